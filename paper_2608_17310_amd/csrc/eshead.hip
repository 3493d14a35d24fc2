// Scoring a member at its head, and a population at its projections
// (include/esopt.h, es_head_*, es_adapt_*).  Host side: checks of arguments, the
// division of a call's workspace and launches; the kernels are in head.hpp,
// adapt.hpp and mm_tile.hpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>

#include "../../include/esopt.h"
#include "es_host.hpp"
#include "adapt.hpp"
#include "head.hpp"

using namespace es_host;
using esmm::kDepth;
using esmm::kSmallTile;
using esmm::kTile;
using esmm::Product;
using esmm::Shape;
using esmm::Side;

namespace {

constexpr uint64_t kMaxStride = uint64_t(1) << 22;
// Results of a product: their tiles' lanes stay below 2^32, a launch's limit.
constexpr uint64_t kMaxResults = uint64_t(1) << 36;
constexpr uint32_t kCus = 256;

// Gradients of logits, and copies of a head's rows, that a call holds at a time:
// what the last cache level keeps between the products that write and read them.
constexpr uint64_t kPieceBytes = uint64_t(256) << 20;

bool odd(const void* p, uintptr_t align) { return reinterpret_cast<uintptr_t>(p) % align != 0; }
uint64_t up(uint64_t x, uint64_t to) { return (x + to - 1) / to * to; }

// `rows` rows of `width` bf16, `stride` elements apart.
uint64_t extent(uint64_t rows, uint64_t width, uint64_t stride) {
    return 2 * ((rows - 1) * stride + width);
}

// A call with strides that mean something: a matrix of one row, or none, takes one of whole words.
uint64_t stride_of(uint64_t rows, uint64_t width, uint64_t stride) { return rows > 1 ? stride : up(width, 8); }

es_head_score_t settled(es_head_score_t x) {
    x.x_stride = stride_of(x.rows, x.hidden, x.x_stride);
    x.w_stride = stride_of(x.vocab, x.hidden, x.w_stride);
    return x;
}
es_head_gradient_t settled(es_head_gradient_t x) {
    x.x_stride = stride_of(x.rows, x.hidden, x.x_stride);
    x.w_stride = stride_of(x.vocab, x.hidden, x.w_stride);
    x.dx_stride = stride_of(x.rows, x.hidden, x.dx_stride);
    x.dw_stride = stride_of(x.vocab, x.hidden, x.dw_stride);
    return x;
}
es_adapt_t settled(es_adapt_t x) {
    x.x_stride = stride_of(x.rows, x.inner, x.x_stride);
    x.w_stride = stride_of(x.outer, x.inner, x.w_stride);
    x.out_stride = stride_of(x.rows, x.outer, x.out_stride);
    return x;
}

// Whether rows of two matrices share memory: rows side by side within a common stride need
// not (with strides that differ, meeting ranges are taken to).
bool meet(const void* a, uint64_t a_rows, uint64_t a_width, uint64_t a_stride, const void* b, uint64_t b_rows,
          uint64_t b_width, uint64_t b_stride) {
    const uint64_t at = reinterpret_cast<uint64_t>(a), bt = reinterpret_cast<uint64_t>(b);
    if (at >= bt + extent(b_rows, b_width, b_stride) || bt >= at + extent(a_rows, a_width, a_stride)) return false;
    if (a_rows < 2 || b_rows < 2 || a_stride != b_stride) return true;
    const uint64_t step = 2 * a_stride, apart = bt >= at ? (bt - at) % step : (step - (at - bt) % step) % step;
    return apart < 2 * a_width || apart + 2 * b_width > step;
}

int launch_error(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ES_OK : hip_fail(e, what);
}

// A workspace handed out in order; without memory, only measured.
struct Room {
    uint8_t* at;
    uint64_t used = 0;
    template <class T>
    T* take(uint64_t n) {
        uint8_t* const p = at == nullptr ? nullptr : at + used;
        used += up(n * sizeof(T), 256);
        return reinterpret_cast<T*>(p);
    }
};

bool word_rows(const void* p, uint64_t stride, uint32_t width) {
    return !odd(p, 16) && stride % 8 == 0 && width % 8 == 0;
}

// How many tiles of `size` an m x n product has.
uint64_t tiles_of(uint64_t m, uint64_t n, uint32_t size) {
    return (m + size - 1) / size * ((n + size - 1) / size);
}

// Tiles of 128 x 128 results where the card holds them at once (two a compute unit), of
// 256 x 256 where there are more.  5120 x 5120: 1000 rows (320 small tiles) 81 and 115 us,
// 2000 (640) 121 and 121; 5120 x 17408: 300 rows (408) 99 and 114; 129 rows against 151936 x
// 2560 (2374) 260 and 211.
uint32_t tile_for(uint64_t m, uint64_t n) {
    return tiles_of(m, n, kSmallTile) <= 2 * kCus ? kSmallTile : kTile;
}

// --------------------------------------------------------------------- head --

int check_head(const char* name, const void* x, const void* weight, uint64_t x_stride,
               uint64_t w_stride, const int64_t* ids, const float* teacher, uint32_t rows,
               uint32_t vocab, uint32_t hidden, uint32_t entries, float scale, uint32_t reserved) {
    if (rows > 65536) return fail_in(ES_ERR_INVALID_ARG, name, "rows above 65536");
    if (vocab == 0 || vocab > (1u << 24))
        return fail_in(ES_ERR_INVALID_ARG, name, "vocab out of range (1 .. 2^24)");
    if (hidden == 0 || hidden > 65536)
        return fail_in(ES_ERR_INVALID_ARG, name, "hidden out of range (1 .. 65536)");
    if (uint64_t(rows) * vocab > kMaxResults)
        return fail_in(ES_ERR_INVALID_ARG, name, "rows times vocab above 2^36");
    if (entries == 0 || entries > eshead::kMaxEntries)
        return fail_in(ES_ERR_INVALID_ARG, name, "entries out of range (1 .. 256)");
    if (!std::isfinite(scale)) return fail_in(ES_ERR_INVALID_ARG, name, "scale is not finite");
    if (reserved != 0) return fail_in(ES_ERR_INVALID_ARG, name, "reserved is not 0");
    if (x_stride > kMaxStride || w_stride > kMaxStride)
        return fail_in(ES_ERR_INVALID_ARG, name, "stride above 2^22");
    if (teacher == nullptr && entries != 1)
        return fail_in(ES_ERR_INVALID_ARG, name, "without a teacher a row has one id");
    if (rows == 0) return ES_OK;
    if (x == nullptr || weight == nullptr || ids == nullptr)
        return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    if (odd(x, 2) || odd(weight, 2) || odd(ids, 8) || odd(teacher, 4))
        return fail_in(ES_ERR_ALIGN, name, "array not aligned to its elements");
    return ES_OK;
}

// The head's rows as the products take them: as they are where each starts at a word
// of 16 bytes, otherwise copied, a piece at a time.
struct HeadRows {
    bool copied;
    uint32_t padded, piece, pieces;        // row width; rows of a piece
    HeadRows(const void* w, uint64_t stride, uint32_t vocab, uint32_t hidden, uint64_t row_bytes) {
        copied = !word_rows(w, stride, hidden);
        padded = static_cast<uint32_t>(up(hidden, kDepth));
        uint64_t each = row_bytes;
        if (copied) each = std::max<uint64_t>(each, 2 * padded);
        const uint64_t whole = up(vocab, kTile);
        const uint64_t most = each == 0 ? whole
                                        : std::max<uint64_t>(kTile, kPieceBytes / each / kTile * kTile);
        pieces = static_cast<uint32_t>((whole + most - 1) / most);
        // pieces of about one size
        piece = static_cast<uint32_t>(up((whole + pieces - 1) / pieces, kTile));
        pieces = static_cast<uint32_t>((whole + piece - 1) / piece);
    }
};

struct Lists {
    uint8_t* flags;
    uint32_t *list, *count;
    uint16_t* x;
    uint32_t rows, padded;                 // of the packed rows
    Lists(Room& room, uint32_t n, uint32_t hidden) {
        rows = static_cast<uint32_t>(up(n, kTile));
        padded = static_cast<uint32_t>(up(hidden, kDepth));
        flags = room.take<uint8_t>(n);
        list = room.take<uint32_t>(n);
        count = room.take<uint32_t>(1);
        x = room.take<uint16_t>(uint64_t(rows) * padded);
    }
    Side deep() const { return Side{x, padded, rows}; }
    Side wide() const { return Side{x, padded, padded}; }
};

// How few rows' products are divided: blocks of 16 rows of the matrix a wave, and
// the waves that share a block's sum.
struct FewPlan {
    uint32_t cols, slices, groups;
    FewPlan(uint32_t rows, uint32_t w_rows, uint32_t width, uint32_t blocks) {
        cols = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
        slices = 1;
        while (slices < esfew::kWaves && width / (2 * slices) >= 128) slices *= 2;
        const uint32_t per = esfew::kWaves / slices * 16 * blocks;
        groups = (w_rows + per - 1) / per;
    }
};

// How a matrix of many rows is divided among a workgroup on each compute unit: an even
// share, in blocks of 16 rows, and as many waves, of `blocks` blocks each, as make equal
// rounds of it (151936 x 1024: three rounds of seven waves where eight left the third
// a third full: 77 rows 63 and 69 us, 1 row 58 and 59; 64 rows of 2560 147 and 145).
struct StreamPlan {
    uint32_t waves, share, groups;
    StreamPlan(uint32_t w_rows, uint32_t blocks) {
        share = 16 * (((w_rows + 15) / 16 + kCus - 1) / kCus);
        const uint32_t each = (share / 16 + blocks - 1) / blocks, rounds = (each + 7) / 8;
        waves = (each + rounds - 1) / rounds;
        groups = (w_rows + share - 1) / share;
    }
};

esstream::StreamArgs stream_args(const void* w, uint64_t w_stride, uint32_t w_rows, const void* x,
                                 uint64_t x_stride, uint32_t rows, uint32_t width, uint32_t share) {
    return esstream::StreamArgs{static_cast<const uint16_t*>(w), static_cast<const uint16_t*>(x), w_stride,
                                x_stride, w_rows, rows, width, share};
}

// Rows of words, few enough that the matrix's bytes are what they cost.  (128 rows of 2560
// against 151936 175 us, 129 in tiles 213.)
bool streams(const es_head_score_t& x) {
    return x.rows <= esstream::kRows && word_rows(x.weight, x.w_stride, x.hidden) &&
           word_rows(x.x, x.x_stride, x.hidden);
}

struct ScorePlan {
    bool few, streamed, ringed;
    uint32_t size;                         // of a tile
    uint32_t share, waves;                 // streamed
    HeadRows head;
    Lists lists;
    FewPlan division;
    uint32_t tiles;
    float* parts;
    uint16_t* w;
    ScorePlan(Room& room, const es_head_score_t& x)
        : few(x.rows <= esfew::kRows || streams(x)),
          head(x.weight, x.w_stride, x.vocab, x.hidden, 0),
          lists(room, few ? 0 : x.rows, x.hidden),
          division(x.rows, x.vocab, x.hidden, 2) {
        if (few) {
            // A small vocabulary leaves the workgroups that stage x too few rows: 3 rows of 5120
            // against 8000 tokens 45 and 21 us (streamed, in rings), 40 of 2560 against 16000
            // 31 and 28, 32 of 1024 against 25000 17 and 26.
            ringed = streams(x) && x.vocab <= 16384;
            streamed = streams(x) && !ringed;
            const StreamPlan stream(x.vocab, 2);
            share = stream.share;
            waves = stream.waves;
            tiles = streamed ? stream.groups : ringed ? (x.vocab + 31) / 32 : division.groups;
            parts = room.take<float>(uint64_t(2) * x.rows * tiles);
            w = nullptr;
            return;
        }
        size = tile_for(head.piece, x.rows);
        tiles = (x.vocab + size - 1) / size;
        parts = room.take<float>(uint64_t(2) * lists.rows * tiles);
        w = head.copied ? room.take<uint16_t>(uint64_t(head.piece) * head.padded) : nullptr;
    }
};

struct GradientPlan {
    Lists lists;
    HeadRows head;
    float *factor, *minus_lse, *parts;
    uint16_t *d, *w;
    uint32_t splits, split_depth, size;    // of the rows' gradient, and its tiles
    GradientPlan(Room& room, const es_head_gradient_t& x)
        : lists(room, x.rows, x.hidden),
          head(x.weight, x.w_stride, x.vocab, x.hidden, 2 * uint64_t(lists.rows)) {
        factor = room.take<float>(lists.rows);
        minus_lse = room.take<float>(lists.rows);
        d = room.take<uint16_t>(uint64_t(lists.rows) * head.piece);
        w = head.copied ? room.take<uint16_t>(uint64_t(head.piece) * head.padded) : nullptr;
        splits = 1;
        split_depth = head.piece;
        parts = nullptr;
        if (x.d_x == nullptr) return;
        // the sum over the vocabulary in as many parts as fill the card
        // (in small tiles where these leave out a quarter of the padded rows: 266 rows against
        // 32003 x 1000 36 and 31 us, and their parts' join 10 and 7.5)
        const bool low = 4 * up(x.rows, kSmallTile) <= 3 * up(x.rows, kTile);
        size = low ? kSmallTile : kTile;
        const uint64_t tiles = tiles_of(x.rows, x.hidden, size);
        const uint32_t most = std::max(1u, head.piece / (low ? 512 : 1024));
        splits = static_cast<uint32_t>(
            std::min<uint64_t>(most, std::max<uint64_t>(1, (low ? 2 * kCus : kCus) / tiles)));
        split_depth = static_cast<uint32_t>(up((head.piece + splits - 1) / splits, kDepth));
        splits = (head.piece + split_depth - 1) / split_depth;
        if (splits > 1 || head.pieces > 1)
            parts = room.take<float>(uint64_t(splits) * lists.rows * lists.padded);
    }
};

Product product(Side a, Side b, uint32_t m, uint32_t n, uint32_t depth, const uint32_t* count,
                uint32_t size) {
    Product p{};
    p.a = a;
    p.b = b;
    p.depth = depth;
    p.m_tiles = (m + size - 1) / size;
    p.n_tiles = (n + size - 1) / size;
    p.splits = 1;
    p.split_depth = depth;
    p.count = count;
    return p;
}

// A kernel over the tiles of a product.
template <int kSize, class Kernel, class Args>
void launch_tiles(Kernel kernel, const Args& a, hipStream_t s) {
    hipLaunchKernelGGL(kernel, dim3(a.p.m_tiles * a.p.n_tiles * a.p.splits), dim3(Shape<kSize>::kThreads),
                       Shape<kSize>::kLds, s, a);
}

// Flags, list and packed rows of a call.
int list_rows(const char* name, const eshead::RowArgs& rows, const Lists& l, const void* x,
              uint64_t x_stride, eshead::PackArgs pack, hipStream_t s) {
    if (rows.entries > 1)
        hipLaunchKernelGGL(eshead::es_head_rows_kernel, dim3((rows.rows + 3) / 4), dim3(256), 0, s, rows);
    // 266 rows against 32003 x 1000: 40.6 and 39.2 us, their gradients 116.7 and 115.1; 1000 rows
    // the same either way
    pack.lists = rows.rows <= 512;
    if (!pack.lists)
        hipLaunchKernelGGL(eshead::es_head_list_kernel, dim3(1), dim3(1024), 0, s,
                           eshead::ListArgs{rows, l.list, l.count});
    pack.out = rows;
    pack.from = static_cast<const uint16_t*>(x);
    pack.to = l.x;
    pack.stride = x_stride;
    pack.list = l.list;
    pack.count = l.count;
    pack.rows = rows.rows;
    pack.width = rows.hidden;
    pack.padded = l.padded;
    hipLaunchKernelGGL(eshead::es_head_pack_kernel, dim3(l.rows / 4), dim3(256), 0, s, pack);
    return launch_error(name);
}

// Rows v0 .. of the head, copied if need be, as a deep side and the stride and start of its rows.
Side head_side(const HeadRows& h, const void* w, uint64_t stride, uint16_t* room, uint32_t v0,
               uint32_t have, uint32_t hidden, hipStream_t s) {
    const uint16_t* const from = static_cast<const uint16_t*>(w) + v0 * stride;
    if (!h.copied) return Side{from, stride, have};
    eshead::PackArgs pack{};
    pack.from = from;
    pack.to = room;
    pack.stride = stride;
    pack.rows = have;
    pack.width = hidden;
    pack.padded = h.padded;
    hipLaunchKernelGGL(eshead::es_head_pack_kernel, dim3(static_cast<uint32_t>(up(have, kTile) / 4)),
                       dim3(256), 0, s, pack);
    return Side{room, h.padded, have};
}

template <int kWaves, int kTokens>
void launch_stream(const eshead::StreamStatsArgs& t, uint32_t groups, hipStream_t s) {
    const auto kernel = eshead::es_head_stream_kernel<kWaves, kTokens>;
    const uint32_t lds = eshead::HeadStream<kWaves, kTokens>::kBytes;
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(64 * kWaves), lds, s, t);
}
template <int kWaves>
void launch_stream(const eshead::StreamStatsArgs& t, uint32_t groups, hipStream_t s) {
    if (t.s.rows <= 32)
        launch_stream<kWaves, 32>(t, groups, s);
    else if (t.s.rows <= 64)
        launch_stream<kWaves, 64>(t, groups, s);
    else if (t.s.rows <= 96)
        launch_stream<kWaves, 96>(t, groups, s);
    else
        launch_stream<kWaves, 128>(t, groups, s);
}

esfew::FewArgs few_args(const void* w, uint64_t w_stride, uint32_t w_rows, const void* x,
                        uint64_t x_stride, uint32_t rows, uint32_t width) {
    esfew::FewArgs f{};
    f.w = static_cast<const uint16_t*>(w);
    f.x = static_cast<const uint16_t*>(x);
    f.w_stride = w_stride;
    f.x_stride = x_stride;
    f.w_rows = w_rows;
    f.rows = rows;
    f.width = width;
    f.slices = 1;
    return f;
}

}  // namespace

extern "C" {

uint64_t es_head_score_bytes(const es_head_score_t* args) {
    if (args == nullptr) return 0;
    const es_head_score_t x = settled(*args);
    if (check_head("es_head_score_bytes", x.x, x.weight, x.x_stride, x.w_stride, x.ids, x.teacher,
                   x.rows, x.vocab, x.hidden, x.entries, x.scale, x.reserved) != ES_OK ||
        x.rows == 0)
        return 0;
    Room room{nullptr};
    const ScorePlan plan(room, x);
    return room.used;
}

int es_head_score(const es_head_score_t* args, es_stream_t stream) try {
    const char* const name = "es_head_score";
    if (args == nullptr) return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    const es_head_score_t x = settled(*args);
    int rc = check_head(name, x.x, x.weight, x.x_stride, x.w_stride, x.ids, x.teacher, x.rows,
                        x.vocab, x.hidden, x.entries, x.scale, x.reserved);
    if (rc != ES_OK) return rc;
    if (x.rows == 0) return ES_OK;
    if (x.logp == nullptr || x.lse == nullptr || (x.loss == nullptr) != (x.teacher == nullptr))
        return fail_in(ES_ERR_INVALID_ARG, name, "logp and lse are needed, and loss with a teacher");
    if (odd(x.logp, 4) || odd(x.lse, 4) || odd(x.loss, 4) || odd(x.status, 4) || odd(x.workspace, 256))
        return fail_in(ES_ERR_ALIGN, name, "array not aligned to its elements");
    int device = -1;
    rc = current_device(&device);
    if (rc != ES_OK) return rc;
    Room room{static_cast<uint8_t*>(x.workspace)};
    const ScorePlan plan(room, x);
    if (x.workspace == nullptr || x.workspace_bytes < room.used)
        return fail_in(ES_ERR_INVALID_ARG, name, "workspace smaller than es_head_score_bytes");
    const uint64_t pairs = uint64_t(x.rows) * x.entries;
    Accesses ok{device, name, {}};
    ok.check(x.x, extent(x.rows, x.hidden, x.x_stride), ": rows");
    ok.check(x.weight, extent(x.vocab, x.hidden, x.w_stride), ": weight");
    ok.check(x.ids, 8 * pairs, ": ids");
    ok.check(x.teacher, x.teacher != nullptr ? 4 * pairs : 0, ": teacher");
    ok.check(x.loss, x.loss != nullptr ? uint64_t(4) * x.rows : 0, ": loss");
    ok.check(x.logp, 4 * pairs, ": logp");
    ok.check(x.lse, uint64_t(4) * x.rows, ": lse");
    ok.check(x.status, x.status != nullptr ? 4 : 0, ": status");
    ok.check(x.workspace, room.used, ": workspace");
    if (ok.rc != ES_OK) return ok.rc;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    eshead::ScoreArgs a{};
    a.parts = plan.parts;
    a.parts_stride = plan.tiles;
    a.n_parts = plan.tiles;
    a.w = static_cast<const uint16_t*>(x.weight);
    a.w_stride = x.w_stride;
    a.ids = x.ids;
    a.teacher = x.teacher;
    a.loss = x.loss;
    a.logp = x.logp;
    a.lse = x.lse;
    a.status = x.status;
    a.hidden = x.hidden;
    a.entries = x.entries;
    a.vocab = x.vocab;
    a.scale = x.scale;
    if (plan.few) {
        a.x = static_cast<const uint16_t*>(x.x);
        a.x_stride = x.x_stride;
    }
    if (plan.few && plan.streamed) {
        eshead::StreamStatsArgs t{};
        t.s = stream_args(x.weight, x.w_stride, x.vocab, x.x, x.x_stride, x.rows, x.hidden, plan.share);
        t.parts = plan.parts;
        t.scale = x.scale;
        switch (plan.waves) {
            case 3: launch_stream<3>(t, plan.tiles, s); break;
            case 4: launch_stream<4>(t, plan.tiles, s); break;
            case 5: launch_stream<5>(t, plan.tiles, s); break;
            case 6: launch_stream<6>(t, plan.tiles, s); break;
            case 7: launch_stream<7>(t, plan.tiles, s); break;
            default: launch_stream<8>(t, plan.tiles, s); break;
        }
        hipLaunchKernelGGL(eshead::es_head_score_kernel, dim3(x.rows), dim3(256), 0, s, a);
        return launch_error("es_head_stream_kernel launch");
    }
    if (plan.few && plan.ringed) {
        eshead::FewStatsArgs f{};
        f.f = few_args(x.weight, x.w_stride, x.vocab, x.x, x.x_stride, x.rows, x.hidden);
        f.parts = plan.parts;
        f.scale = x.scale;
        const auto kernel = x.rows <= 16   ? eshead::es_head_ring_kernel<1, 3>
                            : x.rows <= 32 ? eshead::es_head_ring_kernel<2, 2>
                                           : eshead::es_head_ring_kernel<4, 1>;
        const uint32_t lds = esfew::kWaves * (x.rows <= 16   ? esring::Ring<2, 1, 3>::kBytes
                                              : x.rows <= 32 ? esring::Ring<2, 2, 2>::kBytes
                                                             : esring::Ring<2, 4, 1>::kBytes);
        hipLaunchKernelGGL(kernel, dim3(plan.tiles, (x.rows + 63) / 64), dim3(64 * esfew::kWaves), lds, s, f);
        hipLaunchKernelGGL(eshead::es_head_score_kernel, dim3(x.rows), dim3(256), 0, s, a);
        return launch_error("es_head_ring_kernel launch");
    }
    if (plan.few) {
        eshead::FewStatsArgs f{};
        f.f = few_args(x.weight, x.w_stride, x.vocab, x.x, x.x_stride, x.rows, x.hidden);
        f.f.slices = plan.division.slices;
        f.parts = plan.parts;
        f.scale = x.scale;
        constexpr int b = 2;
        const auto kernel = plan.division.cols == 1   ? eshead::es_head_few_kernel<b, 1>
                            : plan.division.cols == 2 ? eshead::es_head_few_kernel<b, 2>
                                                      : eshead::es_head_few_kernel<b, 4>;
        hipLaunchKernelGGL(kernel, dim3(plan.division.groups), dim3(64 * esfew::kWaves), 0, s, f);
        hipLaunchKernelGGL(eshead::es_head_score_kernel, dim3(x.rows), dim3(256), 0, s, a);
        return launch_error("es_head_few_kernel launch");
    }
    eshead::RowArgs rows{};
    rows.ids = x.ids;
    rows.teacher = x.teacher;
    rows.flags = plan.lists.flags;
    rows.loss = x.loss;
    rows.logp = x.logp;
    rows.lse = x.lse;
    rows.status = x.status;
    rows.rows = x.rows;
    rows.vocab = x.vocab;
    rows.entries = x.entries;
    rows.hidden = x.hidden;
    rc = list_rows(name, rows, plan.lists, x.x, x.x_stride, eshead::PackArgs{}, s);
    if (rc != ES_OK) return rc;
    for (uint32_t v0 = 0; v0 < x.vocab; v0 += plan.head.piece) {
        const uint32_t have = std::min(plan.head.piece, x.vocab - v0);
        const Side w = head_side(plan.head, x.weight, x.w_stride, plan.w, v0, have, x.hidden, s);
        eshead::StatsArgs t{};
        t.p = product(w, plan.lists.deep(), have, x.rows, x.hidden, plan.lists.count, plan.size);
        t.parts = plan.parts;
        t.parts_stride = plan.tiles;
        t.part0 = v0 / plan.size;
        t.scale = x.scale;
        if (plan.size == kTile)
            launch_tiles<kTile>(eshead::es_head_stats_kernel<kTile>, t, s);
        else
            launch_tiles<kSmallTile>(eshead::es_head_stats_kernel<kSmallTile>, t, s);
        rc = launch_error("es_head_stats_kernel launch");
        if (rc != ES_OK) return rc;
    }
    a.list = plan.lists.list;
    a.count = plan.lists.count;
    a.x = plan.lists.x;
    a.x_stride = plan.lists.padded;
    hipLaunchKernelGGL(eshead::es_head_score_kernel, dim3(x.rows), dim3(256), 0, s, a);
    return launch_error("es_head_score_kernel launch");
} catch (const std::bad_alloc&) {
    return fail(ES_ERR_NOMEM, "es_head_score: host allocation failed");
}

uint64_t es_head_gradient_bytes(const es_head_gradient_t* args) {
    if (args == nullptr) return 0;
    const es_head_gradient_t x = settled(*args);
    if (check_head("es_head_gradient_bytes", x.x, x.weight, x.x_stride, x.w_stride, x.ids, x.teacher,
                   x.rows, x.vocab, x.hidden, x.entries, x.scale, x.reserved) != ES_OK ||
        x.rows == 0)
        return 0;
    Room room{nullptr};
    const GradientPlan plan(room, x);
    return room.used;
}

int es_head_gradient(const es_head_gradient_t* args, es_stream_t stream) try {
    const char* const name = "es_head_gradient";
    if (args == nullptr) return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    const es_head_gradient_t x = settled(*args);
    int rc = check_head(name, x.x, x.weight, x.x_stride, x.w_stride, x.ids, x.teacher, x.rows,
                        x.vocab, x.hidden, x.entries, x.scale, x.reserved);
    if (rc != ES_OK) return rc;
    if (x.dx_stride > kMaxStride || x.dw_stride > kMaxStride)
        return fail_in(ES_ERR_INVALID_ARG, name, "stride above 2^22");
    if (x.rows == 0 && x.d_weight != nullptr)
        return fail_in(ES_ERR_INVALID_ARG, name, "no rows: the head's gradient is not written");
    if (x.rows == 0) return ES_OK;
    if (x.logp == nullptr || x.lse == nullptr || x.grad == nullptr)
        return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    if ((x.d_x != nullptr && x.dx_stride < x.hidden) || (x.d_weight != nullptr && x.dw_stride < x.hidden))
        return fail_in(ES_ERR_INVALID_ARG, name, "a gradient's rows overlap");
    if (odd(x.logp, 4) || odd(x.lse, 4) || odd(x.grad, 4) || odd(x.d_x, 2) || odd(x.d_weight, 2) ||
        odd(x.status, 4) || odd(x.workspace, 256))
        return fail_in(ES_ERR_ALIGN, name, "array not aligned to its elements");
    int device = -1;
    rc = current_device(&device);
    if (rc != ES_OK) return rc;
    Room room{static_cast<uint8_t*>(x.workspace)};
    const GradientPlan plan(room, x);
    if (x.workspace == nullptr || x.workspace_bytes < room.used)
        return fail_in(ES_ERR_INVALID_ARG, name, "workspace smaller than es_head_gradient_bytes");
    const uint64_t pairs = uint64_t(x.rows) * x.entries;
    Accesses ok{device, name, {}};
    ok.check(x.x, extent(x.rows, x.hidden, x.x_stride), ": rows");
    ok.check(x.weight, extent(x.vocab, x.hidden, x.w_stride), ": weight");
    ok.check(x.ids, 8 * pairs, ": ids");
    ok.check(x.teacher, x.teacher != nullptr ? 4 * pairs : 0, ": teacher");
    ok.check(x.logp, 4 * pairs, ": logp");
    ok.check(x.lse, uint64_t(4) * x.rows, ": lse");
    ok.check(x.grad, uint64_t(4) * x.rows, ": grad");
    if (x.d_x != nullptr) ok.check(x.d_x, extent(x.rows, x.hidden, x.dx_stride), ": rows' gradient");
    if (x.d_weight != nullptr)
        ok.check(x.d_weight, extent(x.vocab, x.hidden, x.dw_stride), ": weight's gradient");
    ok.check(x.status, x.status != nullptr ? 4 : 0, ": status");
    ok.check(x.workspace, room.used, ": workspace");
    if (ok.rc != ES_OK) return ok.rc;
    if (x.d_x == nullptr && x.d_weight == nullptr) return ES_OK;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Lists& l = plan.lists;
    eshead::RowArgs rows{};
    rows.ids = x.ids;
    rows.teacher = x.teacher;
    rows.flags = l.flags;
    rows.dx = static_cast<uint16_t*>(x.d_x);
    rows.dx_stride = x.dx_stride;
    rows.weighed = x.teacher != nullptr;
    rows.scale = x.scale;
    rows.status = x.status;
    rows.rows = x.rows;
    rows.vocab = x.vocab;
    rows.entries = x.entries;
    rows.hidden = x.hidden;
    const float signed_scale = x.teacher == nullptr ? -x.scale : x.scale;
    eshead::PackArgs pack{};
    pack.grad = x.grad;
    pack.lse = x.lse;
    pack.factor = plan.factor;
    pack.minus_lse = plan.minus_lse;
    pack.scale = signed_scale;
    rc = list_rows(name, rows, l, x.x, x.x_stride, pack, s);
    if (rc != ES_OK) return rc;
    for (uint32_t v0 = 0; v0 < x.vocab; v0 += plan.head.piece) {
        const uint32_t have = std::min(plan.head.piece, x.vocab - v0);
        const Side w = head_side(plan.head, x.weight, x.w_stride, plan.w, v0, have, x.hidden, s);
        eshead::ProbArgs a{};
        const uint32_t size = tile_for(plan.head.piece, x.rows);
        a.p = product(w, l.deep(), have, x.rows, x.hidden, l.count, size);
        a.factor = plan.factor;
        a.minus_lse = plan.minus_lse;
        a.d = plan.d;
        a.d_stride = plan.head.piece;
        a.scale = x.scale;
        if (size == kTile)
            launch_tiles<kTile>(eshead::es_head_prob_kernel<kTile>, a, s);
        else
            launch_tiles<kSmallTile>(eshead::es_head_prob_kernel<kSmallTile>, a, s);
        eshead::EntryArgs e{};
        e.list = l.list;
        e.count = l.count;
        e.ids = x.ids;
        e.teacher = x.teacher;
        e.logp = x.logp;
        e.grad = x.grad;
        e.d = plan.d;
        e.d_stride = plan.head.piece;
        e.entries = x.entries;
        e.v0 = v0;
        e.v_end = v0 + have;
        e.scale = x.scale;
        e.sign_scale = signed_scale;
        hipLaunchKernelGGL(eshead::es_head_entries_kernel, dim3(x.rows), dim3(256), 0, s, e);
        rc = launch_error("es_head_prob_kernel launch");
        if (rc != ES_OK) return rc;
        const Side d_deep{plan.d, plan.head.piece, l.rows};
        if (x.d_x != nullptr) {
            eshead::RowGradArgs g{};
            // along the tile the head's rows are as wide as they are stored
            const uint32_t width = plan.head.copied ? plan.head.padded : x.hidden;
            g.p = product(Side{w.at, w.stride, width}, d_deep, x.hidden, x.rows, have, l.count,
                          plan.size);
            g.p.splits = plan.splits;
            g.p.split_depth = plan.split_depth;
            g.parts = plan.parts;
            g.parts_rows = l.rows;
            g.parts_stride = l.padded;
            g.hidden = x.hidden;
            g.add = v0 != 0;
            if (plan.parts == nullptr) {
                g.out = static_cast<uint16_t*>(x.d_x);
                g.out_stride = x.dx_stride;
                g.list = l.list;
            }
            if (plan.size == kTile)
                launch_tiles<kTile>(eshead::es_head_row_grad_kernel<kTile>, g, s);
            else
                launch_tiles<kSmallTile>(eshead::es_head_row_grad_kernel<kSmallTile>, g, s);
        }
        if (x.d_weight != nullptr) {
            eshead::HeadGradArgs g{};
            const Side d_wide{plan.d, plan.head.piece, plan.head.piece};
            const uint32_t small = tile_for(plan.head.piece, x.hidden);
            g.p = product(l.wide(), d_wide, x.hidden, have, l.rows, l.count, small);
            g.out = static_cast<uint16_t*>(x.d_weight) + v0 * x.dw_stride;
            g.out_stride = x.dw_stride;
            g.n_have = have;
            g.hidden = x.hidden;
            if (small == kTile)
                launch_tiles<kTile>(eshead::es_head_weight_grad_kernel<kTile>, g, s);
            else
                launch_tiles<kSmallTile>(eshead::es_head_weight_grad_kernel<kSmallTile>, g, s);
        }
        rc = launch_error("es_head_gradient kernel launch");
        if (rc != ES_OK) return rc;
    }
    if (x.d_x != nullptr && plan.parts != nullptr) {
        eshead::JoinArgs j{};
        j.parts = plan.parts;
        j.parts_rows = l.rows;
        j.parts_stride = l.padded;
        j.splits = plan.splits;
        j.hidden = x.hidden;
        j.list = l.list;
        j.count = l.count;
        j.out = static_cast<uint16_t*>(x.d_x);
        j.out_stride = x.dx_stride;
        hipLaunchKernelGGL(eshead::es_head_join_kernel, dim3(x.rows, (x.hidden + 1023) / 1024), dim3(256),
                           0, s, j);
    }
    return launch_error("es_head_join_kernel launch");
} catch (const std::bad_alloc&) {
    return fail(ES_ERR_NOMEM, "es_head_gradient: host allocation failed");
}

}  // extern "C"

// ----------------------------------------------------------------- adapters --

namespace {

int check_adapt(const char* name, const es_adapt_t& x) {
    if (x.rows > (1u << 20)) return fail_in(ES_ERR_INVALID_ARG, name, "rows above 2^20");
    if (x.inner == 0 || x.inner % 8 != 0 || x.inner > 65536)
        return fail_in(ES_ERR_INVALID_ARG, name, "inner is not a multiple of 8 up to 65536");
    if (x.outer == 0 || x.outer > (1u << 20))
        return fail_in(ES_ERR_INVALID_ARG, name, "outer out of range (1 .. 2^20)");
    if (uint64_t(x.rows) * x.outer > kMaxResults)
        return fail_in(ES_ERR_INVALID_ARG, name, "rows times outer above 2^36");
    if (x.members == 0 || x.members > 65536)
        return fail_in(ES_ERR_INVALID_ARG, name, "members out of range (1 .. 65536)");
    if (x.rank == 0 || x.rank % 8 != 0 || x.rank > esadapt::kMaxRank)
        return fail_in(ES_ERR_INVALID_ARG, name, "rank is not a multiple of 8 up to 128");
    if (x.reserved != 0) return fail_in(ES_ERR_INVALID_ARG, name, "reserved is not 0");
    if (x.x_stride > kMaxStride || x.w_stride > kMaxStride || x.out_stride > kMaxStride)
        return fail_in(ES_ERR_INVALID_ARG, name, "stride above 2^22");
    if (x.rows == 0) return ES_OK;
    if (x.x == nullptr || x.weight == nullptr || x.out == nullptr || x.a == nullptr ||
        x.b == nullptr || x.index == nullptr)
        return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    if (x.out == x.x) return fail_in(ES_ERR_INVALID_ARG, name, "out is x");
    if (x.out_stride < x.outer)
        return fail_in(ES_ERR_INVALID_ARG, name, "the output's rows overlap");
    const auto meets_out = [&](const void* p, uint64_t rows, uint64_t width, uint64_t stride) {
        return meet(x.out, x.rows, x.outer, x.out_stride, p, rows, width, stride);
    };
    if (meets_out(x.x, x.rows, x.inner, x.x_stride) || meets_out(x.weight, x.outer, x.inner, x.w_stride) ||
        meets_out(x.a, 1, uint64_t(x.members) * x.rank * x.inner, 0) ||
        meets_out(x.b, 1, uint64_t(x.members) * x.rank * x.outer, 0))
        return fail_in(ES_ERR_INVALID_ARG, name, "out shares memory with an input");
    if (odd(x.x, 2) || odd(x.out, 2) || odd(x.scales, 4) || odd(x.index, 4) || odd(x.status, 4))
        return fail_in(ES_ERR_ALIGN, name, "array not aligned to its elements");
    if (odd(x.weight, 16) || x.w_stride % 8 != 0 || odd(x.a, 16) || odd(x.b, 16))
        return fail_in(ES_ERR_ALIGN, name, "weight's rows or adapters not 16-byte aligned");
    return ES_OK;
}

struct AdaptPlan {
    float* u;
    uint16_t* x;
    uint32_t padded, packed_rows;
    AdaptPlan(Room& room, const es_adapt_t& a) {
        u = room.take<float>(uint64_t(a.rows) * a.rank);
        padded = static_cast<uint32_t>(up(a.inner, kDepth));
        packed_rows = static_cast<uint32_t>(up(a.rows, kTile));
        // the products take rows that start at a word of 16 bytes and end in whole stages
        few = a.rows <= esfew::kRows;
        const bool copied = (!few && padded != a.inner) || !word_rows(a.x, a.x_stride, a.inner);
        x = nullptr;
        if (copied) x = room.take<uint16_t>(uint64_t(packed_rows) * padded);
        is_copied = copied;
        const uint64_t tiles = tiles_of(a.outer, a.rows, kSmallTile);
        low = !few && tile_for(a.outer, a.rows) == kSmallTile;
        splits = 1;
        split_depth = static_cast<uint32_t>(up(a.inner, kDepth));
        parts = nullptr;
        parts_stride = up(a.outer, 4);
        // Few tiles' sums are divided, if a part is worth the join: a stage of 64 takes 0.6 us,
        // the join's launch and its bytes the rest.  5120 x 5120, 100 rows (40 tiles) 48 us
        // whole and 25 divided, 300 (120) 48 and 47, 700 (240) 57 and 78.
        uint64_t most = 1;
        const double whole = 0.6 * a.inner / kDepth, join = 8e-6 * a.rows * a.outer / 2.5;
        double best = whole;
        for (uint64_t n = 2; low && n <= 2 * kCus / tiles && n <= a.inner / 1024; ++n)
            if (whole / n + 10 + join * n < best) {
                best = whole / n + 10 + join * n;
                most = n;
            }
        if (most < 2) return;
        split_depth = static_cast<uint32_t>(up((a.inner + most - 1) / most, kDepth));
        splits = (a.inner + split_depth - 1) / split_depth;
        if (splits > 1) parts = room.take<float>(uint64_t(splits) * a.rows * parts_stride);
    }
    bool is_copied, few, low;
    uint32_t splits, split_depth;
    float* parts;
    uint64_t parts_stride;
};

template <int kWaves, int kTokens>
void launch_stream(const esadapt::StreamArgs& t, uint32_t groups, hipStream_t s) {
    const auto kernel = esadapt::es_adapt_stream_kernel<kWaves, kTokens>;
    const uint32_t lds = esadapt::AdaptStream<kWaves, kTokens>::kBytes;
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(64 * kWaves), lds, s, t);
}
template <int kWaves>
void launch_stream(const esadapt::StreamArgs& t, uint32_t groups, hipStream_t s) {
    if (t.s.rows <= 16)
        launch_stream<kWaves, 16>(t, groups, s);
    else if (t.s.rows <= 32)
        launch_stream<kWaves, 32>(t, groups, s);
    else
        launch_stream<kWaves, 64>(t, groups, s);
}

}  // namespace

extern "C" {

uint64_t es_adapt_bytes(const es_adapt_t* args) {
    if (args == nullptr) return 0;
    const es_adapt_t x = settled(*args);
    if (check_adapt("es_adapt_bytes", x) != ES_OK || x.rows == 0) return 0;
    Room room{nullptr};
    const AdaptPlan plan(room, x);
    return room.used;
}

int es_adapt_project(const es_adapt_t* args, es_stream_t stream) try {
    const char* const name = "es_adapt_project";
    if (args == nullptr) return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    const es_adapt_t x = settled(*args);
    int rc = check_adapt(name, x);
    if (rc != ES_OK) return rc;
    if (x.rows == 0) return ES_OK;
    if (odd(x.workspace, 256)) return fail_in(ES_ERR_ALIGN, name, "workspace not 256-byte aligned");
    int device = -1;
    rc = current_device(&device);
    if (rc != ES_OK) return rc;
    Room room{static_cast<uint8_t*>(x.workspace)};
    const AdaptPlan plan(room, x);
    if (x.workspace == nullptr || x.workspace_bytes < room.used)
        return fail_in(ES_ERR_INVALID_ARG, name, "workspace smaller than es_adapt_bytes");
    Accesses ok{device, name, {}};
    ok.check(x.x, extent(x.rows, x.inner, x.x_stride), ": rows");
    ok.check(x.weight, extent(x.outer, x.inner, x.w_stride), ": weight");
    ok.check(x.out, extent(x.rows, x.outer, x.out_stride), ": output");
    ok.check(x.a, 2 * uint64_t(x.members) * x.rank * x.inner, ": a");
    ok.check(x.b, 2 * uint64_t(x.members) * x.rank * x.outer, ": b");
    ok.check(x.scales, x.scales != nullptr ? uint64_t(4) * x.members : 0, ": scales");
    ok.check(x.index, uint64_t(4) * x.rows, ": index");
    ok.check(x.status, x.status != nullptr ? 4 : 0, ": status");
    ok.check(x.workspace, room.used, ": workspace");
    if (ok.rc != ES_OK) return ok.rc;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    Side rows{static_cast<const uint16_t*>(x.x), x.x_stride, x.rows};
    if (plan.is_copied) {
        eshead::PackArgs pack{};
        pack.from = static_cast<const uint16_t*>(x.x);
        pack.to = plan.x;
        pack.stride = x.x_stride;
        pack.rows = x.rows;
        pack.width = x.inner;
        pack.padded = plan.padded;
        hipLaunchKernelGGL(eshead::es_head_pack_kernel, dim3(plan.packed_rows / 4), dim3(256), 0, s, pack);
        rows = Side{plan.x, plan.padded, plan.packed_rows};
    }
    esadapt::SmallArgs small{};
    small.x = rows.at;
    small.x_stride = rows.stride;
    small.a = static_cast<const uint16_t*>(x.a);
    small.scales = x.scales;
    small.index = x.index;
    small.u = plan.u;
    small.status = x.status;
    small.rows = x.rows;
    small.inner = x.inner;
    small.members = x.members;
    small.rank = x.rank;
    small.split = !plan.few && plan.splits == 1;
    const esadapt::AddArgs add{x.index, plan.u, static_cast<const uint16_t*>(x.b), x.rows, x.outer,
                               x.members, x.rank};
    // u: a wave for each of its elements reads two rows of `inner`, which the second cache
    // serves at about 8 TB/s; a workgroup of 32 rows reads them and A once for each member among
    // them, in some 7 us each at 5120.  Rank 16, of 5120: 70 rows of 8 members 4 and 21 us, 300 of
    // 8 12 and 14, 300 of 300 12 and 310, 8403 of 16 (2560, rank 32) about 330 and 25.
    const double one_by_one = 5e-7 * x.rows * x.rank * x.inner;
    const double by_member = (1 + 32.0 * std::min(x.members, x.rows) / x.rows) * (1 + x.inner / 850.0);
    if (plan.few || one_by_one < by_member) {
        hipLaunchKernelGGL(esadapt::es_adapt_few_small_kernel, dim3(x.rows, (x.rank + 3) / 4), dim3(256), 0,
                           s, small);
    } else {
        const auto kernel = x.rank <= 16   ? esadapt::es_adapt_small_kernel<1, 3>
                            : x.rank <= 32 ? esadapt::es_adapt_small_kernel<2, 2>
                                           : esadapt::es_adapt_small_kernel<4, 1>;
        const uint32_t lds = esfew::kWaves * (x.rank <= 16   ? esring::Ring<1, 2, 3>::kBytes
                                              : x.rank <= 32 ? esring::Ring<2, 2, 2>::kBytes
                                                             : esring::Ring<4, 2, 1>::kBytes);
        hipLaunchKernelGGL(kernel, dim3((x.rows + esadapt::kSmallRows - 1) / esadapt::kSmallRows),
                           dim3(64 * esfew::kWaves), lds, s, small);
    }
    if (plan.few) {
        // A matrix of many rows passes through a workgroup on each compute unit, with as many
        // waves as the unit has blocks of 16 rows of it (or half as many and two rounds, and so
        // on); one of few rows among those whose waves share a sum.  5120 x 5120: 1 row 17 and 14
        // us (streamed, in rings), 32 rows 22 and 18; 5120 x 8192: 32 rows 27 and 26; 5120 x
        // 17408: 1 row 38 and 38, 16 rows 39 and 46.
        if (x.outer > 8192) {
            const StreamPlan plan(x.outer, 1);
            esadapt::StreamArgs t{};
            t.s = stream_args(x.weight, x.w_stride, x.outer, rows.at, rows.stride, x.rows, x.inner, plan.share);
            t.add = add;
            t.out = static_cast<uint16_t*>(x.out);
            t.out_stride = x.out_stride;
            switch (plan.waves) {
                case 3: launch_stream<3>(t, plan.groups, s); break;
                case 4: launch_stream<4>(t, plan.groups, s); break;
                case 5: launch_stream<5>(t, plan.groups, s); break;
                case 6: launch_stream<6>(t, plan.groups, s); break;
                case 7: launch_stream<7>(t, plan.groups, s); break;
                default: launch_stream<8>(t, plan.groups, s); break;
            }
            return launch_error("es_adapt_stream_kernel launch");
        }
        esadapt::FewArgs f{};
        f.f = few_args(x.weight, x.w_stride, x.outer, rows.at, rows.stride, x.rows, x.inner);
        f.add = add;
        f.out = static_cast<uint16_t*>(x.out);
        f.out_stride = x.out_stride;
        const auto launch = [&](auto kernel, uint32_t bytes) {
            hipLaunchKernelGGL(kernel, dim3((x.outer + 31) / 32), dim3(64 * esfew::kWaves),
                               esfew::kWaves * bytes, s, f);
        };
        if (x.rows <= 16)
            launch(esadapt::es_adapt_few_kernel<2, 1, 3>, esring::Ring<2, 1, 3>::kBytes);
        else if (x.rows <= 32)
            launch(esadapt::es_adapt_few_kernel<2, 2, 2>, esring::Ring<2, 2, 2>::kBytes);
        else
            launch(esadapt::es_adapt_few_kernel<2, 4, 1>, esring::Ring<2, 4, 1>::kBytes);
        return launch_error("es_adapt_few_kernel launch");
    }
    esadapt::TileArgs a{};
    const Side weight{static_cast<const uint16_t*>(x.weight), x.w_stride, x.outer};
    if (plan.splits > 1) {
        esadapt::PartArgs q{};
        q.p = product(weight, rows, x.outer, x.rows, x.inner, nullptr, kSmallTile);
        q.p.splits = plan.splits;
        q.p.split_depth = plan.split_depth;
        q.parts = plan.parts;
        q.stride = plan.parts_stride;
        q.rows = x.rows;
        q.outer = x.outer;
        launch_tiles<kSmallTile>(esadapt::es_adapt_part_kernel<kSmallTile>, q, s);
        esadapt::JoinArgs j{};
        j.parts = plan.parts;
        j.stride = plan.parts_stride;
        j.splits = plan.splits;
        j.add = add;
        j.out = static_cast<uint16_t*>(x.out);
        j.out_stride = x.out_stride;
        hipLaunchKernelGGL(esadapt::es_adapt_join_kernel, dim3((x.outer + 1023) / 1024, x.rows), dim3(256), 0,
                           s, j);
        return launch_error("es_adapt_join_kernel launch");
    }
    a.p = product(weight, rows, x.outer, x.rows, x.inner, nullptr, plan.low ? kSmallTile : kTile);
    a.add = add;
    a.out = static_cast<uint16_t*>(x.out);
    a.out_stride = x.out_stride;
    if (plan.low && x.rank <= 16)
        launch_tiles<kSmallTile>(esadapt::es_adapt_tile_kernel<kSmallTile, 1>, a, s);
    else if (plan.low)
        launch_tiles<kSmallTile>(esadapt::es_adapt_tile_kernel<kSmallTile, 2>, a, s);
    else if (x.rank <= 16)
        launch_tiles<kTile>(esadapt::es_adapt_tile_kernel<kTile, 1>, a, s);
    else
        launch_tiles<kTile>(esadapt::es_adapt_tile_kernel<kTile, 2>, a, s);
    return launch_error("es_adapt_project kernel launch");
} catch (const std::bad_alloc&) {
    return fail(ES_ERR_NOMEM, "es_adapt_project: host allocation failed");
}

}  // extern "C"
