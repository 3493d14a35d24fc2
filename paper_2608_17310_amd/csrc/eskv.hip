// Scoring a member: the paged cache of keys and values and the attention over
// it (include/esopt.h, es_kv_*).  Host side: checks of arguments, the choice of
// kernels and launches; the kernels are in kv_place.hpp and kv_attend.hpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>

#include "../../include/esopt.h"
#include "es_host.hpp"
#include "kv_attend.hpp"
#include "kv_place.hpp"

using namespace es_host;
using namespace eskv;

// Parts that a launch cuts its histories into at most: they bound the scratch.
static constexpr uint32_t kMaxParts = 512;
static constexpr uint32_t kMinBlocks = 4;          // blocks of a part at least: one a wave
static constexpr uint32_t kTileMinBlocks = 4;      //   and of a part of a tile of many rows
static constexpr uint32_t kPairLength = 1280;      // tokens of a history worth two columns of rows
static constexpr uint32_t kCutBlocks = 16;         // blocks of a history worth cutting for such tiles

struct es_kv {
    int device = -1;
    es_kv_desc_t d{};
    Cache c{};
    float* scratch = nullptr;                      // partial results of es_kv_attend
    uint64_t scratch_bytes = 0;
    float* part_ml = nullptr;                      // behind them, maxima and sums
};

namespace {

int check_kv_device(const es_kv_t* kv, const char* name) {
    int dev = -1;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    if (dev != kv->device)
        return fail_in(ES_ERR_DEVICE, name, "current device differs from the cache's");
    return ES_OK;
}

bool odd(const void* p, uintptr_t align) { return reinterpret_cast<uintptr_t>(p) % align != 0; }

// Elements from row to row at most: 2^24 rows of them are 2^63 bytes, so that the
// extent of an array fits 64 bits.
constexpr uint64_t kMaxStride = uint64_t(1) << 38;

bool too_wide(uint64_t rows, uint64_t stride) { return rows > 1 && stride > kMaxStride; }

// `rows` rows of `width` bf16, `stride` elements apart (at most kMaxStride).
void check_rows(Accesses& x, const void* p, uint64_t rows, uint64_t width, uint64_t stride,
                const char* part) {
    x.check(p, 2 * ((rows - 1) * stride + width), part);
}

int launch_error(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ES_OK : hip_fail(e, what);
}

// Blocks of `per` tokens, a multiple of 8 where there are as many (block_part).
uint32_t token_blocks(uint32_t tokens, uint32_t per) {
    const uint32_t n = (tokens + per - 1) / per;
    return n >= 8 ? (n + 7) / 8 * 8 : n;
}

using AppendKernel = void (*)(AppendArgs);
using ReadKernel = void (*)(ReadArgs);
using AttendKernel = void (*)(AttendArgs);
using JoinKernel = void (*)(AttendArgs, int, int);

template <class K, template <int, int> class Make>
K by_dim_format(uint32_t dim, uint32_t format) {
    switch (dim) {
        case 64: return format == kInt8   ? Make<64, kInt8>::get()
                        : format == kE4M3 ? Make<64, kE4M3>::get()
                                          : Make<64, kBf16>::get();
        case 128: return format == kInt8   ? Make<128, kInt8>::get()
                         : format == kE4M3 ? Make<128, kE4M3>::get()
                                           : Make<128, kBf16>::get();
        default: return format == kInt8   ? Make<256, kInt8>::get()
                        : format == kE4M3 ? Make<256, kE4M3>::get()
                                          : Make<256, kBf16>::get();
    }
}
template <bool kWhole>
struct MakeAppend {
    template <int D, int F>
    struct Of {
        static AppendKernel get() { return es_kv_append_kernel<D, F, kWhole>; }
    };
};
template <int D, int F>
struct MakeRead {
    static ReadKernel get() { return es_kv_read_kernel<D, F>; }
};
template <int kMode, int kCols>
struct MakeSplit {
    template <int D, int F>
    struct Of {
        static AttendKernel get() {
            return es_kv_split_kernel<D, F, kMode, D == 256 || F == kBf16 ? 1 : kCols>;
        }
    };
};
template <int kMode>
struct MakeTile {
    template <int D, int F>
    struct Of {
        static AttendKernel get() { return es_kv_tile_kernel<D, F, kMode>; }
    };
};

struct TileLaunch {
    uint32_t rows, threads, resident;              // of a workgroup; workgroups of the card
    size_t lds;
    uint64_t slots() const { return uint64_t(rows) * resident; }
};
template <int D>
TileLaunch tile_launch() {
    using S = TileShape<D>;
    return TileLaunch{S::kRows, S::kThreads, 256u * S::kPerSimd, S::kLds};
}

constexpr uint64_t kMaxGroups = uint64_t(1) << 24; // workgroups of a launch: below 2^32 lanes

// A kernel that cuts histories into a.target parts, and the join of the parts.
int launch_parts(AttendKernel kernel, AttendArgs a, uint32_t tile_rows, uint32_t threads, size_t lds,
                 uint64_t seq_rows, uint32_t max_length, uint32_t dim, hipStream_t s) {
    const uint32_t heads = a.c.heads;
    // tiles of all sequences, at most and as expected; a history as long as expected
    // leaves no more parts than these
    const uint64_t n_tiles = uint64_t(a.rows) * a.group / tile_rows + a.n_seqs;
    const uint64_t expected =
        std::min<uint64_t>(n_tiles, (seq_rows + tile_rows - 1) / tile_rows * a.n_seqs);
    const uint64_t part = uint64_t(a.min_blocks) * kBlock;
    const uint64_t parts = std::max<uint64_t>(1, (max_length + part - 1) / part);
    a.target = static_cast<uint32_t>(std::min<uint64_t>(a.target, expected * heads * parts));
    // histories expected to be a part each are not cut, however long they turn out
    if (parts == 1) a.min_blocks = 1u << 25;
    // parts: a tile's last may be short, so one more for each
    const uint64_t n_parts = a.target / heads + 1 + n_tiles;
    if (n_parts * heads >= kMaxGroups)
        return fail(ES_ERR_INVALID_ARG, "es_kv_attend: too many rows for one call");
    hipLaunchKernelGGL(kernel, dim3(n_parts * heads), dim3(threads), lds, s, a);
    const int rc = launch_error("es_kv_attend kernel launch");
    if (rc != ES_OK || parts == 1) return rc;
    const JoinKernel join = dim == 64    ? es_kv_join_kernel<64>
                            : dim == 128 ? es_kv_join_kernel<128>
                                         : es_kv_join_kernel<256>;
    // a row in many parts takes a workgroup, rows in few share one
    const uint64_t rows = std::min<uint64_t>(tile_rows, seq_rows);
    const bool spread = rows <= 16 || a.target > 8 * expected * heads;
    const uint64_t together = 4 * kSplitThreads / dim;         // rows of a workgroup's groups
    const uint64_t y = spread ? rows : (rows + together - 1) / together;
    hipLaunchKernelGGL(join, dim3(n_tiles * heads, y), dim3(kSplitThreads), 0, s, a,
                       static_cast<int>(tile_rows), spread ? 1 : 0);
    return launch_error("es_kv_join_kernel launch");
}

}  // namespace

extern "C" {

int es_kv_create(const es_kv_desc_t* desc, es_kv_t** out) try {
    const char* const name = "es_kv_create";
    if (desc == nullptr || out == nullptr) return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    *out = nullptr;
    const es_kv_desc_t& d = *desc;
    if (d.format != ES_KV_BF16 && d.format != ES_KV_INT8 && d.format != ES_KV_E4M3)
        return fail_in(ES_ERR_INVALID_ARG, name, "unknown format");
    if (d.reserved != 0) return fail_in(ES_ERR_INVALID_ARG, name, "reserved is not 0");
    if (d.page < 64 || d.page > 1024 || (d.page & (d.page - 1)) != 0)
        return fail_in(ES_ERR_INVALID_ARG, name, "page is not 64, 128, 256, 512 or 1024");
    if (d.n_pages == 0 || uint64_t(d.n_pages) * d.page > (uint64_t(1) << 31))
        return fail_in(ES_ERR_INVALID_ARG, name, "n_pages out of range (1 .. 2^31 / page)");
    if (d.kv_heads == 0 || d.kv_heads > 1024)
        return fail_in(ES_ERR_INVALID_ARG, name, "kv_heads out of range (1 .. 1024)");
    if (d.head_dim != 64 && d.head_dim != 128 && d.head_dim != 256)
        return fail_in(ES_ERR_INVALID_ARG, name, "head_dim is not 64, 128 or 256");
    const bool scaled = d.format != ES_KV_BF16;
    if (d.k_pages == nullptr || d.v_pages == nullptr ||
        (scaled && (d.k_scales == nullptr || d.v_scales == nullptr)))
        return fail_in(ES_ERR_INVALID_ARG, name, "null pages or scales");
    if (!scaled && (d.k_scales != nullptr || d.v_scales != nullptr))
        return fail_in(ES_ERR_INVALID_ARG, name, "bf16 pages have no scales");
    if (odd(d.k_pages, 16) || odd(d.v_pages, 16) || odd(d.k_scales, 16) || odd(d.v_scales, 16))
        return fail_in(ES_ERR_ALIGN, name, "pages or scales not 16-byte aligned");
    int device = -1;
    int rc = current_device(&device);
    if (rc != ES_OK) return rc;
    const uint64_t rows = uint64_t(d.n_pages) * d.page * d.kv_heads;
    const uint64_t bytes = rows * d.head_dim * (scaled ? 1 : 2);
    const struct { const void* p; uint64_t bytes; const char* what; } parts[] = {
        {d.k_pages, bytes, ": keys"}, {d.v_pages, bytes, ": values"},
        {d.k_scales, scaled ? 4 * rows : 0, ": key scales"},
        {d.v_scales, scaled ? 4 * rows : 0, ": value scales"}};
    for (const auto& p : parts) {
        rc = check_access(p.p, p.bytes, device, name, p.what);
        if (rc != ES_OK) return rc;
    }
    for (const auto& p : parts)
        for (const auto& q : parts) {
            const uintptr_t x = reinterpret_cast<uintptr_t>(p.p), y = reinterpret_cast<uintptr_t>(q.p);
            if (&p != &q && p.bytes != 0 && q.bytes != 0 && x < y + q.bytes && y < x + p.bytes)
                return fail_in(ES_ERR_INVALID_ARG, name, "pages and scales overlap");
        }
    es_kv* kv = new es_kv;
    kv->device = device;
    kv->d = d;
    kv->c = Cache{static_cast<uint8_t*>(d.k_pages), static_cast<uint8_t*>(d.v_pages), d.k_scales,
                  d.v_scales, d.n_pages, d.kv_heads, d.page,
                  static_cast<uint32_t>(__builtin_ctz(d.page))};
    // at most two slots for each part aimed at (a sequence cut into c > 1 parts
    // has more than c - 1 parts' blocks)
    const uint64_t slot_rows = std::max(
        uint64_t(2) * kMaxParts * 2 * kSplitRows,
        uint64_t(2) * (d.head_dim == 64    ? tile_launch<64>().slots()
                       : d.head_dim == 128 ? tile_launch<128>().slots()
                                           : tile_launch<256>().slots()));
    kv->scratch_bytes = slot_rows * (d.head_dim + 2) * 4;
    const hipError_t e = hipMalloc(reinterpret_cast<void**>(&kv->scratch), kv->scratch_bytes);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        delete kv;
        return fail_in(ES_ERR_NOMEM, name, "device allocation of the scratch failed");
    }
    kv->part_ml = kv->scratch + slot_rows * d.head_dim;
    *out = kv;
    return ES_OK;
} catch (const std::bad_alloc&) {
    return fail(ES_ERR_NOMEM, "es_kv_create: host allocation failed");
}

int es_kv_destroy(es_kv_t* kv) {
    if (kv == nullptr) return ES_OK;
    const int rc = release_device_memory(kv->device, kv->scratch, nullptr, "es_kv_destroy");
    delete kv;
    return rc;
}

uint64_t es_kv_device_bytes(const es_kv_t* kv) { return kv == nullptr ? 0 : kv->scratch_bytes; }

int es_kv_append(es_kv_t* kv, const es_kv_append_t* args, es_stream_t stream) try {
    const char* const name = "es_kv_append";
    if (kv == nullptr || args == nullptr) return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    const es_kv_append_t& x = *args;
    const uint32_t dim = kv->d.head_dim;
    if (x.tokens > (1u << 24)) return fail_in(ES_ERR_INVALID_ARG, name, "tokens above 2^24");
    if (x.q_heads > 1024) return fail_in(ES_ERR_INVALID_ARG, name, "q_heads above 1024");
    if ((x.flags & ~ES_KV_ADJACENT) != 0) return fail_in(ES_ERR_INVALID_ARG, name, "unknown flags");
    if (x.rot % 16 != 0 || x.rot > dim)
        return fail_in(ES_ERR_INVALID_ARG, name, "rot not a multiple of 16 up to head_dim");
    if ((x.q_gain != nullptr || x.k_gain != nullptr) && !(x.eps > 0.0f && std::isfinite(x.eps)))
        return fail_in(ES_ERR_INVALID_ARG, name, "eps not positive and finite");
    if (x.rot != 0 && (x.rope == nullptr || x.positions == nullptr || x.rope_rows == 0))
        return fail_in(ES_ERR_INVALID_ARG, name, "rotation without table or positions");
    if (x.tokens == 0) return ES_OK;
    if (x.k == nullptr || x.v == nullptr || x.slots == nullptr ||
        (x.q_heads != 0 && (x.q == nullptr || x.q_out == nullptr)))
        return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    if (x.q_heads != 0 && x.tokens > 1 && x.q_out_stride < uint64_t(x.q_heads) * dim)
        return fail_in(ES_ERR_INVALID_ARG, name, "q_out's rows overlap");
    if (too_wide(x.tokens, x.k_stride) || too_wide(x.tokens, x.v_stride) ||
        (x.q_heads != 0 && (too_wide(x.tokens, x.q_stride) || too_wide(x.tokens, x.q_out_stride))))
        return fail_in(ES_ERR_INVALID_ARG, name, "stride above 2^38");
    if (odd(x.q, 2) || odd(x.k, 2) || odd(x.v, 2) || odd(x.q_out, 2) || odd(x.q_gain, 2) ||
        odd(x.k_gain, 2) || odd(x.rope, 4) || odd(x.positions, 4) || odd(x.slots, 8) ||
        odd(x.status, 4))
        return fail_in(ES_ERR_ALIGN, name, "array not aligned to its elements");
    const uint32_t q_parts = (x.q_heads + kPlaceHeads - 1) / kPlaceHeads;
    const uint32_t q_blocks =
        x.q_heads == 0 ? 0 : token_blocks(x.tokens, kPlaceThreads * 8 / dim);
    const uint32_t kv_blocks = token_blocks(x.tokens, kPlaceTokens);
    const uint64_t groups = uint64_t(kv_blocks) * kv->d.kv_heads + uint64_t(q_blocks) * q_parts;
    if (groups >= kMaxGroups)
        return fail_in(ES_ERR_INVALID_ARG, name, "too many tokens for one call");
    const int rc = check_kv_device(kv, name);
    if (rc != ES_OK) return rc;
    const uint64_t kw = uint64_t(kv->d.kv_heads) * dim, qw = uint64_t(x.q_heads) * dim;
    Accesses ok{kv->device, name, {}};
    check_rows(ok, x.k, x.tokens, kw, x.k_stride, ": keys");
    check_rows(ok, x.v, x.tokens, kw, x.v_stride, ": values");
    if (qw != 0) {
        check_rows(ok, x.q, x.tokens, qw, x.q_stride, ": queries");
        check_rows(ok, x.q_out, x.tokens, qw, x.q_out_stride, ": query output");
    }
    ok.check(x.q_gain, x.q_gain != nullptr ? 2 * dim : 0, ": query gain");
    ok.check(x.k_gain, x.k_gain != nullptr ? 2 * dim : 0, ": key gain");
    ok.check(x.rope, uint64_t(4) * x.rot * x.rope_rows, ": rotation table");
    ok.check(x.positions, x.rot != 0 ? uint64_t(4) * x.tokens : 0, ": positions");
    ok.check(x.slots, uint64_t(8) * x.tokens, ": slots");
    ok.check(x.status, x.status != nullptr ? 4 : 0, ": status");
    if (ok.rc != ES_OK) return ok.rc;
    AppendArgs a{};
    a.q = static_cast<const uint16_t*>(x.q);
    a.k = static_cast<const uint16_t*>(x.k);
    a.v = static_cast<const uint16_t*>(x.v);
    a.q_out = static_cast<uint16_t*>(x.q_out);
    a.q_stride = x.q_stride;
    a.k_stride = x.k_stride;
    a.v_stride = x.v_stride;
    a.q_out_stride = x.q_out_stride;
    a.q_gain = static_cast<const uint16_t*>(x.q_gain);
    a.k_gain = static_cast<const uint16_t*>(x.k_gain);
    a.rope = x.rope;
    a.positions = x.positions;
    a.slots = x.slots;
    a.status = x.status;
    a.tokens = x.tokens;
    a.q_heads = x.q_heads;
    a.rot = x.rot;
    a.rope_rows = x.rope_rows;
    a.eps = x.eps;
    a.adjacent = (x.flags & ES_KV_ADJACENT) != 0;
    a.c = kv->c;
    const AppendKernel kernel =
        x.rot == dim && (x.flags & ES_KV_ADJACENT) == 0
            ? by_dim_format<AppendKernel, MakeAppend<true>::Of>(dim, kv->d.format)
            : by_dim_format<AppendKernel, MakeAppend<false>::Of>(dim, kv->d.format);
    a.q_parts = q_parts;
    a.q_blocks = q_blocks;
    a.kv_blocks = kv_blocks;
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(kPlaceThreads), 0, static_cast<hipStream_t>(stream), a);
    return launch_error("es_kv_append_kernel launch");
} catch (const std::bad_alloc&) {
    return fail(ES_ERR_NOMEM, "es_kv_append: host allocation failed");
}

int es_kv_read(es_kv_t* kv, const int64_t* slots, uint32_t tokens, void* k_out, uint64_t k_stride,
               void* v_out, uint64_t v_stride, uint32_t* status, es_stream_t stream) try {
    const char* const name = "es_kv_read";
    if (kv == nullptr) return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    if (tokens > (1u << 24)) return fail_in(ES_ERR_INVALID_ARG, name, "tokens above 2^24");
    if (tokens == 0) return ES_OK;
    if (slots == nullptr || k_out == nullptr || v_out == nullptr)
        return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    const uint64_t width = uint64_t(kv->d.kv_heads) * kv->d.head_dim;
    if (tokens > 1 && (k_stride < width || v_stride < width))
        return fail_in(ES_ERR_INVALID_ARG, name, "the output's rows overlap");
    if (too_wide(tokens, k_stride) || too_wide(tokens, v_stride))
        return fail_in(ES_ERR_INVALID_ARG, name, "stride above 2^38");
    if (odd(slots, 8) || odd(k_out, 2) || odd(v_out, 2) || odd(status, 4))
        return fail_in(ES_ERR_ALIGN, name, "array not aligned to its elements");
    const uint32_t blocks = token_blocks(tokens, kPlaceTokens);
    if (uint64_t(blocks) * kv->d.kv_heads >= kMaxGroups)
        return fail_in(ES_ERR_INVALID_ARG, name, "too many tokens for one call");
    const int rc = check_kv_device(kv, name);
    if (rc != ES_OK) return rc;
    Accesses ok{kv->device, name, {}};
    ok.check(slots, uint64_t(8) * tokens, ": slots");
    check_rows(ok, k_out, tokens, width, k_stride, ": key output");
    check_rows(ok, v_out, tokens, width, v_stride, ": value output");
    ok.check(status, status != nullptr ? 4 : 0, ": status");
    if (ok.rc != ES_OK) return ok.rc;
    ReadArgs a{};
    a.slots = slots;
    a.k_out = static_cast<uint16_t*>(k_out);
    a.v_out = static_cast<uint16_t*>(v_out);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.status = status;
    a.tokens = tokens;
    a.c = kv->c;
    const ReadKernel kernel = by_dim_format<ReadKernel, MakeRead>(kv->d.head_dim, kv->d.format);
    a.blocks = blocks;
    hipLaunchKernelGGL(kernel, dim3(blocks * kv->d.kv_heads), dim3(kPlaceThreads), 0, static_cast<hipStream_t>(stream), a);
    return launch_error("es_kv_read_kernel launch");
} catch (const std::bad_alloc&) {
    return fail(ES_ERR_NOMEM, "es_kv_read: host allocation failed");
}

int es_kv_attend(es_kv_t* kv, const es_kv_attend_t* args, es_stream_t stream) try {
    const char* const name = "es_kv_attend";
    if (kv == nullptr || args == nullptr) return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    const es_kv_attend_t& x = *args;
    const uint32_t dim = kv->d.head_dim, heads = kv->d.kv_heads;
    if (x.rows > (1u << 24)) return fail_in(ES_ERR_INVALID_ARG, name, "rows above 2^24");
    if (x.n_seqs == 0 || x.n_seqs > 65536)
        return fail_in(ES_ERR_INVALID_ARG, name, "n_seqs out of range (1 .. 65536)");
    if (x.q_heads == 0 || x.q_heads % heads != 0 || x.q_heads / heads > 64)
        return fail_in(ES_ERR_INVALID_ARG, name,
                       "q_heads is not a multiple (1 .. 64) of the cache's kv_heads");
    if (!std::isfinite(x.scale)) return fail_in(ES_ERR_INVALID_ARG, name, "scale is not finite");
    if (!(x.cap >= 0.0f) || !std::isfinite(x.cap))
        return fail_in(ES_ERR_INVALID_ARG, name, "cap is negative or not finite");
    if (x.cap > 0.0f && x.cap < 0x1p-60f)
        return fail_in(ES_ERR_INVALID_ARG, name, "cap below 2^-60");
    if (x.table_stride == 0) return fail_in(ES_ERR_INVALID_ARG, name, "table_stride is 0");
    if (x.rows == 0) return ES_OK;
    if (x.q == nullptr || x.out == nullptr || x.tables == nullptr || x.lengths == nullptr ||
        x.starts == nullptr)
        return fail_in(ES_ERR_INVALID_ARG, name, "null pointer");
    const uint64_t width = uint64_t(x.q_heads) * dim;
    if (x.rows > 1 && x.out_stride < width)
        return fail_in(ES_ERR_INVALID_ARG, name, "the output's rows overlap");
    if (too_wide(x.rows, x.q_stride) || too_wide(x.rows, x.out_stride))
        return fail_in(ES_ERR_INVALID_ARG, name, "stride above 2^38");
    if (odd(x.q, 2) || odd(x.out, 2) || odd(x.tables, 4) || odd(x.lengths, 4) || odd(x.starts, 4) ||
        odd(x.first, 4) || odd(x.limit, 4) || odd(x.slopes, 4) || odd(x.status, 4))
        return fail_in(ES_ERR_ALIGN, name, "array not aligned to its elements");
    int rc = check_kv_device(kv, name);
    if (rc != ES_OK) return rc;
    Accesses ok{kv->device, name, {}};
    check_rows(ok, x.q, x.rows, width, x.q_stride, ": queries");
    check_rows(ok, x.out, x.rows, width, x.out_stride, ": output");
    ok.check(x.tables, uint64_t(4) * x.n_seqs * x.table_stride, ": tables");
    ok.check(x.lengths, uint64_t(4) * x.n_seqs, ": lengths");
    ok.check(x.starts, uint64_t(4) * (uint64_t(x.n_seqs) + 1), ": starts");
    ok.check(x.first, x.first != nullptr ? uint64_t(4) * x.rows : 0, ": first");
    ok.check(x.limit, x.limit != nullptr ? uint64_t(4) * x.rows : 0, ": limit");
    ok.check(x.slopes, x.slopes != nullptr ? uint64_t(4) * x.q_heads : 0, ": slopes");
    ok.check(x.status, x.status != nullptr ? 4 : 0, ": status");
    if (ok.rc != ES_OK) return ok.rc;
    AttendArgs a{};
    a.q = static_cast<const uint16_t*>(x.q);
    a.out = static_cast<uint16_t*>(x.out);
    a.q_stride = x.q_stride;
    a.out_stride = x.out_stride;
    a.tables = x.tables;
    a.lengths = x.lengths;
    a.starts = x.starts;
    a.first = x.first;
    a.limit = x.limit;
    a.slopes = x.slopes;
    a.status = x.status;
    a.part_o = kv->scratch;
    a.part_ml = kv->part_ml;
    a.rows = x.rows;
    a.n_seqs = x.n_seqs;
    a.table_stride = x.table_stride;
    a.group = x.q_heads / heads;
    a.scale = x.scale;
    a.cap = x.cap;
    a.c = kv->c;
    const uint32_t format = kv->d.format;
    const int mode = x.scale <= 0.0f || x.cap > kWideCap || (x.cap > 0.0f && x.slopes != nullptr)
                         ? kAny
                     : x.cap > 0.0f          ? kCapped
                     : x.slopes != nullptr   ? kSloped
                                             : kPlain;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const uint64_t all_rows = uint64_t(x.rows) * a.group;      // of one key head
    const uint64_t seq_rows = std::min<uint64_t>(x.rows, std::max(1u, x.max_rows)) * a.group;
    // Codes of long histories: up to 32 rows of a key head share one conversion in
    // registers, where the tile kernel would turn them for 128 (wide heads leave no
    // registers for it).  20 rows (40 heads over 8 x 128), E4M3, in split and tile
    // kernel: 64 histories of 3000 tokens 88 and 109 us, of 1500 52 and 58, of 800 33
    // and 32, 256 of 800 156 and 136; int8, 20 rows of 16 heads of 64, 64 of 2000 69
    // and 125.  bf16, which the tile kernel loads straight into LDS, 16 of 2000: 36
    // and 32.
    const uint32_t cols = seq_rows > kSplitRows && format != kBf16 && dim < 256 &&
                                  x.max_length >= kPairLength
                              ? 2
                              : 1;
    if (seq_rows <= kSplitRows * cols) {
        // a history's scores cost little beside its bytes: one kernel for every mode but plain
        const AttendKernel kernel =
            cols == 1 ? (mode == kPlain
                             ? by_dim_format<AttendKernel, MakeSplit<kPlain, 1>::Of>(dim, format)
                             : by_dim_format<AttendKernel, MakeSplit<kAny, 1>::Of>(dim, format))
                      : (mode == kPlain
                             ? by_dim_format<AttendKernel, MakeSplit<kPlain, 2>::Of>(dim, format)
                             : by_dim_format<AttendKernel, MakeSplit<kAny, 2>::Of>(dim, format));
        // Two workgroups a compute unit stream as fast as more, and a part left over
        // for a second round costs as long as all of the first: with few histories,
        // room for each one's short last part.  8 histories of 50000 to 65537 tokens
        // (int8) aimed at 512 and 448 parts: 230 and 200 us.  Not 1024, two rounds
        // of half the length: 194 there, but 108 for 100 at 64 of 2000 (bf16) and 136
        // for 127 at 8 of 20000 (bf16, 16 heads over 4 x 256).  How the histories'
        // remainders fall is not looked at: it moves a time by a few percent.
        const uint64_t pairs = uint64_t(x.n_seqs) * heads;
        a.target = kMaxParts - (pairs <= kMaxParts / 4 ? static_cast<uint32_t>(pairs) : 0u);
        a.min_blocks = kMinBlocks;
        return launch_parts(kernel, a, kSplitRows * cols, kSplitThreads, 0, seq_rows, x.max_length, dim, s);
    }
    const AttendKernel kernel =
        mode == kPlain    ? by_dim_format<AttendKernel, MakeTile<kPlain>::Of>(dim, format)
        : mode == kCapped ? by_dim_format<AttendKernel, MakeTile<kCapped>::Of>(dim, format)
        : mode == kSloped ? by_dim_format<AttendKernel, MakeTile<kSloped>::Of>(dim, format)
                          : by_dim_format<AttendKernel, MakeTile<kAny>::Of>(dim, format);
    const TileLaunch tile = dim == 64    ? tile_launch<64>()
                            : dim == 128 ? tile_launch<128>()
                                         : tile_launch<256>();
    // Tiles that fill less than half of the card are cut along long histories.  40
    // heads over 8 x 128, bf16, cut and whole: 13 rows after 12000 tokens 38 and 213
    // us, 200 rows 68 and 214; 800 rows of 3000 tokens (half a card) 69 and 65; a
    // prompt of 517 tokens (16 heads of 64) 14.4 and 12.2.
    const uint64_t n_tiles = all_rows / tile.rows + x.n_seqs;
    const uint64_t expected =
        std::min<uint64_t>(n_tiles, (seq_rows + tile.rows - 1) / tile.rows * x.n_seqs) * heads;
    const uint64_t blocks = (uint64_t(x.max_length) + kBlock - 1) / kBlock;
    if (expected < tile.resident / 2 && blocks >= kCutBlocks) {
        // a part more than its share for each tile, all on the card at once
        a.target = tile.resident - static_cast<uint32_t>(expected);
        a.min_blocks = kTileMinBlocks;
        return launch_parts(kernel, a, tile.rows, tile.threads, tile.lds, seq_rows, x.max_length, dim,
                            s);
    }
    if (n_tiles * heads >= kMaxGroups)
        return fail_in(ES_ERR_INVALID_ARG, name, "too many rows for one call");
    hipLaunchKernelGGL(kernel, dim3(n_tiles * heads), dim3(tile.threads), tile.lds, s, a);
    return launch_error("es_kv_tile_kernel launch");
} catch (const std::bad_alloc&) {
    return fail(ES_ERR_NOMEM, "es_kv_attend: host allocation failed");
}

}  // extern "C"
