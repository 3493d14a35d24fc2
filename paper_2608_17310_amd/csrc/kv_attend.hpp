// Attention over the cache: out = softmax(scores) V for the rows of a batch of
// sequences, each over its own interval of keys.
//
// Both kernels form the transposed products
//   S^T = K Q^T     (keys by rows)        O^T = V^T P^T     (dimensions by rows)
// with rows = query rows in the columns of the matrix instructions.  A
// column of S^T then lives in the lanes n, n + 16, ... (n + 32) of a wave, so a
// row's running maximum and sum are one register a lane, and the exponentials
// are, as they stand in the registers, the second product's right operand: nothing
// moves between lanes.  For that the keys are dealt to the rows of S^T in the
// order in which a lane of V^T reads them: consecutive tokens, one 16-byte word,
// because the cache holds values by dimension.
//
// The rows of a tile are pairs (token, query head of the group of one key
// head), numbered token-major: a group of any size shares its keys' loads.
//
// Softmax in units of log2, in binary32, over one pass with a running maximum.
// Weights are rounded to bf16 (RNE) for the matrix unit, after the product
// with the value's scale; their sum is taken before the rounding.
#pragma once

#include "kv_common.hpp"

namespace eskv {

constexpr int kBlock = 64;                  // keys of a block: never more than a page
// Tokens of a sequence at most: the kernels count keys in 32 bits with a sign, up to 512
// (two steps of a workgroup) past the last.
constexpr int64_t kMaxLength = (int64_t(1) << 31) - 1024;

struct AttendArgs {
    const uint16_t* q;
    uint16_t* out;
    uint64_t q_stride, out_stride;
    const int32_t* tables;
    const int32_t* lengths;
    const int32_t* starts;
    const int32_t* first;
    const int32_t* limit;
    const float* slopes;
    uint32_t* status;
    float* part_o;                          // [slots][rows of a tile][D]
    float* part_ml;                         // [slots][rows of a tile][2]: maximum, sum
    uint32_t rows, n_seqs, table_stride, group;
    uint32_t target, min_blocks;            // parts aimed at (0: none), blocks of a part at least
    float scale, cap;
    Cache c;
};

// A sequence of the batch: its rows [start, start + n) and its length, clamped
// into what q and the table hold.
struct Seq {
    int start, n, len;
};

__device__ __forceinline__ Seq read_seq(const AttendArgs& a, uint32_t s) {
    const int rows = static_cast<int>(a.rows);
    const int s0 = a.starts[s], s1 = a.starts[s + 1], len = a.lengths[s];
    const int64_t room = min(int64_t(a.table_stride) << a.c.page_shift, kMaxLength);
    Seq q;
    q.start = min(max(s0, 0), rows);
    q.n = min(max(s1, q.start), rows) - q.start;
    q.len = static_cast<int>(min(int64_t(max(len, 0)), room));
    if (a.status != nullptr &&
        (q.start != s0 || q.start + q.n != s1 || q.len != len || q.n > q.len))
        atomicOr(a.status, ES_KV_BAD_LENGTH);
    return q;
}

// The keys [first, limit) that row i of a sequence sees, empty as (0, 0).
__device__ __forceinline__ void interval(const AttendArgs& a, const Seq& s, int i, int& lo, int& hi) {
    lo = a.first != nullptr ? max(a.first[s.start + i], 0) : 0;
    hi = a.limit != nullptr ? a.limit[s.start + i] : s.len - s.n + i + 1;
    hi = min(hi, s.len);
    if (lo >= hi) lo = hi = 0;
}

constexpr float kWideCap = 256.0f;

// From the matrix unit's products to the softmax's units (log2), by what a call
// asks for.  A score is kept as x with t = unit x + offset, and a weight is
// 2^(unit x + (offset - base)), so that the last multiply and add are the
// exponential's: plain scores leave the scale to it, capped ones the cap.  kAny
// is several of the others together, a cap too wide for the closed form, or a
// scale that is not positive (which would turn the maximum of unscaled products
// round).
enum Mode : int { kPlain = 0, kCapped = 1, kSloped = 2, kAny = 3 };

struct ScoreMap {
    float factor;                           // of a product, first: log2(e) scale, or, capped,
                                            //   2 log2(e) scale / cap
    float unit, offset;
    float scale, cap;                       // log2(e) times the scale and the cap
    float slope;                            // log2(e) times the slope of this lane's row
    bool capped, wide, sloped;              // read by kAny
};

template <int kMode, bool kBytes>
__device__ __forceinline__ ScoreMap score_map(const AttendArgs& a, uint32_t head) {
    ScoreMap m;
    m.scale = a.scale * kLog2e;
    m.capped = a.cap > 0.0f;
    m.wide = a.cap > kWideCap;
    m.cap = a.cap * kLog2e;
    m.sloped = a.slopes != nullptr;
    m.slope = kMode >= kSloped && m.sloped ? a.slopes[head] * kLog2e : 0.0f;
    m.factor = (kMode == kCapped || kMode == kAny) && m.capped ? 2.0f * kLog2e * a.scale / a.cap
                                                               : m.scale;
    m.unit = kMode == kCapped ? -2.0f * m.cap : kMode == kPlain && !kBytes ? m.scale : 1.0f;
    m.offset = kMode == kCapped ? m.cap : 0.0f;
    return m;
}

// What x starts a maximum as, what stands for an unseen key, and the larger score.
template <int kMode>
__device__ __forceinline__ float unseen() {
    return kMode == kCapped ? inf() : -inf();
}
template <int kMode>
__device__ __forceinline__ float larger(float x, float y) {
    return kMode == kCapped ? __builtin_fminf(x, y) : __builtin_fmaxf(x, y);
}

// The closed form is off by about 2^-23 cap, which a wide cap makes large beside
// a small score: there the series of tanh, to y^9.
__device__ __forceinline__ float wide_cap(const ScoreMap& m, float z, float t) {
    const float y = z * 0.34657359f, y2 = y * y;             // ln(2) / 2
    float f = __builtin_fmaf(y2, 62.0f / 2835.0f, -17.0f / 315.0f);
    f = __builtin_fmaf(y2, f, 2.0f / 15.0f);
    f = __builtin_fmaf(y2, f, -1.0f / 3.0f);
    f = __builtin_fmaf(y2 * y, f, y);
    return __builtin_fabsf(y) < 0.25f ? m.cap * f : t;
}

// Products x of one row with N keys, key i of them at[i] places after a first
// one that lies `away` positions before the row; 8-bit keys' products come
// multiplied by the key's scale and m.factor.  `behind`: none of the keys lies
// ahead of any of the wave's rows.
template <int kMode, bool kBytes, int N, class At>
__device__ __forceinline__ void map_scores(const ScoreMap& m, float (&x)[N], float away, At at,
                                           bool behind) {
    if constexpr (kMode == kPlain) return;
    if constexpr (kMode == kCapped) {
        // tanh(y) = 1 - 2 / (1 + e^(2 y)), and x is the quotient; e^(2 y) may be infinite
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float z = kBytes ? x[i] : x[i] * m.factor;
            x[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z));
        }
    } else if constexpr (kMode == kSloped) {
        const float f = kBytes ? 1.0f : m.factor;
        if (behind) {
            // the distance is away - at: a term of the key and one of the row
            const float row = -m.slope * away;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float bias = __builtin_fmaf(m.slope, static_cast<float>(at(i)), row);
                x[i] = kBytes ? x[i] + bias : __builtin_fmaf(x[i], f, bias);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = __builtin_fabsf(away - static_cast<float>(at(i)));
                x[i] = __builtin_fmaf(-m.slope, d, kBytes ? x[i] : x[i] * f);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t = kBytes ? x[i] : x[i] * m.factor;
            if (m.capped) {
                const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
                const float near = __builtin_fmaf(-2.0f * m.cap, r, m.cap);
                t = m.wide ? wide_cap(m, t, near) : near;
            }
            const float d = __builtin_fabsf(away - static_cast<float>(at(i)));
            x[i] = m.sloped ? __builtin_fmaf(-m.slope, d, t) : t;
        }
    }
}

// A running maximum is kept until a score exceeds it by this much (log2): weights
// are at most 2^8 then, and the accumulators are seldom rescaled.
constexpr float kSlack = 8.0f;

// The larger of a value and the other half-wave's.
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// The largest of a value in the four lanes of a column of a 16-wide tile.
__device__ __forceinline__ float max_quarters(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return max_halves(__builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// ----------------------------------------------------------------------------
// Few rows over long histories: the keys of every sequence are cut into parts,
// a workgroup each, and joined by a second kernel.  Bound by the cache's bytes:
// a wave streams blocks of 64 keys straight from memory into the matrix
// unit's operands, with no LDS and no barrier before the workgroup's own join.
//
// The cut is made on the device from the lengths, so that a step can be
// replayed from a graph while histories grow: all sequences' parts have the same
// number of blocks, C = ceil(all blocks / target), and a workgroup finds its
// sequence by a scan over the batch (a wave, 64 sequences at a time).
//
// The matrix unit's columns are 16 rows of a tile (kCols of them): two share the
// loads and conversions of codes.
//
// Measured (one row, 40 query heads over 8 of 128): 8 histories of 30000, bf16,
// 182 us, 5.4 TB/s; 8 of 60000, E4M3, 181 us, 5.5 TB/s; 32 of 201 to 16384, E4M3, 63
// us with the join.
// ----------------------------------------------------------------------------

constexpr int kSplitThreads = 256;
constexpr int kSplitWaves = kSplitThreads / 64;
constexpr int kSplitRows = 16;              // of a tile's column of operands
// Rows of a sequence whose intervals the scan reads.  One with more counts as its whole
// history: parts in which its tiles see nothing are launched, and joined, empty.  A
// window of 1000 behind 12000 tokens (32 heads over 8 of 128, bf16): 100 rows 35 us, 46
// without the window; 300 rows 34 and 85.  And 64 rows 60 and 38: a lane reads their
// intervals one after another, in the kernel and in the join.
constexpr int kScanRows = 64;

// Waves of a SIMD that the registers leave.
template <int D, int kFmt, int kCols>
constexpr int split_waves() {
    return D == 64 ? 4 / kCols : D == 128 && kFmt == kBf16 && kCols == 1 ? 3 : 2;
}

struct Span {                               // a sequence's blocks
    Seq seq;
    int block0, blocks;                     // the first block that some row sees, and their number
    uint32_t tiles;                         // tiles of rows
};

__device__ __forceinline__ Span read_span(const AttendArgs& a, uint32_t s, int tile_rows) {
    Span p;
    p.seq = Seq{0, 0, 0};
    p.block0 = p.blocks = 0;
    p.tiles = 0;
    if (s >= a.n_seqs) return p;
    p.seq = read_seq(a, s);
    int lo = 0, hi = p.seq.len;
    if (p.seq.n <= kScanRows && (a.first != nullptr || a.limit != nullptr)) {
        lo = p.seq.len;
        hi = 0;
        for (int i = 0; i < p.seq.n; ++i) {
            int f, l;
            interval(a, p.seq, i, f, l);
            if (f < l) {
                lo = min(lo, f);
                hi = max(hi, l);
            }
        }
    }
    p.tiles = (uint32_t(p.seq.n) * a.group + tile_rows - 1) / tile_rows;
    if (lo < hi && p.tiles > 0) {
        p.block0 = lo / kBlock;
        p.blocks = (hi - 1) / kBlock + 1 - p.block0;
    }
    return p;
}

// Inclusive sums over the lanes of a wave, in six adds of neighbouring registers:
// within rows of 16 lanes, then each row's last lane into the next rows.
template <int kControl, int kRows>
__device__ __forceinline__ uint32_t add_moved(uint32_t x) {
    return x + static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
                   0, static_cast<int>(x), kControl, kRows, 0xF, false));
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    constexpr int kRowShr = 0x110, kRowBcast15 = 0x142, kRowBcast31 = 0x143;
    x = add_moved<kRowShr | 1, 0xF>(x);
    x = add_moved<kRowShr | 2, 0xF>(x);
    x = add_moved<kRowShr | 4, 0xF>(x);
    x = add_moved<kRowShr | 8, 0xF>(x);
    x = add_moved<kRowBcast15, 0xA>(x);
    return add_moved<kRowBcast31, 0xC>(x);
}

__device__ __forceinline__ int from_lane(int x, int lane) {
    return __builtin_amdgcn_readlane(x, lane);
}

// A tile of rows of one sequence, and (kParts) one part of its blocks.
struct Place {
    Seq seq;
    uint32_t s;                             // the sequence
    int block0, blocks;                     // the sequence's blocks
    uint32_t tile, chunk, chunks, per;      // per: blocks of a part
    uint32_t slot;                          // of the tile's first part, over the batch (chunks > 1)
    bool found;
};

// The place numbered `unit` among all parts (kParts) or tiles of the batch.
// Every lane of the wave calls it and gets the same answer.
template <bool kParts>
__device__ __forceinline__ Place find_place(const AttendArgs& a, int tile_rows, uint32_t unit) {
    const uint32_t lane = threadIdx.x & 63;
    const Span mine = read_span(a, lane, tile_rows);
    // all blocks of one head, 64 sequences at a time, in two sums of 32 bits (a cache
    // has at most 2^25 blocks); a part of 2^30 blocks or more is all of any history
    uint64_t total = 0;
    for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += 64) {
        const Span p = s0 == 0 ? mine : read_span(a, s0 + lane, tile_rows);
        const uint64_t work = uint64_t(p.blocks) * p.tiles;
        const uint32_t lo = wave_scan(static_cast<uint32_t>(work & 0xFFFFFFu));
        const uint32_t hi = wave_scan(static_cast<uint32_t>(work >> 24) & 0x3FFFFFFu);
        total += (uint64_t(from_lane(hi, 63)) << 24) + uint32_t(from_lane(lo, 63));
    }
    const uint64_t all = total * a.c.heads;
    uint32_t per = a.min_blocks;
    if (all > uint64_t(a.min_blocks) * a.target)
        per = static_cast<uint32_t>(min((all + a.target - 1) / a.target, uint64_t(1) << 30));
    Place r;
    r.per = __builtin_amdgcn_readfirstlane(per);
    r.found = false;
    uint32_t units0 = 0, slots0 = 0;
    for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += 64) {
        const Span p = s0 == 0 ? mine : read_span(a, s0 + lane, tile_rows);
        const uint32_t chunks = max(1u, (uint32_t(p.blocks) + r.per - 1) / r.per);
        const uint32_t units = p.tiles * (kParts ? chunks : 1u);
        const uint32_t slots = chunks > 1 ? p.tiles * chunks : 0u;
        const uint32_t units1 = wave_scan(units), slots1 = wave_scan(slots);
        const uint64_t past = __ballot(units0 + units1 > unit);
        if (past != 0) {
            const int src = __builtin_ctzll(past);
            r.seq = Seq{from_lane(p.seq.start, src), from_lane(p.seq.n, src),
                        from_lane(p.seq.len, src)};
            r.s = s0 + src;
            r.block0 = from_lane(p.block0, src);
            r.blocks = from_lane(p.blocks, src);
            r.chunks = from_lane(chunks, src);
            const uint32_t in = unit - units0 - from_lane(units1 - units, src);
            r.tile = kParts ? in / r.chunks : in;
            r.chunk = kParts ? in % r.chunks : 0u;
            r.slot = slots0 + from_lane(slots1 - slots, src) + r.tile * r.chunks;
            r.found = r.tile < uint32_t(from_lane(p.tiles, src));
            return r;
        }
        units0 += from_lane(units1, 63);
        slots0 += from_lane(slots1, 63);
    }
    return r;
}

template <int D, int kFmt, int kMode, int kCols>
__global__ __launch_bounds__(kSplitThreads, (split_waves<D, kFmt, kCols>())) void
es_kv_split_kernel(AttendArgs a) {
    constexpr int kSteps = D / 32;                           // 32 dimensions a product
    constexpr int kDims = D / 16;                            // 16 dimensions a tile of O^T
    constexpr bool kBytes = kFmt != kBf16;
    // A step takes 4 L keys, as tiles of 16: a lane holds L tokens of each of its
    // dimensions, 16 bytes, or 8 of wide heads, whose registers leave no room for more
    constexpr int L = kBytes && D <= 128 ? 16 : 8;
    constexpr int kKeys = 4 * L, kKeyTiles = L / 4, kPairs = L / 8;
    typedef uint32_t Tokens __attribute__((ext_vector_type(L * kCodeBytes<kFmt> / 4)));
    constexpr int kRowBytes = D * kCodeBytes<kFmt>;
    constexpr int kKeyWords = kRowBytes / 64;                // 16-byte words of a lane of a key's row
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int base_key = L * g;                              // of this lane's keys in a step
    const uint32_t h = blockIdx.x % a.c.heads;

    const Place at = find_place<true>(a, kSplitRows * kCols, blockIdx.x / a.c.heads);
    if (!at.found) return;

    // this lane's rows: columns n, 16 + n of the tile.  Columns past the last row
    // repeat it and are not written.
    const int n_rows = at.seq.n * static_cast<int>(a.group);
    const int row0 = static_cast<int>(at.tile) * kSplitRows * kCols;
    int row_i[kCols], first[kCols], limit[kCols], pos[kCols];
    uint32_t head[kCols];
    ScoreMap map[kCols];
    bf16x8_t q[kCols][kSteps];
    int lo_any = at.seq.len, hi_any = 0, lo_all = 0, hi_all = at.seq.len;
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        const int rr = min(row0 + kSplitRows * c + n, n_rows - 1);
        const int i = rr / static_cast<int>(a.group);
        row_i[c] = i;
        head[c] = h * a.group + (rr - i * static_cast<int>(a.group));
        interval(a, at.seq, i, first[c], limit[c]);
        pos[c] = at.seq.len - at.seq.n + i;
        map[c] = score_map<kMode, kBytes>(a, head[c]);
        lo_any = min(lo_any, first[c] < limit[c] ? first[c] : at.seq.len);
        hi_any = max(hi_any, limit[c]);
        lo_all = max(lo_all, first[c]);
        hi_all = min(hi_all, limit[c]);
        const uint16_t* src =
            a.q + uint64_t(at.seq.start + i) * a.q_stride + uint64_t(head[c]) * D;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            // the dimensions that a lane's words of a key hold: 8 of 32, or 16 of 64
            const int d = kBytes ? 64 * (s / 2) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
            q[c][s] = __builtin_bit_cast(bf16x8_t, load_row8(src + d));
        }
    }
#pragma unroll
    for (int m = 1; m < 16; m *= 2) {
        lo_any = min(lo_any, __shfl_xor(lo_any, m));
        hi_any = max(hi_any, __shfl_xor(hi_any, m));
        lo_all = max(lo_all, __shfl_xor(lo_all, m));
        hi_all = min(hi_all, __shfl_xor(hi_all, m));
    }
    lo_any = __builtin_amdgcn_readfirstlane(lo_any);
    hi_any = __builtin_amdgcn_readfirstlane(hi_any);
    lo_all = __builtin_amdgcn_readfirstlane(lo_all);
    hi_all = __builtin_amdgcn_readfirstlane(hi_all);

    float top[kCols], sum[kCols];
    f32x4_t o[kCols][kDims];
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        top[c] = -inf();
        sum[c] = 0.0f;
#pragma unroll
        for (int d = 0; d < kDims; ++d) o[c][d] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // the part's keys that some row of the tile sees, in whole steps
    const int part0 = at.block0 + static_cast<int>(at.chunk * at.per);
    const int part1 = min(at.block0 + at.blocks, part0 + static_cast<int>(at.per));
    const int k_begin = max(part0 * kBlock, lo_any / kKeys * kKeys);
    const int k_end = min(part1 * kBlock, hi_any);
    const int32_t* table = a.tables + uint64_t(at.s) * a.table_stride;
    const uint32_t val_row = a.c.page * kCodeBytes<kFmt>;    // bytes of a dimension's page
    const uint32_t k_off = (L * (n >> 2) + (n & 3)) * kRowBytes + 16 * g;
    const uint32_t v_off = n * val_row + base_key * kCodeBytes<kFmt>;
    auto page_of = [&](int key0) -> uint32_t {
        return key0 < k_end ? load_uniform(table + (key0 >> a.c.page_shift)) : 0u;
    };
    uint32_t page = page_of(k_begin + wave * kKeys);
    for (int key0 = k_begin + wave * kKeys; key0 < k_end; key0 += kSplitWaves * kKeys) {
        const bool bad = page >= a.c.n_pages;
        const uint64_t head_at = uint64_t(bad ? 0u : page) * a.c.heads + h;
        page = page_of(key0 + kSplitWaves * kKeys);
        const uint32_t off = uint32_t(key0) & (a.c.page - 1);
        const uint64_t token = (head_at << a.c.page_shift) + off;

        // the step's keys: word w of the key that row n of tile t stands for
        const Buffer keys = buffer_of(a.c.k + token * kRowBytes, kKeys * kRowBytes);
        u32x4_t kw[kKeyTiles][kKeyWords];
#pragma unroll
        for (int t = 0; t < kKeyTiles; ++t)
#pragma unroll
            for (int w = 0; w < kKeyWords; ++w)
                kw[t][w] = load_buffer(keys, k_off + 4 * t * kRowBytes + 64 * w);
        // its values: this lane's tokens of dimension 16 d + n
        const Buffer values =
            buffer_of(a.c.v + ((head_at << a.c.page_shift) * D + off) * kCodeBytes<kFmt>,
                      val_row * D - off * kCodeBytes<kFmt>);
        Tokens vw[kDims];
#pragma unroll
        for (int d = 0; d < kDims; ++d)
            vw[d] = load_buffer_as<Tokens>(values, v_off, 16 * d * val_row);
        // its scales
        f32x4_t ks[kKeyTiles], vs[kKeyTiles];
        if constexpr (kBytes) {
            const Buffer k_scales = buffer_of(a.c.ks + token, 4 * kKeys);
            const Buffer v_scales = buffer_of(a.c.vs + token, 4 * kKeys);
#pragma unroll
            for (int t = 0; t < kKeyTiles; ++t) {
                ks[t] = __builtin_bit_cast(f32x4_t, load_buffer(k_scales, 4 * (base_key + 4 * t)));
                vs[t] = __builtin_bit_cast(f32x4_t, load_buffer(v_scales, 4 * (base_key + 4 * t)));
            }
        }

        // slots that a row does not see may hold anything; its weight of zero meets
        // finite values
        const bool masked = key0 < lo_all || key0 + kKeys > hi_all;
        if constexpr (kBytes) {
#pragma unroll
            for (int t = 0; t < kKeyTiles; ++t) ks[t] *= map[0].factor;
            if (masked) {
#pragma unroll
                for (int t = 0; t < L; ++t) vs[t >> 2][t & 3] = finite_scale(vs[t >> 2][t & 3]);
            }
        }
        f32x4_t s[kCols][kKeyTiles];
#pragma unroll
        for (int k = 0; k < kKeyTiles; ++k)
#pragma unroll
            for (int w = 0; w < kKeyWords; ++w) {
                constexpr int kHalves = kBytes ? 2 : 1;
#pragma unroll
                for (int y = 0; y < kHalves; ++y) {
                    bf16x8_t x;
                    if constexpr (kBytes)
                        x = __builtin_bit_cast(
                            bf16x8_t,
                            codes_to_bf16<kFmt>(u32x2_t{kw[k][w][2 * y], kw[k][w][2 * y + 1]}));
                    else
                        x = __builtin_bit_cast(bf16x8_t, kw[k][w]);
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
                        s[c][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            x, q[c][kHalves * w + y], w + y == 0 ? f32x4_t{} : s[c][k], 0, 0, 0);
                }
            }
        bf16x8_t p[kCols][kPairs];
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            // scores of a row and this lane's keys key0 + base_key + 0 .. L - 1
            float x[L];
#pragma unroll
            for (int k = 0; k < L; ++k)
                x[k] = kBytes ? s[c][k >> 2][k & 3] * ks[k >> 2][k & 3] : s[c][k >> 2][k & 3];
            map_scores<kMode, kBytes>(map[c], x, static_cast<float>(pos[c] - key0 - base_key),
                                      [](int i) { return i; }, false);
            if (bad) {
#pragma unroll
                for (int k = 0; k < L; ++k) x[k] = nan();
            }
            if (masked) {
                const int from = first[c] - key0 - base_key, to = limit[c] - key0 - base_key;
#pragma unroll
                for (int k = 0; k < L; ++k)
                    if (k < from || k >= to) x[k] = unseen<kMode>();
            }
            float peak = x[0];
#pragma unroll
            for (int k = 1; k < L; ++k) peak = larger<kMode>(peak, x[k]);
            peak = max_quarters(__builtin_fmaf(peak, map[c].unit, map[c].offset));
            const float now = __builtin_fmaxf(top[c], peak);
            if (__any(now > top[c] + kSlack)) {
                const float shrink = __builtin_amdgcn_exp2f(top[c] - (now == -inf() ? 0.0f : now));
                sum[c] *= shrink;
#pragma unroll
                for (int d = 0; d < kDims; ++d) o[c][d] *= shrink;
                top[c] = now;
            }
            // nothing seen so far: any finite stand-in gives weights of zero
            const float base = map[c].offset - (top[c] == -inf() ? 0.0f : top[c]);
#pragma unroll
            for (int u = 0; u < kPairs; ++u) {
                u32x4_t w;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float e[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int k = 8 * u + 2 * j + y;
                        e[y] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[k], map[c].unit, base));
                        sum[c] += e[y];
                        if constexpr (kBytes) e[y] *= vs[k >> 2][k & 3];
                    }
                    w[j] = pack_bf16(e[0], e[1]);
                }
                p[c][u] = __builtin_bit_cast(bf16x8_t, w);
            }
        }
        if (bad && a.status != nullptr && lane == 0) atomicOr(a.status, ES_KV_BAD_PAGE);
        if (masked && kFmt != kInt8) {
#pragma unroll
            for (int d = 0; d < kDims; ++d)
#pragma unroll
                for (int w = 0; w < L * kCodeBytes<kFmt> / 4; ++w) vw[d][w] = finite<kFmt>(vw[d][w]);
        }
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
#pragma unroll
            for (int u = 0; u < kPairs; ++u) {
                bf16x8_t v;
                if constexpr (kBytes)
                    v = __builtin_bit_cast(
                        bf16x8_t, codes_to_bf16<kFmt>(u32x2_t{vw[d][2 * u], vw[d][2 * u + 1]}));
                else
                    v = __builtin_bit_cast(bf16x8_t, vw[d]);
#pragma unroll
                for (int c = 0; c < kCols; ++c)
                    o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[c][u], o[c][d], 0, 0, 0);
            }
        }
    }

    // join the waves: the others hand their sums to wave 0 through LDS
    __shared__ float ml[kCols][kSplitWaves][2][16];
    __shared__ __attribute__((aligned(16))) f32x4_t part[kCols][kSplitWaves - 1][kDims][64];
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        sum[c] += __shfl_xor(sum[c], 16);
        sum[c] += __shfl_xor(sum[c], 32);
        if (g == 0) {
            ml[c][wave][0][n] = top[c];
            ml[c][wave][1][n] = sum[c];
        }
    }
    __syncthreads();
    float m[kCols], mine[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        m[c] = -inf();
#pragma unroll
        for (int w = 0; w < kSplitWaves; ++w) m[c] = __builtin_fmaxf(m[c], ml[c][w][0][n]);
        mine[c] = __builtin_amdgcn_exp2f(top[c] - (m[c] == -inf() ? 0.0f : m[c]));
        if (wave > 0) {
#pragma unroll
            for (int d = 0; d < kDims; ++d) part[c][wave - 1][d][lane] = o[c][d] * mine[c];
        }
    }
    __syncthreads();
    if (wave > 0) return;
    const bool whole = at.chunks == 1;
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        if (row0 + kSplitRows * c + n >= n_rows) continue;
        const float base = m[c] == -inf() ? 0.0f : m[c];
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < kSplitWaves; ++w)
            total += ml[c][w][1][n] * __builtin_amdgcn_exp2f(ml[c][w][0][n] - base);
        const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
        const uint64_t slot =
            (((uint64_t(at.slot) + at.chunk) * a.c.heads + h) * kCols + c) * kSplitRows + n;
        uint16_t* out =
            a.out + uint64_t(at.seq.start + row_i[c]) * a.out_stride + uint64_t(head[c]) * D;
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
            f32x4_t x = o[c][d] * mine[c];
#pragma unroll
            for (int w = 0; w < kSplitWaves - 1; ++w) x += part[c][w][d][lane];
            if (whole) {
                x *= inv;
                store_row4(out + 16 * d + 4 * g,
                           u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])});
            } else {
                store<f32x4_t>(a.part_o + slot * D + 16 * d + 4 * g, x);
            }
        }
        if (!whole && g == 0) {
            a.part_ml[2 * slot] = m[c];
            a.part_ml[2 * slot + 1] = total;
        }
    }
}

// Join the parts of each row: out = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c.
// D / 4 lanes hold a row.  With `spread` a workgroup takes one row, its lanes'
// groups every so many parts each, joined in LDS (a row in many parts); without,
// every group takes a row of its own.  Rows blockIdx.y, + gridDim.y, ... (of
// groups of rows) of the tile.
template <int D>
__global__ __launch_bounds__(kSplitThreads) void es_kv_join_kernel(AttendArgs a, int tile_rows,
                                                                   int spread) {
    constexpr int kLanes = D / 4;
    constexpr int kGroups = kSplitThreads / kLanes;
    const uint32_t h = blockIdx.x % a.c.heads;
    const Place at = find_place<false>(a, tile_rows, blockIdx.x / a.c.heads);
    if (!at.found || at.chunks <= 1) return;
    const int n_rows = min(at.seq.n * static_cast<int>(a.group) -
                               static_cast<int>(at.tile) * tile_rows, tile_rows);
    const int lane = threadIdx.x % kLanes, grp = threadIdx.x / kLanes;
    __shared__ float ml[kGroups][2];
    __shared__ __attribute__((aligned(16))) f32x4_t part[kGroups][kLanes];
    const int per = spread ? 1 : kGroups;                    // rows of a workgroup at a time
    for (int y0 = blockIdx.y * per; y0 < n_rows; y0 += gridDim.y * per) {
        const int y = spread ? y0 : min(y0 + grp, n_rows - 1);
        float m = -inf(), l = 0.0f;
        f32x4_t o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (uint32_t c = spread ? grp : 0; c < at.chunks; c += spread ? kGroups : 1) {
            const uint64_t slot = ((uint64_t(at.slot) + c) * a.c.heads + h) * tile_rows + y;
            const float mc = a.part_ml[2 * slot], lc = a.part_ml[2 * slot + 1];
            const f32x4_t oc = load<f32x4_t>(a.part_o + slot * D + 4 * lane);
            const float now = __builtin_fmaxf(m, mc);
            const float base = now == -inf() ? 0.0f : now;
            const float x = __builtin_amdgcn_exp2f(m - base), z = __builtin_amdgcn_exp2f(mc - base);
            l = l * x + lc * z;
            o = o * x + oc * z;
            m = now;
        }
        if (spread) {
            if (lane == 0) {
                ml[grp][0] = m;
                ml[grp][1] = l;
            }
            part[grp][lane] = o;
            __syncthreads();
            m = -inf();
#pragma unroll
            for (int k = 0; k < kGroups; ++k) m = __builtin_fmaxf(m, ml[k][0]);
            const float base = m == -inf() ? 0.0f : m;
            o = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            l = 0.0f;
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                const float z = __builtin_amdgcn_exp2f(ml[k][0] - base);
                l += ml[k][1] * z;
                o += part[k][lane] * z;
            }
            __syncthreads();
        }
        if (spread ? grp == 0 : y0 + grp < n_rows) {
            o *= l > 0.0f || l != l ? 1.0f / l : 0.0f;
            const int r = static_cast<int>(at.tile) * tile_rows + y;
            const int i = r / static_cast<int>(a.group);
            const uint32_t head = h * a.group + (r - i * static_cast<int>(a.group));
            store_row4(a.out + uint64_t(at.seq.start + i) * a.out_stride + uint64_t(head) * D +
                           4 * lane,
                       u32x2_t{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])});
        }
    }
}

// ----------------------------------------------------------------------------
// Many rows: a workgroup of four waves takes 128 rows of one key head, 32 to a
// wave, over all blocks that some of them see.  Bound by the matrix unit beside
// the exponentials: keys and values are staged in LDS as bf16, once for all
// waves, double-buffered, the next block on its way under the present one's
// products: bf16 straight into LDS, codes through registers (converted once).
// Two workgroups share a compute unit: with a barrier a block, waves of one
// workgroup compute products and exponentials at the same time, and only
// another workgroup's fill the other unit meanwhile (one of eight waves was as fast
// in bf16 and 8 % slower from codes).
//
// Measured: a prompt of 8192 (40 heads over 8 of 128, bf16) 660 us, 1.04 PFLOP/s of
// visible products, the matrix unit busy 53 % of cycles at 1.95 GHz; without the
// staging loads 14 % less, without the exponentials 7 %.  16 ragged prompts up to
// 2039 (int8, bias) 204 us, 0.57 PFLOP/s; documents of 6001 tokens (E4M3, capped) 138.
//
// LDS rows are 2 D bytes (keys) and 128 bytes (values); their 16-byte words
// are exchanged by the row's number so that 16 rows of one word lie in 16
// different groups of banks.
// ----------------------------------------------------------------------------

template <int D>
struct TileShape {
    static constexpr int kWaves = 4;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kRows = 32 * kWaves;
    static constexpr int kKeyBytes = kBlock * D * 2;
    static constexpr int kBuffer = 2 * kKeyBytes;            // keys, then as many bytes of values
    static constexpr int kLds = 2 * kBuffer + 256 * 4;       //   and the scales of both
    static constexpr int kPerSimd = D == 256 ? 1 : 2;        // waves of a SIMD that the registers leave
};

// Byte offsets of 16-byte words in the staged tiles.
template <int D>
__device__ __forceinline__ int key_word(int row, int w) {
    if constexpr (D == 64) return row * 128 + 16 * (w ^ ((row >> 1) & 7));
    return row * (2 * D) + 16 * (w ^ (row & 15));
}
__device__ __forceinline__ int val_word(int row, int w) {
    return row * 128 + 16 * (w ^ ((row >> 1) & 7));
}

// A workgroup's tile of rows: the sequence and the tile, found like a part.
__device__ __forceinline__ Place find_tile(const AttendArgs& a, int tile_rows, uint32_t unit) {
    const uint32_t lane = threadIdx.x & 63;
    Place r;
    r.found = false;
    uint32_t units0 = 0;
    for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += 64) {
        const uint32_t s = s0 + lane;
        const Seq q = s < a.n_seqs ? read_seq(a, s) : Seq{0, 0, 0};
        const uint32_t units = (uint32_t(q.n) * a.group + tile_rows - 1) / tile_rows;
        const uint32_t units1 = wave_scan(units);
        const uint64_t past = __ballot(units0 + units1 > unit);
        if (past != 0) {
            const int src = __builtin_ctzll(past);
            r.seq = Seq{from_lane(q.start, src), from_lane(q.n, src), from_lane(q.len, src)};
            r.s = s0 + src;
            // the last tiles, which see the most keys, first
            const uint32_t in = unit - units0 - from_lane(units1 - units, src);
            r.found = in < uint32_t(from_lane(units, src));
            r.tile = from_lane(units, src) - 1 - in;
            return r;
        }
        units0 += from_lane(units1, 63);
    }
    return r;
}

template <int D, int kFmt, int kMode>
__global__ __launch_bounds__(TileShape<D>::kThreads, TileShape<D>::kPerSimd) void
es_kv_tile_kernel(AttendArgs a) {
    using S = TileShape<D>;
    constexpr bool kBytes = kFmt != kBf16;
    constexpr int kSteps = D / 16;                           // 16 dimensions a product
    constexpr int kDims = D / 32;                            // 32 dimensions a tile of O^T
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, g = lane >> 5;
    const uint32_t h = blockIdx.x % a.c.heads;

    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ int bounds[4][S::kWaves];

    const bool parts = a.target != 0;
    const Place at = parts ? find_place<true>(a, S::kRows, blockIdx.x / a.c.heads)
                           : find_tile(a, S::kRows, blockIdx.x / a.c.heads);
    if (!at.found) return;

    const int n_rows = at.seq.n * static_cast<int>(a.group);
    const int r = static_cast<int>(at.tile) * S::kRows + 32 * wave + n;
    const int rr = min(r, n_rows - 1);
    const int i = rr / static_cast<int>(a.group);
    const uint32_t head = h * a.group + (rr - i * static_cast<int>(a.group));
    int first, limit;
    interval(a, at.seq, i, first, limit);
    // a wave of no rows (the last tile's) sees nothing and passes every block
    const bool has_rows = static_cast<int>(at.tile) * S::kRows + 32 * wave < n_rows;
    if (!has_rows) first = limit = 0;
    const int pos = at.seq.len - at.seq.n + i;
    const ScoreMap map = score_map<kMode, kBytes>(a, head);
    // positions grow with rows.  Steep slopes take distances one by one: a block's
    // term of the row rounds to 2^-24 of up to 128 slopes
    const int pos_first =
        __any(map.slope > 4.0f || map.slope < -4.0f) ? -1 : __builtin_amdgcn_readfirstlane(pos);

    bf16x8_t q[kSteps];
    {
        const uint16_t* src = a.q + uint64_t(at.seq.start + i) * a.q_stride + uint64_t(head) * D;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            q[s] = __builtin_bit_cast(bf16x8_t, load_row8(src + 16 * s + 8 * g));
    }

    // what the wave's rows see, some and all of them; and the workgroup's (whole: all)
    int lo_any, hi_any, lo_all, hi_all, lo, hi, whole_lo, whole_hi;
    if (a.first == nullptr && a.limit == nullptr) {
        // up to their own positions, which grow with rows: no wave waits for another
        lo_all = lo = whole_lo = 0;
        hi_all = from_lane(limit, 0);
        hi_any = from_lane(limit, 31);
        lo_any = hi_any > 0 ? 0 : at.seq.len;
        const int last = min(static_cast<int>(at.tile + 1) * S::kRows, n_rows) - 1;
        hi = min(at.seq.len, at.seq.len - at.seq.n + last / static_cast<int>(a.group) + 1);
        const int lead = static_cast<int>(at.tile) * S::kRows / static_cast<int>(a.group);
        whole_hi = min(at.seq.len, at.seq.len - at.seq.n + lead + 1);
    } else {
        lo_any = first < limit ? first : at.seq.len;
        hi_any = limit;
        lo_all = first;
        hi_all = limit;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            lo_any = min(lo_any, __shfl_xor(lo_any, m));
            hi_any = max(hi_any, __shfl_xor(hi_any, m));
            lo_all = max(lo_all, __shfl_xor(lo_all, m));
            hi_all = min(hi_all, __shfl_xor(hi_all, m));
        }
        lo_any = __builtin_amdgcn_readfirstlane(lo_any);
        hi_any = __builtin_amdgcn_readfirstlane(hi_any);
        lo_all = __builtin_amdgcn_readfirstlane(lo_all);
        hi_all = __builtin_amdgcn_readfirstlane(hi_all);
        if (lane == 0) {
            bounds[0][wave] = lo_any;
            bounds[1][wave] = hi_any;
            bounds[2][wave] = has_rows ? lo_all : 0;
            bounds[3][wave] = has_rows ? hi_all : at.seq.len;
        }
        __syncthreads();
        lo = whole_hi = at.seq.len;
        hi = whole_lo = 0;
#pragma unroll
        for (int w = 0; w < S::kWaves; ++w) {
            lo = min(lo, bounds[0][w]);
            hi = max(hi, bounds[1][w]);
            whole_lo = max(whole_lo, bounds[2][w]);
            whole_hi = min(whole_hi, bounds[3][w]);
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        hi = __builtin_amdgcn_readfirstlane(hi);
        whole_lo = __builtin_amdgcn_readfirstlane(whole_lo);
        whole_hi = __builtin_amdgcn_readfirstlane(whole_hi);
    }
    int b_begin = lo / kBlock, b_end = hi > lo ? (hi - 1) / kBlock + 1 : b_begin;
    if (parts) {
        const int part0 = at.block0 + static_cast<int>(at.chunk * at.per);
        b_begin = max(b_begin, part0);
        b_end = min(b_end, min(at.block0 + at.blocks, part0 + static_cast<int>(at.per)));
    }

    // staging: 16-byte words of codes, each thread kStage of the keys' and of the values'
    constexpr int kStage = kBlock * D * kCodeBytes<kFmt> / 16 / S::kThreads;
    static_assert(kStage * S::kThreads * 16 == kBlock * D * kCodeBytes<kFmt>,
                  "staging covers the block");
    constexpr int kKeyWords = D * kCodeBytes<kFmt> / 16;     // words of a key's row
    constexpr int kValWords = kBlock * kCodeBytes<kFmt> / 16;    // of a dimension's tokens
    const uint32_t val_row = a.c.page * kCodeBytes<kFmt>;    // bytes of a dimension's page
    // bf16: word p of the staged tile is the 16 bytes at these offsets of the block
    uint32_t k_off[kStage], v_off[kStage];
#pragma unroll
    for (int x = 0; x < kStage; ++x) {
        const int p = (wave * kStage + x) * 64 + lane;
        const int kr = p / kKeyWords, kw = p % kKeyWords, vr = p / kValWords, vw = p % kValWords;
        k_off[x] = key_word<D>(kr, kw);
        v_off[x] = vr * val_row + 16 * (vw ^ ((vr >> 1) & 7));
    }
    // Slots that a row does not see may hold anything: in blocks that not all rows
    // see in full, values that are not finite are cleared, so that a weight of zero
    // gives zero.  (Stored tokens have none; in other blocks every row sees them.)
    // Each lane tests the words that it loaded and writes only where it found some:
    // documents of 6001 tokens 138 us, 136 without and 142 when all are rewritten; a
    // prompt of 517 12.1, 11.7 and 12.3.
    auto unclear = [&](int b) { return b * kBlock < whole_lo || (b + 1) * kBlock > whole_hi; };
    u32x4_t sk[kBytes ? kStage : 1], sv[kBytes ? kStage : 1];
    float sscale = 0.0f;
    bool bad = false, bad_next = false;
    const int32_t* table = a.tables + uint64_t(at.s) * a.table_stride;
    // a block's page, asked for a block ahead of its keys and values
    auto page_of = [&](int b) -> uint32_t {
        return b < b_end ? load_uniform(table + ((b * kBlock) >> a.c.page_shift)) : 0u;
    };
    auto fetch = [&](int b, uint32_t page, uint8_t* buf) {
        bad_next = page >= a.c.n_pages;
        const uint64_t head_at = uint64_t(bad_next ? 0u : page) * a.c.heads + h;
        const uint32_t off = uint32_t(b * kBlock) & (a.c.page - 1);
        const uint64_t token = (head_at << a.c.page_shift) + off;
        const Buffer keys = buffer_of(a.c.k + token * (D * kCodeBytes<kFmt>),
                                      kBlock * D * kCodeBytes<kFmt>);
        const Buffer values =
            buffer_of(a.c.v + ((head_at << a.c.page_shift) * D + off) * kCodeBytes<kFmt>,
                      val_row * D - off * kCodeBytes<kFmt>);
        if constexpr (kBytes) {
#pragma unroll
            for (int x = 0; x < kStage; ++x) {
                const uint32_t w = threadIdx.x + S::kThreads * x;
                sk[x] = load_buffer(keys, 16 * w);
                sv[x] = load_buffer(values, (w / kValWords) * val_row + 16 * (w % kValWords));
            }
            if (threadIdx.x < 2 * kBlock)
                sscale = load_buffer_float(
                    buffer_of((wave < kBlock / 64 ? a.c.ks : a.c.vs) + token, 4 * kBlock),
                    4 * (threadIdx.x & (kBlock - 1)));
        } else {
#pragma unroll
            for (int x = 0; x < kStage; ++x) {
                load_to_lds(keys, k_off[x], buf + (wave * kStage + x) * 1024);
                load_to_lds(values, v_off[x], buf + S::kKeyBytes + (wave * kStage + x) * 1024);
            }
        }
        if (bad_next && a.status != nullptr && threadIdx.x == 0)
            atomicOr(a.status, ES_KV_BAD_PAGE);
    };
    // (keys' scales carry the scores' first factor)
    auto stage = [&](int b, uint8_t* buf, float* scales) {
        if constexpr (kBytes) {
            if (unclear(b)) {
                make_finite<kFmt>(sv);
                if (wave >= kBlock / 64) sscale = finite_scale(sscale);
            }
#pragma unroll
            for (int x = 0; x < kStage; ++x) {
                const int w = threadIdx.x + S::kThreads * x;
                const int kr = w / kKeyWords, kc = w % kKeyWords;
                const int vr = w / kValWords, vc = w % kValWords;
                *reinterpret_cast<u32x4_t*>(buf + key_word<D>(kr, 2 * kc)) =
                    codes_to_bf16<kFmt>(u32x2_t{sk[x][0], sk[x][1]});
                *reinterpret_cast<u32x4_t*>(buf + key_word<D>(kr, 2 * kc + 1)) =
                    codes_to_bf16<kFmt>(u32x2_t{sk[x][2], sk[x][3]});
                *reinterpret_cast<u32x4_t*>(buf + S::kKeyBytes + val_word(vr, 2 * vc)) =
                    codes_to_bf16<kFmt>(u32x2_t{sv[x][0], sv[x][1]});
                *reinterpret_cast<u32x4_t*>(buf + S::kKeyBytes + val_word(vr, 2 * vc + 1)) =
                    codes_to_bf16<kFmt>(u32x2_t{sv[x][2], sv[x][3]});
            }
            if (threadIdx.x < kBlock)
                scales[threadIdx.x] = sscale * map.factor;
            else if (threadIdx.x < 2 * kBlock)
                scales[threadIdx.x] = sscale;
        }
    };
    // the block has landed in LDS for every wave
    auto arrive = [&](int b, uint8_t* buf) {
        if constexpr (!kBytes) {
            wait_loads();
            if (b < b_end && unclear(b)) {
                u32x4_t* const v =               // the words that this lane loaded
                    reinterpret_cast<u32x4_t*>(buf + S::kKeyBytes + wave * kStage * 1024) + lane;
                u32x4_t x[kStage];
#pragma unroll
                for (int y = 0; y < kStage; ++y) x[y] = v[64 * y];
                if (make_finite<kFmt>(x)) {
#pragma unroll
                    for (int y = 0; y < kStage; ++y) v[64 * y] = x[y];
                }
            }
        }
        __syncthreads();
    };

    float top = -inf(), sum = 0.0f;
    f32x16_t o[kDims];
#pragma unroll
    for (int d = 0; d < kDims; ++d)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[d][x] = 0.0f;

    float* const scales0 = reinterpret_cast<float*>(lds + 2 * S::kBuffer);
    // the key that row m of a tile of S^T stands for: bits 2 and 3 exchanged
    const int krow = (n & 0x13) | ((n & 4) << 1) | ((n & 8) >> 1);

    uint32_t page = page_of(b_begin + 1);
    if (b_begin < b_end) {
        fetch(b_begin, page_of(b_begin), lds);
        stage(b_begin, lds, scales0);
        arrive(b_begin, lds);
    }
    for (int b = b_begin; b < b_end; ++b) {
        const int cur = (b - b_begin) & 1;
        uint8_t* const buf = lds + cur * S::kBuffer;
        float* const scales = scales0 + cur * 128;
        const bool more = b + 1 < b_end;
        const int key0 = b * kBlock;
        bad = bad_next;
        if (more) fetch(b + 1, page, lds + (cur ^ 1) * S::kBuffer);
        page = page_of(b + 2);
        if (key0 < hi_any && key0 + kBlock > lo_any) {
            f32x16_t s[2];
#pragma unroll
            for (int c = 0; c < kSteps; ++c)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8_t k = *reinterpret_cast<const bf16x8_t*>(
                        buf + key_word<D>(32 * t + krow, 2 * c + g));
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[c], c == 0 ? f32x16_t{} : s[t],
                                                                   0, 0, 0);
                }
            // four words of keys ahead of the products that take them
            constexpr int kDsRead = 0x100, kMatrix = 0x8;
            __builtin_amdgcn_sched_group_barrier(kDsRead, 4, 0);
#pragma unroll
            for (int c = 0; c < 2 * kSteps - 4; ++c) {
                __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(kMatrix, 4, 0);
            // register x of tile t: key 32 t + 16 (x / 8) + 8 g + x % 8
            float x[32];
#pragma unroll
            for (int y = 0; y < 32; ++y) x[y] = s[y >> 4][y & 15];
            if constexpr (kBytes) {
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    const f32x4_t k4 = *reinterpret_cast<const f32x4_t*>(
                        scales + 32 * (y >> 2) + 16 * ((y >> 1) & 1) + 8 * g + 4 * (y & 1));
#pragma unroll
                    for (int z = 0; z < 4; ++z) x[4 * y + z] *= k4[z];
                }
            }
            const float away = static_cast<float>(pos - (key0 + 8 * g));
            auto place = [](int y) { return 32 * (y >> 4) + 16 * ((y >> 3) & 1) + (y & 7); };
            map_scores<kMode, kBytes>(map, x, away, place, key0 + kBlock - 1 <= pos_first);
            if (bad) {
#pragma unroll
                for (int y = 0; y < 32; ++y) x[y] = nan();
            }
            if (key0 < lo_all || key0 + kBlock > hi_all) {
                // against the key's constant part: no register holds a key's number
                const int from = first - (key0 + 8 * g), to = limit - (key0 + 8 * g);
#pragma unroll
                for (int y = 0; y < 32; ++y) {
                    if (place(y) < from || place(y) >= to) x[y] = unseen<kMode>();
                }
            }
            float peak = x[0];
#pragma unroll
            for (int y = 1; y < 32; ++y) peak = larger<kMode>(peak, x[y]);
            peak = max_halves(__builtin_fmaf(peak, map.unit, map.offset));
            const float now = __builtin_fmaxf(top, peak);
            if (__any(now > top + kSlack)) {
                const float shrink = __builtin_amdgcn_exp2f(top - (now == -inf() ? 0.0f : now));
                sum *= shrink;
#pragma unroll
                for (int d = 0; d < kDims; ++d) o[d] *= shrink;
                top = now;
            }
            // nothing seen so far: any finite stand-in gives weights of zero
            const float base = map.offset - (top == -inf() ? 0.0f : top);
            bf16x8_t p[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                u32x4_t w;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float e[4];
                    f32x4_t v4;
                    if constexpr (kBytes)
                        v4 = *reinterpret_cast<const f32x4_t*>(scales + 64 + 16 * u + 8 * g + 4 * j);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        e[y] = __builtin_amdgcn_exp2f(
                            __builtin_fmaf(x[8 * u + 4 * j + y], map.unit, base));
                        sum += e[y];
                        if constexpr (kBytes) e[y] *= v4[y];
                    }
                    w[2 * j] = pack_bf16(e[0], e[1]);
                    w[2 * j + 1] = pack_bf16(e[2], e[3]);
                }
                p[u] = __builtin_bit_cast(bf16x8_t, w);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int d = 0; d < kDims; ++d) {
                    const bf16x8_t v = *reinterpret_cast<const bf16x8_t*>(
                        buf + S::kKeyBytes + val_word(32 * d + n, 2 * u + g));
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[u], o[d], 0, 0, 0);
                }
        }
        if (more) stage(b + 1, lds + (cur ^ 1) * S::kBuffer, scales0 + (cur ^ 1) * 128);
        arrive(b + 1, lds + (cur ^ 1) * S::kBuffer);
    }

    sum += __shfl_xor(sum, 32);
    if (r >= n_rows) return;
    if (parts && at.chunks > 1) {
        const uint64_t slot =
            ((uint64_t(at.slot) + at.chunk) * a.c.heads + h) * S::kRows + 32 * wave + n;
#pragma unroll
        for (int d = 0; d < kDims; ++d)
#pragma unroll
            for (int y = 0; y < 4; ++y)
                store<f32x4_t>(a.part_o + slot * D + 32 * d + 8 * y + 4 * g,
                               f32x4_t{o[d][4 * y], o[d][4 * y + 1], o[d][4 * y + 2],
                                       o[d][4 * y + 3]});
        if (g == 0) {
            a.part_ml[2 * slot] = top;
            a.part_ml[2 * slot + 1] = sum;
        }
        return;
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    uint16_t* out = a.out + uint64_t(at.seq.start + i) * a.out_stride + uint64_t(head) * D;
#pragma unroll
    for (int d = 0; d < kDims; ++d)
#pragma unroll
        for (int y = 0; y < 4; ++y)
            store_row4(out + 32 * d + 8 * y + 4 * g,
                       u32x2_t{pack_bf16(o[d][4 * y] * inv, o[d][4 * y + 1] * inv),
                               pack_bf16(o[d][4 * y + 2] * inv, o[d][4 * y + 3] * inv)});
}

}  // namespace eskv
