// Appending to the cache and reading it back.
//
// Both move every byte once and compute little: they are bound by memory, and at
// few tokens by latency.  D / 8 lanes hold a row, 8 elements (one 16-byte access)
// each, so a norm is a sum over neighbouring lanes and a rotation's other half an
// exchange with the lane rot / 16 away (the halves' pairing) or nothing (the
// adjacent pairing).
//
// Queries: a workgroup takes one token for each D / 8 of its lanes and up to 8
// heads, so that a token's row of the rotation table is read once for 8
// rows, and 8 rows are on their way at a time.
// Keys and values: a workgroup takes 64 tokens of one head, all of its rows on
// their way at once.  Values are stored by dimension: the tokens are turned in
// LDS and written as runs of tokens, cut where the slots' 16-byte words are: the
// LDS columns are shifted by the first slot's place in its word, so that a word
// whose tokens lie in consecutive slots (a prompt, wherever its page list jumps)
// is read from LDS and written to memory in one access.  The tokens of the other
// words (at the ends of runs, of several sequences, of a generation step) go one
// by one, a lane each, dimension after dimension: neighbours' elements are then
// written by one instruction, into as few lines as there are runs.
//
// Measured: 8362 tokens of 32 ragged prompts (40 query heads over 8 of 128, E4M3)
// appended in 47 us, 4.7 TB/s, and read back in 14; 32771 tokens (16 heads over
// 16 of 64, bf16) in 92 us, 4.4 TB/s, and 58 to 60.  One token: 6.9 to 7.8 and 3.3 to 3.6 us.
#pragma once

#include "kv_common.hpp"

namespace eskv {

constexpr int kPlaceThreads = 256;
constexpr int kPlaceTokens = 64;            // tokens of a workgroup of keys and values
constexpr int kPlaceHeads = 8;              // heads of a workgroup of queries

struct AppendArgs {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    uint16_t* q_out;
    uint64_t q_stride, k_stride, v_stride, q_out_stride;
    const uint16_t* q_gain;
    const uint16_t* k_gain;
    const float* rope;
    const int32_t* positions;
    const int64_t* slots;
    uint32_t* status;
    uint32_t tokens, q_heads, rot, rope_rows;
    float eps;
    uint32_t adjacent;
    uint32_t kv_blocks, q_blocks, q_parts;  // blocks of tokens, for keys and for queries; its parts
    Cache c;
};

struct ReadArgs {
    const int64_t* slots;
    uint16_t* k_out;
    uint16_t* v_out;
    uint64_t k_stride, v_stride;
    uint32_t* status;
    uint32_t tokens, blocks;
    Cache c;
};

// Workgroup `id` of `blocks` blocks of tokens with `parts` parts each: a block's
// parts on one of the eight dies (workgroups go round them), near in time, so that
// a die's L2 holds the block's rows of the rotation table for all of them.  The
// host rounds `blocks` up to a multiple of 8 where there are as many.
__device__ __forceinline__ void block_part(uint32_t id, uint32_t blocks, uint32_t parts,
                                           uint32_t& block, uint32_t& part) {
    const uint32_t dies = blocks >= 8 ? 8 : 1;
    const uint32_t rest = id / dies;
    part = rest % parts;
    block = rest / parts * dies + id % dies;
}

// A register of another lane of the same 16: by data-parallel moves, which cost
// an instruction and no trip through LDS.
template <int kControl>
__device__ __forceinline__ uint32_t moved(uint32_t x) {
    return static_cast<uint32_t>(
        __builtin_amdgcn_update_dpp(0, static_cast<int>(x), kControl, 0xF, 0xF, true));
}
constexpr int kQuadSwap1 = 0xB1, kQuadSwap2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
constexpr int kRor4 = 0x124, kRor8 = 0x128, kRor12 = 0x12C;

// The value of the lane 16 away (of each 32).
__device__ __forceinline__ uint32_t other_row(uint32_t x) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return (threadIdx.x & 16) != 0 ? r[0] : r[1];
}

// `op` over the kLanes lanes of a row, the same in all of them: over pairs, pairs
// of pairs, the mirrored half and the mirrored 16.
template <int kLanes, class Op>
__device__ __forceinline__ uint32_t row_all(uint32_t x, Op op) {
    x = op(x, moved<kQuadSwap1>(x));
    x = op(x, moved<kQuadSwap2>(x));
    x = op(x, moved<kHalfMirror>(x));
    if constexpr (kLanes >= 16) x = op(x, moved<kMirror>(x));
    if constexpr (kLanes >= 32) x = op(x, other_row(x));
    return x;
}
template <int kLanes>
__device__ __forceinline__ float row_sum(float x) {
    return __uint_as_float(row_all<kLanes>(__float_as_uint(x), [](uint32_t p, uint32_t q) {
        return __float_as_uint(__uint_as_float(p) + __uint_as_float(q));
    }));
}
template <int kLanes>
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
    return row_all<kLanes>(x, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
}

// The value of the lane `away` lanes on: the other half's.  kWhole: the halves are
// those of the whole row (rot is D).
template <int kLanes, bool kWhole>
__device__ __forceinline__ float exchanged(float x, int away) {
    const uint32_t u = __float_as_uint(x);
    if constexpr (!kWhole) {
        return __shfl(x, (static_cast<int>(threadIdx.x) & 63) + away);
    } else if constexpr (kLanes == 32) {
        return __uint_as_float(other_row(u));
    } else if constexpr (kLanes == 16) {
        return __uint_as_float(moved<kRor8>(u));
    } else {
        const uint32_t up = moved<kRor12>(u), down = moved<kRor4>(u);
        return __uint_as_float(away > 0 ? up : down);
    }
}

// The largest |x| of 8 elements as bits, which order as magnitudes do with
// infinities and then NaNs above every number.
__device__ __forceinline__ uint32_t max_bits(const float x[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        m = m > b ? m : b;
    }
    return m;
}

// What a row is multiplied by: the gain of this lane's 8 elements, and the
// cosines and sines of its rotation.
struct Turn {
    float c[8], s[8];                       // of its elements, or (adjacent) of its 4 pairs
    int away;                               // lanes to the other half; 0: none
};
constexpr int kUnturned = 1;                // away of an adjacent lane beyond rot

// This lane's part of a row of the rotation table.  The first half takes
// a c - b s and the second b c + a s: the sines carry the sign.
template <int kLanes>
__device__ __forceinline__ Turn load_turn(const float* turn, int lr, uint32_t rot, bool adjacent) {
    Turn t;
    t.away = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        t.c[i] = 1.0f;
        t.s[i] = 0.0f;
    }
    if (8u * lr >= rot) {
        t.away = adjacent ? kUnturned : 0;
        return t;
    }
    const int half = static_cast<int>(rot) / 16;             // lanes of one half
    if (adjacent) {
        const f32x4_t c = load_float4(turn + 4 * lr), s = load_float4(turn + rot / 2 + 4 * lr);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            t.c[i] = c[i];
            t.s[i] = s[i];
        }
    } else {
        t.away = lr < half ? half : -half;
        const float* p = turn + 8 * (lr < half ? lr : lr - half);
        const f32x4_t c0 = load_float4(p), c1 = load_float4(p + 4);
        const f32x4_t s0 = load_float4(p + rot / 2), s1 = load_float4(p + rot / 2 + 4);
        const float sign = lr < half ? -1.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t.c[i] = i < 4 ? c0[i & 3] : c1[i & 3];
            t.s[i] = sign * (i < 4 ? s0[i & 3] : s1[i & 3]);
        }
    }
    return t;
}

// Normalise and rotate the row of which this lane (lane `lr` of the row's
// kLanes) holds x[0..7].
template <int kLanes, bool kWhole>
__device__ __forceinline__ void norm_rotate(float x[8], bool norm, const float gain[8], float eps,
                                            uint32_t rot, bool adjacent, const Turn& t) {
    constexpr float kInvD = 1.0f / (8 * kLanes);
    if (norm) {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
        ss = row_sum<kLanes>(ss);
        if (!(ss < 0x1p120f)) {
            // elements beyond about 2^58: squares are summed in units of 2^160,
            // beside which eps is nothing (eps is at most the largest binary32)
            ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] *= 0x1p-80f;
                ss = __builtin_fmaf(x[i], x[i], ss);
            }
            ss = row_sum<kLanes>(ss);
            eps *= 0x1p-80f * 0x1p-80f;
        }
        const float r = 1.0f / __builtin_sqrtf(__builtin_fmaf(ss, kInvD, eps));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * r * gain[i];
    }
    if (!kWhole && rot == 0) return;
    if (!kWhole && adjacent) {
        // (dimensions beyond rot: cosine 1 and sine 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = t.away == kUnturned ? a : a * t.c[i] - b * t.s[i];
            x[2 * i + 1] = t.away == kUnturned ? b : b * t.c[i] + a * t.s[i];
        }
        return;
    }
    float other[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) other[i] = exchanged<kLanes, kWhole>(x[i], t.away);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = !kWhole && t.away == 0 ? x[i] : x[i] * t.c[i] + other[i] * t.s[i];
}

// LDS of the turned values: a row per dimension of 64 tokens and up to a word's
// shift.  A token's elements of one lane lie 8 rows from the next lane's, which
// is the same bank or its opposite: the words of a row are moved round by the
// number of its 8 rows, so that 16 lanes meet in a bank by twos.
template <int kFmt>
struct Turned {
    static constexpr int kWord = 16 / kCodeBytes<kFmt>;      // tokens of a 16-byte word
    static constexpr int kWords = kPlaceTokens / kWord + 1;
    static constexpr int kRowBytes = 16 * kWords;
    // where word w of dimension d lies
    static __device__ __forceinline__ int at(int d, int w) {
        const int r = w + (d >> 3) % kWords;
        return d * kRowBytes + 16 * (r < kWords ? r : r - kWords);
    }
    // where column c (a token and the shift) of dimension d lies
    static __device__ __forceinline__ int token(int d, int c) {
        return at(d, c / kWord) + c % kWord * kCodeBytes<kFmt>;
    }
    // of dimension 8 lr; the next seven follow kRowBytes apart
    static __device__ __forceinline__ int column(int lr, int c) { return token(8 * lr, c); }
};

// Where token 0 of the workgroup sits in its 16-byte word of slots (the columns'
// shift), and for every word whether its tokens lie in consecutive slots of one
// word: all of them here (kAll: the word is written whole), or those that are (it
// may be read whole; the others of its slots are not used).  The word's first
// slot then, or -1.
template <int kFmt, bool kAll>
__device__ __forceinline__ void find_words(const int64_t* slot, int n, uint64_t pool, int& shift,
                                           int64_t* whole) {
    using T = Turned<kFmt>;
    // the first token that has a slot sets the phase
    const int lane = threadIdx.x & 63;
    const int64_t s = lane < n ? slot[lane] : -1;
    const uint64_t has = __ballot(s >= 0 && uint64_t(s) < pool);
    const int lead = has ? __builtin_ctzll(has) : 0;
    const int at = static_cast<int>(__shfl(static_cast<int>(s & (T::kWord - 1)), lead));
    shift = has ? (at - lead) & (T::kWord - 1) : 0;
    if (threadIdx.x < T::kWords) {
        const int j0 = T::kWord * static_cast<int>(threadIdx.x) - shift;
        const int a = max(j0, 0), b = min(j0 + T::kWord, n);
        const int64_t s0 = a < b ? slot[a] - (a - j0) : -1;
        bool ok = (!kAll || b - a == T::kWord) && s0 >= 0 && uint64_t(s0) + T::kWord <= pool &&
                  (s0 & (T::kWord - 1)) == 0;
        for (int i = a + 1; i < b; ++i) ok = ok && slot[i] == s0 + (i - j0);
        whole[threadIdx.x] = ok ? s0 : -1;
    }
}

__device__ __forceinline__ int log2_up(int x) {              // of 1 .. 2^30
    return x <= 1 ? 0 : 32 - __builtin_clz(static_cast<uint32_t>(x - 1));
}

// Where slot s keeps dimension d of head h's value.
template <int D, int kFmt>
__device__ __forceinline__ uint8_t* value_at(const Cache& c, int64_t s, uint32_t h, int d) {
    const uint64_t page = uint64_t(s) >> c.page_shift;
    const uint32_t off = uint32_t(s) & (c.page - 1);
    return c.v + (((page * c.heads + h) * D + d) * c.page + off) * kCodeBytes<kFmt>;
}

__device__ __forceinline__ void load_gain(const uint16_t* g, int lr, float gain[8]) {
    if (g == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) gain[i] = 1.0f;
    } else {
        unpack8(load_row8(g + 8 * lr), gain);
    }
}

// Queries of one token for each kLanes lanes and up to kPlaceHeads heads.  The
// loop is not unrolled, here and over the passes of keys: a call at few tokens waits
// for its instructions as much as for its data, and one that fills the card has
// other waves' rows on their way.
template <int D, bool kWhole>
__device__ __forceinline__ void append_queries(const AppendArgs& a, uint32_t block) {
    constexpr int kLanes = D / 8;                            // lanes of a row
    constexpr int kTokens = kPlaceThreads / kLanes;
    const int lr = threadIdx.x % kLanes;
    uint32_t tb, part;
    block_part(block, a.q_blocks, a.q_parts, tb, part);
    if (tb * kTokens >= a.tokens) return;
    const uint32_t token = tb * kTokens + threadIdx.x / kLanes;
    const uint32_t t = min(token, a.tokens - 1);             // lanes exchange: none leaves
    const uint32_t h0 = part * kPlaceHeads;
    const int heads = static_cast<int>(min(uint32_t(kPlaceHeads), a.q_heads - h0));
    const uint16_t* src = a.q + t * a.q_stride + h0 * D + 8 * lr;
    uint16_t* dst = a.q_out + t * a.q_out_stride + h0 * D + 8 * lr;
    u32x4_t raw = load_row8(src), next = load_row8(src + min(1, heads - 1) * D);
    const int32_t pos = a.rot != 0 ? a.positions[t] : 0;
    const bool ok = a.rot == 0 || (pos >= 0 && uint32_t(pos) < a.rope_rows);
    float gain[8];
    load_gain(a.q_gain, lr, gain);
    const Turn turn =
        load_turn<kLanes>(a.rope + uint64_t(ok ? pos : 0) * a.rot, lr, a.rot, a.adjacent);
    if (!ok && lr == 0 && a.status != nullptr) atomicOr(a.status, ES_KV_BAD_POSITION);
#pragma unroll 1
    for (int h = 0; h < heads; ++h) {
        const u32x4_t after = load_row8(src + min(h + 2, heads - 1) * D);
        float x[8];
        unpack8(raw, x);
        norm_rotate<kLanes, kWhole>(x, a.q_gain != nullptr, gain, a.eps, a.rot, a.adjacent, turn);
        u32x4_t out;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            out[i] = ok ? pack_bf16(x[2 * i], x[2 * i + 1]) : 0x7FC07FC0u;
        if (token < a.tokens) store_row8(dst + h * D, out);
        raw = next;
        next = after;
    }
}

template <int D, int kFmt, bool kWhole>
__global__ __launch_bounds__(kPlaceThreads) void es_kv_append_kernel(AppendArgs a) {
    // keys and values first: their workgroups take longest
    const uint32_t kv_groups = a.kv_blocks * a.c.heads;
    if (blockIdx.x >= kv_groups) {
        append_queries<D, kWhole>(a, blockIdx.x - kv_groups);
        return;
    }
    using T = Turned<kFmt>;
    constexpr int kLanes = D / 8;
    constexpr int kRows = kPlaceThreads / kLanes;            // rows of a pass
    const int lr = threadIdx.x % kLanes, row = threadIdx.x / kLanes;
    uint32_t tb, h;
    block_part(blockIdx.x, a.kv_blocks, a.c.heads, tb, h);
    const uint32_t t0 = tb * kPlaceTokens;
    if (t0 >= a.tokens) return;
    const int n = static_cast<int>(min(uint32_t(kPlaceTokens), a.tokens - t0));

    __shared__ __attribute__((aligned(16))) uint8_t turned[D * T::kRowBytes];
    __shared__ int64_t slot[kPlaceTokens];
    __shared__ int64_t whole[T::kWords];
    const uint64_t pool = uint64_t(a.c.n_pages) << a.c.page_shift;

    // a pass's rows are asked for a pass ahead (rows past the last repeat it and are
    // not stored: lanes exchange, none leaves)
    struct Ahead {
        u32x4_t k, v;
        int32_t pos;
    };
    auto ask = [&](int p) {
        const uint32_t t = t0 + min(kRows * p + row, n - 1);
        return Ahead{load_row8(a.k + t * a.k_stride + h * D + 8 * lr),
                     load_row8(a.v + t * a.v_stride + h * D + 8 * lr),
                     a.rot != 0 ? a.positions[t] : 0};
    };
    Ahead next = ask(0);
    if (threadIdx.x < kPlaceTokens)
        slot[threadIdx.x] = static_cast<int>(threadIdx.x) < n ? a.slots[t0 + threadIdx.x] : -1;
    float gain[8];
    load_gain(a.k_gain, lr, gain);
    __syncthreads();
    int shift;
    find_words<kFmt, true>(slot, n, pool, shift, whole);

#pragma unroll 1
    for (int p = 0; kRows * p < n; ++p) {
        const int j = kRows * p + row;
        const Ahead now = next;
        const bool ok = a.rot == 0 || (now.pos >= 0 && uint32_t(now.pos) < a.rope_rows);
        const Turn turn =
            load_turn<kLanes>(a.rope + uint64_t(ok ? now.pos : 0) * a.rot, lr, a.rot, a.adjacent);
        next = ask(p + 1);
        float x[8], y[8];
        unpack8(now.k, x);
        unpack8(now.v, y);
        norm_rotate<kLanes, kWhole>(x, a.k_gain != nullptr, gain, a.eps, a.rot, a.adjacent, turn);
        const uint32_t mx = row_max<kLanes>(max_bits(x)), my = row_max<kLanes>(max_bits(y));
        const bool dead = !ok || mx >= 0x7F800000u || my >= 0x7F800000u;
        const int64_t s = slot[min(j, n - 1)];
        const bool in = s >= 0 && uint64_t(s) < pool;
        const bool put = j < n && in;
        if (a.status != nullptr && lr == 0 && h == 0 && j < n) {
            if (!ok) atomicOr(a.status, ES_KV_BAD_POSITION);
            if (s >= 0 && !in) atomicOr(a.status, ES_KV_BAD_SLOT);
        }
        const uint64_t page = uint64_t(in ? s : 0) >> a.c.page_shift;
        const uint32_t off = uint32_t(in ? s : 0) & (a.c.page - 1);
        const uint64_t at = (page * a.c.heads + h) * a.c.page + off;
        uint8_t* column = turned + T::column(lr, j + shift);
        if constexpr (kFmt == kBf16) {
            u32x4_t out;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                out[i] = dead ? 0x7FC07FC0u : pack_bf16(x[2 * i], x[2 * i + 1]);
                const uint32_t w = dead ? 0u : now.v[i];
                if (j < n) {
                    *reinterpret_cast<uint16_t*>(column + 2 * i * T::kRowBytes) =
                        static_cast<uint16_t>(w);
                    *reinterpret_cast<uint16_t*>(column + (2 * i + 1) * T::kRowBytes) =
                        static_cast<uint16_t>(w >> 16);
                }
            }
            if (put) store<u32x4_t>(a.c.k + (at * D + 8 * lr) * 2, out);
        } else {
            // rows that are not finite, or so small that Q / M could overflow, are zeros
            const float fx = __uint_as_float(mx), fy = __uint_as_float(my);
            const bool lx = !dead && fx >= kTinyRow, ly = !dead && fy >= kTinyRow;
            u32x2_t cx = {0u, 0u}, cy = {0u, 0u};
            if (lx) cx = encode8<kFmt>(x, kCodeMax<kFmt> * (1.0f / fx));
            if (ly) cy = encode8<kFmt>(y, kCodeMax<kFmt> * (1.0f / fy));
            if (j < n) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    column[i * T::kRowBytes] = static_cast<uint8_t>(cy[i / 4] >> (8 * (i & 3)));
            }
            if (put) {
                store<u32x2_t>(a.c.k + at * D + 8 * lr, cx);
                if (lr == 0) {
                    store<float>(a.c.ks + at, dead ? nan() : lx ? fx / kCodeMax<kFmt> : 0.0f);
                    store<float>(a.c.vs + at, ly ? fy / kCodeMax<kFmt> : 0.0f);
                }
            }
        }
    }
    __syncthreads();

    // the values' rows of tokens, by words; neighbouring lanes take a row's words
    const int words = (n + shift + T::kWord - 1) / T::kWord;
    const int lanes = log2_up(words);
    for (int i = threadIdx.x; i < D << lanes; i += kPlaceThreads) {
        const int d = i >> lanes, w = i & ((1 << lanes) - 1);
        if (w >= words) continue;
        if (whole[w] >= 0)
            store<u32x4_t>(value_at<D, kFmt>(a.c, whole[w], h, d),
                           *reinterpret_cast<const u32x4_t*>(turned + T::at(d, w)));
    }
    const int j = threadIdx.x & 63;
    const int64_t s = j < n && whole[(j + shift) / T::kWord] < 0 ? slot[j] : -1;
    if (s >= 0 && uint64_t(s) < pool) {
        uint8_t* const dst = value_at<D, kFmt>(a.c, s, h, 0);
        const uint32_t step = a.c.page * kCodeBytes<kFmt>;
#pragma unroll 4
        for (int d = threadIdx.x >> 6; d < D; d += kPlaceThreads / 64) {
            const uint8_t* src = turned + T::token(d, j + shift);
            if constexpr (kFmt == kBf16)
                store<uint16_t>(dst + d * step, *reinterpret_cast<const uint16_t*>(src));
            else
                store<uint8_t>(dst + d * step, *src);
        }
    }
}

template <int D, int kFmt>
__global__ __launch_bounds__(kPlaceThreads) void es_kv_read_kernel(ReadArgs a) {
    using T = Turned<kFmt>;
    constexpr int kLanes = D / 8;
    constexpr int kRows = kPlaceThreads / kLanes;
    constexpr int kPasses = kPlaceTokens / kRows;
    typedef uint32_t Codes __attribute__((ext_vector_type(2 * kCodeBytes<kFmt>)));
    const int lr = threadIdx.x % kLanes, row = threadIdx.x / kLanes;
    uint32_t tb, h;
    block_part(blockIdx.x, a.blocks, a.c.heads, tb, h);
    const uint32_t t0 = tb * kPlaceTokens;
    if (t0 >= a.tokens) return;
    const int n = static_cast<int>(min(uint32_t(kPlaceTokens), a.tokens - t0));
    const uint64_t pool = uint64_t(a.c.n_pages) << a.c.page_shift;

    __shared__ __attribute__((aligned(16))) uint8_t turned[D * T::kRowBytes];
    __shared__ int64_t slot[kPlaceTokens];
    __shared__ int64_t whole[T::kWords];
    if (threadIdx.x < kPlaceTokens)
        slot[threadIdx.x] = static_cast<int>(threadIdx.x) < n ? a.slots[t0 + threadIdx.x] : -1;
    __syncthreads();
    int shift;
    find_words<kFmt, false>(slot, n, pool, shift, whole);
    __syncthreads();

    // this lane's keys and their scales, on their way while the values are turned
    Codes ck[kPasses];
    float sk[kPasses], sv[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int j = kRows * p + row;
        const int64_t s = j < n ? slot[j] : -1;
        const bool in = s >= 0 && uint64_t(s) < pool;
        const uint64_t page = uint64_t(in ? s : 0) >> a.c.page_shift;
        const uint32_t off = uint32_t(in ? s : 0) & (a.c.page - 1);
        const uint64_t at = (page * a.c.heads + h) * a.c.page + off;
        sk[p] = sv[p] = 0.0f;
        if (in) {
            ck[p] = load<Codes>(a.c.k + (at * D + 8 * lr) * kCodeBytes<kFmt>);
            if constexpr (kFmt == kBf16) {
                sk[p] = bf16_lo(load<uint16_t>(a.c.k + at * D * 2));     // NaN: a void token
            } else {
                sk[p] = load<float>(a.c.ks + at);
                sv[p] = load<float>(a.c.vs + at);
            }
        }
    }
    const int words = (n + shift + T::kWord - 1) / T::kWord;
    const int lanes = log2_up(words);
    // kAsk words of a lane at a time, all on their way before the first is used
    constexpr int kAsk = 2;
#pragma unroll 1
    for (int i0 = threadIdx.x; i0 < D << lanes; i0 += kAsk * kPlaceThreads) {
        u32x4_t tokens[kAsk];
        bool run[kAsk];
#pragma unroll
        for (int k = 0; k < kAsk; ++k) {
            const int i = i0 + k * kPlaceThreads, d = i >> lanes, w = i & ((1 << lanes) - 1);
            tokens[k] = u32x4_t{0u, 0u, 0u, 0u};
            run[k] = d < D && w < words && whole[w] >= 0;
            if (run[k]) tokens[k] = load<u32x4_t>(value_at<D, kFmt>(a.c, whole[w], h, d));
        }
#pragma unroll
        for (int k = 0; k < kAsk; ++k) {
            const int i = i0 + k * kPlaceThreads, d = i >> lanes, w = i & ((1 << lanes) - 1);
            if (run[k]) *reinterpret_cast<u32x4_t*>(turned + T::at(d, w)) = tokens[k];
        }
    }
    {
        const int j = threadIdx.x & 63;
        const int64_t s = j < n && whole[(j + shift) / T::kWord] < 0 ? slot[j] : -1;
        if (s >= 0 && uint64_t(s) < pool) {
            const uint8_t* const src = value_at<D, kFmt>(a.c, s, h, 0);
            const uint32_t step = a.c.page * kCodeBytes<kFmt>;
#pragma unroll 8
            for (int d = threadIdx.x >> 6; d < D; d += kPlaceThreads / 64) {
                uint8_t* dst = turned + T::token(d, j + shift);
                if constexpr (kFmt == kBf16)
                    *reinterpret_cast<uint16_t*>(dst) = load<uint16_t>(src + d * step);
                else
                    *dst = load<uint8_t>(src + d * step);
            }
        }
    }
    __syncthreads();

#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int j = kRows * p + row;
        if (j >= n) break;
        const uint32_t t = t0 + j;
        const int64_t s = slot[j];
        const bool in = s >= 0 && uint64_t(s) < pool;
        u32x4_t ko = {0u, 0u, 0u, 0u}, vo = {0u, 0u, 0u, 0u};
        const u32x4_t not_a_number = {0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        if (in) {
            const bool dead = sk[p] != sk[p];
            const uint8_t* column = turned + T::column(lr, j + shift);
            if constexpr (kFmt == kBf16) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t lo =
                        *reinterpret_cast<const uint16_t*>(column + 2 * i * T::kRowBytes);
                    const uint32_t hi =
                        *reinterpret_cast<const uint16_t*>(column + (2 * i + 1) * T::kRowBytes);
                    ko[i] = ck[p][i];
                    vo[i] = lo | (hi << 16);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t cv = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        cv |= uint32_t(column[(4 * i + e) * T::kRowBytes]) << (8 * e);
                    float xk[4], xv[4];
                    decode4<kFmt>(ck[p][i], xk);
                    decode4<kFmt>(cv, xv);
                    ko[2 * i] = pack_bf16(xk[0] * sk[p], xk[1] * sk[p]);
                    ko[2 * i + 1] = pack_bf16(xk[2] * sk[p], xk[3] * sk[p]);
                    vo[2 * i] = pack_bf16(xv[0] * sv[p], xv[1] * sv[p]);
                    vo[2 * i + 1] = pack_bf16(xv[2] * sv[p], xv[3] * sv[p]);
                }
            }
            if (dead) vo = not_a_number;
        } else if (s >= 0) {
            ko = vo = not_a_number;
            if (lr == 0 && h == 0 && a.status != nullptr) atomicOr(a.status, ES_KV_BAD_SLOT);
        }
        store_row8(a.k_out + t * a.k_stride + h * D + 8 * lr, ko);
        store_row8(a.v_out + t * a.v_stride + h * D + 8 * lr, vo);
    }
}

}  // namespace eskv
