// Scores of targets over a large vocabulary and the divergence from a teacher's
// top logits, with their gradients, without keeping the logits.
//
// With z = scale x . w_v and lse = log sum_v exp z_v, a row's scores are z_id - lse;
// its gradient is f (Q softmax(z) - q), q the wanted weights at its ids, Q their
// sum (1; a row whose teacher leaves nothing has no gradient).  The logits of a tile live in
// registers: the scores keep a maximum and a sum of each row and tile, and the
// gradients f Q softmax(z) as bf16, for a piece of the vocabulary at a time.
#pragma once

#include "few.hpp"
#include "mm_tile.hpp"
#include "ring.hpp"
#include "stream.hpp"

namespace eshead {

using namespace esmm;

constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kMaxEntries = 256;

// What becomes of a row, by its ids, and (added to it) that its teacher's weights are NaN.
enum Row : uint8_t { kDead = 0, kLive = 1, kVoid = 2, kKind = 3, kLost = 4 };

// ------------------------------------------------------------------- rows --

struct RowArgs {
    const int64_t* ids;
    const float* teacher;                  // or null
    uint8_t* flags;                        // [rows]
    float *loss, *logp, *lse;              // of dead rows zeros, of void ones NaN; or null
    uint16_t* dx;                          //   likewise
    uint64_t dx_stride;
    uint32_t* status;
    uint32_t rows, vocab, entries, hidden;
    bool weighed;                          // a row whose teacher leaves nothing is dead
    float scale;                           //   at this one
};

// Whether a teacher's logit leaves its entry a weight: what is -infinity at a scale of that
// sign, and -infinity itself, leaves none.  Without a number for it (NaN, or an infinity that
// takes all of the weight) a row's weights are NaN.
__device__ __forceinline__ bool has_weight(float t, float scale) {
    return t != -eskv::inf() && (t != eskv::inf() || !(scale < 0.0f));
}
__device__ __forceinline__ bool is_number(float t, float scale) {
    return __builtin_fabsf(t) < eskv::inf() || !has_weight(t, scale);
}

// What becomes of a row of several ids: one wave a row.
__global__ __launch_bounds__(256) void es_head_rows_kernel(RowArgs a) {
    const uint32_t lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= a.rows) return;
    bool some = false, bad = false, weight = !a.weighed, lost = false;
    for (uint32_t e = lane; e < a.entries; e += 64) {
        const int64_t id = a.ids[uint64_t(r) * a.entries + e];
        some |= id >= 0;
        bad |= id >= int64_t(a.vocab);
        if (id >= 0 && a.weighed) {
            const float t = a.teacher[uint64_t(r) * a.entries + e];
            weight |= has_weight(t, a.scale);
            lost |= !is_number(t, a.scale);
        }
    }
    some = __any(some);
    bad = __any(bad);
    weight = __any(weight);
    lost = __any(lost);
    if (lane == 0) a.flags[r] = (bad ? kVoid : some && weight ? kLive : kDead) | (lost ? kLost : 0);
}

// The same, where a row has one id; of several, what es_head_rows_kernel found.
__device__ __forceinline__ uint8_t kind_of(const RowArgs& a, uint32_t r) {
    if (a.entries > 1) return a.flags[r] & kKind;
    const int64_t id = a.ids[r];
    if (id >= int64_t(a.vocab)) return kVoid;
    return id < 0 || (a.weighed && !has_weight(a.teacher[r], a.scale)) ? kDead : kLive;
}
__device__ __forceinline__ bool is_lost(const RowArgs& a, uint32_t r) {
    if (a.entries > 1) return a.flags[r] & kLost;
    return a.weighed && !is_number(a.teacher[r], a.scale);
}

// Its results, where it has none of its own.  A wave's lanes.
__device__ __forceinline__ void clear_row(const RowArgs& a, uint32_t r, uint32_t lane) {
    const uint8_t kind = kind_of(a, r);
    if (kind == kLive) return;
    const bool bad = kind == kVoid;
    if (bad && lane == 0 && a.status != nullptr) atomicOr(a.status, ES_HEAD_BAD_ID);
    const float v = bad ? eskv::nan() : 0.0f;
    if (lane == 0) {
        if (a.loss != nullptr) a.loss[r] = v;
        if (a.lse != nullptr) a.lse[r] = v;
    }
    if (a.logp != nullptr)
        for (uint32_t e = lane; e < a.entries; e += 64) a.logp[uint64_t(r) * a.entries + e] = v;
    if (a.dx != nullptr)
        for (uint32_t h = lane; h < a.hidden; h += 64) a.dx[r * a.dx_stride + h] = bad ? 0x7FC0u : 0u;
}

struct ListArgs {
    RowArgs rows;
    uint32_t* list;                        // live rows in order
    uint32_t* count;                       // [0]: how many
};

// One workgroup: 16 rows a thread at a time.
__global__ __launch_bounds__(1024) void es_head_list_kernel(ListArgs a) {
    __shared__ uint32_t waves[16];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rows = a.rows.rows;
    uint32_t base = 0;
    for (uint32_t r0 = 0; r0 < rows; r0 += 16384) {
        // (rows of few calls are spread over the threads)
        const uint32_t each = min((rows - r0 + 1023) / 1024, 16u), mine = r0 + each * threadIdx.x;
        uint32_t live = 0;
        for (uint32_t i = 0; i < each; ++i) {
            const uint32_t r = mine + i;
            if (r >= rows) break;
            live |= uint32_t(kind_of(a.rows, r) == kLive) << i;
        }
        const uint32_t n = __popc(live);
        uint32_t sum = n;                  // over this lane and those before it
        for (uint32_t d = 1; d < 64; d *= 2) {
            const uint32_t y = __shfl_up(sum, d);
            if (lane >= d) sum += y;
        }
        if (lane == 63) waves[wave] = sum;
        __syncthreads();
        uint32_t before = base, all = 0;
        for (uint32_t w = 0; w < 16; ++w) {
            if (w < wave) before += waves[w];
            all += waves[w];
        }
        uint32_t at = before + sum - n;
        for (uint32_t i = 0; i < 16; ++i)
            if (live >> i & 1) a.list[at++] = mine + i;
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) *a.count = base;
}

struct PackArgs {
    const uint16_t* from;
    uint16_t* to;
    uint64_t stride;                       // of `from`; `to` has rows of `padded`
    uint32_t *list, *count;                // row i of `to` is row list[i] of `from`; null: row i of `rows`
    bool lists;                            // (they are made here)
    uint32_t rows, width, padded;
    // of the gradients: what a row's products are scaled by (null: none)
    const float *grad, *lse;
    float *factor, *minus_lse;
    float scale;                           // with its sign
    RowArgs out;                           // of a call's rows: those that are not live are cleared
};

// Row i of the copies: row `row` of the others, or zeros.
__device__ __forceinline__ void pack_row(const PackArgs& a, uint32_t i, uint32_t row, bool live, uint32_t lane) {
    const uint16_t* const from = a.from + row * a.stride;
    uint16_t* const to = a.to + uint64_t(i) * a.padded;
    for (uint32_t k = 8 * lane; k < a.padded; k += 512) {
        u32x4_t v = {0, 0, 0, 0};
        if (live && k + 8 <= a.width) {
            v = load_row8(from + k);
        } else if (live) {
            for (uint32_t e = 0; k + e < a.width; ++e)
                v[e / 2] |= uint32_t(load<uint16_t>(from + k + e)) << (16 * (e % 2));
        }
        store<u32x4_t>(to + k, v);
    }
    if (a.factor != nullptr && lane == 0) {
        // (times the sum of the wanted weights, which is 1 if it is a number)
        a.factor[i] = !live ? 0.0f : is_lost(a.out, row) ? eskv::nan() : a.scale * a.grad[row];
        a.minus_lse[i] = live ? -a.lse[row] : 0.0f;
    }
}

// Rows copied to where every row starts at a word of 16 bytes and ends in zeros; the
// rows behind the last one, up to a tile's end, are zeros.  One wave a row.  Where there
// are few rows each wave looks at all of them for its own's place: a launch less.
__global__ __launch_bounds__(256) void es_head_pack_kernel(PackArgs a) {
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t i = uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (a.list != nullptr && i < a.rows) clear_row(a.out, i, lane);
    if (!a.lists) {
        const uint32_t count = a.count != nullptr ? *a.count : a.rows;
        if (i < count)
            pack_row(a, i, a.list != nullptr ? a.list[i] : i, true, lane);
        else if (i < (count + kTile - 1) / kTile * kTile)
            pack_row(a, i, 0, false, lane);
        return;
    }
    uint32_t before = 0, count = 0;
    bool live = false;
    for (uint32_t q0 = 0; q0 < a.rows; q0 += 256) {
        bool is[4];
#pragma unroll
        for (uint32_t y = 0; y < 4; ++y) {
            const uint32_t r = q0 + 64 * y + lane;
            is[y] = r < a.rows && kind_of(a.out, r) == kLive;
        }
#pragma unroll
        for (uint32_t y = 0; y < 4; ++y) {
            const uint32_t r0 = q0 + 64 * y;
            const uint64_t some = __ballot(is[y]);
            count += __popcll(some);
            if (r0 + 64 <= i) {
                before += __popcll(some);
            } else if (r0 <= i) {
                before += __popcll(some & ((uint64_t(1) << (i - r0)) - 1));
                live = some >> (i - r0) & 1;
            }
        }
    }
    if (i == 0 && lane == 0) *a.count = count;
    if (live) {
        if (lane == 0) a.list[before] = i;
        pack_row(a, before, i, true, lane);
    }
    if (i >= count && i < (count + kTile - 1) / kTile * kTile) pack_row(a, i, 0, false, lane);
}

// ----------------------------------------------------------------- scores --

struct StatsArgs {
    Product p;                             // a: the vocabulary's rows, b: the packed rows
    float* parts;                          // [rows][parts_stride] pairs: maximum, sum
    uint64_t parts_stride;
    uint32_t part0;                        // of this launch's first tile
    float scale;
};

// e^x of differences of logits.  The logits themselves stay in their own units: a maximum of some
// thousands times log2(e) would be off by a step of its own, a difference of them is not.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// A tile's rows of logits as maxima and sums.
template <int kSize>
__global__ __launch_bounds__(2 * kSize, 2) void es_head_stats_kernel(StatsArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Place at = place_of(blockIdx.x, a.p);
    const uint32_t m0 = at.m * kSize, n0 = at.n * kSize;
    const uint32_t count = *a.p.count;
    if (n0 >= count) return;
    Tile<kSize> c;
    product_tile<false, false, kSize>(a.p, m0, n0, count - n0, 0, a.p.depth, lds, c);
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t m_have = a.p.a.extent - m0;
    float* const pair = reinterpret_cast<float*>(lds);   // [2 waves of m][n] pairs
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float top = -eskv::inf();
#pragma unroll
        for (int i = 0; i < c.kBlocks; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t m = c.m_of(wave, lane, i) + e;
                const float z = m < m_have ? c.x[i][j][e] * a.scale : -eskv::inf();
                c.x[i][j][e] = z;
                top = fmaxf(top, z);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float from = top == -eskv::inf() ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < c.kBlocks; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += exp_of(c.x[i][j][e] - from);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16) {
            const uint32_t n = 64 * (wave >> 1) + 16 * j + lane;
            pair[2 * (kSize * (wave & 1) + n)] = top;
            pair[2 * (kSize * (wave & 1) + n) + 1] = sum;
        }
    }
    __syncthreads();
    const uint32_t n = threadIdx.x;
    if (n < kSize && n0 + n < count) {
        const float t0 = pair[2 * n], t1 = pair[2 * (kSize + n)];
        const float top = fmaxf(t0, t1), from = top == -eskv::inf() ? 0.0f : top;
        const float sum = pair[2 * n + 1] * exp_of(t0 - from) +
                          pair[2 * (kSize + n) + 1] * exp_of(t1 - from);
        float* const to = a.parts + 2 * ((n0 + n) * a.parts_stride + a.part0 + at.m);
        to[0] = top;
        to[1] = sum;
    }
}

struct FewStatsArgs {
    esfew::FewArgs f;
    float* parts;                          // [rows][workgroups] pairs
    float scale;
};

// The same of up to 64 rows, as they are: a workgroup's blocks are a part.
template <int kBlocks, int kCols>
__global__ __launch_bounds__(512, kCols == 1 ? 4 : 2) void es_head_few_kernel(FewStatsArgs a) {
    using namespace esfew;
    __shared__ __attribute__((aligned(16))) float sums[kWaves][kBlocks * kCols * 256];
    __shared__ float pair[kWaves][16 * kCols][2];
    const uint32_t lane = threadIdx.x & 63;
    const Part<kBlocks, 4> at(a.f);
    Few<kBlocks, kCols, 4> t;
    t.run(a.f, at.row0, at.k0, at.k1);
    if (a.f.slices > 1) {                  // a block's first wave adds the others'
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int j = 0; j < kCols; ++j)
                *reinterpret_cast<f32x4_t*>(&sums[at.wave][(b * kCols + j) * 256 + 4 * lane]) = t.c[b][j];
        __syncthreads();
        if (at.slice == 0) {
            for (uint32_t w = 1; w < a.f.slices; ++w)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int j = 0; j < kCols; ++j) {
                        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(
                            &sums[at.wave + w][(b * kCols + j) * 256 + 4 * lane]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) t.c[b][j][e] += v[e];
                    }
        }
    }
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
        float top = -eskv::inf();
        float z[kBlocks][4];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool here = at.row0 + 16 * b + 4 * (lane >> 4) + e < a.f.w_rows && at.slice == 0;
                z[b][e] = here ? t.c[b][j][e] * a.scale : -eskv::inf();
                top = fmaxf(top, z[b][e]);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float from = top == -eskv::inf() ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += exp_of(z[b][e] - from);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16) {
            pair[at.wave][16 * j + lane][0] = top;
            pair[at.wave][16 * j + lane][1] = sum;
        }
    }
    __syncthreads();
    const uint32_t n = threadIdx.x;
    if (n < 16 * kCols && n < a.f.rows) {
        float top = -eskv::inf();
        for (uint32_t w = 0; w < kWaves; ++w) top = fmaxf(top, pair[w][n][0]);
        const float from = top == -eskv::inf() ? 0.0f : top;
        float sum = 0.0f;
        for (uint32_t w = 0; w < kWaves; ++w)
            sum += pair[w][n][1] * exp_of(pair[w][n][0] - from);
        float* const to = a.parts + 2 * (uint64_t(n) * gridDim.x + blockIdx.x);
        to[0] = top;
        to[1] = sum;
    }
}

// The same of rows of words against a small vocabulary: a workgroup's 32 tokens are a
// part, whose sums its waves share.
template <int kCols, int kParts>
__global__ __launch_bounds__(512, 2) void es_head_ring_kernel(FewStatsArgs a) {
    using R = esring::Ring<2, kCols, kParts>;
    constexpr uint32_t kWaves = esfew::kWaves, kEach = kCols * 512;
    static_assert(kEach * 4 <= R::kBytes, "the waves' sums fit their rings");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    float* const sums = reinterpret_cast<float*>(lds);   // [wave][row of x][token]
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t row0 = blockIdx.x * 32, n0 = blockIdx.y * 64;   // 64 rows of x a workgroup
    a.f.x += n0 * a.f.x_stride;
    a.f.rows = min(a.f.rows - n0, 64u);
    R t;
    t.run(a.f, row0, wave, kWaves, lds + wave * R::kBytes);
    __syncthreads();
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int j = 0; j < kCols; ++j)
            *reinterpret_cast<f32x4_t*>(sums + wave * kEach + (j * 16 + (lane & 15)) * 32 + 16 * b +
                                        4 * (lane >> 4)) = t.c[b][j];
    __syncthreads();
    // half a wave a row: a lane for each token
    for (uint32_t n = threadIdx.x >> 5; n < 16 * kCols && n < a.f.rows; n += 2 * kWaves) {
        const uint32_t i = threadIdx.x & 31;
        float z = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) z += sums[w * kEach + n * 32 + i];
        z = row0 + i < a.f.w_rows ? z * a.scale : -eskv::inf();
        float top = z;
#pragma unroll
        for (int d = 16; d >= 1; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
        float sum = exp_of(z - (top == -eskv::inf() ? 0.0f : top));
#pragma unroll
        for (int d = 16; d >= 1; d /= 2) sum += __shfl_xor(sum, d);
        if (i == 0) {
            float* const to = a.parts + 2 * (uint64_t(n0 + n) * gridDim.x + blockIdx.x);
            to[0] = top;
            to[1] = sum;
        }
    }
}

struct StreamStatsArgs {
    esstream::StreamArgs s;
    float* parts;                          // [rows][workgroups] pairs
    float scale;
};

// The same of up to 128 rows of words: a workgroup's share of the vocabulary is a part,
// whose maxima and sums run along in registers.  Bound by the head's bytes: 32 rows of
// 5120 against 151936 266 us, 5.9 TB/s, with the scores' kernel; 128 of 2560 175 us, 4.5 TB/s
// and, with the operands' reads from LDS, not far from the matrix unit's bound.
template <int kWaves, int kTokens>
using HeadStream = esstream::Stream<
    kWaves, 2, kTokens, 1,
    esstream::stages_for(32 * kWaves, kTokens, 1, 4 + (kTokens / 8 + kWaves - 1) / kWaves)>;

template <int kWaves, int kTokens>
__global__ __launch_bounds__(64 * kWaves, 1) void es_head_stream_kernel(StreamStatsArgs a) {
    using S = HeadStream<kWaves, kTokens>;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float top[S::kCols], sum[S::kCols];
#pragma unroll
    for (int j = 0; j < S::kCols; ++j) {
        top[j] = -eskv::inf();
        sum[j] = 0.0f;
    }
    S t;
    t.run(a.s, lds, [&](uint32_t row0, uint32_t end) {
#pragma unroll
        for (int j = 0; j < S::kCols; ++j) {
            float z[2][4], most = top[j];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool here = row0 + 32 * wave + 16 * b + 4 * (lane >> 4) + e < end;
                    z[b][e] = here ? t.c[b][j][e] * a.scale : -eskv::inf();
                    most = fmaxf(most, z[b][e]);
                }
            const float from = most == -eskv::inf() ? 0.0f : most;
            sum[j] *= exp_of(top[j] - from);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[j] += exp_of(z[b][e] - from);
            top[j] = most;
        }
    });
    __syncthreads();                       // every wave has left the last stage
    float* const pair = reinterpret_cast<float*>(lds);   // [kWaves][kTokens] pairs
#pragma unroll
    for (int j = 0; j < S::kCols; ++j) {
        float most = fmaxf(top[j], __shfl_xor(top[j], 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float from = most == -eskv::inf() ? 0.0f : most;
        float all = sum[j] * exp_of(top[j] - from);
        all += __shfl_xor(all, 16);
        all += __shfl_xor(all, 32);
        if (lane < 16) {
            pair[2 * (kTokens * wave + 16 * j + lane)] = most;
            pair[2 * (kTokens * wave + 16 * j + lane) + 1] = all;
        }
    }
    __syncthreads();
    const uint32_t n = threadIdx.x;
    if (n < kTokens && n < a.s.rows) {
        float most = -eskv::inf();
        for (uint32_t w = 0; w < kWaves; ++w) most = fmaxf(most, pair[2 * (kTokens * w + n)]);
        const float from = most == -eskv::inf() ? 0.0f : most;
        float all = 0.0f;
        for (uint32_t w = 0; w < kWaves; ++w)
            all += pair[2 * (kTokens * w + n) + 1] *
                   exp_of(pair[2 * (kTokens * w + n)] - from);
        float* const to = a.parts + 2 * (uint64_t(n) * gridDim.x + blockIdx.x);
        to[0] = most;
        to[1] = all;
    }
}

struct ScoreArgs {
    const float* parts;
    uint64_t parts_stride;
    uint32_t n_parts;
    const uint32_t *list, *count;          // null: all rows, which are looked at here
    const uint16_t *x, *w;                 // x: the packed rows, or all
    uint64_t x_stride, w_stride;
    const int64_t* ids;
    const float* teacher;
    float *loss, *logp, *lse;
    uint32_t* status;
    uint32_t hidden, entries, vocab;
    float scale;
};

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

// Of 256 threads: sum and maximum, in one order.
__device__ __forceinline__ float block_sum(float x, float* room) {
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
    __syncthreads();
    return (room[0] + room[1]) + (room[2] + room[3]);
}
__device__ __forceinline__ float block_max(float x, float* room) {
    x = wave_max(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
    __syncthreads();
    return fmaxf(fmaxf(room[0], room[1]), fmaxf(room[2], room[3]));
}

// The teacher's weight of thread e's entry (0: absent), and its logarithm.  The likeliest
// entry's logit is taken off before the scale (halves: the difference of two finite logits is
// finite), so that its own exponential is 1 whatever they are, masks of the type's lowest
// value throughout among them.
__device__ __forceinline__ float teacher_weight(bool here, float t, float scale, float* room,
                                                float& log_q) {
    here = here && has_weight(t, scale);
    const float sign = scale < 0.0f ? -1.0f : 1.0f;
    const float top = sign * block_max(here ? sign * t : -eskv::inf(), room);
    const float half = (0.5f * t - 0.5f * top) * scale, z = here ? half + half : -eskv::inf();
    const float e = here ? expf(z) : 0.0f;
    const float sum = block_sum(e, room);
    const float q = sum > 0.0f ? e / sum : e;          // (NaN stays NaN)
    log_q = q > 0.0f ? z - logf(sum) : 0.0f;
    return sum != sum ? sum : q;
}

// A live row's parts joined, and its scores: each id's logit is a product of its own.
// One workgroup a row, waves by turns over the entries.
__global__ __launch_bounds__(256) void es_head_score_kernel(ScoreArgs a) {
    __shared__ float room[4], logits[kMaxEntries];
    const uint32_t i = blockIdx.x;
    if (a.count != nullptr && i >= *a.count) return;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t row = a.list != nullptr ? a.list[i] : i;
    if (a.list == nullptr) {
        const int64_t id = threadIdx.x < a.entries ? a.ids[uint64_t(row) * a.entries + threadIdx.x] : -1;
        const bool some = __syncthreads_or(id >= 0), bad = __syncthreads_or(id >= int64_t(a.vocab));
        if (!some || bad) {                // dead or void
            const float v = bad ? eskv::nan() : 0.0f;
            if (threadIdx.x < a.entries) a.logp[uint64_t(row) * a.entries + threadIdx.x] = v;
            if (threadIdx.x == 0) {
                a.lse[row] = v;
                if (a.loss != nullptr) a.loss[row] = v;
                if (bad && a.status != nullptr) atomicOr(a.status, ES_HEAD_BAD_ID);
            }
            return;
        }
    }
    const float* const parts = a.parts + 2 * i * a.parts_stride;
    float top = -eskv::inf();
    for (uint32_t m = threadIdx.x; m < a.n_parts; m += 256) top = fmaxf(top, parts[2 * m]);
    top = block_max(top, room);
    const float from = top == -eskv::inf() ? 0.0f : top;
    float sum = 0.0f;
    for (uint32_t m = threadIdx.x; m < a.n_parts; m += 256)
        sum += parts[2 * m + 1] * exp_of(parts[2 * m] - from);
    sum = block_sum(sum, room);
    const float lse = from + logf(sum);

    const uint16_t* const x = a.x + i * a.x_stride;
    const uint32_t whole = a.hidden / 8 * 8;
    for (uint32_t e = wave; e < a.entries; e += 4) {
        const int64_t id = a.ids[uint64_t(row) * a.entries + e];
        if (id < 0) continue;
        const uint16_t* const w = a.w + uint64_t(id) * a.w_stride;
        float dot = 0.0f;
        for (uint32_t k = 8 * lane; k < whole; k += 512) {
            float u[8], v[8];
            eskv::unpack8(load_row8(x + k), u);
            eskv::unpack8(load_row8(w + k), v);
#pragma unroll
            for (int y = 0; y < 8; ++y) dot = __builtin_fmaf(u[y], v[y], dot);
        }
        if (whole + lane < a.hidden)
            dot = __builtin_fmaf(eskv::bf16_lo(load<uint16_t>(x + whole + lane)),
                                 eskv::bf16_lo(load<uint16_t>(w + whole + lane)), dot);
        dot = wave_sum(dot);
        if (lane == 0) logits[e] = dot * a.scale;
    }
    __syncthreads();
    const uint32_t e = threadIdx.x;
    const uint64_t at = uint64_t(row) * a.entries + e;
    const bool here = e < a.entries && a.ids[at] >= 0;
    // (a token with nearly all of the weight: its logit's sum and its normaliser's have their own
    // orders, and a probability is at most 1)
    const float diff = here ? logits[e] - lse : 0.0f, logp = diff > 0.0f ? 0.0f : diff;
    if (e < a.entries) a.logp[at] = logp;
    if (e == 0) a.lse[row] = lse;
    if (a.teacher != nullptr) {
        float log_q;
        const float q = teacher_weight(here, here ? a.teacher[at] : 0.0f, a.scale, room, log_q);
        // (a weight of zero takes nothing, whatever the student gives its entry)
        const float loss = block_sum(here && q != 0.0f ? q * (log_q - logp) : 0.0f, room);
        if (e == 0) a.loss[row] = loss;
    }
}

// -------------------------------------------------------------- gradients --

struct ProbArgs {
    Product p;                             // a: a piece of the vocabulary, b: the packed rows
    const float *factor, *minus_lse;       // of a packed row
    uint16_t* d;                           // [rows][d_stride]
    uint64_t d_stride;
    float scale;
};

// The logits' gradients without what their ids add: factor softmax(z), as bf16 (RNE):
// both products that take them have the matrix unit's operands.
template <int kSize>
__global__ __launch_bounds__(2 * kSize, 2) void es_head_prob_kernel(ProbArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Place at = place_of(blockIdx.x, a.p);
    const uint32_t m0 = at.m * kSize, n0 = at.n * kSize;
    const uint32_t count = *a.p.count;
    if (n0 >= count) return;
    Tile<kSize> c;
    product_tile<false, false, kSize>(a.p, m0, n0, count - n0, 0, a.p.depth, lds, c);
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t m_have = a.p.a.extent - m0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t n = n0 + c.n_of(wave, lane, j);
        const uint32_t have = n < count ? m_have : 0;    // rows behind the last: zeros, not 0 times a logit
        const float f = a.factor[n], l = a.minus_lse[n];
#pragma unroll
        for (int i = 0; i < c.kBlocks; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t m = c.m_of(wave, lane, i) + e;
                const float p = f * exp_of(__builtin_fmaf(c.x[i][j][e], a.scale, l));
                c.x[i][j][e] = m < have ? p : 0.0f;
            }
    }
    tile_to_lds(c, lds);
    __syncthreads();
    // (as far as a sum over the rows goes)
    const uint32_t rows = (count + kDepth - 1) / kDepth * kDepth;
    store_rows<kSize>(lds, a.d, a.d_stride, m0, kSize,
                      [&](uint32_t n) { return n0 + n < rows ? int64_t(n0 + n) : int64_t(-1); });
}

struct EntryArgs {
    const uint32_t *list, *count;
    const int64_t* ids;
    const float *teacher, *logp, *grad;
    uint16_t* d;
    uint64_t d_stride;
    uint32_t entries, v0, v_end;           // the piece
    float scale, sign_scale;
};

// The gradients at the ids, f (Q p - q) with the weights of equal ids summed, take
// the places of f Q p: rounded once, where q and p nearly cancel too.
__global__ __launch_bounds__(256) void es_head_entries_kernel(EntryArgs a) {
    __shared__ float room[4], weights[kMaxEntries];
    __shared__ int64_t ids[kMaxEntries];
    const uint32_t i = blockIdx.x;
    if (i >= *a.count) return;
    const uint32_t row = a.list[i], e = threadIdx.x;
    const uint64_t at = uint64_t(row) * a.entries + e;
    const int64_t id = e < a.entries ? a.ids[at] : -1;
    float q = id >= 0 ? 1.0f : 0.0f;
    if (a.teacher != nullptr) {
        float log_q;
        q = teacher_weight(id >= 0, id >= 0 ? a.teacher[at] : 0.0f, a.scale, room, log_q);
    }
    ids[e] = id;
    weights[e] = q;
    __syncthreads();
    if (id < int64_t(a.v0) || id >= int64_t(a.v_end)) return;
    float all = 0.0f;
    for (uint32_t k = 0; k < a.entries; ++k) all += ids[k] == id ? weights[k] : 0.0f;
    const float d = a.sign_scale * a.grad[row] * (expf(a.logp[at]) - all);
    a.d[i * a.d_stride + (id - a.v0)] = static_cast<uint16_t>(pack_bf16(d, 0.0f));
}

struct RowGradArgs {
    Product p;                             // a: the piece (wide), b: d
    float* parts;                          // [splits][rows][parts_stride] binary32
    uint64_t parts_rows, parts_stride;
    uint32_t hidden, add;                  // add: to what is there
    uint16_t* out;                         // or, with one split and one piece, bf16
    uint64_t out_stride;
    const uint32_t* list;
};

template <int kSize>
__global__ __launch_bounds__(2 * kSize, 2) void es_head_row_grad_kernel(RowGradArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Place at = place_of(blockIdx.x, a.p);
    const uint32_t m0 = at.m * kSize, n0 = at.n * kSize;
    const uint32_t count = *a.p.count;
    if (n0 >= count) return;
    const uint32_t k0 = at.split * a.p.split_depth;
    Tile<kSize> c;
    product_tile<true, false, kSize>(a.p, m0, n0, count - n0, k0, min(a.p.depth, k0 + a.p.split_depth), lds, c);
    if (a.out != nullptr) {
        __syncthreads();
        tile_to_lds(c, lds);
        __syncthreads();
        store_rows<kSize>(lds, a.out, a.out_stride, m0, a.hidden - m0, [&](uint32_t n) {
            return n0 + n < count ? int64_t(a.list[n0 + n]) : int64_t(-1);
        });
        return;
    }
    float* const to = a.parts + (at.split * a.parts_rows + n0) * a.parts_stride + m0;
    const uint32_t m_have = a.p.a.extent - m0, n_have = count - n0;
    for_words(c, [&](f32x4_t v, uint32_t m, uint32_t n) {
        if (m >= m_have || n >= n_have) return;          // (extents are multiples of 8)
        float* const q = to + n * a.parts_stride + m;
        if (a.add) {
            const f32x4_t was = load<f32x4_t>(q);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += was[e];
        }
        store<f32x4_t>(q, v);
    });
}

struct JoinArgs {
    const float* parts;
    uint64_t parts_rows, parts_stride;
    uint32_t splits, hidden;
    const uint32_t *list, *count;
    uint16_t* out;
    uint64_t out_stride;
};

// The splits' sums, in one order, rounded once.
__global__ __launch_bounds__(256) void es_head_join_kernel(JoinArgs a) {
    const uint32_t i = blockIdx.x, h = 4 * (blockIdx.y * 256 + threadIdx.x);
    if (i >= *a.count || h >= a.hidden) return;
    const float* p = a.parts + i * a.parts_stride + h;
    f32x4_t v = load<f32x4_t>(p);
    for (uint32_t s = 1; s < a.splits; ++s) {
        const f32x4_t w = load<f32x4_t>(p + s * a.parts_rows * a.parts_stride);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e];
    }
    uint16_t* const to = a.out + a.list[i] * a.out_stride + h;
    const u32x2_t w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    if (h + 4 <= a.hidden) {
        eskv::store_row4(to, w);
    } else {
        for (uint32_t e = 0; h + e < a.hidden; ++e)
            store<uint16_t>(to + e, static_cast<uint16_t>(w[e / 2] >> (16 * (e % 2))));
    }
}

struct HeadGradArgs {
    Product p;                             // a: the packed rows (wide), b: d (wide)
    uint16_t* out;                         // the piece's first row
    uint64_t out_stride;
    uint32_t n_have, hidden;               // rows of the piece
};

template <int kSize>
__global__ __launch_bounds__(2 * kSize, 2) void es_head_weight_grad_kernel(HeadGradArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Place at = place_of(blockIdx.x, a.p);
    const uint32_t m0 = at.m * kSize, n0 = at.n * kSize;
    const uint32_t depth = (*a.p.count + kDepth - 1) / kDepth * kDepth;   // zeros behind the rows
    Tile<kSize> c;
    product_tile<true, true, kSize>(a.p, m0, n0, a.n_have - n0, 0, depth, lds, c);
    __syncthreads();
    tile_to_lds(c, lds);
    __syncthreads();
    store_rows<kSize>(lds, a.out, a.out_stride, m0, a.hidden - m0, [&](uint32_t n) {
        return n0 + n < a.n_have ? int64_t(n0 + n) : int64_t(-1);
    });
}

}  // namespace eshead
