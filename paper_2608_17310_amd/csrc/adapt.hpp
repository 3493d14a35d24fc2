// A shared projection with low-rank adapters beside it, one member's for each row:
//   y = W x + s_i B_i (A_i x).
// The small product u = s_i A_i x comes first, a row at a time as wide as the rank;
// the large one then adds B_i u to its tiles before they are rounded.
#pragma once

#include "few.hpp"
#include "mm_tile.hpp"
#include "ring.hpp"
#include "stream.hpp"

namespace esadapt {

using namespace esmm;

constexpr uint32_t kMaxRank = 128;

struct SmallArgs {
    const uint16_t* x;
    uint64_t x_stride;
    const uint16_t* a;                     // [members][rank][inner]
    const float* scales;                   // or null
    const int32_t* index;
    float* u;                              // [rows][rank]
    uint32_t* status;
    uint32_t rows, inner, members, rank;
    bool split;                            // u as the matrix unit takes it, [rows][2][rank] bf16
};

// Element r of row n of u.  The matrix unit takes it as the sum of two bf16 numbers, cut and
// rounded (RNE): within 2^-15 of it.  Both have its sign, and of a normal number neither is
// 0: an infinity in B times the two is that infinity again, as it is times u.
__device__ __forceinline__ void store_u(const SmallArgs& a, uint32_t n, uint32_t r, float v) {
    if (!a.split) {
        a.u[uint64_t(n) * a.rank + r] = v;
        return;
    }
    const uint32_t word = __float_as_uint(v), sign = word >> 16 & 0x8000u;
    uint32_t high = word >> 16, low = 0;
    if (v != v) {
        high = 0x7FC0u;
    } else if (v != 0.0f) {
        if (__builtin_fabsf(v) < eskv::inf())
            low = pack_bf16(v - __uint_as_float(word & 0xFFFF0000u), 0.0f) & 0x7FFFu;
        low = sign | (low == 0 ? 1u : low);
    }
    uint16_t* const to = reinterpret_cast<uint16_t*>(a.u) + uint64_t(n) * 2 * a.rank + r;
    to[0] = static_cast<uint16_t>(high);
    to[a.rank] = static_cast<uint16_t>(low);
}

constexpr uint32_t kSmallRows = 32;

// A workgroup takes 32 rows, and their members one by one: a product of the member's A
// with those rows, whose sum its waves share.
template <int kBlocks, int kParts>         // blocks of 16 of the rank, at a time
__global__ __launch_bounds__(512, 2) void es_adapt_small_kernel(SmallArgs a) {
    using R = esring::Ring<kBlocks, 2, kParts>;
    constexpr uint32_t kWaves = esfew::kWaves, kEach = kBlocks * 512;
    static_assert(kWaves * kEach * 4 <= kWaves * R::kBytes, "the waves' sums fit their rings");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    float* const sums = reinterpret_cast<float*>(lds);   // [wave][row][of the rank]
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t n0 = blockIdx.x * kSmallRows, n = n0 + (lane & 31);
    const int32_t mine = n < a.rows ? a.index[n] : -1;
    const bool bad = mine >= int32_t(a.members);
    if (bad && wave == 0 && a.status != nullptr) atomicOr(a.status, ES_ADAPT_BAD_INDEX);
    uint32_t left = uint32_t(__ballot(mine >= 0 && !bad));
    esfew::FewArgs f{};
    f.x = a.x + uint64_t(n0) * a.x_stride;
    f.x_stride = a.x_stride;
    f.rows = min(a.rows - n0, kSmallRows);
    f.w_stride = a.inner;
    f.w_rows = a.rank;
    f.width = a.inner;
    while (left != 0) {
        const int32_t member = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
        const uint32_t match = uint32_t(__ballot(mine == member));
        left &= ~match;
        const float s = a.scales != nullptr ? a.scales[member] : 1.0f;
        f.w = a.a + uint64_t(member) * a.rank * a.inner;
        for (uint32_t r0 = 0; r0 < a.rank; r0 += 16 * kBlocks) {
            R t;
            t.run(f, r0, wave, kWaves, lds + wave * R::kBytes);
            __syncthreads();
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<f32x4_t*>(sums + wave * kEach +
                                                (16 * j + (lane & 15)) * (16 * kBlocks) + 16 * b +
                                                4 * (lane >> 4)) = t.c[b][j];
            __syncthreads();
            for (uint32_t e = threadIdx.x; e < kEach; e += 512) {
                const uint32_t i = e / (16 * kBlocks), r = r0 + e % (16 * kBlocks);
                if ((match >> i & 1) == 0 || r >= a.rank) continue;
                float sum = 0.0f;
#pragma unroll
                for (uint32_t w = 0; w < kWaves; ++w) sum += sums[w * kEach + e];
                store_u(a, n0 + i, r, s * sum);
            }
            __syncthreads();               // the rings are free again
        }
    }
}

// u of few rows: a wave for each of its elements.
__global__ __launch_bounds__(256) void es_adapt_few_small_kernel(SmallArgs a) {
    const uint32_t lane = threadIdx.x & 63, n = blockIdx.x;
    const uint32_t r = uniform(blockIdx.y * 4 + (threadIdx.x >> 6));
    const int32_t member = a.index[n];
    if (member >= int32_t(a.members) && a.status != nullptr && blockIdx.y == 0 && threadIdx.x == 0)
        atomicOr(a.status, ES_ADAPT_BAD_INDEX);
    if (member < 0 || member >= int32_t(a.members) || r >= a.rank) return;
    const uint16_t* const x = a.x + uint64_t(n) * a.x_stride;
    const uint16_t* const row = a.a + (uint64_t(member) * a.rank + r) * a.inner;
    float sum[8] = {};
#pragma unroll 4
    for (uint32_t k = 8 * lane; k < a.inner; k += 512) {
        float u[8], v[8];
        eskv::unpack8(load<u32x4_t>(row + k), u);
        eskv::unpack8(load_row8(x + k), v);
#pragma unroll
        for (int y = 0; y < 8; ++y) sum[y] = __builtin_fmaf(u[y], v[y], sum[y]);
    }
    float all = ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) all += __shfl_xor(all, d);
    if (lane == 0) store_u(a, n, r, (a.scales != nullptr ? a.scales[member] : 1.0f) * all);
}

struct AddArgs {
    const int32_t* index;
    const float* u;                        // of a tile split
    const uint16_t* b;                     // [members][outer][rank]
    uint32_t rows, outer, members, rank;
};

// B u added to a tile, for the members of a wave's 64 rows one by one.  Where a
// member has all of 16 rows its products go straight into the tile; otherwise into
// results of their own, of which its rows take theirs: a member that holds
// infinities or NaN reaches no other's rows.  u's two numbers make twice the products (8403
// rows, 2560 to 9728, rank 32: 374 us, with u rounded to one number 369; 16384 rows of 5120, rank
// 64: 728 and 717), but ranks up to 16 (kHalves 1) have both in the length of one instruction.
template <int kHalves, int kSize>
__device__ __forceinline__ void add_adapters(const AddArgs& a, uint32_t m0, uint32_t n0, Tile<kSize>& c) {
    constexpr int kBlocks = Tile<kSize>::kBlocks;
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t n1 = n0 + 64 * (wave >> 1);
    int32_t mine[4];                       // of the lane's row of each block
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t n = n1 + 16 * j + (lane & 15);
        mine[j] = n < a.rows ? a.index[n] : -1;
    }
    const uint16_t* const u = reinterpret_cast<const uint16_t*>(a.u);
    const int32_t every = n1 + lane < a.rows ? a.index[n1 + lane] : -1;
    uint64_t left = __ballot(every >= 0 && every < int32_t(a.members));
    while (left != 0) {
        const int32_t member = __builtin_amdgcn_readlane(every, __builtin_ctzll(left));
        const uint64_t rows = __ballot(every == member);
        left &= ~rows;
        for (uint32_t r0 = 0; r0 < a.rank; r0 += 32) {
            const uint32_t r = r0 + 8 * (lane >> 4), of_b = r < a.rank ? r : r - a.rank;
            const bool here = r < (kHalves == 1 ? 2 * a.rank : a.rank);
            u32x4_t bv[kBlocks];
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                const uint32_t m = min(m0 + kSize / 2 * (wave & 1) + 16 * i + (lane & 15), a.outer - 1);
                bv[i] = here ? load<u32x4_t>(a.b + (uint64_t(member) * a.outer + m) * a.rank + of_b)
                             : u32x4_t{0, 0, 0, 0};
            }
#pragma unroll 1
            for (uint32_t h = 0; h < kHalves; ++h) {     // (unrolled it would spill)
                u32x4_t uv[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    uv[j] = mine[j] == member && here
                                ? load<u32x4_t>(u + (uint64_t(n1 + 16 * j + (lane & 15)) * 2 + h) * a.rank + r)
                                : u32x4_t{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t some = uint32_t(rows >> (16 * j)) & 0xFFFFu;
                    if (some == 0) continue;
                    const bool whole = some == 0xFFFFu;
#pragma unroll
                    for (int i = 0; i < kBlocks; ++i) {
                        const f32x4_t from = whole ? c.x[i][j] : f32x4_t{0, 0, 0, 0};
                        const f32x4_t t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8_t, bv[i]), __builtin_bit_cast(bf16x8_t, uv[j]), from, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            c.x[i][j][e] = whole                ? t[e]
                                           : mine[j] == member ? c.x[i][j][e] + t[e]
                                                               : c.x[i][j][e];
                    }
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (!__any(mine[j] >= int32_t(a.members))) continue;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                c.x[i][j][e] = mine[j] >= int32_t(a.members) ? eskv::nan() : c.x[i][j][e];
    }
}

// Results v of row n, rows m .. of the matrix (before `end`), with their member's B u.
__device__ __forceinline__ f32x4_t with_adapter(const AddArgs& a, f32x4_t v, uint32_t n, uint32_t m,
                                                uint32_t end, int32_t member) {
    if (member >= int32_t(a.members)) return f32x4_t{eskv::nan(), eskv::nan(), eskv::nan(), eskv::nan()};
    if (member < 0) return v;
    const uint16_t* const b = a.b + uint64_t(member) * a.outer * a.rank;
    const float* const u = a.u + uint64_t(n) * a.rank;
    float low[4] = {};
    // (the words of 16 of the rank on their way at a time)
    for (uint32_t r0 = 0; r0 < a.rank; r0 += 16) {
        f32x4_t q[2][2];
        u32x4_t p[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t r = min(r0 + 8 * h, a.rank - 8);
            q[h][0] = load<f32x4_t>(u + r);
            q[h][1] = load<f32x4_t>(u + r + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                p[h][e] = load<u32x4_t>(b + uint64_t(min(m + e, end - 1)) * a.rank + r);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (r0 + 8 * h >= a.rank) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float y[8];
                eskv::unpack8(p[h][e], y);
#pragma unroll
                for (int z = 0; z < 8; ++z) low[e] = __builtin_fmaf(q[h][z / 4][z % 4], y[z], low[e]);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += low[e];
    return v;
}

// Up to four of them, rounded.
__device__ __forceinline__ void store_results(uint16_t* to, f32x4_t v, uint32_t have) {
    const u32x2_t w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    if (have >= 4) {
        eskv::store_row4(to, w);
    } else {
        for (uint32_t e = 0; e < have; ++e)
            store<uint16_t>(to + e, static_cast<uint16_t>(w[e / 2] >> (16 * (e % 2))));
    }
}

struct TileArgs {
    Product p;                             // a: W, b: the rows
    AddArgs add;
    uint16_t* out;
    uint64_t out_stride;
};

template <int kSize, int kHalves>
__global__ __launch_bounds__(2 * kSize, 2) void es_adapt_tile_kernel(TileArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Place at = place_of(blockIdx.x, a.p);
    const uint32_t m0 = at.m * kSize, n0 = at.n * kSize;
    Tile<kSize> c;
    product_tile<false, false, kSize>(a.p, m0, n0, a.add.rows - n0, 0, a.p.depth, lds, c);
    add_adapters<kHalves>(a.add, m0, n0, c);
    __syncthreads();
    tile_to_lds(c, lds);
    __syncthreads();
    store_rows<kSize>(lds, a.out, a.out_stride, m0, a.add.outer - m0, [&](uint32_t n) {
        return n0 + n < a.add.rows ? int64_t(n0 + n) : int64_t(-1);
    });
}

struct PartArgs {
    Product p;
    float* parts;                          // [splits][rows][stride] binary32
    uint64_t stride;
    uint32_t rows, outer;
};

// Where there are few tiles their sums are divided too, and joined with B u.
template <int kSize>
__global__ __launch_bounds__(2 * kSize, 2) void es_adapt_part_kernel(PartArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Place at = place_of(blockIdx.x, a.p);
    const uint32_t m0 = at.m * kSize, n0 = at.n * kSize, k0 = at.split * a.p.split_depth;
    const uint32_t n_have = a.rows - n0, m_have = a.outer - m0;
    Tile<kSize> c;
    product_tile<false, false, kSize>(a.p, m0, n0, n_have, k0, min(a.p.depth, k0 + a.p.split_depth), lds, c);
    float* const to = a.parts + (uint64_t(at.split) * a.rows + n0) * a.stride + m0;
    for_words(c, [&](const f32x4_t& v, uint32_t m, uint32_t n) {
        if (m < m_have && n < n_have) store<f32x4_t>(to + n * a.stride + m, v);   // (stride: a multiple of 4)
    });
}

struct JoinArgs {
    const float* parts;
    uint64_t stride;
    uint32_t splits;
    AddArgs add;
    uint16_t* out;
    uint64_t out_stride;
};

// Four results a lane: their parts in one order, and their row's B u.
__global__ __launch_bounds__(256) void es_adapt_join_kernel(JoinArgs a) {
    const uint32_t n = blockIdx.y, m = 4 * (blockIdx.x * 256 + threadIdx.x);
    if (m >= a.add.outer) return;
    const int32_t member = a.add.index[n];
    const float* const from = a.parts + uint64_t(n) * a.stride + m;
    f32x4_t v = load<f32x4_t>(from);
    for (uint32_t s = 1; s < a.splits; ++s) {
        const f32x4_t w = load<f32x4_t>(from + uint64_t(s) * a.add.rows * a.stride);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e];
    }
    v = with_adapter(a.add, v, n, m, a.add.outer, member);
    store_results(a.out + uint64_t(n) * a.out_stride + m, v, a.add.outer - m);
}

struct FewArgs {
    esfew::FewArgs f;
    AddArgs add;
    uint16_t* out;
    uint64_t out_stride;
};

// Up to 64 rows and a matrix of few: the waves' sums of a block meet in LDS, where each
// result takes its own member's B u.
template <int kBlocks, int kCols, int kParts>
__global__ __launch_bounds__(512, 2) void es_adapt_few_kernel(FewArgs a) {
    using R = esring::Ring<kBlocks, kCols, kParts>;
    constexpr uint32_t kWaves = esfew::kWaves, kEach = kBlocks * kCols * 256;
    static_assert(kEach * 4 <= R::kBytes, "the waves' sums fit their rings");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    float* const sums = reinterpret_cast<float*>(lds);   // [wave][row of x][row of the matrix]
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t row0 = blockIdx.x * 16 * kBlocks;
    R t;
    t.run(a.f, row0, wave, kWaves, lds + wave * R::kBytes);
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int j = 0; j < kCols; ++j)
            *reinterpret_cast<f32x4_t*>(sums + wave * kEach + (j * 16 + (lane & 15)) * (16 * kBlocks) +
                                        16 * b + 4 * (lane >> 4)) = t.c[b][j];
    __syncthreads();
    for (uint32_t y = threadIdx.x; y < kEach; y += 64 * kWaves) {
        const uint32_t n = y / (16 * kBlocks), m = row0 + y % (16 * kBlocks);
        if (n >= a.f.rows || m >= a.f.w_rows) continue;
        float sum = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) sum += sums[w * kEach + y];
        const int32_t member = a.add.index[n];
        if (member >= int32_t(a.add.members)) sum = eskv::nan();
        if (member >= 0 && member < int32_t(a.add.members)) {
            const uint16_t* const b = a.add.b + (uint64_t(member) * a.add.outer + m) * a.add.rank;
            const float* const u = a.add.u + uint64_t(n) * a.add.rank;
            float low = 0.0f;
            for (uint32_t r = 0; r < a.add.rank; r += 8) {
                float p[8];
                eskv::unpack8(load<u32x4_t>(b + r), p);
                const f32x4_t q[2] = {load<f32x4_t>(u + r), load<f32x4_t>(u + r + 4)};
#pragma unroll
                for (int z = 0; z < 8; ++z) low = __builtin_fmaf(p[z], q[z / 4][z % 4], low);
            }
            sum += low;
        }
        store<uint16_t>(a.out + uint64_t(n) * a.out_stride + m, static_cast<uint16_t>(pack_bf16(sum, 0.0f)));
    }
}

struct StreamArgs {
    esstream::StreamArgs s;
    AddArgs add;
    uint16_t* out;
    uint64_t out_stride;
};

// Rows of words and a matrix of many rows: each lane adds its own row's B u to its four
// results.  Bound by the matrix's bytes, so by how many of them are on their way: LDS is
// full of stages.  32 rows of 32 members, 5120 x 17408: 46 us with the small product, where
// two workgroups a compute unit of three stages each took 57.
template <int kWaves, int kTokens>
using AdaptStream = esstream::Stream<
    kWaves, 1, kTokens, 2,
    esstream::stages_for(16 * kWaves, kTokens, 2, 2 * (2 + (kTokens / 8 + kWaves - 1) / kWaves))>;

template <int kWaves, int kTokens>
__global__ __launch_bounds__(64 * kWaves, 1) void es_adapt_stream_kernel(StreamArgs a) {
    using S = AdaptStream<kWaves, kTokens>;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    S t;
    t.run(a.s, lds, [&](uint32_t row0, uint32_t end) {
        const uint32_t m = row0 + 16 * wave + 4 * (lane >> 4);
        if (m >= end) return;
#pragma unroll
        for (int j = 0; j < S::kCols; ++j) {
            const uint32_t n = 16 * j + (lane & 15);
            if (n >= a.s.rows) continue;
            store_results(a.out + uint64_t(n) * a.out_stride + m,
                          with_adapter(a.add, t.c[0][j], n, m, end, a.add.index[n]), end - m);
        }
    });
}

}  // namespace esadapt
