// A shared projection with low-rank adapters beside it, one member's for each row:
//   y = W x + s_i B_i (A_i x).
// The small product u = s_i A_i x comes first, a row at a time as wide as the rank;
// the large one then adds B_i u to its tiles before they are rounded.
#pragma once

#include "mm_tile.hpp"

namespace esadapt {

using namespace esmm;

constexpr uint32_t kMaxRank = 128;

struct SmallArgs {
    const uint16_t* x;
    uint64_t x_stride;
    const uint16_t* a;                     // [members][rank][inner]
    const float* scales;                   // or null
    const int32_t* index;
    uint16_t* u;                           // [rows][rank]
    uint32_t* status;
    uint32_t rows, inner, members, rank;
};

constexpr uint32_t kSmallRows = 32;

// A workgroup takes 32 rows, and their members one by one; its waves share the sum, 16
// of it at a time in turn.  u is rounded to bf16 (RNE) for the matrix unit: it is off by as much
// as y's own rounding, of a smaller term.
__global__ __launch_bounds__(kThreads) void es_adapt_small_kernel(SmallArgs a) {
    __shared__ float part[8][32][33];      // [wave][row of A][row]
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const uint32_t n0 = blockIdx.x * kSmallRows, n = n0 + (lane & 31);
    const int32_t mine = n < a.rows ? a.index[n] : -1;
    const bool bad = mine >= int32_t(a.members);
    if (bad && wave == 0 && a.status != nullptr) atomicOr(a.status, ES_ADAPT_BAD_INDEX);
    uint32_t left = uint32_t(__ballot(mine >= 0 && !bad));
    const uint16_t* const x = a.x + uint64_t(min(n, a.rows - 1)) * a.x_stride;
    while (left != 0) {
        const int32_t member = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
        const uint32_t match = uint32_t(__ballot(mine == member));
        left &= ~match;
        const float s = a.scales != nullptr ? a.scales[member] : 1.0f;
        for (uint32_t r0 = 0; r0 < a.rank; r0 += 32) {
            const uint32_t r = min(r0 + (lane & 31), a.rank - 1);
            const uint16_t* const row = a.a + (uint64_t(member) * a.rank + r) * a.inner;
            f32x16_t c = {};
            for (uint32_t k0 = 16 * wave; k0 < a.inner; k0 += 128) {
                const uint32_t k = k0 + 8 * (lane >> 5);
                u32x4_t av = {0, 0, 0, 0}, xv = {0, 0, 0, 0};
                if (k < a.inner) {                       // (inner is a multiple of 8)
                    av = load_row8(row + k);
                    xv = load_row8(x + k);
                }
                c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, av),
                                                            __builtin_bit_cast(bf16x8_t, xv), c, 0, 0, 0);
            }
            __syncthreads();
#pragma unroll
            for (int y = 0; y < 16; ++y)
                part[wave][8 * (y / 4) + 4 * (lane >> 5) + y % 4][lane & 31] = c[y];
            __syncthreads();
            for (uint32_t e = threadIdx.x; e < 1024; e += kThreads) {
                const uint32_t t = e / 32, q = e % 32;
                if ((match >> t & 1) == 0 || r0 + q >= a.rank) continue;
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) sum += part[w][q][t];
                a.u[uint64_t(n0 + t) * a.rank + r0 + q] =
                    static_cast<uint16_t>(pack_bf16(s * sum, 0.0f));
            }
        }
    }
}

struct AddArgs {
    const int32_t* index;
    const uint16_t* u;
    const uint16_t* b;                     // [members][outer][rank]
    uint32_t rows, outer, members, rank;
};

// B u added to a tile, for the members of each 32 rows one by one.  Where one
// member has all of them its products go straight into the tile; otherwise into
// results of their own, of which its rows take theirs: a member that holds
// infinities or NaN reaches no other's rows.
__device__ __forceinline__ void add_adapters(const AddArgs& a, uint32_t m0, uint32_t n0, Tile& c) {
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t n = n0 + 64 * (wave >> 1) + 32 * j + (lane & 31);
        const int32_t mine = n < a.rows ? a.index[n] : -1;
        const bool bad = mine >= int32_t(a.members);
        uint32_t left = uint32_t(__ballot(mine >= 0 && !bad));
        while (left != 0) {
            const int32_t member = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
            const bool match = mine == member;
            const uint32_t all = uint32_t(__ballot(match));
            left &= ~all;
            f32x16_t t[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int x = 0; x < 16; ++x) t[i][x] = all == ~0u ? c.x[i][j][x] : 0.0f;
            for (uint32_t r0 = 0; r0 < a.rank; r0 += 16) {
                const uint32_t r = r0 + 8 * (lane >> 5);
                u32x4_t uv = {0, 0, 0, 0};
                if (match && r < a.rank) uv = load<u32x4_t>(a.u + uint64_t(n) * a.rank + r);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t m = min(m0 + 128 * (wave & 1) + 32 * i + (lane & 31), a.outer - 1);
                    u32x4_t bv = {0, 0, 0, 0};
                    if (r < a.rank)
                        bv = load<u32x4_t>(a.b + (uint64_t(member) * a.outer + m) * a.rank + r);
                    t[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, bv),
                                                                   __builtin_bit_cast(bf16x8_t, uv),
                                                                   t[i], 0, 0, 0);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    c.x[i][j][x] = all == ~0u ? t[i][x] : match ? c.x[i][j][x] + t[i][x] : c.x[i][j][x];
        }
        if (__any(bad)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int x = 0; x < 16; ++x) c.x[i][j][x] = bad ? eskv::nan() : c.x[i][j][x];
        }
    }
}

struct TileArgs {
    Product p;                             // a: W, b: the rows
    AddArgs add;
    uint16_t* out;
    uint64_t out_stride;
};

__global__ __launch_bounds__(kThreads, 2) void es_adapt_tile_kernel(TileArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Place at = place_of(blockIdx.x, a.p);
    const uint32_t m0 = at.m * kTile, n0 = at.n * kTile;
    Tile c;
    product_tile<false, false>(a.p, m0, n0, 0, a.p.depth, lds, c);
    add_adapters(a.add, m0, n0, c);
    __syncthreads();
    tile_to_lds(c, lds);
    __syncthreads();
    store_rows(lds, a.out, a.out_stride, m0, a.add.outer - m0, [&](uint32_t n) {
        return n0 + n < a.add.rows ? int64_t(n0 + n) : int64_t(-1);
    });
}

}  // namespace esadapt
