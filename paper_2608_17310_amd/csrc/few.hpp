// Products of a large matrix with at most 64 rows: bound by the matrix's bytes.
// Waves stream it from memory into the matrix unit's operands, with no LDS on the
// way; waves of a workgroup share a block's sum where there are few blocks.
// For rows of any alignment: those that start at words of 16 bytes come through LDS, where
// the loads of adjacent lanes belong to one row.
#pragma once

#include "mm_tile.hpp"

namespace esfew {

using namespace esmm;

constexpr uint32_t kRows = 64;             // at most
constexpr uint32_t kWaves = 8;             // of a workgroup

struct FewArgs {
    const uint16_t* w;                     // any alignment to 2 bytes
    const uint16_t* x;
    uint64_t w_stride, x_stride;
    uint32_t w_rows, rows, width;
    uint32_t slices;                       // 1, 2, 4 or 8 waves share a block's sum
};

// Elements k .. k + 7 of a row, zeros from `width` on.
__device__ __forceinline__ u32x4_t load_part(const uint16_t* row, uint32_t k, uint32_t width) {
    if (k + 8 <= width) return load_row8(row + k);
    u32x4_t v = {0, 0, 0, 0};
    for (uint32_t e = 0; k + e < width; ++e)
        v[e / 2] |= uint32_t(load<uint16_t>(row + k + e)) << (16 * (e % 2));
    return v;
}

// The operand of lane l of a block of 16 rows: row l % 16, elements 8 (l / 16) .. of a
// step of 32.  The result: column (a row of x) l % 16, rows 4 (l / 16) .. + 3.
// kSteps steps are on their way at a time, and as many behind them.
template <int kBlocks, int kCols, int kSteps>
struct Few {
    f32x4_t c[kBlocks][kCols];
    const uint16_t *wp[kBlocks], *xp[kCols];

    struct Words {
        u32x4_t w[kSteps][kBlocks], x[kSteps][kCols];
    };
    __device__ __forceinline__ void fetch(Words& q, uint32_t k) const {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) q.w[s][b] = load_row8(wp[b] + k + 32 * s);
#pragma unroll
            for (int j = 0; j < kCols; ++j) q.x[s][j] = load_row8(xp[j] + k + 32 * s);
        }
    }
    __device__ __forceinline__ void multiply(const u32x4_t (&w)[kBlocks], const u32x4_t (&x)[kCols]) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int j = 0; j < kCols; ++j)
                c[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w[b]),
                                                                  __builtin_bit_cast(bf16x8_t, x[j]),
                                                                  c[b][j], 0, 0, 0);
    }
    __device__ __forceinline__ void multiply(const Words& q) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) multiply(q.w[s], q.x[s]);
    }

    // Rows row0 .. of the matrix, elements k0 .. k1 of the sum (k0 a multiple of 32).
    __device__ __forceinline__ void run(const FewArgs& a, uint32_t row0, uint32_t k0, uint32_t k1) {
        const uint32_t lane = threadIdx.x & 63, at = 8 * (lane >> 4);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
            wp[b] = a.w + uint64_t(min(row0 + 16 * b + (lane & 15), a.w_rows - 1)) * a.w_stride + at;
#pragma unroll
        for (int j = 0; j < kCols; ++j)
            xp[j] = a.x + uint64_t(min(16 * j + (lane & 15), a.rows - 1)) * a.x_stride + at;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int j = 0; j < kCols; ++j) c[b][j] = f32x4_t{0, 0, 0, 0};
        // the waves of a block take groups of 128 by turns: together they read its rows in order
        constexpr uint32_t kGroup = 32 * kSteps;
        const uint32_t step = kGroup * a.slices;
        uint32_t k = k0;
        if (k + kGroup <= k1) {
            Words q[2];
            fetch(q[0], k);
            for (; k + 2 * step + kGroup <= k1; k += 2 * step) {
                fetch(q[1], k + step);
                multiply(q[0]);
                fetch(q[0], k + 2 * step);
                multiply(q[1]);
            }
            if (k + step + kGroup <= k1) {
                fetch(q[1], k + step);
                multiply(q[0]);
                multiply(q[1]);
                k += 2 * step;
            } else {
                multiply(q[0]);
                k += step;
            }
        }
        if (k >= k1) return;
        for (; k < k1; k += 32) {
            u32x4_t w[kBlocks], x[kCols];
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) w[b] = load_part(wp[b] - at, k + at, k1);
#pragma unroll
            for (int j = 0; j < kCols; ++j) x[j] = load_part(xp[j] - at, k + at, k1);
            multiply(w, x);
        }
    }
};

// Where a wave works: the first row of its blocks and its first group of the sum.
template <int kBlocks, int kSteps>
struct Part {
    uint32_t wave, group, slice, row0, k0, k1;
    __device__ __forceinline__ explicit Part(const FewArgs& a) {
        wave = uniform(threadIdx.x >> 6);
        slice = wave % a.slices;
        group = wave / a.slices;
        row0 = (blockIdx.x * (kWaves / a.slices) + group) * 16 * kBlocks;
        k0 = slice * 32 * kSteps;
        k1 = a.width;
    }
};

}  // namespace esfew
