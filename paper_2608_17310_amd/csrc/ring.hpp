// Products of a matrix with few rows where a workgroup has only some rows of the
// matrix: its waves share their sum.  Each wave streams its own parts of the sum
// through a ring in LDS of its own, so that no wave waits for another before the end.
#pragma once

#include "few.hpp"
#include "mm_tile.hpp"

namespace esring {

using namespace esmm;
using esfew::FewArgs;

template <int kOutstanding>
__device__ __forceinline__ void wait_part() {
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(kOutstanding) : "memory");
}

// kBlocks blocks of 16 rows of the matrix, kCols of 16 rows beside it, in parts of
// 64 of the sum: rows of 8 words, swizzled as in a tile's stages.  (Loaded straight
// into the matrix unit's operands, adjacent lanes' words belong to different rows,
// and a load takes four times as long: 1 row of 5120 beside 5120 x 5120.)
template <int kBlocks, int kCols, int kParts>
struct Ring {
    static constexpr uint32_t kXAt = kBlocks * 2048, kPart = (kBlocks + kCols) * 2048;
    static constexpr uint32_t kBytes = kParts * kPart;   // of a wave
    static constexpr int kLoads = 2 * (kBlocks + kCols);
    static_assert(kParts * kLoads < 64, "the loads on their way can be counted");

    f32x4_t c[kBlocks][kCols];             // rows 4 (lane / 16) .. of a block, column lane % 16

    // Rows row0 .. of a side of `rows`, from part `first` of the sum on.  Rows behind the last are
    // not fetched (or, where rows overlap, are bytes that are there).
    static __host__ __device__ Window window(const uint16_t* side, uint64_t stride, uint32_t rows,
                                             uint32_t row0, uint32_t width, uint32_t first) {
        Window w{reinterpret_cast<uint64_t>(side) + 2 * (row0 * stride),
                 2 * ((rows - 1 - row0) * stride + width)};
        w.move(uint64_t(first) * (2 * kDepth));
        return w;
    }
    // Load y of a part: the lane's bytes from there.
    static __host__ __device__ uint32_t offset(uint32_t y, uint32_t lane, uint64_t stride) {
        const uint32_t i = 8 * y + (lane >> 3);
        return i * uint32_t(2 * stride) + 16 * ((lane & 7) ^ ((i >> 1) & 7));
    }

    // Rows row0 .. of the matrix (row0 < a.w_rows), parts `first`, first + every, ...; `lds`
    // are the wave's own bytes.
    __device__ __forceinline__ void run(const FewArgs& a, uint32_t row0, uint32_t first, uint32_t every,
                                        uint8_t* lds) {
        const uint32_t lane = threadIdx.x & 63;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int j = 0; j < kCols; ++j) c[b][j] = f32x4_t{0, 0, 0, 0};
        const uint32_t parts = (a.width + kDepth - 1) / kDepth;
        if (first >= parts) return;
        const uint32_t count = (parts - first + every - 1) / every;
        Window ww = window(a.w, a.w_stride, a.w_rows, row0, a.width, first);
        Window xw = window(a.x, a.x_stride, a.rows, 0, a.width, first);
        ww = Window{uniform(ww.at), uniform(ww.bytes)};
        xw = Window{uniform(xw.at), uniform(xw.bytes)};
        uint32_t w_off[2 * kBlocks], x_off[2 * kCols];
#pragma unroll
        for (uint32_t y = 0; y < 2 * kBlocks || y < 2 * kCols; ++y) {
            if (y < 2 * kBlocks) w_off[y] = offset(y, lane, a.w_stride);
            if (y < 2 * kCols) x_off[y] = offset(y, lane, a.x_stride);
        }
        uint32_t at[2];                    // operands of the two steps
#pragma unroll
        for (uint32_t s = 0; s < 2; ++s) {
            const uint32_t i = lane & 15;
            at[s] = i * 128 + (((4 * s + (lane >> 4)) ^ ((i >> 1) & 7)) << 4);
        }
        const uint32_t lds_at = uniform(lds_address(lds));
        uint32_t next = first, next_slot = 0;
        auto issue = [&]() {
            const u32x4_t wb = ww.buffer(), xb = xw.buffer();
            const uint32_t to = lds_at + next_slot;
#pragma unroll
            for (int y = 0; y < 2 * kBlocks; ++y) load_lds(wb, w_off[y], to + 1024 * y);
#pragma unroll
            for (int y = 0; y < 2 * kCols; ++y) load_lds(xb, x_off[y], to + kXAt + 1024 * y);
            ww.move(every * (2 * kDepth));
            xw.move(every * (2 * kDepth));
            next += every;
            next_slot = next_slot + kPart == kBytes ? 0 : next_slot + kPart;
        };
        for (int i = 0; i < kParts; ++i)
            if (next < parts) issue();
        uint32_t slot = 0, p = first;
        for (uint32_t i = 0; i < count; ++i, p += every) {
            if (i + kParts <= count)
                wait_part<(kParts - 1) * kLoads>();
            else
                wait_part<0>();
            bf16x8_t w[2][kBlocks], x[2][kCols];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
                    w[s][b] = *reinterpret_cast<const bf16x8_t*>(lds + slot + at[s] + 2048 * b);
#pragma unroll
                for (int j = 0; j < kCols; ++j)
                    x[s][j] = *reinterpret_cast<const bf16x8_t*>(lds + slot + kXAt + at[s] + 2048 * j);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the part is in registers
            if (next < parts) issue();
            if ((p + 1) * kDepth > a.width) {                    // the sum ends in this part
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (p * kDepth + 32 * s + 8 * (lane >> 4) >= a.width) {
#pragma unroll
                        for (int b = 0; b < kBlocks; ++b) w[s][b] = bf16x8_t{};
#pragma unroll
                        for (int j = 0; j < kCols; ++j) x[s][j] = bf16x8_t{};
                    }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int j = 0; j < kCols; ++j)
                        c[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[s][b], x[s][j], c[b][j], 0, 0, 0);
            slot = slot + kPart == kBytes ? 0 : slot + kPart;
        }
    }
};

}  // namespace esring
