// Products of a large matrix with up to 128 rows: bound by the matrix's bytes, and by
// how often the rows are read beside it.  A workgroup's share of the matrix passes
// through a ring of stages in LDS without passing registers, several stages ahead,
// and the rows' stages beside it serve all of its waves.
#pragma once

#include "mm_tile.hpp"

namespace esstream {

using namespace esmm;

constexpr uint32_t kRows = 128;            // at most

struct StreamArgs {
    const uint16_t *w, *x;                 // rows of 16-byte words: bases, strides and width
    uint64_t w_stride, x_stride;
    uint32_t w_rows, rows, width;
    uint32_t share;                        // rows of the matrix for a workgroup, a multiple of 16
};

// As many stages as LDS holds, and as a wave's loads can be counted.
constexpr int stages_for(int tall, int tokens, int sub, int loads) {
    const int held = 163840 / (sub * (tall + tokens) * 128), counted = 63 / loads + 1;
    return held < counted ? held : counted;
}

template <int kOutstanding>
__device__ __forceinline__ void wait_stage() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kOutstanding) : "memory");
}

// kWaves waves of kBlocks blocks of 16 rows of the matrix, kTokens rows beside them.
// A stage is 64 kSub of the sum, each 64 as rows of 8 words, swizzled as in a tile's
// stages.
template <int kWaves, int kBlocks, int kTokens, int kSub, int kStages>
struct Stream {
    static constexpr uint32_t kTall = 16 * kBlocks * kWaves, kLength = kDepth * kSub;
    static constexpr int kWLoads = 2 * kBlocks;                                   // of a wave and 64
    static constexpr int kXLoads = (kTokens / 8 + kWaves - 1) / kWaves;
    static constexpr int kLoads = kSub * (kWLoads + kXLoads);
    static constexpr uint32_t kXAt = kTall * 128, kPart = kXAt + kTokens * 128, kStage = kSub * kPart;
    static constexpr uint32_t kBytes = kStages * kStage;
    static constexpr int kCols = kTokens / 16;
    static_assert(kBytes <= 163840 && (kStages - 1) * kLoads < 64, "fits");

    f32x4_t c[kBlocks][kCols];             // rows 4 (lane / 16) .. of a block, column lane % 16

    // Rows `row` .. of a side that has those before `end`: rows from there on are not fetched
    // (or, where rows overlap, are bytes that are there).
    static __host__ __device__ Window window(const uint16_t* side, uint64_t stride, uint32_t row,
                                             uint32_t end, uint32_t width) {
        return Window{reinterpret_cast<uint64_t>(side) + 2 * (row * stride),
                      2 * (uint64_t(end - row - 1) * stride + width)};
    }
    // The lane's bytes from there, of rows 8 y .. of a stage.
    static __host__ __device__ uint32_t offset(uint32_t y, uint32_t lane, uint64_t stride) {
        const uint32_t i = 8 * y + (lane >> 3);
        return i * uint32_t(2 * stride) + 16 * ((lane & 7) ^ ((i >> 1) & 7));
    }

    // done(row0, end): c holds rows row0 + 16 kBlocks wave .. of those before `end`.
    template <class F>
    __device__ __forceinline__ void run(const StreamArgs& a, uint8_t* lds, F done) {
        const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
        const uint32_t begin = blockIdx.x * a.share, end = min(begin + a.share, a.w_rows);
        if (begin >= end) return;
        const uint32_t stages = (a.width + kLength - 1) / kLength;
        const uint32_t total = (end - begin + kTall - 1) / kTall * stages;
        uint32_t w_off[kWLoads], x_off[kXLoads];
#pragma unroll
        for (int y = 0; y < kWLoads; ++y) w_off[y] = offset(wave * kWLoads + y, lane, a.w_stride);
#pragma unroll
        for (int y = 0; y < kXLoads; ++y)
            x_off[y] = offset((wave * kXLoads + y) % (kTokens / 8), lane, a.x_stride);
        uint32_t w_at[2], x_at[2];         // operands of the two steps of 64
#pragma unroll
        for (uint32_t s = 0; s < 2; ++s) {
            const uint32_t i = lane & 15, word = ((4 * s + (lane >> 4)) ^ ((i >> 1) & 7)) << 4;
            w_at[s] = (16 * kBlocks * wave + i) * 128 + word;
            x_at[s] = kXAt + i * 128 + word;
        }
        const uint32_t lds_at = uniform(lds_address(lds));
        auto from = [&](const uint16_t* side, uint64_t stride, uint32_t row, uint32_t stop) {
            const Window w = window(side, stride, row, stop, a.width);
            return Window{uniform(w.at), uniform(w.bytes)};
        };
        const Window x_start = from(a.x, a.x_stride, 0, a.rows);
        Window ww = from(a.w, a.w_stride, begin, end), xw = x_start;
        uint32_t next_slot = lds_at, issued = 0, next_k = 0, next_row = begin;
        auto issue = [&]() {
#pragma unroll
            for (int u = 0; u < kSub; ++u) {
                const uint32_t to = next_slot + u * kPart;
                const u32x4_t wb = ww.buffer(), xb = xw.buffer();
#pragma unroll
                for (int y = 0; y < kWLoads; ++y)
                    load_lds(wb, w_off[y], to + (wave * kWLoads + y) * 1024);
#pragma unroll
                for (int y = 0; y < kXLoads; ++y)
                    load_lds(xb, x_off[y], to + kXAt + (wave * kXLoads + y) % (kTokens / 8) * 1024);
                ww.move(2 * kDepth);
                xw.move(2 * kDepth);
            }
            next_k += kLength;
            ++issued;
            next_slot = next_slot + kStage == lds_at + kBytes ? lds_at : next_slot + kStage;
            if (next_k >= a.width) {       // on to the next rows
                next_k = 0;
                next_row += kTall;
                if (next_row < end) ww = from(a.w, a.w_stride, next_row, end);
                xw = x_start;
            }
        };
        auto clear = [&]() {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int j = 0; j < kCols; ++j) c[b][j] = f32x4_t{0, 0, 0, 0};
        };
        clear();
        while (issued < kStages - 1 && issued < total) issue();
        uint32_t slot = 0, k = 0, row0 = begin;
        for (uint32_t q = 0; q < total; ++q) {
            if (q + kStages - 1 <= total)
                wait_stage<(kStages - 2) * kLoads>();
            else
                wait_stage<0>();
            __builtin_amdgcn_s_barrier();  // the stage is there, and all have left the last one
            bf16x8_t wv[2 * kSub][kBlocks], xv[2 * kSub][kCols];
#pragma unroll
            for (int s = 0; s < 2 * kSub; ++s) {
                const uint8_t* const at = lds + slot + s / 2 * kPart;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
                    wv[s][b] = *reinterpret_cast<const bf16x8_t*>(at + w_at[s % 2] + 2048 * b);
#pragma unroll
                for (int j = 0; j < kCols; ++j)
                    xv[s][j] = *reinterpret_cast<const bf16x8_t*>(at + x_at[s % 2] + 2048 * j);
            }
            if (issued < total) issue();
            if (k + kLength > a.width) {   // the sum ends in this stage
#pragma unroll
                for (int s = 0; s < 2 * kSub; ++s)
                    if (k + 32 * s + 8 * (lane >> 4) >= a.width) {
#pragma unroll
                        for (int b = 0; b < kBlocks; ++b) wv[s][b] = bf16x8_t{};
#pragma unroll
                        for (int j = 0; j < kCols; ++j) xv[s][j] = bf16x8_t{};
                    }
            }
#pragma unroll
            for (int s = 0; s < 2 * kSub; ++s)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int j = 0; j < kCols; ++j)
                        c[b][j] =
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[s][b], xv[s][j], c[b][j], 0, 0, 0);
            slot = slot + kStage == kBytes ? 0 : slot + kStage;
            k += kLength;
            if (k >= a.width) {
                done(row0, end);
                clear();
                k = 0;
                row0 += kTall;
            }
        }
    }
};

}  // namespace esstream
