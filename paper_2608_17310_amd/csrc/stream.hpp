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

    // `bytes` from `base` on; what lies beyond them is not fetched
    static __device__ __forceinline__ u32x4_t buffer(uint64_t base, uint64_t bytes) {
        return u32x4_t{uint32_t(base), uint32_t(base >> 32) & 0xFFFFu,
                       bytes > 0xFFFFFFFFull ? 0xFFFFFFFFu : uint32_t(bytes), 0x00020000u};
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
        for (int y = 0; y < kWLoads; ++y) {
            const uint32_t i = (wave * kWLoads + y) * 8 + (lane >> 3);
            w_off[y] = i * uint32_t(2 * a.w_stride) + 16 * ((lane & 7) ^ ((i >> 1) & 7));
        }
#pragma unroll
        for (int y = 0; y < kXLoads; ++y) {
            const uint32_t i = ((wave * kXLoads + y) * 8 + (lane >> 3)) % kTokens;
            x_off[y] = i * uint32_t(2 * a.x_stride) + 16 * ((lane & 7) ^ ((i >> 1) & 7));
        }
        uint32_t w_at[2], x_at[2];         // operands of the two steps of 64
#pragma unroll
        for (uint32_t s = 0; s < 2; ++s) {
            const uint32_t i = lane & 15, word = ((4 * s + (lane >> 4)) ^ ((i >> 1) & 7)) << 4;
            w_at[s] = (16 * kBlocks * wave + i) * 128 + word;
            x_at[s] = kXAt + i * 128 + word;
        }
        const uint32_t lds_at = uniform(lds_address(lds));
        // rows beyond the share and beyond x's are beyond the buffers
        auto share = [&](uint32_t row) {
            return buffer(uniform(reinterpret_cast<uint64_t>(a.w) + 2 * (row * a.w_stride)),
                          uniform(2 * (uint64_t(end - row - 1) * a.w_stride + a.width)));
        };
        const u32x4_t xb = buffer(uniform(reinterpret_cast<uint64_t>(a.x)),
                                  uniform(2 * (uint64_t(a.rows - 1) * a.x_stride + a.width)));
        u32x4_t wb = share(begin);
        uint32_t next_slot = lds_at, issued = 0, next_k = 0, next_row = begin;
        auto issue = [&]() {
#pragma unroll
            for (int u = 0; u < kSub; ++u) {
                const uint32_t to = next_slot + u * kPart;
#pragma unroll
                for (int y = 0; y < kWLoads; ++y)
                    load_lds(wb, w_off[y], next_k, to + (wave * kWLoads + y) * 1024);
#pragma unroll
                for (int y = 0; y < kXLoads; ++y)
                    load_lds(xb, x_off[y], next_k, to + kXAt + (wave * kXLoads + y) % (kTokens / 8) * 1024);
                next_k += 2 * kDepth;
            }
            ++issued;
            next_slot = next_slot + kStage == lds_at + kBytes ? lds_at : next_slot + kStage;
            if (next_k >= 2 * a.width) {   // on to the next rows
                next_k = 0;
                next_row += kTall;
                if (next_row < end) wb = share(next_row);
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
