// The matrix product that the head and the projections are made of: tiles of
// 256 x 256 results (128 x 128 where there are few) on the matrix unit, from operands in either order, with what
// becomes of a tile (its epilogue) as a parameter.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "kv_common.hpp"

namespace esmm {

using eskv::bf16x8_t;
using eskv::f32x16_t;
using eskv::f32x4_t;
using eskv::load;
using eskv::load_row8;
using eskv::pack_bf16;
using eskv::store;
using eskv::store_row8;
using eskv::u32x2_t;
using eskv::u32x4_t;

constexpr int kTile = 256;                 // results of a tile in either direction
constexpr int kSmallTile = 128;            //   where there are few of them
constexpr int kDepth = 64;                 // of the summed dimension, staged at a time

template <int kSize>
struct Shape {
    static constexpr int kThreads = 2 * kSize;                     // waves of kSize / 2 by 64 results
    static constexpr uint32_t kSide = kSize * kDepth * 2;          // bytes of a stage's side
    static constexpr uint32_t kPitch = kSize * 2 + 16;             // of a row of results in LDS
    static constexpr uint32_t kLds = 5 * kSide;                    // three stages of a, two of b
    static_assert(kLds >= kSize * kPitch, "a tile's results fit the stages");
};

// One operand.  Deep: element (i, k) at at[i stride + k], wide: at[k stride + i],
// i along the tile and k along the sum.  16-byte aligned, stride a multiple of 8.
struct Side {
    const uint16_t* at;
    uint64_t stride;
    uint32_t extent;                       // rows i that exist (wide: a multiple of 8)
};

// results[n][m] = sum_k a(m, k) b(n, k).  Beyond the operands' extents the last
// row is read again.  Beyond `depth` b is zero (stored to a multiple of 64), and so
// is a once it is in registers: what it holds elsewhere, infinities too, stays there.
struct Product {
    Side a, b;
    uint32_t depth;
    uint32_t m_tiles, n_tiles, splits;     // splits: of the sum, `split_depth` each
    uint32_t split_depth;                  // a multiple of 64
    const uint32_t* count;                 // rows n that exist, where the device knows it (of a
                                           //   product over them, the sum's length)
};

struct Place {
    uint32_t m, n, split;
};

// Workgroups go round the eight dies in turn: each die takes a contiguous run of
// tiles, ordered in groups of `kGroup` tiles along m over all of n, so that the
// 32 workgroups that a die runs at a time share rows of both operands in its L2.
constexpr uint32_t kGroup = 4;
__device__ __forceinline__ Place place_of(uint32_t id, const Product& p) {
    const uint32_t tiles = p.m_tiles * p.n_tiles, total = tiles * p.splits;
    const uint32_t die = id % 8, q = total / 8, r = total % 8;
    uint32_t at = die * q + (die < r ? die : r) + id / 8;
    Place x;
    x.split = at / tiles;
    at -= x.split * tiles;
    const uint32_t g = at / (kGroup * p.n_tiles);
    at -= g * kGroup * p.n_tiles;
    const uint32_t left = p.m_tiles - g * kGroup, wide = left < kGroup ? left : kGroup;
    x.n = at / wide;
    x.m = g * kGroup + at % wide;
    return x;
}

// An array from some point of it on, as the loads into LDS take it: they bring nothing from
// `bytes` on.  The point moves along the array; the lanes' offsets from it stay.  (The
// instruction's scalar offset is not for that: what the bounds check compares is the lanes'
// offsets, so with it the last row's last words would be read past the array's end.)
struct Window {
    uint64_t at;                           // an address
    uint64_t bytes;                        // from there to the array's end
    __host__ __device__ uint32_t limit() const { return bytes > 0xFFFFFFFFull ? 0xFFFFFFFFu : uint32_t(bytes); }
    __host__ __device__ void move(uint64_t step) {
        at += step;
        bytes -= bytes < step ? bytes : step;
    }
    __device__ __forceinline__ u32x4_t buffer() const {
        return u32x4_t{uint32_t(at), uint32_t(at >> 32) & 0xFFFFu, limit(), 0x00020000u};
    }
};

// 16 bytes a lane from `offset` of the lane into LDS, at byte `dst` (of the wave) + 16 lane.
// (In asm, which has no register output: the compiler would make every later read
// of LDS wait for it; m0 is a reserved register, in which it keeps nothing over a statement.)
// wait_staged() and a barrier before the data are read.
__device__ __forceinline__ void load_lds(u32x4_t buffer, uint32_t offset, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(dst), "v"(offset), "s"(buffer) : "memory");
}
__device__ __forceinline__ void wait_staged() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}
template <int n>                           // but the last n loads
__device__ __forceinline__ void wait_all_but() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(n) : "memory");
}

__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
    return uint64_t(uniform(uint32_t(x >> 32))) << 32 | uniform(uint32_t(x));
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p));   // of the shared aperture
}

// A side's way into LDS, 4 KB a wave and stage of 64 of the sum.  Deep: [kSize rows][8
// words of 16 bytes], word w of row i stored at w ^ ((i >> 1) & 7): sixteen rows' words
// of one w, which a read of an operand takes at a time, fill the banks once.
// Wide: [64][kSize / 8 words], word w of row k at w ^ (4 (k & 3) + 2 (k >> 3 & 1)): the words that
// a transposing read takes at a time, four k's and the four eight further on, do.
template <bool kWide, int kSize>
struct Stage {
    static constexpr uint32_t kWords = kSize / 8;        // of a k's row, where wide
    Window next;                           // the next stage on
    uint64_t step;                         // bytes from stage to stage
    uint32_t off[4];
    uint32_t dst;

    // Load x of a wave: the row (wide: k of a stage) and the word of it that it brings for a lane.
    static __host__ __device__ uint32_t row_of(uint32_t wave, uint32_t x, uint32_t lane) {
        return kWide ? (wave * 4 + x) * (64 / kWords) + lane / kWords : (wave * 4 + x) * 8 + (lane >> 3);
    }
    static __host__ __device__ uint32_t word_of(uint32_t wave, uint32_t x, uint32_t lane) {
        const uint32_t r = row_of(wave, x, lane);
        return kWide ? (lane % kWords) ^ ((r & 3) << 2) ^ ((r >> 3 & 1) << 1) : (lane & 7) ^ ((r >> 1) & 7);
    }

    // The side from rows i0 (< extent) and elements k0 of the sum on, up to k_end.
    static __host__ __device__ Window window(const Side& s, uint32_t i0, uint32_t k0, uint32_t k_end) {
        const uint64_t last = s.extent - 1 - i0, at = reinterpret_cast<uint64_t>(s.at);
        if constexpr (kWide)
            return Window{at + 2 * (k0 * s.stride + i0), 2 * ((k_end - 1 - k0) * s.stride + last + 1)};
        else                               // (rows end with a word)
            return Window{at + 2 * (i0 * s.stride + k0), 2 * (last * s.stride + (k_end + 7) / 8 * 8 - k0)};
    }
    // The lane's bytes from there: of rows behind the last the last one's.
    static __host__ __device__ uint32_t offset(const Side& s, uint32_t i0, uint32_t wave, uint32_t x, uint32_t lane) {
        const uint32_t last = s.extent - 1 - i0, r = row_of(wave, x, lane), w = word_of(wave, x, lane);
        if constexpr (kWide)
            return r * uint32_t(2 * s.stride) + 16 * (w < last / 8 ? w : last / 8);
        else
            return (r < last ? r : last) * uint32_t(2 * s.stride) + 16 * w;
    }
    // Of a last stage of `have` elements of the sum: of those behind them others'.
    static __host__ __device__ uint32_t last_offset(uint32_t o, uint32_t have, const Side& s, uint32_t wave,
                                                    uint32_t x, uint32_t lane) {
        const uint32_t r = row_of(wave, x, lane), w = word_of(wave, x, lane);
        if constexpr (kWide)
            return r >= have ? o - (r - (have - 1)) * uint32_t(2 * s.stride) : o;
        else
            return 8 * w >= have ? o - 16 * w : o;
    }

    __device__ __forceinline__ void init(const Side& s, uint32_t i0, uint32_t k0, uint32_t k_end,
                                         uint32_t wave, uint32_t lane) {
        dst = wave * 4096;
        const Window first = window(s, i0, k0, k_end);
        next = Window{uniform(first.at), uniform(first.bytes)};
        step = uniform(kWide ? 2 * kDepth * s.stride : 2 * kDepth);
#pragma unroll
        for (uint32_t x = 0; x < 4; ++x) off[x] = offset(s, i0, wave, x, lane);
    }

    // The next stage's bytes; load x of it, where it exists in full.
    __device__ __forceinline__ u32x4_t take() {
        const u32x4_t buffer = next.buffer();
        next.move(step);
        return buffer;
    }
    __device__ __forceinline__ void load(u32x4_t buffer, uint32_t lds, uint32_t x) const {
        load_lds(buffer, off[x], lds + dst + 1024 * x);
    }
    // Where only `have` of it exist: others are read again, and cleared in registers.
    __device__ __forceinline__ void load_last(u32x4_t buffer, uint32_t lds, uint32_t x, uint32_t have,
                                              const Side& s, uint32_t wave, uint32_t lane) const {
        const uint32_t o = last_offset(off[x], have, s, wave, x, lane);
        load_lds(buffer, o, lds + dst + 1024 * x);
    }
};

// A wave's reads of a side: block b of 16 rows from row `from`, step s of 32 of the sum.
// The operand of lane l: row l % 16 of the block, elements 8 (l / 16) .. of the step.
template <bool kWide, int kSize, int kBlocks>
struct Reader {
    uint32_t at[kWide ? kBlocks : 2];

    __device__ __forceinline__ void init(uint32_t from, uint32_t lane) {
        if constexpr (kWide) {
            const uint32_t kk = (lane & 15) >> 2, k = 8 * (lane >> 4) + kk;
#pragma unroll
            for (uint32_t b = 0; b < kBlocks; ++b) {
                const uint32_t i = from + 16 * b + 4 * (lane & 3);
                at[b] = k * (2 * kSize) + (((i >> 3) ^ (kk << 2) ^ ((lane >> 4 & 1) << 1)) << 4) + ((i & 4) << 1);
            }
        } else {
            const uint32_t i = from + (lane & 15);
#pragma unroll
            for (uint32_t s = 0; s < 2; ++s)
                at[s] = i * 128 + (((4 * s + (lane >> 4)) ^ ((i >> 1) & 7)) << 4);
        }
    }
    __device__ __forceinline__ bf16x8_t read(const uint8_t* lds, int s, int b) const {
        if constexpr (kWide) {
            typedef short i16x4_t __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) i16x4_t Shared;
            union { i16x4_t half[2]; bf16x8_t whole; } x;
#pragma unroll
            for (int t = 0; t < 2; ++t)
                x.half[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (Shared*)(lds + at[b] + 64 * kSize * s + 8 * kSize * t));
            return x.whole;
        } else {
            return *reinterpret_cast<const bf16x8_t*>(lds + at[s] + 2048 * b);
        }
    }
};

// What a wave holds of a tile: rows m kSize / 2 (wave % 2) + 16 i + 4 (lane / 16) + e in
// element e, and rows n 64 (wave / 2) + 16 j + lane % 16 (the waves' order is m first).
template <int kSize>
struct Tile {
    static constexpr int kBlocks = kSize / 32;
    f32x4_t x[kBlocks][4];
    // the first of the four rows m of block i, and the row n of block j
    static __device__ __forceinline__ uint32_t m_of(uint32_t wave, uint32_t lane, int i) {
        return kSize / 2 * (wave & 1) + 16 * i + 4 * (lane >> 4);
    }
    static __device__ __forceinline__ uint32_t n_of(uint32_t wave, uint32_t lane, int j) {
        return 64 * (wave >> 1) + 16 * j + (lane & 15);
    }
};

template <int n>
struct Count {
    static constexpr int value = n;
};

// Rows n0 .. n0 + n_have of n are there (more than the tile has count as all).  Three
// stages of a and two of b in LDS, all that it holds: while the products of a stage's first
// step are made its second's operands are read; then the stage is in registers and, once
// the next has landed, b's stage after that and a's after that again are asked for, a load
// to some products each: eight waves that ask for all of it at once wait for the loads'
// way in.  4096 rows of 5120 against 151936 (256 x 256): 4.65 ms, 1.37 PFLOP/s; 1024 of 2560
// 672 us.  Two products to a load of b and six to one of a (one each: 4.78 and 697, but with a
// wide, whose reads are twice as many, it is the faster by 3 to 5 %; a's loads in the next stage's first step 4.80 and 693); two stages of a and one product to a
// load 4.82 and 712; without loads in the loop 3.70 and 547.  The clock falls to 1.8 GHz
// at 5120 (the card's power) and stays at 2.2 at 2560.
template <bool kWideA, bool kWideB, int kSize>
__device__ __forceinline__ void product_tile(const Product& p, uint32_t m0, uint32_t n0, uint32_t n_have,
                                             uint32_t k0, uint32_t k_end, uint8_t* lds, Tile<kSize>& c) {
    constexpr int kBlocks = Tile<kSize>::kBlocks, kProducts = 4 * kBlocks;   // of a step
    constexpr uint32_t kSide = Shape<kSize>::kSide;
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c.x[i][j] = f32x4_t{0, 0, 0, 0};
    if (k0 >= k_end) return;
    Stage<kWideA, kSize> sa;
    Stage<kWideB, kSize> sb;
    sa.init(p.a, m0, k0, k_end, wave, lane);
    // (b's rows are stored, as zeros, to the end of its last stage: all of that is brought)
    sb.init(p.b, n0, k0, (k_end + kDepth - 1) / kDepth * kDepth, wave, lane);
    Reader<kWideA, kSize, kBlocks> ra;
    Reader<kWideB, kSize, 4> rb;
    ra.init(kSize / 2 * (wave & 1), lane);
    rb.init(64 * (wave >> 1), lane);
    const uint32_t lds_at = uniform(lds_address(lds));
    uint32_t at_a = 0, at_b = 3 * kSide;                 // of the stage in use
    auto issue_a = [&](uint32_t k, uint32_t at) {
        const u32x4_t buffer = sa.take();
#pragma unroll
        for (uint32_t x = 0; x < 4; ++x) {
            if (k_end - k >= kDepth)
                sa.load(buffer, lds_at + at, x);
            else
                sa.load_last(buffer, lds_at + at, x, k_end - k, p.a, wave, lane);
        }
    };
    auto issue_b = [&](uint32_t at) {                    // (always whole)
        const u32x4_t buffer = sb.take();
#pragma unroll
        for (uint32_t x = 0; x < 4; ++x) sb.load(buffer, lds_at + at, x);
    };
    // The stage after k's has landed for every wave, of a's loads those for the one after it
    // may be out.
    auto landed = [&](uint32_t k) {
        if (k + 2 * kDepth < k_end)
            wait_all_but<4>();
        else
            wait_staged();
        __builtin_amdgcn_s_barrier();
    };
    auto advance = [&]() {
        at_a = at_a == 2 * kSide ? 0 : at_a + kSide;
        at_b = 7 * kSide - at_b;
    };
    bf16x8_t a[2][kBlocks], b[2][4];
    auto read_one = [&](int s, int r) {
        if (r < 4)
            b[s][r] = rb.read(lds + at_b, s, r);
        else
            a[s][r - 4] = ra.read(lds + at_a, s, r - 4);
    };
    auto read = [&](int s) {
#pragma unroll
        for (int r = 0; r < 4 + kBlocks; ++r) read_one(s, r);
    };
    // 16 x 16 x 32 a product: at the clock that the card's power leaves it makes 1.92
    // PFLOP/s with its reads from LDS where 32 x 32 x 16 makes 1.72
    auto one = [&](int s, int y) {
        c.x[y / 4][y % 4] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s][y / 4], b[s][y % 4],
                                                                    c.x[y / 4][y % 4], 0, 0, 0);
    };
    auto multiply = [&](int s) {
#pragma unroll
        for (int y = 0; y < kProducts; ++y) one(s, y);
    };
    // the reads of a step go out one to a product, from the first on
    constexpr int kReads = (kWideA ? 2 : 1) * kBlocks + (kWideB ? 8 : 4), kMatrix = 0x8, kDsRead = 0x100;
    auto interleave = [&](auto products, auto reads) {
        constexpr int n = decltype(products)::value, m = decltype(reads)::value, each = (m + n - 1) / n;
#pragma unroll
        for (int x = 0; x < n; ++x) {
            if (x * each < m) __builtin_amdgcn_sched_group_barrier(kDsRead, each, 0);
            __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    issue_a(k0, 0);
    issue_b(3 * kSide);
    if (k0 + kDepth < k_end) {
        issue_a(k0 + kDepth, kSide);
        issue_b(4 * kSide);
    }
    if (k0 + 2 * kDepth < k_end) {
        issue_a(k0 + 2 * kDepth, 2 * kSide);
        wait_all_but<12>();
    } else if (k0 + kDepth < k_end) {
        wait_all_but<8>();
    } else {
        wait_staged();
    }
    __builtin_amdgcn_s_barrier();
    if (64 * (wave >> 1) >= n_have) {                    // a wave without rows only stages
        for (uint32_t k = k0; k + kDepth < k_end; k += kDepth) {
            landed(k);
            if (k + 2 * kDepth < k_end) issue_b(at_b);
            if (k + 3 * kDepth < k_end) issue_a(k + 3 * kDepth, at_a);
            advance();
        }
        return;
    }
    read(0);
    auto first_step = [&]() {
        read(1);
        multiply(0);
        interleave(Count<kProducts>{}, Count<kReads>{});
    };
    uint32_t k = k0;
    for (; k + 4 * kDepth <= k_end; k += kDepth) {       // the stages to ask for are whole
        first_step();
        // all of the stage is in registers, and the next has landed
        wait_all_but<4>();
        __builtin_amdgcn_s_barrier();
        const uint32_t old_a = lds_at + at_a, old_b = lds_at + at_b;
        advance();
        const u32x4_t ba = sa.take(), bb = sb.take();
        // products to a load of b and of a, and operands read to one of a (wide: behind them all)
        constexpr int kToB = kWideA ? 1 : kProducts / 16, kToA = kWideA ? 1 : 3 * kProducts / 16;
        constexpr int kRow = (4 + kBlocks) / 4, kLeft = kProducts - 4 * kToB - 4 * kToA;
#pragma unroll
        for (uint32_t x = 0; x < 4; ++x) {
            sb.load(bb, old_b, x);
#pragma unroll
            for (int y = 0; y < kToB; ++y) one(1, kToB * x + y);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (uint32_t x = 0; x < 4; ++x) {
            sa.load(ba, old_a, x);
            if constexpr (!kWideA) {
#pragma unroll
                for (int r = kRow * x; r < kRow * int(x + 1); ++r) read_one(0, r);
            }
#pragma unroll
            for (int y = 0; y < kToA; ++y) one(1, 4 * kToB + kToA * x + y);
            if constexpr (!kWideA) interleave(Count<kToA>{}, Count<kReads / 4>{});
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (kWideA) {
            read(0);
#pragma unroll
            for (int y = kProducts - kLeft; y < kProducts; ++y) one(1, y);
            interleave(Count<kLeft>{}, Count<kReads>{});
        }
    }
    for (; k + kDepth < k_end; k += kDepth) {
        first_step();
        landed(k);
        if (k + 2 * kDepth < k_end) issue_b(at_b);
        if (k + 3 * kDepth < k_end) issue_a(k + 3 * kDepth, at_a);
        advance();
        read(0);
        multiply(1);
        interleave(Count<kProducts>{}, Count<kReads>{});
    }
    const uint32_t have = k_end - k;
    // of a's operands of step s, what lies within the sum
    auto keep = [&](int s) {
        const int left = int(have) - int(32 * s + 8 * (lane >> 4));   // of the lane's eight
        u32x4_t kept;
#pragma unroll
        for (int y = 0; y < 4; ++y) kept[y] = left >= 2 * y + 2 ? 0xFFFFFFFFu : left == 2 * y + 1 ? 0xFFFFu : 0u;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i)
            a[s][i] = __builtin_bit_cast(bf16x8_t, __builtin_bit_cast(u32x4_t, a[s][i]) & kept);
    };
    if (have < kDepth) keep(0);
    read(1);
    multiply(0);
    interleave(Count<kProducts>{}, Count<kReads>{});
    if (have < kDepth) keep(1);
    multiply(1);
}

// f(x, m, n): the words of four results, rows m .. m + 3 and row n of the tile.
template <int kSize, class F>
__device__ __forceinline__ void for_words(const Tile<kSize>& c, F f) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < Tile<kSize>::kBlocks; ++i)
            f(c.x[i][j], c.m_of(wave, lane, i), c.n_of(wave, lane, j));
}

// Results as bf16 (RNE) into LDS, [n][m]; all waves have read their last operands.
template <int kSize>
__device__ __forceinline__ void tile_to_lds(const Tile<kSize>& c, uint8_t* lds) {
    for_words(c, [&](const f32x4_t& x, uint32_t m, uint32_t n) {
        *reinterpret_cast<u32x2_t*>(lds + n * Shape<kSize>::kPitch + 2 * m) =
            u32x2_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    });
}

// Rows of the tile from LDS to `out` (bf16, `stride` elements from row to row): row n
// to row_of(n), which is negative for a row that is not written; m_have
// results of each.
template <int kSize, class F>
__device__ __forceinline__ void store_rows(const uint8_t* lds, uint16_t* out, uint64_t stride,
                                           uint32_t m0, uint32_t m_have, F row_of) {
    constexpr uint32_t kWords = kSize / 8;
    const uint32_t word = threadIdx.x % kWords;
#pragma unroll 4
    for (uint32_t n = threadIdx.x / kWords; n < kSize; n += Shape<kSize>::kThreads / kWords) {
        const int64_t row = row_of(n);
        if (row < 0 || 8 * word >= m_have) continue;
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(lds + n * Shape<kSize>::kPitch + 16 * word);
        uint16_t* const to = out + uint64_t(row) * stride + m0 + 8 * word;
        if (8 * word + 8 <= m_have) {
            store_row8(to, v);
        } else {
            for (uint32_t e = 0; 8 * word + e < m_have; ++e)
                store<uint16_t>(to + e, static_cast<uint16_t>(v[e / 2] >> (16 * (e % 2))));
        }
    }
}

}  // namespace esmm
