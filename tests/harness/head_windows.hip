// Replays on the host which bytes the loads into LDS of ring.hpp, stream.hpp and mm_tile.hpp
// address, lane by lane, and what the buffers' bounds check lets through: all of it
// lies in the array, and all of the array's words are there.  The check is taken as the
// compiler's documentation of raw buffer loads has it: a lane's offset against
// the buffer's bytes.  Prints "ok" and exits 0, or names the first failures and exits 1.
#include "../../paper_2608_17310_amd/csrc/ring.hpp"
#include "../../paper_2608_17310_amd/csrc/stream.hpp"

#include <algorithm>
#include <cstdio>
#include <random>
#include <set>

namespace {

int g_failures = 0;

struct Side {
    uint64_t stride;
    uint32_t rows, width;                  // elements; the array ends with its last row
    uint64_t start = uint64_t(1) << 40;
    const uint16_t* at() const { return reinterpret_cast<const uint16_t*>(start); }
    uint64_t end() const { return start + 2 * ((rows - 1) * stride + width); }
};

void fail(const char* what, const Side& s, uint32_t row0, uint32_t k) {
    if (g_failures++ < 20)
        std::printf("FAIL: %s: %u rows of %u, stride %llu, rows from %u, sum from %u\n", what, s.rows, s.width,
                    static_cast<unsigned long long>(s.stride), row0, k);
}

// One load of a wave: rows i0 .. i0 + 7 from row0 on, elements k .. k + 63 of the sum.
template <class Offset>
void replay(const Side& s, const esmm::Window& w, Offset offset, uint32_t row0, uint32_t i0, uint32_t stop,
            uint32_t k) {
    for (uint32_t lane = 0; lane < 64; ++lane) {
        const uint32_t off = offset(lane);
        const bool fetched = off < w.limit();
        if (fetched && (w.at + off < s.start || w.at + off + 16 > s.end())) fail("outside", s, row0, k);
        const uint32_t i = i0 + (lane >> 3), e = k + 8 * ((lane & 7) ^ ((i >> 1) & 7));
        if (row0 + i >= stop || e >= s.width) continue;
        if (!fetched) fail("missing", s, row0, k);
        if (w.at + off != s.start + 2 * ((row0 + i) * s.stride + e)) fail("another word", s, row0, k);
    }
}

template <int kBlocks, int kCols, int kParts>
void ring(const Side& s, uint32_t waves) {
    using R = esring::Ring<kBlocks, kCols, kParts>;
    for (uint32_t row0 = 0; row0 < s.rows; row0 += 16 * kBlocks)
        for (uint32_t first = 0; first < waves; ++first) {
            if (first * 64 >= s.width) break;
            esmm::Window w = R::window(s.at(), s.stride, s.rows, row0, s.width, first);
            for (uint32_t k = 64 * first; k < s.width; k += 64 * waves) {
                for (uint32_t y = 0; y < 2 * kBlocks; ++y)
                    replay(s, w, [&](uint32_t lane) { return R::offset(y, lane, s.stride); }, row0, 8 * y, s.rows,
                           k);
                w.move(waves * 128);
            }
        }
}

template <int kWaves, int kBlocks, int kTokens, int kSub, int kStages>
void stream(const Side& s, uint32_t share) {
    using S = esstream::Stream<kWaves, kBlocks, kTokens, kSub, kStages>;
    for (uint32_t begin = 0; begin < s.rows; begin += share) {
        const uint32_t end = std::min(begin + share, s.rows);
        for (uint32_t row = begin; row < end; row += S::kTall) {
            esmm::Window w = S::window(s.at(), s.stride, row, end, s.width);
            for (uint32_t k0 = 0; k0 < s.width; k0 += S::kLength)
                for (uint32_t u = 0; u < kSub; ++u) {
                    for (uint32_t y = 0; y < kWaves * S::kWLoads; ++y)
                        replay(s, w, [&](uint32_t lane) { return S::offset(y, lane, s.stride); }, row, 8 * y, end,
                               k0 + 64 * u);
                    w.move(128);
                }
        }
    }
}

// A tile's side, stage by stage.  Of a matrix (`whole` false) a last stage brings what there is;
// packed rows (`whole`) are stored to the end of their last stage, and all of it is brought.
template <bool kWide, int kSize>
void tile(uint32_t rows, uint32_t depth, uint64_t stride, uint32_t splits, bool whole) {
    using S = esmm::Stage<kWide, kSize>;
    const uint64_t start = uint64_t(1) << 40;
    const uint32_t stored = whole ? (depth + 63) / 64 * 64 : depth;
    const uint64_t end = start + 2 * (kWide ? (stored - 1) * stride + rows : (rows - 1) * stride + stored);
    const esmm::Side s{reinterpret_cast<const uint16_t*>(start), stride, rows};
    const uint32_t part = ((depth + splits - 1) / splits + 63) / 64 * 64;
    auto bad = [&](const char* what, uint32_t i0, uint32_t k) {
        if (g_failures++ < 20)
            std::printf("FAIL: tile %s: wide %d, %d, %u rows, sum of %u, stride %llu, from %u, %u\n", what, int(kWide),
                        kSize, rows, depth, static_cast<unsigned long long>(stride), i0, k);
    };
    for (uint32_t i0 = 0; i0 < rows; i0 += kSize)
        for (uint32_t k0 = 0; k0 < depth; k0 += part) {
            const uint32_t k_end = std::min(depth, k0 + part), to = whole ? (k_end + 63) / 64 * 64 : k_end;
            esmm::Window w = S::window(s, i0, k0, to);
            for (uint32_t k = k0; k < k_end; k += 64) {
                const uint32_t have = std::min(64u, to - k);
                for (uint32_t wave = 0; wave < kSize / 32; ++wave)
                    for (uint32_t x = 0; x < 4; ++x)
                        for (uint32_t lane = 0; lane < 64; ++lane) {
                            uint32_t off = S::offset(s, i0, wave, x, lane);
                            if (have < 64) off = S::last_offset(off, have, s, wave, x, lane);
                            const bool fetched = off < w.limit();
                            if (!fetched) bad("missing", i0, k);          // (every load is within the array)
                            if (w.at + off < start || w.at + off + 16 > end) bad("outside", i0, k);
                            const uint32_t r = S::row_of(wave, x, lane), e = 8 * S::word_of(wave, x, lane);
                            if (kWide ? i0 + e >= rows || r >= have : i0 + r >= rows || e >= have) continue;
                            const uint64_t want = kWide ? (k + r) * stride + i0 + e : (i0 + r) * stride + k + e;
                            if (w.at + off != start + 2 * want) bad("another word", i0, k);
                        }
                w.move(kWide ? 128 * stride : 128);
            }
        }
}

}  // namespace

int main() {
    std::mt19937_64 rng(1);
    for (int trial = 0; trial < 300; ++trial) {
        Side s;
        s.width = 8 * uint32_t(1 + rng() % (trial % 3 == 0 ? 9 : 90));
        s.rows = 1 + uint32_t(rng() % (trial % 2 ? 12 : 150));
        // rows side by side, apart, and overlapping
        const uint64_t strides[] = {s.width, s.width + 8 * (rng() % 20), 8, 8 * (1 + rng() % (s.width / 8))};
        s.stride = strides[rng() % 4];
        ring<1, 2, 3>(s, 8);
        ring<2, 4, 1>(s, 8);
        stream<3, 2, 32, 1, 4>(s, 16 * (1 + uint32_t(rng() % 9)));
        stream<5, 1, 64, 2, 3>(s, 16 * (1 + uint32_t(rng() % 9)));
    }
    for (int trial = 0; trial < 60; ++trial) {
        const uint32_t rows = 1 + uint32_t(rng() % 600), depth = 8 * uint32_t(1 + rng() % 70);
        const uint32_t wide = (rows + 7) / 8 * 8, splits = 1 + uint32_t(rng() % 3), any = 1 + uint32_t(rng() % 500);
        tile<false, 256>(rows, depth, depth + 8 * (rng() % 3), splits, false);
        tile<false, 128>(rows, depth, depth, splits, false);
        tile<true, 256>(wide, any, wide + 8 * (rng() % 3), splits, false);
        tile<true, 128>(wide, any, wide, splits, false);
        // packed rows, rows of gradients of logits, and both across the sum
        tile<false, 256>(rows, any, (any + 63) / 64 * 64, splits, true);
        tile<false, 128>(rows, any, (any + 255) / 256 * 256, splits, true);
        tile<true, 256>(wide, any, wide, splits, true);
        tile<true, 128>(wide, any, (wide + 255) / 256 * 256, splits, true);
    }
    // a matrix beyond 2^32 bytes
    Side s{uint64_t(1) << 22, 700, 65536};
    ring<2, 1, 3>(s, 8);
    if (g_failures == 0) std::printf("ok\n");
    return g_failures == 0 ? 0 : 1;
}
