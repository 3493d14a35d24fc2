// Appending to the cache and reading it back.
//
// Both move every byte once and compute little: they are bound by memory, and at
// few tokens by latency.  A workgroup takes 64 tokens and one head: a
// query head (normalise, rotate, store), or a key head with its value head.
// D / 8 lanes hold a row, 8 elements (one 16-byte access) each, so a norm is a
// sum over neighbouring lanes and a rotation's other half an exchange with the
// lane rot / 16 away (the halves' pairing) or nothing (the adjacent pairing).
//
// Values are stored by dimension: a workgroup turns its 64 tokens in LDS and
// writes runs of tokens.  Runs are cut where the slots' 16-byte words are: the
// LDS columns are shifted by the first slot's place in its word, so that a word
// whose tokens lie in consecutive slots (a prompt, wherever its page list jumps)
// is read from LDS and written to memory in one access.  Words at the ends of
// runs, and tokens of different sequences (a generation step), go one by one.
#pragma once

#include "kv_common.hpp"

namespace eskv {

constexpr int kPlaceThreads = 256;
constexpr int kPlaceTokens = 64;            // tokens of a workgroup

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
    Cache c;
};

struct ReadArgs {
    const int64_t* slots;
    uint16_t* k_out;
    uint16_t* v_out;
    uint64_t k_stride, v_stride;
    uint32_t* status;
    uint32_t tokens;
    Cache c;
};

template <int kLanes>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int m = 1; m < kLanes; m *= 2) x += __shfl_xor(x, m);
    return x;
}
template <int kLanes>
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
#pragma unroll
    for (int m = 1; m < kLanes; m *= 2) {
        const uint32_t y = __shfl_xor(x, m);
        x = x > y ? x : y;
    }
    return x;
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

// Normalise and rotate the row of which this lane (lane `lr` of the row's
// kLanes) holds x[0..7].  `turn`: the row of the rotation table, or null.
template <int kLanes>
__device__ __forceinline__ void norm_rotate(float x[8], int lr, bool norm, const float gain[8],
                                            float eps, uint32_t rot, bool adjacent,
                                            const float* turn) {
    constexpr float kInvD = 1.0f / (8 * kLanes);
    if (norm) {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
        ss = row_sum<kLanes>(ss);
        float r;
        if (ss < 0x1p120f) {
            r = 1.0f / __builtin_sqrtf(__builtin_fmaf(ss, kInvD, eps));
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * r * gain[i];
        } else {
            // elements beyond about 2^58: squares are summed in units of 2^160,
            // beside which eps is nothing (eps is at most the largest binary32)
            ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] *= 0x1p-80f;
                ss = __builtin_fmaf(x[i], x[i], ss);
            }
            ss = row_sum<kLanes>(ss);
            r = 1.0f / __builtin_sqrtf(__builtin_fmaf(ss, kInvD, eps * 0x1p-80f * 0x1p-80f));
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * r * gain[i];
        }
    }
    if (rot == 0) return;
    if (adjacent) {
        if (8u * lr < rot) {
            const f32x4_t c = load_float4(turn + 4 * lr);
            const f32x4_t s = load_float4(turn + rot / 2 + 4 * lr);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = x[2 * i], b = x[2 * i + 1];
                x[2 * i] = a * c[i] - b * s[i];
                x[2 * i + 1] = b * c[i] + a * s[i];
            }
        }
        return;
    }
    const int half = static_cast<int>(rot) / 16;             // lanes of one half
    const int away = lr < half ? half : lr < 2 * half ? -half : 0;
    const int lane = static_cast<int>(threadIdx.x) & 63;
    float other[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) other[i] = __shfl(x[i], lane + away);
    if (away != 0) {
        const float* t = turn + 8 * (away > 0 ? lr : lr - half);
        const f32x4_t c0 = load_float4(t), c1 = load_float4(t + 4);
        const f32x4_t s0 = load_float4(t + rot / 2), s1 = load_float4(t + rot / 2 + 4);
        const float sign = away > 0 ? -1.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = i < 4 ? c0[i & 3] : c1[i & 3], s = i < 4 ? s0[i & 3] : s1[i & 3];
            x[i] = x[i] * c + sign * (other[i] * s);
        }
    }
}

// LDS of the turned values: a row per dimension of 64 tokens and up to a word's
// shift, padded so that neighbouring rows start in different banks.
template <int kFmt>
struct Turned {
    static constexpr int kWord = 16 / kCodeBytes<kFmt>;      // tokens of a 16-byte word
    static constexpr int kWords = kPlaceTokens / kWord + 1;
    static constexpr int kRowBytes = 16 * kWords + 16;
};

// Where token 0 of the workgroup sits in its 16-byte word of slots (the columns'
// shift), and for every word whether its tokens are all here and in
// consecutive slots of one word.
template <int kFmt>
__device__ __forceinline__ void find_words(const int64_t* slot, int n, uint64_t pool, int& shift,
                                           uint32_t* whole) {
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
        bool ok = j0 >= 0 && j0 + T::kWord <= n;
        if (ok) {
            const int64_t s0 = slot[j0];
            ok = s0 >= 0 && uint64_t(s0) + T::kWord <= pool && (s0 & (T::kWord - 1)) == 0;
            for (int i = 1; i < T::kWord; ++i) ok = ok && slot[j0 + i] == s0 + i;
        }
        whole[threadIdx.x] = ok ? 1u : 0u;
    }
}

template <int D, int kFmt>
__global__ __launch_bounds__(kPlaceThreads) void es_kv_append_kernel(AppendArgs a) {
    using T = Turned<kFmt>;
    constexpr int kLanes = D / 8;                            // lanes of a row
    constexpr int kRows = kPlaceThreads / kLanes;            // rows of a pass
    const int lr = threadIdx.x % kLanes, row = threadIdx.x / kLanes;
    const uint32_t t0 = blockIdx.x * kPlaceTokens;
    const int n = static_cast<int>(min(uint32_t(kPlaceTokens), a.tokens - t0));
    const uint32_t head = blockIdx.y;

    // the row of the rotation table of token t, and whether it has one
    auto turn_of = [&](uint32_t t, bool& ok) -> const float* {
        ok = true;
        if (a.rot == 0) return nullptr;
        const int32_t p = a.positions[t];
        ok = p >= 0 && uint32_t(p) < a.rope_rows;
        return a.rope + uint64_t(ok ? p : 0) * a.rot;
    };
    auto load_gain = [&](const uint16_t* g, float gain[8]) {
        if (g == nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) gain[i] = 1.0f;
        } else {
            unpack8(load_row8(g + 8 * lr), gain);
        }
    };
    float gain[8];

    if (head < a.q_heads) {
        load_gain(a.q_gain, gain);
        for (int j = row; j - row < n; j += kRows) {         // whole passes: lanes exchange
            const uint32_t t = t0 + min(j, n - 1);
            bool ok;
            const float* turn = turn_of(t, ok);
            float x[8];
            unpack8(load_row8(a.q + t * a.q_stride + head * D + 8 * lr), x);
            norm_rotate<kLanes>(x, lr, a.q_gain != nullptr, gain, a.eps, a.rot, a.adjacent, turn);
            if (!ok) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = nan();
                if (lr == 0 && a.status != nullptr) atomicOr(a.status, ES_KV_BAD_POSITION);
            }
            u32x4_t out;
#pragma unroll
            for (int i = 0; i < 4; ++i) out[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
            if (j < n) store_row8(a.q_out + t * a.q_out_stride + head * D + 8 * lr, out);
        }
        return;
    }

    __shared__ __attribute__((aligned(16))) uint8_t turned[D * T::kRowBytes];
    __shared__ int64_t slot[kPlaceTokens];
    __shared__ uint32_t whole[T::kWords];
    const uint32_t h = head - a.q_heads;
    const uint64_t pool = uint64_t(a.c.n_pages) << a.c.page_shift;
    if (threadIdx.x < kPlaceTokens)
        slot[threadIdx.x] = static_cast<int>(threadIdx.x) < n ? a.slots[t0 + threadIdx.x] : -1;
    __syncthreads();
    int shift;
    find_words<kFmt>(slot, n, pool, shift, whole);

    load_gain(a.k_gain, gain);
    for (int j = row; j - row < n; j += kRows) {
        const uint32_t t = t0 + min(j, n - 1);
        bool ok;
        const float* turn = turn_of(t, ok);
        float x[8], y[8];
        unpack8(load_row8(a.k + t * a.k_stride + h * D + 8 * lr), x);
        unpack8(load_row8(a.v + t * a.v_stride + h * D + 8 * lr), y);
        norm_rotate<kLanes>(x, lr, a.k_gain != nullptr, gain, a.eps, a.rot, a.adjacent, turn);
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
        uint8_t* column = turned + (8 * lr) * T::kRowBytes + (j + shift) * kCodeBytes<kFmt>;
        if constexpr (kFmt == kBf16) {
            u32x4_t out;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                out[i] = dead ? 0x7FC07FC0u : pack_bf16(x[2 * i], x[2 * i + 1]);
                const uint32_t w = dead ? 0u : pack_bf16(y[2 * i], y[2 * i + 1]);
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
            if (lx) cx = encode8<kFmt>(x, kCodeMax<kFmt> / fx);
            if (ly) cy = encode8<kFmt>(y, kCodeMax<kFmt> / fy);
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

    // the values' rows of tokens
    for (int i = threadIdx.x; i < D * T::kWords; i += kPlaceThreads) {
        const int d = i / T::kWords, w = i % T::kWords;
        const int j0 = T::kWord * w - shift;
        const uint8_t* src = turned + d * T::kRowBytes + 16 * w;
        auto address = [&](int64_t s) {
            const uint64_t page = uint64_t(s) >> a.c.page_shift;
            const uint32_t off = uint32_t(s) & (a.c.page - 1);
            return a.c.v + (((page * a.c.heads + h) * D + d) * a.c.page + off) * kCodeBytes<kFmt>;
        };
        if (whole[w]) {
            store<u32x4_t>(address(slot[j0]), *reinterpret_cast<const u32x4_t*>(src));
        } else {
            for (int e = max(0, -j0); e < T::kWord && j0 + e < n; ++e) {
                const int64_t s = slot[j0 + e];
                if (s < 0 || uint64_t(s) >= pool) continue;
                if constexpr (kFmt == kBf16)
                    store<uint16_t>(address(s), reinterpret_cast<const uint16_t*>(src)[e]);
                else
                    store<uint8_t>(address(s), src[e]);
            }
        }
    }
}

template <int D, int kFmt>
__global__ __launch_bounds__(kPlaceThreads) void es_kv_read_kernel(ReadArgs a) {
    using T = Turned<kFmt>;
    constexpr int kLanes = D / 8;
    constexpr int kRows = kPlaceThreads / kLanes;
    const int lr = threadIdx.x % kLanes, row = threadIdx.x / kLanes;
    const uint32_t t0 = blockIdx.x * kPlaceTokens;
    const int n = static_cast<int>(min(uint32_t(kPlaceTokens), a.tokens - t0));
    const uint32_t h = blockIdx.y;
    const uint64_t pool = uint64_t(a.c.n_pages) << a.c.page_shift;

    __shared__ __attribute__((aligned(16))) uint8_t turned[D * T::kRowBytes];
    __shared__ int64_t slot[kPlaceTokens];
    __shared__ uint32_t whole[T::kWords];
    if (threadIdx.x < kPlaceTokens)
        slot[threadIdx.x] = static_cast<int>(threadIdx.x) < n ? a.slots[t0 + threadIdx.x] : -1;
    __syncthreads();
    int shift;
    find_words<kFmt>(slot, n, pool, shift, whole);
    __syncthreads();

    for (int i = threadIdx.x; i < D * T::kWords; i += kPlaceThreads) {
        const int d = i / T::kWords, w = i % T::kWords;
        const int j0 = T::kWord * w - shift;
        uint8_t* dst = turned + d * T::kRowBytes + 16 * w;
        auto address = [&](int64_t s) {
            const uint64_t page = uint64_t(s) >> a.c.page_shift;
            const uint32_t off = uint32_t(s) & (a.c.page - 1);
            return a.c.v + (((page * a.c.heads + h) * D + d) * a.c.page + off) * kCodeBytes<kFmt>;
        };
        if (whole[w]) {
            *reinterpret_cast<u32x4_t*>(dst) = load<u32x4_t>(address(slot[j0]));
        } else {
            for (int e = max(0, -j0); e < T::kWord && j0 + e < n; ++e) {
                const int64_t s = slot[j0 + e];
                if (s < 0 || uint64_t(s) >= pool) continue;
                if constexpr (kFmt == kBf16)
                    reinterpret_cast<uint16_t*>(dst)[e] = load<uint16_t>(address(s));
                else
                    dst[e] = load<uint8_t>(address(s));
            }
        }
    }
    __syncthreads();

    for (int j = row; j < n; j += kRows) {
        const uint32_t t = t0 + j;
        const int64_t s = slot[j];
        const bool in = s >= 0 && uint64_t(s) < pool;
        u32x4_t ko, vo;
        ko = u32x4_t{0u, 0u, 0u, 0u};
        vo = ko;
        if (in) {
            const uint64_t page = uint64_t(s) >> a.c.page_shift;
            const uint32_t off = uint32_t(s) & (a.c.page - 1);
            const uint64_t at = (page * a.c.heads + h) * a.c.page + off;
            const uint8_t* column =
                turned + (8 * lr) * T::kRowBytes + (j + shift) * kCodeBytes<kFmt>;
            if constexpr (kFmt == kBf16) {
                ko = load<u32x4_t>(a.c.k + (at * D + 8 * lr) * 2);
                const uint16_t k0 = load<uint16_t>(a.c.k + at * D * 2);
                const bool dead = (k0 & 0x7FFFu) > 0x7F80u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t lo =
                        *reinterpret_cast<const uint16_t*>(column + 2 * i * T::kRowBytes);
                    const uint32_t hi =
                        *reinterpret_cast<const uint16_t*>(column + (2 * i + 1) * T::kRowBytes);
                    vo[i] = dead ? 0x7FC07FC0u : lo | (hi << 16);
                }
            } else {
                const u32x2_t ck = load<u32x2_t>(a.c.k + at * D + 8 * lr);
                const float sk = load<float>(a.c.ks + at);
                const float sv = sk == sk ? load<float>(a.c.vs + at) : nan();
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t cv = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        cv |= uint32_t(column[(4 * i + e) * T::kRowBytes]) << (8 * e);
                    float xk[4], xv[4];
                    decode4<kFmt>(ck[i], xk);
                    decode4<kFmt>(cv, xv);
                    ko[2 * i] = pack_bf16(xk[0] * sk, xk[1] * sk);
                    ko[2 * i + 1] = pack_bf16(xk[2] * sk, xk[3] * sk);
                    vo[2 * i] = pack_bf16(xv[0] * sv, xv[1] * sv);
                    vo[2 * i + 1] = pack_bf16(xv[2] * sv, xv[3] * sv);
                }
            }
        } else if (s >= 0) {
            ko = u32x4_t{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
            vo = ko;
            if (lr == 0 && h == 0 && a.status != nullptr) atomicOr(a.status, ES_KV_BAD_SLOT);
        }
        store_row8(a.k_out + t * a.k_stride + h * D + 8 * lr, ko);
        store_row8(a.v_out + t * a.v_stride + h * D + 8 * lr, vo);
    }
}

}  // namespace eskv
