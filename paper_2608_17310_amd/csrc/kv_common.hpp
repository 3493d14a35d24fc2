// What the cache's kernels share: vector types, the three formats, the
// arguments and the walk over a batch of sequences.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/esopt.h"

namespace eskv {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

#define ESKV_GLOBAL __attribute__((address_space(1)))

template <class T>
__device__ __forceinline__ T load(const void* p) {
    return *reinterpret_cast<const ESKV_GLOBAL T*>(reinterpret_cast<uintptr_t>(p));
}
template <class T>
__device__ __forceinline__ void store(void* p, T v) {
    *reinterpret_cast<ESKV_GLOBAL T*>(reinterpret_cast<uintptr_t>(p)) = v;
}

// Rows of queries, keys and values may start at any bf16, and of the rotation table at
// any float: global memory accesses need no alignment on this part, and the
// types say so.
typedef u32x4_t u32x4_at2_t __attribute__((aligned(2)));
typedef u32x2_t u32x2_at2_t __attribute__((aligned(2)));
typedef f32x4_t f32x4_at4_t __attribute__((aligned(4)));

__device__ __forceinline__ u32x4_t load_row8(const uint16_t* p) {
    return *reinterpret_cast<const ESKV_GLOBAL u32x4_at2_t*>(reinterpret_cast<uintptr_t>(p));
}
__device__ __forceinline__ void store_row8(uint16_t* p, u32x4_t v) {
    *reinterpret_cast<ESKV_GLOBAL u32x4_at2_t*>(reinterpret_cast<uintptr_t>(p)) = v;
}
__device__ __forceinline__ void store_row4(uint16_t* p, u32x2_t v) {
    *reinterpret_cast<ESKV_GLOBAL u32x2_at2_t*>(reinterpret_cast<uintptr_t>(p)) = v;
}
__device__ __forceinline__ f32x4_t load_float4(const float* p) {
    return *reinterpret_cast<const ESKV_GLOBAL f32x4_at4_t*>(reinterpret_cast<uintptr_t>(p));
}

// A value at an address that is the same for the wave, through the scalar cache.
__device__ __forceinline__ int32_t load_uniform(const int32_t* p) {
    return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(
        reinterpret_cast<uintptr_t>(p));
}

enum Format : int { kInt8 = ES_KV_INT8, kE4M3 = ES_KV_E4M3, kBf16 = ES_KV_BF16 };

template <int kFmt>
constexpr int kCodeBytes = kFmt == kBf16 ? 2 : 1;
template <int kFmt>
constexpr float kCodeMax = kFmt == kInt8 ? 127.0f : 448.0f;
constexpr float kTinyRow = 0x1p-100f;       // rows whose largest |x| is below read as zeros

constexpr float kLog2e = 1.4426950408889634f;

// `bytes` bytes of global memory as the buffer instructions address them: a base
// in scalar registers and one 32-bit offset a lane, so that a wave's loads need no
// 64-bit address arithmetic.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}
__device__ __forceinline__ u32x4_t load_buffer(Buffer b, uint32_t offset, uint32_t more = 0) {
    return __builtin_amdgcn_raw_buffer_load_b128(b, offset, more, 0);    // more: of the wave
}
template <class T>
__device__ __forceinline__ T load_buffer_as(Buffer b, uint32_t offset, uint32_t more) {
    if constexpr (sizeof(T) == 16)
        return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b128(b, offset, more, 0));
    else
        return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b64(b, offset, more, 0));
}
__device__ __forceinline__ float load_buffer_float(Buffer b, uint32_t offset) {
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(b, offset, 0, 0));
}
// 16 bytes a lane from memory into LDS, at `dst` (the same for the wave) + 16 lane,
// without passing registers; wait_loads() before the wave's own barrier.
__device__ __forceinline__ void load_to_lds(Buffer b, uint32_t offset, void* dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        b,
        reinterpret_cast<__attribute__((address_space(3))) void*>(
            static_cast<uint32_t>(reinterpret_cast<uintptr_t>(dst))),
        16, offset, 0, 0, 0);
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

__device__ __forceinline__ float inf() { return __builtin_inff(); }
__device__ __forceinline__ float nan() { return __builtin_nanf(""); }

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {     // RNE
    const bf16x2_t p = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
    return __builtin_bit_cast(uint32_t, p);
}

__device__ __forceinline__ void unpack8(u32x4_t w, float x[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
    }
}

// Four codes of a word as binary32, exactly.
template <int kFmt>
__device__ __forceinline__ void decode4(uint32_t w, float v[4]) {
    if constexpr (kFmt == kInt8) {
        v[0] = static_cast<float>(static_cast<int8_t>(w));
        v[1] = static_cast<float>(static_cast<int8_t>(w >> 8));
        v[2] = static_cast<float>(static_cast<int8_t>(w >> 16));
        v[3] = static_cast<float>(static_cast<int32_t>(w) >> 24);
    } else {
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
        const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
        const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
        v[0] = lo.x; v[1] = lo.y; v[2] = hi.x; v[3] = hi.y;
    }
}

// Eight codes (two words) as bf16.  Every int8 and every E4M3 value is a bf16
// value, so nothing is rounded: E4M3 by the hardware's conversion with scale 1,
// int8 through binary32, whose upper halves are the bf16 values.
template <int kFmt>
__device__ __forceinline__ u32x4_t codes_to_bf16(u32x2_t c) {
    u32x4_t out;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (kFmt == kE4M3) {
            out[2 * i] = __builtin_bit_cast(
                uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], 1.0f, false));
            out[2 * i + 1] = __builtin_bit_cast(
                uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], 1.0f, true));
        } else {
            float v[4];
            decode4<kInt8>(c[i], v);
            out[2 * i] = __builtin_amdgcn_perm(__float_as_uint(v[1]), __float_as_uint(v[0]),
                                               0x07060302u);
            out[2 * i + 1] = __builtin_amdgcn_perm(__float_as_uint(v[3]), __float_as_uint(v[2]),
                                                   0x07060302u);
        }
    }
    return out;
}

// Values that are not finite have every exponent bit set in bf16, and every bit but
// the sign in E4M3; no int8 code is one.  One more in that place carries into the
// sign's: these bits of a word, for its values, are the test.
template <int kFmt>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    if constexpr (kFmt == kBf16) return ((w & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u;
    if constexpr (kFmt == kE4M3) return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    return 0u;
}
// The word with zeros for them.
template <int kFmt>
__device__ __forceinline__ uint32_t finite(uint32_t w) {
    const uint32_t top = not_finite<kFmt>(w);
    return w & ~((top << 1) - (top >> (8 * kCodeBytes<kFmt> - 1)));
}
__device__ __forceinline__ float finite_scale(float x) {
    return __builtin_fabsf(x) < __builtin_inff() ? x : 0.0f;
}
// N 16-byte words of values, tested first: one is seldom found.  True: some were.
template <int kFmt, int N>
__device__ __forceinline__ bool make_finite(u32x4_t (&x)[N]) {
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) any |= not_finite<kFmt>(x[i / 4][i % 4]);
    if (any == 0) return false;
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) x[i / 4][i % 4] = finite<kFmt>(x[i / 4][i % 4]);
    return true;
}

// Eight values times `inv` as codes (RNE; |x inv| is at most the format's largest
// value up to roundings of binary32, which the integer rounding and E4M3's
// rounding to 448 both absorb).
template <int kFmt>
__device__ __forceinline__ u32x2_t encode8(const float x[8], float inv) {
    u32x2_t out;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float* y = x + 4 * i;
        if constexpr (kFmt == kInt8) {
            uint32_t w = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int q = static_cast<int>(__builtin_rintf(y[j] * inv));
                w |= (static_cast<uint32_t>(q) & 0xFFu) << (8 * j);
            }
            out[i] = w;
        } else {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * inv, y[1] * inv, 0, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * inv, y[3] * inv, w, true);
            out[i] = static_cast<uint32_t>(w);
        }
    }
    return out;
}

// The cache, as the kernels see it.
struct Cache {
    uint8_t* k;
    uint8_t* v;
    float* ks;
    float* vs;
    uint32_t n_pages, heads, page, page_shift;
};

}  // namespace eskv
