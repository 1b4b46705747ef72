// The 8-bit block format: e4m3 values with a power-of-two scale for each row and block of 128
// columns, held as an e8m0 byte.  The scale is the smallest power of two that brings the block's
// largest finite magnitude to 448 (the largest e4m3 value) or below, so a value keeps its four
// significant bits down to 2^-14 of the block's largest, and value times scale is a bf16 number: one
// conversion instruction makes it from the byte as it is.  An all-zero block has scale 1.  A non-finite element becomes NaN in its own slot and does not enter the scale.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "device_common.h"

namespace spingtp {
namespace {

constexpr int kBlock8 = 128;

__host__ __device__ constexpr int64_t block8_pitch(int64_t D) { return (D + 127) / 128 * 128; }
// bytes of a row of scales: whole 32-bit words, so that a lane reads four blocks' scales at once
__host__ __device__ constexpr int64_t block8_scale_pitch(int64_t D) { return (D + 511) / 512 * 4; }

__device__ __forceinline__ float finite_abs(float v) {
    const float a = fabsf(v);
    return a < __builtin_inff() ? a : 0.f;
}

// The scale's byte of a block with largest finite magnitude `top`: with top = m 2^k, 1 <= m < 2, and
// 448 = 1.75 2^8 the exponent is k - 8, one more where m > 1.75; at least 2^-126.
__device__ __forceinline__ int block8_scale(float top) {
    const uint32_t u = __float_as_uint(top);
    const int b = static_cast<int>(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return u == 0 ? 127 : (b < 1 ? 1 : b);
}
// 1 / scale, a power of two as well
__device__ __forceinline__ float block8_inverse(int scale) { return __uint_as_float(static_cast<uint32_t>(254 - scale) << 23); }
// of any e8m0 byte: 0 is 2^-127, 255 is NaN (as the products' conversion takes them)
__device__ __forceinline__ float block8_power(uint32_t scale) {
    const float power = scale == 0 ? __uint_as_float(0x400000u) : __uint_as_float(scale << 23);
    return scale == 255 ? __builtin_nanf("") : power;
}

// v / scale to e4m3 (nearest, ties to even; |v| / scale <= 448 for finite v, NaN for others), four to
// a word.
__device__ __forceinline__ uint32_t block8_word(float a, float b, float c, float d, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
    return static_cast<uint32_t>(w);
}
typedef float v2f __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void block8_values(uint32_t w, float (&v)[4]) {
    const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
    const v2f hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    v[0] = lo.x, v[1] = lo.y, v[2] = hi.x, v[3] = hi.y;
}

// Largest value over the 16 lanes of a row of lanes (the lanes of one block of 128 columns).
__device__ __forceinline__ float max16(float v) {
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
    return v;
}

// Largest finite magnitude of a block held by 16 lanes, N values each.  Infinities are rare: only a block
// whose plain maximum is one looks at its values again.
template <int N>
__device__ __forceinline__ float block8_top(const float (&v)[N]) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) top = fmaxf(top, fabsf(v[j]));  // a NaN loses
    top = max16(top);
    if (top < __builtin_inff()) return top;
    top = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) top = fmaxf(top, finite_abs(v[j]));
    return max16(top);
}

// Eight neighbouring elements of a row at any element address (global memory takes unaligned wide
// loads), zeros from `n` on.
typedef float u4f __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u4u __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
    if (n >= 8) {
        const u4f a = *reinterpret_cast<const u4f*>(p), b = *reinterpret_cast<const u4f*>(p + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
    }
}
__device__ __forceinline__ void load8(const uint16_t* p, int n, float (&v)[8]) {
    if (n >= 8) {
        const u4u a = *reinterpret_cast<const u4u*>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? bf16_to_f32(p[i]) : 0.f;
    }
}
// load8 of a matrix that is not read again soon: around the caches.
__device__ __forceinline__ void pass8(const float* p, int n, float (&v)[8]) {
    if (n >= 8) {
        const u4f a = __builtin_nontemporal_load(reinterpret_cast<const u4f*>(p));
        const u4f b = __builtin_nontemporal_load(reinterpret_cast<const u4f*>(p + 4));
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
        load8(p, n, v);
    }
}
__device__ __forceinline__ void pass8(const uint16_t* p, int n, float (&v)[8]) {
    if (n >= 8) {
        const u4u a = __builtin_nontemporal_load(reinterpret_cast<const u4u*>(p));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
        load8(p, n, v);
    }
}
// two floats to bf16, nearest with ties to even (one instruction)
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, v2bf{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
    if (n >= 8) {
        *reinterpret_cast<u4f*>(p) = u4f{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<u4f*>(p + 4) = u4f{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = v[i];
    }
}
__device__ __forceinline__ void store8(uint16_t* p, int n, const float (&v)[8]) {
    if (n >= 8) {
        *reinterpret_cast<u4u*>(p) =
            u4u{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = f32_to_bf16(v[i]);
    }
}
// v rounded to the element type
__device__ __forceinline__ float as_type(float v, const float*) { return v; }
__device__ __forceinline__ float as_type(float v, const uint16_t*) { return bf16_to_f32(f32_to_bf16(v)); }

}  // namespace
}  // namespace spingtp
