// A matrix into the 8-bit block format and back: what activation checkpoints and the operands of the
// 8-bit products are made with.  Both are bound by memory.
//
// Along the rows, 16 lanes take four blocks of 128 columns of one row: their loads are in flight
// together and their four scale bytes are one word.  x passes around the caches, which keep the 8-bit
// side for its reader (20,000 x 4,800 fp32 packed and unpacked: 213 -> 177 us, 4.3 -> 5.4 TB/s; stores
// around the caches made it 226).  Along the columns as well (the operand of a
// product that sums over the rows), a workgroup takes a tile of 128 x 128: it is one block of each
// of its rows and of each of its columns, so x is read once for both (4,096 x 4,096 bf16 18.3 us, 3.7 TB/s).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "block8.h"
#include "feedforward.h"
#include "internal.h"

namespace spingtp {
namespace {

template <typename T>
__global__ __launch_bounds__(256) void pack8_rows_kernel(const T* __restrict__ x, int64_t ldx,
                                                         uint8_t* __restrict__ values, uint8_t* __restrict__ scales,
                                                         int64_t R, int64_t D, int quads) {
    const int l = threadIdx.x & 15;
    const int64_t units = R * quads, stride = static_cast<int64_t>(gridDim.x) * 16;
    // the 16 lanes of a unit (a row's four blocks) agree on the loop
    for (int64_t unit = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4); unit < units; unit += stride) {
        const int64_t row = unit / quads;
        const int64_t pitch = block8_pitch(D);
        const int64_t c0 = (unit - row * quads) * 4 * kBlock8 + l * 8;
        const T* px = x + row * ldx;
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t c = c0 + i * kBlock8, left = D - c;
            pass8(px + (left > 0 ? c : 0), left >= 8 ? 8 : static_cast<int>(left), v[i]);
        }
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t c = c0 + i * kBlock8;
            const int e = block8_scale(block8_top(v[i]));  // 127 past the last block
            const float inv = block8_inverse(e);
            word |= static_cast<uint32_t>(e) << (8 * i);
            if (c < pitch)
                *reinterpret_cast<uint2*>(values + row * pitch + c) =
                    make_uint2(block8_word(v[i][0], v[i][1], v[i][2], v[i][3], inv),
                               block8_word(v[i][4], v[i][5], v[i][6], v[i][7], inv));
        }
        if (l == 0) reinterpret_cast<uint32_t*>(scales)[unit] = word;
    }
}

// Two neighbouring columns of a row of the LDS tile.
__device__ __forceinline__ void two(const float* p, float& a, float& b) {
    const float2 v = *reinterpret_cast<const float2*>(p);
    a = v.x, b = v.y;
}
__device__ __forceinline__ void two(const uint16_t* p, float& a, float& b) {
    const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
    a = __uint_as_float(v << 16), b = __uint_as_float(v & 0xffff0000u);
}
__device__ __forceinline__ void keep8(float* p, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(p + 2 * i) = make_float2(v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ void keep8(uint16_t* p, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(p + 2 * i) = bf16_pair(v[2 * i], v[2 * i + 1]);
}

// Tile first + blockIdx.x (rows; `last` is the matrix's last) x blockIdx.y (columns) of 128 x 128.  It lies in LDS in
// its own type.  Along the columns a lane takes two neighbouring ones and a wave a quarter of their rows, so its
// reads of LDS run along the rows, without conflicts, and 32 bytes of each column leave in two stores.
template <typename T, bool ROWS>
__global__ __launch_bounds__(256) void pack8_both_kernel(const T* __restrict__ x, int64_t ldx,
                                                         uint8_t* __restrict__ values, uint8_t* __restrict__ scales,
                                                         uint8_t* __restrict__ t_values,
                                                         uint8_t* __restrict__ t_scales, int64_t R, int64_t D,
                                                         int64_t first, int64_t last) {
    constexpr int ST = 130;  // elements of a tile row
    __shared__ __align__(16) T tile[128 * ST];
    __shared__ float tops[4][128];
    const int64_t rows = first + blockIdx.x, r0 = rows * 128, c0 = static_cast<int64_t>(blockIdx.y) * 128;
    const int l = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t pitch = block8_pitch(D), spitch = block8_scale_pitch(D);
    const int64_t left = D - c0 - l * 8;
    const int n = left >= 8 ? 8 : static_cast<int>(left);
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = r0 + i * 16 + g;
        load8(x + (row < R ? row : 0) * ldx + (n > 0 ? c0 + l * 8 : 0), row < R ? n : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = r0 + i * 16 + g;
        keep8(&tile[(i * 16 + g) * ST + l * 8], v[i]);
        if constexpr (ROWS) {
            const int e = block8_scale(block8_top(v[i]));
            const float inv = block8_inverse(e);
            if (row < R) {
                *reinterpret_cast<uint2*>(values + row * pitch + c0 + l * 8) =
                    make_uint2(block8_word(v[i][0], v[i][1], v[i][2], v[i][3], inv),
                               block8_word(v[i][4], v[i][5], v[i][6], v[i][7], inv));
                if (l == 0) scales[row * spitch + blockIdx.y] = static_cast<uint8_t>(e);
                // the row's scale bytes past its last block
                if (blockIdx.y == gridDim.y - 1 && l >= 1 && blockIdx.y + l < spitch)
                    scales[row * spitch + blockIdx.y + l] = 127;
            }
        }
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float a[32], b[32], ta = 0.f, tb = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        two(&tile[(32 * wave + i) * ST + 2 * lane], a[i], b[i]);
        ta = fmaxf(ta, fabsf(a[i]));
        tb = fmaxf(tb, fabsf(b[i]));
    }
    if (!(fmaxf(ta, tb) < __builtin_inff())) {  // an infinity: the largest finite ones
        ta = tb = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) ta = fmaxf(ta, finite_abs(a[i])), tb = fmaxf(tb, finite_abs(b[i]));
    }
    *reinterpret_cast<float2*>(&tops[wave][2 * lane]) = make_float2(ta, tb);
    __syncthreads();
    const int64_t tpitch = block8_pitch(R), tspitch = block8_scale_pitch(R);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c = 2 * lane + h;
        const int64_t column = c0 + c;
        if (column >= D) continue;
        const float top = fmaxf(fmaxf(tops[0][c], tops[1][c]), fmaxf(tops[2][c], tops[3][c]));
        const int e = block8_scale(top);
        const float inv = block8_inverse(e);
        const float(&w)[32] = h == 0 ? a : b;
        uint8_t* to = t_values + column * tpitch + r0 + 32 * wave;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            *reinterpret_cast<uint4*>(to + 16 * i) =
                make_uint4(block8_word(w[16 * i], w[16 * i + 1], w[16 * i + 2], w[16 * i + 3], inv),
                           block8_word(w[16 * i + 4], w[16 * i + 5], w[16 * i + 6], w[16 * i + 7], inv),
                           block8_word(w[16 * i + 8], w[16 * i + 9], w[16 * i + 10], w[16 * i + 11], inv),
                           block8_word(w[16 * i + 12], w[16 * i + 13], w[16 * i + 14], w[16 * i + 15], inv));
        // the scale, and behind the column's last block the bytes up to the word's end
        if (wave == 0) t_scales[column * tspitch + rows] = static_cast<uint8_t>(e);
        if (wave > 0 && rows == last && rows + wave < tspitch) t_scales[column * tspitch + rows + wave] = 127;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack8_kernel(const uint8_t* __restrict__ values,
                                                      const uint8_t* __restrict__ scales, T* __restrict__ x,
                                                      int64_t ldx, int64_t R, int64_t D, int quads) {
    const int l = threadIdx.x & 15;
    const int64_t units = R * quads, stride = static_cast<int64_t>(gridDim.x) * 16;
    // the 16 lanes of a unit (a row's four blocks) agree on the loop
    for (int64_t unit = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4); unit < units; unit += stride) {
        const int64_t row = unit / quads;
        const int64_t pitch = block8_pitch(D);
        const int64_t c0 = (unit - row * quads) * 4 * kBlock8 + l * 8;
        const uint32_t word = reinterpret_cast<const uint32_t*>(scales)[unit];
        uint2 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t c = c0 + i * kBlock8;
            q[i] = *reinterpret_cast<const uint2*>(values + row * pitch + (c < pitch ? c : 0));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t c = c0 + i * kBlock8, left = D - c;
            const float s = block8_power((word >> (8 * i)) & 255u);
            float a[4], b[4], v[8];
            block8_values(q[i].x, a);
            block8_values(q[i].y, b);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = a[j] * s, v[4 + j] = b[j] * s;
            if (left > 0) store8(x + row * ldx + c, left >= 8 ? 8 : static_cast<int>(left), v);
        }
    }
}

template <typename T>
hipError_t pack(const T* x, int64_t ldx, uint8_t* values, uint8_t* scales, uint8_t* t_values, uint8_t* t_scales,
                int64_t R, int64_t D, hipStream_t stream) {
    if (t_values == nullptr) {
        const int64_t quads = block8_scale_pitch(D) / 4, blocks = (R * quads + 15) / 16;
        hipLaunchKernelGGL((pack8_rows_kernel<T>),
                           dim3(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks)), dim3(256), 0,
                           stream, x, ldx, values, scales, R, D, static_cast<int>(quads));
        return hipGetLastError();
    }
    const int64_t br = (R + 127) / 128, bc = (D + 127) / 128;
    if (bc > 65535) return hipErrorInvalidValue;
    for (int64_t first = 0; first < br; first += kMostBlocks) {  // as many rows as one launch holds
        const dim3 grid(static_cast<unsigned>(br - first < kMostBlocks ? br - first : kMostBlocks),
                        static_cast<unsigned>(bc));
        if (values != nullptr)
            hipLaunchKernelGGL((pack8_both_kernel<T, true>), grid, dim3(256), 0, stream, x, ldx, values, scales,
                               t_values, t_scales, R, D, first, br - 1);
        else
            hipLaunchKernelGGL((pack8_both_kernel<T, false>), grid, dim3(256), 0, stream, x, ldx, values, scales,
                               t_values, t_scales, R, D, first, br - 1);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_pack8(int dtype, const void* x, int64_t ldx, uint8_t* values, uint8_t* scales, uint8_t* t_values,
                        uint8_t* t_scales, int64_t R, int64_t D, hipStream_t stream) {
    return dtype == SPINGTP_FP32
               ? pack(static_cast<const float*>(x), ldx, values, scales, t_values, t_scales, R, D, stream)
               : pack(static_cast<const uint16_t*>(x), ldx, values, scales, t_values, t_scales, R, D, stream);
}

hipError_t launch_unpack8(int dtype, const uint8_t* values, const uint8_t* scales, void* x, int64_t ldx, int64_t R,
                          int64_t D, hipStream_t stream) {
    const int64_t quads = block8_scale_pitch(D) / 4, blocks = (R * quads + 15) / 16;
    const dim3 grid(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks));
    if (dtype == SPINGTP_FP32)
        hipLaunchKernelGGL((unpack8_kernel<float>), grid, dim3(256), 0, stream, values, scales,
                           static_cast<float*>(x), ldx, R, D, static_cast<int>(quads));
    else
        hipLaunchKernelGGL((unpack8_kernel<uint16_t>), grid, dim3(256), 0, stream, values, scales,
                           static_cast<uint16_t*>(x), ldx, R, D, static_cast<int>(quads));
    return hipGetLastError();
}

}  // namespace spingtp
