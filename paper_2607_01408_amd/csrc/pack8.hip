// A matrix into the 8-bit block format and back: what activation checkpoints and the operands of the
// 8-bit products are made with.  Both are bound by memory.
//
// Along the rows, 16 lanes take four blocks of 128 columns of one row: their loads are in flight
// together and their four scale bytes are one word.  Along the columns as well (the operand of a
// product that sums over the rows), a workgroup takes a tile of 128 x 128: it is one block of each
// of its rows and of each of its columns, so x is read once for both.
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
            load8(px + (left > 0 ? c : 0), left >= 8 ? 8 : static_cast<int>(left), v[i]);
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

// Tile blockIdx.x (rows) x blockIdx.y (columns) of 128 x 128.
template <typename T, bool ROWS>
__global__ __launch_bounds__(256) void pack8_both_kernel(const T* __restrict__ x, int64_t ldx,
                                                         uint8_t* __restrict__ values, uint8_t* __restrict__ scales,
                                                         uint8_t* __restrict__ t_values,
                                                         uint8_t* __restrict__ t_scales, int64_t R, int64_t D) {
    constexpr int ST = 132;  // floats of a tile row
    __shared__ float tile[128 * ST];
    const int64_t r0 = static_cast<int64_t>(blockIdx.x) * 128, c0 = static_cast<int64_t>(blockIdx.y) * 128;
    const int l = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t pitch = block8_pitch(D), spitch = block8_scale_pitch(D);
    const int64_t left = D - c0 - l * 8;
    const int n = left >= 8 ? 8 : static_cast<int>(left);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i * 16 + g;
        const int64_t row = r0 + r;
        float v[8];
        load8(x + (row < R ? row : 0) * ldx + (n > 0 ? c0 + l * 8 : 0), row < R ? n : 0, v);
        *reinterpret_cast<float4*>(&tile[r * ST + l * 8]) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(&tile[r * ST + l * 8 + 4]) = make_float4(v[4], v[5], v[6], v[7]);
        if constexpr (ROWS) {
            const int e = block8_scale(block8_top(v));
            const float inv = block8_inverse(e);
            if (row < R) {
                *reinterpret_cast<uint2*>(values + row * pitch + c0 + l * 8) =
                    make_uint2(block8_word(v[0], v[1], v[2], v[3], inv), block8_word(v[4], v[5], v[6], v[7], inv));
                if (l == 0) scales[row * spitch + blockIdx.y] = static_cast<uint8_t>(e);
                // the row's scale bytes past its last block
                if (blockIdx.y == gridDim.y - 1 && l >= 1 && blockIdx.y + l < spitch)
                    scales[row * spitch + blockIdx.y + l] = 127;
            }
        }
    }
    __syncthreads();
    // columns: 16 lanes take the column's 128 rows, 8 neighbouring rows each
    const int64_t tpitch = block8_pitch(R), tspitch = block8_scale_pitch(R);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = i * 16 + g;
        const int64_t column = c0 + c;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = tile[(l * 8 + j) * ST + c];
        const int e = block8_scale(block8_top(v));
        const float inv = block8_inverse(e);
        if (column < D) {
            *reinterpret_cast<uint2*>(t_values + column * tpitch + r0 + l * 8) =
                make_uint2(block8_word(v[0], v[1], v[2], v[3], inv), block8_word(v[4], v[5], v[6], v[7], inv));
            if (l == 0) t_scales[column * tspitch + blockIdx.x] = static_cast<uint8_t>(e);
            if (blockIdx.x == gridDim.x - 1 && l >= 1 && blockIdx.x + l < tspitch)
                t_scales[column * tspitch + blockIdx.x + l] = 127;
        }
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
    if (br > kMostBlocks || bc > 65535) return hipErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(br), static_cast<unsigned>(bc));
    if (values != nullptr)
        hipLaunchKernelGGL((pack8_both_kernel<T, true>), grid, dim3(256), 0, stream, x, ldx, values, scales, t_values,
                           t_scales, R, D);
    else
        hipLaunchKernelGGL((pack8_both_kernel<T, false>), grid, dim3(256), 0, stream, x, ldx, values, scales,
                           t_values, t_scales, R, D);
    return hipGetLastError();
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
