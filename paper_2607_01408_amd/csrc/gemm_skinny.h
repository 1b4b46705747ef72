// The products of gemm_nt.h for at most 64 rows of x (single tokens, small batches): bound by the
// reading of w, once.
//
// A workgroup takes 16 rows of w (of both matrices in the gated form); its eight waves share the
// summed axis, 128 bytes of every row in turn, straight from memory to registers with several steps'
// loads in flight, and their sums meet in LDS in a fixed order.  So N / 16 workgroups of 8 waves read
// at once, which fills the memory system from N of a few hundred on.  x is read from the cache.
// bf16 rows may start at any element and have any length; 8-bit rows are as packed.
// Measured, one row, 8 bits: 4,096 x 4,096 5.6 us, 3.0 TB/s; gated 2,048 x 8,192 8.2 us, 4.1 TB/s.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "gemm_nt.h"

namespace spingtp {
namespace {

constexpr int kSkinnyRows = 64;   // of x
constexpr int kSkinnyWaves = 8;

// Sixteen bytes of a row from byte `at` on, zeros behind its end (bf16).
template <class E>
__device__ __forceinline__ v4i row_chunk(const uint8_t* row, int64_t at, int64_t bytes) {
    if constexpr (E::kScaled) return *reinterpret_cast<const v4i*>(row + at);
    const int64_t left = (bytes - at) / 2;
    if (left >= 8) {
        const u4u v = *reinterpret_cast<const u4u*>(row + at);
        return v4i{static_cast<int>(v.x), static_cast<int>(v.y), static_cast<int>(v.z), static_cast<int>(v.w)};
    }
    const uint16_t* p = reinterpret_cast<const uint16_t*>(row + at);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) w[i / 2] |= static_cast<uint32_t>(p[i]) << (16 * (i & 1));
    return v4i{static_cast<int>(w[0]), static_cast<int>(w[1]), static_cast<int>(w[2]), static_cast<int>(w[3])};
}

// Sums of the tile's 16 columns n0.. and 16 TM rows: done(m, n, sum of w, sum of w2) by one thread each.
// `row_bytes`: of a bf16 row.
template <class E, int TM, bool GATED, class Done>
__device__ __forceinline__ void skinny_tile(const GemmArgs& a, int64_t row_bytes, int64_t n0, const Done& done) {
    constexpr int S = GATED ? 2 : 1, U = TM * S > 4 ? 1 : (TM * S > 2 ? 2 : 4);  // matrices; steps in flight
    __shared__ float part[kSkinnyWaves][S * TM][16][17];
    const int lane = threadIdx.x & 63, row = lane & 15, group = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n = n0 + row < a.N ? n0 + row : a.N - 1;
    const uint8_t* pw[S];
    const uint8_t* qw[S];
    const uint8_t* px[TM];
    const uint8_t* qx[TM];
    pw[0] = a.w + n * a.ldw;
    qw[0] = a.ws + n * a.lds;
    if constexpr (GATED) pw[1] = a.w2 + n * a.ldw, qw[1] = a.ws2 + n * a.lds;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int64_t m = 16 * j + row < a.M ? 16 * j + row : a.M - 1;
        px[j] = a.x + m * a.ldx;
        qx[j] = a.xs + m * a.lds;
    }
    v4f acc[S][TM];
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    for (int first = wave; first < a.steps; first += kSkinnyWaves * U) {
        v4i rw[U][S][2], rx[U][TM][2];
        uint32_t ew[U][S], ex[U][TM];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int step = first + u * kSkinnyWaves < a.steps ? first + u * kSkinnyWaves : first;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int64_t at = static_cast<int64_t>(step) * kStepBytes + c * 64 + group * 16;
#pragma unroll
                for (int i = 0; i < S; ++i) rw[u][i][c] = row_chunk<E>(pw[i], at, row_bytes);
#pragma unroll
                for (int j = 0; j < TM; ++j) rx[u][j][c] = row_chunk<E>(px[j], at, row_bytes);
            }
            if constexpr (E::kScaled) {
#pragma unroll
                for (int i = 0; i < S; ++i) ew[u][i] = qw[i][step];
#pragma unroll
                for (int j = 0; j < TM; ++j) ex[u][j] = qx[j][step];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (first + u * kSkinnyWaves >= a.steps) break;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                v8bf fw[S][E::kParts], fx[TM][E::kParts];
#pragma unroll
                for (int i = 0; i < S; ++i)
                    E::expand(rw[u][i][c], E::kScaled ? __uint_as_float(ew[u][i] << 23) : 1.f, fw[i]);
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    E::expand(rx[u][j][c], E::kScaled ? __uint_as_float(ex[u][j] << 23) : 1.f, fx[j]);
#pragma unroll
                for (int p = 0; p < E::kParts; ++p)
#pragma unroll
                    for (int i = 0; i < S; ++i)
#pragma unroll
                        for (int j = 0; j < TM; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[i][p], fx[j][p], acc[i][j], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) part[wave][i * TM + j][4 * group + r][row] = acc[i][j][r];
    __syncthreads();
    const int at = threadIdx.x & 15;
#pragma unroll
    for (int first = 0; first < 16 * TM; first += 32) {  // 32 rows of 16 columns at a time
        const int m = first + (threadIdx.x >> 4);
        if (m < 16 * TM && m < a.M && n0 + at < a.N) {
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < S; ++i)
#pragma unroll
                for (int w = 0; w < kSkinnyWaves; ++w) s[i] += part[w][i * TM + m / 16][at][m & 15];
            done(m, n0 + at, s[0], s[1]);
        }
    }
}

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = static_cast<uint16_t>(bf16_pair(v, v)); }

template <class E, int TM, typename TO>
__global__ __launch_bounds__(64 * kSkinnyWaves) void gemm_skinny_kernel(GemmArgs a, int64_t row_bytes,
                                                                        TO* __restrict__ out, int64_t ldo) {
    skinny_tile<E, TM, false>(a, row_bytes, static_cast<int64_t>(blockIdx.x) * 16,
                              [&](int64_t m, int64_t n, float s, float) { put(out + m * ldo + n, s); });
}

}  // namespace
}  // namespace spingtp
