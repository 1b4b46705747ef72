// Root-mean-square norm of rows, with the residual's addition before it and the 8-bit block format
// after it, and its gradients.
//   h = x + r (rounded to the element type: the residual stream that is kept)
//   rstd = (mean_d h^2 + eps)^(-1/2),  y = h rstd gain
//   with t = gain dy and xhat = h rstd:  dx = rstd (t - xhat mean_d(t xhat)) + dh,
//   dgain = sum over the rows of dy xhat.
// Sums, statistics and products are fp32.
//
// Bound by memory: a row is read once, stays in registers between the sum of squares and the
// output, and is written once.  TPR threads share a row, each with V groups of 8 neighbouring
// columns; 16 lanes hold a block of 128 columns, so its largest magnitude takes four lane
// exchanges.  Rows too long for that are read twice, the second time from the cache.
// Measured: 16,384 x 4,096 bf16 with the residual 96-105 us, 5.1-5.6 TB/s; its gradients 94-107 us and 5 us for
// the gain's sum, 5.0-5.7 TB/s; 100,000 x 128 fp32 to 8 bits 26 us, 6.4 TB/s (a part from the cache behind the L2); one
// row of 2,048 3.1 us, the latency of its loads and two sums.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "block8.h"
#include "feedforward.h"
#include "internal.h"

namespace spingtp {
namespace {

// Sum over the TPR threads of a row (TPR > 64: over the workgroup, through `part`).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part) {
#pragma unroll
    for (int d = 1; d < (TPR < 64 ? TPR : 64); d <<= 1) v += __shfl_xor(v, d, 64);
    if constexpr (TPR > 64) {
        __syncthreads();  // an earlier sum has been read
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) v += part[w];
    }
    return v;
}

// V = 0: rows of any length, read twice.
template <typename T, int TPR, int V, bool OUT8>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void rms_norm_kernel(
    const T* __restrict__ x, int64_t ldx, const T* __restrict__ r, int64_t ldr, const float* __restrict__ gain,
    float eps, T* __restrict__ h, int64_t ldh, T* __restrict__ y, int64_t ldy, uint8_t* __restrict__ values,
    uint8_t* __restrict__ scales, float* __restrict__ rstd_out, int64_t R, int64_t D) {
    constexpr int THREADS = TPR > 256 ? TPR : 256;
    constexpr int ROWS = THREADS / TPR;
    constexpr int VS = V > 0 ? V : 1;
    __shared__ float part[16];
    const int t = threadIdx.x % TPR;
    // whole rows: the threads of a row agree on the loop
    const int64_t stride = static_cast<int64_t>(gridDim.x) * ROWS;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR; row < R; row += stride) {
        const T* px = x + row * ldx;
        const T* pr = r != nullptr ? r + row * ldr : nullptr;
        T* ph = h != nullptr ? h + row * ldh : nullptr;
        const int64_t steps = V > 0 ? V : (D + 8 * TPR - 1) / (8 * TPR);
        float v[VS][8];
        float s = 0.f;
        auto left = [&](int64_t c) { return D - c >= 8 ? 8 : static_cast<int>(D - c); };  // <= 0 past the row
        auto take = [&](int64_t i, float (&w)[8]) {
            const int64_t c = (i * TPR + t) * 8;
            const int n = left(c);
            load8(px + (n > 0 ? c : 0), n, w);
            if (pr != nullptr) {
                float q[8];
                load8(pr + (n > 0 ? c : 0), n, q);
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = as_type(w[j] + q[j], px);
            }
        };
        if constexpr (V > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) take(i, v[i]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int64_t c = (static_cast<int64_t>(i) * TPR + t) * 8;
                if (ph != nullptr && c < D) store8(ph + c, left(c), v[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) s = fmaf(v[i][j], v[i][j], s);
            }
        } else {
            for (int64_t i = 0; i < steps; ++i) {
                take(i, v[0]);
                const int64_t c = (i * TPR + t) * 8;
                if (ph != nullptr && c < D) store8(ph + c, left(c), v[0]);
#pragma unroll
                for (int j = 0; j < 8; ++j) s = fmaf(v[0][j], v[0][j], s);
            }
        }
        s = row_sum<TPR>(s, part);
        const float rstd = 1.f / sqrtf(s / static_cast<float>(D) + eps);
        if (t == 0 && rstd_out != nullptr) rstd_out[row] = rstd;
        const int64_t pitch = block8_pitch(D), spitch = block8_scale_pitch(D), nb = pitch / kBlock8;
        auto give = [&](int64_t i, float (&w)[8]) {
            const int64_t c = (i * TPR + t) * 8;
            if (c >= pitch) return;  // whole blocks: the 16 lanes of a block leave together
            const int n = left(c);
            float gn[8];
            load8(gain + (n > 0 ? c : 0), n, gn);
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = w[j] * rstd * gn[j];
            if constexpr (OUT8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = j < n ? w[j] : 0.f;  // behind the row, whatever rstd is
                const int e = block8_scale(block8_top(w));
                const float inv = block8_inverse(e);
                *reinterpret_cast<uint2*>(values + row * pitch + c) =
                    make_uint2(block8_word(w[0], w[1], w[2], w[3], inv), block8_word(w[4], w[5], w[6], w[7], inv));
                if ((t & 15) == 0) scales[row * spitch + c / kBlock8] = static_cast<uint8_t>(e);
            } else if (n > 0) {
                store8(y + row * ldy + c, n, w);
            }
        };
        if constexpr (V > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) give(i, v[i]);
        } else {
            for (int64_t i = 0; i < steps; ++i) {
                const int64_t c = (i * TPR + t) * 8;
                const int n = left(c);
                load8((ph != nullptr ? ph : px) + (n > 0 ? c : 0), n, v[0]);  // this thread's own h
                give(i, v[0]);
            }
        }
        if (OUT8 && t < spitch - nb) scales[row * spitch + nb + t] = 127;
    }
}

// One workgroup takes rows blockIdx.x, blockIdx.x + gridDim.x, ... (ROWS at a time) and sums its part
// of dgain in registers; partial[blockIdx.x][D] is summed by norm_gain_kernel, in a fixed order.
template <typename T, int TPR, int V>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void rms_norm_bwd_kernel(
    const T* __restrict__ dy, int64_t lddy, const T* __restrict__ h, int64_t ldh, const float* __restrict__ rstd_in,
    const float* __restrict__ gain, const T* __restrict__ gh, int64_t ldgh, T* __restrict__ dx, int64_t lddx,
    float* __restrict__ partial, int64_t R, int64_t D) {
    constexpr int THREADS = TPR > 256 ? TPR : 256;
    constexpr int ROWS = THREADS / TPR;
    constexpr int VS = V > 0 ? V : 1;
    __shared__ float part[16];
    const int t = threadIdx.x % TPR;
    const int64_t steps = V > 0 ? V : (D + 8 * TPR - 1) / (8 * TPR);
    auto left = [&](int64_t c) { return D - c >= 8 ? 8 : static_cast<int>(D - c); };
    float sum[VS][8], gn[VS][8];
#pragma unroll
    for (int i = 0; i < VS; ++i) {
        const int64_t c = (static_cast<int64_t>(i) * TPR + t) * 8;
        const int n = left(c);
        load8(gain + (n > 0 ? c : 0), n, gn[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[i][j] = 0.f;
    }
    float* mine = partial + blockIdx.x * D;  // V = 0: the sums are kept here
    const int64_t stride = static_cast<int64_t>(gridDim.x) * ROWS;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * ROWS; first < R; first += stride) {
        const int64_t row = first + threadIdx.x / TPR;
        const bool in = row < R;  // TPR <= 64: a row's threads are lanes of one wave and agree
        if (TPR <= 64 && !in) break;
        const T* pd = dy + row * lddy;
        const T* ph = h + row * ldh;
        const float rstd = rstd_in[row];
        float d[VS][8], w[VS][8];
        float s = 0.f;
        for (int64_t i = 0; i < steps; ++i) {
            const int k = V > 0 ? static_cast<int>(i) : 0;
            const int64_t c = (i * TPR + t) * 8;
            const int n = left(c);
            if (V > 0) {  // read once: around the caches (16,384 x 4,096 bf16: 111 -> 107 us)
                pass8(pd + (n > 0 ? c : 0), n, d[k]);
                pass8(ph + (n > 0 ? c : 0), n, w[k]);
            } else {
                load8(pd + (n > 0 ? c : 0), n, d[k]);
                load8(ph + (n > 0 ? c : 0), n, w[k]);
            }
            if (V == 0) load8(gain + (n > 0 ? c : 0), n, gn[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[k][j] *= rstd;
                s = fmaf(d[k][j] * gn[k][j], w[k][j], s);
            }
        }
        const float mean = row_sum<TPR>(s, part) / static_cast<float>(D);
        for (int64_t i = 0; i < steps; ++i) {
            const int k = V > 0 ? static_cast<int>(i) : 0;
            const int64_t c = (i * TPR + t) * 8;
            const int n = left(c);
            if (n <= 0) continue;
            if (V == 0) {
                load8(pd + c, n, d[0]);
                load8(ph + c, n, w[0]);
                load8(gain + c, n, gn[0]);
#pragma unroll
                for (int j = 0; j < 8; ++j) w[0][j] *= rstd;
            }
            float o[8], e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                o[j] = rstd * (d[k][j] * gn[k][j] - w[k][j] * mean);
                if (V > 0) sum[k][j] = fmaf(d[k][j], w[k][j], sum[k][j]);
            }
            if (gh != nullptr) {
                pass8(gh + row * ldgh + c, n, e);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] += e[j];
            }
            store8(dx + row * lddx + c, n, o);
            if (V == 0 && partial != nullptr) {
                float m[8];
                const bool start = first == static_cast<int64_t>(blockIdx.x) * ROWS;
                if (start) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) m[j] = 0.f;
                } else {
                    load8(mine + c, n, m);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) m[j] = fmaf(d[0][j], w[0][j], m[j]);
                store8(mine + c, n, m);
            }
        }
    }
    if (V > 0 && partial != nullptr) {
        if constexpr (ROWS > 1) {  // the workgroup's rows in flight, in order
            __shared__ float all[THREADS][9];
#pragma unroll
            for (int i = 0; i < VS; ++i) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) all[threadIdx.x][j] = sum[i][j];
                __syncthreads();
                if (threadIdx.x < TPR) {
                    const int64_t c = (static_cast<int64_t>(i) * TPR + t) * 8;
                    float o[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        o[j] = 0.f;
#pragma unroll
                        for (int q = 0; q < ROWS; ++q) o[j] += all[q * TPR + t][j];
                    }
                    if (c < D) store8(mine + c, left(c), o);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < VS; ++i) {
                const int64_t c = (static_cast<int64_t>(i) * TPR + t) * 8;
                if (c < D) store8(mine + c, left(c), sum[i]);
            }
        }
    }
}

// dgain[d] = sum of the partial rows, in a fixed order, from column `first` on: 32 columns a workgroup, 32 row
// strides with eight rows in flight each
__global__ __launch_bounds__(1024) void norm_gain_kernel(const float* __restrict__ partial, float* __restrict__ dgain,
                                                         int n, int64_t D, int64_t first) {
    __shared__ float part[32][33];
    const int l = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t c = first + static_cast<int64_t>(blockIdx.x) * 32 + l;
    float s = 0.f;
    if (c < D) {
        for (int i = w; i < n; i += 256) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = i + 32 * j < n ? partial[(i + 32 * j) * D + c] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[j];
        }
    }
    part[w][l] = s;
    __syncthreads();
    if (w == 0 && c < D) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += part[i][l];
        dgain[c] = s;
    }
}

__global__ void norm_gain_zero_kernel(float* dgain, int64_t D) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c < D) dgain[c] = 0.f;
}

struct NormShape {
    int tpr, v;
};
constexpr int kForwardGroups = 4;   // a row in 32 registers
constexpr int kBackwardGroups = 2;  // two rows, the gain and its gradient: 64 registers

// Threads per row and column groups per thread.  Many rows: as few threads as hold the row in `groups_most`
// groups each (4,096 x 4,096 bf16 23 us, with one group a thread 33; 16,384 x 1,024 23 / 30).  Few rows: a group
// per thread, for latency (1 x 2,048 3.2 us, with four groups 5.9; 1,000 x 2,048 5.3 / 7.6).
NormShape norm_shape(int64_t R, int64_t D, int groups_most) {
    const int64_t groups = (D + 7) / 8;
    for (int tpr : {16, 64, 256, 1024}) {
        const int64_t v = (groups + tpr - 1) / tpr;
        const int64_t most = (R * tpr < 256 * 1024 && tpr < 1024) ? 1 : groups_most;
        if (v <= most) return {tpr, v <= 1 ? 1 : (v <= 2 ? 2 : 4)};
    }
    return {1024, 0};
}

template <typename T, int TPR, int V>
hipError_t norm_launch(const NormArgs& a, hipStream_t stream) {
    constexpr int THREADS = TPR > 256 ? TPR : 256, ROWS = THREADS / TPR;
    const int64_t blocks = (a.R + ROWS - 1) / ROWS;
    const dim3 grid(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks));
    if (a.values != nullptr)
        hipLaunchKernelGGL((rms_norm_kernel<T, TPR, V, true>), grid, dim3(THREADS), 0, stream,
                           static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.r), a.ldr, a.gain, a.eps,
                           static_cast<T*>(a.h), a.ldh, static_cast<T*>(a.y), a.ldy, a.values, a.scales, a.rstd, a.R,
                           a.D);
    else
        hipLaunchKernelGGL((rms_norm_kernel<T, TPR, V, false>), grid, dim3(THREADS), 0, stream,
                           static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.r), a.ldr, a.gain, a.eps,
                           static_cast<T*>(a.h), a.ldh, static_cast<T*>(a.y), a.ldy, a.values, a.scales, a.rstd, a.R,
                           a.D);
    return hipGetLastError();
}

template <typename T, int TPR, int V>
hipError_t norm_bwd_launch(const NormBwdArgs& a, hipStream_t stream) {
    constexpr int THREADS = TPR > 256 ? TPR : 256;
    const unsigned grid = static_cast<unsigned>(norm_bwd_blocks(a.R, a.D));
    hipLaunchKernelGGL((rms_norm_bwd_kernel<T, TPR, V>), dim3(grid), dim3(THREADS), 0, stream,
                       static_cast<const T*>(a.dy), a.lddy, static_cast<const T*>(a.h), a.ldh, a.rstd, a.gain,
                       static_cast<const T*>(a.gh), a.ldgh, static_cast<T*>(a.dx), a.lddx,
                       a.dgain != nullptr ? a.partial : nullptr, a.R, a.D);
    hipError_t e = hipGetLastError();
    constexpr int64_t kColumns = 32 * kMostBlocks;  // of a launch
    for (int64_t first = 0; a.dgain != nullptr && e == hipSuccess && first < a.D; first += kColumns) {
        const int64_t columns = a.D - first < kColumns ? a.D - first : kColumns;
        hipLaunchKernelGGL(norm_gain_kernel, dim3(static_cast<unsigned>((columns + 31) / 32)), dim3(1024), 0, stream,
                           a.partial, a.dgain, static_cast<int>(grid), a.D, first);
        e = hipGetLastError();
    }
    return e;
}

#define NORM_SHAPES(CALL, MORE)                                               \
    switch (s.tpr * 8 + s.v) {                                                \
        MORE(CALL)                                                            \
        case 16 * 8 + 1: return CALL(16, 1);                                  \
        case 16 * 8 + 2: return CALL(16, 2);                                  \
        case 64 * 8 + 1: return CALL(64, 1);                                  \
        case 64 * 8 + 2: return CALL(64, 2);                                  \
        case 256 * 8 + 1: return CALL(256, 1);                                \
        case 256 * 8 + 2: return CALL(256, 2);                                \
        case 1024 * 8 + 1: return CALL(1024, 1);                              \
        case 1024 * 8 + 2: return CALL(1024, 2);                              \
        default: return CALL(1024, 0);                                        \
    }

#define NORM_FOUR(CALL)                     \
    case 16 * 8 + 4: return CALL(16, 4);    \
    case 64 * 8 + 4: return CALL(64, 4);    \
    case 256 * 8 + 4: return CALL(256, 4);  \
    case 1024 * 8 + 4: return CALL(1024, 4);
#define NORM_NO_MORE(CALL)

template <typename T>
hipError_t norm_dispatch(const NormArgs& a, hipStream_t stream) {
    const NormShape s = norm_shape(a.R, a.D, kForwardGroups);
#define CALL(TPR, V) (norm_launch<T, TPR, V>(a, stream))
    NORM_SHAPES(CALL, NORM_FOUR)
#undef CALL
}

template <typename T>
hipError_t norm_bwd_dispatch(const NormBwdArgs& a, hipStream_t stream) {
    const NormShape s = norm_shape(a.R, a.D, kBackwardGroups);
#define CALL(TPR, V) (norm_bwd_launch<T, TPR, V>(a, stream))
    NORM_SHAPES(CALL, NORM_NO_MORE)
#undef CALL
}

}  // namespace

int64_t norm_bwd_blocks(int64_t R, int64_t D) {
    const NormShape s = norm_shape(R, D, kBackwardGroups);
    const int64_t rows = s.tpr >= 256 ? 1 : 256 / s.tpr;
    const int64_t all = (R + rows - 1) / rows;
    const int64_t most = s.tpr > 256 ? 256 : 1024;  // 4 waves a SIMD; a partial row of dgain each
    return all < most ? all : most;
}

hipError_t launch_rms_norm(int dtype, const NormArgs& a, hipStream_t stream) {
    return dtype == SPINGTP_FP32 ? norm_dispatch<float>(a, stream) : norm_dispatch<uint16_t>(a, stream);
}

hipError_t launch_rms_norm_bwd(int dtype, const NormBwdArgs& a, hipStream_t stream) {
    if (a.R == 0) {  // no rows: the gain's gradient is zero
        if (a.dgain != nullptr && a.D > 0)
            hipLaunchKernelGGL(norm_gain_zero_kernel, dim3(static_cast<unsigned>((a.D + 255) / 256)), dim3(256), 0,
                               stream, a.dgain, a.D);
        return hipGetLastError();
    }
    return dtype == SPINGTP_FP32 ? norm_bwd_dispatch<float>(a, stream) : norm_bwd_dispatch<uint16_t>(a, stream);
}

}  // namespace spingtp
