// The gated feed-forward block:
//   g = x Wg^T,  u = x Wu^T,  h = act(g) u
// and its gradients
//   dg = dh u act'(g),  du = dh act(g),  dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x.
//
// Forward: one kernel.  A workgroup's tile takes the same 128 outputs from both weight matrices, so
// the lane that holds an output's g holds its u, and h leaves from registers; g and u are written
// only where the backward pass is to have them, in bf16 or as 8-bit blocks (a tile's 128 columns are
// one block of each of its rows).
//
// Backward: dg and du are computed once and written side by side, [M][g | u]; then dx is one product of them
// with the weights, and both weight gradients are one product over M.  The weights' rows and, for the
// weight gradients, both operands' run across the summed axis: the products read them as they are.  An
// 8-bit checkpoint of x is unpacked first.  dg and du are rounded to bf16, as operands of the matrix
// units; sums are fp32.
//
// Bound by power and by what leaves between rounds of tiles.  Measured at 8,192 x 2,048 x 8,192 (550 GFLOP a
// product): forward 404-450 us (8-bit operands 403), 465-480 with g and u kept in bf16, 482-498 in 8 bits; dg and du
// 110 us, 6.1 TB/s; dx 420-470 us, dW 440-460 us, 1.2-1.3 PFLOP/s.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "activation.h"
#include "feedforward.h"
#include "gemm_nt.h"
#include "gemm_skinny.h"
#include "internal.h"
#include "lds_common.h"

namespace spingtp {
namespace {

struct GatedOut {
    void* h;
    int64_t ldh;
    uint8_t* h_scales;
    void* g;
    void* u;
    uint8_t* g_scales;
    uint8_t* u_scales;
    int64_t pitch, spitch;  // of the 8-bit rows
};

// A tile's outputs go through LDS, so that a row's columns leave as whole lines, 16 bytes a lane.
// `value(i, j, r)` is column column(i, r / 4) + r % 4 of row row(j).
constexpr int kPad = 16;  // bytes of an LDS row past its columns: rows start in different banks

// bf16: each wave's own PM rows of PN / 2 columns, in its own place, without barriers.
template <class Tile>
struct WaveOut {
    static constexpr int kColumns = Tile::kRows / Tile::kWavesN, kRows = Tile::TM * Tile::kTile;
    static constexpr int kPitch = 2 * kColumns + kPad, kBytes = kRows * kPitch;
    static constexpr int kLanes = kColumns / 8;  // of a row

    template <class V>
    static __device__ __forceinline__ void stage(const Tile& t, uint8_t* mine, const V& value) {
        const int row = t.wm * kRows, column = t.wn * kColumns;
#pragma unroll
        for (int j = 0; j < Tile::TM; ++j)
#pragma unroll
            for (int i = 0; i < Tile::TN / 2; ++i)
#pragma unroll
                for (int r = 0; r < Tile::kQuads; ++r)
                    *reinterpret_cast<uint2*>(mine + (t.row(j) - row) * kPitch + 2 * (t.column(i, r) - column)) =
                        make_uint2(bf16_pair(value(i, j, 4 * r), value(i, j, 4 * r + 1)),
                                   bf16_pair(value(i, j, 4 * r + 2), value(i, j, 4 * r + 3)));
    }
    static __device__ __forceinline__ void send(const Tile& t, const uint8_t* mine, const GemmArgs& a, int64_t n0,
                                                int64_t m0, void* out, int64_t ldo) {
        constexpr int kAtOnce = 64 / kLanes;
        const int l = t.lane % kLanes, r0 = t.lane / kLanes;
        const int64_t left = a.N - n0 - t.wn * kColumns - 8 * l, m = m0 + t.wm * kRows + r0, rows = a.M - m;
        uint16_t* p = static_cast<uint16_t*>(out) + m * ldo + n0 + t.wn * kColumns + 8 * l;
        uint4 v[kRows / kAtOnce];
#pragma unroll
        for (int q = 0; q < kRows / kAtOnce; ++q)
            v[q] = *reinterpret_cast<const uint4*>(mine + (r0 + q * kAtOnce) * kPitch + 16 * l);
#pragma unroll
        for (int q = 0; q < kRows / kAtOnce; ++q) {
            uint16_t* to = p + q * kAtOnce * ldo;
            if (q * kAtOnce >= rows) continue;
            if (left >= 8) {
                *reinterpret_cast<u4u*>(to) = u4u{v[q].x, v[q].y, v[q].z, v[q].w};
            } else {
                const uint32_t w[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
#pragma unroll
                for (int b = 0; b < 8; ++b)
                    if (b < left) to[b] = static_cast<uint16_t>(w[b / 2] >> (16 * (b & 1)));
            }
        }
    }
};

// The rows as 8-bit blocks: first each wave's largest magnitudes (tops [WN][BM]), then, when all are there,
// the values.
template <class Tile, class V>
__device__ __forceinline__ void block_tops(const Tile& t, float* tops, const V& value) {
#pragma unroll
    for (int j = 0; j < Tile::TM; ++j) {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < Tile::TN / 2; ++i)
#pragma unroll
            for (int r = 0; r < 4 * Tile::kQuads; ++r) top = fmaxf(top, fabsf(value(i, j, r)));
        if (!(top < __builtin_inff())) {
            top = 0.f;
#pragma unroll
            for (int i = 0; i < Tile::TN / 2; ++i)
#pragma unroll
                for (int r = 0; r < 4 * Tile::kQuads; ++r) top = fmaxf(top, finite_abs(value(i, j, r)));
        }
        if constexpr (Tile::kTile == 16) top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        if (t.lane < Tile::kTile) tops[t.wn * Tile::BM + t.row(j)] = top;
    }
}
template <class Tile, int WN, class V>
__device__ __forceinline__ void stage_blocks(const Tile& t, const GemmArgs& a, int64_t n0, int64_t m0,
                                             const float* tops, uint8_t* lds, uint8_t* scales, int64_t spitch,
                                             const V& value) {
    constexpr int PITCH = kBlock8 + kPad;
#pragma unroll
    for (int j = 0; j < Tile::TM; ++j) {
        float top = 0.f;
#pragma unroll
        for (int w = 0; w < WN; ++w) top = fmaxf(top, tops[w * Tile::BM + t.row(j)]);
        const int e = block8_scale(top);
        const float inv = block8_inverse(e);
#pragma unroll
        for (int i = 0; i < Tile::TN / 2; ++i)
#pragma unroll
            for (int r = 0; r < Tile::kQuads; ++r)
                *reinterpret_cast<uint32_t*>(lds + t.row(j) * PITCH + t.column(i, r)) =
                    block8_word(value(i, j, 4 * r), value(i, j, 4 * r + 1), value(i, j, 4 * r + 2),
                                value(i, j, 4 * r + 3), inv);
        const int64_t m = m0 + t.row(j);
        if (t.wn == 0 && t.lane < Tile::kTile && m < a.M) {
            uint8_t* s = scales + m * spitch + n0 / kBlock8;
            s[0] = static_cast<uint8_t>(e);
            if (n0 + kBlock8 >= a.N)  // the row's scale bytes past its last block
                for (int64_t b = n0 / kBlock8 + 1; b < spitch; ++b) scales[m * spitch + b] = 127;
        }
    }
}
template <class Tile>
__device__ __forceinline__ void send_blocks(const uint8_t* lds, const GemmArgs& a, int64_t n0, int64_t m0, void* out,
                                            int64_t pitch) {
    constexpr int PITCH = kBlock8 + kPad;
    const int l = threadIdx.x & 7;
    const int rows = a.M - m0 < Tile::BM ? static_cast<int>(a.M - m0) : Tile::BM;
    uint8_t* p = static_cast<uint8_t*>(out) + m0 * pitch + n0 + 16 * l;  // a block lies in the pitch as a whole
    constexpr int kAtOnce = Tile::kThreads / 8;
    const int r0 = threadIdx.x >> 3;
    uint4 v[Tile::BM / kAtOnce];
#pragma unroll
    for (int q = 0; q < Tile::BM / kAtOnce; ++q)
        v[q] = *reinterpret_cast<const uint4*>(lds + (r0 + q * kAtOnce) * PITCH + 16 * l);
#pragma unroll
    for (int q = 0; q < Tile::BM / kAtOnce; ++q)
        if (r0 + q * kAtOnce < rows) *reinterpret_cast<uint4*>(p + (r0 + q * kAtOnce) * pitch) = v[q];
}

template <class E, int PN, int PM, int WN, int WM, int NS, int ACT, int SAVE, bool OUT8>
__global__ __launch_bounds__(64 * WN * WM) void gated_kernel(GemmArgs a, GatedOut o) {
    using Tile = GemmTile<E, PN, PM, WN, WM, NS, true>;
    static_assert(Tile::kRows == kBlock8, "a tile is one block of its rows");
    constexpr int HALF = Tile::TN / 2, BM = Tile::BM;
    using Out = WaveOut<Tile>;
    constexpr int kPlace = BM * (kBlock8 + kPad);  // of 8-bit rows
    extern __shared__ __align__(16) uint8_t gemm_lds[];
    uint8_t* const place[2] = {gemm_lds, gemm_lds + kPlace};
    uint8_t* const own = gemm_lds + (threadIdx.x >> 6) * 2 * Out::kBytes;
    uint8_t* const mine[2] = {own, own + Out::kBytes};
    float* const tops = reinterpret_cast<float*>(gemm_lds + 2 * kPlace);
    float* const tops2 = tops + WN * BM;
    int tm, tn;
    tile_of(a.tiles_m, a.tiles_n, tm, tn);
    const int64_t n0 = static_cast<int64_t>(tn) * Tile::kRows, m0 = static_cast<int64_t>(tm) * BM;
    Tile t;
    t.run(a, n0, m0, gemm_lds);  // ends with a barrier behind its reads of LDS
    const auto g = [&](int i, int j, int r) { return t.acc[i][j][r]; };
    const auto u = [&](int i, int j, int r) { return t.acc[HALF + i][j][r]; };
    if ((SAVE == kSave8 || OUT8) && n0 + kBlock8 > a.N) {  // 8-bit rows end in zeros
#pragma unroll
        for (int i = 0; i < HALF; ++i)
#pragma unroll
            for (int r = 0; r < 4 * Tile::kQuads; ++r)
                if (n0 + t.column(i, r / 4) + r % 4 >= a.N) {
#pragma unroll
                    for (int j = 0; j < Tile::TM; ++j) t.acc[i][j][r] = t.acc[HALF + i][j][r] = 0.f;
                }
    }
    if constexpr (SAVE == kSaveBf16) {
        Out::stage(t, mine[0], g);
        Out::stage(t, mine[1], u);
    }
    if constexpr (SAVE == kSave8) {
        block_tops(t, tops, g);
        block_tops(t, tops2, u);
        __syncthreads();
        stage_blocks<Tile, WN>(t, a, n0, m0, tops, place[0], o.g_scales, o.spitch, g);
        stage_blocks<Tile, WN>(t, a, n0, m0, tops2, place[1], o.u_scales, o.spitch, u);
        __syncthreads();
        send_blocks<Tile>(place[0], a, n0, m0, o.g, o.pitch);
        send_blocks<Tile>(place[1], a, n0, m0, o.u, o.pitch);
    }
    __builtin_amdgcn_sched_barrier(0);  // here and below: for registers
#pragma unroll
    for (int i = 0; i < HALF; ++i)
#pragma unroll
        for (int j = 0; j < Tile::TM; ++j) {
#pragma unroll
            for (int r = 0; r < 4 * Tile::kQuads; ++r) {
                float h = act<ACT>(t.acc[i][j][r]) * t.acc[HALF + i][j][r];
                asm volatile("" : "+v"(h));  // computed here, not half of it where it is used
                t.acc[i][j][r] = h;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    if constexpr (SAVE == kSaveBf16) {
        wave_lds_order();
        Out::send(t, mine[0], a, n0, m0, o.g, a.N);
        __builtin_amdgcn_sched_barrier(0);
        Out::send(t, mine[1], a, n0, m0, o.u, a.N);
    }
    if constexpr (SAVE == kSave8 || (OUT8 && SAVE != kSaveNone)) __syncthreads();  // g and u have left their places
    if constexpr (OUT8) {
        block_tops(t, tops, g);
        __syncthreads();
        stage_blocks<Tile, WN>(t, a, n0, m0, tops, place[0], o.h_scales, o.spitch, g);
        __syncthreads();
        send_blocks<Tile>(place[0], a, n0, m0, o.h, o.pitch);
    } else {
        wave_lds_order();
        Out::stage(t, mine[0], g);
        wave_lds_order();
        Out::send(t, mine[0], a, n0, m0, o.h, o.ldh);
    }
}

// At most kSkinnyRows rows of x.  What is to be 8-bit blocks leaves in fp32 [M][F] and is packed next (a
// block's 128 columns are eight workgroups'): h with OUT32, g and u with SAVE = kSave8.
template <class E, int TM, int ACT, int SAVE, bool OUT32>
__global__ __launch_bounds__(64 * kSkinnyWaves) void gated_skinny_kernel(GemmArgs a, int64_t row_bytes, GatedOut o) {
    skinny_tile<E, TM, true>(a, row_bytes, static_cast<int64_t>(blockIdx.x) * 16,
                             [&](int64_t m, int64_t n, float g, float u) {
                                 if constexpr (SAVE == kSaveBf16) {
                                     put(static_cast<uint16_t*>(o.g) + m * a.N + n, g);
                                     put(static_cast<uint16_t*>(o.u) + m * a.N + n, u);
                                 }
                                 if constexpr (SAVE == kSave8) {
                                     put(static_cast<float*>(o.g) + m * a.N + n, g);
                                     put(static_cast<float*>(o.u) + m * a.N + n, u);
                                 }
                                 const float h = act<ACT>(g) * u;
                                 if constexpr (OUT32)
                                     put(static_cast<float*>(o.h) + m * a.N + n, h);
                                 else
                                     put(static_cast<uint16_t*>(o.h) + m * o.ldh + n, h);
                             });
}

// Rows of K bf16 elements to rows of a multiple of 64, zeros behind: what the products read where the
// caller's rows do not start and end on 16 bytes.
__global__ __launch_bounds__(256) void stage_rows_kernel(const uint16_t* __restrict__ x, int64_t ldx,
                                                         uint16_t* __restrict__ out, int64_t R, int64_t K,
                                                         int64_t pitch) {
    const int64_t groups = pitch / 8, stride = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < R * groups; i += stride) {
        const int64_t row = i / groups, c = (i - row * groups) * 8, left = K - c;
        float v[8];
        load8(x + row * ldx + (left > 0 ? c : 0), left >= 8 ? 8 : static_cast<int>(left), v);
        store8(out + row * pitch + c, 8, v);
    }
}

// dg and du side by side, [M][2 Fp] (Fp: F up to a multiple of 64, zeros behind): 8 neighbouring columns of both
// per thread.  Everything passes through once, g, u and dh around the caches.
template <int ACT, bool IN8>
__global__ __launch_bounds__(256) void gated_grad_kernel(const uint16_t* __restrict__ dh, int64_t lddh,
                                                         const void* __restrict__ g, const void* __restrict__ u,
                                                         const uint8_t* __restrict__ gs,
                                                         const uint8_t* __restrict__ us, uint16_t* __restrict__ both,
                                                         int64_t M, int64_t F) {
    const int64_t fp = (F + 63) / 64 * 64, stride = static_cast<int64_t>(gridDim.x) * 256;
    const uint32_t groups = static_cast<uint32_t>(fp / 8);
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < M * groups; at += stride) {
        const int64_t m = at / groups, f = (at - m * groups) * 8, left = F - f;
        const int n = left >= 8 ? 8 : static_cast<int>(left);
        const int64_t c = n > 0 ? f : 0;
        float d[8], a[8], b[8];
        pass8(dh + m * lddh + c, n, d);
        if constexpr (IN8) {
            const int64_t p = m * block8_pitch(F) + f, q = m * block8_scale_pitch(F) + f / kBlock8;  // f < the pitch
            const uint2 wa = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(g) + p);
            const uint2 wb = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(u) + p);
            const float sa = block8_power(gs[q]), sb = block8_power(us[q]);
            float lo[4], hi[4];
            block8_values(wa.x, lo);
            block8_values(wa.y, hi);
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = lo[j] * sa, a[4 + j] = hi[j] * sa;
            block8_values(wb.x, lo);
            block8_values(wb.y, hi);
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = lo[j] * sb, b[4 + j] = hi[j] * sb;
        } else {
            pass8(static_cast<const uint16_t*>(g) + m * F + c, n, a);
            pass8(static_cast<const uint16_t*>(u) + m * F + c, n, b);
        }
        float dg[8], du[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float y, dy;
            act_grad<ACT>(a[j], y, dy);
            dg[j] = j < n ? d[j] * b[j] * dy : 0.f;
            du[j] = j < n ? d[j] * y : 0.f;
        }
        store8(both + m * 2 * fp + f, 8, dg);
        store8(both + m * 2 * fp + fp + f, 8, du);
    }
}

__global__ __launch_bounds__(256) void zero_kernel(uint16_t* p, int64_t n) {
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += stride) p[i] = 0;
}

// of 256 threads, for kernels that walk what is left
dim3 walking_grid(int64_t threads) {
    const int64_t blocks = (threads + 255) / 256;
    return dim3(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks));
}

// LDS of a workgroup: the operands' tiles, then the outputs'
template <class Tile, int WN>
constexpr int gated_lds() {
    constexpr int blocks = 2 * Tile::BM * (kBlock8 + kPad) + 2 * WN * Tile::BM * 4;
    constexpr int rows = 2 * Tile::kWaves * WaveOut<Tile>::kBytes, out = blocks > rows ? blocks : rows;
    static_assert(out <= 160 * 1024, "in LDS");
    return out > Tile::kLds ? out : Tile::kLds;
}

template <class E, int PN, int PM, int WN, int WM, int NS, int ACT, int SAVE, bool OUT8>
hipError_t gated_launch(GemmArgs g, const GatedOut& o, hipStream_t stream) {
    using Tile = GemmTile<E, PN, PM, WN, WM, NS, true>;
    const int64_t tm = (g.M + Tile::BM - 1) / Tile::BM, tn = (g.N + Tile::kRows - 1) / Tile::kRows;
    if (tm * tn > kMostTiles) return hipErrorInvalidValue;
    g.tiles_m = static_cast<int>(tm);
    g.tiles_n = static_cast<int>(tn);
    constexpr auto kernel = gated_kernel<E, PN, PM, WN, WM, NS, ACT, SAVE, OUT8>;
    const hipError_t e = raise_lds_limit<kernel>();
    if (e != hipSuccess) return e;
    constexpr int lds = gated_lds<Tile, WN>();
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(tm * tn)), dim3(Tile::kThreads), lds, stream, g, o);
    return hipGetLastError();
}

template <class E, int ACT, int SAVE, bool OUT8>
hipError_t gated_tiles(const GemmArgs& g, const GatedOut& o, hipStream_t stream) {
    switch (gated_tile(g.M, g.N)) {
        case 256: return gated_launch<E, 128, 64, 2, 4, 2, ACT, SAVE, OUT8>(g, o, stream);
        case 128: return gated_launch<E, 64, 64, 4, 2, 3, ACT, SAVE, OUT8>(g, o, stream);
        default: return gated_launch<E, 64, 32, 4, 2, 2, ACT, SAVE, OUT8>(g, o, stream);
    }
}

// Few rows of x, us against the smallest tile's (bf16): one row, 1,024^2 weights 6.0 / 9.5, 4,096^2 13.6 / 43.8,
// 8,192 x 2,048 13.3 / 23.9; 64 rows 8.0 / 9.7, 25.1 / 46.9, 25.7 / 25.8.
template <class E, int ACT, int SAVE, bool OUT32>
hipError_t gated_skinny(const GemmArgs& g, int64_t row_bytes, const GatedOut& o, hipStream_t stream) {
    const int64_t blocks = (g.N + 15) / 16;
    if (blocks > kMostTiles) return hipErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(blocks)), threads(64 * kSkinnyWaves);
    if (g.M <= 16)
        hipLaunchKernelGGL((gated_skinny_kernel<E, 1, ACT, SAVE, OUT32>), grid, threads, 0, stream, g, row_bytes, o);
    else if (g.M <= 32)
        hipLaunchKernelGGL((gated_skinny_kernel<E, 2, ACT, SAVE, OUT32>), grid, threads, 0, stream, g, row_bytes, o);
    else
        hipLaunchKernelGGL((gated_skinny_kernel<E, 4, ACT, SAVE, OUT32>), grid, threads, 0, stream, g, row_bytes, o);
    return hipGetLastError();
}

template <class E, int SAVE, bool OUT32>
hipError_t gated_skinny_act(int act, const GemmArgs& g, int64_t row_bytes, const GatedOut& o, hipStream_t stream) {
    return act == kSilu ? gated_skinny<E, kSilu, SAVE, OUT32>(g, row_bytes, o, stream)
                        : gated_skinny<E, kGelu, SAVE, OUT32>(g, row_bytes, o, stream);
}

template <class E, int SAVE, bool OUT8>
hipError_t gated_act(int act, const GemmArgs& g, const GatedOut& o, hipStream_t stream) {
    return act == kSilu ? gated_tiles<E, kSilu, SAVE, OUT8>(g, o, stream)
                        : gated_tiles<E, kGelu, SAVE, OUT8>(g, o, stream);
}

// whether the products can read these rows as they are
bool rows_fit(int64_t K, int64_t ld) { return K % 8 == 0 && ld % 8 == 0 && 2 * ld <= kMostRowBytes; }
int64_t up64(int64_t n) { return (n + 63) / 64 * 64; }

hipError_t stage(const void* x, int64_t ldx, uint16_t* out, int64_t R, int64_t K, hipStream_t stream) {
    const int64_t pitch = up64(K);
    hipLaunchKernelGGL(stage_rows_kernel, walking_grid(R * (pitch / 8)), dim3(256), 0, stream,
                       static_cast<const uint16_t*>(x), ldx, out, R, K, pitch);
    return hipGetLastError();
}

// The gradients' products: w's columns run along the summed axis, x's with KX.
template <int PN, int PM, int WN, int WM, int NS, bool KX>
hipError_t product_launch(GemmArgs g, void* c, int64_t ldc, hipStream_t stream) {
    using Tile = GemmTile<Bf16, PN, PM, WN, WM, NS, false, true, KX>;
    const int64_t tm = (g.M + Tile::BM - 1) / Tile::BM, tn = (g.N + Tile::BN - 1) / Tile::BN;
    if (tm * tn > kMostTiles) return hipErrorInvalidValue;
    g.tiles_m = static_cast<int>(tm);
    g.tiles_n = static_cast<int>(tn);
    constexpr auto kernel = gemm_nt_kernel<Bf16, PN, PM, WN, WM, NS, uint16_t, true, KX>;
    const hipError_t e = raise_lds_limit<kernel>();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(tm * tn)), dim3(Tile::kThreads), Tile::kLds, stream, g,
                       static_cast<uint16_t*>(c), ldc);
    return hipGetLastError();
}
template <bool KX>
hipError_t product(GemmArgs g, void* c, int64_t ldc, hipStream_t stream) {
    g.tail = kStepBytes;
    switch (product_tile(kPlain16, g.M, g.N)) {
        case 256: return product_launch<128, 64, 2, 4, 2, KX>(g, c, ldc, stream);
        case 128: return product_launch<64, 32, 2, 4, 2, KX>(g, c, ldc, stream);
        default: return product_launch<32, 32, 2, 2, 4, KX>(g, c, ldc, stream);
    }
}

template <int ACT>
hipError_t gated_grad(const GatedBwdArgs& a, uint16_t* both, hipStream_t stream) {
    const dim3 grid = walking_grid(a.M * (up64(a.F) / 8));
    const uint16_t* dh = static_cast<const uint16_t*>(a.dh);
    if (a.save == kSave8)
        hipLaunchKernelGGL((gated_grad_kernel<ACT, true>), grid, dim3(256), 0, stream, dh, a.lddh, a.g, a.u, a.g_scales,
                           a.u_scales, both, a.M, a.F);
    else
        hipLaunchKernelGGL((gated_grad_kernel<ACT, false>), grid, dim3(256), 0, stream, dh, a.lddh, a.g, a.u,
                           a.g_scales, a.u_scales, both, a.M, a.F);
    return hipGetLastError();
}

}  // namespace

size_t gated_workspace(int64_t M, int64_t K, int64_t F, int64_t ldx, int64_t ldw, int save) {
    if (M <= kSkinnyRows) return save == kSave8 ? static_cast<size_t>(2 * M * F) * sizeof(float) : 0;
    const int64_t pitch = up64(K) * 2;
    return static_cast<size_t>((rows_fit(K, ldx) ? 0 : M * pitch) + (rows_fit(K, ldw) ? 0 : 2 * F * pitch));
}

hipError_t launch_gated(const GatedArgs& a, hipStream_t stream) {
    const int64_t pitch = up64(a.K);
    uint16_t* ws = static_cast<uint16_t*>(a.workspace);
    GemmArgs g{};
    g.M = a.M;
    g.N = a.F;
    g.x = static_cast<const uint8_t*>(a.x);
    g.w = static_cast<const uint8_t*>(a.wg);
    g.w2 = static_cast<const uint8_t*>(a.wu);
    g.ldx = 2 * a.ldx;
    g.ldw = 2 * a.ldw;
    const GatedOut o{a.h, a.ldh, nullptr, a.g, a.u, a.g_scales, a.u_scales, block8_pitch(a.F), block8_scale_pitch(a.F)};
    if (a.M <= kSkinnyRows) {  // rows of any alignment are read as they are
        g.steps = static_cast<int>(pitch / 64);
        if (a.save == kSaveNone) return gated_skinny_act<Bf16, kSaveNone, false>(a.act, g, 2 * a.K, o, stream);
        if (a.save == kSaveBf16) return gated_skinny_act<Bf16, kSaveBf16, false>(a.act, g, 2 * a.K, o, stream);
        GatedOut to32 = o;
        to32.g = ws;
        to32.u = reinterpret_cast<float*>(ws) + a.M * a.F;
        hipError_t e = gated_skinny_act<Bf16, kSave8, false>(a.act, g, 2 * a.K, to32, stream);
        if (e == hipSuccess)
            e = launch_pack8(SPINGTP_FP32, to32.g, a.F, static_cast<uint8_t*>(a.g), a.g_scales, nullptr, nullptr, a.M,
                             a.F, stream);
        if (e == hipSuccess)
            e = launch_pack8(SPINGTP_FP32, to32.u, a.F, static_cast<uint8_t*>(a.u), a.u_scales, nullptr, nullptr, a.M,
                             a.F, stream);
        return e;
    }
    hipError_t e = hipSuccess;
    if (!rows_fit(a.K, a.ldx)) {
        e = stage(a.x, a.ldx, ws, a.M, a.K, stream);
        g.x = reinterpret_cast<const uint8_t*>(ws);
        g.ldx = 2 * pitch;
        ws += a.M * pitch;
    }
    if (e == hipSuccess && !rows_fit(a.K, a.ldw)) {
        e = stage(a.wg, a.ldw, ws, a.F, a.K, stream);
        if (e == hipSuccess) e = stage(a.wu, a.ldw, ws + a.F * pitch, a.F, a.K, stream);
        g.w = reinterpret_cast<const uint8_t*>(ws);
        g.w2 = reinterpret_cast<const uint8_t*>(ws + a.F * pitch);
        g.ldw = 2 * pitch;
    }
    if (e != hipSuccess) return e;
    // a staged row next to one that is not has zeros where the other has none: K up to 8 elements
    g.steps = static_cast<int>(pitch / 64);
    const int64_t held = (a.K + 7) / 8 * 16 - (g.steps - 1) * static_cast<int64_t>(kStepBytes);
    g.tail = static_cast<int>(held);
    switch (a.save) {
        case kSaveNone: return gated_act<Bf16, kSaveNone, false>(a.act, g, o, stream);
        case kSaveBf16: return gated_act<Bf16, kSaveBf16, false>(a.act, g, o, stream);
        default: return gated_act<Bf16, kSave8, false>(a.act, g, o, stream);
    }
}

size_t gated8_workspace(int64_t M, int64_t F, bool out8) {
    return out8 && M <= kSkinnyRows ? static_cast<size_t>(M * F) * sizeof(float) : 0;
}

hipError_t launch_gated8(const GatedArgs& a, hipStream_t stream) {
    GemmArgs g{};
    g.M = a.M;
    g.N = a.F;
    g.x = static_cast<const uint8_t*>(a.x);
    g.w = static_cast<const uint8_t*>(a.wg);
    g.w2 = static_cast<const uint8_t*>(a.wu);
    g.ldx = g.ldw = block8_pitch(a.K);
    g.xs = a.x_scales;
    g.ws = a.wg_scales;
    g.ws2 = a.wu_scales;
    g.lds = block8_scale_pitch(a.K);
    g.steps = static_cast<int>(g.ldx / kStepBytes);
    g.tail = kStepBytes;
    const GatedOut o{a.h,     a.ldh,   a.h_scales, nullptr, nullptr, nullptr, nullptr, block8_pitch(a.F),
                     block8_scale_pitch(a.F)};
    if (a.M <= kSkinnyRows) {
        if (a.h_scales == nullptr) return gated_skinny_act<Fp8, kSaveNone, false>(a.act, g, 0, o, stream);
        GatedOut to32 = o;
        to32.h = a.workspace;
        const hipError_t e = gated_skinny_act<Fp8, kSaveNone, true>(a.act, g, 0, to32, stream);
        if (e != hipSuccess) return e;
        return launch_pack8(SPINGTP_FP32, a.workspace, a.F, static_cast<uint8_t*>(a.h), a.h_scales, nullptr, nullptr,
                            a.M, a.F, stream);
    }
    return a.h_scales != nullptr ? gated_act<Fp8, kSaveNone, true>(a.act, g, o, stream)
                                 : gated_act<Fp8, kSaveNone, false>(a.act, g, o, stream);
}

size_t gated_backward_workspace(int64_t M, int64_t K, int64_t F, int64_t ldx, int64_t ldw, bool x8) {
    const int64_t x = x8 || !rows_fit(K, ldx) ? M * up64(K) : 0, w = rows_fit(K, ldw) ? 0 : 2 * F * up64(K);
    return static_cast<size_t>(2 * (M * 2 * up64(F) + x + w));
}

hipError_t launch_gated_backward(const GatedBwdArgs& a, hipStream_t stream) {
    if (a.M == 0) {
        if (a.dw == nullptr) return hipSuccess;
        const int64_t n = 2 * a.F * a.K;
        hipLaunchKernelGGL(zero_kernel, walking_grid(n), dim3(256), 0, stream, static_cast<uint16_t*>(a.dw), n);
        return hipGetLastError();
    }
    const int64_t fp = up64(a.F), kp = up64(a.K);
    uint16_t* both = static_cast<uint16_t*>(a.workspace);
    uint16_t* free_at = both + a.M * 2 * fp;
    hipError_t e = a.act == kSilu ? gated_grad<kSilu>(a, both, stream) : gated_grad<kGelu>(a, both, stream);
    if (e == hipSuccess && a.dx != nullptr) {
        GemmArgs g{};
        g.x = reinterpret_cast<const uint8_t*>(both);
        g.ldx = 4 * fp;
        g.w = static_cast<const uint8_t*>(a.wg);
        g.w2 = static_cast<const uint8_t*>(a.wu);
        g.ldw = 2 * a.ldw;
        if (!rows_fit(a.K, a.ldw)) {
            e = stage(a.wg, a.ldw, free_at, a.F, a.K, stream);
            if (e == hipSuccess) e = stage(a.wu, a.ldw, free_at + a.F * kp, a.F, a.K, stream);
            g.w = reinterpret_cast<const uint8_t*>(free_at);
            g.w2 = reinterpret_cast<const uint8_t*>(free_at + a.F * kp);
            g.ldw = 2 * kp;
            free_at += 2 * a.F * kp;
        }
        g.M = a.M;
        g.N = a.K;
        g.steps = static_cast<int>(2 * fp / 64);
        g.w_rows = a.F;
        g.w_split = static_cast<int>(fp / 64);
        if (e == hipSuccess) e = product<false>(g, a.dx, a.lddx, stream);
    }
    if (e == hipSuccess && a.dw != nullptr) {
        GemmArgs g{};
        if (a.x_scales == nullptr && rows_fit(a.K, a.ldx)) {
            g.w = static_cast<const uint8_t*>(a.x);
            g.ldw = 2 * a.ldx;
        } else {
            g.w = reinterpret_cast<const uint8_t*>(free_at);
            g.ldw = 2 * kp;
        }
        if (a.x_scales != nullptr) {
            e = launch_unpack8(SPINGTP_BF16, static_cast<const uint8_t*>(a.x), a.x_scales, free_at, kp, a.M, a.K, stream);
        } else if (!rows_fit(a.K, a.ldx)) {
            e = stage(a.x, a.ldx, free_at, a.M, a.K, stream);
        }
        g.w2 = g.w;
        g.x = reinterpret_cast<const uint8_t*>(both);
        g.ldx = 4 * fp;
        g.M = fp + a.F;
        g.N = a.K;
        g.steps = static_cast<int>((a.M + 63) / 64);
        g.w_rows = g.x_rows = a.M;
        g.w_split = g.steps;
        g.gap_at = a.F;
        g.gap = fp - a.F;
        if (e == hipSuccess) e = product<true>(g, a.dw, a.K, stream);
    }
    return e;
}

}  // namespace spingtp
