// Product of two matrices in the 8-bit block format: c[m][n] = sum_k a[m][k] b[n][k], both packed
// along k, fp32 accumulators, c in fp32 or bf16.
//
// Bound by the conversion to bf16 beside the matrix units, and at large sizes by power (units busy 64 % of the
// time at 1.9 GHz): 8,192 x 8,192 x 4,096 400-425 us, 1.3 PFLOP/s; 4,096 x 4,096 x 2,048 63 us, 1.1 PFLOP/s;
// 777 x 1,000 x 1,300 8 us, start and end of one round of tiles.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "feedforward.h"
#include "gemm_nt.h"
#include "gemm_skinny.h"
#include "internal.h"
#include "lds_common.h"

namespace spingtp {
namespace {

template <int PN, int PM, int WN, int WM, int NS, typename TO>
hipError_t launch(GemmArgs g, void* out, int64_t ldo, hipStream_t stream) {
    using Tile = GemmTile<Fp8, PN, PM, WN, WM, NS, false>;
    const int64_t tm = (g.M + Tile::BM - 1) / Tile::BM, tn = (g.N + Tile::BN - 1) / Tile::BN;
    if (tm * tn > kMostTiles) return hipErrorInvalidValue;
    g.tiles_m = static_cast<int>(tm);
    g.tiles_n = static_cast<int>(tn);
    constexpr auto kernel = gemm_nt_kernel<Fp8, PN, PM, WN, WM, NS, TO>;
    const hipError_t e = raise_lds_limit<kernel>();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(tm * tn)), dim3(Tile::kThreads), Tile::kLds, stream, g,
                       static_cast<TO*>(out), ldo);
    return hipGetLastError();
}

template <int TM, typename TO>
hipError_t launch_skinny(const GemmArgs& g, void* out, int64_t ldo, hipStream_t stream) {
    // as many rows of w as one launch holds workgroups for
    for (int64_t n = 0; n < g.N; n += 16 * kMostTiles) {
        GemmArgs part = g;
        part.w += n * g.ldw;
        part.ws += n * g.lds;
        part.N = g.N - n < 16 * kMostTiles ? g.N - n : 16 * kMostTiles;
        hipLaunchKernelGGL((gemm_skinny_kernel<Fp8, TM, TO>), dim3(static_cast<unsigned>((part.N + 15) / 16)),
                           dim3(64 * kSkinnyWaves), 0, stream, part, int64_t{0}, static_cast<TO*>(out) + n, ldo);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename TO>
hipError_t dispatch(const GemmArgs& g, int64_t k, void* out, int64_t ldo, hipStream_t stream) {
    // Few rows: the kernel for them, us against the smallest tile's: one row, 1,024^2 2.6 / 5.9, 4,096^2 5.4 / 16.6,
    // 8,192 x 2,048 4.7 / 9.5; 32 rows 3.6 / 5.9, 10.2 / 16.7, 8.7 / 9.6; 64 rows 4.7 / 6.2, 15.7 / 16.9, but
    // 13.3 / 10.2, where there are enough tiles for the sums of 2,048 terms.
    if (g.M <= 16) return launch_skinny<1, TO>(g, out, ldo, stream);
    if (g.M <= 32) return launch_skinny<2, TO>(g, out, ldo, stream);
    if (g.M <= kSkinnyRows && g.N <= 2 * k) return launch_skinny<4, TO>(g, out, ldo, stream);
    switch (product_tile(kPlain8, g.M, g.N)) {
        case 256: return launch<128, 64, 2, 4, 2, TO>(g, out, ldo, stream);
        case 128: return launch<64, 64, 2, 2, 2, TO>(g, out, ldo, stream);
        default: return launch<32, 32, 2, 2, 4, TO>(g, out, ldo, stream);
    }
}

}  // namespace

hipError_t launch_matmul8(int dtype, const Matmul8Args& a, hipStream_t stream) {
    GemmArgs g{};
    g.w = a.b_values;
    g.x = a.a_values;
    g.ldw = g.ldx = block8_pitch(a.K);
    g.ws = a.b_scales;
    g.xs = a.a_scales;
    g.lds = block8_scale_pitch(a.K);
    g.M = a.M;
    g.N = a.N;
    g.steps = static_cast<int>(g.ldx / kStepBytes);
    g.tail = kStepBytes;
    return dtype == SPINGTP_FP32 ? dispatch<float>(g, a.K, a.c, a.ldc, stream)
                                 : dispatch<uint16_t>(g, a.K, a.c, a.ldc, stream);
}

}  // namespace spingtp
