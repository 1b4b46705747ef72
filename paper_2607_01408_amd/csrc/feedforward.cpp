// C entry points of the feed-forward operators: argument checks and launches on the caller's stream.
// The kernels are in norm8.hip, pack8.hip, matmul8.hip and gated.hip.
#include "feedforward.h"

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.h"
#include "tile_rule.h"

namespace {

// Sizes up to 2^31 - 1 each and 2^46 elements per matrix: every offset in bytes fits 64 bits with room.
bool size_ok(int64_t n, int64_t least) { return n >= least && n <= 0x7fffffff; }
bool matrix_ok(int64_t rows, int64_t ld) {
    return ld >= 1 && ld <= (int64_t{1} << 46) && (rows == 0 || ld <= (int64_t{1} << 46) / rows);
}
bool off(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
bool bad(const void* p, uintptr_t a) { return p == nullptr || off(p, a); }
bool dtype_ok(int d) { return d == SPINGTP_FP32 || d == SPINGTP_BF16; }
uintptr_t width(int d) { return d == SPINGTP_FP32 ? 4 : 2; }
spingtp_status of(hipError_t e) { return e == hipSuccess ? SPINGTP_OK : SPINGTP_ERR_HIP; }
hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }
uint8_t* bytes(void* p) { return static_cast<uint8_t*>(p); }
const uint8_t* bytes(const void* p) { return static_cast<const uint8_t*>(p); }

}  // namespace

extern "C" spingtp_status spingtp_pack8(int dtype, const void* x, int64_t ldx, void* values, void* scales,
                                        void* t_values, void* t_scales, int64_t R, int64_t D, void* stream) {
    if (!dtype_ok(dtype) || !size_ok(R, 0) || !size_ok(D, 1) || ldx < D || !matrix_ok(R, ldx) || !matrix_ok(R, D + 511))
        return SPINGTP_ERR_INVALID_ARG;
    if (R == 0) return SPINGTP_OK;
    if (values == nullptr && t_values == nullptr) return SPINGTP_ERR_INVALID_ARG;
    if ((values != nullptr) != (scales != nullptr) || (t_values != nullptr) != (t_scales != nullptr))
        return SPINGTP_ERR_INVALID_ARG;
    if (off(values, 16) || off(scales, 4) || off(t_values, 16) || off(t_scales, 4)) return SPINGTP_ERR_INVALID_ARG;
    if (t_values != nullptr && D > int64_t{65535} * 128) return SPINGTP_ERR_INVALID_ARG;
    if (bad(x, width(dtype))) return SPINGTP_ERR_INVALID_ARG;
    return of(spingtp::launch_pack8(dtype, x, ldx, bytes(values), bytes(scales), bytes(t_values), bytes(t_scales), R, D,
                                    stream_of(stream)));
}

extern "C" spingtp_status spingtp_unpack8(const void* values, const void* scales, int dtype, void* x,
                                          int64_t ldx, int64_t R, int64_t D, void* stream) {
    if (!dtype_ok(dtype) || !size_ok(R, 0) || !size_ok(D, 1) || ldx < D || !matrix_ok(R, ldx) || !matrix_ok(R, D + 511))
        return SPINGTP_ERR_INVALID_ARG;
    if (R == 0) return SPINGTP_OK;
    if (bad(values, 16) || bad(scales, 4) || bad(x, width(dtype))) return SPINGTP_ERR_INVALID_ARG;
    return of(spingtp::launch_unpack8(dtype, bytes(values), bytes(scales), x, ldx, R, D, stream_of(stream)));
}

extern "C" spingtp_status spingtp_rms_norm(int dtype, const void* x, int64_t ldx, const void* residual,
                                           int64_t ldr, const float* gain, float eps, void* h, int64_t ldh, void* y,
                                           int64_t ldy, void* values, void* scales, float* rstd, int64_t R, int64_t D,
                                           void* stream) {
    if (!dtype_ok(dtype) || !size_ok(R, 0) || !size_ok(D, 1) || ldx < D || !matrix_ok(R, ldx) || !matrix_ok(R, D + 511))
        return SPINGTP_ERR_INVALID_ARG;
    if (!(eps >= 0.f)) return SPINGTP_ERR_INVALID_ARG;
    if (R == 0) return SPINGTP_OK;
    if ((y != nullptr) == (values != nullptr) || (values != nullptr) != (scales != nullptr))
        return SPINGTP_ERR_INVALID_ARG;
    if (residual != nullptr && (h == nullptr || ldr < D || !matrix_ok(R, ldr))) return SPINGTP_ERR_INVALID_ARG;
    if (h != nullptr && (ldh < D || !matrix_ok(R, ldh))) return SPINGTP_ERR_INVALID_ARG;
    if (y != nullptr && (ldy < D || !matrix_ok(R, ldy))) return SPINGTP_ERR_INVALID_ARG;
    const uintptr_t w = width(dtype);
    if (off(residual, w) || off(h, w) || off(y, w) || off(values, 16) || off(scales, 4) || off(rstd, 4))
        return SPINGTP_ERR_INVALID_ARG;
    if (bad(x, w) || bad(gain, 4)) return SPINGTP_ERR_INVALID_ARG;
    const spingtp::NormArgs a{x,   ldx, residual, ldr,           gain,          eps,  h, ldh,
                              y,   ldy, bytes(values), bytes(scales), rstd, R, D};
    return of(spingtp::launch_rms_norm(dtype, a, stream_of(stream)));
}

extern "C" spingtp_status spingtp_rms_norm_backward_workspace_size(int64_t R, int64_t D, size_t* size) {
    if (size == nullptr || !size_ok(R, 0) || !size_ok(D, 1)) return SPINGTP_ERR_INVALID_ARG;
    *size = static_cast<size_t>(spingtp::norm_bwd_blocks(R, D) * D) * sizeof(float);
    return SPINGTP_OK;
}

extern "C" spingtp_status spingtp_rms_norm_backward(int dtype, const void* grad_y, int64_t ldg, const void* h,
                                                    int64_t ldh, const float* rstd, const float* gain,
                                                    const void* grad_h, int64_t ldgh, void* grad_x, int64_t ldx,
                                                    float* grad_gain, void* workspace, size_t workspace_bytes,
                                                    int64_t R, int64_t D, void* stream) {
    size_t need = 0;
    if (!dtype_ok(dtype) || spingtp_rms_norm_backward_workspace_size(R, D, &need) != SPINGTP_OK)
        return SPINGTP_ERR_INVALID_ARG;
    if (ldg < D || ldh < D || ldx < D || !matrix_ok(R, ldg) || !matrix_ok(R, ldh) || !matrix_ok(R, ldx))
        return SPINGTP_ERR_INVALID_ARG;
    if (grad_h != nullptr && (ldgh < D || !matrix_ok(R, ldgh))) return SPINGTP_ERR_INVALID_ARG;
    const uintptr_t w = width(dtype);
    if (off(grad_h, w) || off(grad_gain, 4)) return SPINGTP_ERR_INVALID_ARG;
    if (R > 0 && (bad(grad_y, w) || bad(h, w) || bad(rstd, 4) || bad(gain, 4) || bad(grad_x, w)))
        return SPINGTP_ERR_INVALID_ARG;
    if (R > 0 && grad_gain != nullptr && (bad(workspace, 4) || workspace_bytes < need)) return SPINGTP_ERR_INVALID_ARG;
    const spingtp::NormBwdArgs a{grad_y, ldg,    h,   ldh,       rstd, gain, grad_h, ldgh,
                                 grad_x, ldx, grad_gain, static_cast<float*>(workspace), R, D};
    return of(spingtp::launch_rms_norm_bwd(dtype, a, stream_of(stream)));
}

extern "C" spingtp_status spingtp_matmul8(const void* a_values, const void* a_scales, const void* b_values,
                                          const void* b_scales, int dtype, void* c, int64_t ldc, int64_t M,
                                          int64_t N, int64_t K, void* stream) {
    if (!dtype_ok(dtype) || !size_ok(M, 0) || !size_ok(N, 0) || !size_ok(K, 1) || K > int64_t{65535} * 128 ||
        ldc < N || ldc < 1 || !matrix_ok(M, ldc) || !matrix_ok(M, K + 511) || !matrix_ok(N, K + 511) ||
        !spingtp::product_fits(M, N))
        return SPINGTP_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return SPINGTP_OK;
    if (bad(a_values, 16) || bad(a_scales, 4) || bad(b_values, 16) || bad(b_scales, 4) || bad(c, width(dtype)))
        return SPINGTP_ERR_INVALID_ARG;
    const spingtp::Matmul8Args a{bytes(a_values), bytes(a_scales), bytes(b_values), bytes(b_scales), c, ldc, M, N, K};
    return of(spingtp::launch_matmul8(dtype, a, stream_of(stream)));
}

namespace {

bool gated_sizes_ok(int act, int64_t M, int64_t K, int64_t F) {
    return (act == spingtp::kSilu || act == spingtp::kGelu) && size_ok(M, 0) && size_ok(K, 1) && size_ok(F, 1) &&
           K <= int64_t{65535} * 64 && F <= int64_t{65535} * 32 && matrix_ok(M, K + 511) && matrix_ok(M, 2 * (F + 511)) &&
           matrix_ok(F, 2 * (K + 511)) && spingtp::gated_fits(M, F);
}
bool save_ok(int s) { return s == SPINGTP_SAVE_NONE || s == SPINGTP_SAVE_BF16 || s == SPINGTP_SAVE_BLOCK8; }

}  // namespace

extern "C" spingtp_status spingtp_gated_forward_workspace_size(int64_t M, int64_t K, int64_t F, int64_t ldx, int64_t ldw,
                                                               int save, size_t* size) {
    if (size == nullptr || !gated_sizes_ok(spingtp::kSilu, M, K, F) || ldx < K || ldw < K || !matrix_ok(M, ldx) ||
        !matrix_ok(F, ldw) || !save_ok(save))
        return SPINGTP_ERR_INVALID_ARG;
    *size = spingtp::gated_workspace(M, K, F, ldx, ldw, save);
    return SPINGTP_OK;
}

extern "C" spingtp_status spingtp_gated_forward(int act, const void* x, int64_t ldx, const void* w_gate,
                                                const void* w_up, int64_t ldw, void* h, int64_t ldh, int save,
                                                void* g, void* g_scales, void* u, void* u_scales, void* workspace,
                                                size_t workspace_bytes, int64_t M, int64_t K, int64_t F, void* stream) {
    size_t need = 0;
    if (!gated_sizes_ok(act, M, K, F) || ldh < F || !matrix_ok(M, ldh) ||
        spingtp_gated_forward_workspace_size(M, K, F, ldx, ldw, save, &need) != SPINGTP_OK)
        return SPINGTP_ERR_INVALID_ARG;
    if (M == 0) return SPINGTP_OK;
    if (bad(x, 16) || bad(w_gate, 16) || bad(w_up, 16) || bad(h, 2)) return SPINGTP_ERR_INVALID_ARG;
    if (save != SPINGTP_SAVE_NONE && (bad(g, 16) || bad(u, 16))) return SPINGTP_ERR_INVALID_ARG;
    if (save == SPINGTP_SAVE_BLOCK8 && (bad(g_scales, 4) || bad(u_scales, 4))) return SPINGTP_ERR_INVALID_ARG;
    if (need > 0 && (bad(workspace, 16) || workspace_bytes < need)) return SPINGTP_ERR_INVALID_ARG;
    spingtp::GatedArgs a{};
    a.act = act;
    a.x = x;
    a.ldx = ldx;
    a.wg = w_gate;
    a.wu = w_up;
    a.ldw = ldw;
    a.h = h;
    a.ldh = ldh;
    a.save = save;
    a.g = g;
    a.u = u;
    a.g_scales = bytes(g_scales);
    a.u_scales = bytes(u_scales);
    a.workspace = workspace;
    a.M = M;
    a.K = K;
    a.F = F;
    return of(spingtp::launch_gated(a, stream_of(stream)));
}

extern "C" spingtp_status spingtp_gated_forward8_workspace_size(int64_t M, int64_t K, int64_t F, int out8,
                                                                size_t* size) {
    if (size == nullptr || !gated_sizes_ok(spingtp::kSilu, M, K, F)) return SPINGTP_ERR_INVALID_ARG;
    *size = spingtp::gated8_workspace(M, F, out8 != 0);
    return SPINGTP_OK;
}

extern "C" spingtp_status spingtp_gated_forward8(int act, const void* x, const void* x_scales,
                                                 const void* w_gate, const void* w_gate_scales, const void* w_up,
                                                 const void* w_up_scales, void* h, int64_t ldh, void* h_scales,
                                                 void* workspace, size_t workspace_bytes, int64_t M, int64_t K,
                                                 int64_t F, void* stream) {
    size_t need = 0;
    if (!gated_sizes_ok(act, M, K, F) ||
        spingtp_gated_forward8_workspace_size(M, K, F, h_scales != nullptr, &need) != SPINGTP_OK || (h_scales == nullptr && (ldh < F || !matrix_ok(M, ldh))))
        return SPINGTP_ERR_INVALID_ARG;
    if (M == 0) return SPINGTP_OK;
    if (bad(x, 16) || bad(x_scales, 4) || bad(w_gate, 16) || bad(w_gate_scales, 4) || bad(w_up, 16) ||
        bad(w_up_scales, 4) || bad(h, h_scales != nullptr ? 16 : 2) || off(h_scales, 4))
        return SPINGTP_ERR_INVALID_ARG;
    if (need > 0 && (bad(workspace, 16) || workspace_bytes < need)) return SPINGTP_ERR_INVALID_ARG;
    spingtp::GatedArgs a{};
    a.act = act;
    a.x = x;
    a.x_scales = bytes(x_scales);
    a.wg = w_gate;
    a.wg_scales = bytes(w_gate_scales);
    a.wu = w_up;
    a.wu_scales = bytes(w_up_scales);
    a.h = h;
    a.ldh = ldh;
    a.h_scales = bytes(h_scales);
    a.workspace = workspace;
    a.M = M;
    a.K = K;
    a.F = F;
    return of(spingtp::launch_gated8(a, stream_of(stream)));
}

extern "C" spingtp_status spingtp_gated_backward_workspace_size(int64_t M, int64_t K, int64_t F, int64_t ldx,
                                                                int64_t ldw, int x8, size_t* size) {
    if (size == nullptr || !gated_sizes_ok(spingtp::kSilu, M, K, F) || (x8 == 0 && (ldx < K || !matrix_ok(M, ldx))) ||
        ldw < K || !matrix_ok(F, ldw))
        return SPINGTP_ERR_INVALID_ARG;
    *size = spingtp::gated_backward_workspace(M, K, F, ldx, ldw, x8 != 0);
    return SPINGTP_OK;
}

extern "C" spingtp_status spingtp_gated_backward(int act, const void* grad_h, int64_t ldgh,
                                                 int save, const void* g, const void* g_scales, const void* u,
                                                 const void* u_scales, const void* x, int64_t ldx, const void* x_scales,
                                                 const void* w_gate, const void* w_up, int64_t ldw, void* grad_x,
                                                 int64_t ldgx, void* grad_w, void* workspace, size_t workspace_bytes,
                                                 int64_t M, int64_t K, int64_t F, void* stream) {
    size_t need = 0;
    if (!gated_sizes_ok(act, M, K, F) ||
        spingtp_gated_backward_workspace_size(M, K, F, ldx, ldw, x_scales != nullptr, &need) != SPINGTP_OK)
        return SPINGTP_ERR_INVALID_ARG;
    if (ldgh < F || !matrix_ok(M, ldgh) || (save != SPINGTP_SAVE_BF16 && save != SPINGTP_SAVE_BLOCK8))
        return SPINGTP_ERR_INVALID_ARG;
    if ((grad_x != nullptr && (ldgx < K || !matrix_ok(M, ldgx) || off(grad_x, 2))) || off(grad_w, 2))
        return SPINGTP_ERR_INVALID_ARG;
    if (M > 0) {
        if (bad(grad_h, 2) || bad(g, 16) || bad(u, 16)) return SPINGTP_ERR_INVALID_ARG;
        if (save == SPINGTP_SAVE_BLOCK8 && (bad(g_scales, 4) || bad(u_scales, 4))) return SPINGTP_ERR_INVALID_ARG;
        if ((grad_x != nullptr && !spingtp::product_fits(M, K)) ||
            (grad_w != nullptr && !spingtp::product_fits(2 * F + 63, K)))
            return SPINGTP_ERR_INVALID_ARG;
        if (grad_x != nullptr && (bad(w_gate, 16) || bad(w_up, 16))) return SPINGTP_ERR_INVALID_ARG;
        if (grad_w != nullptr && (bad(x, 16) || off(x_scales, 4)))
            return SPINGTP_ERR_INVALID_ARG;
        if (bad(workspace, 16) || workspace_bytes < need) return SPINGTP_ERR_INVALID_ARG;
    }
    if (grad_x == nullptr && grad_w == nullptr) return SPINGTP_OK;
    spingtp::GatedBwdArgs a{};
    a.act = act;
    a.dh = grad_h;
    a.lddh = ldgh;
    a.save = save;
    a.g = g;
    a.u = u;
    a.g_scales = bytes(g_scales);
    a.u_scales = bytes(u_scales);
    a.x = x;
    a.ldx = ldx;
    a.x_scales = bytes(x_scales);
    a.wg = w_gate;
    a.wu = w_up;
    a.ldw = ldw;
    a.dx = grad_x;
    a.lddx = ldgx;
    a.dw = grad_w;
    a.workspace = workspace;
    a.M = M;
    a.K = K;
    a.F = F;
    return of(spingtp::launch_gated_backward(a, stream_of(stream)));
}
