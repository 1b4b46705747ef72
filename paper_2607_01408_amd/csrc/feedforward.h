// Launches of the feed-forward operators (norm8.hip, pack8.hip, matmul8.hip, gated.hip); the C entry
// points that check their arguments are in feedforward.cpp.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace spingtp {

// workgroups of a launch (a launch has fewer than 2^32 threads); the kernels walk what is left
constexpr int64_t kMostBlocks = int64_t{1} << 20;

// dtype 0: fp32 elements, 1: bf16
struct NormArgs {
    const void* x;
    int64_t ldx;
    const void* r;  // may be null
    int64_t ldr;
    const float* gain;
    float eps;
    void* h;  // may be null
    int64_t ldh;
    void* y;  // y or values and scales
    int64_t ldy;
    uint8_t* values;
    uint8_t* scales;
    float* rstd;  // may be null
    int64_t R, D;
};
hipError_t launch_rms_norm(int dtype, const NormArgs& a, hipStream_t stream);

struct NormBwdArgs {
    const void* dy;
    int64_t lddy;
    const void* h;
    int64_t ldh;
    const float* rstd;
    const float* gain;
    const void* gh;  // may be null
    int64_t ldgh;
    void* dx;
    int64_t lddx;
    float* dgain;    // may be null
    float* partial;  // [norm_bwd_blocks(R, D)][D]
    int64_t R, D;
};
int64_t norm_bwd_blocks(int64_t R, int64_t D);
hipError_t launch_rms_norm_bwd(int dtype, const NormBwdArgs& a, hipStream_t stream);

// x [R][D] (row stride ldx) to 8 bits along its rows (values, scales) and / or, as the transposed
// matrix [D][R], along its columns (t_values, t_scales)
hipError_t launch_pack8(int dtype, const void* x, int64_t ldx, uint8_t* values, uint8_t* scales, uint8_t* t_values,
                        uint8_t* t_scales, int64_t R, int64_t D, hipStream_t stream);
hipError_t launch_unpack8(int dtype, const uint8_t* values, const uint8_t* scales, void* x, int64_t ldx, int64_t R,
                          int64_t D, hipStream_t stream);

struct Matmul8Args {
    const uint8_t* a_values;
    const uint8_t* a_scales;
    const uint8_t* b_values;
    const uint8_t* b_scales;
    void* c;
    int64_t ldc;
    int64_t M, N, K;
};
hipError_t launch_matmul8(int dtype, const Matmul8Args& a, hipStream_t stream);

// The gated block's activation
enum { kSilu = 0, kGelu = 1 };

// What the forward keeps of the pre-activations g and u: nothing, bf16 or 8-bit blocks
enum { kSaveNone = 0, kSaveBf16 = 1, kSave8 = 2 };

struct GatedArgs {
    int act;
    // bf16 operands (row strides in elements) ...
    const void* x;
    int64_t ldx;
    const void* wg;
    const void* wu;
    int64_t ldw;
    // ... or 8-bit ones (scales not null)
    const uint8_t* x_scales;
    const uint8_t* wg_scales;
    const uint8_t* wu_scales;
    void* h;  // bf16 [M] rows of ldh elements, or 8-bit values with h_scales
    int64_t ldh;
    uint8_t* h_scales;
    int save;
    void* g;
    void* u;
    uint8_t* g_scales;
    uint8_t* u_scales;
    void* workspace;
    int64_t M, K, F;
};
size_t gated_workspace(int64_t M, int64_t K, int64_t F, int64_t ldx, int64_t ldw, int save);
size_t gated8_workspace(int64_t M, int64_t F, bool out8);
hipError_t launch_gated(const GatedArgs& a, hipStream_t stream);
hipError_t launch_gated8(const GatedArgs& a, hipStream_t stream);

struct GatedBwdArgs {
    int act;
    const void* dh;
    int64_t lddh;
    int save;  // kSaveBf16 or kSave8
    const void* g;
    const void* u;
    const uint8_t* g_scales;
    const uint8_t* u_scales;
    const void* x;  // bf16, or 8-bit values with x_scales
    int64_t ldx;
    const uint8_t* x_scales;
    const void* wg;
    const void* wu;
    int64_t ldw;
    void* dx;  // may be null
    int64_t lddx;
    void* dw;  // [2 F][K], may be null
    void* workspace;
    int64_t M, K, F;
};
size_t gated_backward_workspace(int64_t M, int64_t K, int64_t F, int64_t ldx, int64_t ldw, bool x8);
hipError_t launch_gated_backward(const GatedBwdArgs& a, hipStream_t stream);

}  // namespace spingtp
