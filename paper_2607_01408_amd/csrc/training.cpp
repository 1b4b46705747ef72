// C entry points of the operators of a training step around the layers: argument checks and launches on the caller's
// stream.  The kernels are in sort_index.hip, embedding.hip and adamw.hip.
#include "training.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

namespace {

constexpr int64_t kMostElements = int64_t{1} << 46;  // of a matrix: every offset in bytes fits 64 bits with room
constexpr int64_t kMostColumns = int64_t{65535} * 512;

// n up to 2^31 - 1 entries of an index, V up to 2^31 - 2 rows of a table (V itself stands for none of them)
bool index_ok(int64_t n, int64_t V) { return n >= 0 && n <= 0x7fffffff && V >= 1 && V <= 0x7ffffffe; }
bool matrix_ok(int64_t rows, int64_t columns, int64_t ld) {
    return columns >= 1 && columns <= kMostColumns && ld >= columns && ld <= kMostElements &&
           (rows == 0 || ld <= kMostElements / rows);
}
bool off(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
bool bad(const void* p, uintptr_t a) { return p == nullptr || off(p, a); }
bool dtype_ok(int d) { return d == SPINGTP_FP32 || d == SPINGTP_BF16; }
uintptr_t width(int d) { return d == SPINGTP_FP32 ? 4 : 2; }
bool bytes_ok(int b) { return b == 4 || b == 8; }
spingtp_status of(hipError_t e) { return e == hipSuccess ? SPINGTP_OK : SPINGTP_ERR_HIP; }
hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }

}  // namespace

extern "C" spingtp_status spingtp_embedding(int dtype, const void* table, int64_t ldt, const void* index, int index_bytes,
                                            float scale, void* out, int64_t ldo, int64_t n, int64_t V, int64_t D,
                                            void* stream) {
    if (!dtype_ok(dtype) || !bytes_ok(index_bytes) || !index_ok(n, V) || !matrix_ok(V, D, ldt) || !matrix_ok(n, D, ldo))
        return SPINGTP_ERR_INVALID_ARG;
    if (n == 0) return SPINGTP_OK;
    if (bad(table, width(dtype)) || bad(out, width(dtype)) || bad(index, static_cast<uintptr_t>(index_bytes)))
        return SPINGTP_ERR_INVALID_ARG;
    return of(spingtp::launch_embedding(dtype, table, ldt, index, index_bytes == 8, scale, out, ldo, n, V, D,
                                        stream_of(stream)));
}

extern "C" spingtp_status spingtp_sort_index_workspace_size(int64_t n, int64_t V, size_t* size) {
    if (size == nullptr || !index_ok(n, V)) return SPINGTP_ERR_INVALID_ARG;
    *size = spingtp::sort_index_workspace(n, V);
    return SPINGTP_OK;
}

extern "C" spingtp_status spingtp_sort_index(const void* index, int index_bytes, int32_t* order, int32_t* rows,
                                             void* workspace, size_t workspace_bytes, int64_t n, int64_t V,
                                             void* stream) {
    size_t need = 0;
    if (!bytes_ok(index_bytes) || spingtp_sort_index_workspace_size(n, V, &need) != SPINGTP_OK)
        return SPINGTP_ERR_INVALID_ARG;
    if (n == 0) return SPINGTP_OK;
    if (bad(index, static_cast<uintptr_t>(index_bytes)) || bad(order, 4) || bad(rows, 4) ||
        (need > 0 && (bad(workspace, 16) || workspace_bytes < need)))
        return SPINGTP_ERR_INVALID_ARG;
    return of(spingtp::launch_sort_index(index, index_bytes == 8, order, rows, workspace, n, V, stream_of(stream)));
}

extern "C" spingtp_status spingtp_embedding_backward_workspace_size(int64_t n, int64_t D, size_t* size) {
    if (size == nullptr || !index_ok(n, 1) || !matrix_ok(n, D, D)) return SPINGTP_ERR_INVALID_ARG;
    *size = spingtp::embedding_backward_workspace(n, D);
    return SPINGTP_OK;
}

extern "C" spingtp_status spingtp_embedding_backward(int dtype, const void* grad, int64_t ldg, const int32_t* order,
                                                     const int32_t* rows, float scale, int table_dtype,
                                                     void* grad_table, int64_t ldt, void* workspace,
                                                     size_t workspace_bytes, int64_t n, int64_t V, int64_t D,
                                                     void* stream) {
    size_t need = 0;
    if (!dtype_ok(dtype) || !dtype_ok(table_dtype) || !index_ok(n, V) || !matrix_ok(n, D, ldg) || !matrix_ok(V, D, ldt) ||
        spingtp_embedding_backward_workspace_size(n, D, &need) != SPINGTP_OK)
        return SPINGTP_ERR_INVALID_ARG;
    if (bad(grad_table, width(table_dtype))) return SPINGTP_ERR_INVALID_ARG;
    if (n > 0 && (bad(grad, width(dtype)) || bad(order, 4) || bad(rows, 4) || bad(workspace, 16) || workspace_bytes < need))
        return SPINGTP_ERR_INVALID_ARG;
    const spingtp::EmbeddingBwdArgs a{dtype, grad, ldg, order, rows, scale, table_dtype, grad_table, ldt,
                                      static_cast<float*>(workspace), n, V, D};
    return of(spingtp::launch_embedding_backward(a, stream_of(stream)));
}

extern "C" spingtp_status spingtp_adamw(const spingtp_adamw_tensor* tensors, int64_t count,
                                        const spingtp_adamw_options* options, void* stream) {
    if (count < 0 || options == nullptr || (count > 0 && tensors == nullptr)) return SPINGTP_ERR_INVALID_ARG;
    const spingtp_adamw_options& o = *options;
    if (!(o.beta1 >= 0 && o.beta1 < 1 && o.beta2 >= 0 && o.beta2 < 1 && o.eps >= 0) || !std::isfinite(o.eps) ||
        !std::isfinite(o.lr) || !std::isfinite(o.weight_decay) || (o.device_step == nullptr && o.step < 1) ||
        off(o.device_step, 8) || off(o.device_lr, 4) || off(o.grad_scale, 4))
        return SPINGTP_ERR_INVALID_ARG;
    for (int64_t k = 0; k < count; ++k) {
        const spingtp_adamw_tensor& t = tensors[k];
        if (t.n < 0 || t.n > kMostElements || !dtype_ok(t.param_dtype) || !dtype_ok(t.grad_dtype) ||
            (t.m_scales != nullptr) != (t.v_scales != nullptr))
            return SPINGTP_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        const uintptr_t states = t.m_scales != nullptr ? 16 : 4;
        if (bad(t.param, width(t.param_dtype)) || bad(t.grad, width(t.grad_dtype)) || bad(t.m, states) || bad(t.v, states) ||
            off(t.copy, 2) || (t.copy != nullptr && t.param_dtype != SPINGTP_FP32))
            return SPINGTP_ERR_INVALID_ARG;
    }
    return of(spingtp::launch_adamw(tensors, count, o, stream_of(stream)));
}
