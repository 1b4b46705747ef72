// Launches of the operators of a training step around the layers (sort_index.hip, embedding.hip, adamw.hip); the C
// entry points that check their arguments are in training.cpp.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "feedforward.h"
#include "spingtp.h"

namespace spingtp {

// The sorted form of an index: its places in the order of their rows (equal ones in their own order), and those rows;
// entries outside [0, V) come last, as V.
size_t sort_index_workspace(int64_t n, int64_t V);
hipError_t launch_sort_index(const void* index, bool wide, int32_t* order, int32_t* rows, void* workspace, int64_t n,
                             int64_t V, hipStream_t stream);

// dtype 0: fp32 elements, 1: bf16; index int64 where `wide`, else int32
hipError_t launch_embedding(int dtype, const void* table, int64_t ldt, const void* index, bool wide, float scale, void* out,
                            int64_t ldo, int64_t n, int64_t V, int64_t D, hipStream_t stream);

struct EmbeddingBwdArgs {
    int dtype;  // of grad
    const void* grad;
    int64_t ldg;
    const int32_t* order;
    const int32_t* rows;
    float scale;
    int out_dtype;
    void* out;  // [V] rows of ldo elements
    int64_t ldo;
    float* partial;
    int64_t n, V, D;
};
size_t embedding_backward_workspace(int64_t n, int64_t D);
hipError_t launch_embedding_backward(const EmbeddingBwdArgs& a, hipStream_t stream);

hipError_t launch_adamw(const spingtp_adamw_tensor* tensors, int64_t count, const spingtp_adamw_options& o,
                        hipStream_t stream);

}  // namespace spingtp
