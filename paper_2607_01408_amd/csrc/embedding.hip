// Lookup of a table's rows and its gradient:
//   out[i] = scale table[index[i]],   dtable[v] = scale sum over {i: index[i] = v} of dout[i].
//
// Forward: a row's columns over the lanes of a group, 16 or 32 bytes each; bound by memory, and for few rows by latency:
// 16,384 rows of 2,048 in bf16 22 us (67 MB written, the frequent rows' reads from the caches), 32 rows of 4,096 2.5.
//
// Backward: over the index in sorted order (sort_index.hip), cut into chunks of equal length whatever the rows' numbers
// of entries: a group of lanes walks its chunk and keeps the running sum of a row in fp32.  A row whose entries lie in
// one chunk leaves at once; a row that crosses chunks leaves a part in each, and a second kernel adds the parts in
// order; where all parts of a workgroup belong to one row that began earlier, it leaves their sum too, so that a long row
// has few of them.  So one row with all entries costs little more than many with a few (200,000 rows of 128 in fp32 onto
// one row of 50,000 40 us, onto all of them 30), every row of the result is written once, and no step depends on the
// order of arrival.  The rows without entries are zeroed by workgroups of the same launch: a lane
// looks for its row by bisection.  16,384 entries over 50,000 rows of 2,048 in bf16: 45 us (68 MB in, 205 MB out, 6.0 TB/s)
// and 9 for the rows that cross chunks; 100,000 over 4,000 of 128 in fp32: 14 and 6.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "block8.h"
#include "internal.h"
#include "training.h"

namespace spingtp {
namespace {

// -1: no row of the table
__device__ __forceinline__ int64_t row_of(const void* index, bool wide, int64_t i, int64_t V) {
    const int64_t k = wide ? static_cast<const int64_t*>(index)[i] : static_cast<const int32_t*>(index)[i];
    return k >= 0 && k < V ? k : -1;
}

// A lane's eight columns of its group's 8 LANES: neighbours (16 bytes in bf16) or, of fp32 rows that leave as fp32, two
// fours 4 LANES apart, so that a group's loads and stores are lines without gaps.  `c`: the first; `end`: the row's.
template <int LANES, bool FOURS, typename T>
__device__ __forceinline__ void load_columns(const T* row, int64_t c, int64_t end, float (&v)[8]) {
    if constexpr (FOURS) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = c + 4 * LANES * h;
            if (at + 4 <= end) {
                const u4f x = *reinterpret_cast<const u4f*>(row + at);
                v[4 * h] = x.x, v[4 * h + 1] = x.y, v[4 * h + 2] = x.z, v[4 * h + 3] = x.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[4 * h + i] = at + i < end ? row[at + i] : 0.f;
            }
        }
    } else {
        load8(row + c, end - c >= 8 ? 8 : static_cast<int>(end - c), v);
    }
}
template <int LANES, bool FOURS, typename T>
__device__ __forceinline__ void store_columns(T* row, int64_t c, int64_t end, const float (&v)[8], bool around) {
    if constexpr (FOURS) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = c + 4 * LANES * h;
            if (at + 4 <= end) {
                const u4f x{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                if (around)
                    __builtin_nontemporal_store(x, reinterpret_cast<u4f*>(row + at));
                else
                    *reinterpret_cast<u4f*>(row + at) = x;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (at + i < end) row[at + i] = v[4 * h + i];
            }
        }
    } else {
        pass_store8(row + c, end - c >= 8 ? 8 : static_cast<int>(end - c), v, around);
    }
}

// LANES lanes of eight columns to a row, ROWS rows to a group.
template <int LANES, int ROWS, typename T>
__global__ __launch_bounds__(256) void embedding_kernel(const T* __restrict__ table, int64_t ldt, const void* index,
                                                        bool wide, float scale, T* __restrict__ out, int64_t ldo, int64_t n,
                                                        int64_t V, int64_t D, bool around) {
    constexpr int kGroups = 256 / LANES;
    constexpr bool kFours = sizeof(T) == 4;
    const int l = threadIdx.x % LANES, g = threadIdx.x / LANES;
    const int64_t c = static_cast<int64_t>(blockIdx.y) * LANES * 8 + l * (kFours ? 4 : 8);
    if (c >= D) return;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kGroups * ROWS + g; first < n;
         first += static_cast<int64_t>(gridDim.x) * kGroups * ROWS) {
        int64_t row[ROWS];
        float v[ROWS][8];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) row[r] = first + r * kGroups < n ? row_of(index, wide, first + r * kGroups, V) : -1;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (row[r] >= 0) {
                load_columns<LANES, kFours>(table + row[r] * ldt, c, D, v[r]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[r][i] = 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[r][i] = row[r] >= 0 ? v[r][i] * scale : 0.f;
            if (first + r * kGroups < n) store_columns<LANES, kFours>(out + (first + r * kGroups) * ldo, c, D, v[r], around);
        }
    }
}

// the first place in the sorted rows whose row is `row` or more
__device__ __forceinline__ int64_t place_from(const int32_t* rows, int64_t n, int32_t row) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (rows[mid] < row)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

constexpr int kAhead = 4;  // rows in flight

constexpr int kEmptyRows = 16;  // of the table, that a wave looks after

// Workgroups 0 to sum_blocks - 1: chunks of `chunk` entries, one to a group, `across` workgroups to the columns.  partial
// [chunks][2][D]: the part of a row that began in an earlier chunk, and of one that begins here and goes on.  sums
// [chunks / kGroups][D]: where all chunks of a workgroup start with one row from an earlier workgroup's, the sum of these
// parts (a row with thousands of chunks is joined by them).  The other workgroups: rows of the table without entries.
template <int LANES, typename TG, typename TO>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const TG* __restrict__ grad, int64_t ldg,
                                                            const int32_t* __restrict__ order,
                                                            const int32_t* __restrict__ rows, float scale,
                                                            TO* __restrict__ out, int64_t ldo, float* __restrict__ partial,
                                                            float* __restrict__ sums, int64_t n, int64_t V, int64_t D,
                                                            int64_t chunk, unsigned across, unsigned sum_blocks,
                                                            bool around) {
    constexpr int kGroups = 256 / LANES;
    constexpr bool kFours = sizeof(TG) == 4 && sizeof(TO) == 4;
    if (blockIdx.x >= sum_blocks) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const float zeros[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        constexpr int kAtOnce = 64 / LANES;
        const int64_t stride = static_cast<int64_t>(gridDim.x - sum_blocks) * 4 * kEmptyRows;
        for (int64_t first = (static_cast<int64_t>(blockIdx.x - sum_blocks) * 4 + wave) * kEmptyRows; first < V;
             first += stride) {
            const int64_t mine = first + lane;
            bool empty = false;
            if (lane < kEmptyRows && mine < V) {
                const int64_t at = place_from(rows, n, static_cast<int32_t>(mine));
                empty = at >= n || rows[at] != mine;
            }
            uint64_t left = __ballot(empty);
            // kAtOnce empty rows at a time, LANES lanes to each
            while (left != 0) {
                int64_t row = -1;
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    if (left == 0) break;
                    const int b = __builtin_ctzll(left);
                    left &= left - 1;
                    if (lane / LANES == k) row = first + b;
                }
                if (row >= 0)
                    for (int64_t c = (lane % LANES) * (kFours ? 4 : 8); c < D; c += LANES * 8)
                        store_columns<LANES, kFours>(out + row * ldo, c, D, zeros, around);
            }
        }
        return;
    }
    const int l = threadIdx.x % LANES, g = threadIdx.x / LANES;
    const int64_t c = static_cast<int64_t>(blockIdx.x % across) * LANES * 8 + l * (kFours ? 4 : 8);
    const int64_t window = blockIdx.x / across, k = window * kGroups + g, p0 = k * chunk;
    const int64_t last = ((window + 1) * kGroups - 1) * chunk;  // of the last chunk, its first entry
    const bool one_row = window > 0 && last < n && rows[window * kGroups * chunk - 1] == rows[last];
    if (!one_row && (c >= D || p0 >= n)) return;  // (lanes past the columns load and store nothing)
    const int64_t p1 = p0 + chunk < n ? p0 + chunk : n;
    float sum[8];
    const uint32_t most = static_cast<uint32_t>(n - 1);
    int32_t row = rows[p0];
    bool before = p0 > 0 && rows[p0 - 1] == row;
    const bool after = p1 < n && rows[p1] == rows[p1 - 1];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    const auto leave = [&](bool goes_on) {
        if (static_cast<uint32_t>(row) < V) {
            if (before || goes_on) {
                store_columns<LANES, kFours>(partial + (2 * k + (before ? 0 : 1)) * D, c, D, sum, false);
            } else {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = sum[i] * scale;
                store_columns<LANES, kFours>(out + row * ldo, c, D, v, around);
            }
        }
    };
    for (int64_t p = p0; p < p1; p += kAhead) {
        float v[kAhead][8];
        int32_t r[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t q = p + j < p1 ? p + j : p1 - 1;
            r[j] = rows[q];
            const uint32_t at = static_cast<uint32_t>(order[q]);
            load_columns<LANES, kFours>(grad + (at < most ? at : most) * ldg, c, D, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (p + j >= p1) break;
            if (r[j] != row) {
                leave(false);
                row = r[j];
                before = false;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[j][i];
        }
    }
    leave(after);
    if (!one_row) return;
    __syncthreads();
    if (g != 0 || static_cast<uint32_t>(rows[last]) >= V) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
#pragma unroll 4
    for (int q = 0; q < kGroups; ++q) {
        float v[8];
        load_columns<LANES, kFours>(partial + 2 * (k + q) * D, c, D, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += v[i];
    }
    store_columns<LANES, kFours>(sums + window * D, c, D, sum, false);
}

constexpr int kJoinThreads = 512;
constexpr int kShort = 8;  // chunks beyond the first that a group adds up by itself

// A group to a chunk; those in which a row begins that goes on add its parts: chunk after chunk as long as one starts
// with the row.  A row of more than kShort chunks is added by the whole workgroup, a group every so many chunks (or, where
// there are more than kLong, sums of kWindow of them), and the groups' sums in order.
template <int LANES, int kWindow, typename TO>
__global__ __launch_bounds__(kJoinThreads) void embedding_join_kernel(const float* __restrict__ partial,
                                                                      const float* __restrict__ sums,
                                                                      const int32_t* __restrict__ rows, float scale,
                                                                      TO* __restrict__ out, int64_t ldo, int64_t n,
                                                                      int64_t V, int64_t D, int64_t chunk, int64_t chunks,
                                                                      unsigned across) {
    constexpr int kGroups = kJoinThreads / LANES, kLong = (1 << 18) / (32 * LANES);  // 256 KB of parts
    __shared__ float part[kGroups][LANES * 8 + 4];
    __shared__ int32_t long_row[kGroups];  // -1: none begins in the group's chunk
    __shared__ int first_open;             // the first window that the row does not fill
    const int l = threadIdx.x % LANES, g = threadIdx.x / LANES;
    const int64_t c = (static_cast<int64_t>(blockIdx.x % across) * LANES + l) * 8, left = D - c;
    const int have = left >= 8 ? 8 : (left > 0 ? static_cast<int>(left) : 0);
    const int64_t first = static_cast<int64_t>(blockIdx.x / across) * kGroups;
    // adds the parts of `row` in chunks j, j + step, ... below `end`; whether all of them were its
    const auto add = [&](float (&sum)[8], int32_t row, int64_t j, int64_t step, int64_t end) {
        constexpr int kAtOnce = 4;
        for (; j < end; j += kAtOnce * step) {
            int32_t r[kAtOnce];
            float v[kAtOnce][8];
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                const int64_t at = j + q * step < end ? j + q * step : j;
                r[q] = rows[at * chunk];
                load8(partial + 2 * at * D + (have > 0 ? c : 0), have, v[q]);
            }
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                if (j + q * step >= end) return true;
                if (r[q] != row) return false;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += v[q][i];
            }
        }
        return true;
    };
    const auto finish = [&](float (&sum)[8], int32_t row, int64_t k) {
        float v[8];
        load8(partial + (2 * k + 1) * D + c, have, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (v[i] + sum[i]) * scale;
        store8(out + row * ldo + c, have, v);
    };
    const int64_t k = first + g, p0 = k * chunk, p1 = p0 + chunk;
    int32_t row = -1;
    if (k < chunks && p1 < n) {
        const int32_t last = rows[p1 - 1], next = rows[p1], before = p0 > 0 ? rows[p0 - 1] : -1;
        if (static_cast<uint32_t>(last) < V && next == last && before != last) row = last;
    }
    const int64_t end = k + 1 + kShort < chunks ? k + 1 + kShort : chunks;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    bool more = false;
    if (row >= 0) {
        more = add(sum, row, k + 1, 1, end) && end < chunks && rows[end * chunk] == row;
        if (!more && have > 0) finish(sum, row, k);
    }
    if (l == 0) long_row[g] = more ? row : -1;
    __syncthreads();
    for (int at = 0; at < kGroups; ++at) {
        const int32_t which = long_row[at];
        if (which < 0) continue;
        float mine[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) mine[i] = 0.f;
        const int64_t after = first + at + 1;
        if (after + kLong >= chunks || rows[(after + kLong) * chunk] != which) {
            add(mine, which, after + g, kGroups, chunks);
        } else {
            const int64_t from = (after + kWindow - 1) / kWindow, end = chunks / kWindow;
            if (threadIdx.x == 0) first_open = static_cast<int>(end);
            __syncthreads();
            for (int64_t w = from + threadIdx.x; w < end; w += kJoinThreads)
                if (rows[(w * kWindow + kWindow - 1) * chunk] != which) {
                    atomicMin(&first_open, static_cast<int>(w));
                    break;
                }
            add(mine, which, after + g, kGroups, from * kWindow < chunks ? from * kWindow : chunks);
            __syncthreads();
#pragma unroll 8
            for (int64_t w = from + g; w < first_open; w += kGroups) {
                float v[8];
                load8(sums + w * D + (have > 0 ? c : 0), have, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) mine[i] += v[i];
            }
            add(mine, which, static_cast<int64_t>(first_open) * kWindow + g, kGroups, chunks);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) part[g][8 * l + i] = mine[i];
        __syncthreads();
        if (g == 0 && have > 0) {
#pragma unroll 4
            for (int q = 1; q < kGroups; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) mine[i] += part[q][8 * l + i];
            finish(mine, which, first + at);
        }
        __syncthreads();
    }
}

// matrices of more elements than this leave past the caches
bool large(int64_t elements) { return elements > int64_t{1} << 22; }
int lanes_of(int64_t D) { return D > 256 ? 64 : (D > 128 ? 32 : (D > 64 ? 16 : (D > 32 ? 8 : 4))); }
int64_t across_of(int64_t D, int lanes) { return (D + 8 * lanes - 1) / (8 * lanes); }

// Entries of a chunk: 16 or so many that some 4,096 waves have one chunk for each of their groups.
int64_t chunk_of(int64_t n, int64_t D) {
    const int lanes = lanes_of(D);
    int64_t groups = 4096 * (64 / lanes) / across_of(D, lanes);
    if (groups < 64) groups = 64;
    const int64_t c = (n + groups - 1) / groups;
    return c < 16 ? 16 : c;
}
int64_t chunks_of(int64_t n, int64_t D) { return (n + chunk_of(n, D) - 1) / chunk_of(n, D); }
template <int LANES, typename T>
hipError_t lookup(const void* table, int64_t ldt, const void* index, bool wide, float scale, void* out, int64_t ldo,
                  int64_t n, int64_t V, int64_t D, hipStream_t stream) {
    constexpr int kGroups = 256 / LANES;
    const int64_t across = across_of(D, LANES);
    const bool few = n * across <= 4096 * kGroups;  // one row to a group still leaves CUs without work
    const int64_t at_once = kGroups * (few ? 1 : 4);
    int64_t blocks = (n + at_once - 1) / at_once;
    if (blocks > kMostBlocks / across) blocks = kMostBlocks / across;
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(across));
    const T* t = static_cast<const T*>(table);
    if (few)
        hipLaunchKernelGGL((embedding_kernel<LANES, 1, T>), grid, dim3(256), 0, stream, t, ldt, index, wide, scale,
                           static_cast<T*>(out), ldo, n, V, D, large(n * D));
    else
        hipLaunchKernelGGL((embedding_kernel<LANES, 4, T>), grid, dim3(256), 0, stream, t, ldt, index, wide, scale,
                           static_cast<T*>(out), ldo, n, V, D, large(n * D));
    return hipGetLastError();
}

template <int LANES, typename TG, typename TO>
hipError_t gradient(const EmbeddingBwdArgs& a, hipStream_t stream) {
    const int64_t across = across_of(a.D, LANES), chunks = chunks_of(a.n, a.D), chunk = chunk_of(a.n, a.D);
    const int64_t sums = (chunks + 256 / LANES - 1) / (256 / LANES) * across, looked = 4 * kEmptyRows;
    float* const window_sums = a.partial + 2 * chunks * a.D;
    int64_t empty = (a.V + looked - 1) / looked;
    if (empty > kMostBlocks) empty = kMostBlocks;
    hipLaunchKernelGGL((embedding_sum_kernel<LANES, TG, TO>), dim3(static_cast<unsigned>(sums + empty)), dim3(256), 0,
                       stream, static_cast<const TG*>(a.grad), a.ldg, a.order, a.rows, a.scale, static_cast<TO*>(a.out),
                       a.ldo, a.partial, window_sums, a.n, a.V, a.D, chunk, static_cast<unsigned>(across),
                       static_cast<unsigned>(sums), large(a.V * a.D));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || chunks <= 1) return e;
    constexpr int kJoinLanes = LANES < 32 ? LANES : 32, kGroups = kJoinThreads / kJoinLanes;
    const int64_t join_across = across_of(a.D, kJoinLanes);
    hipLaunchKernelGGL((embedding_join_kernel<kJoinLanes, 256 / LANES, TO>),
                       dim3(static_cast<unsigned>((chunks + kGroups - 1) / kGroups * join_across)), dim3(kJoinThreads), 0, stream,
                       a.partial, window_sums, a.rows, a.scale, static_cast<TO*>(a.out), a.ldo, a.n, a.V, a.D, chunk, chunks,
                       static_cast<unsigned>(join_across));
    return hipGetLastError();
}

template <int LANES>
hipError_t gradient_types(const EmbeddingBwdArgs& a, hipStream_t stream) {
    if (a.dtype == SPINGTP_FP32)
        return a.out_dtype == SPINGTP_FP32 ? gradient<LANES, float, float>(a, stream)
                                           : gradient<LANES, float, uint16_t>(a, stream);
    return a.out_dtype == SPINGTP_FP32 ? gradient<LANES, uint16_t, float>(a, stream)
                                       : gradient<LANES, uint16_t, uint16_t>(a, stream);
}

template <typename T>
hipError_t lookup_lanes(const void* table, int64_t ldt, const void* index, bool wide, float scale, void* out, int64_t ldo,
                        int64_t n, int64_t V, int64_t D, hipStream_t stream) {
    switch (lanes_of(D)) {
        case 64: return lookup<64, T>(table, ldt, index, wide, scale, out, ldo, n, V, D, stream);
        case 32: return lookup<32, T>(table, ldt, index, wide, scale, out, ldo, n, V, D, stream);
        case 16: return lookup<16, T>(table, ldt, index, wide, scale, out, ldo, n, V, D, stream);
        case 8: return lookup<8, T>(table, ldt, index, wide, scale, out, ldo, n, V, D, stream);
        default: return lookup<4, T>(table, ldt, index, wide, scale, out, ldo, n, V, D, stream);
    }
}

}  // namespace

hipError_t launch_embedding(int dtype, const void* table, int64_t ldt, const void* index, bool wide, float scale, void* out,
                            int64_t ldo, int64_t n, int64_t V, int64_t D, hipStream_t stream) {
    return dtype == SPINGTP_FP32 ? lookup_lanes<float>(table, ldt, index, wide, scale, out, ldo, n, V, D, stream)
                                 : lookup_lanes<uint16_t>(table, ldt, index, wide, scale, out, ldo, n, V, D, stream);
}

size_t embedding_backward_workspace(int64_t n, int64_t D) {
    const int64_t chunks = chunks_of(n, D);
    return static_cast<size_t>((2 * chunks + chunks / (256 / lanes_of(D))) * D) * sizeof(float);
}

hipError_t launch_embedding_backward(const EmbeddingBwdArgs& a, hipStream_t stream) {
    switch (lanes_of(a.D)) {
        case 64: return gradient_types<64>(a, stream);
        case 32: return gradient_types<32>(a, stream);
        case 16: return gradient_types<16>(a, stream);
        case 8: return gradient_types<8>(a, stream);
        default: return gradient_types<4>(a, stream);
    }
}

}  // namespace spingtp
