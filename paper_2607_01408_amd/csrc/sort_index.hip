// An index sorted by the rows that it names: the order in which a gradient of a lookup is summed.
//
// Digits of at most 9 bits from the lowest on, each pass stable: a key goes behind all keys of smaller digits, and of
// its own digit behind those before it.  Within a wave the lanes of the same digit are found by ballots of its bits,
// so no step depends on the order of arrival.  Up to 8,192 keys one workgroup sorts in LDS; beyond, a pass is two launches,
// counts per workgroup and the moves, at most 512 workgroups, each of which adds the others' counts up for itself.
//
// A pass's time is launches, ballots and latency, not its bytes.  A call in us, keys / rows: 2,000 / 4,000 7,
// 8,000 / 50,000 17, 16,384 / 50,000 22 (a pass: counts 3, moves 7), 100,000 / 4,000 23 (3 and 8), 1,000,000 / 250,000 105.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.h"
#include "lds_common.h"
#include "training.h"

namespace spingtp {
namespace {

constexpr int kMostBits = 9, kBins = 1 << kMostBits;
constexpr int kSmall = 8192;     // keys that one workgroup sorts
constexpr int kSmallWaves = 16;
constexpr int kSortWaves = 8;
constexpr int kMostSortBlocks = 512;
static_assert(64 * kSortWaves == kBins, "a digit to each thread");

__device__ __forceinline__ uint32_t key_of(const void* index, bool wide, int64_t i, uint32_t V) {
    if (wide) {
        const uint64_t k = static_cast<uint64_t>(static_cast<const int64_t*>(index)[i]);
        return k < V ? static_cast<uint32_t>(k) : V;
    }
    const uint32_t k = static_cast<uint32_t>(static_cast<const int32_t*>(index)[i]);
    return k < V ? k : V;
}

// Lanes with the same digit as this one, among those that have a key.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, bool have) {
    uint64_t same = __ballot(have);
    for (int b = 0; b < bits; ++b) {
        const bool one = (digit >> b) & 1;
        const uint64_t ones = __ballot(one);
        same &= one ? ones : ~ones;
    }
    return same;
}
// The lane's place among the wave's keys of its digit so far, counted on in `counts`.
__device__ __forceinline__ uint32_t place_of(uint32_t digit, int bits, bool have, uint32_t* counts, int lane) {
    const uint64_t same = same_digit(digit, bits, have);
    const uint64_t below = same & ((uint64_t{1} << lane) - 1);
    const uint32_t before = have ? counts[digit] : 0;
    wave_lds_order();
    if (have && below == 0) counts[digit] = before + __popcll(same);
    wave_lds_order();
    return before + __popcll(below);
}

// Thread t (of kBins and more) with digit t's number of keys: those of smaller digits.  `scratch`: kBins / 64 words.
__device__ __forceinline__ uint32_t smaller_digits(uint32_t mine, uint32_t* scratch) {
    const int t = threadIdx.x, lane = t & 63;
    uint32_t sum = mine;  // of the digits up to this one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(sum, d, 64);
        if (lane >= d) sum += o;
    }
    if (t < kBins && lane == 63) scratch[t >> 6] = sum;
    __syncthreads();
    uint32_t base = sum - mine;
    for (int w = 0; w < (t >> 6) && w < kBins / 64; ++w) base += scratch[w];
    return base;
}

// Every wave has its keys, 64 at a time in their order, in registers; LDS takes them once a pass.
__global__ __launch_bounds__(64 * kSmallWaves) void sort_small_kernel(const void* index, bool wide, int32_t* order,
                                                                      int32_t* rows, int n, uint32_t V, int passes,
                                                                      int bits) {
    extern __shared__ __align__(16) uint32_t sort_lds[];
    uint32_t* counts = sort_lds;                       // [kSmallWaves][kBins]
    uint32_t* scratch = counts + kSmallWaves * kBins;  // [16]
    uint32_t* keys = scratch + 16;                     // [kSmall]
    uint16_t* at = reinterpret_cast<uint16_t*>(keys + kSmall);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = (n + 64 * kSmallWaves - 1) / (64 * kSmallWaves) * 64;  // keys of a wave, in a row
    const uint32_t mask = (1u << bits) - 1;
    uint32_t* mine = counts + wave * kBins;
    constexpr int kGroups = kSmall / (64 * kSmallWaves);
    uint32_t key[kGroups], from[kGroups], place[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int i = wave * per + 64 * g + lane;
        const bool have = 64 * g < per && i < n;
        key[g] = have ? key_of(index, wide, i, V) : 0;
        from[g] = i;
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * bits;
        for (int i = threadIdx.x; i < kSmallWaves * kBins; i += 64 * kSmallWaves) counts[i] = 0;
        __syncthreads();
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (64 * g >= per) break;
            place[g] = place_of((key[g] >> shift) & mask, bits, wave * per + 64 * g + lane < n, mine, lane);
        }
        __syncthreads();
        uint32_t whole = 0;
        if (threadIdx.x < kBins) {
#pragma unroll
            for (int w = 0; w < kSmallWaves; ++w) whole += counts[w * kBins + threadIdx.x];
        }
        uint32_t base = smaller_digits(whole, scratch);
        if (threadIdx.x < kBins) {
#pragma unroll
            for (int w = 0; w < kSmallWaves; ++w) {
                const uint32_t c = counts[w * kBins + threadIdx.x];
                counts[w * kBins + threadIdx.x] = base;
                base += c;
            }
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (64 * g >= per) break;
            if (wave * per + 64 * g + lane < n) {
                const uint32_t p = mine[(key[g] >> shift) & mask] + place[g];
                keys[p] = key[g];
                at[p] = static_cast<uint16_t>(from[g]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (64 * g >= per) break;
            const int i = wave * per + 64 * g + lane;
            if (i < n) key[g] = keys[i], from[g] = at[i];
        }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        if (64 * g >= per) break;
        const int i = wave * per + 64 * g + lane;
        if (i < n) rows[i] = static_cast<int32_t>(key[g]), order[i] = static_cast<int32_t>(from[g]);
    }
}

// The keys of a pass: the index itself in the first, what the pass before wrote later.
struct SortFrom {
    const void* index;  // may be null
    bool wide;
    const uint32_t* keys;
    const uint32_t* at;
    uint32_t V;
    int shift, bits;
    int64_t n, per;  // keys of a workgroup
};
__device__ __forceinline__ uint32_t sort_key(const SortFrom& f, int64_t i) {
    return f.index != nullptr ? key_of(f.index, f.wide, i, f.V) : f.keys[i];
}

__global__ __launch_bounds__(64 * kSortWaves) void sort_count_kernel(SortFrom f, uint32_t* counts) {
    __shared__ uint32_t bins[kBins];
    bins[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = blockIdx.x * f.per, end = first + f.per < f.n ? first + f.per : f.n;
    for (int64_t i = first + threadIdx.x; i < end; i += 64 * kSortWaves)
        atomicAdd(&bins[(sort_key(f, i) >> f.shift) & ((1u << f.bits) - 1)], 1u);  // whole numbers: any order
    __syncthreads();
    counts[static_cast<int64_t>(blockIdx.x) * kBins + threadIdx.x] = bins[threadIdx.x];
}

// A workgroup moves its keys in rounds of kRound, in their order.
constexpr int kMoveGroups = 4, kRound = 64 * kSortWaves * kMoveGroups;
__global__ __launch_bounds__(64 * kSortWaves) void sort_move_kernel(SortFrom f, const uint32_t* counts, uint32_t* keys,
                                                                    uint32_t* at) {
    __shared__ uint32_t bins[kSortWaves * kBins];
    __shared__ uint32_t scratch[kBins / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t mask = (1u << f.bits) - 1;
    uint32_t* mine = bins + wave * kBins;
    const int64_t first = blockIdx.x * f.per, end = first + f.per < f.n ? first + f.per : f.n;
    uint32_t key[kMoveGroups], from[kMoveGroups], place[kMoveGroups];
    const auto take = [&](int64_t round) {
#pragma unroll
        for (int g = 0; g < kMoveGroups; ++g) {
            const int64_t i = round + (wave * kMoveGroups + g) * 64 + lane;
            key[g] = i < end ? sort_key(f, i) : 0;
            from[g] = f.index != nullptr || i >= end ? static_cast<uint32_t>(i) : f.at[i];
        }
    };
    take(first);
    // digit by thread, where they are few several threads to one, each with every so many workgroups' counts
    const unsigned parts = kBins >> f.bits, digit = threadIdx.x & mask;
    uint32_t base = 0, total = 0;
#pragma unroll 16
    for (unsigned b = threadIdx.x >> f.bits; b < gridDim.x; b += parts) {
        const uint32_t c = counts[static_cast<int64_t>(b) * kBins + digit];
        base += b < blockIdx.x ? c : 0;
        total += c;
    }
    if (parts > 1) {
        bins[threadIdx.x] = base;
        bins[kBins + threadIdx.x] = total;
        __syncthreads();
        base = total = 0;
        if (threadIdx.x <= mask)
            for (unsigned q = 0; q < parts; ++q) {
                base += bins[(q << f.bits) + threadIdx.x];
                total += bins[kBins + (q << f.bits) + threadIdx.x];
            }
    }
    base += smaller_digits(total, scratch);
    for (int64_t round = first; round < end; round += kRound) {
        if (round > first) take(round);
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) bins[w * kBins + threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int g = 0; g < kMoveGroups; ++g)
            place[g] = place_of((key[g] >> f.shift) & mask, f.bits, round + (wave * kMoveGroups + g) * 64 + lane < end, mine,
                                lane);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = bins[w * kBins + threadIdx.x];
            bins[w * kBins + threadIdx.x] = base;
            base += c;
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < kMoveGroups; ++g) {
            if (round + (wave * kMoveGroups + g) * 64 + lane < end) {
                const uint32_t p = mine[(key[g] >> f.shift) & mask] + place[g];
                keys[p] = key[g];
                at[p] = from[g];
            }
        }
        __syncthreads();
    }
}

// Many keys are moved by digits of 6 bits: with 512 places to go to, four keys of a round lie side by side, and a pass
// over a million keys takes 150 us where it takes 35 with 64.  Up to 65,536 keys the launches count (two passes over
// 60,000 28 us, three 31).
void digits(int64_t n, int64_t V, int& passes, int& bits) {
    int all = 1;  // of the numbers 0 to V
    while (all < 31 && (V >> all) != 0) ++all;
    const int most = n > 65536 ? 6 : kMostBits;
    passes = (all + most - 1) / most;
    bits = (all + passes - 1) / passes;
}
int64_t up4(int64_t n) { return (n + 3) / 4 * 4; }

}  // namespace

size_t sort_index_workspace(int64_t n, int64_t V) {
    int passes, bits;
    digits(n, V, passes, bits);
    if (n <= kSmall) return 0;
    return static_cast<size_t>(kMostSortBlocks * kBins + (passes > 1 ? 2 * up4(n) : 0)) * sizeof(uint32_t);
}

hipError_t launch_sort_index(const void* index, bool wide, int32_t* order, int32_t* rows, void* workspace, int64_t n,
                             int64_t V, hipStream_t stream) {
    int passes, bits;
    digits(n, V, passes, bits);
    if (n <= kSmall) {
        const hipError_t e = raise_lds_limit<sort_small_kernel>();
        if (e != hipSuccess) return e;
        constexpr int lds = (kSmallWaves * kBins + 16 + kSmall) * 4 + kSmall * 2;
        static_assert(lds <= 160 * 1024, "in LDS");
        hipLaunchKernelGGL(sort_small_kernel, dim3(1), dim3(64 * kSmallWaves), lds, stream, index, wide, order, rows,
                           static_cast<int>(n), static_cast<uint32_t>(V), passes, bits);
        return hipGetLastError();
    }
    int64_t per = (n + kMostSortBlocks - 1) / kMostSortBlocks;
    per = (per + kRound - 1) / kRound * kRound;
    const unsigned blocks = static_cast<unsigned>((n + per - 1) / per);
    uint32_t* counts = static_cast<uint32_t*>(workspace);
    uint32_t* tmp = counts + kMostSortBlocks * kBins;
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(rows), tmp};
    uint32_t* at[2] = {reinterpret_cast<uint32_t*>(order), tmp + up4(n)};
    SortFrom f{index, wide, nullptr, nullptr, static_cast<uint32_t>(V), 0, bits, n, per};
    for (int pass = 0; pass < passes; ++pass) {
        const int to = (passes - 1 - pass) & 1;  // the last pass writes the results
        hipLaunchKernelGGL(sort_count_kernel, dim3(blocks), dim3(64 * kSortWaves), 0, stream, f, counts);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(sort_move_kernel, dim3(blocks), dim3(64 * kSortWaves), 0, stream, f, counts, keys[to], at[to]);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        f.index = nullptr;
        f.keys = keys[to];
        f.at = at[to];
        f.shift += bits;
    }
    return hipSuccess;
}

}  // namespace spingtp
