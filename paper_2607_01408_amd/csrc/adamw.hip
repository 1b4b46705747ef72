// AdamW over many tensors:
//   g' = grad_scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = (1 - lr wd) p - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps).
//
// One launch for as many tensors of a kind (types, states) as its arguments hold; a workgroup finds its tensor there and
// takes 2,048 neighbouring elements of it, eight to a lane.  Nothing is uploaded, so a captured launch keeps its own table.
// Bound by memory: 22 million elements in fp32 123 us (28 bytes each, 5.0 TB/s), 44 million with 8-bit states, bf16
// gradients and copies 140 (16 bytes each, 5.1 TB/s); 240 small tensors 29.5, the checks of 960 tensors on the host and
// three launches.
//
// States in 8 bits: m and sqrt(v) (half of v's range of exponents) in blocks of 128 elements, 16 lanes.  A step of v moves
// it by a thousandth, a step of the format is a sixteenth to an eighth: rounded to nearest, v would stay where it is.  So
// each value goes to one of its two neighbours by 16 random bits, with the chance at which the mean of m, and of v, is
// kept.  The bits are a mix of the step, the tensor's place and the element's, so a step gives the same states wherever
// and in however many launches it runs; m and v are computed without contraction for the same reason.  A v that was
// rounded to zero beside an m that was not would make an endless step: v is at least (m / c)^2,
// c = (1 - b1) / sqrt((1 - b2) (1 - b1^2 / b2)), which exact sums of the same gradients keep by themselves
// (Cauchy and Schwarz).  From r = b1^2 / b2 = 1 - 2^-20 on that sum over all steps bounds nothing, and two things take its
// place: the sum over the t steps so far, 1 + r + ... + r^(t-1) in place of 1 / (1 - r), which is no bound either once r^t
// is large; and a v above zero is never rounded to zero but to the smallest number of its block's format.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "block8.h"
#include "internal.h"
#include "training.h"

namespace spingtp {
namespace {

constexpr int kAdamwChunk = 2048;
constexpr int kArgumentBytes = 4096;

// A tensor, or a piece of one: what every kind has, its states in fp32 or 8 bits, the bf16 copy where the list has any.
// The shorter an entry, the more tensors to a launch: 99 in fp32 without copies, 82 where there is room for them.
struct EntryBase {
    uint32_t block;  // first workgroup
    uint32_t n;      // elements
    void* p;
    const void* g;
};
struct Entry32 : EntryBase {
    float* m;
    float* v;
};
struct Entry8 : EntryBase {
    uint8_t* m;
    uint8_t* v;
    uint8_t* ms;
    uint8_t* vs;
    uint32_t place;  // in the list
    uint32_t piece;  // of the tensor, kMostPiece elements each
};
template <typename T, bool COPY>
struct EntryWith : T {};
template <typename T>
struct EntryWith<T, true> : T {
    uint16_t* copy;
};
constexpr int64_t kMostPiece = int64_t{1} << 30;  // elements of an entry
struct AdamwNumbers {
    float b1, c1, b2, c2;  // c: 1 - b
    float eps, least;      // least: 1 / c above, 0 where c is infinite
    float decay, rate;     // 1 - lr wd, lr / (1 - b1^t)
    float root;            // (1 - b2^t)^(-1/2)
    int entries;
    bool around;  // the tensors are too large for the caches
    bool short_bound;  // c is of the steps so far, and no v above zero is rounded to zero
    double wd, lr, log_b1, log_b2;
    int64_t step;
    uint64_t seed;
    const int64_t* device_step;  // may be null: the step, lr and the factor of the gradients
    const float* device_lr;
    const float* grad_scale;
};
template <bool BITS8, bool COPY>
struct AdamwArgs {
    using Entry = EntryWith<std::conditional_t<BITS8, Entry8, Entry32>, COPY>;
    static constexpr int kMost = (kArgumentBytes - sizeof(AdamwNumbers)) / sizeof(Entry);
    AdamwNumbers o;
    Entry entry[kMost];
};
static_assert(sizeof(AdamwArgs<false, false>) <= kArgumentBytes && sizeof(AdamwArgs<true, true>) <= kArgumentBytes);
static_assert(AdamwArgs<false, false>::kMost == 99 && AdamwArgs<false, true>::kMost == 82);
static_assert(AdamwArgs<true, false>::kMost == 62 && AdamwArgs<true, true>::kMost == 55);

// 1 / c of the first t steps: c^2 = (1 - b1)^2 / (1 - b2) (r^t - 1) / (r - 1); 0 where that is infinite
__host__ __device__ inline float least_of_steps(const AdamwNumbers& o, int64_t t) {
    const double log_r = 2.0 * o.log_b1 - o.log_b2;
    const double sum = log_r == 0.0 ? static_cast<double>(t) : expm1(static_cast<double>(t) * log_r) / expm1(log_r);
    const double c1 = -expm1(o.log_b1), c2 = -expm1(o.log_b2);
    return sum > 0.0 && sum < 1e300 ? static_cast<float>(sqrt(c2 / sum) / c1) : 0.f;
}

__host__ __device__ inline uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

// The numbers on either side of t >= 0 in e4m3 (t below 464): three bits behind the leading one, a step of 2^-9 below 2^-6.
__device__ __forceinline__ void neighbours(float t, float& lo, float& hi) {
#pragma clang fp contract(off)
    const float base = t < 0x1p-6f ? 0x1p-6f : 0.f;
    const uint32_t bits = __float_as_uint(t + base) & ~0xFFFFFu;
    lo = __uint_as_float(bits) - base;
    hi = __uint_as_float(bits + 0x100000u) - base;
}
// (r + 1/2) 2^-16 of 16 random bits
__device__ __forceinline__ float share_of(uint32_t r) {
    return (static_cast<float>(r) + 0.5f) * 0x1p-16f;
}

// m, and v by its root, to their blocks: eight elements a lane, 16 lanes a block.
template <bool ROOT>
__device__ __forceinline__ void put_block(const float (&x)[8], const float (&size)[8], const uint32_t (&word)[8],
                                          uint8_t* values, uint8_t* scale, bool leader, bool none_to_zero) {
#pragma clang fp contract(off)
    const int e = block8_scale(block8_top(size));
    const float inv = block8_inverse(e);
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = size[i] * inv;
        float lo, hi;
        neighbours(t, lo, hi);
        const float share = share_of(ROOT ? word[i] >> 16 : word[i] & 0xFFFFu);
        bool more;
        if constexpr (ROOT)
            more = share * ((hi - lo) * (hi + lo)) < x[i] * inv * inv - lo * lo || (none_to_zero && lo == 0.f && x[i] > 0.f);
        else
            more = share * (hi - lo) < t - lo;
        float y = fminf(more ? hi : lo, 448.f);
        y = t <= 448.f ? y : __builtin_nanf("");  // not finite: the block's scale brings all others there
        q[i] = ROOT ? y : copysignf(y, x[i]);
    }
    *reinterpret_cast<uint2*>(values) =
        make_uint2(block8_word(q[0], q[1], q[2], q[3], 1.f), block8_word(q[4], q[5], q[6], q[7], 1.f));
    if (leader) *scale = static_cast<uint8_t>(e);
}

template <bool BITS8, typename TP, typename TG, bool COPY>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwArgs<BITS8, COPY> a) {
    // the last entry that begins here or before, a lane to each: one read of the arguments
    const AdamwNumbers& o = a.o;
    const int lane = threadIdx.x & 63;
    int at = -1;
#pragma unroll
    for (int first = 0; first < AdamwArgs<BITS8, COPY>::kMost; first += 64) {
        const int e = first + lane < o.entries ? first + lane : 0;
        at += __popcll(__ballot(first + lane < o.entries && a.entry[e].block <= blockIdx.x));
    }
    const auto& t = a.entry[at];
    const int64_t n = t.n, i0 = static_cast<int64_t>(blockIdx.x - t.block) * kAdamwChunk + threadIdx.x * 8;
    const int64_t left = n - i0;
    const int have = left >= 8 ? 8 : (left > 0 ? static_cast<int>(left) : 0);
    // a block's sixteen lanes stay together: their places reach past n
    if (i0 >= (BITS8 ? (n + kBlock8 - 1) / kBlock8 * kBlock8 : n)) return;
    const int64_t from = have > 0 ? i0 : 0;
    float p[8], g[8], m[8], v[8];
    pass8(static_cast<const TP*>(t.p) + from, have, p);
    pass8(static_cast<const TG*>(t.g) + from, have, g);
    if constexpr (BITS8) {
        const uint2 wm = *reinterpret_cast<const uint2*>(t.m + i0), wv = *reinterpret_cast<const uint2*>(t.v + i0);
        const float sm = block8_power(t.ms[i0 / kBlock8]), sv = block8_power(t.vs[i0 / kBlock8]);
        float lo[4], hi[4];
        block8_values(wm.x, lo);
        block8_values(wm.y, hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = lo[i] * sm, m[4 + i] = hi[i] * sm;
        block8_values(wv.x, lo);
        block8_values(wv.y, hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = lo[i] * sv, y = hi[i] * sv;
            v[i] = x * x, v[4 + i] = y * y;
        }
    } else {
        pass8(t.m + from, have, m);
        pass8(t.v + from, have, v);
    }
    float decay = o.decay, rate = o.rate, root = o.root, bound = o.least;
    int64_t step = o.step;
    if (o.device_step != nullptr || o.device_lr != nullptr) {
        if (o.device_step != nullptr) step = *o.device_step > 1 ? *o.device_step : 1;
        const double lr = o.device_lr != nullptr ? static_cast<double>(*o.device_lr) : o.lr;
        decay = static_cast<float>(1.0 - lr * o.wd);
        rate = static_cast<float>(lr / -expm1(static_cast<double>(step) * o.log_b1));
        root = static_cast<float>(1.0 / sqrt(-expm1(static_cast<double>(step) * o.log_b2)));
        if (BITS8 && o.short_bound) bound = least_of_steps(o, step);
    }
    const float factor = o.grad_scale != nullptr ? *o.grad_scale : 1.f;
    float size[8], s[8];
    {
#pragma clang fp contract(off)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = g[i] * factor;
            m[i] = o.b1 * m[i] + o.c1 * x;
            v[i] = o.b2 * v[i] + o.c2 * (x * x);
            if constexpr (BITS8) {
                const float y = m[i] * bound, least = y * y;
                v[i] = least > v[i] ? least : v[i];
                if (i >= have) m[i] = v[i] = 0.f;  // zeros behind the tensor whatever lies there
            }
            s[i] = sqrtf(v[i]);
            size[i] = fabsf(m[i]);
            p[i] = p[i] * decay - rate * (m[i] / (s[i] * root + o.eps));
        }
    }
    pass_store8(static_cast<TP*>(t.p) + from, have, p, o.around);
    if constexpr (COPY) {
        if (t.copy != nullptr) pass_store8(t.copy + from, have, p, o.around);
    }
    if constexpr (BITS8) {
        const uint32_t key =
            mix(mix(static_cast<uint32_t>(o.seed) + t.place * 0x9E3779B9u) + static_cast<uint32_t>(step) * 0x3C6EF373u +
                static_cast<uint32_t>(o.seed >> 32));
        const int64_t e = t.piece * kMostPiece + i0;
        const uint32_t high = static_cast<uint32_t>(e >> 32) * 0x3C6EF373u + key;  // of all eight: a multiple of 8
        uint32_t word[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) word[i] = mix((static_cast<uint32_t>(e) + i) * 0x9E3779B9u + high);
        const bool leader = (threadIdx.x & 15) == 0;
        put_block<false>(m, size, word, t.m + i0, t.ms + i0 / kBlock8, leader, false);
        put_block<true>(v, s, word, t.v + i0, t.vs + i0 / kBlock8, leader, o.short_bound);
    } else {
        pass_store8(t.m + from, have, m, o.around);
        pass_store8(t.v + from, have, v, o.around);
    }
}

// The list's tensors of one kind, in as few launches as hold them.
template <bool BITS8, typename TP, typename TG, bool COPY>
hipError_t launch_kind(const spingtp_adamw_tensor* tensors, int64_t count, const AdamwNumbers& o, hipStream_t stream) {
    AdamwArgs<BITS8, COPY> a;
    a.o = o;
    a.o.entries = 0;
    int64_t blocks = 0;
    const auto flush = [&]() {
        if (a.o.entries == 0) return hipSuccess;
        hipLaunchKernelGGL((adamw_kernel<BITS8, TP, TG, COPY>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a);
        a.o.entries = 0;
        blocks = 0;
        return hipGetLastError();
    };
    constexpr int pd = sizeof(TP) == 4 ? SPINGTP_FP32 : SPINGTP_BF16, gd = sizeof(TG) == 4 ? SPINGTP_FP32 : SPINGTP_BF16;
    for (int64_t k = 0; k < count; ++k) {
        const spingtp_adamw_tensor& x = tensors[k];
        if (x.param_dtype != pd || x.grad_dtype != gd || (x.m_scales != nullptr) != BITS8) continue;
        for (int64_t first = 0; first < x.n; first += kMostPiece) {
            const int64_t n = x.n - first < kMostPiece ? x.n - first : kMostPiece;
            const int64_t mine = (n + kAdamwChunk - 1) / kAdamwChunk;
            if (a.o.entries == AdamwArgs<BITS8, COPY>::kMost || blocks + mine > kMostBlocks) {
                const hipError_t e = flush();
                if (e != hipSuccess) return e;
            }
            auto& to = a.entry[a.o.entries++];
            to.block = static_cast<uint32_t>(blocks);
            to.p = static_cast<TP*>(x.param) + first;
            to.g = static_cast<const TG*>(x.grad) + first;
            if constexpr (COPY) to.copy = x.copy != nullptr ? static_cast<uint16_t*>(x.copy) + first : nullptr;
            to.n = static_cast<uint32_t>(n);
            if constexpr (BITS8) {
                to.m = static_cast<uint8_t*>(x.m) + first;
                to.v = static_cast<uint8_t*>(x.v) + first;
                to.ms = static_cast<uint8_t*>(x.m_scales) + first / kBlock8;
                to.vs = static_cast<uint8_t*>(x.v_scales) + first / kBlock8;
                to.place = static_cast<uint32_t>(k);
                to.piece = static_cast<uint32_t>(first / kMostPiece);
            } else {
                to.m = static_cast<float*>(x.m) + first;
                to.v = static_cast<float*>(x.v) + first;
            }
            blocks += mine;
        }
    }
    return flush();
}

}  // namespace

hipError_t launch_adamw(const spingtp_adamw_tensor* tensors, int64_t count, const spingtp_adamw_options& given,
                        hipStream_t stream) {
    AdamwNumbers o{};
    o.b1 = static_cast<float>(given.beta1);
    o.c1 = static_cast<float>(1.0 - given.beta1);
    o.b2 = static_cast<float>(given.beta2);
    o.c2 = static_cast<float>(1.0 - given.beta2);
    o.eps = static_cast<float>(given.eps);
    const double bound = given.beta2 > 0 ? 1.0 - given.beta1 * given.beta1 / given.beta2 : 0.0;
    o.short_bound = !(bound > 0x1p-20);
    o.wd = given.weight_decay;
    o.lr = given.lr;
    o.log_b1 = std::log(given.beta1);
    o.log_b2 = std::log(given.beta2);
    o.step = given.step;
    o.seed = given.seed;
    o.device_step = given.device_step;
    o.device_lr = given.device_lr;
    o.grad_scale = given.grad_scale;
    const double t = static_cast<double>(given.step > 1 ? given.step : 1);
    o.least = o.short_bound ? least_of_steps(o, given.step > 1 ? given.step : 1)
                            : static_cast<float>(std::sqrt((1.0 - given.beta2) * bound) / (1.0 - given.beta1));
    o.decay = static_cast<float>(1.0 - given.lr * given.weight_decay);
    o.rate = static_cast<float>(given.lr / -std::expm1(t * o.log_b1));
    o.root = static_cast<float>(1.0 / std::sqrt(-std::expm1(t * o.log_b2)));
    int64_t elements = 0;
    for (int64_t k = 0; k < count; ++k) elements += tensors[k].n;
    o.around = elements > int64_t{1} << 22;
    bool kinds[8] = {}, copies = false;
    for (int64_t k = 0; k < count; ++k) {
        kinds[(tensors[k].m_scales != nullptr) * 4 + (tensors[k].param_dtype == SPINGTP_BF16) * 2 +
              (tensors[k].grad_dtype == SPINGTP_BF16)] = true;
        copies = copies || tensors[k].copy != nullptr;
    }
    using Launch = hipError_t (*)(const spingtp_adamw_tensor*, int64_t, const AdamwNumbers&, hipStream_t);
    constexpr Launch plain[8] = {
        launch_kind<false, float, float, false>,    launch_kind<false, float, uint16_t, false>,
        launch_kind<false, uint16_t, float, false>, launch_kind<false, uint16_t, uint16_t, false>,
        launch_kind<true, float, float, false>,     launch_kind<true, float, uint16_t, false>,
        launch_kind<true, uint16_t, float, false>,  launch_kind<true, uint16_t, uint16_t, false>};
    // bf16 parameters have no copy
    constexpr Launch copying[8] = {
        launch_kind<false, float, float, true>, launch_kind<false, float, uint16_t, true>, plain[2], plain[3],
        launch_kind<true, float, float, true>,  launch_kind<true, float, uint16_t, true>,  plain[6], plain[7]};
    for (int i = 0; i < 8; ++i)
        if (kinds[i]) {
            const hipError_t e = (copies ? copying : plain)[i](tensors, count, o, stream);
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

}  // namespace spingtp
