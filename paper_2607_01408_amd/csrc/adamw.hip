// AdamW over many tensors:
//   g' = grad_scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = (1 - lr wd) p - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps).
//
// One launch for as many tensors as its arguments hold; a workgroup finds its tensor there and takes 2,048 neighbouring
// elements of it, eight to a lane.  Nothing is uploaded, so a captured launch keeps its own table.
//
// States in 8 bits: m and sqrt(v) (half of v's range of exponents) in blocks of 128 elements, 16 lanes.  A step of v moves
// it by a thousandth, a step of the format is a sixteenth to an eighth: rounded to nearest, v would stay where it is.  So
// each value goes to one of its two neighbours by 16 random bits, with the chance at which the mean of m, and of v, is
// kept.  The bits are a mix of the step, the tensor's place and the element's, so a step gives the same states wherever
// and in however many launches it runs; m and v are computed without contraction for the same reason.  A v that was
// rounded to zero beside an m that was not would make an endless step: v is at least (m / c)^2,
// c = (1 - b1) / sqrt((1 - b2) (1 - b1^2 / b2)), which exact sums of the same gradients keep by themselves
// (Cauchy and Schwarz).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "block8.h"
#include "internal.h"
#include "training.h"

namespace spingtp {
namespace {

struct AdamwEntry {
    void* p;
    const void* g;
    void* m;
    void* v;
    uint8_t* ms;
    uint8_t* vs;
    uint16_t* copy;
    int64_t n;      // elements, of this piece
    int64_t first;  // of the piece in its tensor
    uint32_t place;
    uint32_t kinds;  // kParam16, ...
};
enum : uint32_t { kParam16 = 1, kGrad16 = 2 };
constexpr int kMostEntries = 46;  // with them the arguments stay below 4 KB; at most a wave's lanes
constexpr int kAdamwChunk = 2048;

struct AdamwArgs {
    float b1, c1, b2, c2;  // c: 1 - b
    float eps, least;      // 1 / c above, 0 where there is no bound
    float decay, rate;     // 1 - lr wd, lr / (1 - b1^t)
    float root;            // (1 - b2^t)^(-1/2)
    double wd, log_b1, log_b2;
    int64_t step;
    uint64_t seed;
    const int64_t* device_step;  // may be null: the step, lr and the factor of the gradients
    const float* device_lr;
    const float* grad_scale;
    double lr;
    int entries;
    uint32_t block[kMostEntries];  // an entry's first workgroup
    AdamwEntry entry[kMostEntries];
};
static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");

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
                                          uint8_t* values, uint8_t* scale, bool leader) {
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
            more = share * ((hi - lo) * (hi + lo)) < x[i] * inv * inv - lo * lo;
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

__global__ __launch_bounds__(256) void adamw_kernel(AdamwArgs a) {
    // the last entry that begins here or before, a lane to each: one read of the arguments
    const int lane = threadIdx.x & 63;
    const uint32_t begins = a.block[lane < kMostEntries ? lane : 0];
    const int at = __popcll(__ballot(lane < a.entries && begins <= blockIdx.x)) - 1;
    const AdamwEntry& t = a.entry[at];
    const uint32_t block = blockIdx.x - a.block[at];
    float decay = a.decay, rate = a.rate, root = a.root;
    int64_t step = a.step;
    if (a.device_step != nullptr || a.device_lr != nullptr) {
        if (a.device_step != nullptr) step = *a.device_step > 1 ? *a.device_step : 1;
        const double lr = a.device_lr != nullptr ? static_cast<double>(*a.device_lr) : a.lr;
        decay = static_cast<float>(1.0 - lr * a.wd);
        rate = static_cast<float>(lr / -expm1(static_cast<double>(step) * a.log_b1));
        root = static_cast<float>(1.0 / sqrt(-expm1(static_cast<double>(step) * a.log_b2)));
    }
    const int64_t i0 = static_cast<int64_t>(block) * kAdamwChunk + threadIdx.x * 8;
    const int64_t left = t.n - i0;
    const int have = left >= 8 ? 8 : (left > 0 ? static_cast<int>(left) : 0);
    const bool blocks = t.ms != nullptr;
    // a block's sixteen lanes stay together: their places reach past n
    if (i0 >= (blocks ? (t.n + kBlock8 - 1) / kBlock8 * kBlock8 : t.n)) return;
    const int64_t from = have > 0 ? i0 : 0;
    float p[8], g[8], m[8], v[8];
    if (t.kinds & kParam16)
        pass8(static_cast<const uint16_t*>(t.p) + from, have, p);
    else
        pass8(static_cast<const float*>(t.p) + from, have, p);
    if (t.kinds & kGrad16)
        pass8(static_cast<const uint16_t*>(t.g) + from, have, g);
    else
        pass8(static_cast<const float*>(t.g) + from, have, g);
    if (blocks) {
        const uint2 wm = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.m) + i0);
        const uint2 wv = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + i0);
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
        pass8(static_cast<const float*>(t.m) + from, have, m);
        pass8(static_cast<const float*>(t.v) + from, have, v);
    }
    const float factor = a.grad_scale != nullptr ? *a.grad_scale : 1.f;
    float size[8], s[8];
    {
#pragma clang fp contract(off)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = g[i] * factor;
            m[i] = a.b1 * m[i] + a.c1 * x;
            v[i] = a.b2 * v[i] + a.c2 * (x * x);
            if (blocks) {
                const float y = m[i] * a.least, least = y * y;
                v[i] = least > v[i] ? least : v[i];
                if (i >= have) m[i] = v[i] = 0.f;  // zeros behind the tensor whatever lies there
            }
            s[i] = sqrtf(v[i]);
            size[i] = fabsf(m[i]);
            p[i] = p[i] * decay - rate * (m[i] / (s[i] * root + a.eps));
        }
    }
    if (t.kinds & kParam16) {
        store8(static_cast<uint16_t*>(t.p) + from, have, p);
    } else {
        store8(static_cast<float*>(t.p) + from, have, p);
        if (t.copy != nullptr) store8(t.copy + from, have, p);
    }
    if (!blocks) {
        store8(static_cast<float*>(t.m) + from, have, m);
        store8(static_cast<float*>(t.v) + from, have, v);
        return;
    }
    const uint32_t key =
        mix(mix(static_cast<uint32_t>(a.seed) + t.place * 0x9E3779B9u) + static_cast<uint32_t>(step) * 0x3C6EF373u +
            static_cast<uint32_t>(a.seed >> 32));
    const int64_t e = t.first + i0;
    const uint32_t high = static_cast<uint32_t>(e >> 32) * 0x3C6EF373u + key;  // of all eight: a multiple of 8
    uint32_t word[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) word[i] = mix((static_cast<uint32_t>(e) + i) * 0x9E3779B9u + high);
    const bool leader = (threadIdx.x & 15) == 0;
    put_block<false>(m, size, word, static_cast<uint8_t*>(t.m) + i0, t.ms + i0 / kBlock8, leader);
    put_block<true>(v, s, word, static_cast<uint8_t*>(t.v) + i0, t.vs + i0 / kBlock8, leader);
}

constexpr int64_t kMostPiece = int64_t{1} << 30;  // elements of an entry

}  // namespace

hipError_t launch_adamw(const spingtp_adamw_tensor* tensors, int64_t count, const spingtp_adamw_options& o,
                        hipStream_t stream) {
    AdamwArgs a{};
    a.b1 = static_cast<float>(o.beta1);
    a.c1 = static_cast<float>(1.0 - o.beta1);
    a.b2 = static_cast<float>(o.beta2);
    a.c2 = static_cast<float>(1.0 - o.beta2);
    a.eps = static_cast<float>(o.eps);
    const double bound = o.beta2 > 0 ? 1.0 - o.beta1 * o.beta1 / o.beta2 : 0.0;
    a.least = bound > 0 ? static_cast<float>(std::sqrt((1.0 - o.beta2) * bound) / (1.0 - o.beta1)) : 0.f;
    a.wd = o.weight_decay;
    a.lr = o.lr;
    a.log_b1 = std::log(o.beta1);
    a.log_b2 = std::log(o.beta2);
    a.step = o.step;
    a.seed = o.seed;
    a.device_step = o.device_step;
    a.device_lr = o.device_lr;
    a.grad_scale = o.grad_scale;
    const double t = static_cast<double>(o.step > 1 ? o.step : 1);
    a.decay = static_cast<float>(1.0 - o.lr * o.weight_decay);
    a.rate = static_cast<float>(o.lr / -std::expm1(t * a.log_b1));
    a.root = static_cast<float>(1.0 / std::sqrt(-std::expm1(t * a.log_b2)));
    int64_t blocks = 0;
    const auto flush = [&]() {
        if (a.entries == 0) return hipSuccess;
        hipLaunchKernelGGL(adamw_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a);
        a.entries = 0;
        blocks = 0;
        return hipGetLastError();
    };
    for (int64_t k = 0; k < count; ++k) {
        const spingtp_adamw_tensor& x = tensors[k];
        for (int64_t first = 0; first < x.n; first += kMostPiece) {
            const int64_t n = x.n - first < kMostPiece ? x.n - first : kMostPiece;
            const int64_t mine = (n + kAdamwChunk - 1) / kAdamwChunk;
            if (a.entries == kMostEntries || blocks + mine > kMostBlocks) {
                const hipError_t e = flush();
                if (e != hipSuccess) return e;
            }
            a.block[a.entries] = static_cast<uint32_t>(blocks);
            AdamwEntry& to = a.entry[a.entries++];
            const int64_t pw = x.param_dtype == SPINGTP_FP32 ? 4 : 2, gw = x.grad_dtype == SPINGTP_FP32 ? 4 : 2;
            const bool eight = x.m_scales != nullptr;
            to.p = static_cast<uint8_t*>(x.param) + first * pw;
            to.g = static_cast<const uint8_t*>(x.grad) + first * gw;
            to.m = static_cast<uint8_t*>(x.m) + first * (eight ? 1 : 4);
            to.v = static_cast<uint8_t*>(x.v) + first * (eight ? 1 : 4);
            to.ms = eight ? static_cast<uint8_t*>(x.m_scales) + first / kBlock8 : nullptr;
            to.vs = eight ? static_cast<uint8_t*>(x.v_scales) + first / kBlock8 : nullptr;
            to.copy = x.copy != nullptr ? static_cast<uint16_t*>(x.copy) + first : nullptr;
            to.n = n;
            to.first = first;
            to.place = static_cast<uint32_t>(k);
            to.kinds = (pw == 2 ? kParam16 : 0) | (gw == 2 ? kGrad16 : 0);
            blocks += mine;
        }
    }
    return flush();
}

}  // namespace spingtp
