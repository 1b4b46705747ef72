// Matrix product with bias, activation and residual in its epilogue, and its gradients:
//   z = x w^T + b,  y = act(z) + r,
//   dz = dy act'(z),  dx = dz w,  dw = dz^T x,  db = sum over the rows of dz.
//
// Forward: the products of gemm_nt.h; a wave's accumulators pass through its own LDS, 16 or 32 rows at a time, so that
// a lane gets eight neighbouring columns of a row: bias, residual, z and y are whole lines, each touched once.
// Backward: dz is made once, in bf16, with the columns' partial sums of it before the rounding (for many rows and few
// channels by the launch that makes dx); where there is no activation and dy is bf16 on 16 bytes it is its own dz.  dx sums
// over w's rows, dw over those of dz and x: the products read them as they lie.
//
// Few tiles and a long sum (the weights' gradients of many rows and few channels; dx of few rows) leave most of the
// CUs idle: then the sum is cut into slices, a workgroup to each, whose fp32 sums a second kernel adds in order and
// finishes.
//
// Measured (us, on one card, where a large copy reaches 5.2 TB/s, the library's bf16 product of 8,192^3 1,631 TFLOP/s, its
// products of 8,192 x 2,048 x 8,192 and 8,192 x 8,192 x 2,048 177 and 189, of the latter's gradients 205 and 240):
//   8,192 x 2,048 x 8,192 207, onto a residual 220 (1.25 PFLOP/s, matrix units busy 57 % at 2.0 GHz); 8,192 x 8,192 x 2,048
//   207, with bias and gelu 243, z kept too 253 and among a training step's other launches 298, behind whose epilogue no
//   other workgroup of the CU multiplies; its gradients' products 227 and 211;
//   100,000 x 512 x 128, silu, z kept 49 (205 MB written, 4.7 TB/s), dz and dx 66 (340 MB, 5.1 TB/s; in two launches dz 55,
//   5.6 TB/s, and dx 27), dw 27 in 63 slices, 8 to join them and to add db up;
//   one row by 8,192 x 4,096 weights 12.5 (5.4 TB/s); 24 x 2,048 x 8,192 in 8 bits 9 in slices, 3 to join them; 8 bits,
//   8,192 x 2,048 x 8,192 189, onto a residual 193, 8,192 x 8,192 x 2,048 with bias and gelu 266, 512 x 2,048 x 8,192 25;
//   all gradients of few rows (rows x outputs x inputs), silu: 1 x 8,192 x 4,096 40 (dx 21, dw 20, db 8), 24 46 (26, 24, 8),
//   256 x 2,048 x 2,048 27 (16, 14, 8).
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "activation.h"
#include "feedforward.h"
#include "gemm_nt.h"
#include "gemm_skinny.h"
#include "internal.h"
#include "lds_common.h"

namespace spingtp {
namespace {

struct LinearOut {
    int act;
    bool wide;          // r and y in fp32
    const float* bias;  // may be null
    const void* r;      // may be null
    int64_t ldr;
    void* y;
    int64_t ldy;
    uint16_t* z;     // [M][N], may be null
    bool around;     // y and z are too large for the caches
    float* partial;  // with slices: [slices][M][N] sums, and nothing else leaves
    int slice;       // steps of a slice (without: all)
};

template <int ACT>
__device__ __forceinline__ void activate(float (&v)[8]) {
    if constexpr (ACT != kIdentity) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = act<ACT>(v[i]);
    }
}
__device__ __forceinline__ void residual8(const LinearOut& o, int64_t m, int64_t n, int left, float (&v)[8]) {
    if (o.wide)
        load8(static_cast<const float*>(o.r) + m * o.ldr + n, left, v);
    else
        load8(static_cast<const uint16_t*>(o.r) + m * o.ldr + n, left, v);
}
// Eight neighbouring outputs of row m from their sums on (`bias`, `r`: zeros where there is none); the `left`
// first of them exist.
template <int ACT>
__device__ __forceinline__ void finish8(const LinearOut& o, int64_t N, int64_t m, int64_t n, int left, float (&v)[8],
                                        const float (&bias)[8], const float (&r)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += bias[i];
    if (o.z != nullptr) pass_store8(o.z + m * N + n, left, v, o.around);
    activate<ACT>(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
    if (o.wide)
        pass_store8(static_cast<float*>(o.y) + m * o.ldy + n, left, v, o.around);
    else
        pass_store8(static_cast<uint16_t*>(o.y) + m * o.ldy + n, left, v, o.around);
}

// The part of the sum that is slice `slice`.
template <class E, bool KW, bool KX>
__device__ __forceinline__ void cut_slice(GemmArgs& a, LinearOut& o, int64_t& row_bytes, int slice) {
    const int first = slice * o.slice, left = a.steps - first;
    const bool last = left <= o.slice;
    a.w += KW ? int64_t{64} * first * a.ldw : int64_t{kStepBytes} * first;
    a.x += KX ? int64_t{64} * first * a.ldx : int64_t{kStepBytes} * first;
    if constexpr (E::kScaled) a.ws += first, a.xs += first;  // a multiple of 4: whole words
    a.w_rows -= int64_t{64} * first;
    a.x_rows -= int64_t{64} * first;
    row_bytes -= int64_t{kStepBytes} * first;
    if (!last) {
        a.tail = kStepBytes;
        a.w_rows = a.x_rows = int64_t{64} * o.slice;
        a.steps = o.slice;
    } else {
        a.steps = left;
    }
    a.w_split = a.steps;
    o = LinearOut{kIdentity, true, nullptr, nullptr, 0, o.partial + static_cast<int64_t>(slice) * a.M * a.N, a.N,
                  nullptr,   false, nullptr, 0};
}

// One of PARTS equal parts of the sum, a step more or less: that step is of zeros.
template <class E, bool KW, bool KX, int PARTS>
__device__ __forceinline__ void cut_part(GemmArgs& a, int part) {
    const int first = static_cast<int>(static_cast<int64_t>(a.steps) * part / PARTS);
    const int count = static_cast<int>(static_cast<int64_t>(a.steps) * (part + 1) / PARTS) - first;
    const int most = (a.steps + PARTS - 1) / PARTS;
    a.w += KW ? int64_t{64} * first * a.ldw : int64_t{kStepBytes} * first;
    a.x += KX ? int64_t{64} * first * a.ldx : int64_t{kStepBytes} * first;
    if constexpr (E::kScaled) a.ws += first, a.xs += first;
    const int64_t rows = int64_t{64} * count;
    a.w_rows -= int64_t{64} * first;
    a.x_rows -= int64_t{64} * first;
    if (a.w_rows > rows) a.w_rows = rows;
    if (a.x_rows > rows) a.x_rows = rows;
    if (part < PARTS - 1) a.tail = kStepBytes;
    if (count < most) {
        // (where the part ends inside a step, its last step is one that exists: only the last part does, and it is whole)
        a.tail = 0;
    }
    a.steps = a.w_split = most;
}

// PARTS times the waves of a tile share its sum, each tile's worth in LDS of its own.
template <class E, int PN, int PM, int WN, int WM, int NS, bool KW, bool KX, int PARTS>
struct LinearTile : GemmTile<E, PN, PM, WN, WM, NS, false, KW, KX> {
    using Base = GemmTile<E, PN, PM, WN, WM, NS, false, KW, KX>;
    static constexpr int kPitch = PN + 4;  // floats of a staged row: rows start in different banks
    static constexpr int kStage = Base::kTile * kPitch * 4;
    static constexpr int kStages = PARTS * Base::kWaves * (PARTS > 1 ? Base::TM : 1) * kStage;
    static constexpr int kAllLds = PARTS * Base::kLds > kStages ? PARTS * Base::kLds : kStages;
    static_assert(kAllLds <= 160 * 1024, "in LDS");
};

// ACT: a parameter, for the epilogue's size (with all of them in it the loop over the accumulators is not unrolled,
// and they lie in memory).
template <class E, int PN, int PM, int WN, int WM, int NS, bool KW, bool KX, int PARTS, int ACT>
__global__ __launch_bounds__(64 * WN * WM * PARTS) void linear_kernel(GemmArgs a, LinearOut o) {
    using Tile = LinearTile<E, PN, PM, WN, WM, NS, KW, KX, PARTS>;
    extern __shared__ __align__(16) uint8_t gemm_lds[];
    int tm, tn;
    if (o.partial == nullptr) {
        tile_of(a.tiles_m, a.tiles_n, tm, tn);
    } else {
        // slice after slice, a run of them to each chiplet: its L2 serves the tiles of a slice
        const int tiles = a.tiles_m * a.tiles_n, q = gridDim.x >> 3, rest = gridDim.x & 7;
        const int xcd = blockIdx.x & 7, i = xcd * q + (xcd < rest ? xcd : rest) + (blockIdx.x >> 3);
        const int slice = i / tiles, tile = i - slice * tiles;
        tm = tile / a.tiles_n;
        tn = tile - tm * a.tiles_n;
        int64_t unused = 0;
        cut_slice<E, KW, KX>(a, o, unused, slice);
    }
    const int64_t n0 = static_cast<int64_t>(tn) * Tile::BN, m0 = static_cast<int64_t>(tm) * Tile::BM;
    const int part = PARTS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / Tile::kWaves : 0;
    if constexpr (PARTS > 1) cut_part<E, KW, KX, PARTS>(a, part);
    Tile t;
    t.run(a, n0, m0, gemm_lds + part * Tile::kLds, part * Tile::kWaves);  // ends with a barrier behind its reads of LDS
    constexpr int kLanes = PN / 8, kAtOnce = 64 / kLanes, kTimes = Tile::kTile / kAtOnce;  // lanes of a row
    uint8_t* const mine = gemm_lds + (part * Tile::kWaves + t.wave) * (PARTS > 1 ? Tile::TM : 1) * Tile::kStage;
    const int l = t.lane % kLanes, r0 = t.lane / kLanes, in = t.lane & (Tile::kTile - 1);
    const int64_t n = n0 + t.wn * PN + 8 * l;
    const int left = a.N - n >= 8 ? 8 : (a.N > n ? static_cast<int>(a.N - n) : 0);
    // the gradients' products: sums alone
    [[maybe_unused]] float bias[8], r[kTimes][8];
    if constexpr (!KW) {
#pragma unroll
        for (int i = 0; i < 8; ++i) bias[i] = 0.f;
        if (o.bias != nullptr && left > 0) load8(o.bias + n, left, bias);
    }
    const auto residuals = [&](int64_t m1) {
        if constexpr (!KW) {
#pragma unroll
            for (int q = 0; q < kTimes; ++q) {
#pragma unroll
                for (int i = 0; i < 8; ++i) r[q][i] = 0.f;
                if (o.r != nullptr && left > 0 && m1 + q * kAtOnce < a.M) residual8(o, m1 + q * kAtOnce, n, left, r[q]);
            }
        }
    };
    const auto stage = [&](int j, uint8_t* to) {
#pragma unroll
        for (int i = 0; i < Tile::TN; ++i)
#pragma unroll
            for (int c = 0; c < Tile::kQuads; ++c) {
                const auto& s = t.acc[i][j];
                *reinterpret_cast<float4*>(to + 4 * (in * Tile::kPitch + t.column(i, c) - t.wn * PN)) =
                    make_float4(s[4 * c], s[4 * c + 1], s[4 * c + 2], s[4 * c + 3]);
            }
    };
    // rows m1 + q kAtOnce from their sums, `parts` of them kPart bytes apart
    constexpr int kPart = Tile::kWaves * Tile::TM * Tile::kStage;
    const auto finish = [&](int64_t m1, const uint8_t* at) {
#pragma unroll
        for (int q = 0; q < kTimes; ++q) {
            const float4* from = reinterpret_cast<const float4*>(at + 4 * ((r0 + q * kAtOnce) * Tile::kPitch + 8 * l));
            float4 lo = from[0], hi = from[1];
            float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int p = 1; p < PARTS; ++p) {
                lo = from[p * (kPart / 16)], hi = from[p * (kPart / 16) + 1];
                v[0] += lo.x, v[1] += lo.y, v[2] += lo.z, v[3] += lo.w;
                v[4] += hi.x, v[5] += hi.y, v[6] += hi.z, v[7] += hi.w;
            }
            const int64_t m = m1 + q * kAtOnce;
            if (left <= 0 || m >= a.M) continue;
            if constexpr (!KW) {
                finish8<ACT>(o, a.N, m, n, left, v, bias, r[q]);
            } else if (o.wide) {
                pass_store8(static_cast<float*>(o.y) + m * o.ldy + n, left, v, o.around);
            } else {
                pass_store8(static_cast<uint16_t*>(o.y) + m * o.ldy + n, left, v, o.around);
            }
        }
    };
    const int64_t first = m0 + t.wm * PM + r0;
    if constexpr (PARTS == 1) {
#pragma unroll
        for (int j = 0; j < Tile::TM; ++j) {
            residuals(first + j * Tile::kTile);
            stage(j, mine);
            wave_lds_order();
            finish(first + j * Tile::kTile, mine);
            wave_lds_order();
        }
    } else {
        residuals(first + part * Tile::kTile);  // of the rows below
#pragma unroll
        for (int j = 0; j < Tile::TM; ++j) stage(j, mine + j * Tile::kStage);
        __syncthreads();
        static_assert(Tile::TM <= PARTS);
        if (part < Tile::TM)
            finish(first + part * Tile::kTile, gemm_lds + (t.wave * Tile::TM + part) * Tile::kStage);
    }
}

// At most 16 TM rows of x.
template <class E, int TM>
__global__ __launch_bounds__(64 * kSkinnyWaves) void linear_skinny_kernel(GemmArgs a, int64_t row_bytes, LinearOut o) {
    if (o.partial != nullptr) cut_slice<E, false, false>(a, o, row_bytes, blockIdx.y);
    skinny_tile<E, TM, false>(a, row_bytes, static_cast<int64_t>(blockIdx.x) * 16,
                              [&](int64_t m, int64_t n, float s, float) {
                                  if (o.bias != nullptr) s += o.bias[n];
                                  if (o.z != nullptr) put(o.z + m * a.N + n, s);
                                  s = o.act == kSilu ? act<kSilu>(s) : (o.act == kGelu ? act<kGelu>(s) : s);
                                  if (o.r != nullptr)
                                      s += o.wide ? static_cast<const float*>(o.r)[m * o.ldr + n]
                                                  : bf16_to_f32(static_cast<const uint16_t*>(o.r)[m * o.ldr + n]);
                                  if (o.wide)
                                      put(static_cast<float*>(o.y) + m * o.ldy + n, s);
                                  else
                                      put(static_cast<uint16_t*>(o.y) + m * o.ldy + n, s);
                              });
}

// db: the workgroups' sums of a column added in a fixed order, 16 columns a workgroup of 256, 16 parts of the rows.
struct ColumnSums {
    const float* sums;  // [rows][N]
    int64_t rows, N;
    float* db;  // null: not wanted
    int64_t blocks() const { return db != nullptr ? (N + 15) / 16 : 0; }
};
__device__ __forceinline__ void add_columns(const ColumnSums& d, int64_t block) {
    __shared__ float part[16][17];
    const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t n = block * 16 + c;
    float s = 0.f;
    if (n < d.N) {
#pragma unroll 16
        for (int64_t r = g; r < d.rows; r += 16) s += d.sums[r * d.N + n];
    }
    part[g][c] = s;
    __syncthreads();
    if (threadIdx.x < 16 && n < d.N) {
        float total = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) total += part[k][c];
        d.db[n] = total;
    }
}
__global__ __launch_bounds__(256) void linear_db_kernel(ColumnSums d) { add_columns(d, blockIdx.x); }

// The slices' sums added in a fixed order, and what follows them: eight neighbouring outputs to PARTS threads, each of
// which adds every PARTS-th slice (few outputs of many slices would keep few threads busy).  The workgroups from `blocks` on
// make db, which saves its launch: all gradients of 100,000 x 128 by 32 40 -> 36 us.
template <int PARTS>
__global__ __launch_bounds__(256) void linear_join_kernel(LinearOut o, int slices, int64_t M, int64_t N, unsigned blocks,
                                                          ColumnSums d) {
    if (blockIdx.x >= blocks) {
        add_columns(d, blockIdx.x - blocks);
        return;
    }
    constexpr int kOutputs = 256 / PARTS;
    __shared__ float part[PARTS > 1 ? PARTS : 1][PARTS > 1 ? kOutputs : 1][9];
    const int i0 = threadIdx.x % kOutputs, part_of = threadIdx.x / kOutputs;
    const int64_t groups = (N + 7) / 8, stride = static_cast<int64_t>(blocks) * kOutputs;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kOutputs; first < M * groups; first += stride) {
        const int64_t at = first + i0, m = at / groups, n = (at - m * groups) * 8;
        const bool mine = at < M * groups;
        const int left = !mine ? 0 : (N - n >= 8 ? 8 : static_cast<int>(N - n));
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
        const float* from = o.partial + (mine ? m * N + n : 0);
#pragma unroll 4
        for (int s = part_of; s < slices; s += PARTS) {
            float p[8];
            load8(from + s * M * N, left, p);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += p[i];
        }
        if constexpr (PARTS > 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) part[part_of][i0][i] = v[i];
            __syncthreads();
            if (part_of == 0) {
#pragma unroll
                for (int q = 1; q < PARTS; ++q)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] += part[q][i0][i];
            }
            __syncthreads();
            if (part_of != 0) continue;
        }
        if (!mine) continue;
        float bias[8], r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) bias[i] = r[i] = 0.f;
        if (o.bias != nullptr) load8(o.bias + n, left, bias);
        if (o.r != nullptr) residual8(o, m, n, left, r);
        if (o.act == kSilu)
            finish8<kSilu>(o, N, m, n, left, v, bias, r);
        else if (o.act == kGelu)
            finish8<kGelu>(o, N, m, n, left, v, bias, r);
        else
            finish8<kIdentity>(o, N, m, n, left, v, bias, r);
    }
}

// Rows of K bf16 elements to rows of a multiple of 64, zeros behind: what the products read where the caller's rows do
// not start and end on 16 bytes.  x and w in one launch, eight elements a thread (at any address), `lanes` (a power of two)
// threads to a row, four rows in flight.
struct RowCopy {
    const uint16_t* from;
    int64_t ld, R;
    uint16_t* to;
};
__global__ __launch_bounds__(256) void copy_rows_kernel(RowCopy a, RowCopy b, int64_t K, int64_t pitch, int lanes) {
    constexpr int kRows = 4;
    const int64_t c = (static_cast<int64_t>(blockIdx.y) * lanes + (threadIdx.x & (lanes - 1))) * 8, left = K - c;
    if (c >= pitch) return;
    const int at_once = 256 / lanes;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * at_once * kRows + threadIdx.x / lanes; first < a.R + b.R;
         first += static_cast<int64_t>(gridDim.x) * at_once * kRows) {
        u4u v[kRows];
        uint16_t* to[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t row = first + i * at_once, r = row < a.R ? row : row - a.R;
            const uint16_t* from = (row < a.R ? a.from + r * a.ld : b.from + r * b.ld) + c;
            to[i] = (row < a.R ? a.to : b.to) + r * pitch + c;
            v[i] = u4u{0, 0, 0, 0};
            if (row >= a.R + b.R) continue;
            if (left >= 8) {
                v[i] = *reinterpret_cast<const u4u*>(from);
            } else {
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < left) w[j / 2] |= static_cast<uint32_t>(from[j]) << (16 * (j & 1));
                v[i] = u4u{w[0], w[1], w[2], w[3]};
            }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (first + i * at_once < a.R + b.R) *reinterpret_cast<u4u*>(to[i]) = v[i];
    }
}

// dz [M] rows of `pitch` bf16 elements (zeros behind column N; null: not wanted) and, for each workgroup's rows, the
// sums of its columns before they are rounded (sums [gridDim.y][N]; null: not wanted).  LANES lanes of eight
// columns to a row; a lane keeps its columns.
template <int LANES, typename TD>
__global__ __launch_bounds__(256) void linear_dz_kernel(int kind, const TD* __restrict__ dy, int64_t lddy,
                                                        const uint16_t* __restrict__ z, uint16_t* __restrict__ dz, bool past,
                                                        int64_t pitch, float* __restrict__ sums, int64_t M, int64_t N,
                                                        int64_t rows) {
    constexpr int kAtOnce = 256 / LANES;
    __shared__ float part[kAtOnce][LANES * 8 + 4];
    const int l = threadIdx.x % LANES, g = threadIdx.x / LANES;
    const int64_t n = (static_cast<int64_t>(blockIdx.x) * LANES + l) * 8, left = N - n;
    const int have = left >= 8 ? 8 : (left > 0 ? static_cast<int>(left) : 0);
    const int64_t m1 = static_cast<int64_t>(blockIdx.y) * rows, m2 = m1 + rows < M ? m1 + rows : M;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    if (n < (dz != nullptr ? pitch : N)) {
#pragma unroll 2
        for (int64_t m = m1 + g; m < m2; m += kAtOnce) {
            float v[8];
            if (past)  // large, and lines that no two rows share
                pass8(dy + m * lddy + (have > 0 ? n : 0), have, v);
            else
                load8(dy + m * lddy + (have > 0 ? n : 0), have, v);
            if (kind != kIdentity) {
                float p[8];
                if (past)
                    pass8(z + m * N + (have > 0 ? n : 0), have, p);
                else
                    load8(z + m * N + (have > 0 ? n : 0), have, p);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = kind == kSilu ? slope<kSilu>(p[i]) : slope<kGelu>(p[i]);
                    v[i] = i < have ? v[i] * d : 0.f;
                }
            }
            if (dz != nullptr) store8(dz + m * pitch + n, 8, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        }
    }
    if (sums == nullptr) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[g][8 * l + i] = sum[i];
    __syncthreads();
    for (int c = threadIdx.x; c < 8 * LANES; c += 256) {
        const int64_t column = static_cast<int64_t>(blockIdx.x) * LANES * 8 + c;
        if (column >= N) break;
        float s = 0.f;
#pragma unroll 8
        for (int k = 0; k < kAtOnce; ++k) s += part[k][c];
        sums[static_cast<int64_t>(blockIdx.y) * N + column] = s;
    }
}

// dz, its columns' sums and dx in one launch, for up to 128 columns of w: a workgroup keeps all of them for its rows, so
// dz goes to the product through LDS and is read from memory by dw's alone.
//
// A step is 64 columns of dz by up to 128 rows: a thread makes eight columns of two of them, lays them in LDS beside the
// step's 64 rows of w as a GemmTile with w's columns along the sum has them, and loads the next step's into the
// registers that are free again; eight waves of 32 rows by 64 columns of dx multiply behind the barrier.  Two places for
// either, so one barrier a step.  A column's sum over the wave's 16 rows is made by halving (lane bits 5, 4, 3), over
// the waves by one of them behind the barrier, over the workgroup's rows in `column_sums`.
//
// Memory's rate where every workgroup's rows fill their tiles (dx alone of 65,536 x 512 by 128: 151 MB in 30 us, 5.0 TB/s),
// else a step's arithmetic, which rows that do not exist take part in; 100,000 rows with dz stored 66 us, 5.0 TB/s.  Both
// ways, dz by itself and this one, silu, all gradients (dx alone), us:
//   100,000 x 512 by 128 118 / 100 (81 / 51), 100,000 x 128 by 32 48 / 36, 100,000 x 2,048 by 128 470 / 395, 50,000 x 512 by
//   128 70 / 59 (44 / 26), 50,000 x 256 by 64 40 / 35; 32,768 rows 51 / 51, 31 / 34, 16,384 rows 34 / 46: steps follow one
//   another, some 3 us each.  Hence from 40,000 rows on.  (Without dx: linear_narrow_dz_kernel.)
constexpr int kNarrowRows = 128, kNarrowInputs = 128, kNarrowOutputs = 2048, kNarrowBlocks = 512;
constexpr int64_t kNarrowLeast = 40'000;
constexpr int kNarrowDz = kNarrowRows * kStepBytes, kNarrowW = 64 * 2 * kNarrowInputs, kNarrowPart = 8 * 64 * 4;
constexpr int kNarrowLds = 2 * (kNarrowDz + kNarrowW + kNarrowPart);  // and 4 bytes a column of dz
typedef uint32_t v4w __attribute__((ext_vector_type(4)));
constexpr uint32_t kNowhere = 0x80000000u;  // past every buffer: loads give zeros, stores go nowhere
constexpr int kPast = 2;                    // non-temporal, of a buffer's loads and stores

// 16 bytes to `offset` of a buffer.  The offset goes by the lane's register alone: behind a store of more than 8 bytes the
// first of its data registers may not be written by the next instruction, and the compiler leaves room for that only where
// the store has no scalar offset (seen: lanes with zeros for their first two elements).
__device__ __forceinline__ void store16(v4w v, const uint16_t* base, uint32_t offset) {
    __builtin_amdgcn_raw_buffer_store_b128(v, buffer_of(reinterpret_cast<const uint8_t*>(base), 0x7fffffffu), offset, 0, 0);
}

// Lanes with the bit clear get the pair's sum of a, the others that of b.
__device__ __forceinline__ float halve32(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halve16(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halve8(float a, float b, bool high) {
    const float keep = high ? b : a, send = high ? a : b;
    return keep + __shfl_xor(send, 8);
}

// Eight elements of dz from what was loaded of dy and z.
__device__ __forceinline__ void widen(const v4w& x, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(x[i] << 16);
        v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
    }
}
template <int ACT, int WIDTH>
__device__ __forceinline__ void dz_of(const v4w (&dy)[WIDTH], const v4w& z, float (&v)[8]) {
    if constexpr (WIDTH == 1) {
        widen(dy[0], v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(dy[e / 4][e % 4]);
    }
    if constexpr (ACT != kIdentity) {
        float p[8];
        widen(z, p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= slope<ACT>(p[e]);
    }
}
// (no product is contracted into the sum: both kernels below round alike)
__device__ __forceinline__ void add_rows(float (&sum)[8], const float (&v)[8], bool first) {
#pragma clang fp contract(off)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = first ? v[e] : sum[e] + v[e];
}
// A thread's sums of eight columns to `part` [64] as sums over the wave's rows (lane bits 5, 4, 3); lane bits 2 to 0 are the
// chunk of columns.
__device__ __forceinline__ void leave_column_sums(const float (&sum)[8], float* part, int lane) {
    float four[4], two[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) four[e] = halve32(sum[e], sum[4 + e]);
#pragma unroll
    for (int e = 0; e < 2; ++e) two[e] = halve16(four[e], four[2 + e]);
    part[8 * (lane & 7) + 4 * (lane >> 5) + 2 * ((lane >> 4) & 1) + ((lane >> 3) & 1)] =
        halve8(two[0], two[1], (lane & 8) != 0);
}
// the waves' sums of a column, added in order
__device__ __forceinline__ float add_waves(const float* part, int pitch) {
    float total = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) total += part[k * pitch];
    return total;
}

// Waits until the wave's LDS writes and reads are done, then for all waves; loads and stores of memory go on.
__device__ __forceinline__ void written_and_read() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// WHOLE: dx's rows start and end on 16 bytes (a parameter, for the registers that the other way takes).
template <typename TD, int ACT, bool WHOLE>
__global__ __launch_bounds__(512, 4) void linear_narrow_kernel(const TD* __restrict__ dy, int64_t lddy,
                                                            const uint16_t* __restrict__ z, const uint16_t* __restrict__ w,
                                                            int64_t ldw, uint16_t* __restrict__ dz, int64_t pitch,
                                                            float* __restrict__ sums, uint16_t* __restrict__ dx, int64_t lddx,
                                                            int64_t M, int64_t N, int64_t K, int64_t rows, bool past) {
    using Tile = GemmTile<Bf16, 64, 32, 2, 4, 2, false, true, false>;  // the places of w and its reads
    constexpr int kWidth = sizeof(TD) / 2;                              // loads of eight elements of dy
    extern __shared__ __align__(16) uint8_t narrow_lds[];
    uint8_t* const at_dz = narrow_lds;
    uint8_t* const at_w = at_dz + 2 * kNarrowDz;
    float* const parts = reinterpret_cast<float*>(at_w + 2 * kNarrowW);
    float* const column_sums = parts + 2 * (kNarrowPart / 4);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wn = wave & 1, wm = wave >> 1;
    const int64_t m1 = static_cast<int64_t>(blockIdx.x) * rows, m2 = m1 + rows < M ? m1 + rows : M;
    const int steps = static_cast<int>(pitch / 64);
    for (int s = wave; s < steps; s += 8) column_sums[64 * s + lane] = 0.f;  // by the wave that adds to them

    // the thread's part of a step: rows r and r + 64 of dz, 16-byte chunk c of them; rows of w, chunks of 8 columns
    const int r = tid >> 3, c = tid & 7, wr = tid >> 4, wc = tid & 15;
    v4w at_dy[2][kWidth], at_z[2], at_wr[2];
    const uint32_t dy_row = static_cast<uint32_t>(lddy * sizeof(TD)), z_row = static_cast<uint32_t>(2 * N),
                   w_row = static_cast<uint32_t>(2 * ldw), dz_row = static_cast<uint32_t>(2 * pitch);
    const int columns = static_cast<int>(N), inputs = static_cast<int>(K);
    // half i of step s of the rows from m0 on
    const auto fetch = [&](int64_t m0, int s, int i) {
        const int64_t have = m2 - m0;
        const int count = have < kNarrowRows ? static_cast<int>(have < 0 ? 0 : have) : kNarrowRows;
        const int64_t from = count > 0 ? m0 + 64 * i : 0;
        const Buffer bd = buffer_of(reinterpret_cast<const uint8_t*>(dy + from * lddy), 0x7fffffffu);
        const Buffer bz = buffer_of(reinterpret_cast<const uint8_t*>(z + from * N), 0x7fffffffu);
        const Buffer bw = buffer_of(reinterpret_cast<const uint8_t*>(w + (64 * s + 32 * i) * ldw), 0x7fffffffu);
        const bool in = r < count - 64 * i && 8 * c < columns - 64 * s;
        const uint32_t od = in ? r * dy_row + 8 * sizeof(TD) * c : kNowhere, oz = in ? r * z_row + 16 * c : kNowhere;
        const uint32_t ow = wr < columns - 64 * s - 32 * i && 8 * wc < inputs ? wr * w_row + 16 * wc : kNowhere;
#pragma unroll
        for (int h = 0; h < kWidth; ++h)
            at_dy[i][h] = __builtin_amdgcn_raw_buffer_load_b128(bd, od, 64 * sizeof(TD) * s + 16 * h, kPast);
        if constexpr (ACT != kIdentity) at_z[i] = __builtin_amdgcn_raw_buffer_load_b128(bz, oz, 128 * s, kPast);
        at_wr[i] = __builtin_amdgcn_raw_buffer_load_b128(bw, ow, 0, 0);
    };
    // places of the wave's fragments, as in GemmTile
    const int in = lane & 15, key = (in >> 1) & 7;
    const int wrow = 8 * (lane >> 4) + (in >> 2), wchunk = 8 * wn + ((lane & 3) >> 1);
    const int tw = wrow * 256 + ((wchunk ^ Tile::turn(16, wrow)) << 4) + ((lane & 1) << 3);
    fetch(m1, 0, 0);
    fetch(m1, 0, 1);
    int turn = 0;  // the places of this step
    for (int64_t m0 = m1; m0 < m2; m0 += kNarrowRows) {
        const int count = m2 - m0 < kNarrowRows ? static_cast<int>(m2 - m0) : kNarrowRows;
        v4f acc[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < steps; ++s) {
            const bool last = s + 1 == steps;
            uint8_t* const here_dz = at_dz + turn * kNarrowDz;
            uint8_t* const here_w = at_w + turn * kNarrowW;
            float* const here_part = parts + turn * (kNarrowPart / 4);
            float sum[8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = r + 64 * i, k = wr + 32 * i;
                float v[8];
                dz_of<ACT>(at_dy[i], at_z[i], v);
                const v4w q{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
                *reinterpret_cast<v4w*>(here_dz + row * 128 + ((c ^ ((row >> 1) & 7)) << 4)) = q;
                *reinterpret_cast<v4w*>(here_w + k * 256 + ((wc ^ Tile::turn(16, k)) << 4)) = at_wr[i];
                if (dz != nullptr)
                    store16(q, dz + (m0 + 64 * i) * pitch + 64 * s, row < count ? r * dz_row + 16 * c : kNowhere);
                add_rows(sum, v, i == 0);
                fetch(last ? m0 + kNarrowRows : m0, last ? 0 : s + 1, i);  // into the registers that are free again
                __builtin_amdgcn_sched_barrier(0);
            }
            if (sums != nullptr) leave_column_sums(sum, here_part + wave * 64, lane);
            written_and_read();
            if (sums != nullptr && wave == (s & 7)) column_sums[64 * s + lane] += add_waves(here_part + lane, 64);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                v4i fx[2], fw[4];
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    fx[j] = *reinterpret_cast<const v4i*>(here_dz + (32 * wm + 16 * j + in) * 128 +
                                                          (((4 * q + (lane >> 4)) ^ key) << 4));
#pragma unroll
                for (int i = 0; i < 4; ++i) fw[i] = Tile::turned(here_w + (tw ^ i << 5) + q * 8192, 1024);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = Bf16::product(__builtin_bit_cast(v8bf, fw[i]), __builtin_bit_cast(v8bf, fx[j]), acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
            turn ^= 1;
        }
        // dx by LDS, in dz's places, so that it leaves in whole lines: 16 chunks a row, turned by the row
        written_and_read();
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = 32 * wm + 16 * j + in, chunk = 8 * wn + 2 * i + (lane >> 5);
                *reinterpret_cast<uint2*>(at_dz + row * 256 + ((chunk ^ in) << 4) + ((lane >> 4) & 1) * 8) =
                    make_uint2(bf16_pair(acc[i][j][0], acc[i][j][1]), bf16_pair(acc[i][j][2], acc[i][j][3]));
            }
        written_and_read();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = wr + 32 * i;
            if (row >= count || 8 * wc >= K) continue;
            const uint8_t* const staged = at_dz + row * 256 + ((wc ^ (row & 15)) << 4);
            uint16_t* const out = dx + (m0 + row) * lddx + 8 * wc;
            if constexpr (WHOLE) {
                const v4w v = *reinterpret_cast<const v4w*>(staged);
                if (past)
                    __builtin_nontemporal_store(v, reinterpret_cast<v4w*>(out));
                else
                    *reinterpret_cast<v4w*>(out) = v;
            } else {
#pragma unroll 1
                for (int e = 0; e < 8 && 8 * wc + e < inputs; ++e) out[e] = reinterpret_cast<const uint16_t*>(staged)[e];
            }
        }
        written_and_read();
    }
    if (sums != nullptr)
        for (int s = wave; s < steps; s += 8)
            if (64 * s + lane < N) sums[static_cast<int64_t>(blockIdx.x) * N + 64 * s + lane] = column_sums[64 * s + lane];
}

// dz and its columns' sums without dx, with the bits that the kernel above gives them: the same rows to a workgroup and to a
// wave, the same sums in the same order.  LANES lanes of eight columns to a row (1 KB of 512 columns), so that most of
// the halving is a lane's own: rows 4, 2 and 1 apart, as lane bits 5, 4 and 3 are there.  Columns of a workgroup: 8 LANES;
// the waves meet once in 128 rows.  Memory's rate: db alone of 200,000 x 2,048 270 us (6.1 TB/s).
//
// dw and db, silu, us: the kernel above without its product / linear_dz_kernel, whose sums go in another order / this one
//   100,000 x 2,048 by 128 372 / 349 / 340, 200,000 788 / 699 / 680, 50,000 168 / 158 / 147; 100,000 x 512 by 128 88 / 92 / 89,
//   65,536 61 / 67 / 64, 200,000 182 / 178 / 178; 100,000 x 128 by 32 32 / 39 / 32.
template <int LANES, typename TD, int ACT>
__global__ __launch_bounds__(512, 4) void linear_narrow_dz_kernel(const TD* __restrict__ dy, int64_t lddy,
                                                               const uint16_t* __restrict__ z, uint16_t* __restrict__ dz,
                                                               int64_t pitch, float* __restrict__ sums, int64_t M, int64_t N,
                                                               int64_t rows, unsigned across, unsigned blocks, bool columns_first) {
    constexpr int kWidth = sizeof(TD) / 2, kColumns = 8 * LANES;
    constexpr int kGroups = 64 / LANES, kOwn = 8 / kGroups;  // rows of a wave at a time; of a lane, of the wave's eight
    __shared__ float parts[2][8][kColumns];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned bn = columns_first ? blockIdx.x % across : blockIdx.x / blocks;
    const unsigned bm = columns_first ? blockIdx.x / across : blockIdx.x % blocks;
    const int64_t m1 = static_cast<int64_t>(bm) * rows, m2 = m1 + rows < M ? m1 + rows : M;
    const int64_t n = static_cast<int64_t>(bn) * kColumns + 8 * (lane % LANES);
    const uint32_t dy_row = static_cast<uint32_t>(lddy * sizeof(TD)), z_row = static_cast<uint32_t>(2 * N),
                   dz_row = static_cast<uint32_t>(2 * pitch);
    // of the lane: its row among those of a time, and its places (past the buffers where it has no column)
    const int lane_row = lane / LANES;
    const uint32_t at_od = n < N ? lane_row * dy_row + static_cast<uint32_t>(sizeof(TD) * n) : kNowhere,
                   at_oz = n < N ? lane_row * z_row + static_cast<uint32_t>(2 * n) : kNowhere,
                   at_out = n < pitch ? lane_row * dz_row + static_cast<uint32_t>(2 * n) : kNowhere;
    // row e of time t: rows 64 apart; the times 4, 2 and 1 apart
    const auto row_of = [&](int t, int e) {
        const int first = kOwn == 8 ? (t & 1) * 4 + (t & 2) + (t >> 2) : (kOwn == 4 ? (t & 1) * 4 + (t & 2) : 4 * t);
        return 8 * wave + first + 64 * e;
    };
    v4w at_dy[2][kWidth], at_z[2];
    const auto fetch = [&](int64_t m0, int t, int e) {
        const int64_t have = m2 - m0, from = have > 0 ? m0 : 0;
        const int row = row_of(t, e);
        const Buffer bd = buffer_of(reinterpret_cast<const uint8_t*>(dy + from * lddy), 0x7fffffffu);
        const Buffer bz = buffer_of(reinterpret_cast<const uint8_t*>(z + from * N), 0x7fffffffu);
        const bool in = row + lane_row < have;
        const uint32_t od = in ? at_od : kNowhere, oz = in ? at_oz : kNowhere;
#pragma unroll
        for (int h = 0; h < kWidth; ++h)
            at_dy[e][h] = __builtin_amdgcn_raw_buffer_load_b128(bd, od, row * dy_row + 16 * h, kPast);
        if constexpr (ACT != kIdentity) at_z[e] = __builtin_amdgcn_raw_buffer_load_b128(bz, oz, row * z_row, kPast);
    };
#pragma unroll
    for (int e = 0; e < 2; ++e) fetch(m1, 0, e);
    float total = 0.f;  // of the thread's column
    int turn = 0;
    for (int64_t m0 = m1; m0 < m2; m0 += kNarrowRows) {
        float sum[8], half[8], pair[8], one[8];
        // (not unrolled: the additions would move behind all loads, whose registers do not suffice)
#pragma unroll 1
        for (int t = 0; t < kOwn; ++t) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float v[8];
                dz_of<ACT>(at_dy[e], at_z[e], v);
                const bool last = t + 1 == kOwn;
                fetch(last ? m0 + kNarrowRows : m0, last ? 0 : t + 1, e);  // into the registers that are free again
                const int row = row_of(t, e);
                if (dz != nullptr)
                    store16(v4w{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])},
                            dz + (m0 + row) * pitch, row + lane_row < m2 - m0 ? at_out : kNowhere);
                add_rows(one, v, e == 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            add_rows(pair, one, (t & 1) == 0);
            if (kOwn == 1 || (t & 1) == 1) add_rows(half, pair, (t & 2) == 0);
            if (kOwn < 4 || (t & 3) == 3) add_rows(sum, half, (t & 4) == 0);
        }
#pragma unroll
        for (int d = 32; d >= LANES; d >>= 1) {
            if (d > 4 * LANES) continue;
            float other[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) other[i] = __shfl_xor(sum[i], d);
            add_rows(sum, other, false);
        }
        if (lane < LANES) {
            float4* const to = reinterpret_cast<float4*>(&parts[turn][wave][8 * lane]);
            to[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            to[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
        }
        written_and_read();
        if (tid < kColumns) total += add_waves(&parts[turn][0][tid], kColumns);
        turn ^= 1;
    }
    const int64_t at = static_cast<int64_t>(bn) * kColumns + tid;
    if (sums != nullptr && tid < kColumns && at < N) sums[static_cast<int64_t>(bm) * N + at] = total;
}

template <typename T>
__global__ __launch_bounds__(256) void linear_zero_kernel(T* p, int64_t n) {
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += stride) p[i] = 0;
}

// of 256 threads, for kernels that walk what is left
dim3 walking(int64_t threads) {
    const int64_t blocks = (threads + 255) / 256;
    return dim3(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks));
}
int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
// whether the products can read these rows as they are
bool rows_fit(const void* p, int64_t K, int64_t ld) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && K % 8 == 0 && ld % 8 == 0 && 2 * ld <= kMostRowBytes;
}
hipError_t copy_rows(const RowCopy& a, const RowCopy& b, int64_t K, hipStream_t stream) {
    const int64_t pitch = up(K, 64), rows = a.R + b.R, groups = pitch / 8;
    int lanes = 8;
    while (lanes < 64 && lanes < groups) lanes *= 2;
    const int64_t across = (groups + lanes - 1) / lanes, most = kMostBlocks / across;
    const int64_t at_once = 4 * (256 / lanes), down = (rows + at_once - 1) / at_once;
    hipLaunchKernelGGL(copy_rows_kernel,
                       dim3(static_cast<unsigned>(down < most ? down : most), static_cast<unsigned>(across)), dim3(256), 0,
                       stream, a, b, K, pitch, lanes);
    return hipGetLastError();
}

// What a product of [M][N] outputs over `steps` steps takes: the tile (0: the few-rows kernel) and the slices of its sum.
struct Shape : SumShape {
    size_t bytes(int64_t M, int64_t N) const { return slices > 1 ? static_cast<size_t>(slices * M * N) * sizeof(float) : 0; }
};
Shape shape_of(const SliceCosts& costs, int64_t M, int64_t N, int64_t steps, int64_t grain) {
    return Shape{sum_shape(costs, M, N, steps, grain)};
}
// Up to 16 rows of x the weights' bytes are all that counts, and the few-rows kernel reads them with the least
// latency: us against the best tile (sum x columns), one row bf16 4,096 x 8,192 12.7 / 14.7, 1,024^2 4.1 / 5.9; 24 rows
// 23 / 16 and 6.7 / 6.2.  8 bits, 17 rows 8,192 x 2,048 13.5 / 11.5, 4,096^2 8.1 / 9.5, 2,048 x 8,192 7.3 / 8.2, 8,192^2
// 26 / 18; 24 rows 15.6 / 11.5, 9.1 / 9.6, 8.1 / 8.1, 30 / 18; 32 rows 17.7 / 11.6, 10.2 / 9.9, 9.0 / 8.1, 34 / 18; 64 rows
// 28 / 12, 16 / 12, 10 / 8, 55 / 19: sums of up to 4,096 could go on to 24 rows for 1 us.  Its eight waves have four steps
// each in flight: a longer sum over few columns is cut, one row of 8,192 x 128 10.6 -> 6.7.
constexpr int64_t kFewRows = 16;
Shape few_shape(int64_t N, int64_t steps, int64_t grain) {
    const int64_t groups = (N + 15) / 16, at_once = 4 * kSkinnyWaves;
    int64_t slices = 256 / groups;
    if (slices > steps / at_once) slices = steps / at_once;
    if (slices < 2) return Shape{{0, 1, 1, steps}};
    const int64_t per = up((steps + slices - 1) / slices, grain);
    return Shape{{0, 1, (steps + per - 1) / per, per}};
}

template <class E, int PN, int PM, int WN, int WM, int NS, bool KW, bool KX, int PARTS, int ACT>
hipError_t launch_tile(GemmArgs g, const LinearOut& o, int64_t slices, hipStream_t stream) {
    using Tile = LinearTile<E, PN, PM, WN, WM, NS, KW, KX, PARTS>;
    const int64_t tm = (g.M + Tile::BM - 1) / Tile::BM, tn = (g.N + Tile::BN - 1) / Tile::BN;
    if (tm * tn > kMostTiles) return hipErrorInvalidValue;
    g.tiles_m = static_cast<int>(tm);
    g.tiles_n = static_cast<int>(tn);
    constexpr auto kernel = linear_kernel<E, PN, PM, WN, WM, NS, KW, KX, PARTS, ACT>;
    const hipError_t e = raise_lds_limit<kernel>();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(tm * tn * slices)), dim3(Tile::kThreads * PARTS), Tile::kAllLds,
                       stream, g, o);
    return hipGetLastError();
}

template <class E, bool KW, bool KX, int ACT>
hipError_t launch_tiles(const Shape& s, const GemmArgs& g, const LinearOut& o, hipStream_t stream) {
    // 128: 8 bits in four waves, for registers
    constexpr int PM = E::kScaled ? 64 : 32, WM = E::kScaled ? 2 : 4;
    switch (s.tile) {
        case 256: return launch_tile<E, 128, 64, 2, 4, 2, KW, KX, 1, ACT>(g, o, s.slices, stream);
        case 128:
            if (s.parts == 2) return launch_tile<E, 64, PM, 2, WM, 2, KW, KX, 2, ACT>(g, o, s.slices, stream);
            return launch_tile<E, 64, PM, 2, WM, 2, KW, KX, 1, ACT>(g, o, s.slices, stream);
        default:
            if (s.parts == 2) return launch_tile<E, 32, 32, 2, 2, 4, KW, KX, 2, ACT>(g, o, s.slices, stream);
            return launch_tile<E, 32, 32, 2, 2, 4, KW, KX, 1, ACT>(g, o, s.slices, stream);
    }
}

template <class E>
hipError_t launch_few(const GemmArgs& g, int64_t row_bytes, const LinearOut& o, int64_t slices, hipStream_t stream) {
    const int64_t blocks = (g.N + 15) / 16;
    if (blocks > kMostTiles) return hipErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(slices)), threads(64 * kSkinnyWaves);
    hipLaunchKernelGGL((linear_skinny_kernel<E, 1>), grid, threads, 0, stream, g, row_bytes, o);
    return hipGetLastError();
}

template <int PARTS>
void join(const Shape& s, const GemmArgs& g, const LinearOut& o, const ColumnSums& d, hipStream_t stream) {
    const unsigned blocks = walking(g.M * ((g.N + 7) / 8) * PARTS).x;
    hipLaunchKernelGGL(linear_join_kernel<PARTS>, dim3(blocks + static_cast<unsigned>(d.blocks())), dim3(256), 0, stream, o,
                       static_cast<int>(s.slices), g.M, g.N, blocks, d);
}

// The product, its slices in `partial`, and what follows; where there are slices, db in the launch that joins them.
template <class E, bool KW, bool KX>
hipError_t product(const Shape& s, GemmArgs g, int64_t row_bytes, LinearOut o, float* partial, hipStream_t stream,
                   const ColumnSums& d = ColumnSums{}) {
    o.partial = s.slices > 1 ? partial : nullptr;
    o.slice = static_cast<int>(s.per);
    hipError_t e;
    if (s.tile > 0) {
        // slices leave as sums
        const int act = KW || s.slices > 1 ? static_cast<int>(kIdentity) : o.act;
        if constexpr (!KW) {
            if (act == kSilu) return launch_tiles<E, KW, KX, kSilu>(s, g, o, stream);
            if (act == kGelu) return launch_tiles<E, KW, KX, kGelu>(s, g, o, stream);
        }
        e = launch_tiles<E, KW, KX, kIdentity>(s, g, o, stream);
    } else {
        if constexpr (KW)
            e = hipErrorInvalidValue;
        else
            e = launch_few<E>(g, row_bytes, o, s.slices, stream);
    }
    if (e != hipSuccess || s.slices == 1) return e;
    const int64_t outputs = g.M * ((g.N + 7) / 8);
    if (outputs < 32768 && s.slices >= 8)
        join<8>(s, g, o, d, stream);
    else
        join<1>(s, g, o, d, stream);
    return hipGetLastError();
}

Shape forward_shape(int64_t M, int64_t K, int64_t N) {
    const int64_t steps = (K + 63) / 64;
    return M <= kFewRows ? few_shape(N, steps, 1) : shape_of(kSlices16, M, N, steps, 1);
}
Shape forward8_shape(int64_t M, int64_t K, int64_t N) {
    const int64_t steps = (K + 127) / 128;
    return M <= kFewRows ? few_shape(N, steps, 4) : shape_of(kSlices8, M, N, steps, 4);
}
// of dx, and of dw
Shape dx_shape(int64_t M, int64_t K, int64_t N) { return shape_of(kSlices16, M, K, (N + 63) / 64, 1); }
Shape dw_shape(int64_t M, int64_t K, int64_t N) { return shape_of(kSlices16, N, K, (M + 63) / 64, 1); }

// Outputs of more elements than this leave past the caches: 100,000 x 512 of 128 terms with silu, z kept, 66 -> 49 us
// (without either 34 -> 32), 8,192 x 8,192 of 2,048 with gelu 262 -> 243, z kept too 279 -> 253.  Smaller ones stay for
// who reads them next.
bool large(int64_t elements) { return elements > int64_t{1} << 24; }

LinearOut out_of(const LinearArgs& a) {
    return LinearOut{a.act,
                     a.dtype == SPINGTP_FP32,
                     a.bias,
                     a.r,
                     a.ldr,
                     a.y,
                     a.ldy,
                     static_cast<uint16_t*>(a.z),
                     large(a.M * a.N),
                     nullptr,
                     0};
}

// lanes of a row of dz, and how many rows a workgroup takes
int dz_lanes(int64_t N) { return N > 256 ? 64 : (N > 64 ? 32 : 8); }
int64_t dz_rows(int64_t M, int64_t N) {
    const int lanes = dz_lanes(N), at_once = 256 / lanes;
    const int64_t across = (up(N, 64) / 8 + lanes - 1) / lanes;
    int64_t blocks = 2048 / across;
    if (blocks < 1) blocks = 1;
    const int64_t rows = up((M + blocks - 1) / blocks, 4 * at_once);
    return rows < int64_t{1} << 31 ? rows : int64_t{1} << 31;
}
int64_t dz_blocks(int64_t M, int64_t N) {
    const int64_t rows = dz_rows(M, N);
    return (M + rows - 1) / rows;
}
bool own_dz(const LinearBwdArgs& a) {
    return a.act == kIdentity && a.dtype == SPINGTP_BF16 && rows_fit(a.dy, a.N, a.lddy);
}

template <int LANES, typename TD>
hipError_t launch_dz(const LinearBwdArgs& a, uint16_t* dz, float* sums, hipStream_t stream) {
    const int64_t pitch = up(a.N, 64), across = (pitch / 8 + LANES - 1) / LANES;
    hipLaunchKernelGGL((linear_dz_kernel<LANES, TD>),
                       dim3(static_cast<unsigned>(across), static_cast<unsigned>(dz_blocks(a.M, a.N))), dim3(256), 0, stream,
                       a.act, static_cast<const TD*>(a.dy), a.lddy, static_cast<const uint16_t*>(a.z), dz,
                       large(a.M * a.N) && a.N % 8 == 0, pitch, sums, a.M,
                       a.N, dz_rows(a.M, a.N));
    return hipGetLastError();
}
template <typename TD>
hipError_t make_dz(const LinearBwdArgs& a, uint16_t* dz, float* sums, hipStream_t stream) {
    switch (dz_lanes(a.N)) {
        case 64: return launch_dz<64, TD>(a, dz, sums, stream);
        case 32: return launch_dz<32, TD>(a, dz, sums, stream);
        default: return launch_dz<8, TD>(a, dz, sums, stream);
    }
}
template <typename T>
hipError_t zero(void* p, int64_t n, hipStream_t stream) {
    hipLaunchKernelGGL(linear_zero_kernel<T>, walking(n), dim3(256), 0, stream, static_cast<T*>(p), n);
    return hipGetLastError();
}
size_t larger(size_t a, size_t b) { return a > b ? a : b; }
size_t up16(size_t n) { return (n + 15) / 16 * 16; }

}  // namespace

size_t linear_workspace(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t M, int64_t K, int64_t N) {
    const Shape s = forward_shape(M, K, N);
    const size_t row = static_cast<size_t>(up(K, 64)) * 2;
    size_t n = s.bytes(M, N);
    if (s.tile > 0) n = up16(n) + (rows_fit(x, K, ldx) ? 0 : M * row) + (rows_fit(w, K, ldw) ? 0 : N * row);
    return n;
}

hipError_t launch_linear(const LinearArgs& a, hipStream_t stream) {
    const Shape s = forward_shape(a.M, a.K, a.N);
    GemmArgs g{};
    g.M = a.M;
    g.N = a.N;
    g.x = static_cast<const uint8_t*>(a.x);
    g.w = static_cast<const uint8_t*>(a.w);
    g.ldx = 2 * a.ldx;
    g.ldw = 2 * a.ldw;
    g.steps = static_cast<int>((a.K + 63) / 64);
    g.tail = static_cast<int>(up(a.K, 8) * 2 - (g.steps - 1) * static_cast<int64_t>(kStepBytes));
    if (s.tile > 0) {
        const int64_t pitch = up(a.K, 64);
        uint16_t* free_at = reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(a.workspace) + up16(s.bytes(a.M, a.N)));
        RowCopy x{static_cast<const uint16_t*>(a.x), a.ldx, 0, nullptr}, w{static_cast<const uint16_t*>(a.w), a.ldw, 0, nullptr};
        if (!rows_fit(a.x, a.K, a.ldx)) {
            x.R = a.M;
            x.to = free_at;
            free_at += a.M * pitch;
            g.x = reinterpret_cast<const uint8_t*>(x.to);
            g.ldx = 2 * pitch;
        }
        if (!rows_fit(a.w, a.K, a.ldw)) {
            w.R = a.N;
            w.to = free_at;
            g.w = reinterpret_cast<const uint8_t*>(w.to);
            g.ldw = 2 * pitch;
        }
        if (x.R + w.R > 0) {
            const hipError_t e = copy_rows(x, w, a.K, stream);
            if (e != hipSuccess) return e;
        }
    }
    return product<Bf16, false, false>(s, g, 2 * a.K, out_of(a), static_cast<float*>(a.workspace), stream);
}

size_t linear8_workspace(int64_t M, int64_t K, int64_t N) { return forward8_shape(M, K, N).bytes(M, N); }

hipError_t launch_linear8(const LinearArgs& a, hipStream_t stream) {
    GemmArgs g{};
    g.M = a.M;
    g.N = a.N;
    g.x = static_cast<const uint8_t*>(a.x);
    g.w = static_cast<const uint8_t*>(a.w);
    g.ldx = g.ldw = block8_pitch(a.K);
    g.xs = a.x_scales;
    g.ws = a.w_scales;
    g.lds = block8_scale_pitch(a.K);
    g.steps = static_cast<int>(g.ldx / kStepBytes);
    g.tail = kStepBytes;
    return product<Fp8, false, false>(forward8_shape(a.M, a.K, a.N), g, 0, out_of(a), static_cast<float*>(a.workspace),
                                      stream);
}

// Whether linear_narrow_kernel makes dz and dx (without dx linear_narrow_dz_kernel dz): whatever w, dx and the gradients that
// are wanted, so that db has the same bits with any of them.
bool narrow(const LinearBwdArgs& a) {
    const int64_t width = a.dtype == SPINGTP_FP32 ? 4 : 2;
    const auto whole = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    return !own_dz(a) && a.M >= kNarrowLeast && a.K <= kNarrowInputs && a.N <= kNarrowOutputs && a.N % 8 == 0 &&
           whole(a.dy) && a.lddy * width % 16 == 0 && a.lddy * width <= kMostRowBytes && (a.act == kIdentity || whole(a.z));
}
// of a workgroup, all of them on the CUs at once (whole tiles, 782 workgroups for 100,000 x 512 by 128: 158 us of the training
// step against 156)
int64_t narrow_rows(int64_t M) { return up((M + kNarrowBlocks - 1) / kNarrowBlocks, 16); }
int64_t narrow_blocks(int64_t M) { return (M + narrow_rows(M) - 1) / narrow_rows(M); }
template <typename TD, int ACT, bool WHOLE>
hipError_t launch_narrow(const LinearBwdArgs& a, const uint16_t* w, int64_t ldw, uint16_t* dz, float* sums,
                         hipStream_t stream) {
    const int64_t pitch = up(a.N, 64);
    const size_t lds = kNarrowLds + static_cast<size_t>(pitch) * 4;
    static_assert(2 * (kNarrowLds + 4 * kNarrowOutputs) <= 160 * 1024, "two workgroups to a CU");
    constexpr auto kernel = linear_narrow_kernel<TD, ACT, WHOLE>;
    const hipError_t e = raise_lds_limit<kernel>();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(narrow_blocks(a.M))), dim3(512), lds, stream,
                       static_cast<const TD*>(a.dy), a.lddy, static_cast<const uint16_t*>(a.z), w, ldw, dz, pitch, sums,
                       static_cast<uint16_t*>(a.dx), a.lddx, a.M, a.N, a.K, narrow_rows(a.M),
                       large(a.M * a.K));
    return hipGetLastError();
}
template <typename TD, bool WHOLE>
hipError_t make_narrow(const LinearBwdArgs& a, const uint16_t* w, int64_t ldw, uint16_t* dz, float* sums,
                       hipStream_t stream) {
    switch (a.act) {
        case kSilu: return launch_narrow<TD, kSilu, WHOLE>(a, w, ldw, dz, sums, stream);
        case kGelu: return launch_narrow<TD, kGelu, WHOLE>(a, w, ldw, dz, sums, stream);
        default: return launch_narrow<TD, kIdentity, WHOLE>(a, w, ldw, dz, sums, stream);
    }
}
template <int LANES, typename TD, int ACT>
hipError_t launch_narrow_dz(const LinearBwdArgs& a, uint16_t* dz, float* sums, hipStream_t stream) {
    const int64_t pitch = up(a.N, 64);
    const unsigned across = static_cast<unsigned>((pitch + 8 * LANES - 1) / (8 * LANES));
    const unsigned blocks = static_cast<unsigned>(narrow_blocks(a.M));
    hipLaunchKernelGGL((linear_narrow_dz_kernel<LANES, TD, ACT>), dim3(across * blocks), dim3(512), 0, stream,
                       static_cast<const TD*>(a.dy), a.lddy, static_cast<const uint16_t*>(a.z), dz, pitch, sums, a.M, a.N,
                       narrow_rows(a.M), across, blocks, across > 2);  // long rows: all of their columns at once (2,048
                                                                       // columns of 65,536 rows 221 us, else 239)
    return hipGetLastError();
}
template <typename TD, int ACT>
hipError_t launch_narrow_dz(const LinearBwdArgs& a, uint16_t* dz, float* sums, hipStream_t stream) {
    if (a.N > 512) return launch_narrow_dz<64, TD, ACT>(a, dz, sums, stream);
    if (a.N > 256) return launch_narrow_dz<32, TD, ACT>(a, dz, sums, stream);
    if (a.N > 128) return launch_narrow_dz<16, TD, ACT>(a, dz, sums, stream);
    return launch_narrow_dz<8, TD, ACT>(a, dz, sums, stream);
}
template <typename TD>
hipError_t make_narrow_dz(const LinearBwdArgs& a, uint16_t* dz, float* sums, hipStream_t stream) {
    switch (a.act) {
        case kSilu: return launch_narrow_dz<TD, kSilu>(a, dz, sums, stream);
        case kGelu: return launch_narrow_dz<TD, kGelu>(a, dz, sums, stream);
        default: return launch_narrow_dz<TD, kIdentity>(a, dz, sums, stream);
    }
}
hipError_t make_narrow(const LinearBwdArgs& a, const uint16_t* w, int64_t ldw, uint16_t* dz, float* sums,
                       hipStream_t stream) {
    if (a.dx == nullptr)
        return a.dtype == SPINGTP_FP32 ? make_narrow_dz<float>(a, dz, sums, stream)
                                       : make_narrow_dz<uint16_t>(a, dz, sums, stream);
    const bool whole = rows_fit(a.dx, a.K, a.lddx);
    if (a.dtype == SPINGTP_FP32)
        return whole ? make_narrow<float, true>(a, w, ldw, dz, sums, stream)
                     : make_narrow<float, false>(a, w, ldw, dz, sums, stream);
    return whole ? make_narrow<uint16_t, true>(a, w, ldw, dz, sums, stream)
                 : make_narrow<uint16_t, false>(a, w, ldw, dz, sums, stream);
}
// rows of the columns' sums
int64_t sum_rows(const LinearBwdArgs& a) { return narrow(a) ? narrow_blocks(a.M) : dz_blocks(a.M, a.N); }

// dz, the sums of its columns, copies of w and x, and the slices' sums of a product
bool makes_dz(const LinearBwdArgs& a) { return (a.dx != nullptr || a.dw != nullptr) && !own_dz(a); }
bool copies_w(const LinearBwdArgs& a) { return a.dx != nullptr && !rows_fit(a.w, a.K, a.ldw); }
bool copies_x(const LinearBwdArgs& a) { return a.dw != nullptr && !rows_fit(a.x, a.K, a.ldx); }
size_t linear_backward_workspace(const LinearBwdArgs& a) {
    const size_t row = static_cast<size_t>(up(a.K, 64)) * 2;
    const size_t dx = a.dx == nullptr ? 0 : dx_shape(a.M, a.K, a.N).bytes(a.M, a.K);
    const size_t dw = a.dw == nullptr ? 0 : dw_shape(a.M, a.K, a.N).bytes(a.N, a.K);
    const size_t copies = ((copies_w(a) ? a.N : 0) + (copies_x(a) ? a.M : 0)) * row;
    const size_t dz = makes_dz(a) ? static_cast<size_t>(a.M * up(a.N, 64)) * 2 : 0;
    int64_t blocks = dz_blocks(a.M, a.N);  // either kernel's
    if (narrow_blocks(a.M) > blocks) blocks = narrow_blocks(a.M);
    const size_t sums = a.db == nullptr ? 0 : static_cast<size_t>(blocks * a.N) * sizeof(float);
    return dz + up16(sums) + copies + larger(dx, dw);
}

hipError_t launch_linear_backward(const LinearBwdArgs& a, hipStream_t stream) {
    if (a.M == 0) {
        hipError_t e = hipSuccess;
        if (a.dw != nullptr)
            e = a.w_dtype == SPINGTP_FP32 ? zero<float>(a.dw, a.N * a.K, stream) : zero<uint16_t>(a.dw, a.N * a.K, stream);
        if (e == hipSuccess && a.db != nullptr) e = zero<float>(a.db, a.N, stream);
        return e;
    }
    const int64_t np = up(a.N, 64), kp = up(a.K, 64);
    const bool own = own_dz(a);
    uint8_t* at = static_cast<uint8_t*>(a.workspace);
    const bool one_launch = narrow(a);
    uint16_t* dz = makes_dz(a) && (a.dw != nullptr || !one_launch) ? reinterpret_cast<uint16_t*>(at) : nullptr;
    if (dz != nullptr) at += 2 * a.M * np;
    float* sums = a.db != nullptr ? reinterpret_cast<float*>(at) : nullptr;
    if (a.db != nullptr) at += up16(static_cast<size_t>(sum_rows(a) * a.N) * sizeof(float));
    RowCopy w{static_cast<const uint16_t*>(a.w), a.ldw, 0, nullptr}, x{static_cast<const uint16_t*>(a.x), a.ldx, 0, nullptr};
    if (copies_w(a)) {
        w.R = a.N;
        w.to = reinterpret_cast<uint16_t*>(at);
        at += 2 * a.N * kp;
    }
    if (copies_x(a)) {
        x.R = a.M;
        x.to = reinterpret_cast<uint16_t*>(at);
        at += 2 * a.M * kp;
    }
    hipError_t e = hipSuccess;
    if (w.R + x.R > 0) e = copy_rows(w, x, a.K, stream);
    const uint16_t* const w_rows = w.R > 0 ? w.to : static_cast<const uint16_t*>(a.w);
    const int64_t ldw = w.R > 0 ? kp : a.ldw;
    if (e == hipSuccess && one_launch)
        e = make_narrow(a, w_rows, ldw, dz, sums, stream);
    else if (e == hipSuccess && (dz != nullptr || sums != nullptr))
        e = a.dtype == SPINGTP_FP32 ? make_dz<float>(a, dz, sums, stream) : make_dz<uint16_t>(a, dz, sums, stream);
    ColumnSums d{sums, sums != nullptr ? sum_rows(a) : 0, a.N, sums != nullptr ? a.db : nullptr};
    const bool joined = a.dw != nullptr && dw_shape(a.M, a.K, a.N).slices > 1 && d.blocks() <= kMostBlocks;
    if (e == hipSuccess && sums != nullptr && !joined) {
        hipLaunchKernelGGL(linear_db_kernel, dim3(static_cast<unsigned>(d.blocks())), dim3(256), 0, stream, d);
        e = hipGetLastError();
    }
    const uint8_t* from = own ? static_cast<const uint8_t*>(a.dy) : reinterpret_cast<const uint8_t*>(dz);
    const int64_t ldz = 2 * (own ? a.lddy : np);
    if (e == hipSuccess && a.dx != nullptr && !one_launch) {
        const Shape s = dx_shape(a.M, a.K, a.N);
        GemmArgs g{};
        g.x = from;
        g.ldx = ldz;
        g.w = reinterpret_cast<const uint8_t*>(w_rows);
        g.ldw = 2 * ldw;
        g.w2 = g.w;
        g.M = a.M;
        g.N = a.K;
        g.steps = static_cast<int>(np / 64);
        g.tail = own ? static_cast<int>(2 * a.N - (g.steps - 1) * static_cast<int64_t>(kStepBytes)) : kStepBytes;
        g.w_rows = a.N;
        g.w_split = g.steps;
        const LinearOut o{kIdentity, false, nullptr, nullptr, 0, a.dx, a.lddx, nullptr, large(a.M * a.K), nullptr, 0};
        if (e == hipSuccess) e = product<Bf16, true, false>(s, g, 0, o, reinterpret_cast<float*>(at), stream);
    }
    if (e == hipSuccess && a.dw != nullptr) {
        const Shape s = dw_shape(a.M, a.K, a.N);
        GemmArgs g{};
        g.w = x.R > 0 ? reinterpret_cast<const uint8_t*>(x.to) : static_cast<const uint8_t*>(a.x);
        g.ldw = 2 * (x.R > 0 ? kp : a.ldx);
        g.w2 = g.w;
        g.x = from;
        g.ldx = ldz;
        g.M = a.N;
        g.N = a.K;
        g.steps = static_cast<int>((a.M + 63) / 64);
        g.tail = kStepBytes;
        g.w_rows = g.x_rows = a.M;
        g.w_split = g.steps;
        const LinearOut o{kIdentity, a.w_dtype == SPINGTP_FP32, nullptr, nullptr, 0, a.dw, a.K, nullptr, false, nullptr, 0};
        if (e == hipSuccess) e = product<Bf16, true, true>(s, g, 0, o, reinterpret_cast<float*>(at), stream, joined ? d : ColumnSums{});
    }
    return e;
}

}  // namespace spingtp
