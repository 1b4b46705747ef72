// Matrix product of two matrices, here with rows that run along the summed axis:
//   c[m][n] = sum_k x[m][k] w[n][k],
// bf16 or 8-bit block format (block8.h) operands, bf16 matrix units, fp32 accumulators, one workgroup per tile of BN
// rows of w and BM rows of x.  The epilogue gets the accumulators.  In the gated form half of the
// tile's w rows come from a second matrix, so a lane holds both products of an output.
//
// A step takes 128 bytes of every row (64 bf16, or 128 8-bit elements: one scale block).  The tiles
// of two to four steps lie in LDS: the loads of the next go straight from memory to LDS while one is
// multiplied.  A row's eight 16-byte chunks are stored rotated by an exclusive or with the row, which
// the loading lanes bring about by which chunk each of them fetches; so the lanes of a fragment read,
// which hold one chunk of 16 rows, spread over all banks.
//
// Either operand may instead have columns that run along the summed axis (bf16: w[k][n], x[k][m]; the
// gradients' products).  A step is then 64 of its rows, the tile's columns of each; they lie in LDS as
// they come, and the fragment reads transpose (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 columns and
// each gets a column's four).  The order of k is the same as of the other form, so the two can meet.  Here
// 32-byte pairs of chunks are rotated by the row, so that the 16 rows of a read spread over all banks
// (counted: no conflicts).  What it saves is the transposed copies: 8,192 x 2,048 x 8,192 forward and backward
// 1,603 -> 1,485 us.
//
// w rows are the matrix unit's rows, x rows its columns, so that a lane's accumulators are one x row and
// runs of four neighbouring w rows: four neighbouring outputs.  The order of k inside a step is the same
// for both operands and otherwise free.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "block8.h"
#include "tile_rule.h"

namespace spingtp {

struct GemmArgs {
    const uint8_t* w;   // [N] rows of ldw bytes
    const uint8_t* w2;  // the second matrix of the gated form
    const uint8_t* x;   // [M] rows of ldx bytes
    int64_t ldw, ldx;   // at most kMostRowBytes
    const uint8_t* ws;  // scales of the 8-bit format
    const uint8_t* ws2;
    const uint8_t* xs;
    int64_t lds;        // bytes of a row of scales (both operands: the same K)
    int64_t M, N;
    int steps;          // of 128 bytes
    int tail;           // bf16: bytes of the last step that exist, a multiple of 16 (128: all)
    int tiles_m, tiles_n;
    // columns along k: rows of w (of each matrix) and x, the step from which on w2 is read, and output rows left
    // out: [gap_at, gap_at + gap), those behind move up
    int64_t w_rows, x_rows;
    int w_split;
    int64_t gap_at, gap;
};

namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int kStepBytes = 128;

// An operand's 16 bytes of a row as bf16 operands of the matrix units, and their shape: bf16 16 x 16 x 32,
// which takes less power for the same products than 32 x 32 x 16 (the clock falls with the power: 2,048 x
// 16,384 outputs of 8,192 terms 438 against 410 us); 8 bits 32 x 32 x 16, for registers.
struct Bf16 {
    static constexpr bool kScaled = false;
    static constexpr int kTile = 16, kParts = 1;
    typedef v4f Acc;
    static __device__ __forceinline__ void expand(v4i raw, float, v8bf (&p)[1]) { p[0] = __builtin_bit_cast(v8bf, raw); }
    static __device__ __forceinline__ Acc product(v8bf a, v8bf b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
// e4m3 values times their block's power of two are bf16 numbers exactly, and v_cvt_scalef32 makes them
// in one instruction for two (but below 2^-133, where bf16 ends), so the products are exact in fp32 and only
// their sum rounds.  (The matrix units' own 8-bit products, at twice the rate, are not taken: of eight products
// summed together they cut what lies below 2^-13 of the largest, 1.5e-5 of a result of normal values against 1e-8 to 8e-8.)
struct Fp8 {
    static constexpr bool kScaled = true;
    static constexpr int kTile = 32, kParts = 2;
    typedef v16f Acc;
    static __device__ __forceinline__ void expand(v4i raw, float scale, v8bf (&p)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t lo = static_cast<uint32_t>(raw[2 * i]), hi = static_cast<uint32_t>(raw[2 * i + 1]);
            const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
            const v2bf b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
            const v2bf c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
            const v2bf d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
            p[i] = v8bf{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
        }
    }
    static __device__ __forceinline__ Acc product(v8bf a, v8bf b, Acc c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};

// Rows from `base` on as a buffer of `bytes` bytes: what a load asks for past them is zero.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const uint8_t* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, static_cast<int>(bytes), 0x00027000);
}
// 16 bytes per lane from the buffer to LDS at `to` + 16 lane.  (As a buffer instruction: the compiler
// takes a global load to LDS for one that may touch LDS in any order, and lets every later read of
// LDS wait for all before it.)
__device__ __forceinline__ void to_lds(Buffer from, uint32_t lane_at, int at, uint8_t* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16,
                                             static_cast<int>(lane_at), at, 0, 0);
}
// Waits until at most LEFT of the wave's loads are in flight (they return in order) and its LDS reads are
// done, then for all waves of the workgroup.  Written out: what __syncthreads waits for is the compiler's
// account, which has lost loads to LDS here where register loads of one branch came between.
template <int LEFT>
__device__ __forceinline__ void arrived_and_read() {
    static_assert(LEFT < 64, "the counter's range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}
// Most bytes between the rows of an operand: a tile's 256 rows in a buffer's 32-bit offsets.
constexpr int64_t kMostRowBytes = (int64_t{1} << 23);

// The tile of this workgroup.  Neighbouring workgroups go to the 8 chiplets in turn: each chiplet
// takes a run of tiles, 8 tiles of x by as many of w, so that its L2 serves both operands.
__device__ __forceinline__ void tile_of(int tiles_m, int tiles_n, int& tm, int& tn) {
    const int total = tiles_m * tiles_n, q = total >> 3, rest = total & 7;
    const int xcd = blockIdx.x & 7, at = blockIdx.x >> 3;
    const int i = xcd * q + (xcd < rest ? xcd : rest) + at;
    const int group = i / (8 * tiles_n), in = i - group * 8 * tiles_n;
    const int rows = tiles_m - 8 * group < 8 ? tiles_m - 8 * group : 8;
    tn = in / rows;
    tm = 8 * group + in - tn * rows;
}

// A wave's tile is PN rows of w by PM rows of x; WN x WM waves; NS steps in LDS.
// KW, KX: the columns of w, x run along the summed axis.
template <class E, int PN, int PM, int WN, int WM, int NS, bool GATED, bool KW = false, bool KX = false>
struct GemmTile {
    static constexpr int kTile = E::kTile, TN = PN / kTile, TM = PM / kTile;  // accumulators of kTile x kTile
    static constexpr int kPhases = kTile == 16 ? 2 : 4;                    // fragment reads of a step
    static constexpr int kQuads = kTile == 16 ? 1 : 4;                     // runs of four outputs in an accumulator
    static constexpr int kWavesN = WN, kWaves = WN * WM, kThreads = 64 * kWaves;
    static constexpr int BN = PN * WN, BM = PM * WM;
    static constexpr int kRows = GATED ? BN / 2 : BN;  // of one matrix
    static constexpr int kStage = (BN + BM) * kStepBytes;
    static constexpr int kLds = NS * kStage + (E::kScaled ? 2 * (BN + BM) * 4 : 0);
    static constexpr int kScaleLoads = (BN + BM + 64 * kWaves - 1) / (64 * kWaves);  // 64-row loads per wave and group
    static constexpr int LW = BN / 8 / kWaves, LX = BM / 8 / kWaves;  // 8-row loads per wave and step
    static_assert(LW * 8 * kWaves == BN && LX * 8 * kWaves == BM && kWaves % 2 == 0, "whole loads");
    static_assert(BN % 64 == 0 && (!GATED || kRows % 64 == 0), "a load of scales is one operand's");
    static_assert(!KX || KW);
    static_assert(!KW || (E::kTile == 16 && !E::kScaled && !GATED), "bf16");
    static_assert(!GATED || (TN % 2 == 0 && LW % 2 == 0), "both halves in a wave, and in its loads");

    typename E::Acc acc[TN][TM];
    int lane, wave, wn, wm;

    // first w row (of its matrix) of accumulator i, and of the tile in LDS
    static __device__ __forceinline__ int row_in(int i, int wn) {
        if constexpr (GATED) return (i % (TN / 2)) * kTile + wn * (PN / 2);
        return wn * PN + i * kTile;
    }
    static __device__ __forceinline__ int lds_row(int i, int wn) {
        return (GATED && i >= TN / 2 ? kRows : 0) + row_in(i, wn);
    }

    // columns along k: what the chunk's number in row r of `cpr` chunks is turned by
    static __device__ __forceinline__ int turn(int cpr, int r) {
        return cpr >= 16 ? 2 * ((r & 3) | ((r >> 3) & 1) << 2) : 2 * (((r >> 1) & 1) | ((r >> 3) & 1) << 1);
    }
    // Eight rows of the lane's column: four at `from`'s row and four `four` bytes on.  (__restrict__: what is known
    // of a pointer keeps the compiler from waiting here for every load to LDS in flight, as with the plain
    // reads' types; dx of 8,192 x 2,048 x 8,192 565 -> 498 us.)
    static __device__ __forceinline__ v4i turned(const uint8_t* __restrict__ from, int four) {
        typedef short v4s __attribute__((ext_vector_type(4)));
        typedef int v2i __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) v4s* P;
        const v2i lo = __builtin_bit_cast(v2i, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(from)));
        const v2i hi = __builtin_bit_cast(v2i, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(from + four)));
        return v4i{lo.x, lo.y, hi.x, hi.y};
    }

    __device__ __forceinline__ void run(const GemmArgs& a, int64_t n0, int64_t m0, uint8_t* lds) {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wn = wave % WN;
        wm = wave / WN;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int r = 0; r < 4 * kQuads; ++r) acc[i][j][r] = 0.f;

        // where the lane's chunk of each load lies: row lane / 8 of the load's eight
        const int key = (4 * (wave & 1) + (lane >> 4)) & 7;  // (row >> 1) & 7
        const int chunk = ((lane & 7) ^ key) * 16;
        const uint32_t ldw = static_cast<uint32_t>(a.ldw), ldx = static_cast<uint32_t>(a.ldx);
        const int rows_w = a.N - n0 < kRows ? static_cast<int>(a.N - n0) : kRows;
        const int rows_x = a.M - m0 < BM ? static_cast<int>(a.M - m0) : BM;
        const uint32_t held = static_cast<uint32_t>(a.steps - 1) * kStepBytes + (E::kScaled ? kStepBytes : a.tail);
        const uint32_t bytes_w = (rows_w - 1) * ldw + held, bytes_x = (rows_x - 1) * ldx + held;
        const Buffer bw = buffer_of(a.w + n0 * a.ldw, bytes_w);
        const Buffer bw2 = buffer_of((GATED ? a.w2 : a.w) + n0 * a.ldw, bytes_w);
        const Buffer bx = buffer_of(a.x + m0 * a.ldx, bytes_x);
        // Columns along k: the next step's rows of an operand as a buffer from the tile's first column on, and the
        // lane's place in load t, `cpr` chunks a row; zeros past the matrix's last row and column.
        const uint8_t* aw = a.w + 2 * n0;
        const uint8_t* ax = a.x + 2 * m0;
        const uint32_t all_w = 64 * ldw - 2 * n0, all_x = 64 * ldx - 2 * m0;
        const uint32_t last_w = KW ? (a.w_rows - 64 * (a.w_split - 1)) * ldw - 2 * n0 : 0;
        const uint32_t last_x = KX ? (a.x_rows - 64 * (a.steps - 1)) * ldx - 2 * m0 : 0;
        const auto size_w = [&](int k) { return k + 1 == a.w_split || k + 1 == a.steps ? last_w : all_w; };
        const auto size_x = [&](int k) { return k + 1 == a.steps ? last_x : all_x; };
        uint32_t sw = size_w(0), sx = size_x(0);
        const auto place = [&](int t, int cpr, uint32_t ld, int64_t column, int64_t columns) {
            const int r = (wave + kWaves * t) * (64 / cpr) + lane / cpr, c = (lane % cpr) ^ turn(cpr, r);
            return column + 8 * c < columns ? r * ld + 16 * c : 0x80000000u;
        };
        uint32_t ow[LW], ox[LX];
#pragma unroll
        for (int t = 0; t < LW; ++t) {
            if constexpr (KW) {
                ow[t] = place(t, BN / 8, ldw, n0, a.N);
                continue;
            }
            const int r = 8 * (wave + kWaves * t) + (lane >> 3) - (GATED && t >= LW / 2 ? kRows : 0);
            ow[t] = (r < rows_w ? r : rows_w - 1) * ldw + chunk;  // rows past the end are not stored
        }
#pragma unroll
        for (int t = 0; t < LX; ++t) {
            if constexpr (KX) {
                ox[t] = place(t, BM / 8, ldx, m0, a.M);
                continue;
            }
            const int r = 8 * (wave + kWaves * t) + (lane >> 3);
            ox[t] = (r < rows_x ? r : rows_x - 1) * ldx + chunk;
        }
        // load t of the wave's LW + LX of step k; steps and loads in order
        auto load_part = [&](int t, int k, uint8_t* to) {
            if (t < LW) {
                uint8_t* const at = to + (wave + kWaves * t) * 1024;
                if constexpr (KW) {
                    to_lds(buffer_of(aw, sw), ow[t < LW ? t : 0], 0, at);
                    if (t == LW - 1) {  // here, among the products, not ahead of them
                        aw = k + 1 == a.w_split ? a.w2 + 2 * n0 : aw + 64 * a.ldw;
                        sw = size_w(k + 1);
                    }
                } else
                    to_lds(GATED && t >= LW / 2 ? bw2 : bw, ow[t < LW ? t : 0], k * kStepBytes, at);
            } else {
                uint8_t* const at = to + (BN / 8 + wave + kWaves * (t - LW)) * 1024;
                if constexpr (KX) {
                    to_lds(buffer_of(ax, sx), ox[t < LW ? 0 : t - LW], 0, at);
                    if (t == LW + LX - 1) ax += 64 * a.ldx, sx = size_x(k + 1);
                } else
                    to_lds(bx, ox[t < LW ? 0 : t - LW], k * kStepBytes, at);
            }
        };
        auto load = [&](int k, uint8_t* to) {
#pragma unroll
            for (int t = 0; t < LW + LX; ++t) load_part(t, k, to);
        };
        // the last step, where its rows end inside: zeros past their end
        auto load_any = [&](int k, uint8_t* to) {
            if (!E::kScaled && !KW && a.tail < kStepBytes && k == a.steps - 1) {
                const bool cut = chunk >= a.tail;
#pragma unroll
                for (int t = 0; t < LW; ++t) ow[t] = cut ? 0x80000000u : ow[t];  // past the buffer
#pragma unroll
                for (int t = 0; t < LX; ++t) ox[t] = cut ? 0x80000000u : ox[t];
            }
            load(k, to);
        };

        // Scales (8 bits): four steps' bytes of a row are a word, the words of the tile's rows a group in LDS;
        // two groups, and in registers the bytes of the lane's rows for a step, read half a step ahead.
        uint8_t* const groups = lds + NS * kStage;
        constexpr int kGroup = E::kScaled ? (BN + BM) * 4 : 0;
        constexpr int LS = kScaleLoads;
        const int last_word = (a.steps - 1) >> 2;
        const uint32_t lds_w = static_cast<uint32_t>(a.lds);
        Buffer bs[LS];
        uint32_t os[LS];
        if constexpr (E::kScaled) {
#pragma unroll
            for (int t = 0; t < LS; ++t) {
                const int first = 64 * (wave + kWaves * t);  // 64 rows of one operand
                const bool in_x = first >= BN, second = GATED && !in_x && first >= kRows;
                const int rows = in_x ? rows_x : rows_w;
                const int r = first - (in_x ? BN : (second ? kRows : 0)) + lane;
                bs[t] = buffer_of(in_x ? a.xs + m0 * a.lds : (second ? a.ws2 : a.ws) + n0 * a.lds,
                                  (rows - 1) * lds_w + (last_word + 1) * 4);
                os[t] = (r < rows ? r : rows - 1) * lds_w;
            }
        }
        auto load_scales = [&](int g) {
            if constexpr (E::kScaled) {
#pragma unroll
                for (int t = 0; t < LS; ++t)
                    if (kScaleLoads * kWaves * 64 == BN + BM || 64 * (wave + kWaves * t) < BN + BM)
                        __builtin_amdgcn_raw_ptr_buffer_load_lds(
                            bs[t],
                            (__attribute__((address_space(3))) void*)(groups + (g & 1) * kGroup + 256 * (wave + kWaves * t)),
                            4, static_cast<int>(os[t]), (g < last_word ? g : last_word) * 4, 0, 0);
            }
        };
        uint32_t ew[TN], ex[TM];
        auto read_scales = [&](int k) {
            if constexpr (E::kScaled) {
                const uint8_t* from = groups + ((k >> 2) & 1) * kGroup + (lane & (kTile - 1)) * 4 + (k & 3);
#pragma unroll
                for (int i = 0; i < TN; ++i) ew[i] = from[lds_row(i, wn) * 4];
#pragma unroll
                for (int j = 0; j < TM; ++j) ex[j] = from[(BN + wm * PM + j * kTile) * 4];
            }
        };

        const int fkey = (lane >> 1) & 7, in = lane & (kTile - 1);
        int at[kPhases];  // the lane's chunk of phase q
#pragma unroll
        for (int q = 0; q < kPhases; ++q) at[q] = in * 128 + (((8 / kPhases * q + lane / kTile) ^ fkey) << 4);

        // The lane's place in the tile's columns along k: row lane / 16 * 8 + lane % 16 / 4, four columns of the
        // wave's first 16; those of fragment i lie 2 i chunks on, bits 5 to 7 of the address, which rows leave free.
        const auto corner = [&](int column, int cpr) {
            const int r = 8 * (lane >> 4) + ((lane & 15) >> 2), c = (column >> 3) + ((lane & 3) >> 1);
            return r * 16 * cpr + ((c ^ turn(cpr, r)) << 4) + ((lane & 1) << 3);
        };
        const int tw = KW ? corner(wn * PN, BN / 8) : 0, tx = KX ? corner(wm * PM, BM / 8) : 0;

        // Fragments are read a phase ahead, and the last phase of a step is multiplied behind the barrier that
        // ends its reads, so the matrix units have work while the next step's first fragments come.
        v4i rw[2][TN], rx[2][TM];
        auto read = [&](const uint8_t* from, int q, int buffer) {
#pragma unroll
            for (int j = 0; j < TM; ++j)
                rx[buffer][j] = KX ? turned(from + BN * 128 + (tx ^ j << 5) + q * 64 * BM, 8 * BM)
                                   : *reinterpret_cast<const v4i*>(from + (BN + wm * PM + j * kTile) * 128 + at[q]);
#pragma unroll
            for (int i = 0; i < TN; ++i)
                rw[buffer][i] = KW ? turned(from + (tw ^ i << 5) + q * 64 * BN, 8 * BN)
                                   : *reinterpret_cast<const v4i*>(from + lds_row(i, wn) * 128 + at[q]);
            __builtin_amdgcn_sched_barrier(0);  // before the products that do not need them
        };
        float fsw[TN], fsx[TM];
        // `between(n)` comes behind the n-th product
        auto multiply = [&](int buffer, auto between) {
            v8bf fw[TN][E::kParts], fx[TM][E::kParts];
#pragma unroll
            for (int j = 0; j < TM; ++j) E::expand(rx[buffer][j], fsx[j], fx[j]);
#pragma unroll
            for (int i = 0; i < TN; ++i) E::expand(rw[buffer][i], fsw[i], fw[i]);
            int n = 0;
#pragma unroll
            for (int p = 0; p < E::kParts; ++p)
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int j = 0; j < TM; ++j) {
                        acc[i][j] = E::product(fw[i][p], fx[j][p], acc[i][j]);
                        between(n++);
                    }
            __builtin_amdgcn_sched_barrier(0);
        };
        const auto nothing = [](int) {};

        load_scales(0);
        load_scales(1);
#pragma unroll
        for (int k = 0; k < NS; ++k)
            if (k < a.steps) load_any(k, lds + k * kStage);
        if (a.steps >= NS)
            arrived_and_read<(NS - 1) * (LW + LX)>();
        else
            arrived_and_read<0>();
        read(lds, 0, 0);
        read_scales(0);
        int at_step = 0;  // where the step lies
        // step k: its products, the loads of step k + NS into its place (MORE = 2: some step before the last, 1:
        // any), the first fragments of step k + 1
        auto step = [&](int k, auto more, auto follows) {
            uint8_t* here = lds + at_step;
            at_step = at_step + kStage < NS * kStage ? at_step + kStage : 0;
            uint8_t* next = lds + at_step;
            if constexpr (E::kScaled) {
#pragma unroll
                for (int i = 0; i < TN; ++i) fsw[i] = __uint_as_float(ew[i] << 23);
#pragma unroll
                for (int j = 0; j < TM; ++j) fsx[j] = __uint_as_float(ex[j] << 23);
            }
#pragma unroll
            for (int q = 0; q < kPhases - 1; ++q) {
                read(here, q + 1, (q + 1) & 1);
                multiply(q & 1, nothing);
            }
            // Step k has been read by all, and step k + 1 has arrived: of the loads in flight, in order, only those
            // of the NS - 2 steps behind it may be left.  (Scales between them make the wait longer, not
            // shorter; a group's are waited for two steps after their issue and read four steps after it.)
            arrived_and_read<decltype(more)::value == 2 ? (NS - 2) * (LW + LX) : 0>();
            if constexpr (decltype(follows)::value) {
                read_scales(k + 1);
                read(next, 0, 0);
            }
            if constexpr (decltype(more)::value == 1) load_any(k + NS, here);
            // the group of this step's scales has been read by all
            if (E::kScaled && (k & 3) == 3 && (k >> 2) + 2 <= last_word) load_scales((k >> 2) + 2);
            // loads spread over the products: a burst of them would hold the wave up at their issue
            multiply(1, [&](int n) {
                constexpr int products = TN * TM * E::kParts, all = LW + LX;
                if (decltype(more)::value == 2 && (n + 1) * all / products > n * all / products) {
#pragma unroll
                    for (int t = n * all / products; t < (n + 1) * all / products; ++t) load_part(t, k + NS, here);
                    __builtin_amdgcn_sched_barrier(0);
                }
            });
        };
        using std::integral_constant;
        int k = 0;
        for (; k + NS + 1 < a.steps; ++k) step(k, integral_constant<int, 2>{}, std::true_type{});
        if (k + NS < a.steps) step(k++, integral_constant<int, 1>{}, std::true_type{});
        for (; k + 1 < a.steps; ++k) step(k, integral_constant<int, 0>{}, std::true_type{});
        step(k, integral_constant<int, 0>{}, std::false_type{});
    }

    // the output column (w row) of the first of run r of tile i's accumulators, and the output row of tile j
    __device__ __forceinline__ int column(int i, int r) const { return row_in(i, wn) + 8 * r + 4 * (lane / kTile); }
    __device__ __forceinline__ int row(int j) const { return wm * PM + j * kTile + (lane & (kTile - 1)); }
};

// Four neighbouring outputs of a row, those before column N.
__device__ __forceinline__ void store4(float* p, int64_t left, float a, float b, float c, float d) {
    if (left >= 4) {
        *reinterpret_cast<u4f*>(p) = u4f{a, b, c, d};
    } else {
        if (left > 0) p[0] = a;
        if (left > 1) p[1] = b;
        if (left > 2) p[2] = c;
    }
}
typedef uint32_t u2u __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void store4(uint16_t* p, int64_t left, float a, float b, float c, float d) {
    const uint32_t lo = bf16_pair(a, b), hi = bf16_pair(c, d);
    if (left >= 4) {
        *reinterpret_cast<u2u*>(p) = u2u{lo, hi};
    } else {
        if (left > 0) p[0] = static_cast<uint16_t>(lo);
        if (left > 1) p[1] = static_cast<uint16_t>(lo >> 16);
        if (left > 2) p[2] = static_cast<uint16_t>(hi);
    }
}

// The product itself, to out [M] rows of ldo elements.
template <class E, int PN, int PM, int WN, int WM, int NS, typename TO, bool KW = false, bool KX = false>
__global__ __launch_bounds__(64 * WN * WM) void gemm_nt_kernel(GemmArgs a, TO* __restrict__ out, int64_t ldo) {
    using Tile = GemmTile<E, PN, PM, WN, WM, NS, false, KW, KX>;
    extern __shared__ __align__(16) uint8_t gemm_lds[];
    int tm, tn;
    tile_of(a.tiles_m, a.tiles_n, tm, tn);
    const int64_t n0 = static_cast<int64_t>(tn) * Tile::BN, m0 = static_cast<int64_t>(tm) * Tile::BM;
    Tile t;
    t.run(a, n0, m0, gemm_lds);
#pragma unroll
    for (int j = 0; j < Tile::TM; ++j) {
        int64_t m = m0 + t.row(j);
        if (m >= a.M) continue;
        if (KX && m >= a.gap_at) {
            m -= a.gap;
            if (m < a.gap_at) continue;
        }
        TO* p = out + m * ldo;
#pragma unroll
        for (int i = 0; i < Tile::TN; ++i)
#pragma unroll
            for (int r = 0; r < Tile::kQuads; ++r) {
                const int64_t n = n0 + t.column(i, r);
                const auto& c = t.acc[i][j];
                store4(p + n, a.N - n, c[4 * r], c[4 * r + 1], c[4 * r + 2], c[4 * r + 3]);
            }
    }
}

}  // namespace
}  // namespace spingtp
