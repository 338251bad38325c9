// The matrix-core tile of the gated feed-forward update and of a classifier's loss: three kinds of product of one shape of kernel.
//
//   FORWARD  G, U [R,C]    = A [R,Kc] B0, B1 [Kc,C]         and the gate in the epilogue
//   ROWS     dX   [R,C]    = sum over groups of A [R,Kc] B [C,Kc]^T
//   WEIGHTS  dWg, dWu [R,C] = A [Kc,R]^T B0, B1 [Kc,C]
//
// and with one result the loss's (fastgl_loss.h)
//
//   SCORES   z [R,C] = A [R,Kc] B [Kc,C], of which each wavefront leaves maximum and sum of exponentials of its columns of every row
//   GRADIENT the same, of which dZ is left as the next products take it, and its column sums
//   ROWS_ADD sums of slabs as ROWS has them, added to what a piece of the classes before left there
//   WEIGHTS_ONE  dW [R,C] = A [Kc,R]^T B [Kc,C] into columns of a wider matrix
//
// All operands are bf16 with rows of a multiple of 16 bytes; fp32 operands come as three planes of pieces, and a
// product of two such is a sequence of six segments, each a product of one plane of either.
//
// * A wavefront has 64 rows and 128 (or 64) columns of a tile: of two results, half the columns each, so that a lane
//   holds G and U of the same elements.  Contracted 32 at a time through a ring of LDS buffers.
// * Operands go from memory to LDS without passing registers (16 bytes a lane).  An operand whose contracted
//   index is contiguous lies as [row][32], read 16 bytes a lane; one whose other index is contiguous lies as [32][column] and is
//   turned on its way out of LDS by the transposing reads.  The 16-byte pieces of a row are permuted (by the addresses they
//   are loaded from) so that the lanes of a read meet different banks.
// * Buffer resources end the operands: what lies beyond is read as 0.  Pieces beyond the contracted range that lie inside an
//   operand are given an address beyond the end.
// * What bounds it: the matrix instructions at the clock that the card holds under them (1.7 to 1.9 GHz of 2.4).  Kernel times, the least of
//   150 passes on one card: dWg, dWu of 16 384 rows 1024 x 4096 bf16 215 us, 1279 TFLOP/s, the matrix cores busy 82 to 87 % of a compute unit's
//   cycles; dX there 222 us, 1238 TFLOP/s (a library product of that shape 215); forward 16 384 rows 1024 -> 4096 242 us without G and U, 1136
//   TFLOP/s; 115 000 rows 256 -> 1024 with them 174 us, bound by its 706 MB of results (4.4 TB/s with what is read).  No LDS bank conflicts
//   in dX and dW.  fp32 runs at a sixth: 207 TFLOP/s at 16 384 rows 1024 -> 4096 with GELU.
// * Results are turned through LDS, 64 x 64 at a time for each wavefront alone, into whole 128-byte lines.
#pragma once
#include <type_traits>

#include "rows_device.h"
#include "fastgl_gated.h"

namespace fastgl {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#define FASTGL_LDS __attribute__((address_space(3)))

enum TileMode { kForward = 0, kRows = 1, kWeights = 2, kScores = 3, kGradient = 4, kRowsAdd = 5, kWeightsOne = 6 };

constexpr int kStep = 32;                       // contracted elements of an LDS buffer
constexpr uint32_t kNoSuchOffset = 0x7FFFFF00u; // beyond every buffer
constexpr int kTileRsrc = 0x00020000;

struct TileArgs {
    const uint16_t *a[2], *b[2];   // FORWARD, WEIGHTS: a[0] and b[0], b[1]; ROWS: group g has a[g], b[g]
    int64_t a_plane, b_plane;      // elements between planes of pieces
    int64_t lda, ldb;              // elements between rows, multiples of 8; contiguous contracted elements are 0 from Kc on to a multiple of 8
    int64_t a_blocks, b_blocks;    // 0, or ROWS' A and WEIGHTS' B lie in blocks of 32 columns, [block][row][32], so many elements a block
    int64_t R, C, Kc;
    int32_t pairs, groups;         // segments: groups x pairs of a plane of A and a plane of B
    uint32_t planes_a, planes_b;   // the planes of pair i: four bits each from bit 4 i
    int32_t tiles_r, tiles_c, slabs;      // slabs: the steps of all segments are dealt to as many workgroups a tile
    const float *bias[2];          // FORWARD, or NULL
    void *out[3];                  // FORWARD: P, G, U (G, U or NULL); ROWS: dX; WEIGHTS: dWg, dWu
    float *part;                   // slabs > 1: their sums, [slab][results][R][C]
};

struct LossTileArgs : TileArgs {
    int64_t shift;                 // SCORES, GRADIENT: the column of B that column 0 is
    int64_t ldo;                   // WEIGHTS_ONE: elements between rows of the result
    int32_t add;                   // ROWS_ADD: whether `part` holds sums to add to
    const int64_t *label;          // [R]
    int64_t first, classes;        // the class of column 0, and all of them
    float *stats;                  // SCORES: [column tile and wavefront][R][2]
    float *picked;                 // SCORES: [R] the score of the label
    const float *lse, *dloss;      // GRADIENT: [R]
    uint16_t *dz;                  // GRADIENT: planes of dZ; column c of row r at (c >> 5) * dz_block + r * dz_ld + (c & 31)
    int64_t dz_plane, dz_ld, dz_block;
    float *db;                     // GRADIENT: [row tile and wavefront][C] column sums, or NULL
};
template <int MODE> struct TileArgsOf { typedef TileArgs type; };
template <> struct TileArgsOf<kScores> { typedef LossTileArgs type; };
template <> struct TileArgsOf<kGradient> { typedef LossTileArgs type; };
template <> struct TileArgsOf<kRowsAdd> { typedef LossTileArgs type; };
template <> struct TileArgsOf<kWeightsOne> { typedef LossTileArgs type; };

// Pairs of planes, smallest products first: six of three planes and three (0 2, 2 0, 1 1, 0 1, 1 0, 0 0), and two of two and one.
constexpr uint32_t kSixA = 0x001120, kSixB = 0x010102, kTwo = 0x01;

// exp(-x), x >= 0 or any: 2^(-x log2 e).  Relative error 2^-23 (1 + |x|): the rounding of the exponent.
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(-1.44269504089f * x); }

// The normal distribution below -x and what exp(-x^2 / 2) is there, x >= 0 (not NaN): the distribution times exp(x^2 / 2) is a
// polynomial in t = 1 / (1 + c x) without a constant term, its coefficients fitted here to the function in 64 bits so that the largest relative
// error is least over 0 <= x <= 13.5.  Relative, so that the products of large negative gates keep their digits.
//   fp32   nine terms (2e-8), t to the last bit, the square of x in two parts and its exponent too: at most 8.4 x 2^-24 altogether
//   bf16   six terms (4e-5, a hundredth of a bf16 rounding; 2e-7 of the largest value)
// us a call, fp32, with a series of five terms that bounds the absolute error (7.5e-8: 5e-5 relative at -3, 4e-3 at -6) / so: 60 000 rows
// 64 -> 512 81 / 87, 16 384 rows 1024 -> 4096 1307 / 1329; bf16: the same with five and six terms.
template <bool BF16>
__device__ __forceinline__ float normal_tail(float x, float *density)
{
    if constexpr (BF16) {
        const float t = __builtin_amdgcn_rcpf(fmaf(0.296984851f, x, 1.f));
        *density = __builtin_amdgcn_exp2f(-0.721347520f * (x * x));
        const float p = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.0816464052f, 0.237926498f), -0.0390622281f), 0.153226212f), 0.110543162f), 0.119012617f);
        return t * p * *density;
    } else {
        x = fminf(x, 32.f);                                  // the square stays finite; the result is 0 from 13.3 on
        const float d = fmaf(0.26870057f, x, 1.f), t0 = __builtin_amdgcn_rcpf(d), t = fmaf(fmaf(-d, t0, 1.f), t0, t0);
        const float square = x * x, square_rest = fmaf(x, x, -square);
        const float a = square * 0.721347520f;               // log2(e) / 2 in two parts
        const float a_rest = fmaf(square_rest, 0.721347520f, fmaf(square, 0.721347520f, -a) + square * 9.62981517e-09f);
        const float e = __builtin_amdgcn_exp2f(-a);
        *density = fmaf(e, -0.693147181f * a_rest, e);
        const float p = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.0294481106f, -0.130960837f), 0.18154034f), -0.080257751f),
                        0.114666335f), 0.069482483f), 0.10191007f), 0.106966197f), 0.107205063f);
        return t * p * *density;
    }
}

// act(g) and, where wanted, its derivative.  The sigmoid is 1 / (1 + exp(-g)).
template <int ACT, bool GRAD, bool BF16>
__device__ __forceinline__ float gate(float g, float *grad)
{
    if constexpr (ACT == FASTGL_ACT_RELU) {
        if (GRAD) *grad = g > 0.f ? 1.f : g != g ? g : 0.f;
        return g < 0.f ? 0.f : g;                            // NaN stays NaN
    } else if constexpr (ACT == FASTGL_ACT_GELU) {
        float e;
        const float tail = normal_tail<BF16>(fabsf(g), &e);
        const float cdf = g < 0.f ? tail : 1.f - tail;
        if (GRAD) *grad = fmaf(g * 0.39894228040f, e, cdf);
        return g * cdf;
    } else {
        const float s = __builtin_amdgcn_rcpf(1.f + exp_neg(g));
        if constexpr (ACT == FASTGL_ACT_SIGMOID) {
            if (GRAD) *grad = s * (1.f - s);
            return s;
        } else {
            if (GRAD) *grad = s * fmaf(g, 1.f - s, 1.f);
            return g * s;
        }
    }
}

// Tiles: rows, columns (of all results together), wavefronts, LDS buffers.  A compute unit has one workgroup of the large
// tile, two of the others.
enum TileSize { kLarge = 0, kMiddle = 1, kSmall = 2 };

template <int MODE, int SIZE>
struct Tile {
    static constexpr int NW = SIZE == kLarge ? 8 : 4, BM = SIZE == kLarge ? 256 : 128, BNV = SIZE == kSmall ? 128 : 256;
    static constexpr int BUFS = SIZE == kMiddle ? 3 : 5;
    static constexpr int WM = SIZE == kLarge ? 4 : 2, WN = 2;
    static constexpr int TM = BM / WM / 32, TN = BNV / WN / 32;          // blocks of 32 x 32 a wavefront
    static constexpr bool FORWARD = MODE == kForward || MODE == kScores || MODE == kGradient, ROWS = MODE == kRows || MODE == kRowsAdd;
    static constexpr bool WEIGHTS = MODE == kWeights || MODE == kWeightsOne, DUAL = MODE == kForward || MODE == kWeights;
    static constexpr int RESULTS = DUAL ? 2 : 1, BC = BNV / RESULTS;     // columns of one result
    static constexpr bool A_T = WEIGHTS, B_T = !ROWS;                    // other index contiguous
    static constexpr int A_BYTES = BM * kStep * 2, B_BYTES = BNV * kStep * 2, STAGE = A_BYTES + B_BYTES;
    static constexpr int THREADS = NW * kWave;
    static constexpr int LA = A_BYTES / (THREADS * 16), LB = B_BYTES / (THREADS * 16);      // 16-byte loads a lane
    static_assert(TM == 2 && LA == 2, "tile shape");
};

// The tile of a product and how many workgroups share the steps of one.
struct Cut {
    int size;
    int64_t slabs;
};

// The cut that a model of the launch finds fastest.  A compute unit needs single_us for a step of a workgroup that it has alone and
// pair_us for one of each of two (large tiles: one at a time), and tile_us for what is around the steps; slabs cost the sums that they
// write and that are read again (4 bytes each way at some 6 TB/s), and a launch.
// Measured (bf16, us for large / middle / small tiles; kernel times, the least of 150 passes on one card):
//   forward 16 384 rows 1024 -> 4096, G and U kept 273 / 269 / -, alone 241 / 253 / -;  115 000 rows 256 -> 1024 193 / 174 / -, 162 / 140 / -
//   dX of 16 384 rows 1024 -> 4096 223 / 278 / 310, dWg and dWu there 218 / 241 / 401 (the first two in two slabs)
//   all kernels of a backward call of 300 rows 256 -> 1024 (medians) 36 / 32 / 31, of 2000 rows 52 / 47 / 43, of 8000 rows 256 -> 683 73 / 67 / 60
// The loss's products have one result of twice the columns (`one`); scores are not summed over slabs (`whole`), and what becomes of them hides
// behind another workgroup's products where there are two: us a call, large / middle tiles, 8192 rows -> 16 384 bf16, forward and dZ (one piece): 256 inputs 93 + 162 / 83 + 142,
// 512 144 + 210 / 135 + 195, 1024 239 + 307 / 240 + 303, 2048 418 + 517 / 452 + 513; fp32 128 inputs 199 + 372 / 192 + 326, 512 633 + 807 / 682 + 820.
inline Cut cut_of(int mode, int64_t R, int64_t C, int64_t Kc, int64_t segments, bool one = false, bool whole = false)
{
    static const double single_us[3][3] = {{0.80, 0.60, 0.36}, {0.93, 0.65, 0.38}, {0.80, 0.60, 0.42}};      // [mode][size]
    static const double pair_us[3][3] = {{1.60, 0.92, 0.64}, {1.86, 1.10, 0.70}, {1.60, 0.92, 0.80}};
    static const double tile_us[2][3] = {{6.0, 2.6, 1.6}, {4.0, 2.0, 1.2}};
    Cut best = {kLarge, 1};
    double least = 1e300;
    const int64_t all = ceil_div(Kc, kStep) * segments;
    for (int size = kLarge; size <= kSmall; ++size) {
        const int64_t bm = size == kLarge ? 256 : 128, bc = (size == kSmall ? 128 : 256) / (mode == kRows || one ? 1 : 2);
        const int64_t tiles = ceil_div(R, bm) * ceil_div(C, bc);
        for (int64_t slabs = 1; slabs <= (whole ? 1 : 64) && (slabs == 1 || (all / slabs >= 4 && R * C <= (int64_t)1 << 30)); slabs = slabs < 8 ? slabs + 1 : slabs * 5 / 4) {
            const int64_t of_unit = ceil_div(tiles * slabs, 256);
            const double step = (double)(of_unit / 2) * pair_us[mode][size] + (double)(of_unit % 2) * single_us[mode][size];
            const double us = (double)ceil_div(all, slabs) * step + (double)of_unit * (tile_us[mode != kForward][size] + (whole && size == kLarge ? 4.0 : 0.0)) +
                              (slabs > 1 ? 4.0 + (double)slabs * (double)R * (double)C * (mode == kRows || one ? 1.3e-6 : 2.6e-6) : 0.0);
            if (us < least) {
                least = us;
                best = {size, slabs};
            }
        }
    }
    return best;
}

// Which 16-byte piece of row k a [32][columns] buffer has at place p: rows of RB bytes.  Reads take 64 bytes of four
// consecutive rows at a time, which this puts 64 bytes apart modulo 256.
template <int RB>
__device__ __forceinline__ int turned(int k) { return RB >= 256 ? 4 * (k & 3) : 4 * ((k >> 1) & 1); }
// The same for a [row][32] buffer (rows of 64 bytes), read one piece of 32 consecutive rows at a time: 16 rows meet all
// the banks once.
__device__ __forceinline__ int twisted(int row) { return (row >> 2) & 3; }

namespace {

// Sums v[0 .. N) over the lanes that differ in the bits O, O / 2, ... FROM: at each bit a lane keeps one half of what it holds and
// gives the other away, so that N - 1 exchanges (not N for each bit) are enough.  A lane ends with N FROM / 64 values (one at
// least), of the returned index onwards.
template <int N, int O, int FROM, int NV>
__device__ __forceinline__ int scatter_sum(float (&v)[NV], int lane)
{
    if constexpr (O < FROM) {
        return 0;
    } else if constexpr (N > 1) {
        const bool up = lane & O;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float give = up ? v[i] : v[i + N / 2], keep = up ? v[i + N / 2] : v[i];
            v[i] = keep + __shfl_xor(give, O, kWave);
        }
        return (up ? N / 2 : 0) + scatter_sum<N / 2, O / 2, FROM>(v, lane);
    } else {
        v[0] += __shfl_xor(v[0], O, kWave);
        return scatter_sum<1, O / 2, FROM>(v, lane);
    }
}

// Whether log2 e times a finite score is no float.
__device__ __forceinline__ bool beyond_log2e(float z) { return fabsf(z) > 2.3586e38f && fabsf(z) < INFINITY; }

// A wavefront's scores: rows row0 + 32 i + lane % 32, columns col0 + 32 j + 8 (e / 4) + 4 (lane / 32) + e % 4 in acc[i][j][e].
// SCORES: maximum and sum of exponentials (of what the maximum leaves) of its columns of each row, and the label's score where it is among them.  The
// exponents are taken from the rounded product of the maximum and log2 e, which costs one operation a score; what its rounding left is a factor of the
// sum.  Where that product is no float (scores of the type's lowest value rule a class out as well as -inf does) the maximum is subtracted first.
// GRADIENT: dZ = g (exp(z - lse) - [label]), 0 in rows without a label and in columns that do not exist (to a multiple of 32), as
// `planes` bf16 whose sum is it (one: rounded), and its column sums.
// Labels are looked for only by wavefronts that have one.
template <int MODE, class T, int PLANES, class ARGS>
__device__ __forceinline__ void loss_epilogue(const ARGS &g, f32x16 (&acc)[T::TM][T::TN], int64_t row0, int64_t col0, int64_t row_slot, int64_t col_slot)
{
    constexpr float kLog2e = 1.44269504089f;
    const int lane = threadIdx.x & (kWave - 1), h = lane >> 5, l32 = lane & 31;
    const int64_t far = g.C - col0;                                       // columns that exist, less this lane's first
    const int left = (int)(far < T::TN * 32 ? far : T::TN * 32) - 4 * h;
    if (far <= 0) return;                                                 // the same for a wavefront
    if (far < T::TN * 32) {                                               // columns that do not exist weigh nothing
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 32 * j + 8 * (e >> 2) + (e & 3) < left ? acc[i][j][e] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < T::TM; ++i) {
        const int64_t row = row0 + i * 32 + l32;
        const bool in = row < g.R;
        const int64_t label = in ? g.label[row] : -1, at = label - g.first - col0 - 4 * h;      // of the label among this lane's columns
        const int mine = label >= 0 && at >= 0 && at < left ? (int)at : -1;
        const bool any = __any(mine >= 0);
        if constexpr (MODE == kScores) {
            float most = -INFINITY, sum = 0.f;
#pragma unroll
            for (int j = 0; j < T::TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) most = fmaxf(most, acc[i][j][e]);
            most = fmaxf(most, __shfl_xor(most, 32, kWave));
            const float base = most == -INFINITY ? 0.f : most * kLog2e;
            if (beyond_log2e(most)) {
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f((acc[i][j][e] - most) * kLog2e);
            } else {
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], kLog2e, -base));
                if (most != -INFINITY) sum *= __builtin_amdgcn_exp2f(-fmaf(most, kLog2e, -base));
            }
            sum += __shfl_xor(sum, 32, kWave);
            if (h == 0 && in) {
                typedef float f2 __attribute__((ext_vector_type(2)));
                reinterpret_cast<f2 *>(g.stats)[col_slot * g.R + row] = f2{most, sum};
            }
            if (any) {
                float z = 0.f;
                bool has = false;
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const bool is = 32 * j + 8 * (e >> 2) + (e & 3) == mine;
                        z = is ? acc[i][j][e] : z;
                        has = has || is;
                    }
                if (has) g.picked[row] = z;
            }
        } else {
            const float lse = label >= 0 ? g.lse[row] : 0.f, base = lse * kLog2e;
            const float scale = label >= g.classes ? NAN : label >= 0 ? g.dloss[row] : 0.f;
            if (label < 0) {                                              // whatever the scores are: a NaN of the weights or the bias times 0
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
            } else if (beyond_log2e(lse)) {
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] = __builtin_amdgcn_exp2f((acc[i][j][e] - lse) * kLog2e) * scale;
            } else {
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[i][j][e] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], kLog2e, -base)) * scale;
            }
            if (any) {
#pragma unroll
                for (int j = 0; j < T::TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        acc[i][j][e] = 32 * j + 8 * (e >> 2) + (e & 3) == mine ? acc[i][j][e] - scale : acc[i][j][e];
            }
        }
    }
    if constexpr (MODE == kGradient) {
        if (g.db) {
            constexpr int NV = T::TN * 16;
            float sums[NV];
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                sums[c] = 0.f;
#pragma unroll
                for (int i = 0; i < T::TM; ++i) sums[c] += acc[i][c / 16][c % 16];
            }
            const int at = scatter_sum<NV, 16, 1>(sums, lane);
#pragma unroll
            for (int k = 0; k < NV / 32; ++k) {
                const int e = at + k, c = 32 * (e >> 4) + 8 * ((e >> 2) & 3) + (e & 3);
                if (c < left) g.db[row_slot * g.C + col0 + 4 * h + c] = sums[k];
            }
        }
        // Eight columns a lane: the lower 32 lanes have those of an even group of eight, the upper ones those of the odd one beside it.
#pragma unroll
        for (int i = 0; i < T::TM; ++i) {
            const int64_t row = row0 + i * 32 + l32;
            if (row >= g.R) continue;
#pragma unroll
            for (int j = 0; j < T::TN; ++j) {
                if (32 * j >= far) break;
                uint16_t *to = g.dz + (col0 / 32 + j) * g.dz_block + row * g.dz_ld + 8 * h;
#pragma unroll
                for (int p = 0; p < PLANES; ++p)
#pragma unroll
                    for (int q = 0; q < 4; q += 2) {
                        uint32_t w[2][2];
#pragma unroll
                        for (int o = 0; o < 2; ++o)
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                float &lo = reinterpret_cast<float *>(&acc[i][j])[4 * (q + o) + 2 * x], &hi = reinterpret_cast<float *>(&acc[i][j])[4 * (q + o) + 2 * x + 1];
                                w[o][x] = pack_bf16(lo, hi);
                                if (p + 1 < PLANES) {
                                    lo -= __uint_as_float(w[o][x] << 16);
                                    hi -= __uint_as_float(w[o][x] & 0xFFFF0000u);
                                }
                            }
                        const auto a = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false), b = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
                        *reinterpret_cast<u32x4 *>(to + p * g.dz_plane + 8 * q) = u32x4{a[0], b[0], a[1], b[1]};
                    }
            }
        }
    }
}

// PART: sums of a slab instead of results.  ONCE: whole lines of results go past the caches.  ACT: of GRADIENT the planes of dZ.
template <int MODE, int SIZE, class OUT, int ACT, bool PART, bool ONCE>
__global__ __launch_bounds__((Tile<MODE, SIZE>::THREADS), 2) void k_gated_tile(typename TileArgsOf<MODE>::type g)
{
#ifdef __HIP_DEVICE_COMPILE__                    // the host pass makes no launch stub of a body with these builtins
    using T = Tile<MODE, SIZE>;
    constexpr int NW = T::NW;
    __shared__ __attribute__((aligned(1024))) char lds[T::BUFS * T::STAGE];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wm = wave / T::WN, wn = wave % T::WN, h = lane >> 5, l32 = lane & 31;

    // Workgroups are dealt to the eight L2 domains in turn: each gets a run of consecutive tiles, taken four rows of
    // tiles at a time, column after column, so that those under way at once share their operands.
    const uint32_t per_slab = (uint32_t)g.tiles_r * (uint32_t)g.tiles_c, total = per_slab * (uint32_t)g.slabs;
    uint32_t at = blockIdx.x;
    {
        const uint32_t q = total / kXcds, rest = total % kXcds, x = at % kXcds;
        at = x * q + (x < rest ? x : rest) + at / kXcds;
    }
    const uint32_t slab = at / per_slab;
    at -= slab * per_slab;
    const uint32_t band = at / (4u * (uint32_t)g.tiles_c), first = 4u * band;
    const uint32_t high = (uint32_t)g.tiles_r - first < 4u ? (uint32_t)g.tiles_r - first : 4u;
    at -= first * (uint32_t)g.tiles_c;
    const int64_t row0 = (int64_t)(first + at % high) * T::BM, col0 = (int64_t)(at / high) * T::BC;

    const int steps = (int)((g.Kc + kStep - 1) / kStep), nseg = g.pairs * g.groups;
    const int first_step = PART ? (int)((int64_t)steps * nseg * slab / g.slabs) : 0;
    const int all = (PART ? (int)((int64_t)steps * nseg * (slab + 1) / g.slabs) : steps * nseg) - first_step;

    const int64_t a_blocks = T::ROWS ? g.a_blocks : 0, b_blocks = T::WEIGHTS ? g.b_blocks : 0;

    // Where this lane's 16-byte pieces of a step come from.
    uint32_t off_a[T::LA], off_b[T::LB];
    const int piece_k = (lane & 3) ^ twisted(lane >> 2);                 // [row][32]: sixteen rows an instruction
    auto place = [&](auto other, auto columns, int64_t ld, int64_t blocks, int inst) __attribute__((always_inline)) {
        if (blocks) ld = 32;
        if constexpr (!decltype(other)::value) {
            return (uint32_t)((inst * 16 + (lane >> 2)) * ld * 2) + 16u * (uint32_t)piece_k;
        } else {
            constexpr int COLS = decltype(columns)::value, PER_ROW = COLS / 8;
            const int k = (inst * kWave + lane) / PER_ROW, c = (lane & (PER_ROW - 1)) ^ turned<COLS * 2>(k);
            if (blocks) return (uint32_t)(k * 64 + (c >> 2) * blocks * 2) + 16u * (uint32_t)(c & 3);
            return (uint32_t)(k * ld * 2) + 16u * (uint32_t)c;
        }
    };
    typedef std::integral_constant<int, T::BM> ColsA;
    typedef std::integral_constant<int, T::BC> ColsB;
#pragma unroll
    for (int i = 0; i < T::LA; ++i) off_a[i] = place(std::integral_constant<bool, T::A_T>(), ColsA(), g.lda, a_blocks, i * NW + wave);
#pragma unroll
    for (int i = 0; i < T::LB; ++i)
        off_b[i] = place(std::integral_constant<bool, T::B_T>(), ColsB(), g.ldb, b_blocks, i % (T::LB / T::RESULTS) * NW + wave);

    // The operands of the step that is loaded next.  Resources begin at the step's first element and end, for an operand
    // whose contracted index is contiguous, with the tile's last row (a row's pieces beyond the contracted range are given an
    // address beyond every end, in a segment's last step), for the others with the step's last contracted row.
    int seg = PART ? first_step / (steps > 0 ? steps : 1) : 0, t = first_step - seg * steps, loaded = 0;
    int into = 0;                                                        // bytes to the LDS buffer it goes to
    const uint16_t *next_a, *next_b[2];
    const int64_t step_a = T::A_T ? kStep * g.lda : a_blocks ? a_blocks : kStep, step_b = T::B_T ? kStep * (b_blocks ? 32 : g.ldb) : kStep;
    const int64_t row_a = a_blocks ? 32 : g.lda;
    const int last_rows = (int)(g.Kc - (int64_t)(steps - 1) * kStep);     // contracted elements of a segment's last step
    const int64_t rows_a = g.R - row0 < T::BM ? g.R - row0 : T::BM, rows_b = g.C - col0 < T::BNV ? g.C - col0 : T::BNV;
    const int bytes_a = (int)(2 * (T::A_T ? kStep * g.lda - row0 : rows_a * row_a));
    // blocks of columns: what the tile has of them; where a block's own rows end, only masks tell
    int64_t left_blocks = b_blocks ? (g.C - col0 + 31) / 32 : 0;
    left_blocks = left_blocks < T::BC / 32 ? left_blocks : T::BC / 32;
    int64_t col_b = col0;                                                // of B
    if constexpr (MODE == kScores || MODE == kGradient) col_b += g.shift;
    const int bytes_b = (int)(2 * (b_blocks ? left_blocks * b_blocks : T::B_T ? kStep * g.ldb - col_b : rows_b * g.ldb));
    const int64_t base_b = b_blocks ? col0 / 32 * b_blocks : T::B_T ? col_b : col0 * g.ldb;
    const int last_a = T::A_T ? (int)(2 * (last_rows * g.lda - row0)) : bytes_a, last_b = T::B_T && !b_blocks ? (int)(2 * (last_rows * g.ldb - col_b)) : bytes_b;
    const bool beyond = piece_k * 8 >= last_rows;                        // rows are padded with zeros to whole pieces
    uint32_t last_off_b[T::LB];
#pragma unroll
    for (int i = 0; i < T::LB; ++i) {
        const int k = (i % (T::LB / T::RESULTS) * NW * kWave + wave * kWave + lane) / (T::BC / 8);         // of this lane's piece
        last_off_b[i] = (T::B_T ? T::WEIGHTS && k >= last_rows : beyond) ? kNoSuchOffset : off_b[i];
    }
    auto begin_segment = [&]() __attribute__((always_inline)) {
        const int grp = T::ROWS ? seg / g.pairs : 0, pair = T::ROWS ? seg - grp * g.pairs : seg;
        const int pa = (int)(g.planes_a >> (4 * pair)) & 15, pb = (int)(g.planes_b >> (4 * pair)) & 15;
        next_a = g.a[grp] + pa * g.a_plane + (T::A_T ? row0 : row0 * row_a) + t * step_a;
#pragma unroll
        for (int q = 0; q < T::RESULTS; ++q)
            next_b[q] = (T::ROWS ? g.b[grp] : g.b[q]) + pb * g.b_plane + base_b + t * step_b;
    };
    auto load_next = [&]() __attribute__((always_inline)) {
        if (loaded >= all) return;
        const bool last = t + 1 == steps;
        FASTGL_LDS char *to = (FASTGL_LDS char *)lds + into + wave * 1024;
        auto rsrc = [&](const uint16_t *p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(p), 0, bytes, kTileRsrc); };
        const auto ra = rsrc(next_a, last ? last_a : bytes_a);
#pragma unroll
        for (int i = 0; i < T::LA; ++i) {
            const uint32_t o = !T::A_T && last && beyond ? kNoSuchOffset : off_a[i];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (FASTGL_LDS void *)(to + i * NW * 1024), 16, (int)o, 0, 0, 0);
        }
#pragma unroll
        for (int q = 0; q < T::RESULTS; ++q) {
            const auto rb = rsrc(next_b[q], last ? last_b : bytes_b);
#pragma unroll
            for (int i = q * (T::LB / T::RESULTS); i < (q + 1) * (T::LB / T::RESULTS); ++i) {
                const uint32_t o = !T::FORWARD && last ? last_off_b[i] : off_b[i];
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (FASTGL_LDS void *)(to + T::A_BYTES + i * NW * 1024), 16, (int)o, 0, 0, 0);
            }
            next_b[q] += step_b;
        }
        next_a += step_a;
        ++loaded;
        into = into == (T::BUFS - 1) * T::STAGE ? 0 : into + T::STAGE;
        if (++t == steps) {
            t = 0;
            ++seg;
            if (loaded < all) begin_segment();
        }
    };

    // Where a lane reads its fragments: row (or column) l32 of a block of 32, contracted elements 8 h .. 8 h + 7 of 16.
    // [row][32]: piece 2 kk + h.  [32][column]: two transposing reads of four contracted rows each; of sixteen lanes four read one
    // row, and lane i gets column i of the four rows.
    const int i16 = lane & 15, g2 = (lane >> 4) & 1;
    uint32_t read_k[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) read_k[kk] = (uint32_t)(l32 * 64 + (((2 * kk + h) ^ twisted(l32)) << 4));
    auto read_t = [&](auto columns, int block) {                        // block: of 32 columns
        constexpr int RB = decltype(columns)::value * 2;
        const int k = 8 * h + (i16 >> 2), piece = (4 * block + 2 * g2 + ((i16 & 3) >> 1)) ^ turned<RB>(k);
        return (uint32_t)(k * RB + piece * 16 + (i16 & 1) * 8);
    };
    constexpr int ONE = T::TN / T::RESULTS;                               // column blocks of one result
    uint32_t at_a[T::TM], at_b[ONE];
#pragma unroll
    for (int i = 0; i < T::TM; ++i) at_a[i] = T::A_T ? read_t(ColsA(), wm * T::TM + i) : 0;
#pragma unroll
    for (int j = 0; j < ONE; ++j) at_b[j] = T::B_T ? read_t(ColsB(), wn * ONE + j) : 0;

    auto frag_k = [&](uint32_t base) { return *(FASTGL_LDS bf16x8 *)((FASTGL_LDS char *)lds + base); };
    auto frag_t = [&](uint32_t base, int row_bytes) {
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FASTGL_LDS i16x4 *)((FASTGL_LDS char *)lds + base));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FASTGL_LDS i16x4 *)((FASTGL_LDS char *)lds + base + 4 * row_bytes));
        struct { i16x4 l, h; } both = {lo, hi};
        return __builtin_bit_cast(bf16x8, both);
    };
    struct Frags { bf16x8 a[T::TM], b[T::TN]; };
    auto read = [&](int buf, int kk) __attribute__((always_inline)) {
        Frags f;
        const uint32_t base = (uint32_t)buf;
#pragma unroll
        for (int i = 0; i < T::TM; ++i) {
            if constexpr (T::A_T) f.a[i] = frag_t(base + at_a[i] + (uint32_t)(kk * 16 * 2 * T::BM), 2 * T::BM);
            else f.a[i] = frag_k(base + read_k[kk] + (uint32_t)((wm * T::TM + i) * 32 * 64));
        }
#pragma unroll
        for (int j = 0; j < T::TN; ++j) {
            if constexpr (T::B_T)
                f.b[j] = frag_t(base + T::A_BYTES + j / ONE * (T::B_BYTES / T::RESULTS) + at_b[j % ONE] + (uint32_t)(kk * 16 * 2 * T::BC), 2 * T::BC);
            else f.b[j] = frag_k(base + T::A_BYTES + read_k[kk] + (uint32_t)((wn * T::TN + j) * 32 * 64));
        }
        return f;
    };

    // Sums start from the biases.  Operands are multiplied columns first: lane l then holds, of row l32 of a block, columns
    // 8 q + 4 h + (0 .. 3) in elements 4 q + (0 .. 3).
    f32x16 acc[T::TM][T::TN];
#pragma unroll
    for (int j = 0; j < T::TN; ++j) {
        f32x16 start;
#pragma unroll
        for (int e = 0; e < 16; ++e) start[e] = 0.f;
        if constexpr (T::FORWARD && !PART)
            if (const float *bias = g.bias[j / ONE]) {
                const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(bias), 0, (int)(g.C * 4), kTileRsrc);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)(4 * (col0 + (wn * ONE + j % ONE) * 32 + 8 * q + 4 * h)), 0, 0);
#pragma unroll
                    for (int x = 0; x < 4; ++x) start[4 * q + x] = __uint_as_float(v[x]);
                }
            }
#pragma unroll
        for (int i = 0; i < T::TM; ++i) acc[i][j] = start;
    }
    auto multiply = [&](const Frags &f) {
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int i = 0; i < T::TM; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.b[j], f.a[i], acc[i][j], 0, 0, 0);
    };
    // The reads of the next fragments go between the matrix instructions of this one, the first of them in front.
    auto interleave = [&]() {
        constexpr int READS = T::TM * (T::A_T ? 2 : 1) + T::TN * (T::B_T ? 2 : 1), MATRIX = T::TM * T::TN;
#pragma unroll
        for (int i = 0; i < MATRIX; ++i) {
            if (i * 2 < READS) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
        if (READS > 2 * MATRIX) __builtin_amdgcn_sched_group_barrier(0x100, READS - 2 * MATRIX, 0);
        __builtin_amdgcn_sched_barrier(0);
    };

    // A step multiplies what lies in its buffer, in two halves.  Between them is its barrier: everybody has read the buffer,
    // and everybody's loads of the next step have arrived, so that the next step's first fragments are read during the second half.
    // The loads that a step begins go where the step before it was, and have BUFS - 3/2 steps to arrive.
    constexpr int IN_FLIGHT = T::LA + T::LB;                 // loads of a step
    if (all > 0) {
        begin_segment();
#pragma unroll
        for (int i = 0; i < T::BUFS - 1; ++i) load_next();
        if (all >= T::BUFS - 1) __builtin_amdgcn_s_waitcnt(0x0F70 | (T::BUFS - 2) * IN_FLIGHT);
        else __builtin_amdgcn_s_waitcnt(0x0F70);
        __builtin_amdgcn_s_barrier();
        Frags f = read(0, 0);
        int now = 0;                                         // bytes to the step's buffer
        auto step = [&](auto arrived) __attribute__((always_inline)) {
            load_next();
            __builtin_amdgcn_sched_barrier(0);
            const Frags n = read(now, 1);
            multiply(f);
            interleave();
            __builtin_amdgcn_s_waitcnt(decltype(arrived)::value);       // and lgkmcnt 0: the fragments are here
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            now = now == (T::BUFS - 1) * T::STAGE ? 0 : now + T::STAGE;
            f = read(now, 0);                                // of no use after the last step
            multiply(n);
            interleave();
        };
        int s = 0;
        for (; s < all - (T::BUFS - 1); ++s) step(std::integral_constant<int, 0x0070 | (T::BUFS - 2) * IN_FLIGHT>());
        for (; s < all; ++s) step(std::integral_constant<int, 0x0070>());
    }

    // ------------------------------------------------------------------ epilogue
    __builtin_amdgcn_s_waitcnt(0xC07F);              // lgkmcnt 0
    __builtin_amdgcn_s_barrier();                    // the LDS buffers are free: each wavefront has a part for itself
    constexpr int OB = (int)sizeof(OUT), PARTB = T::BUFS * T::STAGE / NW & ~1023;
    constexpr int ROWB = 64 * OB;                                        // 64 columns of a row
    static_assert(64 * ROWB <= PARTB, "a block of 64 x 64 results fits a wavefront's part");
    FASTGL_LDS char *mine = (FASTGL_LDS char *)lds + wave * PARTB;
    const int64_t r_base = row0 + wm * 64;
    int64_t ldo = g.C;                                                   // elements between rows of the result
    if constexpr (MODE == kWeightsOne && !PART) ldo = g.ldo;
    // NB blocks of 32 columns from column c_base of the wavefront's 64 rows, element by element from value(i, block, e).
    auto store_block = [&](auto blocks, void *out, int64_t c_base, auto value) {
        constexpr int NB = decltype(blocks)::value, LPR = NB * 32 * OB / 16, PER = 16 / OB;      // lanes a row: PER elements each
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < T::TM; ++i)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = i * 32 + l32, col = b * 32 + 8 * q + 4 * h;
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = value(i, b, 4 * q + e);
                    const int piece = (col * OB / 16) ^ (row & 7), within = (col * OB) & 15;
                    FASTGL_LDS char *p = mine + row * ROWB + piece * 16 + within;
                    if constexpr (OB == 2) {
                        u32x2 o;
                        o[0] = pack_bf16(v[0], v[1]);
                        o[1] = pack_bf16(v[2], v[3]);
                        *(FASTGL_LDS u32x2 *)p = o;
                    } else {
                        u32x4 o;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(v[e]);
                        *(FASTGL_LDS u32x4 *)p = o;
                    }
                }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        typedef typename Words<OB>::x4 W4;
        constexpr int ROUNDS = 64 * LPR / kWave, ROWS = kWave / LPR;       // rows a round
        const int row = lane / LPR, c = lane % LPR;
        FASTGL_LDS char *from = mine + row * ROWB;
        auto piece = [&](int n) { return *(FASTGL_LDS u32x4 *)(from + n * ROWS * ROWB + ((c ^ ((row + n * ROWS) & 7)) * 16)); };
        OUT *base = static_cast<OUT *>(out) + r_base * ldo + c_base;
        if (r_base + 64 <= g.R && c_base + NB * 32 <= g.C) {              // all of it exists
            uint32_t o = (uint32_t)((row * ldo + c * PER) * OB);
            const uint32_t down = (uint32_t)(ROWS * ldo * OB);
#pragma unroll
            for (int n = 0; n < ROUNDS; ++n, o += down) {
                u32x4 v = piece(n);
                W4 *p = reinterpret_cast<W4 *>(reinterpret_cast<char *>(base) + o);
                if constexpr (MODE == kRowsAdd)
                    if (g.add) {
                        const W4 w = *p;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) + __uint_as_float(w[e]));
                    }
                if constexpr (ONCE) __builtin_nontemporal_store(W4{v[0], v[1], v[2], v[3]}, p);
                else *p = W4{v[0], v[1], v[2], v[3]};
            }
        } else {
            const int64_t left = g.C - c_base - c * PER;
            for (int n = 0; n < ROUNDS; ++n) {
                if (r_base + row + n * ROWS >= g.R || left <= 0) continue;
                u32x4 v = piece(n);
                OUT *p = base + (row + n * ROWS) * ldo + c * PER;
                if constexpr (MODE == kRowsAdd)
                    if (g.add) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (e < left) v[e] = __float_as_uint(__uint_as_float(v[e]) + p[e]);
                    }
                if (left >= PER) {
                    *reinterpret_cast<W4 *>(p) = W4{v[0], v[1], v[2], v[3]};
                } else {
#pragma unroll
                    for (int e = 0; e < PER - 1; ++e)
                        if (e < left) {
                            const uint32_t word = v[e * OB / 4];           // a copy: a bit cast of v[e] itself takes v[0]
                            if constexpr (OB == 2) p[e] = (uint16_t)(word >> (16 * (e & 1)));
                            else p[e] = __uint_as_float(word);
                        }
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    typedef std::integral_constant<int, ONE < 2 ? 1 : 2> NB;             // 64 columns at a time at most
    auto store_result = [&](int q, void *out, auto value) {               // value(i, block, e): of this result's blocks
#pragma unroll
        for (int n = 0; n < ONE; n += NB::value)
            store_block(NB(), out, col0 + (wn * ONE + n) * 32, [&](int i, int b, int e) { return value(i, n + b, e); });
    };
    if constexpr (MODE == kScores || MODE == kGradient) {
        loss_epilogue<MODE, T, ACT>(g, acc, r_base, col0 + wn * T::TN * 32, (row0 / T::BM) * T::WM + wm, (col0 / T::BC) * T::WN + wn);
    } else if constexpr (PART) {
#pragma unroll
        for (int q = 0; q < T::RESULTS; ++q)
            if (MODE == kForward || MODE == kRowsAdd || MODE == kWeightsOne || g.out[q])
                store_result(q, g.part + ((int64_t)slab * T::RESULTS + q) * g.R * g.C, [&](int i, int b, int e) { return acc[i][q * ONE + b][e]; });
    } else if constexpr (MODE == kForward) {
        if (g.out[1]) store_result(0, g.out[1], [&](int i, int b, int e) { return acc[i][b][e]; });
        if (g.out[2]) store_result(1, g.out[2], [&](int i, int b, int e) { return acc[i][ONE + b][e]; });
        store_result(0, g.out[0], [&](int i, int b, int e) { return gate<ACT, false, sizeof(OUT) == 2>(acc[i][b][e], nullptr) * acc[i][ONE + b][e]; });
    } else {
#pragma unroll
        for (int q = 0; q < T::RESULTS; ++q)
            if (g.out[q]) store_result(q, g.out[q], [&](int i, int b, int e) { return acc[i][q * ONE + b][e]; });
    }
#endif
}

}  // namespace
}  // namespace fastgl
