// Softmax cross entropy of class scores that are not kept (fastgl_loss.h has the formulas): what is around the products of gated_tile.h.
//
//   forward   for a piece of the classes at a time: [operands packed] -> scores by tiles, of which maximum and sum of exponentials of some columns of
//             each row remain -> k_loss_join
//   backward  the same: [W packed] -> scores again, of which dZ remains (as the matrix cores take it: fp32 calls in three bf16
//             pieces, bf16 calls in two, or rounded to one for a caller who asks for that; with column sums)
//             -> dH += dZ W^T -> dW = H^T dZ -> k_loss_sum
//
// Small calls go another way, through k_loss_block: a workgroup has 32 rows and 64 classes, the scores in LDS, and all of a pass that these take part in.
//
// dZ of a bf16 call in two pieces, rounded to one (us, backward): 8192 rows 512 -> 65 536 2940, 1780; 16 384 rows 512 -> 1000 128, 89.  Rounded, dH and dW are
// 2.4e-3 of themselves off instead of 1.7e-3, which is their own rounding.
//
// The rows of H are packed once for all pieces of a backward pass, 0 where there is no label: dZ is 0 there, and what H holds there must not
// reach dW (0 times NaN).
#include <initializer_list>

#include "fastgl_loss.h"
#include "gated_tile.h"
#include "update_internal.h"

namespace fastgl {
namespace {

constexpr int64_t kMostClasses = (int64_t)1 << 21, kMostInputs = (int64_t)1 << 20;
// dZ, and packed weights, of a piece of the classes.  8192 rows 512 -> 65 536 bf16, dZ rounded, the kernels of a backward pass: 256 MiB (four pieces) 1953 us, 512 MiB
// 1783, 1 GiB (one) 1720: fewer sums of pieces, although dZ no longer stays in the last cache.
constexpr int64_t kPieceBytes = (int64_t)1 << 30;
constexpr int kPieceCols = 256;                           // one of several pieces has a multiple of them

// ------------------------------------------------------------------ packing
// Matrices [rows][cols] (rows ld_src apart) as planes of bf16 with rows of ld elements, 0 beyond cols and in rows whose label is negative.
struct LossPackArgs {
    const void *src[2];
    uint16_t *out[2];
    const int64_t *label[2];
    int64_t rows[2], ld_src[2], end[2];      // end: elements from src to the array's end
    int32_t cols[2], ld[2];
};

template <bool BF16>
__global__ __launch_bounds__(kBlock) void k_loss_pack(LossPackArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    const int m = blockIdx.y;
    const T *src = static_cast<const T *>(m ? a.src[1] : a.src[0]);
    uint16_t *out = m ? a.out[1] : a.out[0];
    const int64_t *label = m ? a.label[1] : a.label[0];
    const int64_t rows = m ? a.rows[1] : a.rows[0], ld_src = m ? a.ld_src[1] : a.ld_src[0], end = m ? a.end[1] : a.end[0];
    const int32_t cols = m ? a.cols[1] : a.cols[0], ld = m ? a.ld[1] : a.ld[0], chunks = ld / kChunk;
    const int64_t n = rows * chunks;
    for (int64_t u = (int64_t)blockIdx.x * kBlock + threadIdx.x; u < n; u += (int64_t)gridDim.x * kBlock) {
        const int64_t row = u / chunks;
        const int col = (int)(u - row * chunks) * kChunk, left = cols - col;
        const int64_t at = row * ld_src + col;
        Chunk<BF16> c;
        float v[8];
        c.load(src + at, left > 0 && at + kChunk <= end ? kChunk : left);
        const bool on = !label || label[row] >= 0;
        c.get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = on && j < left ? v[j] : 0.f;
        uint16_t *to = out + row * ld + col;
        Chunk<true>::store(to, v, 8);
        if constexpr (!BF16) {
#pragma unroll
            for (int p = 1; p < 3; ++p) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] -= (float)(__bf16)v[j];
                Chunk<true>::store(to + p * rows * ld, v, 8);
            }
        }
    }
}

// ------------------------------------------------------------------ joining
// A row's maxima and sums from all column tiles of a piece of the classes and what the pieces before left (before, or NULL), 2^lg rows and as many
// threads a row as are left; after: not the last piece, the row's pair goes there.
__global__ __launch_bounds__(kBlock) void k_loss_join(const float *stats, int64_t slots, const float *before, float *after, const float *picked,
                                                      const int64_t *label, int64_t M, int64_t N, int lg, float *loss, float *lse)
{
    constexpr float kLog2e = 1.44269504089f, kLn2 = 0.69314718056f;
    __shared__ float most[kBlock], sums[kBlock];
    const int parts = kBlock >> lg, part = threadIdx.x >> lg, r = threadIdx.x & ((1 << lg) - 1);
    const int64_t row = ((int64_t)blockIdx.x << lg) + r;
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 *p = reinterpret_cast<const f2 *>(stats) + (row < M ? row : M - 1);
    float m = -INFINITY, s = 0.f;
    if (before && part == 0 && row < M) {
        const f2 x = reinterpret_cast<const f2 *>(before)[row];
        m = x[0];
        s = x[1];
    }
#pragma unroll 4
    for (int64_t t = part; t < slots; t += parts) {
        const f2 x = p[t * M];
        const float next = fmaxf(m, x[0]), base = next == -INFINITY ? 0.f : next;
        s = s * __builtin_amdgcn_exp2f((m - base) * kLog2e) + x[1] * __builtin_amdgcn_exp2f((x[0] - base) * kLog2e);
        m = next;
    }
    most[threadIdx.x] = m;
    sums[threadIdx.x] = s;
    __syncthreads();
    if (part != 0 || row >= M) return;
    for (int q = 1; q < parts; ++q) m = fmaxf(m, most[(q << lg) + r]);
    const float base = m == -INFINITY ? 0.f : m;
    s = 0.f;
    for (int q = 0; q < parts; ++q) s += sums[(q << lg) + r] * __builtin_amdgcn_exp2f((most[(q << lg) + r] - base) * kLog2e);
    if (after) {
        reinterpret_cast<f2 *>(after)[row] = f2{m, s};
        return;
    }
    const float all = m == -INFINITY && s == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(s) * kLn2;
    if (lse) lse[row] = all;
    const int64_t y = label[row];
    loss[row] = y < 0 ? 0.f : y >= N ? NAN : all - picked[row];
}

// ------------------------------------------------------------------ sums of slabs, column sums
struct LossSumArgs {
    const float *part;               // slab s at part + s * R * C, or NULL
    void *out;                       // rows ldo apart
    int64_t R, C, ldo;
    int32_t slabs;
    int32_t blocks;                  // workgroups of the slabs, before those of the columns
    const float *db_part;            // [db_rows][db_cols], or NULL
    float *db;
    int32_t db_rows, db_cols;
};

template <bool BF16>
__global__ __launch_bounds__(kBlock) void k_loss_sum(LossSumArgs a)
{
    if ((int)blockIdx.x < a.blocks) {
        const int64_t n = a.R * a.C;
        for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t)a.blocks * kBlock) {
            double v = 0.0;
#pragma unroll 8
            for (int s = 0; s < a.slabs; ++s) v += (double)a.part[(int64_t)s * n + i];
            const int64_t row = i / a.C, to = row * a.ldo + (i - row * a.C);
            if constexpr (BF16) static_cast<uint16_t *>(a.out)[to] = __builtin_bit_cast(uint16_t, (__bf16)(float)v);
            else static_cast<float *>(a.out)[to] = (float)v;
        }
        return;
    }
    __shared__ double sums[kBlock / 8][9];                             // eight columns, 32 threads a column
    const int c = threadIdx.x & 7, r = threadIdx.x >> 3;
    const int64_t col = ((int64_t)blockIdx.x - a.blocks) * 8 + c;
    double v = 0.0;
    if (col < a.db_cols) {
#pragma unroll 8
        for (int i = r; i < a.db_rows; i += kBlock / 8) v += (double)a.db_part[(int64_t)i * a.db_cols + col];
    }
    sums[r][c] = v;
    __syncthreads();
    if (r == 0 && col < a.db_cols) {
        v = 0.0;
        for (int i = 0; i < kBlock / 8; ++i) v += sums[i][c];
        a.db[col] = (float)v;
    }
}

// ------------------------------------------------------------------ small calls
// 32 rows and 64 classes a workgroup, with fp32 matrix instructions from rows and weights as they lie in memory: nothing is packed, dZ stays
// in LDS and is not rounded.
//   scores  the wavefronts take eight inputs each in turn; their sums are joined in LDS, where the tile then has its statistics or dZ
//   dH      32 inputs a wavefront at a time: sums over the tile's classes, one for each strip of classes, joined afterwards
//   dW      the same over the tile's rows
// COARSE: dH and dW are of dZ rounded to one bf16, as the caller asked for.
struct LossBlockArgs {
    const void *H, *W;
    const float *b;
    const int64_t *label;
    const float *lse_in, *dloss;
    int64_t M, N;
    int32_t K;
    float *loss, *lse;             // forward, one strip
    float *stats, *picked;         // forward, several
    void *dH, *dW;                 // or NULL
    float *db;
    float *part_h, *part_w, *part_b;       // [strip][M][K], [tile][K][N], [tile][N]; NULL: results go where they belong
};

constexpr int kBlockRows = 32, kBlockCols = 64, kPad = 68;
constexpr int kAddThreads = 1024, kAddLg = 10;

// Elements by 32-bit offsets: arrays of small calls have fewer than 2^27 elements.
template <bool BF16>
__device__ __forceinline__ float element(const void *p, uint32_t i)
{
    if constexpr (BF16) return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(static_cast<const char *>(p) + 2 * i) << 16);
    else return *reinterpret_cast<const float *>(static_cast<const char *>(p) + 4 * i);
}

// Four elements from i on, at any alignment to an element.
template <bool BF16>
__device__ __forceinline__ void four(const void *p, uint32_t i, float (&v)[4])
{
    if constexpr (BF16) {
        const Words<2>::x2 q = *reinterpret_cast<const Words<2>::x2 *>(static_cast<const char *>(p) + 2 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(j & 1 ? q[j >> 1] & 0xFFFF0000u : q[j >> 1] << 16);
    } else {
        const Words<4>::x4 q = *reinterpret_cast<const Words<4>::x4 *>(static_cast<const char *>(p) + 4 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(q[j]);
    }
}

template <bool BF16>
__device__ __forceinline__ void put_result(void *out, float *part, uint32_t at, float x)
{
    if (part) *reinterpret_cast<float *>(reinterpret_cast<char *>(part) + 4 * at) = x;
    else if constexpr (BF16) *reinterpret_cast<uint16_t *>(static_cast<char *>(out) + 2 * at) = __builtin_bit_cast(uint16_t, (__bf16)x);
    else *reinterpret_cast<float *>(static_cast<char *>(out) + 4 * at) = x;
}

template <bool BF16, bool BACKWARD, int THREADS, bool COARSE>
__global__ __launch_bounds__(THREADS) void k_loss_block(LossBlockArgs a)
{
    constexpr float kLog2e = 1.44269504089f, kLn2 = 0.69314718056f;
    constexpr int WAVES = THREADS / kWave, PER = THREADS / kBlockRows, CE = kBlockCols / PER;      // threads a row, columns of each
    __shared__ float z[WAVES][kBlockRows][kPad];
    __shared__ float on[kBlockRows];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r = lane & 31, h = lane >> 5;
    const int strip = blockIdx.x, tile = blockIdx.y;
    const int64_t col0 = (int64_t)strip * kBlockCols;
    const int left = (int)(a.N - col0 < kBlockCols ? a.N - col0 : kBlockCols);
    const uint32_t N = (uint32_t)a.N, K = (uint32_t)a.K;
    uint32_t col[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) col[q] = (uint32_t)col0 + (32 * q + r < left ? 32 * q + r : left - 1);        // columns that do not exist are not used
    float *part_h = a.part_h ? a.part_h + (int64_t)strip * a.M * a.K : nullptr, *part_w = a.part_w ? a.part_w + (int64_t)tile * a.K * a.N : nullptr;
    const int64_t row0 = (int64_t)tile * kBlockRows;
    const int rows = (int)(a.M - row0 < kBlockRows ? a.M - row0 : kBlockRows);
    // ---- scores
    f32x16 acc[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[0][e] = acc[1][e] = 0.f;
    const uint32_t first = (uint32_t)row0 * K, my_row = first + (uint32_t)(r < rows ? r : rows - 1) * K;
    const int whole = a.K & ~7;
#pragma unroll 2
    for (int k = wave * 8; k < whole; k += WAVES * 8) {
        float x[4], w[2][4];
        four<BF16>(a.H, my_row + k + 4 * h, x);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 2; ++q) w[q][j] = element<BF16>(a.W, (uint32_t)(k + 4 * h + j) * N + col[q]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 2; ++q) acc[q] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], w[q][j], acc[q], 0, 0, 0);
    }
    if (whole < a.K && wave == (whole / 8) % WAVES) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = whole + 4 * h + j;
            const bool in = k < a.K;
            const float x = in ? element<BF16>(a.H, my_row + k) : 0.f;
#pragma unroll
            for (int q = 0; q < 2; ++q)
                acc[q] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, in ? element<BF16>(a.W, (uint32_t)k * N + col[q]) : 0.f, acc[q], 0, 0, 0);
        }
    }
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int e = 0; e < 16; ++e) z[wave][8 * (e >> 2) + 4 * h + (e & 3)][32 * q + r] = acc[q][e];
    __syncthreads();
    // ---- statistics or dZ: some columns of a row each thread
    {
        const int row = threadIdx.x / PER, c0 = threadIdx.x % PER * CE;
        const int64_t label = row < rows ? a.label[row0 + row] : -1;
        const int mine = label >= col0 && label < col0 + left ? (int)(label - col0) - c0 : -1;       // of the label among these columns
        float v[CE];
#pragma unroll
        for (int c = 0; c < CE; ++c) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) s += z[i][row][c0 + c];
            if (a.b && c0 + c < left) s += a.b[col0 + c0 + c];
            v[c] = c0 + c < left ? s : -INFINITY;
        }
        if constexpr (!BACKWARD) {
            float most = -INFINITY, sum = 0.f, at = 0.f;
#pragma unroll
            for (int c = 0; c < CE; ++c) most = fmaxf(most, v[c]);
#pragma unroll
            for (int d = 1; d < PER; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, kWave));
            const float base = most == -INFINITY ? 0.f : most;
#pragma unroll
            for (int c = 0; c < CE; ++c) {
                sum += __builtin_amdgcn_exp2f((v[c] - base) * kLog2e);
                at = c == mine ? v[c] : at;
            }
#pragma unroll
            for (int d = 1; d < PER; d <<= 1) {
                sum += __shfl_xor(sum, d, kWave);
                at += __shfl_xor(at, d, kWave);
            }
            if (row < rows && c0 == 0) {
                if (a.stats) {
                    a.stats[2 * (strip * a.M + row0 + row)] = most;
                    a.stats[2 * (strip * a.M + row0 + row) + 1] = sum;
                    if (label >= col0 && label < col0 + left) a.picked[row0 + row] = at;
                } else {
                    const float all = most == -INFINITY && sum == 0.f ? -INFINITY : most + __builtin_amdgcn_logf(sum) * kLn2;
                    if (a.lse) a.lse[row0 + row] = all;
                    a.loss[row0 + row] = label < 0 ? 0.f : label >= a.N ? NAN : all - at;
                }
            }
        } else {
            const float lse = label >= 0 ? a.lse_in[row0 + row] : 0.f;
            const float scale = label >= a.N ? NAN : label >= 0 ? a.dloss[row0 + row] : 0.f;
#pragma unroll
            for (int c = 0; c < CE; ++c) {
                const float p = __builtin_amdgcn_exp2f((v[c] - lse) * kLog2e), x = c == mine ? p - 1.f : p;
                z[0][row][c0 + c] = label >= 0 && c0 + c < left ? x * scale : 0.f;
            }
            if (c0 == 0) on[row] = label >= 0 ? 1.f : 0.f;
        }
    }
    if constexpr (BACKWARD) {
        __syncthreads();
        float db = 0.f;
        if (a.db && threadIdx.x < kBlockCols) {
#pragma unroll 8
            for (int i = 0; i < kBlockRows; ++i) db += z[0][i][threadIdx.x];
        }
        auto dz = [&](int row, int c) __attribute__((always_inline)) { return COARSE ? (float)(__bf16)z[0][row][c] : z[0][row][c]; };
        // ---- dH
        auto rows_of = [&](int k0) __attribute__((always_inline)) {
            const int k = k0 + r;
            const uint32_t w0 = (uint32_t)(k < a.K ? k : a.K - 1) * N + (uint32_t)col0;
            f32x16 out;
#pragma unroll
            for (int e = 0; e < 16; ++e) out[e] = 0.f;
            auto eight = [&](int c, const float (&w)[4]) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) out = __builtin_amdgcn_mfma_f32_32x32x2f32(dz(r, 8 * c + 4 * h + j), w[j], out, 0, 0, 0);
            };
            if (left == kBlockCols) {
                float w[8][4];
#pragma unroll
                for (int c = 0; c < 8; ++c) four<BF16>(a.W, w0 + 8 * c + 4 * h, w[c]);
#pragma unroll
                for (int c = 0; c < 8; ++c) eight(c, w[c]);
            } else
                for (int c = 0; 8 * c < left; ++c) {
                    float w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = 8 * c + 4 * h + j < left ? element<BF16>(a.W, w0 + 8 * c + 4 * h + j) : 0.f;
                    eight(c, w);
                }
            if (k < a.K) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int row = 8 * (e >> 2) + 4 * h + (e & 3);
                    if (row < rows) put_result<BF16>(a.dH, part_h, first + (uint32_t)row * K + (uint32_t)k, out[e]);
                }
            }
        };
        // ---- dW, of NQ times 32 classes from q0 on
        auto weights_of = [&](int k0, int q0, auto nq) __attribute__((always_inline)) {
            constexpr int NQ = decltype(nq)::value;
            f32x16 out[NQ];
#pragma unroll
            for (int q = 0; q < NQ; ++q)
#pragma unroll
                for (int e = 0; e < 16; ++e) out[q][e] = 0.f;
            const int k = k0 + r < a.K ? k0 + r : a.K - 1;
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int row = 8 * (i >> 2) + 4 * h + (i & 3);
                x[i] = element<BF16>(a.H, first + (uint32_t)(row < rows ? row : rows - 1) * K + (uint32_t)k);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int row = 8 * (i >> 2) + 4 * h + (i & 3);
                const float v = on[row] != 0.f ? x[i] : 0.f;                   // rows without a label: whatever they hold
#pragma unroll
                for (int q = 0; q < NQ; ++q) out[q] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, dz(row, 32 * (q0 + q) + r), out[q], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);    // one block's rows in registers at a time
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                if (32 * (q0 + q) + r >= left) continue;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int to = k0 + 8 * (e >> 2) + 4 * h + (e & 3);
                    if (to < a.K) put_result<BF16>(a.dW, part_w, (uint32_t)to * N + (uint32_t)col0 + 32 * (q0 + q) + r, out[q][e]);
                }
            }
        };
        // Blocks of 32 inputs are dealt to the wavefronts; where there are fewer of them, dH and each half of the classes of dW by themselves.  us, all of a block to
        // one wavefront / so: 15 507 rows 11 -> 10 080, f32, 819 / 654;  24 241 rows 31 -> 1548 259 / 221;  8000 rows 16 -> 7 11.8 / 10.3.
        const int blocks = (a.K + 31) / 32;
        if (blocks >= WAVES) {
            if (a.dH)
                for (int k = wave; k < blocks; k += WAVES) rows_of(32 * k);
            if (a.dW)
                for (int k = wave; k < blocks; k += WAVES) weights_of(32 * k, 0, std::integral_constant<int, 2>());
        } else
            for (int job = wave; job < 3 * blocks; job += WAVES) {
                if (job < blocks) {
                    if (a.dH) rows_of(32 * job);
                } else if (a.dW)
                    weights_of(32 * ((job - blocks) >> 1), (job - blocks) & 1, std::integral_constant<int, 1>());
            }
        if (a.db && threadIdx.x < (unsigned)left) {
            if (a.part_b) a.part_b[(int64_t)tile * a.N + col0 + threadIdx.x] = db;
            else a.db[col0 + threadIdx.x] = db;
        }
    }
}

// The sums of small calls: up to three results of n elements from so many parts each, 2^lg elements a workgroup and as many threads an element
// as are left, in fp64 and a fixed order.
struct LossAddArgs {
    const float *part[3];
    void *out[3];
    int64_t n[3], blocks[3];
    int32_t parts[3], lg[3], bf16[3];
};

__global__ __launch_bounds__(kAddThreads) void k_loss_add(LossAddArgs a)
{
    __shared__ double sums[kAddThreads];
    int64_t block = blockIdx.x;
    int m = 0;
    for (; m < 2 && block >= a.blocks[m]; ++m) block -= a.blocks[m];
    const float *part = m == 0 ? a.part[0] : m == 1 ? a.part[1] : a.part[2];
    void *out = m == 0 ? a.out[0] : m == 1 ? a.out[1] : a.out[2];
    const int64_t n = m == 0 ? a.n[0] : m == 1 ? a.n[1] : a.n[2];
    const int parts = m == 0 ? a.parts[0] : m == 1 ? a.parts[1] : a.parts[2], lg = m == 0 ? a.lg[0] : m == 1 ? a.lg[1] : a.lg[2];
    const int bf16 = m == 0 ? a.bf16[0] : m == 1 ? a.bf16[1] : a.bf16[2];
    const int c = threadIdx.x & ((1 << lg) - 1), t = threadIdx.x >> lg, threads = kAddThreads >> lg;
    const int64_t i = (block << lg) + c;
    double v = 0.0;
    if (i < n) {
#pragma unroll 8
        for (int s = t; s < parts; s += threads) v += (double)part[(int64_t)s * n + i];
    }
    if (threads > 1) {
        sums[threadIdx.x] = v;
        __syncthreads();
        for (int d = threads / 2; d > 0; d >>= 1) {
            if (t < d) sums[threadIdx.x] += sums[threadIdx.x + (d << lg)];
            __syncthreads();
        }
        v = sums[threadIdx.x];
    }
    if (t != 0 || i >= n) return;
    if (bf16) static_cast<uint16_t *>(out)[i] = __builtin_bit_cast(uint16_t, (__bf16)(float)v);
    else static_cast<float *>(out)[i] = (float)v;
}

// ------------------------------------------------------------------ host side
bool misaligned_to(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

struct Shape {
    bool bf16, backward, pack_h, pack_w;
    int planes, z_planes;          // of H and W, of dZ
    int64_t M, K, N, ldk, pairs, z_pairs;
    Shape(fastgl_dtype dtype, int64_t M_, int64_t K_, int64_t N_, bool aligned, bool backward_, bool coarse)
        : bf16(dtype == FASTGL_BF16), backward(backward_), pack_h(backward_ || !bf16 || !aligned || K_ % 8), pack_w(!bf16 || !aligned || N_ % 8),
          planes(bf16 ? 1 : 3), z_planes(!bf16 ? 3 : coarse ? 1 : 2), M(M_), K(K_), N(N_), ldk((int64_t)align_up((size_t)K_, 8)), pairs(bf16 ? 1 : 6),
          z_pairs(bf16 ? z_planes : 6)
    {
    }
    int64_t rows() const { return (int64_t)align_up((size_t)M, 256); }
    // Classes of a piece: dZ, a forward pass's statistics (8 bytes for 64 classes of a row at most) and packed weights stay below kPieceBytes, the
    // pieces are of one size.
    int64_t piece() const
    {
        int64_t most = backward ? kPieceBytes / (2 * z_planes * rows()) : kPieceBytes / 8 * 64 / M;
        if (pack_w && K > 0 && kPieceBytes / (2 * planes * K) < most) most = kPieceBytes / (2 * planes * K);
        if (most >= N) return (int64_t)align_up((size_t)N, 32);            // the columns of dZ that are written and read
        most = most < 2 * kPieceCols ? kPieceCols : most / kPieceCols * kPieceCols;
        return (int64_t)align_up((size_t)ceil_div(N, ceil_div(N, most)), kPieceCols);
    }
    int64_t pieces() const { return ceil_div(N, piece()); }
    int64_t widest() const { return piece() < N ? piece() : N; }          // columns that exist of the largest piece
    // dZ in blocks of 32 columns, [block][row][32], a block 2304 bytes more than a multiple of 4096 (the gated update's layout and reasons);
    // rows lie whole where eight blocks pass 32-bit offsets.
    bool blocks() const { return M <= (int64_t)1 << 21; }
    int64_t z_block() const { return blocks() ? (int64_t)(align_up((size_t)rows() * 64, 4096) + 2304) / 2 : 32; }
    int64_t z_ld() const { return blocks() ? 32 : piece(); }
    int64_t z_plane() const { return blocks() ? piece() / 32 * z_block() : rows() * piece(); }
    Cut scores_cut() const { return cut_of(kForward, M, widest(), K, pairs, true, true); }
    Cut rows_cut() const { return cut_of(kRows, M, K, widest(), z_pairs); }
    Cut weights_cut() const { return cut_of(kWeights, K, widest(), M, z_pairs, true); }
    static int64_t tile_rows(const Cut &c) { return c.size == kLarge ? 256 : 128; }
    static int64_t wave_cols(const Cut &c) { return c.size == kSmall ? 64 : 128; }
    int64_t slots() const { return ceil_div(widest(), wave_cols(scores_cut())); }      // of statistics: column tiles and wavefronts of a piece
    int64_t db_rows() const { return ceil_div(M, tile_rows(scores_cut())) * (scores_cut().size == kLarge ? 4 : 2); }
    bool parts_h() const { return pieces() > 1 || rows_cut().slabs > 1; }

    // ---- k_loss_block
    int64_t tiles() const { return ceil_div(M, kBlockRows); }
    int64_t strips() const { return ceil_div(N, kBlockCols); }
    // Whether every workgroup has a compute unit to itself: twice the wavefronts then, which share what one waits for.  us a backward pass, f32, 256
    // threads / 512: 1 row 256 -> 47 15.8 / 12.6;  8000 rows 256 -> 47 27.6 / 24.7;  300 rows 500 -> 464 35.5 / 31.1;  with more workgroups 4000 rows
    // 64 -> 1000 48 / 60.
    bool one_each() const { return tiles() * strips() <= 256; }
    // Whether k_loss_block is taken: a model of both ways, in us, that the sizes go into as they are padded.  In a forward pass a workgroup of it costs
    // 1.4 us and 0.009 us an input, four at a time a compute unit.  A backward pass is one workgroup's chain, or 6 M N K multiply-adds at 110 TFLOP/s, and
    // the launch of its sums, written and read.  The other way costs its launches, the steps of one tile where there are few, the products at what they
    // reach, and dZ and packed rows at 4 (bf16: 5) TB/s.  us a call, k_loss_block / tiles (bf16 backward: dZ in two pieces; rounded 24 241 rows 229 / 76):
    //                                 f32 forward   f32 backward  bf16 forward  bf16 backward
    //       1 row  256 ->     47       6.5 / 36      12.8 / 42      6.4 / 20      14.8 / 21.4
    //    8000 rows 256 ->     47       7.0 / 35        25 / 71      6.9 / 13      26.4 / 36.3
    //    8000 rows 512 ->     47      10.5 / 64        38 / 92      9.2 / 17      43.3 / 46.1
    //  70 000 rows 256 ->     47        41 / 88       112 / 255    31.5 / 22       118 / 103
    //      16 rows 512 -> 50 000        35 / 92        81 / 182      34 / 18        81 / 65
    //     512 rows 256 ->   1000                                                  29.5 / 37.1
    //  20 000 rows 128 ->     60                                                  34.0 / 43.8
    //    1645 rows 1070 ->  2113        90 / 145      614 / 277      82 / 38       584 / 105
    //     667 rows  25 -> 18 287        34 / 21        73 / 92       34 / 16        75 / 55
    //  24 241 rows  31 ->   1548       101 / 39       221 / 220      95 / 26       226 / 115
    //  16 384 rows 512 ->   1000       183 / 100     1130 / 341     169 / 24      1047 / 128
    bool small() const
    {
        if (tiles() > 65535 || K * N >= (int64_t)1 << 27 || M * K >= (int64_t)1 << 27) return false;      // its grid and offsets
        const double groups = (double)(tiles() * strips()), k = (double)K, m = (double)M;
        const double all = (double)align_up((size_t)M, 128) * (double)align_up((size_t)N, 128) * (double)align_up((size_t)K, 128);
        if (!backward) {
            const double one = 0.015 * k, many = groups / 256.0 * (1.43 + 0.0094 * k);
            const double here = 4.5 + (strips() > 1 ? 3.2 : 0.0) + (one > many ? one : many);
            const double there = bf16 ? 9.5 + (pack_h || pack_w ? 4.0 : 0.0) + 0.006 * k + all * 2.0 / 0.6e9 : 15.0 + 0.085 * k + all * 2.0 / 0.17e9;
            return here < there;
        }
        const double sums = 4.0 * ((tiles() > 1 ? (double)tiles() * k * (double)N : 0.0) + (strips() > 1 ? (double)strips() * m * k : 0.0));
        if (sums > 512e6) return false;
        const double here = ((one_each() ? 4.0 + 0.034 * k : 10.0 + 0.035 * k + groups * (0.004 + 6.0 * kBlockRows * kBlockCols * k / 110e6)) +
                             (sums > 0.0 ? 4.5 + 2.0 * sums / (one_each() ? 4e6 : 5e6) : 0.0)) * (!bf16 ? 1.0 : one_each() ? 1.15 : 1.08);
        const double z = m * (double)align_up((size_t)N, 32);
        const double there = z_planes == 1   ? 23.0 + 0.015 * k + all * 6.0 / 0.6e9 + (10.0 * z + 8.0 * m * k) / 5e6
                             : z_planes == 2 ? 27.5 + 0.024 * k + all * 10.0 / 0.8e9 + (10.0 * z + 8.0 * m * k) / 5e6
                                             : 40.0 + 0.06 * k + all * 6.0 / 0.2e9 + (18.0 * z + 12.0 * m * k) / 4e6;
        return here < there;
    }
};

struct Scratch {
    size_t used = 0;
    char *base;
    uint16_t *h, *w, *dz;
    float *stats, *picked, *joined, *db, *part_h, *part_w;
    template <class T>
    T *take(size_t n)
    {
        char *p = base ? base + used : nullptr;
        used += align_up(n * sizeof(T), 256);
        return reinterpret_cast<T *>(p);
    }
    Scratch(const Shape &s, char *at) : base(at)
    {
        h = w = dz = nullptr;
        stats = picked = joined = db = part_h = part_w = nullptr;
        if (s.small()) {
            if (!s.backward && s.strips() > 1) {
                stats = take<float>((size_t)(2 * s.strips() * s.M));
                picked = take<float>((size_t)s.M);
            }
            if (s.backward && s.strips() > 1) part_h = take<float>((size_t)(s.strips() * s.M * s.K));
            if (s.backward && s.tiles() > 1) {
                part_w = take<float>((size_t)(s.tiles() * s.K * s.N));
                db = take<float>((size_t)(s.tiles() * s.N));
            }
            return;
        }
        if (s.pack_h) h = take<uint16_t>((size_t)(s.planes * s.M * s.ldk));
        if (s.pack_w) w = take<uint16_t>((size_t)(s.planes * s.K * s.piece()));
        if (!s.backward) {
            stats = take<float>((size_t)(2 * s.slots() * s.M));
            picked = take<float>((size_t)s.M);
            if (s.pieces() > 1) joined = take<float>((size_t)(2 * s.M));
            return;
        }
        dz = take<uint16_t>((size_t)(s.z_planes * s.z_plane()));
        db = take<float>((size_t)(s.db_rows() * s.widest()));
        if (s.parts_h()) part_h = take<float>((size_t)(s.rows_cut().slabs * s.M * s.K));
        const Cut c = s.weights_cut();
        if (c.slabs > 1) part_w = take<float>((size_t)(c.slabs * s.K * s.widest()));
    }
};

fastgl_status check(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N)
{
    if (dtype != FASTGL_F32 && dtype != FASTGL_BF16) {
        set_error("bad dtype %d", (int)dtype);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (M < 0 || K < 0 || N < 0 || (M > 0 && N == 0)) {
        set_error("negative size, or rows without classes (M=%lld K=%lld N=%lld)", (long long)M, (long long)K, (long long)N);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (M > kMaxIndex || K > kMostInputs || N > kMostClasses) {
        set_error("M must stay below 2^31-1-1024, K at 2^20 and N at 2^21 or below");
        return FASTGL_ERR_UNSUPPORTED;
    }
    return FASTGL_OK;
}

fastgl_status check_workspace(const void *ws, size_t bytes, size_t need)
{
    if (need == 0) return FASTGL_OK;
    if (!ws || misaligned_to(ws, 256)) {
        set_error("workspace must be a 256-byte aligned device buffer");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (bytes < need) {
        set_error("workspace too small: %zu < %zu bytes", bytes, need);
        return FASTGL_ERR_WORKSPACE;
    }
    return FASTGL_OK;
}

size_t workspace(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, bool aligned, bool backward, bool coarse = false)
{
    if (check(dtype, M, K, N) != FASTGL_OK || M == 0) return 0;
    const size_t whole = Scratch(Shape(dtype, M, K, N, true, backward, coarse), nullptr).used;
    if (aligned) return whole;
    const size_t any = Scratch(Shape(dtype, M, K, N, false, backward, coarse), nullptr).used;
    return any > whole ? any : whole;
}

// A small call: one launch, and one for the sums of several strips or workgroups a strip.
fastgl_status launch_block(const Shape &d, LossBlockArgs a, hipStream_t s, const char *what)
{
    a.M = d.M; a.N = d.N;
    a.K = (int32_t)d.K;
    const dim3 grid((unsigned)d.strips(), (unsigned)d.tiles());
    auto typed = [&](auto bf16, auto threads) {
        constexpr bool B = decltype(bf16)::value;
        constexpr int T = decltype(threads)::value;
        if (!d.backward) hipLaunchKernelGGL((k_loss_block<B, false, T, false>), grid, dim3(T), 0, s, a);
        else if (B && d.z_planes == 1) hipLaunchKernelGGL((k_loss_block<B, true, T, B>), grid, dim3(T), 0, s, a);
        else hipLaunchKernelGGL((k_loss_block<B, true, T, false>), grid, dim3(T), 0, s, a);
    };
    auto sized = [&](auto bf16) {
        if (d.one_each()) typed(bf16, std::integral_constant<int, 512>());
        else typed(bf16, std::integral_constant<int, 256>());
    };
    if (d.bf16) sized(std::true_type());
    else sized(std::false_type());
    FASTGL_LAUNCH_CHECK(what);
    return FASTGL_OK;
}

fastgl_status launch_join(const Scratch &o, int64_t slots, bool first, bool last, const int64_t *label, int64_t M, int64_t N, float *loss, float *lse, hipStream_t s)
{
    int lg = 0;
    while ((lg < 5 && ((int64_t)1 << lg) < M) || (lg < 8 && M >> lg >= (int64_t)1 << 22)) ++lg;       // a launch has less than 2^32 threads
    hipLaunchKernelGGL(k_loss_join, dim3((unsigned)ceil_div(M, (int64_t)1 << lg)), dim3(kBlock), 0, s, (const float *)o.stats, slots,
                       first ? nullptr : (const float *)o.joined, last ? nullptr : o.joined, (const float *)o.picked, label, M, N, lg, loss, lse);
    FASTGL_LAUNCH_CHECK("fastgl_loss_fwd (rows)");
    return FASTGL_OK;
}

// What of H and of classes n0 .. n0 + n of W a call needs packed, in one launch.
fastgl_status pack(const Shape &d, const Scratch &o, const void *H, const void *W, const int64_t *label, int64_t n0, int64_t n, bool h, bool w, hipStream_t s)
{
    const int64_t el = d.bf16 ? 2 : 4;
    LossPackArgs a = {};
    int m = 0;
    int64_t most = 0;
    auto add = [&](const void *src, uint16_t *out, const int64_t *on, int64_t rows, int64_t cols, int64_t ld_src, int64_t end, int64_t ld) {
        if (rows == 0 || cols == 0) return;
        a.src[m] = src;
        a.out[m] = out;
        a.label[m] = on;
        a.rows[m] = rows; a.ld_src[m] = ld_src; a.end[m] = end;
        a.cols[m] = (int32_t)cols; a.ld[m++] = (int32_t)ld;
        if (rows * (ld / kChunk) > most) most = rows * (ld / kChunk);
    };
    if (h) add(H, o.h, d.backward ? label : nullptr, d.M, d.K, d.K, d.M * d.K, d.ldk);
    if (w) add(static_cast<const char *>(W) + n0 * el, o.w, nullptr, d.K, n, d.N, d.K * d.N - n0, (int64_t)align_up((size_t)n, 8));
    if (m == 0) return FASTGL_OK;
    const int64_t blocks = ceil_div(most, kBlock);
    const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384), (unsigned)m);
    if (d.bf16) hipLaunchKernelGGL(k_loss_pack<true>, grid, dim3(kBlock), 0, s, a);
    else hipLaunchKernelGGL(k_loss_pack<false>, grid, dim3(kBlock), 0, s, a);
    FASTGL_LAUNCH_CHECK("fastgl_loss (pack)");
    return FASTGL_OK;
}

// One product.  PART: sums of slabs.  PLANES: of dZ.
template <int MODE, bool PART, int PLANES = 0>
fastgl_status launch(const LossTileArgs &args, const Cut &cut, bool bf16, hipStream_t s, const char *what)
{
    typename TileArgsOf<MODE>::type g = args;
    const int64_t tr = ceil_div(g.R, Shape::tile_rows(cut)), tc = ceil_div(g.C, cut.size == kSmall ? 128 : 256), total = tr * tc * cut.slabs;
    if (total > (int64_t)UINT32_MAX / (cut.size == kLarge ? Tile<MODE, kLarge>::THREADS : Tile<MODE, kSmall>::THREADS) || 4 * tc > 0x7FFFFFFFLL) {
        set_error("%s: too many tiles (%lld)", what, (long long)total);
        return FASTGL_ERR_UNSUPPORTED;
    }
    g.tiles_r = (int32_t)tr;
    g.tiles_c = (int32_t)tc;
    g.slabs = (int32_t)cut.slabs;
    auto sized = [&](auto size) {
        constexpr int S = decltype(size)::value;
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)total), dim3(Tile<MODE, S>::THREADS), 0, s, g); };
        if constexpr (PART || MODE == kScores || MODE == kGradient) go(k_gated_tile<MODE, S, float, PLANES, PART, false>);
        else if (bf16) go(k_gated_tile<MODE, S, uint16_t, 0, false, false>);
        else go(k_gated_tile<MODE, S, float, 0, false, false>);
    };
    if (cut.size == kLarge) sized(std::integral_constant<int, kLarge>());
    else if (cut.size == kMiddle) sized(std::integral_constant<int, kMiddle>());
    else sized(std::integral_constant<int, kSmall>());
    FASTGL_LAUNCH_CHECK(what);
    return FASTGL_OK;
}

fastgl_status launch_sum(LossSumArgs a, bool bf16, hipStream_t s, const char *what)
{
    const int64_t blocks = a.part ? ceil_div(a.R * a.C, kBlock) : 0, most = (int64_t)1 << 20;        // a launch has less than 2^32 threads
    a.blocks = (int32_t)(blocks < most ? blocks : most);
    const dim3 grid((unsigned)(a.blocks + (a.db_part ? ceil_div((int64_t)a.db_cols, 8) : 0)));
    if (bf16) hipLaunchKernelGGL(k_loss_sum<true>, grid, dim3(kBlock), 0, s, a);
    else hipLaunchKernelGGL(k_loss_sum<false>, grid, dim3(kBlock), 0, s, a);
    FASTGL_LAUNCH_CHECK(what);
    return FASTGL_OK;
}

// The scores' product of classes n0 .. n0 + n.
LossTileArgs scores_of(const Shape &d, const Scratch &o, const void *H, const void *W, const float *b, const int64_t *label, int64_t n0, int64_t n)
{
    LossTileArgs g = {};
    g.a[0] = d.pack_h ? o.h : (const uint16_t *)H;
    g.b[0] = d.pack_w ? o.w : (const uint16_t *)W;
    g.lda = d.ldk;
    g.ldb = d.pack_w ? (int64_t)align_up((size_t)n, 8) : d.N;
    g.shift = d.pack_w ? 0 : n0;
    g.a_plane = d.M * d.ldk; g.b_plane = d.K * g.ldb;
    g.R = d.M; g.C = n; g.Kc = d.K;
    g.pairs = (int32_t)d.pairs; g.groups = 1;
    if (!d.bf16) {
        g.planes_a = kSixA;
        g.planes_b = kSixB;
    }
    g.bias[0] = b ? b + n0 : nullptr;
    g.label = label;
    g.first = n0; g.classes = d.N;
    return g;
}

bool starts_whole(std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if (misaligned_to(p, 16)) return false;
    return true;
}

fastgl_status loss_bwd(bool coarse, fastgl_dtype dtype, const void *H, const void *W, const float *b, const int64_t *label, const float *lse,
                       const float *dloss, int64_t M, int64_t K, int64_t N, void *dH, void *dW, float *db, void *ws, size_t ws_bytes, void *stream)
{
    fastgl_status st = check(dtype, M, K, N);
    if (st != FASTGL_OK) return st;
    const bool want_h = dH && M > 0 && K > 0, want_w = dW && K > 0 && N > 0, want_b = db && N > 0;
    if (!want_h && !want_w && !want_b) return FASTGL_OK;
    if (M > 0 && (!label || !lse || !dloss || (K > 0 && (!H || !W)))) {
        set_error("H, W, label, lse or dloss is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    const uintptr_t el = dtype == FASTGL_BF16 ? 2 : 4;
    if (misaligned_to(H, el) || misaligned_to(W, el) || misaligned_to(b, 4) || misaligned_to(label, 8) || misaligned_to(lse, 4) ||
        misaligned_to(dloss, 4) || misaligned_to(dH, el) || misaligned_to(dW, el) || misaligned_to(db, 4)) {
        set_error("buffers must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    hipStream_t s = (hipStream_t)stream;
    if (M == 0) {                                     // sums without terms
        if (want_w && (st = launch_no_terms(dtype == FASTGL_BF16, dW, nullptr, K, N, false, s, "fastgl_loss_bwd (dW, M = 0)")) != FASTGL_OK) return st;
        if (want_b) return launch_no_terms(false, db, nullptr, 1, N, false, s, "fastgl_loss_bwd (db, M = 0)");
        return FASTGL_OK;
    }
    const Shape d(dtype, M, K, N, starts_whole({H, W}), true, coarse);
    if ((st = check_workspace(ws, ws_bytes, Scratch(d, nullptr).used)) != FASTGL_OK) return st;
    const Scratch o(d, (char *)ws);
    if (d.small()) {
        LossBlockArgs a = {};
        a.H = H; a.W = W; a.b = b;
        a.label = label;
        a.lse_in = lse; a.dloss = dloss;
        a.dH = want_h ? dH : nullptr; a.dW = want_w ? dW : nullptr;
        a.db = want_b ? db : nullptr;
        a.part_h = o.part_h; a.part_w = o.part_w; a.part_b = o.db;
        if ((st = launch_block(d, a, s, "fastgl_loss_bwd (small)")) != FASTGL_OK) return st;
        LossAddArgs t = {};
        int64_t total = 0;
        auto add = [&](int m, const float *part, void *out, int64_t n, int64_t parts, bool bf16) {
            if (!part || !out) return;
            t.part[m] = part;
            t.out[m] = out;
            t.n[m] = n;
            t.parts[m] = (int32_t)parts;
            t.bf16[m] = bf16;
            // Fewer elements a workgroup where there are few of many parts, 128 bytes of a part at least.  250 parts of 12 032 elements: 256 threads
            // and 32 bytes of a part a workgroup 10.6 us, 1024 and 128 bytes 5.2.
            t.lg[m] = kAddLg;
            while (t.lg[m] > 5 && (parts >> (kAddLg - t.lg[m])) > 8 && ceil_div(n, (int64_t)1 << t.lg[m]) < 1024) --t.lg[m];
            t.blocks[m] = ceil_div(n, (int64_t)1 << t.lg[m]);
            total += t.blocks[m];
        };
        add(0, a.part_h, a.dH, M * K, d.strips(), d.bf16);
        add(1, a.part_w, a.dW, K * N, d.tiles(), d.bf16);
        add(2, a.part_b, a.db, N, d.tiles(), false);
        if (total == 0) return FASTGL_OK;
        hipLaunchKernelGGL(k_loss_add, dim3((unsigned)total), dim3(kAddThreads), 0, s, t);
        FASTGL_LAUNCH_CHECK("fastgl_loss_bwd (sums)");
        return FASTGL_OK;
    }
    const Cut scores = d.scores_cut(), rows = d.rows_cut(), weights = d.weights_cut();
    for (int64_t n0 = 0; n0 < N; n0 += d.piece()) {
        const int64_t n = N - n0 < d.piece() ? N - n0 : d.piece();
        if ((st = pack(d, o, H, W, label, n0, n, n0 == 0, d.pack_w, s)) != FASTGL_OK) return st;
        LossTileArgs z = scores_of(d, o, H, W, b, label, n0, n);
        z.lse = lse;
        z.dloss = dloss;
        z.dz = o.dz; z.dz_plane = d.z_plane(); z.dz_ld = d.z_ld(); z.dz_block = d.z_block();
        z.db = want_b ? o.db : nullptr;
        st = !d.bf16            ? launch<kGradient, false, 3>(z, scores, d.bf16, s, "fastgl_loss_bwd (dZ)")
             : d.z_planes == 2 ? launch<kGradient, false, 2>(z, scores, d.bf16, s, "fastgl_loss_bwd (dZ)")
                               : launch<kGradient, false, 1>(z, scores, d.bf16, s, "fastgl_loss_bwd (dZ)");
        if (st != FASTGL_OK) return st;
        LossSumArgs sum = {};                         // the sums at the end of the piece
        if (want_b) {
            sum.db_part = o.db;
            sum.db = db + n0;
            sum.db_rows = (int32_t)d.db_rows(); sum.db_cols = (int32_t)n;
        }
        if (want_h) {
            LossTileArgs g = {};
            g.a[0] = o.dz;
            g.b[0] = d.pack_w ? o.w : (const uint16_t *)W + n0;
            g.a_plane = d.z_plane(); g.lda = d.z_ld();
            g.a_blocks = d.blocks() ? d.z_block() : 0;
            g.ldb = z.ldb; g.b_plane = z.b_plane;
            g.R = M; g.C = K; g.Kc = n;
            g.pairs = (int32_t)d.z_pairs; g.groups = 1;
            g.planes_a = !d.bf16 ? kSixA : d.z_planes == 2 ? kTwo : 0;
            g.planes_b = !d.bf16 ? kSixB : 0;
            g.out[0] = dH;
            g.part = o.part_h;
            g.add = n0 > 0;
            st = d.parts_h() ? launch<kRowsAdd, true>(g, rows, d.bf16, s, "fastgl_loss_bwd (dH)") : launch<kRows, false>(g, rows, d.bf16, s, "fastgl_loss_bwd (dH)");
            if (st != FASTGL_OK) return st;
        }
        if (want_w) {
            LossTileArgs g = {};
            g.a[0] = o.h;
            g.b[0] = o.dz;
            g.a_plane = M * d.ldk; g.lda = d.ldk;
            g.b_plane = d.z_plane(); g.ldb = d.z_ld();
            g.b_blocks = d.blocks() ? d.z_block() : 0;
            g.R = K; g.C = n; g.Kc = M;
            g.pairs = (int32_t)d.z_pairs; g.groups = 1;
            g.planes_a = !d.bf16 ? kSixA : 0;
            g.planes_b = !d.bf16 ? kSixB : d.z_planes == 2 ? kTwo : 0;
            g.out[0] = static_cast<char *>(dW) + n0 * (int64_t)el;
            g.ldo = N;
            g.part = o.part_w;
            st = weights.slabs > 1 ? launch<kWeightsOne, true>(g, weights, d.bf16, s, "fastgl_loss_bwd (dW)")
                                   : launch<kWeightsOne, false>(g, weights, d.bf16, s, "fastgl_loss_bwd (dW)");
            if (st != FASTGL_OK) return st;
            if (weights.slabs > 1) {
                sum.part = o.part_w;
                sum.out = g.out[0];
                sum.R = K; sum.C = n; sum.ldo = N;
                sum.slabs = (int32_t)weights.slabs;
            }
        }
        if ((sum.part || sum.db_part) && (st = launch_sum(sum, d.bf16, s, "fastgl_loss_bwd (sums)")) != FASTGL_OK) return st;
    }
    if (!want_h || !d.parts_h()) return FASTGL_OK;
    LossSumArgs sum = {};
    sum.part = o.part_h;
    sum.out = dH;
    sum.R = M; sum.C = K; sum.ldo = K;
    sum.slabs = (int32_t)rows.slabs;
    return launch_sum(sum, d.bf16, s, "fastgl_loss_bwd (dH, sums)");
}

}  // namespace
}  // namespace fastgl

using namespace fastgl;

extern "C" {

size_t fastgl_loss_fwd_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned)
{
    return workspace(dtype, M, K, N, aligned != 0, false);
}

size_t fastgl_loss_bwd_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned)
{
    return workspace(dtype, M, K, N, aligned != 0, true);
}

size_t fastgl_loss_bwd_coarse_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned)
{
    return workspace(dtype, M, K, N, aligned != 0, true, true);
}

fastgl_status fastgl_loss_fwd(fastgl_dtype dtype, const void *H, const void *W, const float *b, const int64_t *label, int64_t M,
                              int64_t K, int64_t N, float *loss, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    fastgl_status st = check(dtype, M, K, N);
    if (st != FASTGL_OK) return st;
    if (M == 0) return FASTGL_OK;
    if (!label || !loss || (K > 0 && (!H || !W))) {
        set_error("H, W, label or loss is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    const uintptr_t el = dtype == FASTGL_BF16 ? 2 : 4;
    if (misaligned_to(H, el) || misaligned_to(W, el) || misaligned_to(b, 4) || misaligned_to(label, 8) || misaligned_to(loss, 4) || misaligned_to(lse, 4)) {
        set_error("buffers must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    const Shape d(dtype, M, K, N, starts_whole({H, W}), false, false);
    if ((st = check_workspace(ws, ws_bytes, Scratch(d, nullptr).used)) != FASTGL_OK) return st;
    const Scratch o(d, (char *)ws);
    hipStream_t s = (hipStream_t)stream;
    if (d.small()) {
        LossBlockArgs a = {};
        a.H = H; a.W = W; a.b = b;
        a.label = label;
        a.loss = loss; a.lse = lse;
        a.stats = o.stats; a.picked = o.picked;
        st = launch_block(d, a, s, "fastgl_loss_fwd (small)");
        return st != FASTGL_OK || d.strips() == 1 ? st : launch_join(o, d.strips(), true, true, label, M, N, loss, lse, s);
    }
    const Cut cut = d.scores_cut();
    for (int64_t n0 = 0; n0 < N; n0 += d.piece()) {
        const int64_t n = N - n0 < d.piece() ? N - n0 : d.piece();
        if ((st = pack(d, o, H, W, label, n0, n, d.pack_h && n0 == 0, d.pack_w, s)) != FASTGL_OK) return st;
        LossTileArgs g = scores_of(d, o, H, W, b, label, n0, n);
        g.stats = o.stats;
        g.picked = o.picked;
        if ((st = launch<kScores, false>(g, cut, d.bf16, s, "fastgl_loss_fwd")) != FASTGL_OK) return st;
        if ((st = launch_join(o, ceil_div(n, Shape::wave_cols(cut)), n0 == 0, n0 + n == N, label, M, N, loss, lse, s)) != FASTGL_OK) return st;
    }
    return FASTGL_OK;
}

fastgl_status fastgl_loss_bwd(fastgl_dtype dtype, const void *H, const void *W, const float *b, const int64_t *label,
                              const float *lse, const float *dloss, int64_t M, int64_t K, int64_t N, void *dH, void *dW, float *db,
                              void *ws, size_t ws_bytes, void *stream)
{
    return loss_bwd(false, dtype, H, W, b, label, lse, dloss, M, K, N, dH, dW, db, ws, ws_bytes, stream);
}

fastgl_status fastgl_loss_bwd_coarse(fastgl_dtype dtype, const void *H, const void *W, const float *b, const int64_t *label,
                                     const float *lse, const float *dloss, int64_t M, int64_t K, int64_t N, void *dH, void *dW, float *db,
                                     void *ws, size_t ws_bytes, void *stream)
{
    return loss_bwd(true, dtype, H, W, b, label, lse, dloss, M, K, N, dH, dW, db, ws, ws_bytes, stream);
}

}  // extern "C"
