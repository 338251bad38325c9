// Gated feed-forward update, forward and backward (fastgl_gated.h has the formulas): what is around the products of
// gated_tile.h.
//
//   forward   [operands packed] -> one product for G and U with the gate in its epilogue; few rows: k_gated_rows alone
//   backward  k_gated_dz (dG, dU as the matrix cores take them, column sums) -> dX: one product over both halves
//             -> dWg and dWu: one product
//   where a product has few tiles, its steps are dealt to several workgroups a tile, whose sums are added in fp64 afterwards
#include "gated_tile.h"
#include "update_internal.h"

namespace fastgl {
namespace {

// Rows that k_gated_rows takes, by the elements of a weight matrix: its time grows with the rows, that of the tiles hardly, but they pack
// operands that are fp32 or no multiple of 16 bytes.  us a call, k_gated_rows / tiles, on both sides of each line:
//   bf16, nothing to pack: 1024 -> 4096 2 rows 8.2 / 10.5, 3 rows 11.4 / 10.5, 8 rows 12.8 / 11.0; 2048 -> 1024 8 rows 9.3 / 9.9; 512 -> 2048 8 rows
//   6.6 / 9.0; 256 -> 1024 8 rows 5.6 / 5.6, 16 rows 5.6 / 5.6, 32 rows 7.2 / 5.6
//   bf16, packed: 1000 -> 4095 12 rows 16.6 / 19.0, 16 rows 19.6 / 18.9, 32 rows 34.5 / 19.2; 500 -> 2001 24 rows 13.8 / 15.5, 32 rows 17.1 / 15.5, 48 rows
//   23.0 / 15.7; 257 -> 1023 32 rows 8.3 / 9.6, 48 rows 12.1 / 9.8; 2000 -> 300 32 rows 11.8 / 13.1, 64 rows 15.6 / 13.6; 100 -> 300 64 rows 5.6 / 9.1
//   fp32: 1024 -> 4096 48 rows 34.5 / 48.4, 64 rows 43.6 / 48.9, 80 rows 51.9 / 49.4; 1000 -> 1000 64 rows 23.1 / 26.3, 80 rows 27.1 / 26.4; 256 -> 1024
//   64 rows 11.0 / 15.8, 128 rows 17.1 / 18.0; 100 -> 300 64 rows 5.6 / 12.5
inline int64_t few_rows_of(bool bf16, bool packed, int64_t weights)
{
    if (bf16 && !packed) return weights > (int64_t)1 << 21 ? 2 : 8;
    if (bf16 && weights > (int64_t)1 << 16) return weights > (int64_t)1 << 21 ? 16 : 32;
    return 60;
}
constexpr int kSumGroups = 2048;       // workgroups of the gradient of the gate
constexpr int64_t kMostWidth = (int64_t)1 << 20;

// x as three bf16 whose sum is x exactly (each rounding to nearest).
__device__ __forceinline__ void pieces(float x, float (&p)[3])
{
    p[0] = (float)(__bf16)x;
    const float r = x - p[0];
    p[1] = (float)(__bf16)r;
    p[2] = r - p[1];
}

// Eight columns into `planes` bf16 planes.
template <int PLANES>
__device__ __forceinline__ void store_planes(uint16_t *p, int64_t plane, const float (&v)[8])
{
    if constexpr (PLANES == 1) {
        Chunk<true>::store(p, v, 8);
    } else {
        float q[3][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float c[3];
            pieces(v[j], c);
            q[0][j] = c[0];
            q[1][j] = c[1];
            q[2][j] = c[2];
        }
#pragma unroll
        for (int i = 0; i < PLANES; ++i) Chunk<true>::store(p + i * plane, q[i], 8);
    }
}

// ------------------------------------------------------------------------------------ packing
// Matrices [rows][cols] as planes of bf16 with rows of ld elements, 0 beyond cols.
struct PackArgs {
    const void *src[3];
    uint16_t *out[3];
    int64_t rows[3];
    int32_t cols[3], ld[3];
};

template <bool BF16>
__global__ __launch_bounds__(kBlock) void k_gated_pack(PackArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    const int m = blockIdx.y;
    const T *src = static_cast<const T *>(m == 0 ? a.src[0] : m == 1 ? a.src[1] : a.src[2]);
    uint16_t *out = m == 0 ? a.out[0] : m == 1 ? a.out[1] : a.out[2];
    const int64_t rows = m == 0 ? a.rows[0] : m == 1 ? a.rows[1] : a.rows[2];
    const int32_t cols = m == 0 ? a.cols[0] : m == 1 ? a.cols[1] : a.cols[2], ld = m == 0 ? a.ld[0] : m == 1 ? a.ld[1] : a.ld[2];
    const int32_t chunks = ld / kChunk;
    const int64_t n = rows * chunks;
    for (int64_t u = (int64_t)blockIdx.x * kBlock + threadIdx.x; u < n; u += (int64_t)gridDim.x * kBlock) {
        const int64_t row = u / chunks;
        const int col = (int)(u - row * chunks) * kChunk;
        Chunk<BF16> c;
        float v[8];
        const int64_t wave_u = u - (threadIdx.x & (kWave - 1));
        const bool inside = __builtin_amdgcn_readfirstlane((int)(wave_u + kWave + kChunk <= n));
        load_row(c, src, row * cols + col, cols - col, inside);
        c.get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < cols - col ? v[j] : 0.f;
        store_planes<BF16 ? 1 : 3>(out + row * ld + col, rows * ld, v);
    }
}

// ------------------------------------------------------------------------------------ few rows
struct RowsArgs {
    const void *X, *Wg, *Wu;
    const float *bg, *bu;
    void *P, *G, *U;
    int32_t M, K, N, act;
    int32_t strips, groups;          // strips of columns, groups of rows
};

// MR rows of a strip of columns by one workgroup: 2^LG lanes hold eight columns of both weights each, the lanes beyond them
// the next k; the sums of a column are joined through the lanes of a wavefront, then through LDS, in a fixed order.
// Bound by the weights: neighbouring strips, which share lines, are given to one L2 domain.
template <bool BF16, int MR, int LG>
__global__ __launch_bounds__(kBlock) void k_gated_rows(RowsArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    constexpr int LANES = 1 << LG, SLOTS = kBlock >> LG, NV = MR * 16, LEFT = NV * LANES > kWave ? NV * LANES / kWave : 1;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    uint32_t at = blockIdx.x;
    {
        const uint32_t total = (uint32_t)a.strips * (uint32_t)a.groups, q = total / kXcds, rest = total % kXcds, x = at % kXcds;
        at = x * q + (x < rest ? x : rest) + at / kXcds;
    }
    const int strip = (int)(at / (uint32_t)a.groups), m0 = (int)(at - (uint32_t)strip * (uint32_t)a.groups) * MR;
    const int c = threadIdx.x & (LANES - 1), col = (strip * LANES + c) * kChunk, left = a.N - col;
    const T *X = static_cast<const T *>(a.X), *Wg = static_cast<const T *>(a.Wg), *Wu = static_cast<const T *>(a.Wu);
    float v[NV];                                                     // [row][gate, up][column]
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = 0.f;
#pragma unroll 4
    for (int k = threadIdx.x >> LG; k < a.K; k += SLOTS) {
        const bool inside = k - (int)(threadIdx.x >> LG) + wave_first(LG) + (kWave >> LG) + kChunk <= a.K;
        Chunk<BF16> qg, qu;
        float g[8], u[8];
        load_row(qg, Wg, (int64_t)k * a.N + col, left, inside);       // columns that do not exist are summed and not stored
        load_row(qu, Wu, (int64_t)k * a.N + col, left, inside);
        float x[MR];
#pragma unroll
        for (int m = 0; m < MR; ++m) {
            const int64_t row = m0 + m < a.M ? m0 + m : a.M - 1;
            if constexpr (BF16) x[m] = __uint_as_float((uint32_t)X[row * a.K + k] << 16);
            else x[m] = X[row * a.K + k];
        }
        qg.get(g);
        qu.get(u);
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[m * 16 + j] = fmaf(x[m], g[j], v[m * 16 + j]);
                v[m * 16 + 8 + j] = fmaf(x[m], u[j], v[m * 16 + 8 + j]);
            }
    }
    __shared__ float sums[kBlock / kWave][LANES][NV];
    const int first = scatter_sum<NV, kWave / 2, LANES>(v, lane);
#pragma unroll
    for (int i = 0; i < LEFT; ++i) sums[wave][c][first + i] = v[i];
    __syncthreads();
    for (int i = threadIdx.x; i < MR * LANES * 8; i += kBlock) {
        const int m = i / (LANES * 8), j = i - m * (LANES * 8), row = m0 + m, e = m * 16 + (j & 7), l = j >> 3;
        const int64_t n = (int64_t)strip * (LANES * 8) + j;
        if (row >= a.M || n >= a.N) continue;
        float g = (sums[0][l][e] + sums[1][l][e]) + (sums[2][l][e] + sums[3][l][e]);
        float u = (sums[0][l][e + 8] + sums[1][l][e + 8]) + (sums[2][l][e + 8] + sums[3][l][e + 8]);
        if (a.bg) g += a.bg[n];
        if (a.bu) u += a.bu[n];
        const int64_t to = (int64_t)row * a.N + n;
        auto put = [&](void *out, float x) {
            if constexpr (BF16) static_cast<T *>(out)[to] = __builtin_bit_cast(uint16_t, (__bf16)x);
            else static_cast<T *>(out)[to] = x;
        };
        float act;
        switch (a.act) {
            case FASTGL_ACT_SILU: act = gate<FASTGL_ACT_SILU, false, BF16>(g, nullptr); break;
            case FASTGL_ACT_GELU: act = gate<FASTGL_ACT_GELU, false, BF16>(g, nullptr); break;
            case FASTGL_ACT_RELU: act = gate<FASTGL_ACT_RELU, false, BF16>(g, nullptr); break;
            default: act = gate<FASTGL_ACT_SIGMOID, false, BF16>(g, nullptr); break;
        }
        put(a.P, act * u);
        if (a.G) put(a.G, g);
        if (a.U) put(a.U, u);
    }
}

// ------------------------------------------------------------------------------------ gradient of the gate
struct DzArgs {
    const void *G, *U, *dP;
    uint16_t *dG, *dU;               // planes [M][ld], or NULL
    int64_t M, plane, ld, block;     // ld: elements between rows, block: between blocks of 32 columns (32: rows lie whole)
    int32_t N, lg;                   // 2^lg lanes of eight columns a row
    float *part;                     // [gridDim.y][2][N] column sums, or NULL
};

// dG = dP U act'(G), dU = dP act(G), rounded to what the matrix cores take: three pieces of fp32, or bf16, whose rounding adds an error
// of the size of the results' own, as rounding any bf16 tensor between two products does (results are off by sqrt 2 of what their own
// rounding costs, root mean square), or, where the caller asks for it, two pieces (2^-17) at twice the products: us a bf16 call, one piece /
// two: 1 row 256 -> 1024 22 / 22, 300 rows 28 / 37, 8000 rows 72 / 91, 130 000 rows 32 -> 64 72 / 119, 16 384 rows 1024 -> 4096 586 / 1042.
// One rule for all sizes: a row's gradient has the same error in a small batch and in a large one.  The column sums are formed from the
// unrounded values.
// Bound by memory: 16 384 x 4096 bf16 119 us, 671 MB at 5.6 TB/s.
template <bool BF16, int ACT, int PLANES>
__global__ __launch_bounds__(kBlock) void k_gated_dz(DzArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    const int lanes = 1 << a.lg, c = threadIdx.x & (lanes - 1), rows = kBlock >> a.lg;
    const int col = (int)(blockIdx.x * lanes + c) * kChunk, left = a.N - col;
    const T *G = static_cast<const T *>(a.G), *U = static_cast<const T *>(a.U), *dP = static_cast<const T *>(a.dP);
    float sg[8], su[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sg[j] = su[j] = 0.f;
    if (left > 0) {
        for (int64_t row = (int64_t)blockIdx.y * rows + (threadIdx.x >> a.lg); row < a.M; row += (int64_t)gridDim.y * rows) {
            const int64_t at = row * a.N + col;
            const bool inside = row - (threadIdx.x >> a.lg) + wave_first(a.lg) + (kWave >> a.lg) + kChunk <= a.M;
            Chunk<BF16> qg, qu, qp;
            float g[8], u[8], p[8];
            load_row(qg, G, at, left, inside);
            load_row(qu, U, at, left, inside);
            load_row(qp, dP, at, left, inside);
            qg.get(g);
            qu.get(u);
            qp.get(p);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float grad;
                const float v = gate<ACT, true, BF16>(g[j], &grad);
                g[j] = p[j] * u[j] * grad;
                u[j] = p[j] * v;
                if (j >= left) g[j] = u[j] = 0.f;                  // padding
                sg[j] += g[j];
                su[j] += u[j];
            }
            if (a.dG) {
                const int64_t to = (col >> 5) * a.block + row * a.ld + (col & 31);
                store_planes<PLANES>(a.dG + to, a.plane, g);
                store_planes<PLANES>(a.dU + to, a.plane, u);
            }
        }
    }
    if (!a.part) return;
    __shared__ float sums[2][kBlock * kChunk];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        sums[0][threadIdx.x * kChunk + j] = sg[j];
        sums[1][threadIdx.x * kChunk + j] = su[j];
    }
    __syncthreads();
    const int width = lanes * kChunk;
    for (int i = threadIdx.x; i < 2 * width; i += kBlock) {
        const int q = i >= width, j = i - q * width;
        const int64_t n = (int64_t)blockIdx.x * width + j;
        float v = 0.f;
        for (int r = 0; r < rows; ++r) v += sums[q][r * width + j];
        if (n < a.N) a.part[((int64_t)blockIdx.y * 2 + q) * a.N + n] = v;
    }
}

// What a backward pass adds up at its end, in fp64 and a fixed order: slabs of up to two results of n elements, and the
// column sums of dG and dU.
struct SumArgs {
    const float *part;               // slab s of result q at part + s * stride + q * n
    void *out[2];                    // or NULL
    int64_t n, stride;
    int32_t slabs, results;
    int32_t blocks;                  // workgroups of the slabs, before those of the columns
    const float *db;                 // [rows][2][N]
    float *dbg, *dbu;
    int32_t rows, N;
};

template <bool BF16>
__global__ __launch_bounds__(kBlock) void k_gated_sum(SumArgs a)
{
    if ((int)blockIdx.x < a.blocks) {
        const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
        if (i >= a.n * a.results) return;
        const int q = i >= a.n;
        if (!a.out[q]) return;
        double v = 0.0;
#pragma unroll 8
        for (int s = 0; s < a.slabs; ++s) v += (double)a.part[(int64_t)s * a.stride + i];
        if constexpr (BF16) static_cast<uint16_t *>(a.out[q])[i - q * a.n] = __builtin_bit_cast(uint16_t, (__bf16)(float)v);
        else static_cast<float *>(a.out[q])[i - q * a.n] = (float)v;
        return;
    }
    __shared__ double sums[kBlock / 8][9];                             // eight columns, 32 threads a column
    const int c = threadIdx.x & 7, r = threadIdx.x >> 3;
    const int64_t col = ((int64_t)blockIdx.x - a.blocks) * 8 + c;
    double v = 0.0;
    if (col < 2 * (int64_t)a.N) {
#pragma unroll 8
        for (int i = r; i < a.rows; i += kBlock / 8) v += (double)a.db[(int64_t)i * 2 * a.N + col];
    }
    sums[r][c] = v;
    __syncthreads();
    if (r == 0 && col < 2 * (int64_t)a.N) {
        v = 0.0;
        for (int i = 0; i < kBlock / 8; ++i) v += sums[i][c];
        float *out = col < a.N ? a.dbg : a.dbu;
        if (out) out[col < a.N ? col : col - a.N] = (float)v;
    }
}

// The forward pass's slabs: sums, biases and the gate.
template <bool BF16, int ACT>
__global__ __launch_bounds__(kBlock) void k_gated_join(const float *__restrict__ part, int32_t slabs, int64_t n, int32_t N, const float *bg,
                                                       const float *bu, void *P, void *G, void *U)
{
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i >= n) return;
    const int c = (int)(i % N);
    double sg = bg ? (double)bg[c] : 0.0, su = bu ? (double)bu[c] : 0.0;
#pragma unroll 4
    for (int s = 0; s < slabs; ++s) {
        sg += (double)part[(int64_t)(2 * s) * n + i];
        su += (double)part[(int64_t)(2 * s + 1) * n + i];
    }
    const float g = (float)sg, u = (float)su;
    auto put = [&](void *out, float v) {
        if constexpr (BF16) static_cast<uint16_t *>(out)[i] = __builtin_bit_cast(uint16_t, (__bf16)v);
        else static_cast<float *>(out)[i] = v;
    };
    put(P, gate<ACT, false, BF16>(g, nullptr) * u);
    if (G) put(G, g);
    if (U) put(U, u);
}

// ------------------------------------------------------------------------------------ host side
bool misaligned_to(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

// Where a call's scratch lies; base NULL: only the size is wanted.
struct Layout {
    size_t used = 0;
    char *base = nullptr;
    template <class T>
    T *take(size_t n)
    {
        char *p = base ? base + used : nullptr;
        used += align_up(n * sizeof(T), 256);
        return reinterpret_cast<T *>(p);
    }
};

struct Shape {
    bool bf16, aligned, fine;
    int planes;
    int64_t M, K, N, ldk, ldn, ldz;
    Shape(fastgl_dtype dtype, int64_t M_, int64_t K_, int64_t N_, bool aligned_, bool fine_ = false)
        : bf16(dtype == FASTGL_BF16), aligned(aligned_), fine(fine_), planes(dtype == FASTGL_BF16 ? 1 : 3), M(M_), K(K_), N(N_),
          ldk((int64_t)align_up((size_t)K_, 8)), ldn((int64_t)align_up((size_t)N_, 8)), ldz((int64_t)align_up((size_t)N_, 32))
    {
    }
    bool pack_x() const { return !bf16 || !aligned || K % 8; }
    bool pack_w() const { return !bf16 || !aligned || N % 8; }
    bool few_rows() const { return M <= few_rows_of(bf16, pack_x() || pack_w(), K * N); }
    // Elements of a block of 32 columns of dG and dU, which lie [block][row][32]: dX then reads whole lines although it takes 32
    // columns a step (16 384 x 8192 times 8192 x 1024: 245 -> 221 us).  A block is 2304 bytes more than a multiple of 4096: the tiles
    // of the weight gradients read the same rows of many blocks at a time, which should not meet in the same memory channels.  0: rows lie
    // whole, where there are few or four blocks pass 32-bit offsets.  us a backward call, blocks / whole rows, 1024 -> 4096: 512 rows bf16
    // 50.5 / 50.2, fp32 154 / 155; 1024 rows 65.7 / 66.4, 249 / 253; 2000 rows 110 / 109, 403 / 413; 4000 rows 189 / 190, 752 / 779; 16 000 rows
    // 574 / 594, 2750 / 2839; bf16 256 -> 1024 1000 rows 35.8 / 37.1, 4000 rows 53.1 / 51.5, 16 000 rows 96.9 / 101.7.
    int64_t z_block() const { return M >= 1024 && M <= (int64_t)1 << 22 ? (int64_t)(align_up((size_t)M * 64, 4096) + 2304) / 2 : 0; }
    int64_t z_plane() const { return z_block() ? ldz / 32 * z_block() : M * ldz; }
    int z_planes() const { return !bf16 ? 3 : fine ? 2 : 1; }               // of dG and dU
    int64_t pairs() const { return bf16 ? 1 : 6; }
    int64_t z_pairs() const { return bf16 ? z_planes() : 6; }
    Cut forward_cut() const { return cut_of(kForward, M, N, K, pairs()); }
    Cut rows_cut() const { return cut_of(kRows, M, K, N, 2 * z_pairs()); }
    Cut weights_cut() const { return cut_of(kWeights, K, N, M, z_pairs()); }
    // workgroups of k_gated_dz: (columns, rows); 2^lg lanes a row
    int lg() const
    {
        int lg = 0;
        while (lg < 5 && ((int64_t)8 << lg) < N) ++lg;
        return lg;
    }
    int64_t dz_cols() const { return ceil_div(N, (int64_t)8 << lg()); }
    int64_t dz_rows() const
    {
        const int64_t most = ceil_div(M, (int64_t)(kBlock >> lg()) * 4), some = ceil_div(kSumGroups, dz_cols() > 0 ? dz_cols() : 1);
        return most < some ? (most > 0 ? most : 1) : some;
    }
};

struct Scratch {
    uint16_t *x, *wg, *wu, *dg, *du;
    float *db, *part;                // part: of one product at a time
};

Scratch carve(const Shape &s, bool backward, Layout &l)
{
    Scratch o = {};
    if (s.pack_x()) o.x = l.take<uint16_t>((size_t)(s.planes * s.M * s.ldk));
    if (s.pack_w()) {
        o.wg = l.take<uint16_t>((size_t)(s.planes * s.K * s.ldn));
        o.wu = l.take<uint16_t>((size_t)(s.planes * s.K * s.ldn));
    }
    auto sums = [](const Cut &c, int64_t n) { return c.slabs > 1 ? (size_t)(c.slabs * n) : (size_t)0; };
    if (backward) {
        o.dg = l.take<uint16_t>((size_t)(s.z_planes() * s.z_plane()));
        o.du = l.take<uint16_t>((size_t)(s.z_planes() * s.z_plane()));
        o.db = l.take<float>((size_t)(s.dz_rows() * 2 * s.N));
        const size_t x = sums(s.rows_cut(), s.M * s.K), w = sums(s.weights_cut(), 2 * s.K * s.N);
        o.part = l.take<float>(x > w ? x : w);
    } else
        o.part = l.take<float>(sums(s.forward_cut(), 2 * s.M * s.N));
    return o;
}

fastgl_status check(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, fastgl_act act)
{
    if (dtype != FASTGL_F32 && dtype != FASTGL_BF16) {
        set_error("bad dtype %d", (int)dtype);
        return FASTGL_ERR_INVALID_ARG;
    }
    if ((int)act < FASTGL_ACT_SILU || (int)act > FASTGL_ACT_SIGMOID) {
        set_error("bad activation %d", (int)act);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (M < 0 || K < 0 || N < 0) {
        set_error("negative size (M=%lld K=%lld N=%lld)", (long long)M, (long long)K, (long long)N);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (M > kMaxIndex || K > kMostWidth || N > kMostWidth) {
        set_error("M must stay below 2^31-1-1024, K and N at 2^20 or below");
        return FASTGL_ERR_UNSUPPORTED;
    }
    return FASTGL_OK;
}

fastgl_status check_workspace(const void *workspace, size_t bytes, size_t need)
{
    if (need == 0) return FASTGL_OK;
    if (!workspace || misaligned_to(workspace, 256)) {
        set_error("workspace must be a 256-byte aligned device buffer");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (bytes < need) {
        set_error("workspace too small: %zu < %zu bytes", bytes, need);
        return FASTGL_ERR_WORKSPACE;
    }
    return FASTGL_OK;
}

// What of X, Wg and Wu a product needs packed, in one launch.
fastgl_status pack(const Shape &d, const Scratch &o, const void *X, const void *Wg, const void *Wu, bool x, bool w, hipStream_t st)
{
    PackArgs a = {};
    int n = 0;
    int64_t most = 0;
    auto add = [&](const void *src, uint16_t *out, int64_t rows, int64_t cols, int64_t ld) {
        if (rows == 0 || cols == 0) return;
        a.src[n] = src;
        a.out[n] = out;
        a.rows[n] = rows;
        a.cols[n] = (int32_t)cols;
        a.ld[n++] = (int32_t)ld;
        if (rows * (ld / kChunk) > most) most = rows * (ld / kChunk);
    };
    if (x && d.pack_x()) add(X, o.x, d.M, d.K, d.ldk);
    if (w && d.pack_w()) {
        add(Wg, o.wg, d.K, d.N, d.ldn);
        add(Wu, o.wu, d.K, d.N, d.ldn);
    }
    if (n == 0) return FASTGL_OK;
    const int64_t blocks = ceil_div(most, kBlock);
    const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384), (unsigned)n);
    if (d.bf16) hipLaunchKernelGGL(k_gated_pack<true>, grid, dim3(kBlock), 0, st, a);
    else hipLaunchKernelGGL(k_gated_pack<false>, grid, dim3(kBlock), 0, st, a);
    FASTGL_LAUNCH_CHECK("fastgl_gated (pack)");
    return FASTGL_OK;
}

template <class F>
void by_act(fastgl_act act, F f)
{
    switch (act) {
        case FASTGL_ACT_SILU: f(std::integral_constant<int, FASTGL_ACT_SILU>()); break;
        case FASTGL_ACT_GELU: f(std::integral_constant<int, FASTGL_ACT_GELU>()); break;
        case FASTGL_ACT_RELU: f(std::integral_constant<int, FASTGL_ACT_RELU>()); break;
        default: f(std::integral_constant<int, FASTGL_ACT_SIGMOID>()); break;
    }
}

// One product: results in bf16 or fp32, or sums of slabs.
//
// Results of the forward pass go past the caches where the tiles' rows are whole 128-byte lines.  us, through the caches / past them (bf16; kernel
// times, the least of 150 passes on one card): 115 000 rows 256 -> 1024, G and U kept 246 / 174, alone 167 / 141; 8000 rows 16.9 / 16.2, 13.8 / 12.4;
// 16 384 rows 1024 -> 4096 302 / 273, 253 / 242.  Rows that are not: 60 000 rows 128 -> 520 49 / 92; 20 000 rows 104 -> 1000 31 / 63.
template <int MODE, class ACT>
fastgl_status launch_tile(TileArgs g, const Cut &cut, bool bf16, ACT, hipStream_t s, const char *what)
{
    constexpr int A = ACT::value;
    const int64_t bm = cut.size == kLarge ? 256 : 128, bc = (cut.size == kSmall ? 128 : 256) / (MODE == kRows ? 1 : 2);
    const int64_t line = bf16 ? 64 : 32;                             // elements
    const bool once = cut.size != kSmall && g.C % line == 0 && !misaligned_to(g.out[0], 128) && !misaligned_to(g.out[1], 128) && !misaligned_to(g.out[2], 128);
    const int64_t tr = ceil_div(g.R, bm), tc = ceil_div(g.C, bc), total = tr * tc * cut.slabs;
    if (total > 0x7FFFFFFFLL || 4 * tc > 0x7FFFFFFFLL) {
        set_error("%s: too many tiles (%lld)", what, (long long)total);
        return FASTGL_ERR_UNSUPPORTED;
    }
    g.tiles_r = (int32_t)tr;
    g.tiles_c = (int32_t)tc;
    g.slabs = (int32_t)cut.slabs;
    auto sized = [&](auto size) {
        constexpr int S = decltype(size)::value;
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)total), dim3(Tile<MODE, S>::THREADS), 0, s, g); };
        if (cut.slabs > 1) return go(k_gated_tile<MODE, S, float, 0, true, false>);
        if constexpr (MODE == kForward) {
            if (once) return bf16 ? go(k_gated_tile<MODE, S, uint16_t, A, false, true>) : go(k_gated_tile<MODE, S, float, A, false, true>);
        }
        if (bf16) go(k_gated_tile<MODE, S, uint16_t, A, false, false>);
        else go(k_gated_tile<MODE, S, float, A, false, false>);
    };
    if (cut.size == kLarge) sized(std::integral_constant<int, kLarge>());
    else if (cut.size == kMiddle) sized(std::integral_constant<int, kMiddle>());
    else sized(std::integral_constant<int, kSmall>());
    FASTGL_LAUNCH_CHECK(what);
    return FASTGL_OK;
}

fastgl_status launch_sum(SumArgs a, bool bf16, hipStream_t s, const char *what)
{
    a.blocks = (int32_t)ceil_div(a.n * a.results, kBlock);
    const dim3 grid((unsigned)(a.blocks + (a.db ? ceil_div(2 * (int64_t)a.N, 8) : 0)));
    if (bf16) hipLaunchKernelGGL(k_gated_sum<true>, grid, dim3(kBlock), 0, s, a);
    else hipLaunchKernelGGL(k_gated_sum<false>, grid, dim3(kBlock), 0, s, a);
    FASTGL_LAUNCH_CHECK(what);
    return FASTGL_OK;
}

bool starts_whole(std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if (misaligned_to(p, 16)) return false;
    return true;
}

size_t workspace(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, bool aligned, bool backward, bool fine = false)
{
    if (check(dtype, M, K, N, FASTGL_ACT_SILU) != FASTGL_OK) return 0;
    const Shape d(dtype, M, K, N, aligned, fine);
    Layout l;
    if (backward || !d.few_rows()) carve(d, backward, l);
    if (aligned) return l.used;
    const size_t whole = workspace(dtype, M, K, N, true, backward, fine);      // the tiles may be taken from fewer rows on
    return l.used > whole ? l.used : whole;
}

fastgl_status gated_bwd(bool fine, fastgl_dtype dtype, const void *X, const void *Wg, const void *Wu, const void *G, const void *U,
                        const void *dP, int64_t M, int64_t K, int64_t N, fastgl_act act, void *dX, void *dWg, void *dWu, float *dbg,
                        float *dbu, void *ws, size_t ws_bytes, void *stream)
{
    fastgl_status st = check(dtype, M, K, N, act);
    if (st != FASTGL_OK) return st;
    const uintptr_t el = dtype == FASTGL_BF16 ? 2 : 4;
    const bool want_x = dX && M > 0 && K > 0, want_w = (dWg || dWu) && K > 0 && N > 0, want_b = (dbg || dbu) && N > 0;
    const bool terms = M > 0 && N > 0;
    if (terms && (want_x || want_w || want_b) && (!G || !U || !dP)) {
        set_error("G, U or dP is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (want_x && terms && (!Wg || !Wu)) {
        set_error("dX needs Wg and Wu");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (want_w && terms && !X) {
        set_error("dWg and dWu need X");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (misaligned_to(X, el) || misaligned_to(Wg, el) || misaligned_to(Wu, el) || misaligned_to(G, el) || misaligned_to(U, el) ||
        misaligned_to(dP, el) || misaligned_to(dX, el) || misaligned_to(dWg, el) || misaligned_to(dWu, el) || misaligned_to(dbg, 4) ||
        misaligned_to(dbu, 4)) {
        set_error("matrices must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    hipStream_t s = (hipStream_t)stream;
    if (!terms) {                                     // sums without terms
        const bool bf16 = dtype == FASTGL_BF16;
        if (want_x && (st = launch_no_terms(bf16, dX, nullptr, M, K, false, s, "fastgl_gated_bwd (dX, N = 0)")) != FASTGL_OK) return st;
        for (void *w : {dWg, dWu})
            if (w && want_w && (st = launch_no_terms(bf16, w, nullptr, K, N, false, s, "fastgl_gated_bwd (dW, M = 0)")) != FASTGL_OK) return st;
        for (float *b : {dbg, dbu})
            if (b && want_b && (st = launch_no_terms(false, b, nullptr, 1, N, false, s, "fastgl_gated_bwd (db, M = 0)")) != FASTGL_OK) return st;
        return FASTGL_OK;
    }
    if (!want_x && !want_w && !want_b) return FASTGL_OK;
    const Shape d(dtype, M, K, N, starts_whole({want_w ? X : nullptr, want_x ? Wg : nullptr, want_x ? Wu : nullptr}), fine);
    Layout l;
    carve(d, true, l);
    st = check_workspace(ws, ws_bytes, l.used);
    if (st != FASTGL_OK) return st;
    l = Layout();
    l.base = (char *)ws;
    const Scratch o = carve(d, true, l);

    DzArgs z = {};
    z.G = G; z.U = U; z.dP = dP;
    z.dG = want_x || want_w ? o.dg : nullptr;
    z.dU = o.du;
    z.M = M; z.plane = d.z_plane();
    z.N = (int32_t)N; z.lg = d.lg();
    z.ld = d.z_block() ? 32 : d.ldz;
    z.block = d.z_block() ? d.z_block() : 32;
    z.part = want_b ? o.db : nullptr;
    const dim3 dz((unsigned)d.dz_cols(), (unsigned)d.dz_rows());
    by_act(act, [&](auto A) {
        constexpr int ACT = decltype(A)::value;
        if (d.z_planes() == 1) hipLaunchKernelGGL((k_gated_dz<true, ACT, 1>), dz, dim3(kBlock), 0, s, z);
        else if (d.bf16) hipLaunchKernelGGL((k_gated_dz<true, ACT, 2>), dz, dim3(kBlock), 0, s, z);
        else hipLaunchKernelGGL((k_gated_dz<false, ACT, 3>), dz, dim3(kBlock), 0, s, z);
    });
    FASTGL_LAUNCH_CHECK("fastgl_gated_bwd (dG, dU)");
    SumArgs last = {};                                 // the sums at the end
    if (want_b) {
        last.db = o.db;
        last.dbg = dbg; last.dbu = dbu;
        last.rows = (int32_t)dz.y; last.N = (int32_t)N;
    }
    if ((st = pack(d, o, X, Wg, Wu, want_w, want_x, s)) != FASTGL_OK) return st;
    const std::integral_constant<int, 0> none;
    if (want_x) {
        TileArgs g = {};
        g.a[0] = o.dg; g.a[1] = o.du;
        g.b[0] = d.pack_w() ? o.wg : (const uint16_t *)Wg;
        g.b[1] = d.pack_w() ? o.wu : (const uint16_t *)Wu;
        g.a_plane = d.z_plane(); g.b_plane = K * d.ldn;
        g.lda = d.ldz; g.ldb = d.ldn;
        g.a_blocks = d.z_block();
        g.R = M; g.C = K; g.Kc = N;
        g.pairs = (int32_t)d.z_pairs(); g.groups = 2;
        g.planes_a = !d.bf16 ? kSixA : d.z_planes() == 2 ? kTwo : 0;
        g.planes_b = !d.bf16 ? kSixB : 0;
        g.out[0] = dX;
        g.part = o.part;
        const Cut cut = d.rows_cut();
        if ((st = launch_tile<kRows>(g, cut, d.bf16, none, s, "fastgl_gated_bwd (dX)")) != FASTGL_OK) return st;
        if (cut.slabs > 1) {
            SumArgs a = {};
            a.part = o.part; a.out[0] = dX;
            a.n = a.stride = M * K;
            a.slabs = (int32_t)cut.slabs; a.results = 1;
            if ((st = launch_sum(a, d.bf16, s, "fastgl_gated_bwd (dX, sums)")) != FASTGL_OK) return st;
        }
    }
    if (want_w) {
        TileArgs g = {};
        g.a[0] = d.pack_x() ? o.x : (const uint16_t *)X;
        g.b[0] = o.dg; g.b[1] = o.du;
        g.a_plane = M * d.ldk; g.b_plane = d.z_plane();
        g.lda = d.ldk; g.ldb = d.ldz;
        g.b_blocks = d.z_block();
        g.R = K; g.C = N; g.Kc = M;
        g.pairs = (int32_t)d.z_pairs(); g.groups = 1;
        g.planes_a = !d.bf16 ? kSixA : 0;
        g.planes_b = !d.bf16 ? kSixB : d.z_planes() == 2 ? kTwo : 0;
        g.out[0] = dWg; g.out[1] = dWu;
        g.part = o.part;
        const Cut cut = d.weights_cut();
        if ((st = launch_tile<kWeights>(g, cut, d.bf16, none, s, "fastgl_gated_bwd (dW)")) != FASTGL_OK) return st;
        if (cut.slabs > 1) {
            last.part = o.part;
            last.out[0] = dWg; last.out[1] = dWu;
            last.n = K * N; last.stride = 2 * K * N;
            last.slabs = (int32_t)cut.slabs; last.results = 2;
        }
    }
    if (want_b || last.results) return launch_sum(last, d.bf16, s, "fastgl_gated_bwd (sums)");
    return FASTGL_OK;
}

}  // namespace
}  // namespace fastgl

using namespace fastgl;

extern "C" {

size_t fastgl_gated_fwd_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned)
{
    return workspace(dtype, M, K, N, aligned != 0, false);
}

size_t fastgl_gated_bwd_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned)
{
    return workspace(dtype, M, K, N, aligned != 0, true);
}

size_t fastgl_gated_bwd_fine_workspace_bytes(fastgl_dtype dtype, int64_t M, int64_t K, int64_t N, int aligned)
{
    return workspace(dtype, M, K, N, aligned != 0, true, true);
}

fastgl_status fastgl_gated_fwd(fastgl_dtype dtype, const void *X, const void *Wg, const void *Wu, const float *bg,
                               const float *bu, int64_t M, int64_t K, int64_t N, fastgl_act act, void *P, void *G, void *U,
                               void *ws, size_t ws_bytes, void *stream)
{
    fastgl_status st = check(dtype, M, K, N, act);
    if (st != FASTGL_OK) return st;
    if (M == 0 || N == 0) return FASTGL_OK;
    if (!P || (K > 0 && (!X || !Wg || !Wu))) {
        set_error("X, Wg, Wu or P is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    const uintptr_t el = dtype == FASTGL_BF16 ? 2 : 4;
    if (misaligned_to(X, el) || misaligned_to(Wg, el) || misaligned_to(Wu, el) || misaligned_to(P, el) || misaligned_to(G, el) ||
        misaligned_to(U, el) || misaligned_to(bg, 4) || misaligned_to(bu, 4)) {
        set_error("matrices must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    hipStream_t s = (hipStream_t)stream;
    const Shape d(dtype, M, K, N, starts_whole({X, Wg, Wu}));
    if (d.few_rows()) {
        int lg = 3;                                     // strips as wide as leaves enough of them
        while (lg > 0 && ceil_div(N, (int64_t)8 << lg) < 192) --lg;
        const int rows = M == 1 ? 1 : M == 2 ? 2 : 4;
        RowsArgs a = {X, Wg, Wu, bg, bu, P, G, U, (int32_t)M, (int32_t)K, (int32_t)N, (int32_t)act, (int32_t)ceil_div(N, (int64_t)8 << lg),
                      (int32_t)ceil_div(M, rows)};
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(a.strips * a.groups)), dim3(kBlock), 0, s, a); };
        auto wide = [&](auto bf16, auto mr) {
            constexpr bool B = decltype(bf16)::value;
            constexpr int R = decltype(mr)::value;
            switch (lg) {
                case 0: go(k_gated_rows<B, R, 0>); break;
                case 1: go(k_gated_rows<B, R, 1>); break;
                case 2: go(k_gated_rows<B, R, 2>); break;
                default: go(k_gated_rows<B, R, 3>); break;
            }
        };
        auto typed = [&](auto bf16) {
            if (rows == 1) wide(bf16, std::integral_constant<int, 1>());
            else if (rows == 2) wide(bf16, std::integral_constant<int, 2>());
            else wide(bf16, std::integral_constant<int, 4>());
        };
        if (dtype == FASTGL_BF16) typed(std::true_type());
        else typed(std::false_type());
        FASTGL_LAUNCH_CHECK("fastgl_gated_fwd (few rows)");
        return FASTGL_OK;
    }
    Layout l;
    carve(d, false, l);
    st = check_workspace(ws, ws_bytes, l.used);
    if (st != FASTGL_OK) return st;
    l = Layout();
    l.base = (char *)ws;
    const Scratch o = carve(d, false, l);
    if ((st = pack(d, o, X, Wg, Wu, true, true, s)) != FASTGL_OK) return st;
    TileArgs g = {};
    g.a[0] = d.pack_x() ? o.x : (const uint16_t *)X;
    g.b[0] = d.pack_w() ? o.wg : (const uint16_t *)Wg;
    g.b[1] = d.pack_w() ? o.wu : (const uint16_t *)Wu;
    g.a_plane = M * d.ldk; g.b_plane = K * d.ldn;
    g.lda = d.ldk; g.ldb = d.ldn;
    g.R = M; g.C = N; g.Kc = K;
    g.pairs = (int32_t)d.pairs(); g.groups = 1;
    if (!d.bf16) {
        g.planes_a = kSixA;
        g.planes_b = kSixB;
    }
    g.bias[0] = bg; g.bias[1] = bu;
    g.out[0] = P; g.out[1] = G; g.out[2] = U;
    g.part = o.part;
    const Cut cut = d.forward_cut();
    by_act(act, [&](auto A) { st = launch_tile<kForward>(g, cut, d.bf16, A, s, "fastgl_gated_fwd"); });
    if (st != FASTGL_OK || cut.slabs == 1) return st;
    by_act(act, [&](auto A) {
        constexpr int ACT = decltype(A)::value;
        const dim3 grid((unsigned)ceil_div(M * N, kBlock));
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, (const float *)o.part, (int32_t)cut.slabs, M * N, (int32_t)N, bg, bu, P, G, U);
        };
        if (d.bf16) go(k_gated_join<true, ACT>);
        else go(k_gated_join<false, ACT>);
    });
    FASTGL_LAUNCH_CHECK("fastgl_gated_fwd (sum of slabs)");
    return FASTGL_OK;
}

fastgl_status fastgl_gated_bwd(fastgl_dtype dtype, const void *X, const void *Wg, const void *Wu, const void *G,
                               const void *U, const void *dP, int64_t M, int64_t K, int64_t N, fastgl_act act, void *dX,
                               void *dWg, void *dWu, float *dbg, float *dbu, void *ws, size_t ws_bytes, void *stream)
{
    return gated_bwd(false, dtype, X, Wg, Wu, G, U, dP, M, K, N, act, dX, dWg, dWu, dbg, dbu, ws, ws_bytes, stream);
}

fastgl_status fastgl_gated_bwd_fine(fastgl_dtype dtype, const void *X, const void *Wg, const void *Wu, const void *G,
                                    const void *U, const void *dP, int64_t M, int64_t K, int64_t N, fastgl_act act, void *dX,
                                    void *dWg, void *dWu, float *dbg, float *dbu, void *ws, size_t ws_bytes, void *stream)
{
    return gated_bwd(true, dtype, X, Wg, Wu, G, U, dP, M, K, N, act, dX, dWg, dWu, dbg, dbu, ws, ws_bytes, stream);
}

}  // extern "C"
