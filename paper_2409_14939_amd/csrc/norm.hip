// Root-mean-square norm of rows with the residual's addition and dropout in front of it, and its backward pass
// (fastgl_norm.h has the formulas).
//
// A row is read once: its columns stay in registers between the sum of squares and the result.  A lane holds eight
// columns at a time (one 16-byte word of bf16, two of fp32, one answer of the generator).  A row has 1 to 64 lanes
// of a wavefront, NC chunks each, and beyond 1536 columns a workgroup; beyond 8192 it is read twice (to 8 bits
// three times, backward with column sums three times).  Groups of lanes walk the rows with
// the grid's stride, so that the weights stay in registers and the backward pass keeps its column sums there.
//
// Bound by memory; a copy runs at 4.7 to 5.0 TB/s on the same cards.  us a call and TB/s of what has to move: 512 000 bf16 rows of 256
// with residual and dropout 207 (5.1); gradient of 115 000 fp32 rows of 602 with both 283 (4.9); 400 003 bf16 rows of 128 to 8 bits 37
// (4.2); plain norm of 115 000 bf16 rows of 602 47 (5.9).  One row: 1.9 us of kernel, the rest of a call is the host.
#include "fastgl_norm.h"
#include "rows_device.h"

#include <type_traits>

namespace fastgl {
namespace {

constexpr int kMaxGroupsOfRows = 2048;    // workgroups of a launch: eight per compute unit
constexpr int kReduceCols = 16;

struct NormArgs {
    const void *X, *R;
    const float *w;
    int64_t M;
    int32_t F;
    float eps, inv_F;
    const int64_t *rng;
    uint32_t threshold;
    float drop_scale;
    void *sum_out, *Y;
    float *row_scale, *rstd;
};

struct NormBwdArgs {
    const void *S, *dY, *dS;
    const float *w, *rstd;
    int64_t M;
    int32_t F;
    float inv_F;
    const int64_t *rng;
    uint32_t threshold;
    float drop_scale;
    void *dX, *dR;
    float *part;               // [workgroups][F] column sums of dY n, or NULL
};

// What load_row() read beyond the row counts as 0.
__device__ __forceinline__ void only(float (&v)[8], int left)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < left ? v[j] : 0.f;
}

struct Plus {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// The value of another lane of the same sixteen: CTRL 0xB1 the neighbour, 0x4E the neighbour pair's, 0x141 and 0x140 the
// mirrored place of eight and of sixteen (sums of four and of eight lanes, which their lanes all hold, meet their others).
template <int CTRL>
__device__ __forceinline__ float lane_of_16(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}

// Over the 2^LG lanes of a row (LG = 8: the workgroup, through `buf`, two halves in turn so that one barrier is
// enough); the order of the terms is fixed.
template <int LG, class OP>
__device__ __forceinline__ float row_reduce(float v, OP op, float (&buf)[2][4], int &turn)
{
    if constexpr (LG > 0) v = op(v, lane_of_16<0xB1>(v));
    if constexpr (LG > 1) v = op(v, lane_of_16<0x4E>(v));
    if constexpr (LG > 2) v = op(v, lane_of_16<0x141>(v));
    if constexpr (LG > 3) v = op(v, lane_of_16<0x140>(v));
    if constexpr (LG > 4) v = op(v, __shfl_xor(v, 16, kWave));
    if constexpr (LG > 5) v = op(v, __shfl_xor(v, 32, kWave));
    if constexpr (LG == 8) {
        if ((threadIdx.x & (kWave - 1)) == 0) buf[turn][threadIdx.x / kWave] = v;
        __syncthreads();
        v = op(op(buf[turn][0], buf[turn][1]), op(buf[turn][2], buf[turn][3]));
        turn ^= 1;
    }
    return v;
}

// The scale of a row of e4m3 values and quotients by it, all rounded as a division rounds them: the product with the rounded reciprocal,
// then what that leaves of the dividend (exact), times the reciprocal.  us a call for 400 003 bf16 rows of 128, by divisions 46, so 37, by
// the product alone 34, which stores a value or two in 10^7 of normal data a step off.
struct RowScale {
    float scale, s, inv;
    bool tiny;
    __device__ __forceinline__ explicit RowScale(float most)
    {
        const float q = most * (1.f / 448.f);
        scale = fmaxf(most < __builtin_inff() ? fmaf(fmaf(-q, 448.f, most), 1.f / 448.f, q) : most, 0x1p-126f);
        tiny = scale < 0x1p-90f;                        // what is left would not be a whole number of the least subnormal
        s = tiny ? scale * 0x1p64f : scale;
        inv = 1.f / s;
        s = inv > 0.f ? s : 0.f;                        // an infinite scale: the product alone, 0 (or NaN)
    }
    __device__ __forceinline__ void divide(float (&v)[8]) const
    {
        if (tiny) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= 0x1p64f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float q = v[j] * inv;
            v[j] = fmaf(fmaf(-q, s, v[j]), inv, q);
        }
    }
};

// y of eight columns as e4m3.
__device__ __forceinline__ void store_e4m3(uint8_t *p, const float (&v)[8], int left)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(1)));
    int a = 0, b = 0;
    a = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], a, false);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], a, true);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], b, false);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], b, true);
    if (left >= 8) {
        *reinterpret_cast<u32x2 *>(p) = u32x2{(uint32_t)a, (uint32_t)b};
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < left) p[j] = (uint8_t)((uint32_t)(j < 4 ? a : b) >> (8 * (j & 3)));
    }
}

template <bool BF16, int LG, int NC, bool DROP, bool E4M3>
__global__ __launch_bounds__(kBlock) void k_norm(NormArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    constexpr int LANES = 1 << LG, ROWS = kBlock >> LG;
    __shared__ float buf[2][4];
    int turn = 0;
    const int lane = threadIdx.x & (LANES - 1), F = a.F;
    const T *X = static_cast<const T *>(a.X), *R = static_cast<const T *>(a.R);
    Philox gen;
    if constexpr (DROP) gen.load(a.rng);
    float w[NC][8];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        Chunk<false> q;
        const int col = (c * LANES + lane) * kChunk;
        q.load(a.w + col, F - col);
        q.get(w[c]);
    }
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const bool ragged = F % kChunk != 0;
    // the rows of a step; the next step's are under way while this one's are worked on, where registers allow
    auto fetch = [&](int64_t row0, Chunk<BF16>(&x)[NC], Chunk<BF16>(&r)[NC]) {
        const int64_t row = row0 + (threadIdx.x >> LG), at = row * F;
        // of the rows of a wavefront, each of an element at least, the last is followed by eight
        const bool inside = row0 + (int64_t)wave_first(LG) + (kWave >> (LG < 6 ? LG : 6)) + kChunk <= a.M;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * LANES + lane) * kChunk;
            load_row(x[c], X, at + col, row < a.M ? F - col : 0, inside);
        }
        if (R) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (c * LANES + lane) * kChunk;
                load_row(r[c], R, at + col, row < a.M ? F - col : 0, inside);
            }
        }
    };
    constexpr bool AHEAD = BF16 ? NC <= 3 : NC == 1;
    Chunk<BF16> x[NC], r[NC], next_x[NC], next_r[NC];
    if (AHEAD) fetch((int64_t)blockIdx.x * ROWS, next_x, next_r);
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.M; row0 += step) {
        const int64_t row = row0 + (threadIdx.x >> LG), at = row * F;
        const bool live = row < a.M;                                  // no row: nothing is read or written
        if (AHEAD) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                x[c] = next_x[c];
                r[c] = next_r[c];
            }
            if (row0 + step < a.M) fetch(row0 + step, next_x, next_r);
        } else
            fetch(row0, x, r);
        float h[NC][8], sq = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * LANES + lane) * kChunk;
            uint32_t words[4];
            if constexpr (DROP) gen.words((uint32_t)(col / kChunk), (uint32_t)row, words);
            x[c].get(h[c]);
            if constexpr (DROP) drop8(h[c], words, a.threshold, a.drop_scale);
            if (R) {
                float v[8];
                r[c].get(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[c][j] += v[j];
            }
            if (ragged) only(h[c], live ? F - col : 0);
            if (a.sum_out) Chunk<BF16>::store(static_cast<T *>(a.sum_out) + at + col, h[c], live ? F - col : 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) sq = fmaf(h[c][j], h[c][j], sq);
        }
        sq = row_reduce<LG>(sq, Plus(), buf, turn);
        const float rstd = 1.f / sqrtf(sq * a.inv_F + a.eps);
        if (a.rstd && lane == 0 && live) a.rstd[row] = rstd;
        float most = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[c][j] = h[c][j] * rstd * w[c][j];
                if constexpr (E4M3) most = fmaxf(most, fabsf(h[c][j]));
            }
        if constexpr (E4M3) {
            most = row_reduce<LG>(most, Max(), buf, turn);
            const RowScale by(most);
            if (lane == 0 && live) a.row_scale[row] = by.scale;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (c * LANES + lane) * kChunk;
                by.divide(h[c]);
                store_e4m3(static_cast<uint8_t *>(a.Y) + at + col, h[c], live ? F - col : 0);
            }
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (c * LANES + lane) * kChunk;
                Chunk<BF16>::store(static_cast<T *>(a.Y) + at + col, h[c], live ? F - col : 0);
            }
        }
    }
}

// Rows beyond what registers hold: one workgroup a row, h formed in every pass over it.
template <bool BF16, bool DROP, bool E4M3>
__global__ __launch_bounds__(kBlock) void k_norm_wide(NormArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    __shared__ float buf[2][4];
    int turn = 0;
    const int F = a.F;
    const T *X = static_cast<const T *>(a.X), *R = static_cast<const T *>(a.R);
    Philox gen;
    if constexpr (DROP) gen.load(a.rng);
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
        const int64_t at = row * F;
        auto sum = [&](int col, float(&h)[8]) {
            Chunk<BF16> x;
            x.load(X + at + col, F - col);
            x.get(h);
            if constexpr (DROP) {
                uint32_t words[4];
                gen.words((uint32_t)(col / kChunk), (uint32_t)row, words);
                drop8(h, words, a.threshold, a.drop_scale);
            }
            if (R) {
                float v[8];
                x.load(R + at + col, F - col);
                x.get(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[j] += v[j];
            }
        };
        auto scaled = [&](int col, float rstd, float(&h)[8]) {
            float w[8];
            Chunk<false> q;
            q.load(a.w + col, F - col);
            q.get(w);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = h[j] * rstd * w[j];
        };
        float sq = 0.f;
        for (int col = threadIdx.x * kChunk; col < F; col += kBlock * kChunk) {
            float h[8];
            sum(col, h);
            if (a.sum_out) Chunk<BF16>::store(static_cast<T *>(a.sum_out) + at + col, h, F - col);
#pragma unroll
            for (int j = 0; j < 8; ++j) sq = fmaf(h[j], h[j], sq);
        }
        sq = row_reduce<8>(sq, Plus(), buf, turn);
        const float rstd = 1.f / sqrtf(sq * a.inv_F + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
        float most = 0.f;
        if constexpr (E4M3) {
            for (int col = threadIdx.x * kChunk; col < F; col += kBlock * kChunk) {
                float h[8];
                sum(col, h);
                scaled(col, rstd, h);
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(h[j]));
            }
            most = row_reduce<8>(most, Max(), buf, turn);
        }
        const RowScale by(most);
        if constexpr (E4M3)
            if (threadIdx.x == 0) a.row_scale[row] = by.scale;
        for (int col = threadIdx.x * kChunk; col < F; col += kBlock * kChunk) {
            float h[8];
            sum(col, h);
            scaled(col, rstd, h);
            if constexpr (E4M3) {
                by.divide(h);
                store_e4m3(static_cast<uint8_t *>(a.Y) + at + col, h, F - col);
            } else
                Chunk<BF16>::store(static_cast<T *>(a.Y) + at + col, h, F - col);
        }
    }
}

// ------------------------------------------------------------------------------------ backward
template <bool BF16, int LG, int NC, bool DROP>
__global__ __launch_bounds__(kBlock) void k_norm_bwd(NormBwdArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    constexpr int LANES = 1 << LG, ROWS = kBlock >> LG;
    __shared__ float buf[2][4];
    int turn = 0;
    const int lane = threadIdx.x & (LANES - 1), F = a.F;
    const T *S = static_cast<const T *>(a.S), *dY = static_cast<const T *>(a.dY), *dS = static_cast<const T *>(a.dS);
    Philox gen;
    if constexpr (DROP) gen.load(a.rng);
    float w[NC][8], dw[NC][8];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        Chunk<false> q;
        const int col = (c * LANES + lane) * kChunk;
        q.load(a.w + col, F - col);
        q.get(w[c]);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[c][j] = 0.f;
    }
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const bool ragged = F % kChunk != 0;
    auto fetch = [&](int64_t row0, Chunk<BF16>(&qs)[NC], Chunk<BF16>(&qy)[NC], Chunk<BF16>(&qd)[NC], float &rstd) {
        const int64_t row = row0 + (threadIdx.x >> LG), at = row * F;
        const bool inside = row0 + (int64_t)wave_first(LG) + (kWave >> (LG < 6 ? LG : 6)) + kChunk <= a.M;
        rstd = row < a.M ? a.rstd[row] : 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * LANES + lane) * kChunk, left = row < a.M ? F - col : 0;
            load_row(qs[c], S, at + col, left, inside);
            load_row(qy[c], dY, at + col, left, inside);
        }
        if (dS) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (c * LANES + lane) * kChunk;
                load_row(qd[c], dS, at + col, row < a.M ? F - col : 0, inside);
            }
        }
    };
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.M; row0 += step) {
        const int64_t row = row0 + (threadIdx.x >> LG), at = row * F;
        const bool live = row < a.M;
        Chunk<BF16> qs[NC], qy[NC], qd[NC];
        float rstd;
        fetch(row0, qs, qy, qd, rstd);                               // loading a step ahead gained nothing here
        float n[NC][8], t[NC][8], dot = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            qs[c].get(n[c]);
            qy[c].get(t[c]);
            if (ragged) {
                only(n[c], F - (c * LANES + lane) * kChunk);
                only(t[c], F - (c * LANES + lane) * kChunk);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                n[c][j] *= rstd;
                dw[c][j] = fmaf(t[c][j], n[c][j], dw[c][j]);
                t[c][j] *= w[c][j];
                dot = fmaf(t[c][j], n[c][j], dot);
            }
        }
        dot = row_reduce<LG>(dot, Plus(), buf, turn) * a.inv_F;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * LANES + lane) * kChunk;
            float d[8];
            if (dS) qd[c].get(d);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = fmaf(rstd, t[c][j] - n[c][j] * dot, d[j]);
            if (a.dR) Chunk<BF16>::store(static_cast<T *>(a.dR) + at + col, d, live ? F - col : 0);
            if (a.dX) {
                if constexpr (DROP) {
                    uint32_t words[4];
                    gen.words((uint32_t)(col / kChunk), (uint32_t)row, words);
                    drop8(d, words, a.threshold, a.drop_scale);
                }
                Chunk<BF16>::store(static_cast<T *>(a.dX) + at + col, d, live ? F - col : 0);
            }
        }
    }
    if (!a.part) return;
    // the column sums of the workgroup's groups of lanes, in the order of the groups
    if constexpr (LG == 8) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * LANES + lane) * kChunk;
            Chunk<false>::store(a.part + (int64_t)blockIdx.x * F + col, dw[c], F - col);
        }
    } else {
        constexpr int STRIDE = LANES * kChunk + 4;
        __shared__ float sums[4][STRIDE];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int o = LANES; o < kWave; o <<= 1) dw[c][j] += __shfl_xor(dw[c][j], o, kWave);
            __syncthreads();
            if ((threadIdx.x & (kWave - 1)) < LANES)
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[threadIdx.x / kWave][lane * kChunk + j] = dw[c][j];
            __syncthreads();
            for (int i = threadIdx.x; i < LANES * kChunk; i += kBlock) {
                const int col = c * LANES * kChunk + i;
                if (col < F) a.part[(int64_t)blockIdx.x * F + col] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
            }
        }
    }
}

// Rows beyond what registers hold.  Column sums: a second kernel over the rows (k_norm_dw_wide).
template <bool BF16, bool DROP>
__global__ __launch_bounds__(kBlock) void k_norm_bwd_wide(NormBwdArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    __shared__ float buf[2][4];
    int turn = 0;
    const int F = a.F;
    const T *S = static_cast<const T *>(a.S), *dY = static_cast<const T *>(a.dY), *dS = static_cast<const T *>(a.dS);
    Philox gen;
    if constexpr (DROP) gen.load(a.rng);
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
        const int64_t at = row * F;
        const float rstd = a.rstd[row];
        auto terms = [&](int col, float(&n)[8], float(&t)[8]) {
            Chunk<BF16> q;
            Chunk<false> qw;
            float w[8];
            q.load(S + at + col, F - col);
            q.get(n);
            q.load(dY + at + col, F - col);
            q.get(t);
            qw.load(a.w + col, F - col);
            qw.get(w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                n[j] *= rstd;
                t[j] *= w[j];
            }
        };
        float dot = 0.f;
        for (int col = threadIdx.x * kChunk; col < F; col += kBlock * kChunk) {
            float n[8], t[8];
            terms(col, n, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) dot = fmaf(t[j], n[j], dot);
        }
        dot = row_reduce<8>(dot, Plus(), buf, turn) * a.inv_F;
        for (int col = threadIdx.x * kChunk; col < F; col += kBlock * kChunk) {
            float n[8], t[8], d[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            terms(col, n, t);
            if (dS) {
                Chunk<BF16> q;
                q.load(dS + at + col, F - col);
                q.get(d);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = fmaf(rstd, t[j] - n[j] * dot, d[j]);
            if (a.dR) Chunk<BF16>::store(static_cast<T *>(a.dR) + at + col, d, F - col);
            if (a.dX) {
                if constexpr (DROP) {
                    uint32_t words[4];
                    gen.words((uint32_t)(col / kChunk), (uint32_t)row, words);
                    drop8(d, words, a.threshold, a.drop_scale);
                }
                Chunk<BF16>::store(static_cast<T *>(a.dX) + at + col, d, F - col);
            }
        }
    }
}

// part[y][col] = sum over the rows y, y + gridDim.y, ... of dY n: wide rows, a workgroup holds 2048 columns.
template <bool BF16>
__global__ __launch_bounds__(kBlock) void k_norm_dw_wide(NormBwdArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    const int F = a.F, col = (int)(blockIdx.x * kBlock + threadIdx.x) * kChunk;
    if (col >= F) return;
    float dw[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t row = blockIdx.y; row < a.M; row += gridDim.y) {
        Chunk<BF16> q;
        float n[8], y[8];
        const float rstd = a.rstd[row];
        q.load(static_cast<const T *>(a.S) + row * F + col, F - col);
        q.get(n);
        q.load(static_cast<const T *>(a.dY) + row * F + col, F - col);
        q.get(y);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[j] = fmaf(y[j], n[j] * rstd, dw[j]);
    }
    Chunk<false>::store(a.part + (int64_t)blockIdx.y * F + col, dw, F - col);
}

// dw[col] = sum of part[0 .. n)[col] in fp64: 16 columns a workgroup, 64 threads a column, a fixed order.
__global__ __launch_bounds__(1024) void k_norm_dw(const float *__restrict__ part, int32_t n, int32_t F, float *__restrict__ dw)
{
    __shared__ double sums[64][kReduceCols + 1];
    const int c = threadIdx.x % kReduceCols, s = threadIdx.x / kReduceCols;
    const int col = blockIdx.x * kReduceCols + c;
    double v = 0.0;
    if (col < F) {
#pragma unroll 8
        for (int i = s; i < n; i += 64) v += (double)part[(int64_t)i * F + col];
    }
    sums[s][c] = v;
    __syncthreads();
    if (s < 8) {
        v = 0.0;
        for (int i = 0; i < 8; ++i) v += sums[s * 8 + i][c];
    }
    __syncthreads();
    if (s < 8) sums[s][c] = v;
    __syncthreads();
    if (s == 0 && col < F) {
        v = 0.0;
        for (int i = 0; i < 8; ++i) v += sums[i][c];
        dw[col] = (float)v;
    }
}

// ------------------------------------------------------------------------------------ host side
// How a row of F columns is spread over lanes: f(integral_constant LG, integral_constant NC); false beyond registers.  As few lanes as have
// columns: us a call, 1 M rows, residual and dropout, eight lanes / two for 16 columns, four for 32: bf16 44.0 / 22.7, 50.9 / 42.4; fp32 60.7 / 45.6,
// 108 / 101; backward bf16 59.6 / 33.1, 70.7 / 63.4, fp32 74.7 / 63.0, 131 / 129.
template <class GO>
bool spread(int64_t F, GO go)
{
    const int64_t chunks = ceil_div(F, kChunk);
    auto is = [&](auto lg, auto nc) {
        go(lg, nc);
        return true;
    };
    using std::integral_constant;
    if (chunks <= 1) return is(integral_constant<int, 0>(), integral_constant<int, 1>());
    if (chunks <= 2) return is(integral_constant<int, 1>(), integral_constant<int, 1>());
    if (chunks <= 4) return is(integral_constant<int, 2>(), integral_constant<int, 1>());
    if (chunks <= 8) return is(integral_constant<int, 3>(), integral_constant<int, 1>());
    if (chunks <= 16) return is(integral_constant<int, 4>(), integral_constant<int, 1>());
    if (chunks <= 24) return is(integral_constant<int, 3>(), integral_constant<int, 3>());
    if (chunks <= 32) return is(integral_constant<int, 5>(), integral_constant<int, 1>());
    if (chunks <= 48) return is(integral_constant<int, 4>(), integral_constant<int, 3>());
    if (chunks <= 64) return is(integral_constant<int, 6>(), integral_constant<int, 1>());
    if (chunks <= 96) return is(integral_constant<int, 5>(), integral_constant<int, 3>());
    if (chunks <= 128) return is(integral_constant<int, 6>(), integral_constant<int, 2>());
    if (chunks <= 192) return is(integral_constant<int, 6>(), integral_constant<int, 3>());
    if (chunks <= 256) return is(integral_constant<int, 8>(), integral_constant<int, 1>());
    if (chunks <= 512) return is(integral_constant<int, 8>(), integral_constant<int, 2>());
    if (chunks <= 1024) return is(integral_constant<int, 8>(), integral_constant<int, 4>());
    return false;
}

int rows_per_group(int64_t F)
{
    int rows = 1;
    spread(F, [&](auto lg, auto) { rows = kBlock >> decltype(lg)::value; });
    return rows;
}

// Workgroups of the backward pass that leave column sums: one has eight rows at least, so that the sums are little beside the
// rows, unless that leaves compute units without one.
int64_t bwd_groups(int64_t M, int64_t F)
{
    const int64_t most = ceil_div(M, rows_per_group(F)), some = ceil_div(M, 8);
    const int64_t enough = some > 256 ? some : 256, n = most < enough ? most : enough;
    return n < kMaxGroupsOfRows ? n : kMaxGroupsOfRows;
}

bool misaligned_to(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

fastgl_status check_rows(fastgl_dtype dtype, int64_t M, int64_t F, const int64_t *rng, double p, uint32_t *threshold, float *scale)
{
    if (dtype != FASTGL_F32 && dtype != FASTGL_BF16) {
        set_error("bad dtype %d", (int)dtype);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (M < 0 || F < 1) {
        set_error("negative size or no columns (M=%lld F=%lld)", (long long)M, (long long)F);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (M > kMaxIndex || F > (int64_t)1 << 24) {
        set_error("M must stay below 2^31-1-1024 and F at 2^24 or below");
        return FASTGL_ERR_UNSUPPORTED;
    }
    if (!drop_constants(p, threshold, scale)) {
        set_error("the dropout probability must be in [0, 1]");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (p > 0.0 && (!rng || misaligned_to(rng, 8))) {
        set_error("dropout needs rng: two int64 {seed, offset} in device memory, aligned to 8 bytes");
        return FASTGL_ERR_INVALID_ARG;
    }
    return FASTGL_OK;
}

fastgl_status norm_fwd(bool e4m3, fastgl_dtype dtype, const void *X, const void *R, const float *w, int64_t M, int64_t F,
                       float eps, const int64_t *rng, double p, void *sum_out, void *Y, float *row_scale, float *rstd, hipStream_t s)
{
    NormArgs a = {};
    const fastgl_status st = check_rows(dtype, M, F, rng, p, &a.threshold, &a.drop_scale);
    if (st != FASTGL_OK) return st;
    if (!(eps >= 0.f) || eps > 3.4e38f) {
        set_error("eps must be finite and not negative");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (M == 0) return FASTGL_OK;
    const uintptr_t el = dtype == FASTGL_BF16 ? 2 : 4;
    if (!X || !w || !Y || (e4m3 && !row_scale)) {
        set_error("X, w or an output is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (misaligned_to(X, el) || misaligned_to(R, el) || misaligned_to(sum_out, el) || misaligned_to(Y, e4m3 ? 1 : el) ||
        misaligned_to(w, 4) || misaligned_to(rstd, 4) || misaligned_to(row_scale, 4)) {
        set_error("arrays must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    a.X = X; a.R = R; a.w = w;
    a.M = M; a.F = (int32_t)F;
    a.eps = eps; a.inv_F = (float)(1.0 / (double)F);
    a.rng = rng;
    a.sum_out = sum_out; a.Y = Y; a.row_scale = row_scale; a.rstd = rstd;
    const int64_t groups = ceil_div(M, rows_per_group(F));
    const dim3 grid((unsigned)(groups < kMaxGroupsOfRows ? groups : kMaxGroupsOfRows));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, a); };
    auto typed = [&](auto bf16, auto drop, auto to8) {
        constexpr bool B = decltype(bf16)::value, D = decltype(drop)::value, E = decltype(to8)::value;
        if (!spread(F, [&](auto lg, auto nc) { go(k_norm<B, decltype(lg)::value, decltype(nc)::value, D, E>); }))
            go(k_norm_wide<B, D, E>);
    };
    auto dropped = [&](auto bf16, auto drop) { e4m3 ? typed(bf16, drop, std::true_type()) : typed(bf16, drop, std::false_type()); };
    auto both = [&](auto bf16) { p > 0.0 ? dropped(bf16, std::true_type()) : dropped(bf16, std::false_type()); };
    if (dtype == FASTGL_BF16) both(std::true_type());
    else both(std::false_type());
    FASTGL_LAUNCH_CHECK("fastgl_norm_fwd");
    return FASTGL_OK;
}

}  // namespace
}  // namespace fastgl

using namespace fastgl;

extern "C" {

fastgl_status fastgl_norm_fwd(fastgl_dtype dtype, const void *X, const void *R, const float *w, int64_t M, int64_t F,
                              float eps, const int64_t *rng, double p, void *sum_out, void *Y, float *rstd, void *stream)
{
    return norm_fwd(false, dtype, X, R, w, M, F, eps, rng, p, sum_out, Y, nullptr, rstd, (hipStream_t)stream);
}

fastgl_status fastgl_norm_fwd_e4m3(fastgl_dtype dtype, const void *X, const void *R, const float *w, int64_t M, int64_t F,
                                   float eps, const int64_t *rng, double p, void *sum_out, uint8_t *Q, float *scale,
                                   float *rstd, void *stream)
{
    return norm_fwd(true, dtype, X, R, w, M, F, eps, rng, p, sum_out, Q, scale, rstd, (hipStream_t)stream);
}

size_t fastgl_norm_bwd_workspace_bytes(int64_t M, int64_t F)
{
    if (M < 0 || F < 1 || M > kMaxIndex || F > (int64_t)1 << 24) return 0;
    return align_up((size_t)bwd_groups(M, F) * (size_t)F * sizeof(float), 256);
}

fastgl_status fastgl_norm_bwd(fastgl_dtype dtype, const void *S, const float *w, const float *rstd, const void *dY,
                              const void *dS, int64_t M, int64_t F, const int64_t *rng, double p, void *dX, void *dR,
                              float *dw, void *workspace, size_t workspace_bytes, void *stream)
{
    NormBwdArgs a = {};
    const fastgl_status st = check_rows(dtype, M, F, rng, p, &a.threshold, &a.drop_scale);
    if (st != FASTGL_OK) return st;
    const uintptr_t el = dtype == FASTGL_BF16 ? 2 : 4;
    if (M > 0 && (!S || !w || !rstd || !dY)) {
        set_error("S, w, rstd or dY is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (misaligned_to(S, el) || misaligned_to(dY, el) || misaligned_to(dS, el) || misaligned_to(dX, el) || misaligned_to(dR, el) ||
        misaligned_to(w, 4) || misaligned_to(rstd, 4) || misaligned_to(dw, 4)) {
        set_error("arrays must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (dw && M > 0) {
        if (!workspace || misaligned_to(workspace, 256)) {
            set_error("workspace must be a 256-byte aligned device buffer");
            return FASTGL_ERR_INVALID_ARG;
        }
        if (workspace_bytes < fastgl_norm_bwd_workspace_bytes(M, F)) {
            set_error("workspace too small: %zu < %zu bytes", workspace_bytes, fastgl_norm_bwd_workspace_bytes(M, F));
            return FASTGL_ERR_WORKSPACE;
        }
    }
    if (!dX && !dR && !dw) return FASTGL_OK;
    hipStream_t s = (hipStream_t)stream;
    a.S = S; a.dY = dY; a.dS = dS;
    a.w = w; a.rstd = rstd;
    a.M = M; a.F = (int32_t)F;
    a.inv_F = (float)(1.0 / (double)F);
    a.rng = rng;
    a.dX = dX; a.dR = dR;
    a.part = dw ? (float *)workspace : nullptr;
    const int64_t groups = bwd_groups(M, F);
    if (M > 0) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kBlock), 0, s, a); };
        auto typed = [&](auto bf16, auto drop) {
            constexpr bool B = decltype(bf16)::value, D = decltype(drop)::value;
            if (spread(F, [&](auto lg, auto nc) { go(k_norm_bwd<B, decltype(lg)::value, decltype(nc)::value, D>); })) return;
            if (dX || dR) go(k_norm_bwd_wide<B, D>);
            if (dw)
                hipLaunchKernelGGL(k_norm_dw_wide<B>, dim3((unsigned)ceil_div(F, kBlock * kChunk), (unsigned)groups),
                                   dim3(kBlock), 0, s, a);
        };
        auto both = [&](auto bf16) { p > 0.0 ? typed(bf16, std::true_type()) : typed(bf16, std::false_type()); };
        if (dtype == FASTGL_BF16) both(std::true_type());
        else both(std::false_type());
        FASTGL_LAUNCH_CHECK("fastgl_norm_bwd");
    }
    if (dw) {
        hipLaunchKernelGGL(k_norm_dw, dim3((unsigned)ceil_div(F, kReduceCols)), dim3(1024), 0, s, (const float *)workspace,
                           (int32_t)(M > 0 ? groups : 0), (int32_t)F, dw);
        FASTGL_LAUNCH_CHECK("fastgl_norm_bwd (dw)");
    }
    return FASTGL_OK;
}

}  // extern "C"
