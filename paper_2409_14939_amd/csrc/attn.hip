// Attention over the sampled neighbours of a block, forward and backward (fastgl_attn.h has the formulas).
//
//   forward   k_attn_fwd (rows, and chunks of long rows) -> [k_attn_join: chunks to rows]
//   backward  k_attn_dq  (the same walk: dQ, and maximum, sum and sum p dp of every row) -> [k_attn_join]
//             k_attn_dkv (rows of the transposed block: dK, dV; ds of every edge where dbias is wanted) -> [k_attn_join]
//             k_attn_dbias -> k_attn_dbias_sum
//
// A group of lanes has one row and one head, 16 bytes of the head a lane whatever its width and alignment: the last lane's piece
// ends with the head, and what it has in common with the one before counts once in a dot product (it is 0 in the row's own operand) and is
// the same in both lanes' sums.  A group walks its row's edges some at a time: the dot products are joined across its lanes, the running
// maximum is raised once for all of them, and the sums stay in registers.
//
// The backward pass forms maximum and sum of every row again, with dQ: rounded to one number (the forward pass's lse) they lose the sum where
// scores are large (a row of scores of -1e9, or of the type's lowest value, has weights 1 / n, and exp(s - lse) = 1).
#include <type_traits>

#include "fastgl_attn.h"
#include "internal.h"

namespace fastgl {
namespace {

constexpr float kLog2e = 1.44269504089f, kLn2 = 0.69314718056f;
constexpr int kAttnUnroll = 4;            // edges a group has under way
constexpr int kBiasBlocks = 1024;         // workgroups of k_attn_dbias
constexpr int kBiasTile = 64;             // buckets of one of its passes

// ------------------------------------------------------------------ lanes and pieces
template <bool BF16, bool WHOLE>
struct Piece;

template <>
struct Piece<false, true> {
    typedef float elem;
    static constexpr int N = 4;
    Words<4>::x4 w;
    __device__ __forceinline__ void load(const float *p) { w = *reinterpret_cast<const Words<4>::x4 *>(p); }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(w[i]); }
    __device__ __forceinline__ void keep(bool on)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = on ? w[i] : 0u;
    }
    __device__ static __forceinline__ void store(float *p, const float (&v)[4])
    {
        *reinterpret_cast<Words<4>::x4 *>(p) = Words<4>::x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
};

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

template <>
struct Piece<true, true> {
    typedef uint16_t elem;
    static constexpr int N = 8;
    Words<2>::x4 w;
    __device__ __forceinline__ void load(const uint16_t *p) { w = *reinterpret_cast<const Words<2>::x4 *>(p); }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16); }
    __device__ __forceinline__ void keep(bool on)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = on ? w[i] : 0u;
    }
    __device__ static __forceinline__ void store(uint16_t *p, const float (&v)[8])
    {
        *reinterpret_cast<Words<2>::x4 *>(p) = Words<2>::x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
    }
};

// Heads narrower than 16 bytes: an element a lane.
template <>
struct Piece<false, false> {
    typedef float elem;
    static constexpr int N = 1;
    float w;
    __device__ __forceinline__ void load(const float *p) { w = *p; }
    __device__ __forceinline__ float get(int) const { return w; }
    __device__ __forceinline__ void keep(bool on) { w = on ? w : 0.f; }
    __device__ static __forceinline__ void store(float *p, const float (&v)[1]) { *p = v[0]; }
};

template <>
struct Piece<true, false> {
    typedef uint16_t elem;
    static constexpr int N = 1;
    uint32_t w;
    __device__ __forceinline__ void load(const uint16_t *p) { w = *p; }
    __device__ __forceinline__ float get(int) const { return __uint_as_float(w << 16); }
    __device__ __forceinline__ void keep(bool on) { w = on ? w : 0u; }
    __device__ static __forceinline__ void store(uint16_t *p, const float (&v)[1]) { *p = __builtin_bit_cast(uint16_t, (__bf16)v[0]); }
};

// exp(x) of a difference of scores, x <= 0: 2^(x log2 e).  Relative error 2^-23 (1 + |x|).
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// x + x of the lane across: the first four exchanges stay within sixteen lanes and need no LDS.  After them both lanes of a pair
// hold the same sum, so that mirrored lanes are as good as those across.
template <int CTRL>
__device__ __forceinline__ float plus_dpp(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}

template <int LG>
__device__ __forceinline__ float over_lanes(float v)
{
    if constexpr (LG > 0) v = plus_dpp<0xB1>(v);          // lanes 1, 0, 3, 2 of four
    if constexpr (LG > 1) v = plus_dpp<0x4E>(v);          // 2, 3, 0, 1
    if constexpr (LG > 2) v = plus_dpp<0x141>(v);         // eight lanes mirrored
    if constexpr (LG > 3) v = plus_dpp<0x140>(v);         // sixteen lanes mirrored
    if constexpr (LG > 4) v += __shfl_xor(v, 16, kWave);
    if constexpr (LG > 5) v += __shfl_xor(v, 32, kWave);
    return v;
}

struct AttnArgs {
    const int32_t *ptr, *col;      // rows of the block, or of its transpose
    const int32_t *eid;            // transposed: the edge's number in edge order; NULL: the position is the number
    const int32_t *bucket;         // or NULL
    const float *bias;             // or NULL
    const void *Q, *K, *V, *dO;
    int64_t ldq, ldk, ldv, lddo;
    typedef float f4 __attribute__((ext_vector_type(4)));
    f4 *stats;                     // [num_dst][heads]: maximum, 1 / sum, sum p dp of a row
    void *O, *dQ, *dK, *dV;        // or NULL
    int64_t ldo, lddq, lddk, lddv;
    float *lse;                    // [rows][heads], or NULL
    float *ds;                     // [position][heads], or NULL
    int64_t units;                 // rows x heads (transposed: x key heads)
    uint64_t heads_inv;            // ceil(2^64 / heads of a unit), 0 for one
    uint32_t shared_inv;           // ceil(2^32 / shared), 0 for one: exact for 2^20 query heads of edges at most 4096 of which share
    uint32_t buckets;              // edges of this bucket and above are left out
    int32_t heads, unit_heads, shared, width;
    float scale;
    int32_t long_thr;              // rows of more edges are taken in chunks
    const int32_t *long_rows, *chunk_ptr, *n_long, *n_chunks;
    float *part, *part_more;       // sums of chunks: [chunk][unit head][width], and what else a pass has
    int32_t chunk_blocks;          // workgroups that take chunks, before those of the rows
    int64_t part_stride;           // between the two arrays of `part` that a backward pass has
};

// Where a lane is: its group's place in the workgroup and its piece of a head.
template <class P, int LG, bool WHOLE>
struct Where {
    int l, g, off, skip;
    bool active;
    __device__ __forceinline__ Where(int width)
    {
        l = threadIdx.x & ((1 << LG) - 1);
        g = threadIdx.x >> LG;
        const int at = l * P::N, last = width - P::N;
        off = at < last ? at : last;
        skip = at - off;                              // elements that the lane before has too; all of them beyond the head
        active = at < width;
    }
    // This row's own operand, times `by`; 0 where another lane has it.
    __device__ __forceinline__ void own(const typename P::elem *p, float by, float (&v)[P::N]) const
    {
        P x;
        x.load(p + off);
#pragma unroll
        for (int i = 0; i < P::N; ++i) v[i] = i >= skip ? x.get(i) * by : 0.f;
    }
};

__device__ __forceinline__ uint64_t over(uint64_t n, uint64_t inv) { return inv ? __umul64hi(n, inv) : n; }
__device__ __forceinline__ uint32_t over(uint32_t n, uint32_t inv) { return inv ? __umulhi(n, inv) : n; }

// The chunk's row and its edges.
struct ChunkOf {
    int row, beg, end;
    __device__ __forceinline__ ChunkOf(const AttnArgs &a, int chunk, int n_long)
    {
        int lo = 0, hi = n_long;                      // chunk_ptr[lo] <= chunk < chunk_ptr[hi]
        while (hi - lo > 1) {
            const int mid = lo + ((hi - lo) >> 1);
            if (a.chunk_ptr[mid] <= chunk) lo = mid; else hi = mid;
        }
        row = a.long_rows[lo];
        beg = a.ptr[row] + (chunk - a.chunk_ptr[lo]) * kLongChunk;
        const int last = a.ptr[row + 1];
        end = beg + kLongChunk < last ? beg + kLongChunk : last;
    }
};

// body(row, unit head, beg, end, chunk or -1) for the units of this launch: a group takes one row, or chunks of long rows in turn.
template <int LG, class BODY>
__device__ __forceinline__ void for_units(const AttnArgs &a, int g, BODY body)
{
    constexpr int GROUPS = kBlock >> LG;
    if ((int)blockIdx.x < a.chunk_blocks) {
        const int n_long = *a.n_long;
        const int64_t total = (int64_t)*a.n_chunks * a.unit_heads;
        for (int64_t unit = (int64_t)blockIdx.x * GROUPS + g; unit < total; unit += (int64_t)a.chunk_blocks * GROUPS) {
            const int chunk = (int)over((uint64_t)unit, a.heads_inv), h = (int)(unit - (int64_t)chunk * a.unit_heads);
            const ChunkOf c(a, chunk, n_long);
            body(c.row, h, c.beg, c.end, (int64_t)chunk);
        }
        return;
    }
    const int64_t unit = (int64_t)(blockIdx.x - a.chunk_blocks) * GROUPS + g;
    if (unit >= a.units) return;
    const int64_t row = (int64_t)over((uint64_t)unit, a.heads_inv);
    const int h = (int)(unit - row * a.unit_heads);
    const int beg = a.ptr[row], end = a.ptr[row + 1];
    if (end - beg > a.long_thr) return;
    body(row, h, beg, end, (int64_t)-1);
}

// Columns (and buckets) of the next edges, the last of them again beyond the end.
struct Ahead {
    int col[kAttnUnroll], bucket[kAttnUnroll];
    __device__ __forceinline__ void load(const AttnArgs &a, int e, int end)
    {
#pragma unroll
        for (int j = 0; j < kAttnUnroll; ++j) {
            const int at = e + j < end ? e + j : end - 1;
            col[j] = a.col[at];
            bucket[j] = a.bucket ? a.bucket[at] : 0;
        }
    }
};

// The bias of an edge; -inf where the edge is left out.
__device__ __forceinline__ float bias_of(const AttnArgs &a, int bucket, int h)
{
    const bool in = (uint32_t)bucket < a.buckets;
    const float b = a.bias ? a.bias[(int64_t)(in ? bucket : 0) * a.heads + h] : 0.f;
    return in ? b : -INFINITY;
}

// ------------------------------------------------------------------ forward
template <bool BF16, int LG, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_attn_fwd(AttnArgs a)
{
    typedef Piece<BF16, WHOLE> P;
    typedef typename P::elem T;
    constexpr int N = P::N, U = kAttnUnroll;
    const Where<P, LG, WHOLE> w(a.width);
    for_units<LG>(a, w.g, [&](int64_t row, int h, int beg, int end, int64_t chunk) __attribute__((always_inline)) {
        const int hk = (int)over((uint32_t)h, a.shared_inv);
        const T *K = static_cast<const T *>(a.K) + hk * a.width + w.off, *V = static_cast<const T *>(a.V) + hk * a.width + w.off;
        float q[N], acc[N], m = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = 0.f;
        Ahead next;
        if (beg < end) {
            next.load(a, beg, end);
            w.own(static_cast<const T *>(a.Q) + row * a.ldq + h * a.width, a.scale, q);
        }
        for (int e = beg; e < end; e += U) {
            P k[U], v[U];
            float s[U];
#pragma unroll
            for (int j = 0; j < U; ++j) k[j].load(K + next.col[j] * a.ldk);
#pragma unroll
            for (int j = 0; j < U; ++j) v[j].load(V + next.col[j] * a.ldv);
#pragma unroll
            for (int j = 0; j < U; ++j) s[j] = e + j < end ? bias_of(a, next.bucket[j], h) : -INFINITY;
            if (e + U < end) next.load(a, e + U, end);
            float most = m;
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float d = 0.f;
#pragma unroll
                for (int i = 0; i < N; ++i) d = fmaf(q[i], k[j].get(i), d);
                d = over_lanes<LG>(d);
                s[j] = s[j] == -INFINITY ? s[j] : d + s[j];
                most = fmaxf(most, s[j]);
            }
            const float base = most == -INFINITY ? 0.f : most, old = exp_of(m - base);
            m = most;
            sum *= old;
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] *= old;
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const float p = exp_of(s[j] - base);
                sum += p;
                v[j].keep(p != 0.f);
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = fmaf(p, v[j].get(i), acc[i]);
            }
        }
        if (chunk >= 0) {
            const int64_t at = chunk * a.unit_heads + h;
            if (w.active) {
#pragma unroll
                for (int i = 0; i < N; ++i) a.part[at * a.width + w.off + i] = acc[i];
            }
            if (w.l == 0) {
                a.part_more[2 * at] = m;
                a.part_more[2 * at + 1] = sum;
            }
            return;
        }
        const float by = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] *= by;
        if (w.active) P::store(static_cast<T *>(a.O) + row * a.ldo + h * a.width + w.off, acc);
        if (a.lse && w.l == 0) a.lse[row * a.heads + h] = sum == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(sum) * kLn2;
    });
}

// ------------------------------------------------------------------ dQ
// sum p dp comes with the sums of p dp K and p K in one walk: dQ = scale (sum p dp K - (sum p dp) sum p K), all of them of e^(s - maximum)
// first and divided by its sum at the end.
template <bool BF16, int LG, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_attn_dq(AttnArgs a)
{
    typedef Piece<BF16, WHOLE> P;
    typedef typename P::elem T;
    constexpr int N = P::N, U = kAttnUnroll;
    const Where<P, LG, WHOLE> w(a.width);
    for_units<LG>(a, w.g, [&](int64_t row, int h, int beg, int end, int64_t chunk) __attribute__((always_inline)) {
        const int hk = (int)over((uint32_t)h, a.shared_inv);
        const T *K = static_cast<const T *>(a.K) + hk * a.width + w.off, *V = static_cast<const T *>(a.V) + hk * a.width + w.off;
        float q[N], g[N], pk[N], pdk[N], m = -INFINITY, sum = 0.f, delta = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) pk[i] = pdk[i] = 0.f;
        Ahead next;
        if (beg < end) {
            next.load(a, beg, end);
            w.own(static_cast<const T *>(a.Q) + row * a.ldq + h * a.width, a.scale, q);
            w.own(static_cast<const T *>(a.dO) + row * a.lddo + h * a.width, 1.f, g);
        }
        for (int e = beg; e < end; e += U) {
            P k[U], v[U];
            float s[U];
#pragma unroll
            for (int j = 0; j < U; ++j) k[j].load(K + next.col[j] * a.ldk);
#pragma unroll
            for (int j = 0; j < U; ++j) v[j].load(V + next.col[j] * a.ldv);
#pragma unroll
            for (int j = 0; j < U; ++j) s[j] = e + j < end ? bias_of(a, next.bucket[j], h) : -INFINITY;
            if (e + U < end) next.load(a, e + U, end);
            float most = m, dp[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float d = 0.f;
                dp[j] = 0.f;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    d = fmaf(q[i], k[j].get(i), d);
                    dp[j] = fmaf(g[i], v[j].get(i), dp[j]);
                }
                d = over_lanes<LG>(d);
                dp[j] = over_lanes<LG>(dp[j]);
                s[j] = s[j] == -INFINITY ? s[j] : d + s[j];
                most = fmaxf(most, s[j]);
            }
            const float base = most == -INFINITY ? 0.f : most, old = exp_of(m - base);
            m = most;
            sum *= old;
            delta *= old;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                pk[i] *= old;
                pdk[i] *= old;
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const float p = exp_of(s[j] - base), pd = p == 0.f ? 0.f : p * dp[j];
                sum += p;
                delta += pd;
                k[j].keep(p != 0.f);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    pk[i] = fmaf(p, k[j].get(i), pk[i]);
                    pdk[i] = fmaf(pd, k[j].get(i), pdk[i]);
                }
            }
        }
        if (chunk >= 0) {
            const int64_t at = chunk * a.unit_heads + h;
            if (w.active) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    a.part[at * a.width + w.off + i] = pdk[i];
                    a.part[a.part_stride + at * a.width + w.off + i] = pk[i];
                }
            }
            if (w.l == 0) reinterpret_cast<AttnArgs::f4 *>(a.part_more)[at] = AttnArgs::f4{m, sum, delta, 0.f};
            return;
        }
        const float by = sum == 0.f ? 0.f : 1.f / sum;
        delta *= by;
#pragma unroll
        for (int i = 0; i < N; ++i) pdk[i] = a.scale * by * fmaf(-delta, pk[i], pdk[i]);
        if (a.dQ && w.active) P::store(static_cast<T *>(a.dQ) + row * a.lddq + h * a.width + w.off, pdk);
        if (w.l == 0) a.stats[row * a.heads + h] = AttnArgs::f4{m, by, delta, 0.f};
    });
}

// ------------------------------------------------------------------ dK, dV
// Rows are sources; a group has one of the key heads and walks the edges of its row once for each query head that shares it.
template <bool BF16, int LG, bool WHOLE>
__global__ __launch_bounds__(kBlock) void k_attn_dkv(AttnArgs a)
{
    typedef Piece<BF16, WHOLE> P;
    typedef typename P::elem T;
    constexpr int N = P::N, U = kAttnUnroll;
    const Where<P, LG, WHOLE> w(a.width);
    for_units<LG>(a, w.g, [&](int64_t row, int hk, int beg, int end, int64_t chunk) __attribute__((always_inline)) {
        const T *Q = static_cast<const T *>(a.Q) + w.off, *G = static_cast<const T *>(a.dO) + w.off;
        float k[N], v[N], dk[N], dv[N];
#pragma unroll
        for (int i = 0; i < N; ++i) dk[i] = dv[i] = 0.f;
        if (beg < end) {
            w.own(static_cast<const T *>(a.K) + row * a.ldk + hk * a.width, a.scale, k);
            w.own(static_cast<const T *>(a.V) + row * a.ldv + hk * a.width, 1.f, v);
        }
        const uint32_t steps = (uint32_t)(end - beg) * (uint32_t)a.shared;       // rows of a transposed block are chunked: 2^8 x 2^12 at most
        for (uint32_t at = 0; at < steps; at += U) {
            P q[U], g[U];
            float s[U];
            AttnArgs::f4 stats[U];
            int pos[U], head[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const uint32_t i = at + j < steps ? at + j : steps - 1, e = over(i, a.shared_inv);
                pos[j] = beg + (int)e;
                head[j] = hk * a.shared + (int)(i - e * (uint32_t)a.shared);
            }
            int u[U], b[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                u[j] = a.col[pos[j]];
                b[j] = a.bucket ? a.bucket[a.eid[pos[j]]] : 0;
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                q[j].load(Q + u[j] * a.ldq + head[j] * a.width);
                g[j].load(G + u[j] * a.lddo + head[j] * a.width);
                stats[j] = a.stats[(int64_t)u[j] * a.heads + head[j]];
                s[j] = at + j < steps ? bias_of(a, b[j], head[j]) : -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float d = 0.f, dp = 0.f;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    d = fmaf(k[i], q[j].get(i), d);
                    dp = fmaf(v[i], g[j].get(i), dp);
                }
                d = over_lanes<LG>(d);
                dp = over_lanes<LG>(dp);
                const float z = s[j] == -INFINITY ? s[j] : d + s[j], p = z == -INFINITY ? 0.f : exp_of(z - stats[j][0]) * stats[j][1];
                const float ds = p == 0.f ? 0.f : p * (dp - stats[j][2]);
                if (a.ds && w.l == 0 && at + j < steps) a.ds[(int64_t)pos[j] * a.heads + head[j]] = ds;
                q[j].keep(p != 0.f);
                g[j].keep(p != 0.f);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    dk[i] = fmaf(ds, q[j].get(i), dk[i]);
                    dv[i] = fmaf(p, g[j].get(i), dv[i]);
                }
            }
        }
        if (chunk >= 0) {
            const int64_t to = chunk * a.unit_heads + hk;
            if (w.active) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    a.part[to * a.width + w.off + i] = dk[i];
                    a.part[a.part_stride + to * a.width + w.off + i] = dv[i];
                }
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) dk[i] *= a.scale;
        if (!w.active) return;
        if (a.dK) P::store(static_cast<T *>(a.dK) + row * a.lddk + hk * a.width + w.off, dk);
        if (a.dV) P::store(static_cast<T *>(a.dV) + row * a.lddv + hk * a.width + w.off, dv);
    });
}

// ------------------------------------------------------------------ chunks of long rows
// A workgroup has one long row and 2^lg of its columns at a time, and as many parts of its chunks as threads are left; the parts are joined in
// order.  KIND 0: O and lse, 1: dQ and the row's numbers, 2: dK and dV.
template <bool BF16, int KIND>
__global__ __launch_bounds__(kBlock) void k_attn_join(AttnArgs a, int lg)
{
    typedef typename Piece<BF16, true>::elem T;
    constexpr int MORE = KIND == 1 ? 4 : 2, NS = KIND == 0 ? 2 : KIND == 1 ? 4 : 2;       // sums: columns' (one or two), the row's
    const int cols = a.unit_heads * a.width, tiles = (cols + (1 << lg) - 1) >> lg, parts = kBlock >> lg;
    const int c = threadIdx.x & ((1 << lg) - 1), part = threadIdx.x >> lg;
    __shared__ float sums[NS][kBlock], most[kBlock];
    const int64_t total = (int64_t)*a.n_long * tiles;
    for (int64_t unit = blockIdx.x; unit < total; unit += gridDim.x) {
        const int li = (int)(unit / tiles), col = ((int)(unit - (int64_t)li * tiles) << lg) + c;
        const int64_t row = a.long_rows[li];
        const int first = a.chunk_ptr[li], n = a.chunk_ptr[li + 1] - first, per = (n + parts - 1) / parts;
        const int lo = first + part * per, hi = lo + per < first + n ? lo + per : first + n;
        const int h = col < cols ? col / a.width : 0;
        const float *p = a.part + (col < cols ? col : 0), *more = a.part_more;
        float v[NS], m = -INFINITY;
#pragma unroll
        for (int i = 0; i < NS; ++i) v[i] = 0.f;
        if (KIND != 2)
            for (int k = lo; k < hi; ++k) m = fmaxf(m, more[MORE * ((int64_t)k * a.unit_heads + h)]);
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 4
        for (int k = lo; k < hi; ++k) {
            const int64_t at = MORE * ((int64_t)k * a.unit_heads + h), to = (int64_t)k * cols;
            if constexpr (KIND == 2) {
                v[0] += p[to];
                v[1] += p[a.part_stride + to];
            } else {
                const float by = exp_of(more[at] - base);
                v[0] += by == 0.f ? 0.f : by * p[to];
                v[1] += by * more[at + 1];
                if constexpr (KIND == 1) {
                    v[2] += by == 0.f ? 0.f : by * p[a.part_stride + to];
                    v[3] += by == 0.f ? 0.f : by * more[at + 2];
                }
            }
        }
        __syncthreads();                              // the row before has been read
#pragma unroll
        for (int i = 0; i < NS; ++i) sums[i][threadIdx.x] = v[i];
        if (KIND != 2) most[threadIdx.x] = m;
        __syncthreads();
        if (part != 0 || col >= cols) continue;       // the barriers of the next row are reached by all
        if (KIND != 2)
            for (int r = 1; r < parts; ++r) m = fmaxf(m, most[(r << lg) + c]);
        const float all = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < NS; ++i) v[i] = 0.f;
        for (int r = 0; r < parts; ++r) {
            const float by = KIND == 2 ? 1.f : exp_of(most[(r << lg) + c] - all);
#pragma unroll
            for (int i = 0; i < NS; ++i) v[i] += by == 0.f ? 0.f : by * sums[i][(r << lg) + c];
        }
        auto put = [&](void *out, int64_t ld, float x) {
            if (!out) return;
            T *to = static_cast<T *>(out) + row * ld + col;
            if constexpr (BF16) *to = __builtin_bit_cast(uint16_t, (__bf16)x);
            else *to = x;
        };
        if constexpr (KIND == 2) {
            put(a.dK, a.lddk, v[0] * a.scale);
            put(a.dV, a.lddv, v[1]);
        } else {
            const float by = v[1] == 0.f ? 0.f : 1.f / v[1];
            if constexpr (KIND == 0) {
                put(a.O, a.ldo, v[0] * by);
                if (a.lse && col == h * a.width) a.lse[row * a.heads + h] = v[1] == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(v[1]) * kLn2;
            } else {
                const float delta = v[3] * by;
                put(a.dQ, a.lddq, a.scale * by * fmaf(-delta, v[2], v[0]));
                if (col == h * a.width) a.stats[row * a.heads + h] = AttnArgs::f4{m, by, delta, 0.f};
            }
        }
    }
}

// ------------------------------------------------------------------ dbias
// A workgroup adds up ds of a run of edges into tables of its own in LDS: one for every edge that it has under way, so that no two threads
// meet; then table by table.  Buckets are taken kBiasTile at a time, heads 2^lg at a time.
struct BiasArgs {
    const float *ds;               // [position][heads]
    const int32_t *eid, *bucket;
    float *part;                   // [workgroup][buckets][heads]
    int64_t positions;
    int32_t heads, buckets, lg;
};

__global__ __launch_bounds__(kBlock) void k_attn_dbias(BiasArgs a)
{
    __shared__ float table[kBiasTile * kBlock];       // [bucket][edge under way][head]
    const int hs = 1 << a.lg, slots = kBlock >> a.lg, head0 = (int)blockIdx.z * hs, first = (int)blockIdx.y * kBiasTile;
    const int h = head0 + (threadIdx.x & (hs - 1)), slot = threadIdx.x >> a.lg;
    for (int i = 0; i < kBiasTile; ++i) table[i * kBlock + threadIdx.x] = 0.f;
    __syncthreads();
    const int64_t per = (a.positions + gridDim.x - 1) / gridDim.x, beg = per * blockIdx.x, last = beg + per < a.positions ? beg + per : a.positions;
#pragma unroll 4
    for (int64_t t = beg + slot; t < last; t += slots) {
        const uint32_t b = (uint32_t)(a.bucket[a.eid[t]] - first);
        if (b < (uint32_t)kBiasTile && h < a.heads) table[b * kBlock + threadIdx.x] += a.ds[t * a.heads + h];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kBiasTile * hs; i += kBlock) {
        const int b = i >> a.lg, c = i & (hs - 1);
        float v = 0.f;
        for (int r = 0; r < slots; ++r) v += table[b * kBlock + (r << a.lg) + c];
        if (first + b < a.buckets && head0 + c < a.heads) a.part[((int64_t)blockIdx.x * a.buckets + first + b) * a.heads + head0 + c] = v;
    }
}

// Eight entries of the table a workgroup, 32 threads each.
__global__ __launch_bounds__(kBlock) void k_attn_dbias_sum(const float *part, int blocks, int64_t n, float *dbias)
{
    __shared__ double sums[kBlock / 8][9];
    const int c = threadIdx.x & 7, r = threadIdx.x >> 3;
    const int64_t at = (int64_t)blockIdx.x * 8 + c;
    double v = 0.0;
    if (at < n) {
#pragma unroll 4
        for (int i = r; i < blocks; i += kBlock / 8) v += (double)part[(int64_t)i * n + at];
    }
    sums[r][c] = v;
    __syncthreads();
    if (r == 0 && at < n) {
        v = 0.0;
        for (int i = 0; i < kBlock / 8; ++i) v += sums[i][c];
        dbias[at] = (float)v;
    }
}

// ------------------------------------------------------------------ host side
bool misaligned_to(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

fastgl_status check_sizes(const fastgl_attn_desc &d)
{
    if (d.num_dst < 0 || d.num_src < 0 || d.num_edges < 0 || d.num_buckets < 0) {
        set_error("negative size (num_dst=%lld num_src=%lld num_edges=%lld num_buckets=%lld)", (long long)d.num_dst, (long long)d.num_src,
                  (long long)d.num_edges, (long long)d.num_buckets);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (d.num_dst > kMaxIndex || d.num_src > kMaxIndex || d.num_edges > kMaxIndex) {
        set_error("sizes must not exceed 2^31-1-%d", INT32_MAX - (int)kMaxIndex);
        return FASTGL_ERR_UNSUPPORTED;
    }
    if (d.num_edges > 0 && (d.num_dst == 0 || d.num_src == 0)) {
        set_error("edges need at least one destination and one source node");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (d.dtype != FASTGL_F32 && d.dtype != FASTGL_BF16) {
        set_error("bad dtype %d", (int)d.dtype);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (d.heads < 1 || d.kv_heads < 1 || d.heads % d.kv_heads || d.width < 1) {
        set_error("heads (%lld) must be a multiple of kv_heads (%lld) and width (%lld) positive", (long long)d.heads, (long long)d.kv_heads,
                  (long long)d.width);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (d.width > 256 || d.heads > 4096 || d.heads * d.width > 65536 || (d.bias && d.num_buckets > 65536)) {
        set_error("width must stay at 256, heads at 4096, heads * width at 65536 and num_buckets at 65536 or below");
        return FASTGL_ERR_UNSUPPORTED;
    }
    if (d.bias && ((!d.bucket && d.num_edges > 0) || d.num_buckets < 1)) {
        set_error("a bias needs buckets");
        return FASTGL_ERR_INVALID_ARG;
    }
    return FASTGL_OK;
}

fastgl_status check(const fastgl_attn_desc *desc, bool backward, const fastgl_plan *plan)
{
    if (!desc) {
        set_error("desc is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    const fastgl_attn_desc &d = *desc;
    const fastgl_status st = check_sizes(d);
    if (st != FASTGL_OK) return st;
    if (!d.indptr || (!d.indices && d.num_edges > 0)) {
        set_error("indptr or indices is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    if ((d.num_dst > 0 && !d.Q) || (d.num_src > 0 && (!d.K || !d.V))) {
        set_error("Q, K or V is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (d.ldq < d.heads * d.width || d.ldk < d.kv_heads * d.width || d.ldv < d.kv_heads * d.width) {
        set_error("ldq, ldk and ldv must not be below a row's length");
        return FASTGL_ERR_INVALID_ARG;
    }
    const uintptr_t el = d.dtype == FASTGL_BF16 ? 2 : 4;
    if (misaligned_to(d.Q, el) || misaligned_to(d.K, el) || misaligned_to(d.V, el) || misaligned_to(d.indptr, 4) || misaligned_to(d.indices, 4) ||
        misaligned_to(d.bucket, 4) || misaligned_to(d.bias, 4)) {
        set_error("buffers must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (!plan) return FASTGL_OK;
    const int need = !backward ? FASTGL_PLAN_FWD : FASTGL_PLAN_ALL | (d.bucket ? FASTGL_PLAN_PERM : 0);
    if (plan->indptr != d.indptr || plan->indices != d.indices || plan->num_dst != d.num_dst || plan->num_src != d.num_src ||
        plan->num_edges != d.num_edges) {
        set_error("plan was built for a different block");
        return FASTGL_ERR_INVALID_ARG;
    }
    if ((plan->parts & need) != need) {
        set_error("plan lacks the parts this pass needs (has %d, needs %d)", plan->parts, need);
        return FASTGL_ERR_INVALID_ARG;
    }
    return FASTGL_OK;
}

// Where a call's scratch lies; base NULL: only the size is wanted.
struct Scratch {
    size_t used = 0;
    char *base;
    float *part, *part_more, *stats, *ds, *bias;
    char *plan;
    int64_t part_stride;
    float *take(int64_t n)
    {
        char *p = base ? base + used : nullptr;
        used += align_up((size_t)n * sizeof(float), 256);
        return reinterpret_cast<float *>(p);
    }
    Scratch(const fastgl_attn_desc &d, bool backward, bool own_plan, char *at) : base(at)
    {
        part = part_more = stats = ds = bias = nullptr;
        plan = nullptr;
        const int64_t chunks = d.num_edges > kLongThreshold ? cap_chunks(d.num_edges) : 0;
        part_stride = chunks * d.heads * d.width;
        part = take(part_stride * (backward ? 2 : 1));
        part_more = take(chunks * d.heads * (backward ? 4 : 2));
        if (backward) {
            stats = take(d.num_dst * d.heads * 4);
            if (d.bias) {
                ds = take(d.num_edges * d.heads);
                bias = take(bias_blocks(d) * d.num_buckets * d.heads);
            }
        }
        if (own_plan && (backward || chunks)) {
            plan = base ? base + used : nullptr;
            used += plan_layout(nullptr, nullptr, d.num_dst, d.num_src, d.num_edges, !backward);
        }
    }
    // Workgroups of the bias gradient: some hundred edges each, and tables of 64 MiB together at most.
    static int64_t bias_blocks(const fastgl_attn_desc &d)
    {
        const int64_t some = ceil_div(d.num_edges, 512), most = ((int64_t)16 << 20) / (d.num_buckets * d.heads + 1);
        const int64_t n = some < kBiasBlocks ? some : kBiasBlocks;
        return n < most ? (n > 0 ? n : 1) : (most > 0 ? most : 1);
    }
};

template <class F>
fastgl_status by_shape(fastgl_dtype dtype, int64_t width, F f)
{
    const bool bf16 = dtype == FASTGL_BF16;
    const int n = bf16 ? 8 : 4;
    typedef std::true_type Yes;
    typedef std::false_type No;
    if (width < n) return bf16 ? f(Yes(), std::integral_constant<int, 3>(), No()) : f(No(), std::integral_constant<int, 2>(), No());
    const int64_t pieces = ceil_div(width, n);
    auto lanes = [&](auto b) {
        if (pieces <= 1) return f(b, std::integral_constant<int, 0>(), Yes());
        if (pieces <= 2) return f(b, std::integral_constant<int, 1>(), Yes());
        if (pieces <= 4) return f(b, std::integral_constant<int, 2>(), Yes());
        if (pieces <= 8) return f(b, std::integral_constant<int, 3>(), Yes());
        if (pieces <= 16) return f(b, std::integral_constant<int, 4>(), Yes());
        if constexpr (decltype(b)::value) return f(b, std::integral_constant<int, 5>(), Yes());
        else {
            if (pieces <= 32) return f(b, std::integral_constant<int, 5>(), Yes());
            return f(b, std::integral_constant<int, 6>(), Yes());
        }
    };
    return bf16 ? lanes(Yes()) : lanes(No());
}

enum Pass { kPassFwd = 0, kPassDq = 1, kPassDkv = 2 };

// One walk and the launch that joins its chunks.
template <int PASS>
fastgl_status launch_walk(AttnArgs a, const fastgl_attn_desc &d, const fastgl_plan *pl, hipStream_t s)
{
    static const char *const names[3] = {"fastgl_attn_fwd", "fastgl_attn_bwd (dQ)", "fastgl_attn_bwd (dK, dV)"};
    constexpr bool T = PASS == kPassDkv;
    const int64_t rows = T ? d.num_src : d.num_dst;
    a.unit_heads = (int32_t)(T ? d.kv_heads : d.heads);
    a.units = rows * a.unit_heads;
    a.heads_inv = a.unit_heads > 1 ? UINT64_MAX / (uint64_t)a.unit_heads + 1 : 0;
    const bool chunked = d.num_edges > kLongThreshold && (T || !(pl->parts & FASTGL_PLAN_SHORT_DST_ROWS));
    a.long_thr = chunked ? kLongThreshold : INT32_MAX;
    if (chunked) {
        a.long_rows = T ? pl->long_src : pl->long_dst;
        a.chunk_ptr = T ? pl->chunk_ptr_src : pl->chunk_ptr_dst;
        a.n_long = pl->counters + (T ? 2 : 0);
        a.n_chunks = pl->counters + (T ? 3 : 1);
    }
    if (a.units == 0) return FASTGL_OK;
    const fastgl_status st = by_shape(d.dtype, d.width, [&](auto bf16, auto lg, auto whole) {
        constexpr bool B = decltype(bf16)::value, W = decltype(whole)::value;
        constexpr int LG = decltype(lg)::value;
        const int64_t groups = kBlock >> LG;
        if (chunked) {
            const int64_t n = ceil_div(cap_chunks(d.num_edges) * a.unit_heads, groups);
            a.chunk_blocks = (int32_t)(n < 1024 ? n : 1024);
        }
        const int64_t blocks = ceil_div(a.units, groups) + a.chunk_blocks;
        if (blocks > INT32_MAX) {
            set_error("%s: too many rows and heads", names[PASS]);
            return FASTGL_ERR_UNSUPPORTED;
        }
        if constexpr (PASS == kPassFwd) hipLaunchKernelGGL((k_attn_fwd<B, LG, W>), dim3((unsigned)blocks), dim3(kBlock), 0, s, a);
        else if constexpr (PASS == kPassDq) hipLaunchKernelGGL((k_attn_dq<B, LG, W>), dim3((unsigned)blocks), dim3(kBlock), 0, s, a);
        else hipLaunchKernelGGL((k_attn_dkv<B, LG, W>), dim3((unsigned)blocks), dim3(kBlock), 0, s, a);
        FASTGL_LAUNCH_CHECK(names[PASS]);
        return FASTGL_OK;
    });
    if (st != FASTGL_OK || !chunked) return st;
    const int cols = a.unit_heads * a.width;
    int lg = 5;
    while (lg < 8 && (1 << lg) < cols) ++lg;
    const int64_t units = cap_long_rows(d.num_edges) * ceil_div(cols, (int64_t)1 << lg);
    const dim3 grid((unsigned)(units < 1024 ? units : 1024));
    if (d.dtype == FASTGL_BF16) hipLaunchKernelGGL((k_attn_join<true, PASS>), grid, dim3(kBlock), 0, s, a, lg);
    else hipLaunchKernelGGL((k_attn_join<false, PASS>), grid, dim3(kBlock), 0, s, a, lg);
    FASTGL_LAUNCH_CHECK("fastgl_attn (long rows)");
    return FASTGL_OK;
}

AttnArgs args_of(const fastgl_attn_desc &d, const Scratch &o)
{
    AttnArgs a = {};
    a.ptr = d.indptr; a.col = d.indices;
    a.bucket = d.bucket; a.bias = d.bias;
    a.buckets = d.bias ? (uint32_t)d.num_buckets : 0x80000000u;
    a.Q = d.Q; a.K = d.K; a.V = d.V;
    a.ldq = d.ldq; a.ldk = d.ldk; a.ldv = d.ldv;
    a.heads = (int32_t)d.heads; a.shared = (int32_t)(d.heads / d.kv_heads); a.width = (int32_t)d.width;
    a.shared_inv = a.shared > 1 ? (uint32_t)(0xFFFFFFFFu / (uint32_t)a.shared + 1) : 0;
    a.scale = d.scale;
    a.stats = reinterpret_cast<AttnArgs::f4 *>(o.stats);
    a.part = o.part; a.part_more = o.part_more; a.part_stride = o.part_stride;
    return a;
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

// The caller's plan, or one built in the workspace.
fastgl_status plan_for(const fastgl_attn_desc &d, const fastgl_plan **plan, fastgl_plan *local, char *mem, int parts, hipStream_t s)
{
    if (*plan || !mem) return FASTGL_OK;
    local->num_dst = d.num_dst; local->num_src = d.num_src; local->num_edges = d.num_edges;
    local->indptr = d.indptr; local->indices = d.indices;
    plan_layout(local, mem, d.num_dst, d.num_src, d.num_edges, parts == FASTGL_PLAN_FWD);
    *plan = local;
    return plan_build(local, parts, false, s);
}

}  // namespace
}  // namespace fastgl

using namespace fastgl;

extern "C" {

size_t fastgl_attn_workspace_bytes(const fastgl_attn_desc *desc, int backward)
{
    if (!desc || check_sizes(*desc) != FASTGL_OK) return 0;
    return Scratch(*desc, backward != 0, true, nullptr).used;
}

fastgl_status fastgl_attn_fwd(const fastgl_attn_desc *desc, void *O, int64_t ldo, float *lse, const fastgl_plan *plan, void *ws,
                              size_t ws_bytes, void *stream)
{
    fastgl_status st = check(desc, false, plan);
    if (st != FASTGL_OK) return st;
    const fastgl_attn_desc &d = *desc;
    if (d.num_dst == 0) return FASTGL_OK;
    if (!O || ldo < d.heads * d.width || misaligned_to(O, d.dtype == FASTGL_BF16 ? 2 : 4) || misaligned_to(lse, 4)) {
        set_error("O is NULL or misaligned, ldo below a row's length, or lse misaligned");
        return FASTGL_ERR_INVALID_ARG;
    }
    st = check_workspace(ws, ws_bytes, Scratch(d, false, !plan, nullptr).used);
    if (st != FASTGL_OK) return st;
    hipStream_t s = (hipStream_t)stream;
    const Scratch o(d, false, !plan, (char *)ws);
    fastgl_plan local;
    if ((st = plan_for(d, &plan, &local, o.plan, FASTGL_PLAN_FWD, s)) != FASTGL_OK) return st;
    AttnArgs a = args_of(d, o);
    a.O = O; a.ldo = ldo;
    a.lse = lse;
    return launch_walk<kPassFwd>(a, d, plan, s);
}

fastgl_status fastgl_attn_bwd(const fastgl_attn_desc *desc, const void *dO, int64_t lddo, void *dQ, int64_t lddq, void *dK,
                              int64_t lddk, void *dV, int64_t lddv, float *dbias, const fastgl_plan *plan, void *ws, size_t ws_bytes,
                              void *stream)
{
    fastgl_status st = check(desc, true, plan);
    if (st != FASTGL_OK) return st;
    const fastgl_attn_desc &d = *desc;
    const uintptr_t el = d.dtype == FASTGL_BF16 ? 2 : 4;
    const int64_t n = d.heads * d.width, k = d.kv_heads * d.width;
    if (!dQ && !dK && !dV && !dbias) return FASTGL_OK;
    if (d.num_dst > 0 && !dO) {
        set_error("dO is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (dbias && !d.bias) {
        set_error("dbias needs the bias and its buckets");
        return FASTGL_ERR_INVALID_ARG;
    }
    if ((dO && lddo < n) || (dQ && lddq < n) || (dK && lddk < k) || (dV && lddv < k)) {
        set_error("lddo, lddq, lddk and lddv must not be below a row's length");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (misaligned_to(dO, el) || misaligned_to(dQ, el) || misaligned_to(dK, el) || misaligned_to(dV, el) || misaligned_to(dbias, 4)) {
        set_error("buffers must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    st = check_workspace(ws, ws_bytes, Scratch(d, true, !plan, nullptr).used);
    if (st != FASTGL_OK) return st;
    hipStream_t s = (hipStream_t)stream;
    const Scratch o(d, true, !plan, (char *)ws);
    fastgl_plan local;
    st = plan_for(d, &plan, &local, o.plan, FASTGL_PLAN_ALL | (d.bucket ? FASTGL_PLAN_PERM : 0), s);
    if (st != FASTGL_OK) return st;

    AttnArgs a = args_of(d, o);
    a.dO = dO; a.lddo = lddo;
    a.dQ = dQ; a.lddq = lddq;
    if ((st = launch_walk<kPassDq>(a, d, plan, s)) != FASTGL_OK) return st;
    if (!dK && !dV && !dbias) return FASTGL_OK;
    AttnArgs b = args_of(d, o);
    b.ptr = plan->indptr_T; b.col = plan->indices_T; b.eid = plan->perm;
    b.dO = dO; b.lddo = lddo;
    b.dK = dK; b.lddk = lddk;
    b.dV = dV; b.lddv = lddv;
    b.ds = dbias ? o.ds : nullptr;
    if ((st = launch_walk<kPassDkv>(b, d, plan, s)) != FASTGL_OK) return st;
    if (!dbias) return FASTGL_OK;
    BiasArgs c = {};
    c.ds = o.ds;
    c.eid = plan->perm; c.bucket = d.bucket;
    c.part = o.bias;
    c.positions = d.num_edges;
    c.heads = (int32_t)d.heads; c.buckets = (int32_t)d.num_buckets;
    while (c.lg < 5 && (1 << c.lg) < d.heads) ++c.lg;
    const int64_t blocks = Scratch::bias_blocks(d), table = d.num_buckets * d.heads;
    const dim3 grid((unsigned)blocks, (unsigned)ceil_div(d.num_buckets, kBiasTile), (unsigned)ceil_div(d.heads, (int64_t)1 << c.lg));
    hipLaunchKernelGGL(k_attn_dbias, grid, dim3(kBlock), 0, s, c);
    FASTGL_LAUNCH_CHECK("fastgl_attn_bwd (dbias)");
    hipLaunchKernelGGL(k_attn_dbias_sum, dim3((unsigned)ceil_div(table, 8)), dim3(kBlock), 0, s, (const float *)o.bias, (int)blocks, table, dbias);
    FASTGL_LAUNCH_CHECK("fastgl_attn_bwd (dbias, sums)");
    return FASTGL_OK;
}

}  // extern "C"
