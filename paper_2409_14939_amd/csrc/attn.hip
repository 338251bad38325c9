// Attention over the sampled neighbours of a block, forward and backward (fastgl_attn.h has the formulas).
//
//   forward   k_attn_fwd (rows, and chunks of long rows) -> [k_attn_join: chunks to rows]
//   backward  k_attn_dq  (the same walk: dQ, and maximum, sum and sum p dp of every row) -> [k_attn_join]
//             k_attn_dkv (rows of the transposed block: dK, dV; ds of every edge where dbias is wanted) -> [k_attn_join]
//             k_attn_dbias -> k_attn_dbias_sum
//
// A group of lanes has one row and one head, one or two pieces of 16 bytes of the head a lane whatever its width and alignment: the last piece
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
constexpr int kSegment = 16;              // steps that a group takes where a neighbour has more
constexpr int kSlack = 8;                 // steps more than shorter segments have that a group takes alone rather than have them cut
constexpr int kTransposedSteps = 6;       // of a group, on average, that a wavefront of the transposed pass takes units for
constexpr int kBiasBlocks = 1024;         // workgroups of k_attn_dbias
constexpr int64_t kHintEdges = (int64_t)1 << 24;      // blocks of more have their long rows looked for whatever the plan's hint says
constexpr int kJoin = 1024;               // threads of a workgroup that joins chunks
constexpr int kBiasTile = 64;             // buckets of one of its passes

// ------------------------------------------------------------------ lanes and pieces
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// What a lane holds of a head: PC pieces of 16 bytes, `lanes` pieces apart; PC 0: one element, for heads narrower than 16 bytes.
template <bool BF16, int PC>
struct Piece {
    typedef typename std::conditional<BF16, uint16_t, float>::type elem;
    typedef typename Words<BF16 ? 2 : 4>::x4 word;
    static constexpr int ES = sizeof(elem), CE = 16 / ES, PIECES = PC, N = PC * CE;
    word w[PC];
    __device__ __forceinline__ void load(const char *p, int c) { w[c] = *reinterpret_cast<const word *>(p); }
    __device__ __forceinline__ float get(int i) const
    {
        const uint32_t x = w[i / CE][i % CE * ES / 4];
        if constexpr (BF16) return __uint_as_float(i & 1 ? x & 0xFFFF0000u : x << 16);
        else return __uint_as_float(x);
    }
    __device__ __forceinline__ void keep(bool on)
    {
#pragma unroll
        for (int c = 0; c < PC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[c][i] = on ? w[c][i] : 0u;
    }
    // Without the first `skip` elements of piece c.
    __device__ __forceinline__ void cut(int c, int skip)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) w[c][i] &= 2 * i >= skip ? 0xFFFFFFFFu : 2 * i + 1 >= skip ? 0xFFFF0000u : 0u;
            else w[c][i] = i >= skip ? w[c][i] : 0u;
        }
    }
    // The sum of products in fp32: of bf16 two at a time, exact.
    __device__ __forceinline__ float dot(const Piece &o) const
    {
        float d = 0.f;
#pragma unroll
        for (int c = 0; c < PC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (BF16) {
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                    const uint32_t x = w[c][i], y = o.w[c][i];
                    d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, y), d, false);
                } else
                    d = fmaf(__uint_as_float(w[c][i]), __uint_as_float(o.w[c][i]), d);
            }
        return d;
    }
    __device__ static __forceinline__ void store(char *p, int c, const float (&v)[N])
    {
        word o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) o[i] = pack2(v[c * CE + 2 * i], v[c * CE + 2 * i + 1]);
            else o[i] = __float_as_uint(v[c * CE + i]);
        }
        *reinterpret_cast<word *>(p) = o;
    }
};

template <bool BF16>
struct Piece<BF16, 0> {
    typedef typename std::conditional<BF16, uint16_t, float>::type elem;
    static constexpr int ES = sizeof(elem), CE = 1, PIECES = 1, N = 1;
    float x;
    __device__ __forceinline__ void load(const char *p, int)
    {
        if constexpr (BF16) x = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(p) << 16);
        else x = *reinterpret_cast<const float *>(p);
    }
    __device__ __forceinline__ float get(int) const { return x; }
    __device__ __forceinline__ void keep(bool on) { x = on ? x : 0.f; }
    __device__ __forceinline__ void cut(int, int skip) { x = skip > 0 ? 0.f : x; }
    __device__ __forceinline__ float dot(const Piece &o) const { return x * o.x; }
    __device__ static __forceinline__ void store(char *p, int, const float (&v)[1])
    {
        if constexpr (BF16) *reinterpret_cast<uint16_t *>(p) = __builtin_bit_cast(uint16_t, (__bf16)v[0]);
        else *reinterpret_cast<float *>(p) = v[0];
    }
};

// exp(x) of a difference of scores, x <= 0: 2^(x log2 e).  Relative error 2^-23 (1 + |x|).
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// x + x of the lane across: the first four exchanges stay within sixteen lanes and need no LDS.  After them both lanes of a pair
// hold the same sum, so that mirrored lanes are as good as those across: a product of one element a lane is rounded before it is added.
template <int CTRL>
__device__ __forceinline__ float plus_dpp(float v)
{
#pragma clang fp contract(off)
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

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    const int32_t *ptr, *col;      // rows of the block, or of its transpose
    const int32_t *bucket;         // by position in col, or NULL
    const float *bias;             // or NULL
    const void *Q, *K, *V, *dO;
    int64_t ldq, ldk, ldv, lddo;
    f32x4 *stats;                  // [num_dst][heads]: maximum, 1 / sum, sum p dp of a row
    void *O, *dQ, *dK, *dV;        // or NULL
    int64_t ldo, lddq, lddk, lddv;
    float *lse;                    // [rows][heads], or NULL
    float *ds;                     // [position][heads], or NULL
    const int32_t *bucket_from, *eid;      // dQ: the transposed block's buckets are brought into its order on the way: bucket_to[i] =
    int32_t *bucket_to;                    // bucket_from[eid[i]] for so many edges
    int64_t edges;
    int64_t units;                 // rows (dealt: to a multiple of 512) x heads (transposed: x key heads)
    int64_t rows;
    int32_t dealt;                 // rows are taken 64 apart
    int32_t units_a_wave;          // the groups of a wavefront or fewer
    uint64_t heads_inv;            // ceil(2^64 / heads of a unit), 0 for one
    uint32_t shared_inv;           // ceil(2^32 / shared), 0 for one: exact for 2^20 query heads of edges at most 4096 of which share
    uint32_t buckets;              // edges of this bucket and above are left out
    int32_t heads, unit_heads, shared, width;
    float scale;
    int32_t long_thr;              // rows of more edges are taken in chunks
    const int32_t *long_rows, *chunk_ptr, *n_long, *n_chunks;
    int32_t chunk_waves;           // wavefronts that take chunks
    float *part, *part_more;       // sums of chunks: [chunk][unit head][width], and what else a pass has
    int64_t part_stride;           // between the two arrays of `part` that a backward pass has
};

// Launches of more than 2^32 threads have two dimensions.
__device__ __forceinline__ int64_t block_of() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

__device__ __forceinline__ uint64_t over(uint64_t n, uint64_t inv) { return inv ? __umul64hi(n, inv) : n; }
__device__ __forceinline__ uint32_t over(uint32_t n, uint32_t inv) { return inv ? __umulhi(n, inv) : n; }

// Where a lane is: its group's place in the wavefront and its pieces of a head.  A row's place in an array is a 32-bit offset where the
// array is NEAR (us, so / 64-bit offsets: 8000 rows of 15, four f32 heads of 47 on one, forward 15.7 / 16.7, dQ 18.6 / 19.3, dK and dV 50.0 / 51.3;  91 331
// rows of 10, eight bf16 heads of 32, dK and dV 334 / 341;  where memory bounds a walk the same).
template <class P, int LG, bool NEAR>
struct Where {
    int l, g, off[P::PIECES], skip[P::PIECES];        // off: bytes
    bool active[P::PIECES];
    __device__ __forceinline__ Where(int width)
    {
        const int lane = threadIdx.x & (kWave - 1);
        l = lane & ((1 << LG) - 1);
        g = lane >> LG;
#pragma unroll
        for (int c = 0; c < P::PIECES; ++c) {
            const int at = (l + (c << LG)) * P::CE, last = width - P::CE, from = at < last ? at : last;
            off[c] = from * P::ES;
            skip[c] = at - from;                      // elements that the piece before has too; all of them beyond the head
            active[c] = at < width;
        }
    }
    __device__ __forceinline__ void load(P &x, const void *base, int64_t row, int64_t ld, int col) const
    {
#pragma unroll
        for (int c = 0; c < P::PIECES; ++c) {
            if constexpr (NEAR) x.load(static_cast<const char *>(base) + ((uint32_t)row * (uint32_t)(ld * P::ES) + (uint32_t)(col * P::ES + off[c])), c);
            else x.load(static_cast<const char *>(base) + (row * ld + col) * P::ES + off[c], c);
        }
    }
    // A row's own operand without what another piece has too.
    __device__ __forceinline__ void cut(P &x) const
    {
#pragma unroll
        for (int c = 0; c < P::PIECES; ++c) x.cut(c, skip[c]);
    }
    __device__ __forceinline__ void store(void *base, int64_t row, int64_t ld, int col, const float (&v)[P::N]) const
    {
#pragma unroll
        for (int c = 0; c < P::PIECES; ++c)
            if (active[c]) P::store(static_cast<char *>(base) + (row * ld + col) * P::ES + off[c], c, v);
    }
    __device__ __forceinline__ void store_sums(float *base, int64_t at, const float (&v)[P::N]) const       // of a chunk
    {
#pragma unroll
        for (int c = 0; c < P::PIECES; ++c)
            if (active[c]) {
#pragma unroll
                for (int i = 0; i < P::CE; ++i) base[at + off[c] / P::ES + i] = v[c * P::CE + i];
            }
    }
};

// The next edges of a row: columns and buckets, the last of them again beyond the end.  Transposed, an edge counts once for each query
// head that shares the key head: step i is head i % shared of edge i / shared.
template <bool T, int U>
struct Ahead {
    int col[U], bucket[U], pos[T ? U : 1], head[T ? U : 1];
    __device__ __forceinline__ void load(const AttnArgs &a, int beg, int i, int steps)
    {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            int at = i + j < steps ? i + j : steps - 1;
            if constexpr (T) {
                const int e = (int)over((uint32_t)at, a.shared_inv);
                head[j] = at - e * a.shared;
                pos[j] = beg + e;
                at = e;
            }
            col[j] = a.col[beg + at];
            bucket[j] = a.bucket ? a.bucket[beg + at] : 0;
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

// ------------------------------------------------------------------ the walk
// ROW has the operands and sums of one row and head (or of a part of its edges), the pass's arithmetic and where its results go.
//
// A group takes one row and head, a unit; where there are few units a wavefront has fewer of them than groups.  Where a unit of the wavefront has more
// than kSegment steps, all its units' steps are cut into segments of so many, which the groups take in turn, so that nobody waits long for a
// neighbour's row: segments of one unit lie side by side, their sums are joined across the groups and then with what earlier turns left in LDS.  Where
// there are few units segments are as short as gives every group one.  Chunks of long rows, which the first wavefronts take after their own rows,
// are units too, as many at a time as give every group a segment.
//
// Rows of sources are dealt to the wavefronts 64 apart: those that are neighbours of many often have numbers that lie together.
//
// What bounds it: the gathers of neighbours' rows.  With heads of 128 bytes and 4.4 edges a row (512 345 rows, 1.1 million sources) the forward pass takes 295 us:
// 1.15 GB of K and V from memory and caches and 0.52 GB of Q and O, 5.7 TB/s.  With heads of 32 bytes (65 536 rows, 1.7 million edges: forward 104 us, dQ 143, dK and
// dV 133) three quarters of the forward pass's and dQ's lines are not in L2, 0.49 and 0.61 GB at 4.7 and 4.3 TB/s, and the vector ALUs are busy for 33, 40 and 54 % of
// the time: a step's rows are asked for after the step before, so that a wavefront waits for them once a step (two thirds of its time and more, with the four wavefronts that a SIMD has here).
// Segments: 65 536 rows of eight edges beside rows of up to 18 000, forward 201 us without them, 103 with;  8000 rows of 15, dK and dV for heads that share
// theirs 121 and 50.  Two pieces a lane instead of one: the 512 345 rows 451 and 345 us (then with 64-bit offsets).
template <class ROW>
__device__ __forceinline__ void walk_units(const AttnArgs &a)
{
    constexpr int LG = ROW::LG, G = kWave >> LG, L = 1 << LG;
    constexpr bool T = ROW::T;
    constexpr int U = ROW::UNROLL;
    __shared__ float kept[kBlock / kWave][ROW::VALUES][kWave];
    ROW r(a);
    const int lane = threadIdx.x & (kWave - 1), gw = r.w.g, mult = T ? a.shared : 1;
    const int in_block = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t wave = block_of() * (kBlock / kWave) + in_block;
    float (&slots)[ROW::VALUES][kWave] = kept[in_block];
    // Steps i .. steps of a row, U at a time; the last U / 2 in one of half the size.
    auto walk = [&](int row, int h, int beg, int i, int steps) __attribute__((always_inline)) {
        Ahead<T, U> next;
        if (i < steps) {
            next.load(a, beg, i, steps);
            r.own(row, h);
        }
        r.start(h);
        for (; i + U / 2 < steps; i += U) r.template step<U>(next, beg, i, steps);
        if constexpr (U > 1)
            if (i < steps) r.template step<U / 2>(next, beg, i, steps);
    };
    const int64_t chunks = a.long_rows && wave < a.chunk_waves ? (int64_t)*a.n_chunks * a.unit_heads : 0;
    constexpr int AT_ONCE = G * kSegment / kLongChunk > 0 ? G * kSegment / kLongChunk : 1;       // chunks
    for (int64_t at = -1; at < chunks; at = at < 0 ? wave * AT_ONCE : at + (int64_t)a.chunk_waves * AT_ONCE) {
        int row = 0, h = 0, beg = 0, steps = 0;
        int64_t chunk = -1;
        bool on;
        if (at < 0) {
            const int64_t unit = wave * a.units_a_wave + gw;
            int64_t to = (int64_t)over((uint64_t)unit, a.heads_inv);
            h = (int)(unit - to * a.unit_heads);
            if (T && a.dealt) to = (to & ~(int64_t)511) | ((to & 7) << 6) | ((to >> 3) & 63);
            on = gw < a.units_a_wave && unit < a.units && to < a.rows;
            if (on) {
                row = (int)to;
                beg = a.ptr[row];
                const int len = a.ptr[row + 1] - beg;
                on = len <= a.long_thr;
                steps = on ? len * mult : 0;
            }
        } else {
            chunk = at + gw;
            on = gw < AT_ONCE && chunk < chunks;
            if (on) {
                const int c = (int)over((uint64_t)chunk, a.heads_inv);
                h = (int)(chunk - (int64_t)c * a.unit_heads);
                int lo = 0, hi = *a.n_long;           // chunk_ptr[lo] <= c < chunk_ptr[hi]
                while (hi - lo > 1) {
                    const int mid = lo + ((hi - lo) >> 1);
                    if (a.chunk_ptr[mid] <= c) lo = mid; else hi = mid;
                }
                row = a.long_rows[lo];
                beg = a.ptr[row] + (c - a.chunk_ptr[lo]) * kLongChunk;
                const int last = a.ptr[row + 1];
                steps = ((beg + kLongChunk < last ? beg + kLongChunk : last) - beg) * mult;
            }
        }
        int size = kSegment, slack = 0;               // steps of a segment
        if (a.units_a_wave < G) {
            int sum = steps;
#pragma unroll
            for (int d = L; d < kWave; d <<= 1) sum += __shfl_xor(sum, d, kWave);
            const int fair = (sum + G * U - 1) / (G * U) * U;
            size = fair < U ? U : fair < kSegment ? fair : kSegment;
            slack = kSlack;
        }
        const int segments = (steps + size - 1) / size;
        int upto = segments, total = 1;               // of this group and those before, and of all
        const bool cut = __any(steps > size + slack);
        auto fence = []() __attribute__((always_inline)) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");          // a wavefront's LDS accesses are carried out in order
            __builtin_amdgcn_wave_barrier();
        };
        if (cut) {
#pragma unroll
            for (int d = L; d < kWave; d <<= 1) {
                const int before = __shfl_up(upto, d, kWave);
                upto += lane >= d ? before : 0;
            }
            total = __builtin_amdgcn_readlane(upto, kWave - 1);
            r.start(h);
            r.leave(slots, lane);
            fence();
        }
        for (int first = 0; first < total; first += G) {
            int its_row = row, its_h = h, its_beg = beg, i = 0, its_end = steps, of = gw;
            const int segment = first + gw;
            if (cut) {
                of = 0;                               // the group whose unit it belongs to: the first with upto > segment
#pragma unroll
                for (int d = G / 2; d > 0; d >>= 1) of += __shfl(upto, (of + d - 1) * L, kWave) <= segment ? d : 0;
                const int from = of * L;
                its_row = __shfl(row, from, kWave);
                its_h = __shfl(h, from, kWave);
                its_beg = __shfl(beg, from, kWave);
                its_end = __shfl(steps, from, kWave);
                i = (segment - __shfl(upto - segments, from, kWave)) * size;
                if (i + size < its_end) its_end = i + size;
                if (segment >= total) i = its_end = 0;
            }
            walk(its_row, its_h, its_beg, i, its_end);
            if (cut) {
                const bool mine = segment < total;
                const int id = mine ? of : -1;
#pragma unroll
                for (int d = L; d < kWave; d <<= 1) {
                    const int other = __shfl_down(id, d, kWave);
                    r.join(d, lane + d < kWave && other == id && mine);
                }
                const int before = __shfl_up(id, L, kWave);
                if (mine && (gw == 0 || before != id)) r.add(slots, of * L + r.w.l);
                fence();
            }
        }
        if (cut) {
            r.start(h);
            r.add_from(slots, lane);
            fence();
        }
        if (!on) continue;
        if (chunk >= 0) r.store_chunk(chunk);
        else r.store(row, h);
    }
}

// ------------------------------------------------------------------ forward
template <bool BF16, int PC, int LG_, bool NEAR>
struct ForwardRow {
    typedef Piece<BF16, PC> P;
    static constexpr int LG = LG_, N = P::N, UNROLL = LG >= 4 ? 4 : 2;
    static constexpr bool T = false;
    const AttnArgs &a;
    const Where<P, LG, NEAR> w;
    P q;                           // this row's own operand
    int head, col;                 // col: of the key head
    float acc[N], m, sum;
    __device__ __forceinline__ ForwardRow(const AttnArgs &args) : a(args), w(args.width) {}
    __device__ __forceinline__ void own(int64_t row, int h) { w.load(q, a.Q, row, a.ldq, h * a.width); }
    __device__ __forceinline__ void start(int h)
    {
        head = h;
        col = (int)over((uint32_t)h, a.shared_inv) * a.width;
        w.cut(q);
        m = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int x = 0; x < N; ++x) acc[x] = 0.f;
    }
    template <int U>
    __device__ __forceinline__ void step(Ahead<T, UNROLL> &next, int beg, int i, int steps)
    {
        P k[U], v[U];
        float s[U];
#pragma unroll
        for (int j = 0; j < U; ++j) w.load(k[j], a.K, next.col[j], a.ldk, col);
#pragma unroll
        for (int j = 0; j < U; ++j) w.load(v[j], a.V, next.col[j], a.ldv, col);
#pragma unroll
        for (int j = 0; j < U; ++j) s[j] = i + j < steps ? bias_of(a, next.bucket[j], head) : -INFINITY;
        if (i + U < steps) next.load(a, beg, i + U, steps);
        float most = m;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const float d = over_lanes<LG>(q.dot(k[j]));
            s[j] = s[j] == -INFINITY ? s[j] : fmaf(d, a.scale, s[j]);
            most = fmaxf(most, s[j]);
        }
        const float base = most == -INFINITY ? 0.f : most, old = exp_of(m - base);
        m = most;
        sum *= old;
#pragma unroll
        for (int x = 0; x < N; ++x) acc[x] *= old;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const float p = exp_of(s[j] - base);
            sum += p;
            v[j].keep(p != 0.f);
#pragma unroll
            for (int x = 0; x < N; ++x) acc[x] = fmaf(p, v[j].get(x), acc[x]);
        }
    }
    // What another part of the row left: its maximum, sum and sums of rows.
    __device__ __forceinline__ void merge(float m2, float sum2, const float (&acc2)[N])
    {
        const float most = fmaxf(m, m2), base = most == -INFINITY ? 0.f : most, by = exp_of(m - base), by2 = exp_of(m2 - base);
        m = most;
        sum = sum * by + sum2 * by2;
#pragma unroll
        for (int x = 0; x < N; ++x) acc[x] = acc[x] * by + acc2[x] * by2;
    }
    __device__ __forceinline__ void join(int d, bool on)
    {
        const float m2 = __shfl_down(m, d, kWave), sum2 = __shfl_down(sum, d, kWave);
        float acc2[N];
#pragma unroll
        for (int x = 0; x < N; ++x) acc2[x] = __shfl_down(acc[x], d, kWave);
        if (on) merge(m2, sum2, acc2);
    }
    static constexpr int VALUES = N + 2;
    __device__ __forceinline__ void leave(float (&slots)[VALUES][kWave], int at) const
    {
        slots[0][at] = m;
        slots[1][at] = sum;
#pragma unroll
        for (int x = 0; x < N; ++x) slots[2 + x][at] = acc[x];
    }
    __device__ __forceinline__ void add_from(float (&slots)[VALUES][kWave], int at)
    {
        float acc2[N];
#pragma unroll
        for (int x = 0; x < N; ++x) acc2[x] = slots[2 + x][at];
        merge(slots[0][at], slots[1][at], acc2);
    }
    __device__ __forceinline__ void add(float (&slots)[VALUES][kWave], int at)
    {
        add_from(slots, at);
        leave(slots, at);
    }
    __device__ __forceinline__ void store_chunk(int64_t at)
    {
        w.store_sums(a.part, at * a.width, acc);
        if (w.l == 0) {
            a.part_more[2 * at] = m;
            a.part_more[2 * at + 1] = sum;
        }
    }
    __device__ __forceinline__ void store(int64_t row, int h)
    {
        const float by = sum == 0.f ? 0.f : 1.f / sum;
        float o[N];
#pragma unroll
        for (int x = 0; x < N; ++x) o[x] = acc[x] * by;
        w.store(a.O, row, a.ldo, h * a.width, o);
        if (a.lse && w.l == 0) a.lse[row * a.heads + h] = sum == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(sum) * kLn2;
    }
};

// Wavefronts a SIMD hide the gathers' latency: the 512 345 rows with four edges under way and three wavefronts 345 us, with two and four 297.
template <bool BF16, int PC, int LG, bool NEAR>
__global__ __launch_bounds__(kBlock, LG >= 4 ? 3 : 4) void k_attn_fwd(AttnArgs a)
{
    walk_units<ForwardRow<BF16, PC, LG, NEAR>>(a);
}

// ------------------------------------------------------------------ dQ
// sum p dp comes with the sums of p dp K and p K in one walk: dQ = scale (sum p dp K - (sum p dp) sum p K), all of them of e^(s - maximum)
// first and divided by its sum at the end.  dp is taken less a reference, the mean of p dp so far, to which the sums are brought in every step and
// where parts are joined: one operation an element and step.  It changes no result but its error, which goes with |dp - delta| as if delta were known before (dp itself loses where V
// or K have a mean, dp less that of any one edge where K has), and a row of one edge has none.  Relative errors in float32 arithmetic with dp as it is / less the first edge's /
// so / from a delta known before, 100 edges: no means 3.0e-7 / 7.0e-7 / 3.1e-7 / 2.9e-7; K's mean 1 4.6e-7 / 2.0e-6 / 3.5e-7 / 4.0e-7; V's 4, K's 2 1.6e-5 / 3.9e-6 / 5.8e-7 / 1.1e-5.
template <bool BF16, int PC, int LG_, bool NEAR>
struct QueryRow {
    typedef Piece<BF16, PC> P;
    static constexpr int LG = LG_, N = P::N, UNROLL = LG >= 4 ? 4 : 2;
    static constexpr bool T = false;
    const AttnArgs &a;
    const Where<P, LG, NEAR> w;
    P q, g;                        // this row's own operands
    int head, col;
    float pk[N], pdk[N], m, sum, delta, ref;      // pdk and delta: of dp - ref
    __device__ __forceinline__ QueryRow(const AttnArgs &args) : a(args), w(args.width) {}
    __device__ __forceinline__ void own(int64_t row, int h)
    {
        w.load(q, a.Q, row, a.ldq, h * a.width);
        w.load(g, a.dO, row, a.lddo, h * a.width);
    }
    __device__ __forceinline__ void start(int h)
    {
        head = h;
        col = (int)over((uint32_t)h, a.shared_inv) * a.width;
        w.cut(q);
        w.cut(g);
        m = -INFINITY;
        sum = delta = ref = 0.f;
#pragma unroll
        for (int x = 0; x < N; ++x) pk[x] = pdk[x] = 0.f;
    }
    template <int U>
    __device__ __forceinline__ void step(Ahead<T, UNROLL> &next, int beg, int i, int steps)
    {
        P k[U], v[U];
        float s[U];
#pragma unroll
        for (int j = 0; j < U; ++j) w.load(k[j], a.K, next.col[j], a.ldk, col);
#pragma unroll
        for (int j = 0; j < U; ++j) w.load(v[j], a.V, next.col[j], a.ldv, col);
#pragma unroll
        for (int j = 0; j < U; ++j) s[j] = i + j < steps ? bias_of(a, next.bucket[j], head) : -INFINITY;
        if (i + U < steps) next.load(a, beg, i + U, steps);
        float most = m, dp[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const float d = over_lanes<LG>(q.dot(k[j]));
            dp[j] = over_lanes<LG>(g.dot(v[j]));
            s[j] = s[j] == -INFINITY ? s[j] : fmaf(d, a.scale, s[j]);
            most = fmaxf(most, s[j]);
        }
        const float base = most == -INFINITY ? 0.f : most, old = exp_of(m - base);
        m = most;
        sum *= old;
        delta *= old;
        float p[U], all = sum, off = delta;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            p[j] = exp_of(s[j] - base);
            all += p[j];
            off += p[j] == 0.f ? 0.f : p[j] * (dp[j] - ref);
        }
        const float more = to_mean(off, all);
        delta = fmaf(more, sum, delta);
        sum = all;
#pragma unroll
        for (int x = 0; x < N; ++x) {
            pk[x] *= old;
            pdk[x] = fmaf(more, pk[x], pdk[x] * old);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const float pd = p[j] == 0.f ? 0.f : p[j] * (dp[j] - ref);
            delta += pd;
            k[j].keep(p[j] != 0.f);
#pragma unroll
            for (int x = 0; x < N; ++x) {
                pk[x] = fmaf(p[j], k[j].get(x), pk[x]);
                pdk[x] = fmaf(pd, k[j].get(x), pdk[x]);
            }
        }
    }
    // Brings the reference to the mean of sums off / all; what a sum of p (dp - ref) has to be given for each p.
    __device__ __forceinline__ float to_mean(float off, float all)
    {
        const float before = ref;
        ref = all > 0.f ? fmaf(off, __builtin_amdgcn_rcpf(all), ref) : ref;
        return before - ref;
    }
    __device__ __forceinline__ void merge(const float (&v)[2 * N + 4])
    {
        const float most = fmaxf(m, v[0]), base = most == -INFINITY ? 0.f : most, by = exp_of(m - base), by2 = exp_of(v[0] - base);
        const float off = delta * by + fmaf(v[3] - ref, v[1], v[2]) * by2, all = sum * by + v[1] * by2;
        const float more = to_mean(off, all), more2 = v[3] - ref;             // of a part that has nothing: times sums that are 0
        m = most;
        delta = fmaf(more, sum, delta) * by + fmaf(more2, v[1], v[2]) * by2;
        sum = all;
#pragma unroll
        for (int x = 0; x < N; ++x) {
            pdk[x] = fmaf(more, pk[x], pdk[x]) * by + fmaf(more2, v[4 + x], v[4 + N + x]) * by2;
            pk[x] = pk[x] * by + v[4 + x] * by2;
        }
    }
    __device__ __forceinline__ void join(int d, bool on)
    {
        float v[2 * N + 4];
        v[0] = __shfl_down(m, d, kWave);
        v[1] = __shfl_down(sum, d, kWave);
        v[2] = __shfl_down(delta, d, kWave);
        v[3] = __shfl_down(ref, d, kWave);
#pragma unroll
        for (int x = 0; x < N; ++x) {
            v[4 + x] = __shfl_down(pk[x], d, kWave);
            v[4 + N + x] = __shfl_down(pdk[x], d, kWave);
        }
        if (on) merge(v);
    }
    static constexpr int VALUES = 2 * N + 4;
    __device__ __forceinline__ void leave(float (&slots)[VALUES][kWave], int at) const
    {
        slots[0][at] = m;
        slots[1][at] = sum;
        slots[2][at] = delta;
        slots[3][at] = ref;
#pragma unroll
        for (int x = 0; x < N; ++x) {
            slots[4 + x][at] = pk[x];
            slots[4 + N + x][at] = pdk[x];
        }
    }
    __device__ __forceinline__ void add_from(float (&slots)[VALUES][kWave], int at)
    {
        float v[2 * N + 4];
#pragma unroll
        for (int x = 0; x < VALUES; ++x) v[x] = slots[x][at];
        merge(v);
    }
    __device__ __forceinline__ void add(float (&slots)[VALUES][kWave], int at)
    {
        add_from(slots, at);
        leave(slots, at);
    }
    __device__ __forceinline__ void store_chunk(int64_t at)
    {
        w.store_sums(a.part, at * a.width, pdk);
        w.store_sums(a.part + a.part_stride, at * a.width, pk);
        if (w.l == 0) reinterpret_cast<f32x4 *>(a.part_more)[at] = f32x4{m, sum, delta, ref};
    }
    __device__ __forceinline__ void store(int64_t r, int h)
    {
        const float by = sum == 0.f ? 0.f : 1.f / sum, d = delta * by;
        float o[N];
#pragma unroll
        for (int x = 0; x < N; ++x) o[x] = a.scale * by * fmaf(-d, pk[x], pdk[x]);
        if (a.dQ) w.store(a.dQ, r, a.lddq, h * a.width, o);
        if (w.l == 0) a.stats[r * a.heads + h] = f32x4{m, by, ref + d, 0.f};
    }
};

// 91 331 rows of 10, eight bf16 heads of 32: four edges under way 160 us, two 148 (0.96 GB, most of it gathered, at 6.5 TB/s).  The transposed order's buckets come along
// in place of a launch of their own.
template <bool BF16, int PC, int LG, bool NEAR>
__global__ __launch_bounds__(kBlock, LG >= 4 ? 2 : BF16 ? 3 : 4) void k_attn_dq(AttnArgs a)
{
    if (a.bucket_to)
        for (int64_t i = block_of() * kBlock + threadIdx.x; i < a.edges; i += (int64_t)gridDim.x * gridDim.y * kBlock) a.bucket_to[i] = a.bucket_from[a.eid[i]];
    walk_units<QueryRow<BF16, PC, LG, NEAR>>(a);
}

// ------------------------------------------------------------------ dK, dV
// Rows are sources; a unit has one of the key heads, and its row's edges once for each query head that shares it.
template <bool BF16, int PC, int LG_, bool NEAR, int U_>
struct KeyRow {
    typedef Piece<BF16, PC> P;
    static constexpr int LG = LG_, N = P::N, UNROLL = U_;
    static constexpr bool T = true;
    const AttnArgs &a;
    const Where<P, LG, NEAR> w;
    P k, v;                        // this row's own operands
    int head;                      // the first of the query heads
    float dk[N], dv[N];
    __device__ __forceinline__ KeyRow(const AttnArgs &args) : a(args), w(args.width) {}
    __device__ __forceinline__ void own(int64_t row, int hk)
    {
        w.load(k, a.K, row, a.ldk, hk * a.width);
        w.load(v, a.V, row, a.ldv, hk * a.width);
    }
    __device__ __forceinline__ void start(int hk)
    {
        head = hk * a.shared;
        w.cut(k);
        w.cut(v);
#pragma unroll
        for (int x = 0; x < N; ++x) dk[x] = dv[x] = 0.f;
    }
    template <int U>
    __device__ __forceinline__ void step(Ahead<T, UNROLL> &next, int beg, int i, int steps)
    {
        P q[U], g[U];
        float s[U];
        f32x4 stats[U];
        int pos[U], its[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int h = head + next.head[j];
            w.load(q[j], a.Q, next.col[j], a.ldq, h * a.width);
            w.load(g[j], a.dO, next.col[j], a.lddo, h * a.width);
            stats[j] = a.stats[(int64_t)next.col[j] * a.heads + h];
            s[j] = i + j < steps ? bias_of(a, next.bucket[j], h) : -INFINITY;
            pos[j] = next.pos[j];
            its[j] = h;
        }
        const int last = steps - i;
        if (i + U < steps) next.load(a, beg, i + U, steps);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const float d = over_lanes<LG>(k.dot(q[j])), dp = over_lanes<LG>(v.dot(g[j]));
            const float z = s[j] == -INFINITY ? s[j] : fmaf(d, a.scale, s[j]), p = z == -INFINITY ? 0.f : exp_of(z - stats[j][0]) * stats[j][1];
            const float ds = p == 0.f ? 0.f : p * (dp - stats[j][2]);
            if (a.ds && w.l == 0 && j < last) a.ds[(int64_t)pos[j] * a.heads + its[j]] = ds;
            q[j].keep(p != 0.f);
            g[j].keep(p != 0.f);
#pragma unroll
            for (int x = 0; x < N; ++x) {
                dk[x] = fmaf(ds, q[j].get(x), dk[x]);
                dv[x] = fmaf(p, g[j].get(x), dv[x]);
            }
        }
    }
    __device__ __forceinline__ void join(int d, bool on)
    {
#pragma unroll
        for (int x = 0; x < N; ++x) {
            const float k2 = __shfl_down(dk[x], d, kWave), v2 = __shfl_down(dv[x], d, kWave);
            dk[x] += on ? k2 : 0.f;
            dv[x] += on ? v2 : 0.f;
        }
    }
    static constexpr int VALUES = 2 * N;
    __device__ __forceinline__ void leave(float (&slots)[VALUES][kWave], int at) const
    {
#pragma unroll
        for (int x = 0; x < N; ++x) {
            slots[x][at] = dk[x];
            slots[N + x][at] = dv[x];
        }
    }
    __device__ __forceinline__ void add_from(float (&slots)[VALUES][kWave], int at)
    {
#pragma unroll
        for (int x = 0; x < N; ++x) {
            dk[x] += slots[x][at];
            dv[x] += slots[N + x][at];
        }
    }
    __device__ __forceinline__ void add(float (&slots)[VALUES][kWave], int at)
    {
        add_from(slots, at);
        leave(slots, at);
    }
    __device__ __forceinline__ void store_chunk(int64_t at)
    {
        w.store_sums(a.part, at * a.width, dk);
        w.store_sums(a.part + a.part_stride, at * a.width, dv);
    }
    __device__ __forceinline__ void store(int64_t r, int hk)
    {
        float o[N];
#pragma unroll
        for (int x = 0; x < N; ++x) o[x] = dk[x] * a.scale;
        if (a.dK) w.store(a.dK, r, a.lddk, hk * a.width, o);
        if (a.dV) w.store(a.dV, r, a.lddv, hk * a.width, dv);
    }
};

// A source has few edges, and its own rows are read and written: 512 345 sources of 1.6 edges, eight bf16 heads of 32, 334 us: 1.05 GB of own rows and 0.92
// gathered, 5.9 TB/s.  One edge under way where heads share no key head: that 332 us, two 372;  two where they do, as a row then has as many steps more: 8000 rows of 15,
// four f32 heads of 47 on one, 49 us, one 66.
template <bool BF16, int PC, int LG, bool NEAR, int U>
__global__ __launch_bounds__(kBlock, U == 1 ? 4 : 3) void k_attn_dkv(AttnArgs a)
{
    walk_units<KeyRow<BF16, PC, LG, NEAR, U>>(a);
}

// ------------------------------------------------------------------ chunks of long rows
// A workgroup has one long row and 2^lg of its columns at a time, and as many parts of its chunks as threads are left; the parts are joined in
// order.  Latency bounds it: 4.5 us where there is no long row (the host does not know), 13 to 16 where 65 536 rows have chunks by the thousand.  KIND 0: O and lse, 1: dQ and the row's numbers, 2: dK and dV.
template <bool BF16, int KIND>
__global__ __launch_bounds__(kJoin) void k_attn_join(AttnArgs a, int lg)
{
    typedef typename std::conditional<BF16, uint16_t, float>::type T;
    constexpr int MORE = KIND == 1 ? 4 : 2, NS = KIND == 0 ? 2 : KIND == 1 ? 4 : 2;       // sums: columns' (one or two), the row's
    const int cols = a.unit_heads * a.width, tiles = (cols + (1 << lg) - 1) >> lg, parts = kJoin >> lg;
    const int c = threadIdx.x & ((1 << lg) - 1), part = threadIdx.x >> lg;
    __shared__ float sums[NS][kJoin], most[kJoin], refs[KIND == 1 ? kJoin : 1];
    const int64_t total = (int64_t)*a.n_long * tiles;
    for (int64_t unit = blockIdx.x; unit < total; unit += gridDim.x) {
        const int li = (int)(unit / tiles), col = ((int)(unit - (int64_t)li * tiles) << lg) + c;
        const int64_t row = a.long_rows[li];
        const int first = a.chunk_ptr[li], n = a.chunk_ptr[li + 1] - first, per = (n + parts - 1) / parts;
        const int lo = first + part * per, hi = lo + per < first + n ? lo + per : first + n;
        const int h = col < cols ? col / a.width : 0;
        const float *p = a.part + (col < cols ? col : 0), *more = a.part_more;
        float v[NS], m = -INFINITY, ref = 0.f;        // ref: of the chunk with the maximum, see dQ's walk
#pragma unroll
        for (int i = 0; i < NS; ++i) v[i] = 0.f;
        if (KIND != 2)
#pragma unroll 4
            for (int k = lo; k < hi; ++k) {
                const int64_t at = MORE * ((int64_t)k * a.unit_heads + h);
                const float its = more[at];
                if constexpr (KIND == 1) ref = its > m ? more[at + 3] : ref;
                m = fmaxf(m, its);
            }
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 4
        for (int k = lo; k < hi; ++k) {
            const int64_t at = MORE * ((int64_t)k * a.unit_heads + h), to = (int64_t)k * cols;
            if constexpr (KIND == 2) {
                v[0] += p[to];
                v[1] += p[a.part_stride + to];
            } else {
                const float by = exp_of(more[at] - base);
                v[1] += by * more[at + 1];
                if constexpr (KIND == 0) {
                    v[0] += by == 0.f ? 0.f : by * p[to];
                } else {
                    const float x = more[at + 3] - ref, pk = p[a.part_stride + to];
                    v[0] += by == 0.f ? 0.f : by * fmaf(x, pk, p[to]);
                    v[2] += by == 0.f ? 0.f : by * pk;
                    v[3] += by == 0.f ? 0.f : by * fmaf(x, more[at + 1], more[at + 2]);
                }
            }
        }
        __syncthreads();                              // the row before has been read
#pragma unroll
        for (int i = 0; i < NS; ++i) sums[i][threadIdx.x] = v[i];
        if (KIND != 2) most[threadIdx.x] = m;
        if (KIND == 1) refs[threadIdx.x] = ref;
        __syncthreads();
        if (part != 0 || col >= cols) continue;       // the barriers of the next row are reached by all
        if (KIND != 2)
            for (int r = 1; r < parts; ++r) {
                const float its = most[(r << lg) + c];
                if constexpr (KIND == 1) ref = its > m ? refs[(r << lg) + c] : ref;
                m = fmaxf(m, its);
            }
        const float all = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < NS; ++i) v[i] = 0.f;
        for (int r = 0; r < parts; ++r) {
            const float by = KIND == 2 ? 1.f : exp_of(most[(r << lg) + c] - all);
            const float x = KIND == 1 ? refs[KIND == 1 ? (r << lg) + c : 0] - ref : 0.f;
#pragma unroll
            for (int i = 0; i < NS; ++i) {            // a sum of NaN (its scores leave no maximum) stays: every result is divided by it
                const bool none = by == 0.f && (KIND == 2 || i != 1);
                float its = sums[i][(r << lg) + c];
                if (KIND == 1 && (i == 0 || i == 3)) its = fmaf(x, sums[i == 0 ? 2 : 1][(r << lg) + c], its);
                v[i] += none ? 0.f : by * its;
            }
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
                if (col == h * a.width) a.stats[row * a.heads + h] = f32x4{m, by, ref + delta, 0.f};
            }
        }
    }
}

// ------------------------------------------------------------------ dbias
// A workgroup adds up ds of a run of edges into tables of its own in LDS: one for every edge that it has under way, so that no two threads
// meet; then table by table.  Buckets are taken kBiasTile at a time, heads 2^lg at a time.
struct BiasArgs {
    const float *ds;               // [position][heads]
    const int32_t *bucket;         // [position]
    float *part;                   // [workgroup][buckets][heads]
    int64_t positions;
    int32_t heads, buckets, lg;
};

__global__ __launch_bounds__(kBlock) void k_attn_dbias(BiasArgs a)
{
    extern __shared__ float table[];                  // [bucket][edge under way][head]
    const int hs = 1 << a.lg, slots = kBlock >> a.lg, head0 = (int)blockIdx.z * hs, first = (int)blockIdx.y * kBiasTile;
    const int tile = a.buckets - first < kBiasTile ? a.buckets - first : kBiasTile;
    const int h = head0 + (threadIdx.x & (hs - 1)), slot = threadIdx.x >> a.lg;
    for (int i = 0; i < tile; ++i) table[i * kBlock + threadIdx.x] = 0.f;
    const int64_t per = (a.positions + gridDim.x - 1) / gridDim.x, beg = per * blockIdx.x, last = beg + per < a.positions ? beg + per : a.positions;
    if (h < a.heads) {                                // a thread's column is its own: no barrier before the tables are read
        int64_t t = beg + slot;
        constexpr int U = 8;
        for (; t + (U - 1) * slots < last; t += U * slots) {
            int b[U];
            float x[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                b[j] = a.bucket[t + j * slots] - first;
                x[j] = a.ds[(t + j * slots) * a.heads + h];
            }
#pragma unroll
            for (int j = 0; j < U; ++j)
                if ((uint32_t)b[j] < (uint32_t)tile) table[b[j] * kBlock + threadIdx.x] += x[j];
        }
        for (; t < last; t += slots) {
            const int b = a.bucket[t] - first;
            if ((uint32_t)b < (uint32_t)tile) table[b * kBlock + threadIdx.x] += a.ds[t * a.heads + h];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < tile * hs; i += kBlock) {
        const int b = i >> a.lg, c = i & (hs - 1);
        float v = 0.f;
        for (int r = 0; r < slots; ++r) v += table[b * kBlock + (r << a.lg) + c];
        if (head0 + c < a.heads) a.part[((int64_t)blockIdx.x * a.buckets + first + b) * a.heads + head0 + c] = v;
    }
}

// Eight entries of the table a workgroup, 32 threads each.
__global__ __launch_bounds__(kBlock) void k_attn_dbias_sum(const float *part, int blocks, int64_t n, float *dbias)
{
    __shared__ double sums[kBlock / 8][9];
    const int c = threadIdx.x & 7, r = threadIdx.x >> 3;
    const int64_t at = block_of() * 8 + c;
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
    int32_t *bucket;
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
        bucket = nullptr;
        plan = nullptr;
        const int64_t chunks = d.num_edges > kLongThreshold ? cap_chunks(d.num_edges) : 0;
        part_stride = chunks * d.heads * d.width;
        part = take(part_stride * (backward ? 2 : 1));
        part_more = take(chunks * d.heads * (backward ? 4 : 2));
        if (backward) {
            stats = take(d.num_dst * d.heads * 4);
            if (d.bucket) bucket = reinterpret_cast<int32_t *>(take(d.num_edges));
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

// Lanes of a head: two pieces each, so that what is done once an edge and lane counts less; one piece where there is no more.
// near: whether offsets into all arrays of rows are below 2^32.
template <class F>
fastgl_status by_shape(fastgl_dtype dtype, int64_t width, bool near, F f)
{
    const bool bf16 = dtype == FASTGL_BF16;
    const int64_t n = bf16 ? 8 : 4, pieces = ceil_div(width, n);
    typedef std::true_type Yes;
    typedef std::false_type No;
    typedef std::integral_constant<int, 0> I0;
    typedef std::integral_constant<int, 1> I1;
    typedef std::integral_constant<int, 2> I2;
    if (width < n) return bf16 ? f(Yes(), I0(), std::integral_constant<int, 3>(), No()) : f(No(), I0(), I2(), No());
    auto lanes = [&](auto b, auto near_) {
        if (pieces <= 1) return f(b, I1(), I0(), near_);
        if (pieces <= 2) return f(b, I2(), I0(), near_);
        if (pieces <= 4) return f(b, I2(), I1(), near_);
        if (pieces <= 8) return f(b, I2(), I2(), near_);
        if (pieces <= 16) return f(b, I2(), std::integral_constant<int, 3>(), near_);
        if constexpr (decltype(b)::value) return f(b, I2(), std::integral_constant<int, 4>(), near_);
        else {
            if (pieces <= 32) return f(b, I2(), std::integral_constant<int, 4>(), near_);
            return f(b, I2(), std::integral_constant<int, 5>(), near_);
        }
    };
    if (near) return bf16 ? lanes(Yes(), Yes()) : lanes(No(), Yes());
    return bf16 ? lanes(Yes(), No()) : lanes(No(), No());
}

dim3 grid_of(int64_t blocks)                          // blocks beyond the last have nothing
{
    const int64_t x = (int64_t)1 << 20;
    return blocks <= x ? dim3((unsigned)blocks) : dim3((unsigned)x, (unsigned)ceil_div(blocks, x));
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
    a.rows = rows;
    a.dealt = T && rows >= 512;
    a.units = (a.dealt ? (int64_t)align_up((size_t)rows, 512) : rows) * a.unit_heads;
    a.heads_inv = a.unit_heads > 1 ? UINT64_MAX / (uint64_t)a.unit_heads + 1 : 0;
    // The hint may be wrong: a wavefront's units together then have up to 64 num_edges steps, which are counted in 32 bits.
    const bool chunked = d.num_edges > kLongThreshold && (T || !(pl->parts & FASTGL_PLAN_SHORT_DST_ROWS) || d.num_edges > kHintEdges);
    a.long_thr = chunked ? kLongThreshold : INT32_MAX;
    if (chunked) {
        a.long_rows = T ? pl->long_src : pl->long_dst;
        a.chunk_ptr = T ? pl->chunk_ptr_src : pl->chunk_ptr_dst;
        a.n_long = pl->counters + (T ? 2 : 0);
        a.n_chunks = pl->counters + (T ? 3 : 1);
    }
    if (a.units == 0) return FASTGL_OK;
    const int64_t el = d.dtype == FASTGL_BF16 ? 2 : 4, far = (int64_t)UINT32_MAX / el;
    const bool near = d.num_dst * d.ldq <= far && d.num_src * d.ldk <= far && d.num_src * d.ldv <= far && d.num_dst * a.lddo <= far;
    const fastgl_status st = by_shape(d.dtype, d.width, near, [&](auto bf16, auto pc, auto lg, auto near_) {
        constexpr bool B = decltype(bf16)::value, NEAR = decltype(near_)::value;
        constexpr int PC = decltype(pc)::value, LG = decltype(lg)::value;
        // Fewer units a wavefront where there are few: so many that four wavefronts a compute unit have some, sixteen for rows of sources and wide heads
        // (few groups a wavefront).  us, units to all groups / so: 105 rows of 15 heads, 93 sources, dK and dV 59 / 9;  597 rows of up to 350 edges, heads
        // of 160 fp32 columns, forward 87 / 46;  16 843 rows of 16, 2 heads of 12 columns, dQ 10.4 / 10.4, with sixteen 17.
        const int64_t groups = kWave >> LG, few = ceil_div(a.units, T || LG >= 4 ? 4096 : 1024);
        a.units_a_wave = (int32_t)(few <= groups / 2 ? few : groups);
        // Rows of sources with many steps: as few as have kTransposedSteps a group on average, so that the neighbours of many do not meet in one wavefront.
        // us, dK and dV: 2350 sources of 28 edges, 32 heads of one f32 column, eight to a key head 146 / 76 (8: 76, 16: 110);  45 157 sources of 4, 40 heads of 12 on
        // five 357 / 238 (8: 248, 16: 282);  19 239 of 5, 18 of 19 on six 137 / 115.  Rows of targets, of alike lengths, lose by it: 30 / 49.
        if (T && d.num_edges > 0) {
            const int64_t so = ceil_div(groups * kTransposedSteps * rows, d.num_edges * a.shared);
            if (so < a.units_a_wave) a.units_a_wave = (int32_t)so;
        }
        const int64_t blocks = ceil_div(a.units, (int64_t)a.units_a_wave * (kBlock / kWave));
        if (blocks > (int64_t)65535 << 20) {
            set_error("%s: too many rows and heads", names[PASS]);
            return FASTGL_ERR_UNSUPPORTED;
        }
        a.chunk_waves = (int32_t)((blocks < 2048 ? blocks : 2048) * (kBlock / kWave));
        if constexpr (PASS == kPassFwd) hipLaunchKernelGGL((k_attn_fwd<B, PC, LG, NEAR>), grid_of(blocks), dim3(kBlock), 0, s, a);
        else if constexpr (PASS == kPassDq) hipLaunchKernelGGL((k_attn_dq<B, PC, LG, NEAR>), grid_of(blocks), dim3(kBlock), 0, s, a);
        else if (a.shared == 1) hipLaunchKernelGGL((k_attn_dkv<B, PC, LG, NEAR, 1>), grid_of(blocks), dim3(kBlock), 0, s, a);
        else hipLaunchKernelGGL((k_attn_dkv<B, PC, LG, NEAR, 2>), grid_of(blocks), dim3(kBlock), 0, s, a);
        FASTGL_LAUNCH_CHECK(names[PASS]);
        return FASTGL_OK;
    });
    if (st != FASTGL_OK || !chunked) return st;
    const int cols = a.unit_heads * a.width;
    int lg = 5;
    while (lg < 8 && (1 << lg) < cols) ++lg;
    const int64_t units = cap_long_rows(d.num_edges) * ceil_div(cols, (int64_t)1 << lg);
    const dim3 grid((unsigned)(units < 1024 ? units : 1024));
    if (d.dtype == FASTGL_BF16) hipLaunchKernelGGL((k_attn_join<true, PASS>), grid, dim3(kJoin), 0, s, a, lg);
    else hipLaunchKernelGGL((k_attn_join<false, PASS>), grid, dim3(kJoin), 0, s, a, lg);
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
    a.stats = reinterpret_cast<f32x4 *>(o.stats);
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
    if (d.bucket && (dK || dV || dbias)) {
        a.bucket_from = d.bucket; a.eid = plan->perm;
        a.bucket_to = o.bucket;
        a.edges = d.num_edges;
    }
    if ((st = launch_walk<kPassDq>(a, d, plan, s)) != FASTGL_OK) return st;
    if (!dK && !dV && !dbias) return FASTGL_OK;
    AttnArgs b = args_of(d, o);
    b.ptr = plan->indptr_T; b.col = plan->indices_T;
    b.bucket = o.bucket;
    b.dO = dO; b.lddo = lddo;
    b.dK = dK; b.lddk = lddk;
    b.dV = dV; b.lddv = lddv;
    b.ds = dbias ? o.ds : nullptr;
    if ((st = launch_walk<kPassDkv>(b, d, plan, s)) != FASTGL_OK) return st;
    if (!dbias) return FASTGL_OK;
    BiasArgs c = {};
    c.ds = o.ds;
    c.bucket = o.bucket;
    c.part = o.bias;
    c.positions = d.num_edges;
    c.heads = (int32_t)d.heads; c.buckets = (int32_t)d.num_buckets;
    while (c.lg < 5 && (1 << c.lg) < d.heads) ++c.lg;
    const int64_t blocks = Scratch::bias_blocks(d), table = d.num_buckets * d.heads;
    const dim3 grid((unsigned)blocks, (unsigned)ceil_div(d.num_buckets, kBiasTile), (unsigned)ceil_div(d.heads, (int64_t)1 << c.lg));
    const size_t lds = sizeof(float) * kBlock * (size_t)(d.num_buckets < kBiasTile ? d.num_buckets : kBiasTile);
    hipLaunchKernelGGL(k_attn_dbias, grid, dim3(kBlock), lds, s, c);
    FASTGL_LAUNCH_CHECK("fastgl_attn_bwd (dbias)");
    hipLaunchKernelGGL(k_attn_dbias_sum, grid_of(ceil_div(table, 8)), dim3(kBlock), 0, s, (const float *)o.bias, (int)blocks, table, dbias);
    FASTGL_LAUNCH_CHECK("fastgl_attn_bwd (dbias, sums)");
    return FASTGL_OK;
}

}  // extern "C"
