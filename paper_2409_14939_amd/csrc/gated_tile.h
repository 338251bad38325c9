// The matrix-core tile of the gated feed-forward update: three kinds of product of one shape of kernel.
//
//   FORWARD  G, U [R,C]    = A [R,Kc] B0, B1 [Kc,C]         and the gate in the epilogue
//   ROWS     dX   [R,C]    = sum over groups of A [R,Kc] B [C,Kc]^T
//   WEIGHTS  dWg, dWu [R,C] = A [Kc,R]^T B0, B1 [Kc,C]       contracted range cut into slabs
//
// All operands are bf16 with rows of a multiple of 16 bytes; fp32 operands come as three planes of pieces, and a
// product of two such is a sequence of six segments, each a product of one plane of either.
//
// * A tile is 256 x 256 (eight wavefronts, 64 x 128 each) or 128 x 128 (four, 64 x 64): of two results, half the
//   columns each, so that a lane holds G and U of the same elements.  Contracted 64 at a time through two LDS buffers.
// * Operands go from memory to LDS without passing registers (16 bytes a lane).  An operand whose contracted
//   index is contiguous lies as [row][64], read 16 bytes a lane; one whose other index is contiguous lies as [64][column] and is
//   turned on its way out of LDS by the transposing reads.  The 16-byte pieces of a row are permuted (by the addresses they
//   are loaded from) so that the lanes of a read meet different banks.
// * Buffer resources end the operands: what lies beyond is read as 0.  A row's last pieces beyond the contracted
//   range are given an address beyond the end.
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

enum TileMode { kForward = 0, kRows = 1, kWeights = 2 };

constexpr int kStep = 64;                       // contracted elements of an LDS buffer
constexpr uint32_t kNoSuchOffset = 0x7FFFFF00u; // beyond every buffer
constexpr int64_t kMostRecords = 0x7FFF0000;
constexpr int kTileRsrc = 0x00020000;

struct TileArgs {
    const uint16_t *a[2], *b[2];   // FORWARD, WEIGHTS: a[0] and b[0], b[1]; ROWS: group g has a[g], b[g]
    int64_t a_plane, b_plane;      // elements between planes of pieces
    int64_t lda, ldb;              // elements between rows, multiples of 8; contiguous contracted elements are 0 from Kc to there
    int64_t R, C, Kc;
    int32_t pairs, groups;         // segments: groups x pairs; pairs is 1 (bf16) or 6 (three planes)
    int64_t slab;                  // WEIGHTS: contracted elements of a slab, a multiple of kStep
    int32_t tiles_r, tiles_c, slabs;
    const float *bias[2];          // FORWARD, or NULL
    int32_t act;
    void *out[3];                  // FORWARD: P, G, U (G, U or NULL); ROWS: dX; WEIGHTS: dWg, dWu, or their partial sums
    int64_t out_slab;              // WEIGHTS with partial sums: elements between those of two slabs
};

// Segment i of six: the planes of A and of B, smallest products first.
__device__ __forceinline__ int plane_a(int i) { return (0x001120 >> (4 * i)) & 15; }       // 0 2 1 1 0 0
__device__ __forceinline__ int plane_b(int i) { return (0x010102 >> (4 * i)) & 15; }       // 2 0 1 0 1 0

// exp(-x), x >= 0 or any: 2^(-x log2 e).  Relative error 2^-23 (1 + |x|): the rounding of the exponent.
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(-1.44269504089f * x); }

// act(g) and, where wanted, its derivative.  The sigmoid is 1 / (1 + exp(-g)).  The normal distribution of GELU:
// erfc(x) = (a1 t + ... + a5 t^5) exp(-x^2), t = 1 / (1 + p x) (Hastings; Abramowitz and Stegun 7.1.26, error below
// 1.5e-7), whose exponential is that of the density, so the derivative costs two products more.
template <int ACT, bool GRAD>
__device__ __forceinline__ float gate(float g, float *grad)
{
    if constexpr (ACT == FASTGL_ACT_RELU) {
        if (GRAD) *grad = g > 0.f ? 1.f : g != g ? g : 0.f;
        return g < 0.f ? 0.f : g;                            // NaN stays NaN
    } else if constexpr (ACT == FASTGL_ACT_GELU) {
        const float x = fabsf(g) * 0.70710678118f;
        const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
        const float e = exp_neg(x * x);
        const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
        const float tail = 0.5f * poly * e;
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

template <int MODE, int NW>
struct Tile {
    static constexpr int BM = NW == 8 ? 256 : 128, BNV = BM;             // rows and columns of all results together
    static constexpr int WM = NW == 8 ? 4 : 2, WN = 2;
    static constexpr int TM = BM / WM / 32, TN = BNV / WN / 32;
    static constexpr bool DUAL = MODE != kRows;
    static constexpr int BC = DUAL ? BNV / 2 : BNV;                     // columns of one result
    static constexpr bool A_T = MODE == kWeights, B_T = MODE != kRows;  // other index contiguous
    static constexpr int A_BYTES = BM * kStep * 2, B_BYTES = BNV * kStep * 2, STAGE = A_BYTES + B_BYTES;
    static constexpr int THREADS = NW * kWave;
    static constexpr int LOADS = A_BYTES / (THREADS * 16);              // 16-byte loads a lane, of either operand
    static_assert(TM == 2 && LOADS == 4 && B_BYTES == A_BYTES, "tile shape");
};

// Which 16-byte piece of row k a [64][columns] buffer has at place p: rows of RB bytes.  Reads take 64 bytes of four
// consecutive rows at a time, which this puts 64 bytes apart modulo 256.
template <int RB>
__device__ __forceinline__ int turned(int k) { return RB >= 256 ? 4 * (k & 3) : 4 * ((k >> 1) & 1); }
// The same for a [row][64] buffer (rows of 128 bytes), read one piece of 32 consecutive rows at a time.
__device__ __forceinline__ int twisted(int row) { return row & 7; }

namespace {

template <int MODE, int NW, class OUT, int ACT>
__global__ __launch_bounds__(NW * kWave, NW == 8 ? 2 : 2) void k_gated_tile(TileArgs g)
{
#ifdef __HIP_DEVICE_COMPILE__                    // the host pass makes no launch stub of a body with these builtins
    using T = Tile<MODE, NW>;
    __shared__ __attribute__((aligned(1024))) char lds[2 * T::STAGE];
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

    const int64_t k_first = MODE == kWeights ? (int64_t)slab * g.slab : 0;
    const int64_t k_len = MODE == kWeights ? (g.Kc - k_first < g.slab ? g.Kc - k_first : g.slab) : g.Kc;
    const int steps = (int)((k_len + kStep - 1) / kStep), nseg = g.pairs * g.groups;

    // Where this lane's 16-byte pieces come from, within a step, and to which step's pieces they belong.
    uint32_t off_a[4], off_b[4];
    const int piece_k = (lane & 7) ^ twisted(lane >> 3);                 // [row][64]: eight rows an instruction
    auto place = [&](auto turned_layout, int64_t ld, int columns, uint32_t(&off)[4], bool dual) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (!decltype(turned_layout)::value) {
                const int row = (i * NW + wave) * 8 + (lane >> 3);
                off[i] = (uint32_t)(row * ld * 2) + 16u * (uint32_t)piece_k;
            } else {
                // dual: the first two instructions load one operand, the others the other
                const int inst = dual ? (i & 1) * NW + wave : i * NW + wave;
                const int per_row = columns / 8, k = (inst * kWave + lane) / per_row, p = lane & (per_row - 1);
                const int c = p ^ (columns * 2 >= 256 ? turned<256>(k) : turned<128>(k));
                off[i] = (uint32_t)(k * ld * 2) + 16u * (uint32_t)c;
            }
        }
    };
    place(std::integral_constant<bool, T::A_T>(), g.lda, T::BM, off_a, false);
    place(std::integral_constant<bool, T::B_T>(), g.ldb, T::BC, off_b, T::DUAL);

    // The operands' places at segment `seg`, step `t`, and the loads of that step into LDS buffer `buf`.
    auto load_step = [&](int seg, int t, int buf) {
        const int grp = MODE == kRows ? seg / g.pairs : 0, pair = MODE == kRows ? seg - grp * g.pairs : seg;
        const int pa = g.pairs == 1 ? 0 : plane_a(pair), pb = g.pairs == 1 ? 0 : plane_b(pair);
        const uint16_t *a = g.a[grp] + pa * g.a_plane;
        const int64_t k = k_first + (int64_t)t * kStep, k_end = k_first + k_len;
        auto rsrc = [&](const uint16_t *p, int64_t start, int64_t end) {
            int64_t bytes = (end - start) * 2;
            bytes = bytes < 0 ? 0 : bytes > kMostRecords ? kMostRecords : bytes;
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(p + start), 0, (int)bytes, kTileRsrc);
        };
        const bool tail = !(T::A_T && T::B_T) && k + kStep > k_end;
        const uint32_t left = (uint32_t)(k_end - k + 7) / 8;             // pieces: rows are padded with zeros to a multiple of 8
        FASTGL_LDS char *to = (FASTGL_LDS char *)lds + buf * T::STAGE + wave * 1024;
        {
            const auto r = T::A_T ? rsrc(a, k * g.lda + row0, k_end * g.lda) : rsrc(a, row0 * g.lda + k, g.R * g.lda);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t o = off_a[i];
                if (!T::A_T && tail && (uint32_t)piece_k >= left) o = kNoSuchOffset;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (FASTGL_LDS void *)(to + i * NW * 1024), 16, (int)o, 0, 0, 0);
            }
        }
#pragma unroll
        for (int q = 0; q < (T::DUAL ? 2 : 1); ++q) {
            const uint16_t *b = (MODE == kRows ? g.b[grp] : g.b[q]) + pb * g.b_plane;
            const auto r = T::B_T ? rsrc(b, k * g.ldb + col0, k_end * g.ldb) : rsrc(b, col0 * g.ldb + k, g.C * g.ldb);
#pragma unroll
            for (int i = T::DUAL ? 2 * q : 0; i < (T::DUAL ? 2 * q + 2 : 4); ++i) {
                uint32_t o = off_b[i];
                if (!T::B_T && tail && (uint32_t)piece_k >= left) o = kNoSuchOffset;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (FASTGL_LDS void *)(to + T::A_BYTES + i * NW * 1024), 16, (int)o, 0, 0, 0);
            }
        }
    };

    // Where a lane reads its fragments: row (or column) l32 of a block of 32, contracted elements 8 h .. 8 h + 7 of 16.
    // [row][64]: piece 2 kk + h.  [64][column]: two transposing reads of four contracted rows each; of sixteen lanes four read one
    // row, and lane i gets column i of the four rows.
    const int i16 = lane & 15, g2 = (lane >> 4) & 1;
    uint32_t read_k[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) read_k[kk] = (uint32_t)(l32 * 128 + (((2 * kk + h) ^ twisted(l32)) << 4));
    auto read_t = [&](auto row_bytes, int block) {                      // block: of 32 columns
        constexpr int RB = decltype(row_bytes)::value;
        const int k = 8 * h + (i16 >> 2), piece = (4 * block + 2 * g2 + ((i16 & 3) >> 1)) ^ turned<RB>(k);
        return (uint32_t)(k * RB + piece * 16 + (i16 & 1) * 8);
    };
    typedef std::integral_constant<int, T::BM * 2> RowA;
    typedef std::integral_constant<int, T::BC * 2> RowB;
    constexpr int HALF_N = T::DUAL ? T::TN / 2 : T::TN;                   // column blocks of one result
    uint32_t at_a[T::TM], at_b[HALF_N];
#pragma unroll
    for (int i = 0; i < T::TM; ++i) at_a[i] = T::A_T ? read_t(RowA(), wm * T::TM + i) : 0;
#pragma unroll
    for (int j = 0; j < HALF_N; ++j) at_b[j] = T::B_T ? read_t(RowB(), wn * HALF_N + j) : 0;

    auto frag_k = [&](uint32_t base) { return *(FASTGL_LDS bf16x8 *)((FASTGL_LDS char *)lds + base); };
    auto frag_t = [&](uint32_t base, int row_bytes) {
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FASTGL_LDS i16x4 *)((FASTGL_LDS char *)lds + base));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FASTGL_LDS i16x4 *)((FASTGL_LDS char *)lds + base + 4 * row_bytes));
        struct { i16x4 l, h; } both = {lo, hi};
        return __builtin_bit_cast(bf16x8, both);
    };

    f32x16 acc[T::TM][T::TN];
#pragma unroll
    for (int i = 0; i < T::TM; ++i)
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    struct Frags { bf16x8 a[T::TM], b[T::TN]; };
    auto read = [&](int buf, int kk) {
        Frags f;
        const uint32_t base = (uint32_t)(buf * T::STAGE);
#pragma unroll
        for (int i = 0; i < T::TM; ++i) {
            if constexpr (T::A_T) f.a[i] = frag_t(base + at_a[i] + (uint32_t)(kk * 16 * RowA::value), RowA::value);
            else f.a[i] = frag_k(base + read_k[kk] + (uint32_t)((wm * T::TM + i) * 32 * 128));
        }
#pragma unroll
        for (int j = 0; j < T::TN; ++j) {
            if constexpr (T::B_T) {
                const int q = T::DUAL && j >= HALF_N ? 1 : 0;
                f.b[j] = frag_t(base + T::A_BYTES + q * (T::B_BYTES / 2) + at_b[j - q * HALF_N] + (uint32_t)(kk * 16 * RowB::value), RowB::value);
            } else
                f.b[j] = frag_k(base + T::A_BYTES + read_k[kk] + (uint32_t)((wn * T::TN + j) * 32 * 128));
        }
        return f;
    };
    // the columns first: a lane then holds four consecutive columns of one row
    auto multiply = [&](const Frags &f) {
#pragma unroll
        for (int j = 0; j < T::TN; ++j)
#pragma unroll
            for (int i = 0; i < T::TM; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.b[j], f.a[i], acc[i][j], 0, 0, 0);
    };

    const int all = steps * nseg;
    int seg = 0, t = 0;
    if (all > 0) load_step(0, 0, 0);
    for (int s = 0; s < all; ++s) {
        const int buf = s & 1;
        __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt 0: this wavefront's loads of the step are in LDS
        __builtin_amdgcn_s_barrier();                // everybody's are, and the other buffer has been read
        __builtin_amdgcn_sched_barrier(0);
        if (++t == steps) {
            t = 0;
            ++seg;
        }
        if (s + 1 < all) load_step(seg, t, buf ^ 1);
        Frags f = read(buf, 0);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            Frags n;
            if (kk < 3) n = read(buf, kk + 1);
            multiply(f);
            f = n;
        }
    }

    // ------------------------------------------------------------------ epilogue
    __builtin_amdgcn_s_waitcnt(0xC07F);              // lgkmcnt 0
    __builtin_amdgcn_s_barrier();                    // the LDS buffers are free: each wavefront has a part for itself
    constexpr int OB = (int)sizeof(OUT), PART = 2 * T::STAGE / NW;         // 16 KB a wavefront
    constexpr int ROWB = 64 * OB;                                        // 64 columns of a row
    static_assert(64 * ROWB <= PART, "a block of 64 x 64 results fits a wavefront's part");
    FASTGL_LDS char *mine = (FASTGL_LDS char *)lds + wave * PART;
    const int64_t r_base = row0 + wm * 64;
    // Columns c .. c + 32 B - 1 (B = 1 or 2 blocks) of the wavefront's 64 rows, element by element from `value(i, block, e)`.
    auto store_block = [&](auto blocks, void *out, int64_t ld, int64_t c_base, auto value) {
        constexpr int NB = decltype(blocks)::value, LPR = NB * 32 * OB / 16;        // lanes a row: 16 bytes each
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
                        o[0] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[0]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[1]) << 16;
                        o[1] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[3]) << 16;
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
#pragma unroll
        for (int n = 0; n < 64 * LPR / kWave; ++n) {
            const int row = (n * kWave + lane) / LPR, c = lane % LPR;
            const u32x4 o = *(FASTGL_LDS u32x4 *)(mine + row * ROWB + ((c ^ (row & 7)) * 16));
            const int64_t r = r_base + row, col = c_base + c * (16 / OB);
            if (r < g.R && col < g.C) {
                OUT *p = static_cast<OUT *>(out) + r * ld + col;
                if (col + 16 / OB <= g.C) {
                    *reinterpret_cast<W4 *>(p) = W4{o[0], o[1], o[2], o[3]};
                } else {
#pragma unroll
                    for (int e = 0; e < 16 / OB - 1; ++e)
                        if (col + e < g.C) {
                            const uint32_t word = o[e * OB / 4];             // a copy: a bit cast of o[e] itself takes o[0]
                            if constexpr (OB == 2) p[e] = (uint16_t)(word >> (16 * (e & 1)));
                            else p[e] = __uint_as_float(word);
                        }
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    if constexpr (MODE == kForward) {
        const int64_t c_base = col0 + wn * HALF_N * 32;
        typedef std::integral_constant<int, HALF_N> NB;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (!g.bias[q]) continue;
            const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(g.bias[q]), 0, (int)(g.C * 4), kTileRsrc);
#pragma unroll
            for (int b = 0; b < HALF_N; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)(4 * (c_base + b * 32 + 8 * e + 4 * h)), 0, 0);
#pragma unroll
                    for (int i = 0; i < T::TM; ++i)
#pragma unroll
                        for (int x = 0; x < 4; ++x) acc[i][q * HALF_N + b][4 * e + x] += __uint_as_float(v[x]);
                }
        }
        if (g.out[1]) store_block(NB(), g.out[1], g.C, c_base, [&](int i, int b, int e) { return acc[i][b][e]; });
        if (g.out[2]) store_block(NB(), g.out[2], g.C, c_base, [&](int i, int b, int e) { return acc[i][HALF_N + b][e]; });
        store_block(NB(), g.out[0], g.C, c_base,
                    [&](int i, int b, int e) { return gate<ACT, false>(acc[i][b][e], nullptr) * acc[i][HALF_N + b][e]; });
    } else if constexpr (MODE == kRows) {
#pragma unroll
        for (int n = 0; n < T::TN / 2; ++n)
            store_block(std::integral_constant<int, 2>(), g.out[0], g.C, col0 + (wn * T::TN + 2 * n) * 32,
                        [&](int i, int b, int e) { return acc[i][2 * n + b][e]; });
    } else {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (!g.out[q]) continue;
            store_block(std::integral_constant<int, HALF_N>(), static_cast<OUT *>(g.out[q]) + (int64_t)slab * g.out_slab, g.C,
                        col0 + wn * HALF_N * 32, [&](int i, int b, int e) { return acc[i][q * HALF_N + b][e]; });
        }
    }
#endif
}

}  // namespace
}  // namespace fastgl
