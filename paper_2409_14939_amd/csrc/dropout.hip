// Dropout from the counter-based generator, with an optional addition (fastgl_norm.h has the formula), and the row
// gather of tables held in 8 bits.  Both are one pass over memory.
//
// Dropout is bound by memory: 1.15 M fp32 rows of 100 take 175 us, 5.3 TB/s (a copy runs at 4.7 to 5.0 here).  An answer of the
// generator serves eight elements: its twenty 32-bit products take about as long as the moves of eight bf16, and fit beside them.
// A workgroup has consecutive chunks whatever the rows' length, four a lane under way at once.
//
// The gather is bound by its random rows: 390 000 rows of 128 from a table of 2.6 GB take 37 us, 4.1 TB/s of what has to move (each row's scale,
// 4 bytes, costs a sector of its own); 44 in calls that take three tables in turn.
#include "fastgl_norm.h"
#include "rows_device.h"

#include <type_traits>

namespace fastgl {
namespace {

constexpr int kUnits = 4;           // chunks of eight columns a lane of the dropout takes
constexpr int kMany = 4;            // rows that a lane of the gather has under way where the result has kManyBytes at least
constexpr int64_t kManyBytes = (int64_t)64 << 20;
constexpr int kWide = 2048;         // chunks a row from which a workgroup's units touch at most two rows

struct DropArgs {
    const void *X, *R;
    void *Y;
    int64_t M;
    int32_t F, chunks;
    uint32_t inv;                   // ceil(2^32 / chunks), for rows of fewer than kWide chunks
    const int64_t *rng;
    uint32_t threshold;
    float scale;
};

// Unit u = (row, chunk) in row-major order; a workgroup has kBlock * kUnits consecutive ones.
template <bool BF16, bool DROP>
__global__ __launch_bounds__(kBlock) void k_dropout(DropArgs a)
{
    typedef typename Chunk<BF16>::elem T;
    Philox gen;
    if constexpr (DROP) gen.load(a.rng);
    const uint64_t first = (uint64_t)blockIdx.x * (kBlock * kUnits);
    const int64_t row0 = (int64_t)(first / (uint32_t)a.chunks);
    const uint32_t c0 = (uint32_t)(first - (uint64_t)row0 * (uint32_t)a.chunks);
    const bool inside = first + kBlock * kUnits + kChunk <= (uint64_t)a.M * (uint32_t)a.chunks;      // units follow, of an element at least
    Chunk<BF16> x[kUnits], r[kUnits];
    int64_t at[kUnits];
    uint32_t rows[kUnits], cs[kUnits];
    int left[kUnits];
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        // c0 + the unit's place: below chunks + kBlock * kUnits, so below kWide chunks the product with `inv` is exact
        // (both factors below 2^12) and beyond them the quotient is 0 or 1; one chunk a row divides by itself
        const uint32_t u = c0 + (uint32_t)(i * kBlock) + threadIdx.x;
        const uint32_t q = a.chunks == 1 ? u : a.chunks < kWide ? __umulhi(u, a.inv) : (u >= (uint32_t)a.chunks ? 1u : 0u);
        const int64_t row = row0 + q;
        rows[i] = (uint32_t)row;
        cs[i] = u - q * (uint32_t)a.chunks;
        const int col = (int)cs[i] * kChunk;
        at[i] = row * a.F + col;
        left[i] = row < a.M ? a.F - col : 0;
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) load_row(x[i], static_cast<const T *>(a.X), at[i], left[i], inside);
    if (a.R) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) load_row(r[i], static_cast<const T *>(a.R), at[i], left[i], inside);
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        float v[8];
        uint32_t words[4];
        if constexpr (DROP) gen.words(cs[i], rows[i], words);
        x[i].get(v);
        if constexpr (DROP) drop8(v, words, a.threshold, a.scale);
        if (a.R) {
            float y[8];
            r[i].get(y);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += y[j];
        }
        Chunk<BF16>::store(static_cast<T *>(a.Y) + at[i], v, left[i]);
    }
}

// ------------------------------------------------------------------------------------ 8-bit rows
struct Gather8Args {
    const uint8_t *table;
    const float *scale;
    int64_t table_rows;
    const int64_t *ids;
    int64_t n;
    int32_t F;
    int32_t slices;                 // of 16 bytes a row of the result
    int32_t lg;                     // 2^lg lanes a row
    void *out;
};

// A lane writes 16 bytes of a row: V columns, of MANY rows whose IDs, scales and columns are under way together.  In rows of V
// and more the last slice starts V before the row's end, and what two slices share is written twice alike; shorter rows go
// column by column.
template <bool BF16, bool SHORT, int MANY>
__global__ __launch_bounds__(kBlock) void k_gather_e4m3(Gather8Args a)
{
    typedef uint32_t bytes4 __attribute__((aligned(1)));
    typedef typename Chunk<BF16>::elem T;
    constexpr int V = 16 / (int)sizeof(T);
    const int groups = kBlock >> a.lg, lanes = 1 << a.lg;
    const int64_t first = (int64_t)blockIdx.x * (groups * MANY) + (threadIdx.x >> a.lg);
    const uint8_t *q[MANY];
    float scale[MANY];
    bool there[MANY];
#pragma unroll
    for (int m = 0; m < MANY; ++m) {
        const int64_t row = first + m * groups;
        const int64_t id = row < a.n ? a.ids[row] : -1;
        there[m] = (uint64_t)id < (uint64_t)a.table_rows;
        q[m] = a.table + (there[m] ? id : 0) * a.F;
        scale[m] = there[m] ? a.scale[id] : __uint_as_float(0x7FC00000u);
    }
    if constexpr (SHORT) {
        for (int c = threadIdx.x & (lanes - 1); c < a.F; c += lanes)
#pragma unroll
            for (int m = 0; m < MANY; ++m) {
                const int64_t row = first + m * groups;
                if (row >= a.n) continue;
                const uint32_t b = there[m] ? q[m][c] : 0u;
                const float v = __builtin_amdgcn_cvt_f32_fp8((int)b, 0) * scale[m];
                T *out = static_cast<T *>(a.out) + row * a.F + c;
                if constexpr (BF16) *out = __builtin_bit_cast(uint16_t, (__bf16)v);
                else *out = v;
            }
    } else {
        for (int c = threadIdx.x & (lanes - 1); c < a.slices; c += lanes) {
            const int col = c * V < a.F - V ? c * V : a.F - V;
            uint32_t w[MANY][V / 4];
#pragma unroll
            for (int m = 0; m < MANY; ++m)
#pragma unroll
                for (int i = 0; i < V / 4; ++i) w[m][i] = there[m] ? *reinterpret_cast<const bytes4 *>(q[m] + col + 4 * i) : 0u;
#pragma unroll
            for (int m = 0; m < MANY; ++m) {
                const int64_t row = first + m * groups;
                if (row >= a.n) continue;
                T *out = static_cast<T *>(a.out) + row * a.F + col;
                float v[V];
#pragma unroll
                for (int i = 0; i < V / 4; ++i) {
                    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[m][i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[m][i], true);
                    v[4 * i] = lo[0] * scale[m];
                    v[4 * i + 1] = lo[1] * scale[m];
                    v[4 * i + 2] = hi[0] * scale[m];
                    v[4 * i + 3] = hi[1] * scale[m];
                }
                if constexpr (BF16) {
                    Chunk<true>::store(out, v, 8);
                } else
                    *reinterpret_cast<Words<4>::x4 *>(out) =
                        Words<4>::x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
            }
        }
    }
}

bool misaligned_to(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

}  // namespace
}  // namespace fastgl

using namespace fastgl;

extern "C" {

fastgl_status fastgl_dropout(fastgl_dtype dtype, const void *X, const void *R, int64_t M, int64_t F, const int64_t *rng,
                             double p, void *Y, void *stream)
{
    DropArgs a = {};
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
    if (!drop_constants(p, &a.threshold, &a.scale)) {
        set_error("the dropout probability must be in [0, 1]");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (p > 0.0 && (!rng || misaligned_to(rng, 8))) {
        set_error("dropout needs rng: two int64 {seed, offset} in device memory, aligned to 8 bytes");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (M == 0) return FASTGL_OK;
    const uintptr_t el = dtype == FASTGL_BF16 ? 2 : 4;
    if (!X || !Y) {
        set_error("X or Y is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (misaligned_to(X, el) || misaligned_to(R, el) || misaligned_to(Y, el)) {
        set_error("arrays must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    a.X = X; a.R = R; a.Y = Y;
    a.M = M; a.F = (int32_t)F;
    a.chunks = (int32_t)ceil_div(F, kChunk);
    a.inv = (uint32_t)ceil_div((int64_t)1 << 32, a.chunks > 1 ? a.chunks : 2);
    a.rng = rng;
    const int64_t blocks = ceil_div(M * a.chunks, kBlock * kUnits);
    if (blocks > 0x7FFFFFFFLL) {
        set_error("dropout too large for one launch");
        return FASTGL_ERR_UNSUPPORTED;
    }
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, (hipStream_t)stream, a); };
    if (dtype == FASTGL_BF16) p > 0.0 ? go(k_dropout<true, true>) : go(k_dropout<true, false>);
    else p > 0.0 ? go(k_dropout<false, true>) : go(k_dropout<false, false>);
    FASTGL_LAUNCH_CHECK("fastgl_dropout");
    return FASTGL_OK;
}

fastgl_status fastgl_gather_rows_e4m3(const uint8_t *table, const float *scale, int64_t table_rows, const int64_t *ids,
                                      int64_t n, int64_t F, fastgl_dtype dtype, void *out, void *stream)
{
    if (dtype != FASTGL_F32 && dtype != FASTGL_BF16) {
        set_error("bad dtype %d", (int)dtype);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (n < 0 || table_rows < 0 || F < 1) {
        set_error("negative size or no columns (n=%lld table_rows=%lld F=%lld)", (long long)n, (long long)table_rows, (long long)F);
        return FASTGL_ERR_INVALID_ARG;
    }
    if (n > kMaxIndex || F > (int64_t)1 << 24) {
        set_error("n must stay below 2^31-1-1024 and F at 2^24 or below");
        return FASTGL_ERR_UNSUPPORTED;
    }
    if (n == 0) return FASTGL_OK;
    if (!ids || !out || (table_rows > 0 && (!table || !scale))) {
        set_error("table, scale, ids or out is NULL");
        return FASTGL_ERR_INVALID_ARG;
    }
    if (misaligned_to(scale, 4) || misaligned_to(ids, 8) || misaligned_to(out, dtype == FASTGL_BF16 ? 2 : 4)) {
        set_error("arrays must be aligned to their element size");
        return FASTGL_ERR_INVALID_ARG;
    }
    Gather8Args a = {};
    a.table = table; a.scale = scale; a.table_rows = table_rows;
    a.ids = ids; a.n = n; a.F = (int32_t)F; a.out = out;
    const int64_t V = dtype == FASTGL_BF16 ? 8 : 4;
    a.slices = (int32_t)ceil_div(F, V);
    const int64_t units = F < V ? F : a.slices;
    while (a.lg < 6 && ((int64_t)1 << a.lg) < units) ++a.lg;
    // us a call, one row under way / four: 390 000 rows of 128 to bf16 42 / 37, to fp32 81 / 63; 30 000 of 2048 to fp32 79 / 64;
    // 80 000 of 128 to fp32 11.3 / 11.6; 100 000 of 16 to bf16 5.8 / 6.6
    const bool many = n * F * (dtype == FASTGL_BF16 ? 2 : 4) >= kManyBytes;
    const int64_t blocks = ceil_div(n, (int64_t)(kBlock >> a.lg) * (many ? kMany : 1));
    if (blocks > 0x7FFFFFFFLL) {
        set_error("gather too large for one launch");
        return FASTGL_ERR_UNSUPPORTED;
    }
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, (hipStream_t)stream, a); };
    auto typed = [&](auto bf16, auto many_rows) {
        constexpr bool B = decltype(bf16)::value;
        constexpr int N = decltype(many_rows)::value;
        F < V ? go(k_gather_e4m3<B, true, N>) : go(k_gather_e4m3<B, false, N>);
    };
    auto both = [&](auto bf16) { many ? typed(bf16, std::integral_constant<int, kMany>()) : typed(bf16, std::integral_constant<int, 1>()); };
    if (dtype == FASTGL_BF16) both(std::true_type());
    else both(std::false_type());
    FASTGL_LAUNCH_CHECK("fastgl_gather_rows_e4m3");
    return FASTGL_OK;
}

}  // extern "C"
