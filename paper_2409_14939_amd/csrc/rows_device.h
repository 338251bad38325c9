// Device helpers of the row-wise kernels (norm, dropout): eight columns at a time, and the counter-based
// generator that says which of them a dropout keeps.
#pragma once
#include "internal.h"

namespace fastgl {

constexpr int kChunk = 8;              // columns a lane holds at a time: one answer of the generator, 16 bytes of bf16

// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011).
// Key: the seed; counter: (block of eight columns, row, offset).  The mask is a function of these alone, so it is
// computed again wherever it is needed and never stored, and does not depend on the launch or on the rows beside it.
struct Philox {
    uint32_t k0, k1, n2, n3;
    __device__ __forceinline__ void load(const int64_t *state)      // the same address for every lane: scalar loads
    {
        const uint64_t seed = (uint64_t)state[0], offset = (uint64_t)state[1];
        k0 = (uint32_t)seed;
        k1 = (uint32_t)(seed >> 32);
        n2 = (uint32_t)offset;
        n3 = (uint32_t)(offset >> 32);
    }
    __device__ __forceinline__ void words(uint32_t block, uint32_t row, uint32_t (&w)[4]) const
    {
        uint32_t x0 = block, x1 = row, x2 = n2, x3 = n3, a = k0, b = k1;
#pragma unroll
        for (int r = 0; r < 10; ++r) {
            const uint64_t p = (uint64_t)x0 * 0xD2511F53u, q = (uint64_t)x2 * 0xCD9E8D57u;
            x0 = (uint32_t)(q >> 32) ^ x1 ^ a;
            x1 = (uint32_t)q;
            x2 = (uint32_t)(p >> 32) ^ x3 ^ b;
            x3 = (uint32_t)p;
            a += 0x9E3779B9u;
            b += 0xBB67AE85u;
        }
        w[0] = x0;
        w[1] = x1;
        w[2] = x2;
        w[3] = x3;
    }
};

// Sixteen bits decide an element: kept where its half word is >= threshold = round(65536 p).  The probability is p to
// 2^-17, and the scale 65536 / (65536 - threshold) is the reciprocal of the probability that is realised, so the
// expectation is exact; 32 bits would cost twice the integer products, which is what bounds the generator.
// What is dropped is 0 whatever it was (NaN and infinity too): a selection, not a product.
__device__ __forceinline__ void drop8(float (&v)[8], const uint32_t (&w)[4], uint32_t threshold, float scale)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t h = j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu;
        v[j] = h >= threshold ? v[j] * scale : 0.f;
    }
}

// Two fp32 as bf16, to the nearest, even, in one instruction.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// Eight columns as they lie in memory, at any alignment to an element; columns from `left` on (left < 8 in a row's last
// chunk) are neither read nor written, and read as 0.  A last chunk of bf16 moves in a word of four columns, one of two and
// one of one, as many as it has; of fp32 in a word of four and column by column.  Column by column throughout, 1.15 M bf16 rows
// of 100 take 149 us for the plain norm, this way 98 (dropout 137 / 103).
template <bool BF16>
struct Chunk;

template <>
struct Chunk<true> {
    typedef uint16_t elem;
    uint32_t w[4];
    __device__ __forceinline__ void load(const uint16_t *p, int left)
    {
        if (left >= 8) {
            const Words<2>::x4 q = *reinterpret_cast<const Words<2>::x4 *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = q[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = 0;
            if (left <= 0) return;
            if (left & 4) {
                const Words<2>::x2 q = *reinterpret_cast<const Words<2>::x2 *>(p);
                w[0] = q[0];
                w[1] = q[1];
            }
            uint32_t tail = 0;
            if (left & 2) tail = *reinterpret_cast<const Words<2>::x1 *>(p + (left & 4));
            uint32_t one = 0;
            if (left & 1) one = p[left & 6];
            const uint32_t lo = left & 2 ? tail : one, hi = left & 2 ? one : 0u;
            if (left & 4) {
                w[2] = lo;
                w[3] = hi;
            } else {
                w[0] = lo;
                w[1] = hi;
            }
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ static __forceinline__ void store(uint16_t *p, const float (&v)[8], int left)
    {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        if (left >= 8) {
            *reinterpret_cast<Words<2>::x4 *>(p) = Words<2>::x4{o[0], o[1], o[2], o[3]};
        } else if (left > 0) {
            if (left & 4) *reinterpret_cast<Words<2>::x2 *>(p) = Words<2>::x2{o[0], o[1]};
            const uint32_t lo = left & 4 ? o[2] : o[0], hi = left & 4 ? o[3] : o[1];
            if (left & 2) *reinterpret_cast<Words<2>::x1 *>(p + (left & 4)) = lo;
            if (left & 1) p[left & 6] = (uint16_t)(left & 2 ? hi : lo);
        }
    }
};

template <>
struct Chunk<false> {
    typedef float elem;
    float w[8];
    __device__ __forceinline__ void four(const float *p, int i)
    {
        const Words<4>::x4 a = *reinterpret_cast<const Words<4>::x4 *>(p + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[i + j] = __uint_as_float(a[j]);
    }
    __device__ __forceinline__ void load(const float *p, int left)
    {
        if (left >= 8) {
            four(p, 0);
            four(p, 4);
        } else if (left >= 4) {
            four(p, 0);
#pragma unroll
            for (int j = 4; j < 8; ++j) w[j] = j < left ? p[j] : 0.f;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = j < 3 && j < left ? p[j] : 0.f;
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = w[j];
    }
    __device__ static __forceinline__ void store(float *p, const float (&v)[8], int left)
    {
        auto four = [&](int i) {
            *reinterpret_cast<Words<4>::x4 *>(p + i) =
                Words<4>::x4{__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])};
        };
        if (left >= 8) {
            four(0);
            four(4);
        } else if (left >= 4) {
            four(0);
#pragma unroll
            for (int j = 4; j < 7; ++j)
                if (j < left) p[j] = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (j < left) p[j] = v[j];
        }
    }
};

// A chunk of a row, at element `at` of an array: where the array goes on for eight elements at least (`inside`, the same for a
// whole wavefront), a row's last chunk is read beyond the row, as one word, and masked where it is used (not here: nothing should
// wait for the load yet); by load() only at the array's end.
// us a call, by load() throughout / so: gradient of the plain norm of 115 000 bf16 rows of 602 116 / 94.
template <class C, class T>
__device__ __forceinline__ void load_row(C &c, const T *p, int64_t at, int left, bool inside)
{
    if (__builtin_expect(inside, 1)) {
        c = C{};                                       // columns that do not exist: 0
        if (left > 0) c.load(p + at, kChunk);
    } else
        c.load(p + at, left);
}

// The number of a wavefront's first thread, over 2^lg.
__device__ __forceinline__ int wave_first(int lg) { return __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> lg; }

// Host side of a dropout probability: false where it is not in [0, 1].
inline bool drop_constants(double p, uint32_t *threshold, float *scale)
{
    if (!(p >= 0.0 && p <= 1.0)) return false;
    const double t = __builtin_nearbyint(65536.0 * p);
    *threshold = (uint32_t)t;
    *scale = t < 65536.0 ? (float)(65536.0 / (65536.0 - t)) : 0.f;
    return true;
}

}  // namespace fastgl
