// Rows of 16- or 32-bit elements, eight at a time, and the bits that dropout decides by (gfx950).
#pragma once
#include "common.h"

namespace {

typedef _Float16 f16_t;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(4 * sizeof(_Float16)))) _Float16 f16x4;
typedef __attribute__((__vector_size__(8 * sizeof(float)))) float f32x8;

template <class T>
struct Vec8;
template <>
struct Vec8<float> {
    typedef f32x8 type;
};
template <>
struct Vec8<bf16_t> {
    typedef bf16x8 type;
};
template <>
struct Vec8<f16_t> {
    typedef f16x8 type;
};

// Eight elements of a row, as they lie in memory.  Rows start wherever their stride puts them: the accesses ask for the alignment of one element,
// and the hardware takes 16 bytes from any address.
template <class T>
struct Raw8 {
    typename Vec8<T>::type v;
    // the first n of the eight; the others are 0
    __device__ inline void load(const T *p, int n)
    {
        if (n >= 8) {
            __builtin_memcpy(&v, p, sizeof(v));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : (T)0.f;
        }
    }
    __device__ inline f32x8 wide() const { return __builtin_convertvector(v, f32x8); }
    __device__ inline void round(const f32x8 &f) { v = __builtin_convertvector(f, typename Vec8<T>::type); }  // to nearest, ties to even
    __device__ inline void store(T *p, int n, bool streaming = false) const
    {
        if (n >= 8 && streaming) {
            typedef typename Vec8<T>::type V;
            typedef V Anywhere __attribute__((aligned(sizeof(T))));
            __builtin_nontemporal_store(v, reinterpret_cast<Anywhere *>(p));
        } else if (n >= 8) {
            __builtin_memcpy(p, &v, sizeof(v));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) p[i] = v[i];
        }
    }
};

// Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011): 128 bits that are a function of
// a 128-bit counter and a 64-bit key.
__device__ inline u32x4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

// Dropout of a matrix: element (row, col) has the 16 bits number col & 7 of the counter (col / 8, row, offset) under the key `seed`, low halves of
// the words first, and is dropped where they are below `below`.  16 bits: one counter serves the eight elements of an access, and the rate is met to
// 2^-17; the factor is that of the rate that is met.
struct Drop {
    uint32_t k0, k1, o0, o1;
    uint32_t below;  // 0: nothing is dropped, 65536: everything
    float factor;
};

__device__ inline f32x8 dropped(f32x8 v, const Drop &d, int chunk, int64_t row)
{
    const u32x4 w = philox((uint32_t)chunk, (uint32_t)row, d.o0, d.o1, d.k0, d.k1);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
        v[i] = u < d.below ? 0.f : v[i] * d.factor;  // a choice, not a product: infinities and NaN that are dropped are gone
    }
    return v;
}

}  // namespace
