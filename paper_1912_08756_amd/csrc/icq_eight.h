// Eight neighbouring values of a row, and comparisons of their magnitudes' bits, for the quantisers.
#pragma once
#include "icq_types.h"

// Eight values of one row as they were loaded, and the bits of their magnitudes: pairs of halves, or words.
template <int TYPE>
struct Eight {
    static constexpr int WORDS = TYPE == ICQ_F32 ? 8 : 4;
    uint32_t w[WORDS];
};

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t icq_u32x4 __attribute__((ext_vector_type(4), aligned(2)));             // 16 bytes at any value's address

// The larger magnitudes, pair by pair or word by word.
template <int TYPE>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    if constexpr (TYPE == ICQ_F32) return max(a, b);
    else return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

template <int TYPE>
__device__ __forceinline__ uint32_t magnitude(uint32_t w) { return w & (TYPE == ICQ_F32 ? 0x7fffffffu : 0x7fff7fffu); }

// A magnitude's bits as those of a float.
template <int TYPE>
__device__ __forceinline__ uint32_t float_bits(uint32_t half) {
    if constexpr (TYPE == ICQ_F32) return half;
    else if constexpr (TYPE == ICQ_F16) return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)half));
    else return half << 16;
}

// Values c .. c + 7 of row r, zeros where there are none.  ONCE: nobody reads them again soon, let them not put out what is.
template <int TYPE, bool ONCE = false>
__device__ __forceinline__ Eight<TYPE> read8(const void *x, int64_t rows, int64_t cols, int64_t ldx, int64_t r, int64_t c) {
    typedef typename IcqElem<TYPE>::raw raw;
    Eight<TYPE> v;
#pragma unroll
    for (int i = 0; i < Eight<TYPE>::WORDS; ++i) v.w[i] = 0;
    if (r >= rows) return v;
    const raw *p = static_cast<const raw *>(x) + r * ldx + c;
    if (c + 8 <= cols) {
        if constexpr (ONCE) {
#pragma unroll
            for (int k = 0; k < Eight<TYPE>::WORDS / 4; ++k) {
                const icq_u32x4 q = __builtin_nontemporal_load(reinterpret_cast<const icq_u32x4 *>(p) + k);
                __builtin_memcpy(v.w + 4 * k, &q, 16);
            }
        } else {
            __builtin_memcpy(v.w, p, sizeof v.w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) {
                if constexpr (TYPE == ICQ_F32) v.w[i] = __float_as_uint(p[i]);
                else v.w[i >> 1] |= (uint32_t)__builtin_bit_cast(uint16_t, p[i]) << (16 * (i & 1));
            }
    }
    return v;
}

template <int TYPE>
__device__ __forceinline__ void values8(const Eight<TYPE> &v, float *x) {
#pragma unroll
    for (int h = 0; h < Eight<TYPE>::WORDS / 4; ++h) IcqElem<TYPE>::unpack(make_uint4(v.w[4 * h], v.w[4 * h + 1], v.w[4 * h + 2], v.w[4 * h + 3]), x + 4 * h);
}
