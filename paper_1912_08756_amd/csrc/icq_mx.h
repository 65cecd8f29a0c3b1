// Shared by the kernels of microscaled 4-bit floating point.
#pragma once
#include "icq_matmul.h"
#include "icq_mx_plan.h"

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// A block's scale byte from the bits of its largest magnitude: 255 where that is no number.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax, bool fit) {
    constexpr uint32_t least = 27u << 23, six = 0x400000u;                     // 2^-100; the mantissa of 6
    if (amax >= 0x7f800000u) return 255u;
    amax = max(amax, least);
    return min((amax >> 23) - 2u + (fit && (amax & 0x7fffffu) > six ? 1u : 0u), 252u);
}

// The scale of a byte in 25 .. 252 (what the quantiser makes); of 255 some number.
__device__ __forceinline__ float mx_divisor(uint32_t byte) { return __uint_as_float(min(byte, 252u) << 23); }

// The scale of any byte.
__device__ __forceinline__ float mx_scale(uint32_t byte) { return byte == 255u ? __uint_as_float(0x7fc00000u) : byte == 0u ? __uint_as_float(0x400000u) : __uint_as_float(byte << 23); }

// Two neighbouring values as they were loaded (a word of halves, or two words) to codes, in byte SEL of `old`: nearest, ties to even, saturating.
template <int TYPE, int SEL>
__device__ __forceinline__ uint32_t mx_codes2(const uint32_t *w, float scale, uint32_t old) {
    if constexpr (TYPE == ICQ_F32) return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, __uint_as_float(w[0]), __uint_as_float(w[1]), scale, SEL);
    else if constexpr (TYPE == ICQ_F16) return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(f16x2, w[0]), scale, SEL);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, w[0]), scale, SEL);
}

// Eight neighbouring values to eight codes.
template <int TYPE>
__device__ __forceinline__ uint32_t mx_codes8(const uint32_t *w, float scale) {
    constexpr int PER = TYPE == ICQ_F32 ? 2 : 1;                               // words of two values
    uint32_t c = mx_codes2<TYPE, 0>(w, scale, 0u);
    c = mx_codes2<TYPE, 1>(w + PER, scale, c);
    c = mx_codes2<TYPE, 2>(w + 2 * PER, scale, c);
    return mx_codes2<TYPE, 3>(w + 3 * PER, scale, c);
}

// A product of held matrices: sizes, result and parts as of the 8-bit products (a step along K: p.kb, p.per), and where codes and scales lie.
struct MxProduct {
    Product p;                 // a, b: codes; lda, ldb: bytes; sa, sb: not used
    const uint8_t *ea, *eb;    // scales
    int64_t ld_ea, ld_eb;
    int blocks;                // of 32 along K
};

// The first n < 32 of 32 codes, zeros after them.
__device__ __forceinline__ uint4 first_codes(const uint4 &v, int n) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = n - 8 * i;
        w[i] = left >= 8 ? w[i] : left <= 0 ? 0u : w[i] & ((1u << (4 * left)) - 1u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct MxQuantize {
    const void *x;
    int64_t rows, cols, ldx;
    uint8_t *codes, *codes_t, *scales, *scales_t;
    int64_t ld, ld_t, ld_s, ld_st;
    int across, down;          // groups of 128 along a row, along a column
    int fit;
};

// Rows of blocks of 32 (icq_mx.hip): what icq_mx_quantize does for `codes` alone with block_rows = 1.
int icq_launch_mx_rows(const MxQuantize &a, int x_type, hipStream_t s);
// The product in tiles, p.splits parts of the contraction; a step along K is 256 values (icq_mx_tiles.hip).
int icq_launch_mx_tiles(const MxProduct &q, icq_tiles tiles, int num_cu, int out_type, hipStream_t s);
// The product of few rows of a, held (a_type ICQ_E2M1) or as values x (icq_mx_few.hip).
int icq_launch_mx_few(const MxProduct &q, const icq_mx_plan &plan, int num_cu, const void *x, int a_type, int64_t ldx, bool fit, int out_type, hipStream_t s);
