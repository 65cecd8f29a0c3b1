// Shared by the kernels of icq_block_matmul.
#pragma once
#include "icq_matmul_plan.h"
#include "icq_types.h"

struct Product {
    const uint8_t *a, *b;
    int64_t lda, ldb;
    const float *sa, *sb;
    int64_t M, N, K;
    int kb;                    // blocks along K
    void *out;
    int64_t ldo;
    float *part;               // [splits][M][N] partial sums where splits > 1
    int splits, per;           // blocks along K per split
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 16 codes (words 2 q, 2 q + 1 of a lane's eight hold eight of them) as the bf16 values they stand for: exact for both formats.
template <int FORMAT>
__device__ __forceinline__ bf16x8 widen(const icq_i32x8 &v, int q) {
    bf16x8 r;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const uint32_t w = (uint32_t)v[2 * q + (h >> 1)];
        bf16x2 d;
        if constexpr (FORMAT == ICQ_E4M3) d = (h & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
        else d = (h & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, false);
        r[2 * h] = d.x; r[2 * h + 1] = d.y;
    }
    return r;
}

template <int TYPE>
__device__ __forceinline__ void store4(const Product &p, int64_t m, int64_t n, const icq_f32x4 &v) {
    typedef IcqElem<TYPE> E;
    typedef typename E::raw raw;
    raw *o = static_cast<raw *>(p.out) + m * p.ldo + n;
    if (n + 4 <= p.N) {                                // (the memory pipe takes 8 or 16 bytes to any address)
        if constexpr (TYPE == ICQ_F32) __builtin_memcpy(o, &v, 16);
        else {
            const uint2 w = make_uint2(E::pack2(v[0], v[1]), E::pack2(v[2], v[3]));
            __builtin_memcpy(o, &w, 8);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.N) o[i] = E::put(v[i]);
    }
}

__device__ __forceinline__ void store_part(const Product &p, int split, int64_t m, int64_t n, const icq_f32x4 &v) {
    float *o = p.part + ((int64_t)split * p.M + m) * p.N + n;
    if (p.N % 4 == 0 && n < p.N) *reinterpret_cast<icq_f32x4 *>(o) = v;
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.N) o[e] = v[e];
}

// Blocks of up to 512 threads of one launch, a multiple of 8: the threads of a launch are counted in 32 bits.
constexpr uint32_t ICQ_PRODUCT_BLOCKS = 1u << 22;

// The first n < 16 of 16 bytes, zeros after them.
__device__ __forceinline__ uint4 first_bytes(const uint4 &v, int n) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = n - 4 * i;
        w[i] = left >= 4 ? w[i] : left <= 0 ? 0u : w[i] & ((1u << (8 * left)) - 1u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The product in tiles, p.splits parts of the contraction (icq_matmul_tiles.hip).
int icq_launch_product_tiles(const Product &p, icq_tiles tiles, int a_format, int b_format, bool rows, bool pow2, int out_type, hipStream_t s);
// The product of few rows of a (icq_matmul_few.hip).
int icq_launch_product_few(const Product &p, int num_cu, int a_format, int b_format, bool rows, int out_type, hipStream_t s);
