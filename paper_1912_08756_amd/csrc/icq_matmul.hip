// Products of matrices held in 8-bit floating point with one scale per block of 128 along the contraction:
//     out[m][n] = sum_kb sa[m][kb] * sb[.][kb] * sum_{k in block kb} a[m][k] * b[n][k],
// sb per row n (b in blocks of 1 x 128) or per 128 rows (128 x 128).
//
// One scale block is the contraction of one 16x16x128 or two 32x32x64 matrix instructions, so their result, summed from zero, takes the
// product of the two scales as it is added to the accumulator: one multiply-add per element and block on the vector pipe,
// beside 128 on the matrix pipe; scales of powers of two go into the instructions themselves.  Which of a block's 128 positions
// meets which lane is free as long as both operands agree, so a lane takes whatever 32 bytes are convenient.  b's rows are the
// instruction's rows: a lane then ends up with four consecutive n of one m, one scale of a, and stores of 8 or 16 bytes.
//
// The 8-bit matrix instructions add each eight neighbouring products to about 13 bits below the largest of them (1.4e-5 of the result
// in the 2-norm for normal values, against 1.7e-3 and 2e-4 of rounding to bf16 and f16), so a result that stays in 32 bits takes
// the 16-bit ones, which hold 32, over codes widened to bf16 (exact for both formats).
#include "icq_matmul.h"

#include <algorithm>

namespace {

// The splits' partial sums added in order; four columns a thread.
template <int TYPE>
__global__ __launch_bounds__(256) void product_join_kernel(Product p) {
    const int64_t m = blockIdx.y + (int64_t)blockIdx.z * 32768, n = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (m >= p.M || n >= p.N) return;
    const int64_t total = p.M * p.N;
    const float *from = p.part + m * p.N + n;
    icq_f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (n + 4 <= p.N) {
        for (int k = 0; k < p.splits; ++k) {
            icq_f32x4 v;
            __builtin_memcpy(&v, from + k * total, 16);
            s += v;
        }
    } else {
        for (int k = 0; k < p.splits; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < p.N) s[e] += from[k * total + e];
    }
    store4<TYPE>(p, m, n, s);
}

}  // namespace

bool icq_product_extents_ok(int64_t M, int64_t N, int64_t K) {
    return M >= 0 && N >= 0 && K >= 0 && M <= ICQ_MAX_EXTENT && N <= ICQ_MAX_EXTENT && K <= ICQ_MAX_EXTENT &&
           ((M + 63) / 64) * ((N + 63) / 64) <= 0x7fffffff;
}

int icq_launch_product_join(const Product &p, int out_type, hipStream_t s) {
    const auto go = [&](const Product &q) {
        const dim3 by_four((uint32_t)((q.N + 1023) / 1024), (uint32_t)(q.M < 32768 ? q.M : 32768), (uint32_t)((q.M + 32767) / 32768));
        ICQ_FOR_TYPE(out_type, hipLaunchKernelGGL(HIP_KERNEL_NAME(product_join_kernel<TYPE>), by_four, dim3(256), 0, s, q))
    };
    if (p.splits > 0) go(p);                                                  // (few tiles, then: far from a launch's 2^32 threads)
    else {
        const int64_t step = std::max<int64_t>(1, ICQ_PRODUCT_BLOCKS / ((p.N + 1023) / 1024));
        for (int64_t m = 0; m < p.M; m += step) {
            Product q = p;
            q.M = std::min(step, p.M - m);
            q.out = static_cast<char *>(p.out) + m * p.ldo * icq_type_bytes(out_type);
            go(q);
        }
    }
    return icq_check_launch();
}

ICQ_EXPORT int icq_block_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, size_t *out) {
    if (!out || !icq_product_extents_ok(M, N, K)) return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    const int fast = icq_plan_product(M, N, K, false, cu).splits, exact = icq_plan_product(M, N, K, true, cu).splits, splits = fast > exact ? fast : exact;
    *out = splits > 1 ? icq_align_up((size_t)splits * M * N * sizeof(float), ICQ_ALIGN) : 0;
    return ICQ_OK;
}

ICQ_EXPORT int icq_block_matmul(const uint8_t *a, int a_format, int64_t lda, const float *a_scales, const uint8_t *b, int b_format,
                                int64_t ldb, const float *b_scales, int b_block_rows, int scaling, int64_t M, int64_t N, int64_t K,
                                void *out, int out_type, int64_t ldo, void *workspace, size_t workspace_bytes, void *stream) {
    const int size = icq_type_bytes(out_type);
    if (size == 0 || (a_format != ICQ_E4M3 && a_format != ICQ_E5M2) || (b_format != ICQ_E4M3 && b_format != ICQ_E5M2) ||
        (scaling != ICQ_SCALES_F32 && scaling != ICQ_SCALES_POW2) || (b_block_rows != 1 && b_block_rows != ICQ_BLOCK) || !icq_product_extents_ok(M, N, K))
        return ICQ_ERR_ARG;
    if (M == 0 || N == 0) return ICQ_OK;
    if (!out || (uintptr_t)out % size != 0 || ldo < N) return ICQ_ERR_ARG;
    if (K > 0 && (!a || !b || !a_scales || !b_scales || lda < K || ldb < K || lda > ICQ_MAX_CODE_LD || ldb > ICQ_MAX_CODE_LD || lda % 16 != 0 || ldb % 16 != 0 || (uintptr_t)a % 16 != 0 ||
                  (uintptr_t)b % 16 != 0))
        return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    Product p;
    p.a = a; p.b = b; p.lda = lda; p.ldb = ldb; p.sa = a_scales; p.sb = b_scales;
    p.M = M; p.N = N; p.K = K;
    p.kb = (int)((K + 127) / 128);
    p.out = out; p.ldo = ldo;
    const icq_product_plan plan = icq_plan_product(M, N, K, out_type == ICQ_F32, cu);
    p.splits = plan.splits;
    p.per = (p.kb + p.splits - 1) / p.splits;
    p.part = static_cast<float *>(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (K == 0) {
        p.splits = 0;                                                         // (a sum of nothing)
        return icq_launch_product_join(p, out_type, s);
    }
    if (p.splits > 1 && (!workspace || (uintptr_t)workspace % ICQ_ALIGN != 0 || workspace_bytes < (size_t)p.splits * M * N * sizeof(float)))
        return ICQ_ERR_WORKSPACE;
    const bool rows = b_block_rows == 1;
    const int rc = plan.few ? icq_launch_product_few(p, cu, a_format, b_format, rows, out_type, s)
                            : icq_launch_product_tiles(p, plan.tiles, a_format, b_format, rows, scaling == ICQ_SCALES_POW2, out_type, s);
    if (rc != ICQ_OK || p.splits == 1) return rc;
    return icq_launch_product_join(p, out_type, s);
}
