// Products of matrices held in 8-bit floating point with one scale per block of 128 along the contraction:
//     out[m][n] = sum_kb sa[m][kb] * sb[.][kb] * sum_{k in block kb} a[m][k] * b[n][k],
// sb per row n (b in blocks of 1 x 128) or per 128 rows (128 x 128).
//
// One 16x16x128 matrix instruction contracts exactly one scale block, so its result, summed from zero, takes
// the product of the two scales as it is added to the accumulator: one multiply-add per element and block on the vector
// pipe, beside 128 on the matrix pipe.  Which of a block's 128 positions meets which lane is free as long as both operands
// agree, so a lane takes whatever 32 bytes are convenient.  b's rows are the instruction's rows: a lane then ends up with four
// consecutive n of one m, a scalar scale of a, and stores of 8 or 16 bytes.
#include "icq_matmul.h"

namespace {

constexpr int BM = 128, BN = 128;

// The contraction of one scale block.  The 8-bit matrix instructions add each eight neighbouring products to about 13 bits below the
// largest of them (1.4e-5 of the result in the 2-norm for normal values, against 1.7e-3 and 2e-4 of rounding to bf16 and f16), so a
// result that stays in 32 bits takes the 16-bit ones, which hold 32: EXACT.
template <int FA, int FB, bool EXACT>
__device__ __forceinline__ icq_f32x4 dot128(const icq_i32x8 &n, const icq_i32x8 &m) {
    icq_f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
    // first operand: rows of b, second: rows of a; scales of one
    if constexpr (!EXACT) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(n, m, c, FB, FA, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
    else {
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FB>(n, q), widen<FA>(m, q), c, 0, 0, 0);
        return c;
    }
}

// A 128 x 128 tile of the result per block, 64 x 64 per wavefront.  ROWS: b has a scale per row.
template <int FA, int FB, bool ROWS, int TYPE>
__global__ __launch_bounds__(256) void product_tile_kernel(Product p) {
    __shared__ __attribute__((aligned(16))) uint8_t s_a[BM * 128], s_b[BN * 128];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t m0 = (int64_t)blockIdx.x * BM, n0 = (int64_t)blockIdx.y * BN;
    const int split = blockIdx.z, k0 = split * p.per, k1 = min(p.kb, k0 + p.per);
    const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64, at = lane & 15, quarter = lane >> 4;
    icq_f32x4 acc[4][4] = {};
    for (int kb = k0; kb < k1; ++kb) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = u * 256 + tid, r = i >> 3, c = i & 7;       // 16-byte piece c of row r sits at place c ^ (r & 7)
            const int64_t k = (int64_t)kb * 128 + c * 16;
            *reinterpret_cast<uint4 *>(&s_a[r * 128 + ((c ^ (r & 7)) << 4)]) = load16(p.a, p.lda, p.M, p.K, m0 + r, k);
            *reinterpret_cast<uint4 *>(&s_b[r * 128 + ((c ^ (r & 7)) << 4)]) = load16(p.b, p.ldb, p.N, p.K, n0 + r, k);
        }
        __syncthreads();
        icq_i32x8 fa[4], fb[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = h * 4 + quarter, ra = wm + t * 16 + at, rb = wn + t * 16 + at;
                const uint4 va = *reinterpret_cast<const uint4 *>(&s_a[ra * 128 + ((c ^ (ra & 7)) << 4)]);
                const uint4 vb = *reinterpret_cast<const uint4 *>(&s_b[rb * 128 + ((c ^ (rb & 7)) << 4)]);
                fa[t][4 * h] = (int)va.x; fa[t][4 * h + 1] = (int)va.y; fa[t][4 * h + 2] = (int)va.z; fa[t][4 * h + 3] = (int)va.w;
                fb[t][4 * h] = (int)vb.x; fb[t][4 * h + 1] = (int)vb.y; fb[t][4 * h + 2] = (int)vb.z; fb[t][4 * h + 3] = (int)vb.w;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t m = m0 + wm + i * 16 + at;
            const float sa = m < p.M ? p.sa[m * p.kb + kb] : 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const icq_f32x4 d = dot128<FA, FB, TYPE == ICQ_F32>(fb[j], fa[i]);
                const int64_t n = n0 + wn + j * 16 + quarter * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t row = ROWS ? n + e : (n0 + wn) >> 7;
                    const float sb = n + e < p.N ? p.sb[row * p.kb + kb] : 0.0f;
                    acc[i][j][e] = fmaf(d[e], sa * sb, acc[i][j][e]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + wm + i * 16 + at;
        if (m >= p.M) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + wn + j * 16 + quarter * 4;
            if (p.splits == 1) {
                store4<TYPE>(p, m, n, acc[i][j]);
            } else {
                float *o = p.part + ((int64_t)split * p.M + m) * p.N + n;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e < p.N) o[e] = acc[i][j][e];
            }
        }
    }
}

// The splits' partial sums added in order.
template <int TYPE>
__global__ __launch_bounds__(256) void product_join_kernel(Product p) {
    typedef IcqElem<TYPE> E;
    const int64_t total = p.M * p.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        float s = p.part[i];
        for (int k = 1; k < p.splits; ++k) s += p.part[k * total + i];
        static_cast<typename E::raw *>(p.out)[i / p.N * p.ldo + i % p.N] = E::put(s);
    }
}

template <int TYPE>
__global__ __launch_bounds__(256) void product_zero_kernel(Product p) {
    typedef IcqElem<TYPE> E;
    const int64_t total = p.M * p.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256)
        static_cast<typename E::raw *>(p.out)[i / p.N * p.ldo + i % p.N] = E::put(0.0f);
}

// Splits of the contraction: enough blocks for the chip, eight scale blocks at least in each.
int splits_of(int64_t M, int64_t N, int64_t K, int num_cu) {
    const int64_t tiles = ((M + BM - 1) / BM) * ((N + BN - 1) / BN), kb = (K + 127) / 128;
    const int64_t want = 2ll * num_cu / (tiles > 0 ? tiles : 1), most = kb / 8;
    const int64_t n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n);
}

template <int FA, int FB, bool ROWS, int TYPE>
void launch(const Product &p, hipStream_t s) {
    const dim3 grid((uint32_t)((p.M + BM - 1) / BM), (uint32_t)((p.N + BN - 1) / BN), (uint32_t)p.splits);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(product_tile_kernel<FA, FB, ROWS, TYPE>), grid, dim3(256), 0, s, p);
}

template <int TYPE, bool ROWS>
void launch_formats(const Product &p, int fa, int fb, hipStream_t s) {
    if (fa == ICQ_E4M3) {
        if (fb == ICQ_E4M3) launch<ICQ_E4M3, ICQ_E4M3, ROWS, TYPE>(p, s);
        else launch<ICQ_E4M3, ICQ_E5M2, ROWS, TYPE>(p, s);
    } else {
        if (fb == ICQ_E4M3) launch<ICQ_E5M2, ICQ_E4M3, ROWS, TYPE>(p, s);
        else launch<ICQ_E5M2, ICQ_E5M2, ROWS, TYPE>(p, s);
    }
}

bool extents_ok(int64_t M, int64_t N, int64_t K) {
    return M >= 0 && N >= 0 && K >= 0 && M <= ICQ_MAX_EXTENT && N <= ICQ_MAX_EXTENT && K <= ICQ_MAX_EXTENT &&
           (N + BN - 1) / BN <= 65535;
}

}  // namespace

ICQ_EXPORT int icq_block_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, size_t *out) {
    if (!out || !extents_ok(M, N, K)) return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    const int splits = splits_of(M, N, K, cu);
    *out = splits > 1 ? icq_align_up((size_t)splits * M * N * sizeof(float), ICQ_ALIGN) : 0;
    return ICQ_OK;
}

ICQ_EXPORT int icq_block_matmul(const uint8_t *a, int a_format, int64_t lda, const float *a_scales, const uint8_t *b, int b_format,
                                int64_t ldb, const float *b_scales, int b_block_rows, int scaling, int64_t M, int64_t N, int64_t K,
                                void *out, int out_type, int64_t ldo, void *workspace, size_t workspace_bytes, void *stream) {
    const int size = icq_type_bytes(out_type);
    if (size == 0 || (a_format != ICQ_E4M3 && a_format != ICQ_E5M2) || (b_format != ICQ_E4M3 && b_format != ICQ_E5M2) ||
        (scaling != ICQ_SCALES_F32 && scaling != ICQ_SCALES_POW2) || (b_block_rows != 1 && b_block_rows != ICQ_BLOCK) || !extents_ok(M, N, K))
        return ICQ_ERR_ARG;
    if (M == 0 || N == 0) return ICQ_OK;
    if (!out || (uintptr_t)out % size != 0 || ldo < N) return ICQ_ERR_ARG;
    if (K > 0 && (!a || !b || !a_scales || !b_scales || lda < K || ldb < K || lda % 16 != 0 || ldb % 16 != 0 || (uintptr_t)a % 16 != 0 ||
                  (uintptr_t)b % 16 != 0))
        return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    Product p;
    p.a = a; p.b = b; p.lda = lda; p.ldb = ldb; p.sa = a_scales; p.sb = b_scales;
    p.M = M; p.N = N; p.K = K;
    p.kb = (int)((K + 127) / 128);
    p.out = out; p.ldo = ldo;
    p.splits = splits_of(M, N, K, cu);
    p.per = (p.kb + p.splits - 1) / p.splits;
    p.part = static_cast<float *>(workspace);
    p.vec = (uintptr_t)out % (4 * size) == 0 && ldo % 4 == 0;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t total = M * N;
    const dim3 flat((uint32_t)(total / 256 + 1 < 65536 ? total / 256 + 1 : 65536));
    if (K == 0) {
        ICQ_FOR_TYPE(out_type, hipLaunchKernelGGL(HIP_KERNEL_NAME(product_zero_kernel<TYPE>), flat, dim3(256), 0, s, p))
        return icq_check_launch();
    }
    if (p.splits > 1 && (!workspace || (uintptr_t)workspace % ICQ_ALIGN != 0 || workspace_bytes < (size_t)p.splits * M * N * sizeof(float)))
        return ICQ_ERR_WORKSPACE;
    if (p.splits == 1 && icq_product_wide_usable(M, N, K, lda, ldb, cu))
        return icq_launch_product_wide(p, a_format, b_format, b_block_rows == 1, scaling == ICQ_SCALES_POW2, out_type, s);
    ICQ_FOR_TYPE(out_type,
        if (b_block_rows == 1) launch_formats<TYPE, true>(p, a_format, b_format, s);
        else launch_formats<TYPE, false>(p, a_format, b_format, s);
        if (p.splits > 1) hipLaunchKernelGGL(HIP_KERNEL_NAME(product_join_kernel<TYPE>), flat, dim3(256), 0, s, p))
    return icq_check_launch();
}
