// Products of 8-bit matrices with block scales for up to 32 rows of a: reading b is all that counts.
//
// A block of eight wavefronts has 16 NT rows of b; each wavefront takes every eighth scale block of them, straight from memory into
// the registers in the matrix instruction's layout, the next one requested before the present one is multiplied; a's rows come
// from the caches the same way.  The eight partial sums meet in the LDS, in a fixed order.  Bound by memory: 1 x 16384 x 4096
// 13.0 us, 5.2 TB/s of b, into f32 over widened codes the same (16 rows 14.4 and 14.7); where b is small, by the launch and one chain of loads (1 x 4096 x 4096: 8 us with the host's share).
#include "icq_matmul.h"

#include <algorithm>

namespace {

constexpr int WAVES = ICQ_PRODUCT_FEW_WAVES;

template <int FA, int FB, bool EXACT>
__device__ __forceinline__ icq_f32x4 dot128(const icq_i32x8 &n, const icq_i32x8 &m) {
    icq_f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (!EXACT) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(n, m, c, FB, FA, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
    else {
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FB>(n, q), widen<FA>(m, q), c, 0, 0, 0);
        return c;
    }
}

// One scale block's operands of a wavefront.
template <int MT, int NT, bool ROWS>
struct Operands {
    icq_i32x8 a[MT], b[NT];
    float sa[MT], sb[NT][ROWS ? 4 : 1];
};

template <int FA, int FB, bool ROWS, bool EXACT, int MT, int NT>
__global__ __launch_bounds__(64 * WAVES) void product_few_kernel(Product p, int out_type, uint32_t first_block) {
    __shared__ icq_f32x4 s_part[WAVES / 2][NT * MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = lane & 15, quarter = lane >> 4;
    const int64_t n0 = (int64_t)(first_block + blockIdx.x) * (16 * NT);
    const int whole = (int)(p.K / 128), ragged = (int)(p.K % 128);
    const uint8_t *row_a[MT], *row_b[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) row_a[i] = p.a + min((int64_t)(16 * i + at), p.M - 1) * p.lda;
#pragma unroll
    for (int j = 0; j < NT; ++j) row_b[j] = p.b + min(n0 + 16 * j + at, p.N - 1) * p.ldb;
    auto fragment = [&](const uint8_t *row, int kb) {                         // 32 bytes from 32 quarter on, zeros from K on
        const int64_t k = (int64_t)kb * 128;
        const int from = 32 * quarter, left = kb == whole ? ragged - from : 128;
        const uint4 *q = reinterpret_cast<const uint4 *>(row + k + (left > 0 ? from : 0));
        uint4 u = q[0], v = q[left > 16 ? 1 : 0];
        if (kb == whole) {
            u = first_bytes(u, left);
            v = first_bytes(v, left - 16);
        }
        icq_i32x8 f = {(int)u.x, (int)u.y, (int)u.z, (int)u.w, (int)v.x, (int)v.y, (int)v.z, (int)v.w};
        return f;
    };
    auto load = [&](Operands<MT, NT, ROWS> &o, int kb) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            o.b[j] = fragment(row_b[j], kb);
            if constexpr (ROWS) {
#pragma unroll
                for (int e = 0; e < 4; ++e) o.sb[j][e] = p.sb[min(n0 + 16 * j + 4 * quarter + e, p.N - 1) * p.kb + kb];
            } else {
                o.sb[j][0] = p.sb[min((n0 + 16 * j) >> 7, (p.N - 1) >> 7) * p.kb + kb];
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            o.a[i] = fragment(row_a[i], kb);
            o.sa[i] = p.sa[min((int64_t)(16 * i + at), p.M - 1) * p.kb + kb];
        }
    };
    icq_f32x4 acc[MT][NT] = {};
    auto multiply = [&](const Operands<MT, NT, ROWS> &o) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const icq_f32x4 d = dot128<FA, FB, EXACT>(o.b[j], o.a[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(d[e], o.sa[i] * o.sb[j][ROWS ? e : 0], acc[i][j][e]);
            }
    };
    Operands<MT, NT, ROWS> even, odd;
    const int end = min(p.kb, ((int)blockIdx.y + 1) * p.per);
    int kb = blockIdx.y * p.per + wave;
    if (kb < end) {
        load(even, kb);
        for (;;) {
            if (kb + WAVES < end) load(odd, kb + WAVES);
            multiply(even);
            if ((kb += WAVES) >= end) break;
            if (kb + WAVES < end) load(even, kb + WAVES);
            multiply(odd);
            if ((kb += WAVES) >= end) break;
        }
    }
#pragma unroll
    for (int h = WAVES / 2; h > 0; h >>= 1) {
        if (h < WAVES / 2) __syncthreads();
        if (wave >= h && wave < 2 * h) {
#pragma unroll
            for (int t = 0; t < NT * MT; ++t) s_part[wave - h][t][lane] = acc[t % MT][t / MT];
        }
        __syncthreads();
        if (wave < h) {
#pragma unroll
            for (int t = 0; t < NT * MT; ++t) acc[t % MT][t / MT] += s_part[wave][t][lane];
        }
    }
    if (wave != 0) return;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = 16 * i + at;
        if (m >= p.M) continue;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t n = n0 + 16 * j + 4 * quarter;
            if (p.splits > 1) store_part(p, blockIdx.y, m, n, acc[i][j]);
            else if (EXACT) store4<ICQ_F32>(p, m, n, acc[i][j]);
            else if (out_type == ICQ_BF16) store4<ICQ_BF16>(p, m, n, acc[i][j]);
            else store4<ICQ_F16>(p, m, n, acc[i][j]);
        }
    }
}

template <int FA, int FB, bool ROWS, bool EXACT>
int launch(const Product &p, int num_cu, int out_type, hipStream_t s) {
    auto go = [&](auto kernel, int nt) {
        const uint32_t blocks = (uint32_t)((p.N + 16 * nt - 1) / (16 * nt));
        for (uint32_t i = 0; i < blocks; i += ICQ_PRODUCT_BLOCKS)
            hipLaunchKernelGGL(kernel, dim3(std::min(blocks - i, ICQ_PRODUCT_BLOCKS), (uint32_t)p.splits), dim3(64 * WAVES), 0, s, p, out_type, i);
    };
    if (p.M > 16) go(product_few_kernel<FA, FB, ROWS, EXACT, 2, 1>, 1);
    else if (icq_product_few_wide(p.M, p.N, num_cu)) go(product_few_kernel<FA, FB, ROWS, EXACT, 1, 4>, 4);
    else go(product_few_kernel<FA, FB, ROWS, EXACT, 1, 1>, 1);
    return icq_check_launch();
}

template <bool ROWS, bool EXACT>
int launch_formats(const Product &p, int num_cu, int fa, int fb, int out_type, hipStream_t s) {
    if (fa == ICQ_E4M3) return fb == ICQ_E4M3 ? launch<ICQ_E4M3, ICQ_E4M3, ROWS, EXACT>(p, num_cu, out_type, s) : launch<ICQ_E4M3, ICQ_E5M2, ROWS, EXACT>(p, num_cu, out_type, s);
    return fb == ICQ_E4M3 ? launch<ICQ_E5M2, ICQ_E4M3, ROWS, EXACT>(p, num_cu, out_type, s) : launch<ICQ_E5M2, ICQ_E5M2, ROWS, EXACT>(p, num_cu, out_type, s);
}

}  // namespace

int icq_launch_product_few(const Product &p, int num_cu, int fa, int fb, bool rows, int out_type, hipStream_t s) {
    if (out_type == ICQ_F32)
        return rows ? launch_formats<true, true>(p, num_cu, fa, fb, out_type, s) : launch_formats<false, true>(p, num_cu, fa, fb, out_type, s);
    return rows ? launch_formats<true, false>(p, num_cu, fa, fb, out_type, s) : launch_formats<false, false>(p, num_cu, fa, fb, out_type, s);
}
