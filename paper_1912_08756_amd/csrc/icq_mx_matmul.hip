// Products of matrices held in microscaled 4-bit floating point:
//     out[m][n] = sum_kb sa[m][kb] sb[n][kb] sum_{k in block kb} a[m][k] b[n][k].
//
// The matrix instructions take 32 codes of a row and their scale's byte from each lane and sum in 32 bits: products of two codes are whole quarters up to 36, and
// unlike those of 8 bits none of their bits are lost (4096 products of 32 x 32 x 64 with random codes and scales within 2^6 of each
// other: equal to the sums in 64 bits).  So one kernel serves results of any type.  A scale byte of 255 makes the row NaN.
//
// A wavefront has 16 rows of a and 16 of b, straight from memory in the instruction's layout; b's rows are the instruction's rows, so a lane ends up
// with four consecutive n of one m.
#include "icq_mx.h"

#include <algorithm>

namespace {

constexpr int WAVES = 4;

__global__ __launch_bounds__(64 * WAVES) void mx_product_kernel(MxProduct q, int tiles_n, int out_type, int64_t first_tile, int64_t end_tile) {
    const Product &p = q.p;
    const int lane = threadIdx.x & 63, at = lane & 15, quarter = lane >> 4;
    const int64_t tile = first_tile + (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
    if (tile >= end_tile) return;
    const int64_t m0 = tile / tiles_n * 16, n0 = tile % tiles_n * 16;
    const int64_t ra = min(m0 + at, p.M - 1), rb = min(n0 + at, p.N - 1);
    const uint8_t *row_a = p.a + ra * p.lda, *row_b = p.b + rb * p.ldb, *scale_a = q.ea + ra * q.ld_ea, *scale_b = q.eb + rb * q.ld_eb;
    icq_f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int kb = 0; kb < p.kb; ++kb) {
        const int block = 4 * kb + quarter;
        const int64_t left = p.K - (int64_t)block * 32;
        const int64_t from = left > 0 ? (int64_t)block * 16 : 0;
        const auto codes = [&](const uint8_t *row) {
            const uint4 v = first_codes(*reinterpret_cast<const uint4 *>(row + from), (int)min(max(left, (int64_t)0), (int64_t)32));
            icq_i32x8 f = {(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
            return f;
        };
        const int ea = left > 0 ? scale_a[block] : 127, eb = left > 0 ? scale_b[block] : 127;
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes(row_b), codes(row_a), acc, 4, 4, 0, eb, 0, ea);
    }
    const int64_t m = m0 + at, n = n0 + 4 * quarter;
    if (m >= p.M) return;
    if (out_type == ICQ_F32) store4<ICQ_F32>(p, m, n, acc);
    else if (out_type == ICQ_BF16) store4<ICQ_BF16>(p, m, n, acc);
    else store4<ICQ_F16>(p, m, n, acc);
}

bool values(int a_type) { return icq_type_bytes(a_type) > 0; }

// The workspace: the parts' sums, then a's codes and scales if it comes as values.
struct Held { int64_t ld, ld_s; size_t codes, scales, bytes; };
Held held(int64_t M, int64_t N, int64_t K, bool values, const icq_mx_plan &plan) {
    Held h = {};
    h.codes = plan.splits > 1 ? icq_align_up((size_t)plan.splits * M * N * sizeof(float), ICQ_ALIGN) : 0;
    h.bytes = h.codes;
    if (!values) return h;
    h.ld = (K + 31) / 32 * 16;
    h.ld_s = (K + 127) / 128 * 4;
    h.scales = h.codes + icq_align_up((size_t)M * h.ld, ICQ_ALIGN);
    h.bytes = h.scales + icq_align_up((size_t)M * h.ld_s, ICQ_ALIGN);
    return h;
}

}  // namespace

ICQ_EXPORT int icq_mx_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int a_type, size_t *out) {
    if (!out || !icq_product_extents_ok(M, N, K) || (a_type != ICQ_E2M1 && !values(a_type))) return ICQ_ERR_ARG;
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    *out = M > 0 && N > 0 && K > 0 ? held(M, N, K, values(a_type), icq_plan_mx(M, N, K, cu)).bytes : 0;
    return ICQ_OK;
}

ICQ_EXPORT int icq_mx_matmul(const void *a, int a_type, int64_t lda, const uint8_t *a_scales, int64_t ld_a_scales, int scaling, const uint8_t *b, int64_t ldb,
                             const uint8_t *b_scales, int64_t ld_b_scales, int64_t M, int64_t N, int64_t K, void *out, int out_type, int64_t ldo, void *workspace,
                             size_t workspace_bytes, void *stream) {
    const int size = icq_type_bytes(out_type);
    if (size == 0 || (a_type != ICQ_E2M1 && !values(a_type)) || (scaling != ICQ_MX_FLOOR && scaling != ICQ_MX_FIT) || !icq_product_extents_ok(M, N, K)) return ICQ_ERR_ARG;
    if (M == 0 || N == 0) return ICQ_OK;
    if (!out || (uintptr_t)out % size != 0 || ldo < N) return ICQ_ERR_ARG;
    const int64_t bytes = (K + 1) / 2, blocks = (K + 31) / 32;
    const auto held_ok = [&](const void *p, int64_t ld, const uint8_t *scales, int64_t ld_s) {
        return p && scales && ld >= bytes && ld <= ICQ_MAX_CODE_LD && ld % 16 == 0 && (uintptr_t)p % 16 == 0 && ld_s >= blocks && ld_s <= ICQ_MAX_CODE_LD && ld_s % 4 == 0 &&
               (uintptr_t)scales % 4 == 0;
    };
    if (K > 0) {
        if (!held_ok(b, ldb, b_scales, ld_b_scales)) return ICQ_ERR_ARG;
        if (values(a_type) ? !a || a_scales || lda < K || (uintptr_t)a % icq_type_bytes(a_type) != 0 || bytes > ICQ_MAX_CODE_LD : !held_ok(a, lda, a_scales, ld_a_scales)) return ICQ_ERR_ARG;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    MxProduct q;
    Product &p = q.p;
    p.a = static_cast<const uint8_t *>(a); p.b = b; p.lda = lda; p.ldb = ldb; p.sa = p.sb = nullptr;
    p.M = M; p.N = N; p.K = K;
    p.kb = (int)((K + 127) / 128);
    p.out = out; p.ldo = ldo;
    p.part = nullptr; p.splits = 1; p.per = p.kb;
    q.ea = a_scales; q.eb = b_scales; q.ld_ea = ld_a_scales; q.ld_eb = ld_b_scales; q.blocks = (int)blocks;
    if (K == 0) {
        p.splits = 0;                                                         // (a sum of nothing)
        return icq_launch_product_join(p, out_type, s);
    }
    const int cu = icq_num_cu();
    if (cu <= 0) return ICQ_ERR_HIP;
    const icq_mx_plan plan = icq_plan_mx(M, N, K, cu);
    const Held h = held(M, N, K, values(a_type), plan);
    if (h.bytes > 0 && (!workspace || (uintptr_t)workspace % ICQ_ALIGN != 0 || workspace_bytes < h.bytes)) return ICQ_ERR_WORKSPACE;
    if (values(a_type)) {
        MxQuantize z = {};
        z.x = a; z.rows = M; z.cols = K; z.ldx = lda;
        z.codes = static_cast<uint8_t *>(workspace) + h.codes; z.scales = static_cast<uint8_t *>(workspace) + h.scales; z.ld = h.ld; z.ld_s = h.ld_s;
        z.across = (int)((K + 127) / 128);
        z.fit = scaling == ICQ_MX_FIT;
        const int rc = icq_launch_mx_rows(z, a_type, s);
        if (rc != ICQ_OK) return rc;
        p.a = z.codes; p.lda = h.ld; q.ea = z.scales; q.ld_ea = h.ld_s;
    }
    if (!plan.few) {
        p.kb = (int)((K + 255) / 256);
        p.splits = plan.splits; p.per = plan.per;
        p.part = static_cast<float *>(workspace);
        const int rc = icq_launch_mx_tiles(q, plan.tiles, out_type, s);
        return rc != ICQ_OK || p.splits == 1 ? rc : icq_launch_product_join(p, out_type, s);
    }
    const int64_t tiles_n = (N + 15) / 16, tiles = (M + 15) / 16 * tiles_n, step = (int64_t)ICQ_PRODUCT_BLOCKS * WAVES;
    for (int64_t t = 0; t < tiles; t += step) {
        const int64_t end = std::min(tiles, t + step);
        hipLaunchKernelGGL(mx_product_kernel, dim3((uint32_t)((end - t + WAVES - 1) / WAVES)), dim3(64 * WAVES), 0, s, q, (int)tiles_n, out_type, t, end);
    }
    return icq_check_launch();
}
