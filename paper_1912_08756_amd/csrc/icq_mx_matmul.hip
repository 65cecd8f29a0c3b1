// Products of matrices held in microscaled 4-bit floating point:
//     out[m][n] = sum_kb sa[m][kb] sb[n][kb] sum_{k in block kb} a[m][k] b[n][k].
//
// The matrix instructions take 32 codes of a row and their scale's byte from each lane and sum in 32 bits: products of two codes are whole quarters up to 36, and
// unlike those of 8 bits none of their bits are lost (4096 products of 32 x 32 x 64 with random codes and scales within 2^6 of each
// other: equal to the sums in 64 bits).  So one kernel serves results of any type.  A scale byte of 255 makes the row NaN.
#include "icq_mx.h"

namespace {

bool values(int a_type) { return icq_type_bytes(a_type) > 0; }

// The workspace: the parts' sums, then a's codes and scales if it comes as values.
struct Held { int64_t ld, ld_s; size_t codes, scales, bytes; };
Held held(int64_t M, int64_t N, int64_t K, bool values, const icq_mx_plan &plan) {
    Held h = {};
    h.codes = plan.splits > 1 ? icq_align_up((size_t)plan.splits * M * N * sizeof(float), ICQ_ALIGN) : 0;
    h.bytes = h.codes;
    if (!values || (plan.few && icq_mx_few_quantises(M, plan.per))) return h;      // (the kernel for few rows quantises them itself)
    h.ld = (K + 255) / 256 * 128;                                                  // (whole lines to a row: 4096 x 10000 x 960 48.4 us against 50 in rows of 480 bytes)
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
    p.kb = (int)((K + 255) / 256);
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
    p.splits = plan.splits; p.per = plan.per;
    p.part = static_cast<float *>(workspace);
    int rc = ICQ_OK;
    if (h.scales > 0) {
        MxQuantize z = {};
        z.x = a; z.rows = M; z.cols = K; z.ldx = lda;
        z.codes = static_cast<uint8_t *>(workspace) + h.codes; z.scales = static_cast<uint8_t *>(workspace) + h.scales; z.ld = h.ld; z.ld_s = h.ld_s;
        z.across = (int)((K + 127) / 128);
        z.fit = scaling == ICQ_MX_FIT;
        if ((rc = icq_launch_mx_rows(z, a_type, s)) != ICQ_OK) return rc;
        p.a = z.codes; p.lda = h.ld; q.ea = z.scales; q.ld_ea = h.ld_s;
        a_type = ICQ_E2M1;
    }
    rc = plan.few ? icq_launch_mx_few(q, plan, cu, a, a_type, lda, scaling == ICQ_MX_FIT, out_type, s) : icq_launch_mx_tiles(q, plan.tiles, cu, out_type, s);
    return rc != ICQ_OK || p.splits == 1 ? rc : icq_launch_product_join(p, out_type, s);
}
