// Large products of 8-bit matrices with block scales: a 256 x 256 tile of the result per block, 128 x 64 per wavefront.
//
// The operands' tiles of one scale block (64 KB) go from memory straight into the LDS, one stage ahead of the matrix instructions; a
// row's eight 16-byte pieces are permuted by its number, by the choice of each lane's address, so that a fragment's reads
// spread over the banks.  Eight wavefronts, two per SIMD: one's multiply-adds and LDS reads run beside the other's matrix instructions.
#include "icq_matmul.h"

namespace {

constexpr int TM = 256, TN = 256, STAGE = (TM + TN) * 128, SCALES = 4 * (TM + TN);     // bytes of a stage; scales of four blocks along K
constexpr int LDS_BYTES = 2 * STAGE + 2 * SCALES * 4;

typedef float f32x16 __attribute__((ext_vector_type(16)));

enum Mode { FAST, FAST_POW2, EXACT };      // 8-bit matrix instructions; those with their own scales; 16-bit ones over widened codes

template <int FA, int FB, int MODE>
__device__ __forceinline__ f32x16 dot64(const icq_i32x8 &n, const icq_i32x8 &m, f32x16 c, int sn, int sm) {
    if constexpr (MODE == FAST) return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(n, m, c, FB, FA, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
    else if constexpr (MODE == FAST_POW2) return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(n, m, c, FB, FA, 0, sn, 0, sm);
    else {
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen<FB>(n, q), widen<FA>(m, q), c, 0, 0, 0);
        return c;
    }
}

__device__ __forceinline__ icq_i32x8 two_pieces(const uint8_t *row, int c0, int c1) {
    const uint4 u = *reinterpret_cast<const uint4 *>(row + c0 * 16), v = *reinterpret_cast<const uint4 *>(row + c1 * 16);
    icq_i32x8 f = {(int)u.x, (int)u.y, (int)u.z, (int)u.w, (int)v.x, (int)v.y, (int)v.z, (int)v.w};
    return f;
}

typedef __attribute__((address_space(3))) void lds_void;

template <int FA, int FB, bool ROWS, int MODE>
__global__ __launch_bounds__(512, 2) void product_wide_kernel(Product p, int tiles_m, int tiles_n, int out_type) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    float *s_scales = reinterpret_cast<float *>(smem + 2 * STAGE);            // [2][a: 4 x 256, b: 4 x 256]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // XCD blockIdx % 8 takes a contiguous share of the tiles, eight tiles of m at a time
    const int total = tiles_m * tiles_n, q8 = total / 8, r8 = total % 8, xcd = blockIdx.x % 8, at8 = blockIdx.x / 8;
    const int tile = xcd * q8 + (xcd < r8 ? xcd : r8) + at8;
    const int group = tile / (8 * tiles_n), in = tile % (8 * tiles_n), high = min(8, tiles_m - group * 8);
    const int64_t m0 = (int64_t)(group * 8 + in % high) * TM, n0 = (int64_t)(in / high) * TN;
    const int k0 = blockIdx.y * p.per, k1 = min(p.kb, k0 + p.per);
    const int wm = (wave & 1) * 128, wn = (wave >> 1) * 64, at = lane & 31, half = lane >> 5;
    const int whole = (int)(p.K / 128), ragged = (int)(p.K % 128);            // blocks along K, and what is in one more

    // this lane's place in the tile loads: instruction u of a wavefront brings rows 64 u + 8 wave .. + 7
    const int piece = (lane & 7) ^ (lane >> 3);                               // row r's piece c sits at place c ^ (r & 7)
    uint32_t off_a[4], off_b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int r = 64 * u + 8 * wave + (lane >> 3);
        const int64_t ra = min((int64_t)r, p.M - 1 - m0), rb = min((int64_t)r, p.N - 1 - n0);
        off_a[u] = (uint32_t)(ra * p.lda) + piece * 16;
        off_b[u] = (uint32_t)(rb * p.ldb) + piece * 16;
    }
    const auto rsrc_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.a + m0 * p.lda), 0, 0xffffffffu, 0x00027000);
    const auto rsrc_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.b + n0 * p.ldb), 0, 0xffffffffu, 0x00027000);

    auto load_stage = [&](int kb, int buf) {
        uint8_t *to = smem + buf * STAGE + wave * 1024;
        const int beyond = kb == whole && piece * 16 >= ragged ? piece * 16 : 0;   // pieces beyond the row: any of its bytes will do
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_a, (lds_void *)(to + u * 8192), 16, off_a[u] - beyond, kb * 128, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_b, (lds_void *)(to + TM * 128 + u * 8192), 16, off_b[u] - beyond, kb * 128, 0, 0);
        }
    };
    // the last block's bytes from K on become zero: thread t has row t of the stage (a's rows, then b's)
    auto clear_beyond = [&](int buf) {
        uint8_t *row = smem + buf * STAGE + tid * 128;
        for (int c = ragged >> 4; c < 8; ++c) {
            uint4 *w = reinterpret_cast<uint4 *>(row + ((c ^ (tid & 7)) << 4));
            *w = c * 16 < ragged ? first_bytes(*w, ragged & 15) : make_uint4(0, 0, 0, 0);
        }
    };
    int place[2][2];                                                          // this lane's two pieces of each half of a block
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 2; ++c) place[h][c] = (4 * h + 2 * half + c) ^ (at & 7);
    // scales of blocks k .. k + 3: thread t has rows t % 256, blocks 2 (t / 256) and the next
    const int64_t row_a = min(m0 + (tid & 255), p.M - 1) * p.kb;
    const int64_t row_b = (ROWS ? min(n0 + (tid & 255), p.N - 1) : min((n0 >> 7) + (tid & 1), (p.N - 1) >> 7)) * p.kb;
    float sc[4];
    auto read_scales = [&](int k) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int kb = min(k + 2 * (tid >> 8) + h, p.kb - 1);
            sc[h] = p.sa[row_a + kb];
            sc[2 + h] = p.sb[row_b + kb];
        }
    };
    auto write_scales = [&](int buf) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at4 = 2 * (tid >> 8) + h;
            s_scales[buf * SCALES + at4 * TM + (tid & 255)] = sc[h];
            s_scales[buf * SCALES + 4 * TM + at4 * TN + (tid & 255)] = sc[2 + h];
        }
    };

    f32x16 acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    if (k0 < k1) {
        load_stage(k0, 0);
        read_scales(k0);
        write_scales(0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int kb = k0; kb < k1; ++kb) {
        const int step = kb - k0, buf = step & 1;
        if (kb == whole) {
            clear_beyond(buf);
            __syncthreads();
        }
        if (kb + 1 < k1) load_stage(kb + 1, buf ^ 1);
        if ((step & 3) == 3) write_scales(((step >> 2) & 1) ^ 1);             // (read three steps ago)
        if ((step & 3) == 0) read_scales(kb + 4);
        const uint8_t *tile_a = smem + buf * STAGE + (wm + at) * 128, *tile_b = smem + buf * STAGE + (TM + wn + at) * 128;
        const float *sc_a = s_scales + ((step >> 2) & 1) * SCALES + (step & 3) * TM + wm + at;
        const float *sc_b = s_scales + ((step >> 2) & 1) * SCALES + 4 * TM + (step & 3) * TN + (ROWS ? wn : wn >> 7);
        icq_i32x8 fb[2][2], fa[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < 2; ++j) fb[j][h] = two_pieces(tile_b + j * 32 * 128, place[h][0], place[h][1]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) fa[h] = two_pieces(tile_a + i * 32 * 128, place[h][0], place[h][1]);
            const float sa = sc_a[i * 32];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if constexpr (MODE == FAST_POW2) {
                    const float sb = ROWS ? sc_b[j * 32 + at] : sc_b[0];
                    const int em = (int)(__float_as_uint(sa) >> 23), en = (int)(__float_as_uint(sb) >> 23);
#pragma unroll
                    for (int h = 0; h < 2; ++h) acc[i][j] = dot64<FA, FB, MODE>(fb[j][h], fa[h], acc[i][j], en, em);
                } else {
                    f32x16 d;
#pragma unroll
                    for (int e = 0; e < 16; ++e) d[e] = 0.0f;
#pragma unroll
                    for (int h = 0; h < 2; ++h) d = dot64<FA, FB, MODE>(fb[j][h], fa[h], d, 0, 0);
                    if constexpr (ROWS) {
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const icq_f32x4 sb = *reinterpret_cast<const icq_f32x4 *>(sc_b + j * 32 + 8 * g + 4 * half);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] = fmaf(d[4 * g + e], sa * sb[e], acc[i][j][4 * g + e]);
                        }
                    } else {
                        const float s = sa * sc_b[0];
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[i][j][e] = fmaf(d[e], s, acc[i][j][e]);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);                                // (later fragments would be read early, beyond the registers)
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + wm + i * 32 + at;
        if (m >= p.M) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int64_t n = n0 + wn + j * 32 + 8 * g + 4 * half;
                const icq_f32x4 v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                if (p.splits > 1) {
                    float *o = p.part + ((int64_t)blockIdx.y * p.M + m) * p.N + n;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n + e < p.N) o[e] = v[e];
                } else if (MODE == EXACT) {
                    store4<ICQ_F32>(p, m, n, v);
                } else if (out_type == ICQ_BF16) {
                    store4<ICQ_BF16>(p, m, n, v);
                } else {
                    store4<ICQ_F16>(p, m, n, v);
                }
            }
    }
}

template <int FA, int FB, bool ROWS>
int launch(const Product &p, bool pow2, int out_type, hipStream_t s) {
    const int tm = (int)((p.M + TM - 1) / TM), tn = (int)((p.N + TN - 1) / TN);
    const dim3 grid((uint32_t)((int64_t)tm * tn), (uint32_t)p.splits);
    auto go = [&](auto kernel) {
        if (icq_allow_lds(reinterpret_cast<const void *>(kernel), LDS_BYTES) != hipSuccess) return ICQ_ERR_HIP;
        hipLaunchKernelGGL(kernel, grid, dim3(512), LDS_BYTES, s, p, tm, tn, out_type);
        return icq_check_launch();
    };
    if (out_type == ICQ_F32) return go(product_wide_kernel<FA, FB, ROWS, EXACT>);
    if (pow2) return go(product_wide_kernel<FA, FB, ROWS, FAST_POW2>);
    return go(product_wide_kernel<FA, FB, ROWS, FAST>);
}

}  // namespace

// Rows of the tile within 32 bits of its first, and tiles for most of the chip.
bool icq_product_wide_usable(int64_t M, int64_t N, int64_t K, int64_t lda, int64_t ldb, int num_cu) {
    const int64_t tiles = ((M + TM - 1) / TM) * ((N + TN - 1) / TN);
    return K >= 128 && lda < (1 << 23) && ldb < (1 << 23) && tiles >= num_cu / 2 && tiles < (1 << 28);
}

int icq_launch_product_wide(const Product &p, int fa, int fb, bool rows, bool pow2, int out_type, hipStream_t s) {
    if (fa == ICQ_E4M3 && fb == ICQ_E4M3) return rows ? launch<ICQ_E4M3, ICQ_E4M3, true>(p, pow2, out_type, s) : launch<ICQ_E4M3, ICQ_E4M3, false>(p, pow2, out_type, s);
    if (fa == ICQ_E4M3) return rows ? launch<ICQ_E4M3, ICQ_E5M2, true>(p, pow2, out_type, s) : launch<ICQ_E4M3, ICQ_E5M2, false>(p, pow2, out_type, s);
    if (fb == ICQ_E4M3) return rows ? launch<ICQ_E5M2, ICQ_E4M3, true>(p, pow2, out_type, s) : launch<ICQ_E5M2, ICQ_E4M3, false>(p, pow2, out_type, s);
    return rows ? launch<ICQ_E5M2, ICQ_E5M2, true>(p, pow2, out_type, s) : launch<ICQ_E5M2, ICQ_E5M2, false>(p, pow2, out_type, s);
}
