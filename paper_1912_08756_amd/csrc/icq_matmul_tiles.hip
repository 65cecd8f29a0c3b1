// Products of 8-bit matrices with block scales: tiles of 256 x 256 (eight wavefronts of 128 x 64), 128 x 128 (four of 64 x 64)
// or 64 x 64 (four of 32 x 32).
//
// The operands' tiles of one scale block go from memory straight into the LDS, two stages deep; a row's eight 16-byte pieces are
// permuted by its number, by the choice of each lane's address, so that 16 rows' pieces fall on all 64 banks.
// The one barrier of a step stands before its last rows' matrix instructions: by then the next stage has arrived (requested a whole step
// earlier) and this one's last fragments are in registers, so the next step's first fragments are read, and the stage after it
// requested, beside the matrix instructions that are left.
//
// What bounds them (8192^3, us; the library's 8-bit product with one scale a matrix 403, its bf16 product 899): with scales of powers of
// two 447, the matrix pipe 68 % busy at the 1.7 GHz that such operands leave, without any loads 399; with other scales 504, the
// multiply-adds beside; into f32 1050, the matrix pipe 61 % busy and the widening beside.  What the steps gave: the
// loads' requests spread over the multiplication, and no wait of the compiler's own for them, 597 -> 476; scales four blocks at a time
// (a quarter of the requests to the second-level cache); results stored in whole rows 470 -> 447, 2048 x 16384 x 960 91 -> 46.
#include "icq_matmul.h"

#include <algorithm>

namespace {

// Rows and columns of a wavefront's part in units of 32, wavefronts along m and n, stages in the LDS.
template <int NI_, int NJ_, int WM_, int WN_, int DEPTH_>
struct Shape {
    static constexpr int NI = NI_, NJ = NJ_, WM = WM_, WN = WN_, DEPTH = DEPTH_, WAVES = WM * WN, THREADS = 64 * WAVES, T = 32 * NI * WM;
    static constexpr int PARTS = T / (8 * WAVES), LOADS = 2 * PARTS;          // of a wavefront for a stage: eight rows of each operand a part
    static constexpr int STAGE = 2 * T * 128;                                 // bytes of a stage
    static constexpr int LDS_BYTES = DEPTH * STAGE + 3 * 8 * T * 4;
    static_assert(32 * NJ * WN == T && THREADS >= 2 * T && PARTS == 2 * NJ && DEPTH * STAGE / WAVES >= 32 * (32 * NJ + 4) * 4, "square tiles, a thread for every row of a stage; a stage's parts over a wavefront's columns twice; results fit the stages");
};
typedef Shape<4, 2, 2, 4, 2> Wide;
typedef Shape<2, 2, 2, 2, 2> Small;    // two blocks share a compute unit
typedef Shape<2, 2, 2, 2, 4> Deep;     // one has it to itself
typedef Shape<1, 1, 2, 2, 4> Little;   // 64 x 64: two blocks a compute unit

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

// s_waitcnt: at most n loads still under way, the other counters left alone
constexpr int loads_left(int n) { return 0x0f70 | (n & 15) | (n >> 4) << 14; }

typedef int i32x4 __attribute__((ext_vector_type(4)));

// A buffer descriptor of the memory from p on (a wavefront's own: scalar).
__device__ __forceinline__ i32x4 bytes_from(const void *p) {
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    i32x4 r = {__builtin_amdgcn_readfirstlane((int)(uint32_t)u), __builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32) & 0xffff), -1, 0x00027000};
    return r;
}

#pragma clang diagnostic ignored "-Winline-asm"       // (M0, which the next two name as overwritten, is no register of the allocator's: a warning each)

// 16 bytes per lane from base + off + by into the LDS at `to` + 16 * lane.  Written out because the compiler makes every later LDS read
// wait for loads of its own built-in; they have no destination registers, and the waits for them are those of loads_left(0).
__device__ __forceinline__ void load_to_lds(const i32x4 &base, uint32_t off, int by, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(base), "s"(by) : "memory", "m0");
}

// 32 rows and 32 NJ columns of the result from a wavefront's accumulators, whole rows at a time: in the accumulators a lane has four
// neighbours of one row and the lanes 32 rows, whose stores would be 16 bytes here and there.
template <int TYPE, int NJ>
__device__ __forceinline__ void store_rows(uint8_t *turn, const f32x16 (&acc)[NJ], void *out, int64_t ldo, int64_t M, int64_t N, int64_t m0, int64_t n0,
                                           int lane) {
    typedef IcqElem<TYPE> E;
    typedef typename E::raw raw;
    constexpr int PER = E::PER, WIDTH = 32 * NJ, STRIDE = WIDTH + PER;                            // (16 bytes more than a row: other banks)
    const int at = lane & 31, half = lane >> 5;
    raw *mine = reinterpret_cast<raw *>(turn);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            raw *to = mine + at * STRIDE + j * 32 + 8 * g + 4 * half;
            const float v[4] = {acc[j][4 * g], acc[j][4 * g + 1], acc[j][4 * g + 2], acc[j][4 * g + 3]};
            if constexpr (TYPE == ICQ_F32) *reinterpret_cast<uint4 *>(to) = E::pack(v);
            else *reinterpret_cast<uint2 *>(to) = make_uint2(E::pack2(v[0], v[1]), E::pack2(v[2], v[3]));
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    constexpr int LANES = WIDTH / PER, ROWS_AT_ONCE = 64 / LANES;
    const int c = lane % LANES * PER;
    raw *to = static_cast<raw *>(out) + (m0 + lane / LANES) * ldo + n0 + c;
    const int left = (int)min((int64_t)PER, N - n0 - c), rows = (int)min((int64_t)32, M - m0);
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += ROWS_AT_ONCE, to += ROWS_AT_ONCE * ldo) {
        const int r = r0 + lane / LANES;
        const raw *from = mine + r * STRIDE + c;
        if (r >= rows) continue;
        if (left == PER) {
            const uint4 v = *reinterpret_cast<const uint4 *>(from);
            __builtin_memcpy(to, &v, 16);                                     // (to any address)
        } else {
            for (int e = 0; e < left; ++e) to[e] = from[e];
        }
    }
}

// The same for 4 bytes per lane, to `to` + 4 * lane.
__device__ __forceinline__ void load_word_to_lds(const i32x4 &base, uint32_t off, int by, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(base), "s"(by) : "memory", "m0");
}

template <typename S, int FA, int FB, bool ROWS, int MODE>
__global__ __launch_bounds__(S::THREADS, 2) void product_kernel(Product p, int tiles_m, int tiles_n, int out_type, uint32_t first_block) {
    constexpr int T = S::T, NI = S::NI, NJ = S::NJ, DEPTH = S::DEPTH, WAVES = S::WAVES, PARTS = S::PARTS, LOADS = S::LOADS;
    // loads under way that the barrier need not wait for: those of the stages after the next
    constexpr int LATER = (DEPTH - 2) * LOADS - (NI == 1 ? LOADS / 2 : 0);
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    float *s_scales = reinterpret_cast<float *>(smem + DEPTH * S::STAGE);     // [3][four blocks along K][a: T, b: T]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // XCD blockIdx % 8 takes a contiguous share of the tiles, eight tiles of m at a time (first_block: a multiple of 8)
    const uint32_t block_id = first_block + blockIdx.x;
    const int total = tiles_m * tiles_n, q8 = total / 8, r8 = total % 8, xcd = block_id % 8, at8 = block_id / 8;
    const int tile = xcd * q8 + (xcd < r8 ? xcd : r8) + at8;
    const int group = tile / (8 * tiles_n), in = tile % (8 * tiles_n), high = min(8, tiles_m - group * 8);
    const int64_t m0 = (int64_t)(group * 8 + in % high) * T, n0 = (int64_t)(in / high) * T;
    const int k0 = blockIdx.y * p.per, k1 = min(p.kb, k0 + p.per);
    const int wm = (wave % S::WM) * 32 * NI, wn = (wave / S::WM) * 32 * NJ, at = lane & 31, half = lane >> 5;
    const int whole = (int)(p.K / 128), ragged = (int)(p.K % 128);            // blocks along K, and what is in one more

    // this lane's place in the tile loads: instruction u of a wavefront brings rows 8 (WAVES u + wave) .. + 7;
    // row r's piece c sits at place c ^ (r / 2 % 8)
    uint32_t off_a[PARTS], off_b[PARTS];
    const int piece = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
        const int r = 8 * (WAVES * u + wave) + (lane >> 3);
        const int64_t ra = min((int64_t)r, p.M - 1 - m0), rb = min((int64_t)r, p.N - 1 - n0);
        off_a[u] = (uint32_t)(ra * p.lda) + piece * 16;
        off_b[u] = (uint32_t)(rb * p.ldb) + piece * 16;
    }
    const i32x4 rsrc_a = bytes_from(p.a + m0 * p.lda), rsrc_b = bytes_from(p.b + n0 * p.ldb);
    auto load_part = [&](int kb, int buf, int u, uint32_t back) {
        const uint32_t to = buf * S::STAGE + wave * 1024 + u * WAVES * 1024;
        load_to_lds(rsrc_a, off_a[u] - back, kb * 128, to);
        load_to_lds(rsrc_b, off_b[u] - back, kb * 128, to + T * 128);
    };
    // the last block's bytes from K on become zero: thread t has row t of the stage (a's rows, then b's)
    auto clear_beyond = [&](int buf) {
        uint8_t *row = smem + buf * S::STAGE + tid * 128;
        for (int c = ragged >> 4; c < 8 && tid < 2 * T; ++c) {
            uint4 *w = reinterpret_cast<uint4 *>(row + ((c ^ (tid >> 1 & 7)) << 4));
            *w = c * 16 < ragged ? first_bytes(*w, ragged & 15) : make_uint4(0, 0, 0, 0);
        }
        __syncthreads();
    };
    int place[2][2];                                                          // this lane's two pieces of each half of a block
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 2; ++c) place[h][c] = (4 * h + 2 * half + c) ^ (at >> 1 & 7);
    // thread t brings the scale of row t of the stage (a's rows, then b's)
    const float *scale_row = tid < T ? p.sa + min(m0 + tid, p.M - 1) * p.kb
                                     : p.sb + (ROWS ? min(n0 + tid % T, p.N - 1) : min((n0 >> 7) + (tid & 1), (p.N - 1) >> 7)) * p.kb;
    // ... of blocks kb .. kb + 3, as far as there are any
    struct Four { float v[4]; };
    auto read_scales = [&](int kb) {
        Four f;
        if (p.kb >= 4) {
            const int from = min(kb, p.kb - 4), by = kb - from;
            __builtin_memcpy(&f, scale_row + from, 16);
            for (int k = 0; k < by; ++k) { f.v[0] = f.v[1]; f.v[1] = f.v[2]; f.v[2] = f.v[3]; }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) f.v[k] = scale_row[min(kb + k, p.kb - 1)];
        }
        return f;
    };
    // the same straight into the LDS, a block along K at a time: loads of the compiler's own would have to be waited for with all others,
    // and four stages are to stay under way (two are not: at the barrier nothing is)
    const i32x4 rsrc_scale = bytes_from(wave < T / 64 ? p.sa + m0 * p.kb : p.sb + (ROWS ? n0 : n0 >> 7) * p.kb);
    const uint32_t off_scale = (uint32_t)((tid < T ? min((int64_t)tid, p.M - 1 - m0)
                                                   : ROWS ? min((int64_t)(tid % T), p.N - 1 - n0) : min((int64_t)(tid & 1), ((p.N - 1) >> 7) - (n0 >> 7))) * p.kb * 4);
    auto scales_to_lds = [&](int third, int kb) {
        if (wave >= 2 * T / 64) return;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            load_word_to_lds(rsrc_scale, off_scale, min(kb + k, p.kb - 1) * 4, DEPTH * S::STAGE + ((third * 4 + k) * 2 * T + wave * 64) * 4);
    };
    auto write_scales = [&](int third, const Four &f) {
#pragma unroll
        for (int k = 0; k < 4; ++k) s_scales[(third * 4 + k) * 2 * T + tid] = f.v[k];
    };

    f32x16 acc[NI][NJ];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    icq_i32x8 fa[2][2], fb[NJ][2];
    float sa[2], sb[NJ];
    // rows 32 i .. of this wavefront times columns 32 j ..; sc: the block's scales
    auto multiply = [&](int i, int j, const float *sc) {
        if constexpr (MODE == FAST_POW2) {
            const int em = (int)(__float_as_uint(sa[i & 1]) >> 23), en = (int)(__float_as_uint(ROWS ? sb[j] : sb[0]) >> 23);
#pragma unroll
            for (int h = 0; h < 2; ++h) acc[i][j] = dot64<FA, FB, MODE>(fb[j][h], fa[i & 1][h], acc[i][j], en, em);
        } else {
            f32x16 d;
#pragma unroll
            for (int e = 0; e < 16; ++e) d[e] = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h) d = dot64<FA, FB, MODE>(fb[j][h], fa[i & 1][h], d, 0, 0);
            if constexpr (ROWS) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const icq_f32x4 s = *reinterpret_cast<const icq_f32x4 *>(sc + T + wn + j * 32 + 8 * g + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] = fmaf(d[4 * g + e], sa[i & 1] * s[e], acc[i][j][4 * g + e]);
                }
            } else {
                const float s = sa[i & 1] * sb[0];
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = fmaf(d[e], s, acc[i][j][e]);
            }
        }
    };
    auto read_a = [&](int i, int buf, const float *sc) {
        sa[i & 1] = sc[wm + at + i * 32];
#pragma unroll
        for (int h = 0; h < 2; ++h) fa[i & 1][h] = two_pieces(smem + buf * S::STAGE + (wm + i * 32 + at) * 128, place[h][0], place[h][1]);
    };
    auto read_b = [&](int j, int buf, const float *sc) {
        if (ROWS && MODE == FAST_POW2) sb[j] = sc[T + wn + j * 32 + at];
        if (!ROWS && j == NJ - 1) sb[0] = sc[T + (wn >> 7)];
#pragma unroll
        for (int h = 0; h < 2; ++h) fb[j][h] = two_pieces(smem + buf * S::STAGE + (T + wn + j * 32 + at) * 128, place[h][0], place[h][1]);
    };

    const int kw = min(k1, whole), last = k1 - 1;                             // whole blocks: [k0, kw); a ragged one may follow
    const uint32_t beyond = piece * 16 >= ragged ? piece * 16 : 0;            // there, pieces beyond the row: any of its bytes will do
    int block = 0;
    if (k0 < k1) {
#pragma unroll
        for (int u = 0; u < PARTS; ++u) load_part(k0, 0, u, k0 == whole ? beyond : 0);
        if constexpr (DEPTH > 2) scales_to_lds(0, k0);
        else write_scales(0, read_scales(k0));
    }
    uint32_t back = 0;                                                        // of the stage under way
    if (k0 < kw) {
#pragma unroll
        for (int d = 1; d < DEPTH; ++d) {
            back = min(k0 + d, last) == whole ? beyond : 0;
#pragma unroll
            for (int u = 0; u < (d == DEPTH - 1 ? PARTS / 2 : PARTS); ++u) load_part(min(k0 + d, last), d, u, back);
        }
        __builtin_amdgcn_s_waitcnt(loads_left((DEPTH - 2) * LOADS + LOADS / 2));
    } else {
        __builtin_amdgcn_s_waitcnt(loads_left(0));
    }
    __syncthreads();
    if (k0 < kw) {
        Four next;
        if constexpr (DEPTH == 2) next = read_scales(min(k0 + 4, last));
        read_a(0, 0, s_scales);
#pragma unroll
        for (int j = 0; j < NJ; ++j) read_b(j, 0, s_scales);
        int kb = k0, third = 0, buf = 0;
        do {                                                                  // four blocks: their scales are in the LDS
            block = third * 4;
            third = third == 2 ? 0 : third + 1;
            if constexpr (DEPTH > 2) scales_to_lds(third, min(kb + 4, last)); // (nobody reads that third any more: four barriers since)
            else {
                write_scales(third, next);
                next = read_scales(min(kb + 8, last));
            }
            const int end = min(kb + 4, kw);
            // no branch in the loop: behind one, the compiler would put off matrix instructions and keep their fragments;
            // the last steps request the last stage again
            do {
                const int next_buf = buf == DEPTH - 1 ? 0 : buf + 1, last_buf = buf == 0 ? DEPTH - 1 : buf - 1;
                const float *sc = s_scales + block * 2 * T;
                block = block == 11 ? 0 : block + 1;
                const float *sc_next = s_scales + block * 2 * T;
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    if (i < NI - 1) {
                        read_a(i + 1, buf, sc);
                    } else {
                        __builtin_amdgcn_s_waitcnt(loads_left(LATER));                    // the next stage is here, later ones may not be
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
                        __builtin_amdgcn_s_barrier();
                    }
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        // a stage's requests are spread over four parts of the multiplication: all at once they hold up the wavefront
                        if (i == 0) load_part(min(kb + DEPTH - 1, last), last_buf, NJ + j, back);
                        if (i == NI - 1) {
                            back = min(kb + DEPTH, last) == whole ? beyond : 0;
                            load_part(min(kb + DEPTH, last), buf, j, back);
                        }
                        multiply(i, j, sc);
                        if (i == NI - 1) {                                    // the next step's first fragments (after the last step: not used)
                            if (j == 0) read_a(0, next_buf, sc_next);
                            read_b(j, next_buf, sc_next);
                        }
                        __builtin_amdgcn_sched_barrier(0);                    // (later fragments would be read early, beyond the registers)
                    }
                }
                buf = next_buf;
            } while (++kb < end);
        } while (kb < kw);
        __builtin_amdgcn_s_waitcnt(loads_left(0));
        __syncthreads();
    }
    if (k0 < k1 && kw < k1) {                                                // the ragged end: its stage has arrived
        const int buf = (kw - k0) % DEPTH;
        const float *sc = s_scales + block * 2 * T;
        clear_beyond(buf);
#pragma unroll
        for (int j = 0; j < NJ; ++j) read_b(j, buf, sc);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            read_a(i, buf, sc);
#pragma unroll
            for (int j = 0; j < NJ; ++j) multiply(i, j, sc);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __syncthreads();                                                          // (a wavefront's part of the stages takes its results)
    uint8_t *turn = smem + wave * (DEPTH * S::STAGE / WAVES);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int64_t m = m0 + wm + i * 32, n = n0 + wn;
        if (p.splits > 1) store_rows<ICQ_F32, NJ>(turn, acc[i], p.part + (int64_t)blockIdx.y * p.M * p.N, p.N, p.M, p.N, m, n, lane);
        else if (MODE == EXACT) store_rows<ICQ_F32, NJ>(turn, acc[i], p.out, p.ldo, p.M, p.N, m, n, lane);
        else if (out_type == ICQ_BF16) store_rows<ICQ_BF16, NJ>(turn, acc[i], p.out, p.ldo, p.M, p.N, m, n, lane);
        else store_rows<ICQ_F16, NJ>(turn, acc[i], p.out, p.ldo, p.M, p.N, m, n, lane);
    }
}

template <typename S, int FA, int FB, bool ROWS>
int launch(const Product &p, bool pow2, int out_type, hipStream_t s) {
    const int tm = (int)((p.M + S::T - 1) / S::T), tn = (int)((p.N + S::T - 1) / S::T);
    const uint32_t blocks = (uint32_t)((int64_t)tm * tn);
    auto go = [&](auto kernel) {
        if (icq_allow_lds(reinterpret_cast<const void *>(kernel), S::LDS_BYTES, true) != hipSuccess) return ICQ_ERR_HIP;
        for (uint32_t i = 0; i < blocks; i += ICQ_PRODUCT_BLOCKS)
            hipLaunchKernelGGL(kernel, dim3(std::min(blocks - i, ICQ_PRODUCT_BLOCKS), (uint32_t)p.splits), dim3(S::THREADS), S::LDS_BYTES, s, p, tm, tn, out_type, i);
        return icq_check_launch();
    };
    if (out_type == ICQ_F32) {
        if constexpr (S::T <= 128) return go(product_kernel<S, FA, FB, ROWS, EXACT>);
        return ICQ_ERR_ARG;                                                   // (not asked for: widened fragments beside 128 accumulators do not fit the registers)
    }
    if (pow2) return go(product_kernel<S, FA, FB, ROWS, FAST_POW2>);
    return go(product_kernel<S, FA, FB, ROWS, FAST>);
}

template <typename S>
int launch_formats(const Product &p, int fa, int fb, bool rows, bool pow2, int out_type, hipStream_t s) {
    if (fa == ICQ_E4M3 && fb == ICQ_E4M3) return rows ? launch<S, ICQ_E4M3, ICQ_E4M3, true>(p, pow2, out_type, s) : launch<S, ICQ_E4M3, ICQ_E4M3, false>(p, pow2, out_type, s);
    if (fa == ICQ_E4M3) return rows ? launch<S, ICQ_E4M3, ICQ_E5M2, true>(p, pow2, out_type, s) : launch<S, ICQ_E4M3, ICQ_E5M2, false>(p, pow2, out_type, s);
    if (fb == ICQ_E4M3) return rows ? launch<S, ICQ_E5M2, ICQ_E4M3, true>(p, pow2, out_type, s) : launch<S, ICQ_E5M2, ICQ_E4M3, false>(p, pow2, out_type, s);
    return rows ? launch<S, ICQ_E5M2, ICQ_E5M2, true>(p, pow2, out_type, s) : launch<S, ICQ_E5M2, ICQ_E5M2, false>(p, pow2, out_type, s);
}

}  // namespace

int icq_launch_product_tiles(const Product &p, icq_tiles tiles, int fa, int fb, bool rows, bool pow2, int out_type, hipStream_t s) {
    if (tiles == ICQ_TILES_WIDE) return launch_formats<Wide>(p, fa, fb, rows, pow2, out_type, s);
    if (tiles == ICQ_TILES_LITTLE) return launch_formats<Little>(p, fa, fb, rows, pow2, out_type, s);
    return tiles == ICQ_TILES_DEEP ? launch_formats<Deep>(p, fa, fb, rows, pow2, out_type, s) : launch_formats<Small>(p, fa, fb, rows, pow2, out_type, s);
}
