// Products of matrices in microscaled 4-bit floating point for up to 16 rows of a: reading b is all that counts.
//
// A wavefront has 16 NT rows of b and takes steps of 256 values: their codes and scales go from memory straight into its own part of the LDS, DEPTH steps
// ahead, also from one group of rows to the next, and from there into matrix instructions; nobody else reads them, so there is no barrier in the
// loop.  Which 32 values of a step meet which lane is free as long as both operands agree: a lane's two neighbouring blocks are the operands of
// two instructions.  a lies in the LDS whole: values are quantised by each block behind its first requests of b, which saves a launch and
// its wait.  A block's eight wavefronts share rows of b in `along` parts of the contraction, whose sums meet in the LDS, in a fixed order.
//
// Bound by memory: 8 x 1000000 x 960 into f32 108 us, 5.0 TB/s of b's codes and scales and of the results (a copy 5.1); 8 x 100000 x 2048, which the last-level
// cache holds, 20.5; 1 x 16384 x 4096 over the same memory 7.0 held or as values, over other memory each time 9.2 and 9.4.  Requests into
// registers instead, one step ahead, were bound by the lines that the first-level cache holds under way, scales' among them: 27.4 for 8 x 100000 x 2048
// (20 without scales, 38 two steps ahead; through the LDS 19.9 then).
#include "icq_eight.h"
#include "icq_mx.h"
#include "icq_tiles.h"

#include <algorithm>

namespace {

constexpr int WAVES = ICQ_MX_FEW_WAVES;

struct Few {
    MxProduct q;
    const void *x;             // a as values, rows ldx apart
    int64_t ldx;
    int fit, along;
};

// Bytes of a's steps in the LDS.
__host__ __device__ constexpr int held_bytes(int steps, int rows) { return (steps * rows * 136 + 15) & ~15; }

// TYPE: of a's values, or ICQ_E2M1 where it is held.  NT: 16 rows of b to a wavefront.  DEPTH: steps in the LDS.
template <int TYPE, int NT, int DEPTH>
__global__ __launch_bounds__(64 * WAVES, 2) void mx_few_kernel(Few f, int out_type, int64_t tiles) {
    constexpr bool VALUES = TYPE != ICQ_E2M1;
    constexpr int LOADS = 2 * NT + 1, CODES = NT * 2048, STAGE = CODES + 256;  // of a wavefront's step: requests, bytes of codes, with scales
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];          // the wavefronts' steps; a: steps' codes [piece][row] of 16 bytes, steps' scales [row] of 8 bytes; parts' sums
    const Product &p = f.q.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), at = lane & 15, quarter = lane >> 4;
    const int by = f.along, part = wave % by, blocks = f.q.blocks, words = (blocks + 3) >> 2;
    const int begin = blockIdx.y * p.per, end = min(p.kb, begin + p.per), steps = end - begin, rows = (int)p.M;
    const int ra = min(at, rows - 1);                                         // this lane's row of a: beyond M again M - 1's
    const int whole = (int)(p.K / 256), ragged = (int)(p.K % 256);
    uint8_t *const s_a = smem + WAVES * DEPTH * STAGE, *const s_scales = s_a + steps * rows * 128;
    icq_f32x4 *const s_part = reinterpret_cast<icq_f32x4 *>(smem + WAVES * DEPTH * STAGE + held_bytes(p.per, rows)) + quarter * rows + ra;   // [place][16 rows of b][quarter][row of a]
    const uint32_t mine = (uint32_t)(wave * DEPTH * STAGE);                   // (there is no other LDS: smem is at 0)

    // Requests, of a tile and step that run ahead: instruction i brings rows 8 i .. + 7, row r's piece c to place c ^ (r / 2 % 8), so that 16 rows' pieces fall on all
    // banks; the last one the rows' two words of scales.  Pieces beyond a row's end are taken from its beginning.
    int64_t asked = begin + part < end ? (int64_t)blockIdx.x : tiles;
    int asked_step = begin + part, asked_slot = 0;
    const uint8_t *row_b = nullptr, *scale_b = nullptr;
    uint32_t off_b[2 * NT], off_e = 0;
    auto first_row = [&](int64_t t) { return (t * (WAVES / by) + wave / by) * (16 * NT); };
    auto piece_of = [&](int i) { return (lane & 7) ^ ((4 * i + (lane >> 4)) & 7); };
    auto aim = [&]() {
        const int64_t n = min(first_row(asked), p.N - 1);
        row_b = p.b + n * p.ldb;
        scale_b = f.q.eb + n * f.q.ld_eb;
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) off_b[i] = (uint32_t)(min((int64_t)(8 * i + (lane >> 3)), p.N - 1 - n) * p.ldb) + piece_of(i) * 16;
        off_e = (uint32_t)(min((int64_t)(lane >> 1 & (16 * NT - 1)), p.N - 1 - n) * f.q.ld_eb);
    };
    auto ask = [&]() {
        if (asked >= tiles) return;
        const uint32_t to = mine + asked_slot * STAGE;
        const i32x4 codes = bytes_from(row_b), scales = bytes_from(scale_b);
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) load_to_lds(codes, off_b[i] - (asked_step == whole && piece_of(i) * 32 >= ragged ? piece_of(i) * 16 : 0), asked_step * 128, to + i * 1024);
        load_word_to_lds(scales, off_e + min(2 * asked_step + (lane & 1), words - 1) * 4, 0, to + CODES);
        asked_slot = (asked_slot + 1) & (DEPTH - 1);
        if ((asked_step += by) < end) return;
        asked_step = begin + part;
        if ((asked += gridDim.x) < tiles) aim();
    };
    if (asked < tiles) aim();
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) ask();
    if constexpr (VALUES) {
        // four neighbouring threads have a block, eight values each
        const int pieces = steps * 8 * 4;
        for (int i = tid; i < rows * pieces; i += 64 * WAVES) {
            const int r = i / pieces, k = i % pieces;
            const Eight<TYPE> x = read8<TYPE>(f.x, p.M, p.K, f.ldx, r, (int64_t)begin * 256 + 8 * k);
            uint32_t m = magnitude<TYPE>(x.w[0]);
#pragma unroll
            for (int w = 1; w < Eight<TYPE>::WORDS; ++w) m = larger<TYPE>(m, magnitude<TYPE>(x.w[w]));
            m = larger<TYPE>(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, true));
            m = larger<TYPE>(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, true));
            if constexpr (TYPE != ICQ_F32) m = float_bits<TYPE>(max(m & 0xffffu, m >> 16));
            const uint32_t byte = mx_scale_byte(m, f.fit), codes = byte == 255u ? 0u : mx_codes8<TYPE>(x.w, mx_divisor(byte));
            const int block = k >> 2;
            *reinterpret_cast<uint32_t *>(s_a + (block * rows + r) * 16 + (k & 3) * 4) = codes;
            if ((k & 3) == 0) s_scales[((block >> 3) * rows + r) * 8 + (block & 7)] = (uint8_t)byte;
        }
    } else {
        const int pieces = steps * 8;
        for (int i = tid; i < rows * pieces; i += 64 * WAVES) {
            const int r = i / pieces, k = i % pieces, block = begin * 8 + k;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (block < blocks) v = first_codes(*reinterpret_cast<const uint4 *>(p.a + r * p.lda + (int64_t)block * 16), (int)min(p.K - (int64_t)block * 32, (int64_t)32));
            *reinterpret_cast<uint4 *>(s_a + (k * rows + r) * 16) = v;
            s_scales[((k >> 3) * rows + r) * 8 + (k & 7)] = block < blocks ? f.q.ea[r * f.q.ld_ea + block] : (uint8_t)127;
        }
    }
    __syncthreads();
    int slot = 0;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        icq_f32x4 acc[NT] = {};
        for (int step = begin + part; step < end; step += by) {
            // the step's requests have arrived when as many are left as came after them (stores among them make the wait longer, never shorter)
            if (asked < tiles) __builtin_amdgcn_s_waitcnt(loads_left((DEPTH - 1) * LOADS));
            else __builtin_amdgcn_s_waitcnt(loads_left(0));
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_sched_barrier(0);
            const uint8_t *stage = smem + mine + slot * STAGE, *of_a = s_a + (step - begin) * rows * 128 + ra * 16;
            uint4 b[NT][2], a[2];
            uint32_t eb[NT];
            const uint32_t ea = *reinterpret_cast<const uint16_t *>(s_scales + ((step - begin) * rows + ra) * 8 + 2 * quarter);
#pragma unroll
            for (int h = 0; h < 2; ++h) a[h] = *reinterpret_cast<const uint4 *>(of_a + (2 * quarter + h) * rows * 16);
            const int left = blocks - 8 * step - 2 * quarter;                 // beyond the row's end the scale 1
#pragma unroll
            for (int j = 0; j < NT; ++j) {
#pragma unroll
                for (int h = 0; h < 2; ++h) b[j][h] = *reinterpret_cast<const uint4 *>(stage + (16 * j + at) * 128 + (((2 * quarter + h) ^ (at >> 1 & 7)) << 4));
                eb[j] = *reinterpret_cast<const uint16_t *>(stage + CODES + (16 * j + at) * 8 + 2 * quarter);
                eb[j] = left >= 2 ? eb[j] : left > 0 ? (eb[j] & 0xffu) | 0x7f00u : 0x7f7fu;
            }
            __builtin_amdgcn_s_waitcnt(0xc07f);                               // (all LDS reads are done: the place may be written)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_sched_barrier(0);
            ask();
            auto codes = [](const uint4 &v) {
                icq_i32x8 r = {(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
                return r;
            };
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes(b[j][0]), codes(a[0]), acc[j], 4, 4, 0, (int)eb[j], 0, (int)ea);
                acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes(b[j][1]), codes(a[1]), acc[j], 4, 4, 1, (int)eb[j], 1, (int)ea);
            }
            slot = (slot + 1) & (DEPTH - 1);
        }
        // the parts' sums: halves onto halves
        for (int h = by / 2; h > 0; h >>= 1) {
            const int place = wave / by * (by / 2);
            if (part >= h && part < 2 * h && at < rows) {
#pragma unroll
                for (int j = 0; j < NT; ++j) s_part[((place + part - h) * NT + j) * 4 * rows] = acc[j];
            }
            __syncthreads();
            if (part < h) {
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[j] += s_part[((place + part) * NT + j) * 4 * rows];
            }
            __syncthreads();
        }
        if (part == 0 && at < p.M) {
            const int64_t n0 = first_row(tile);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int64_t n = n0 + 16 * j + 4 * quarter;
                if (p.splits > 1) store_part(p, blockIdx.y, at, n, acc[j]);
                else if (out_type == ICQ_F32) store4<ICQ_F32>(p, at, n, acc[j]);
                else if (out_type == ICQ_BF16) store4<ICQ_BF16>(p, at, n, acc[j]);
                else store4<ICQ_F16>(p, at, n, acc[j]);
            }
        }
    }
}

template <int TYPE>
int launch(const Few &f, bool wide, int num_cu, int out_type, hipStream_t s) {
    const Product &p = f.q.p;
    const auto lds = [&](int nt, int depth) { return WAVES * depth * (nt * 2048 + 256) + held_bytes(p.per, (int)p.M) + (f.along > 1 ? WAVES / 2 * nt * 64 * (int)p.M : 0); };
    const auto tiles = [&](int nt) { const int64_t rows = (int64_t)16 * nt * (WAVES / f.along); return (p.N + rows - 1) / rows; };
    const auto go = [&](auto kernel, int nt, int depth) {
        const int bytes = lds(nt, depth);
        if (icq_allow_lds(reinterpret_cast<const void *>(kernel), bytes, true) != hipSuccess) return ICQ_ERR_HIP;
        const int64_t room = (int64_t)num_cu * (2 * bytes <= ICQ_MX_FEW_LDS ? 2 : 1);
        hipLaunchKernelGGL(kernel, dim3((uint32_t)std::min(tiles(nt), room), (uint32_t)p.splits), dim3(64 * WAVES), bytes, s, f, out_type, tiles(nt));
        return icq_check_launch();
    };
    // Four steps ahead where a compute unit has one block in any case (1 x 16384 x 4096: 7.3 us, two steps 7.6), two where it can have two blocks (8 x 100000 x 2048:
    // 20.4, four steps 21.3; 8 x 300000 x 512 16.7 and 18.0; 8 x 1000000 x 960 106.3 and 105.0)
    const int nt = wide ? 2 : 1;
    if (tiles(nt) * p.splits <= num_cu && lds(nt, 4) <= ICQ_MX_FEW_LDS) return wide ? go(mx_few_kernel<TYPE, 2, 4>, 2, 4) : go(mx_few_kernel<TYPE, 1, 4>, 1, 4);
    return wide ? go(mx_few_kernel<TYPE, 2, 2>, 2, 2) : go(mx_few_kernel<TYPE, 1, 2>, 1, 2);
}

}  // namespace

int icq_launch_mx_few(const MxProduct &q, const icq_mx_plan &plan, int num_cu, const void *x, int a_type, int64_t ldx, bool fit, int out_type, hipStream_t s) {
    Few f;
    f.q = q;
    f.x = x; f.ldx = ldx; f.fit = fit; f.along = plan.along;
    if (a_type == ICQ_E2M1) return launch<ICQ_E2M1>(f, plan.wide, num_cu, out_type, s);
    int rc = ICQ_OK;
    ICQ_FOR_TYPE(a_type, rc = launch<TYPE>(f, plan.wide, num_cu, out_type, s))
    return rc;
}
