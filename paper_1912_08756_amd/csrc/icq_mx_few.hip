// Products of matrices in microscaled 4-bit floating point for up to 16 rows of a: reading b is all that counts.
//
// A wavefront has 16 NT rows of b and takes steps of 256 values: 32 bytes of codes and two scales of each row to a lane, straight from memory
// into the registers, the next step's requested before the present one's are multiplied, also from one group of rows to the next.
// Which 32 values of a step meet which lane is free as long as both operands agree: a lane's two neighbouring blocks are the operands of
// two instructions, so that four lanes read 128 bytes of a row.
// a as values: each block quantises the part it needs into the LDS, behind its first requests of b; that saves a launch and its wait.
// A block's eight wavefronts share rows of b in `along` parts of the contraction, whose sums meet in the LDS, in a fixed order.
#include "icq_eight.h"
#include "icq_mx.h"

#include <algorithm>

namespace {

constexpr int WAVES = ICQ_MX_FEW_WAVES;

struct Few {
    MxProduct q;
    const void *x;             // a as values, rows ldx apart
    int64_t ldx;
    int fit, along;
};

// Two blocks of 32 codes and their scales in the two low bytes.
struct Blocks {
    uint4 v[2];
    uint32_t e;
};

// What a held row has for this lane in step s: its blocks 8 s + 2 quarter and the next; beyond the row's end any codes under the scale 1.
__device__ __forceinline__ Blocks held_blocks(const uint8_t *row, const uint8_t *scales, int blocks, int first) {
    Blocks b;
    const int left = blocks - first;
    b.v[0] = *reinterpret_cast<const uint4 *>(row + (left > 0 ? (int64_t)first * 16 : 0));
    b.v[1] = *reinterpret_cast<const uint4 *>(row + (left > 1 ? (int64_t)first * 16 + 16 : 0));
    b.e = *reinterpret_cast<const uint16_t *>(scales + (left > 0 ? first : 0));
    if (left < 2) b.e = left > 0 ? (b.e & 0xffu) | 0x7f00u : 0x7f7fu;
    return b;
}

// TYPE: of a's values, or ICQ_E2M1 where it is held.  NT: 16 rows of b to a wavefront.
template <int TYPE, int NT>
__global__ __launch_bounds__(64 * WAVES, 4) void mx_few_kernel(Few f, int out_type, int64_t tiles) {
    constexpr bool VALUES = TYPE != ICQ_E2M1;
    __shared__ icq_f32x4 s_part[WAVES / 2][NT][64];
    extern __shared__ __attribute__((aligned(16))) uint8_t s_a[];             // steps' codes [piece][row] of 16 bytes, then their scales [row] of 8 bytes
    const Product &p = f.q.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = lane & 15, quarter = lane >> 4;
    const int part = wave % f.along, by = f.along, blocks = f.q.blocks;
    const int begin = blockIdx.y * p.per, end = min(p.kb, begin + p.per);
    const int ra = (int)min((int64_t)at, p.M - 1);                            // this lane's row of a: beyond M again M - 1's
    const uint8_t *row_a = VALUES ? nullptr : p.a + ra * p.lda, *scale_a = VALUES ? nullptr : f.q.ea + ra * f.q.ld_ea;

    struct Operand { Blocks b[NT], a; };                                      // (a: where it is held)
    // rows of b of the tile under way; of the one whose steps are requested
    int64_t tile = blockIdx.x, n0 = 0;
    const uint8_t *row_b[NT], *scale_b[NT];
    auto first_row = [&](int64_t t) { return (t * (WAVES / f.along) + wave / f.along) * (16 * NT); };
    auto point = [&](int64_t t) {
        const int64_t n = first_row(t);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t r = min(n + 16 * j + at, p.N - 1);
            row_b[j] = p.b + r * p.ldb;
            scale_b[j] = f.q.eb + r * f.q.ld_eb;
        }
    };
    auto request = [&](Operand &o, int step) {
#pragma unroll
        for (int j = 0; j < NT; ++j) o.b[j] = held_blocks(row_b[j], scale_b[j], blocks, 8 * step + 2 * quarter);
        if constexpr (!VALUES) o.a = held_blocks(row_a, scale_a, blocks, 8 * step + 2 * quarter);
    };
    auto blocks_of_a = [&](const Operand &o, int step) {
        Blocks a;
        if constexpr (VALUES) {
            const uint8_t *from = s_a + (step - begin) * 2048;
            a.v[0] = *reinterpret_cast<const uint4 *>(from + (2 * quarter * 16 + ra) * 16);
            a.v[1] = *reinterpret_cast<const uint4 *>(from + ((2 * quarter + 1) * 16 + ra) * 16);
            a.e = *reinterpret_cast<const uint16_t *>(s_a + (end - begin) * 2048 + (step - begin) * 128 + ra * 8 + 2 * quarter);
        } else {
            const int64_t c = (int64_t)step * 256 + 64 * quarter;
            a = o.a;
            if (c + 64 > p.K)                                                 // (zero in a: what b holds there does not matter)
#pragma unroll
                for (int h = 0; h < 2; ++h) a.v[h] = first_codes(a.v[h], (int)min(max(p.K - c - 32 * h, (int64_t)0), (int64_t)32));
        }
        return a;
    };
    Operand even, odd;
    const bool some = begin + part < end;                                     // this wavefront has steps
    if (some) {
        point(tile);
        request(even, begin + part);
    }
    n0 = first_row(tile);
    if constexpr (VALUES) {
        // four neighbouring threads have a block, eight values each
        const int pieces = (end - begin) * 8 * 4, rows = (int)p.M;
        for (int i = threadIdx.x; i < rows * pieces; i += 64 * WAVES) {
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
            *reinterpret_cast<uint32_t *>(s_a + (block * 16 + r) * 16 + (k & 3) * 4) = codes;
            if ((k & 3) == 0) s_a[(end - begin) * 2048 + (block >> 3) * 128 + r * 8 + (block & 7)] = (uint8_t)byte;
        }
        __syncthreads();
    }
    icq_f32x4 acc[NT] = {};
    int step = begin + part;
    // multiplies the step that `now` holds, with the next one's requests into `then`; false after the last
    auto advance = [&](const Operand &now, Operand &then) {
        const bool last = step + by >= end, more = tile + gridDim.x < tiles;
        if (some) {
            if (last && more) point(tile + gridDim.x);
            if (!last || more) request(then, last ? begin + part : step + by);
            const Blocks a = blocks_of_a(now, step);
            auto codes = [](const uint4 &v) {
                icq_i32x8 r = {(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
                return r;
            };
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes(now.b[j].v[0]), codes(a.v[0]), acc[j], 4, 4, 0, (int)now.b[j].e, 0, (int)a.e);
                acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes(now.b[j].v[1]), codes(a.v[1]), acc[j], 4, 4, 1, (int)now.b[j].e, 1, (int)a.e);
            }
        }
        step += by;
        if (!last) return true;
        // the parts' sums: halves onto halves
        for (int h = by / 2; h > 0; h >>= 1) {
            const int place = wave / by * (by / 2);
            if (part >= h && part < 2 * h) {
#pragma unroll
                for (int j = 0; j < NT; ++j) s_part[place + part - h][j][lane] = acc[j];
            }
            __syncthreads();
            if (part < h) {
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[j] += s_part[place + part][j][lane];
            }
            __syncthreads();
        }
        if (part == 0 && at < p.M) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int64_t n = n0 + 16 * j + 4 * quarter;
                if (p.splits > 1) store_part(p, blockIdx.y, at, n, acc[j]);
                else if (out_type == ICQ_F32) store4<ICQ_F32>(p, at, n, acc[j]);
                else if (out_type == ICQ_BF16) store4<ICQ_BF16>(p, at, n, acc[j]);
                else store4<ICQ_F16>(p, at, n, acc[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] = icq_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        tile += gridDim.x;
        n0 = first_row(tile);
        step = begin + part;
        return more;
    };
    // (wavefronts of a block have a different number of steps by one at most: one that has done its last waits in the reduction, as often as the others)
    while (advance(even, odd) && advance(odd, even)) {}
}

template <int TYPE>
int launch(const Few &f, bool wide, int num_cu, int out_type, hipStream_t s) {
    const Product &p = f.q.p;
    const int lds = TYPE == ICQ_E2M1 ? 0 : std::min(p.kb, p.per) * (2048 + 128);
    auto go = [&](auto kernel, int nt) {
        if (lds > 0 && icq_allow_lds(reinterpret_cast<const void *>(kernel), lds) != hipSuccess) return ICQ_ERR_HIP;
        const int64_t rows = (int64_t)16 * nt * (WAVES / f.along), tiles = (p.N + rows - 1) / rows;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)std::min<int64_t>(tiles, 2 * num_cu), (uint32_t)p.splits), dim3(64 * WAVES), lds, s, f, out_type, tiles);
        return icq_check_launch();
    };
    return wide ? go(mx_few_kernel<TYPE, 2>, 2) : go(mx_few_kernel<TYPE, 1>, 1);
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
