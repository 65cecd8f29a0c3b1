// Products of matrices in microscaled 4-bit floating point for up to 32 rows of a: reading b is all that counts.
//
// A wavefront has 16 NT rows of b and takes steps of 256 values: 32 bytes of codes and two scales of each row to a lane, straight from memory
// into the registers, the next step requested before the present one is multiplied.  Which 32 values of a step meet which lane is free as
// long as both operands agree: a lane's two neighbouring blocks are the operands of two instructions, so that four lanes read 128 bytes of a row.
// a's rows come from the caches the same way; as values, a lane has its two blocks whole and quantises them in its registers, which is
// little beside the loads of b and saves a launch and its wait.
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

// The 64 values of a row from c on as they lie in memory, zeros from K on.
template <int TYPE>
struct Raw {
    Eight<TYPE> v[8];
};

template <int TYPE>
__device__ __forceinline__ Blocks quantised(const Raw<TYPE> &x, int fit) {
    Blocks b;
    b.e = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int w = 0; w < Eight<TYPE>::WORDS; ++w) m = larger<TYPE>(m, magnitude<TYPE>(x.v[4 * h + k].w[w]));
        if constexpr (TYPE != ICQ_F32) m = float_bits<TYPE>(max(m & 0xffffu, m >> 16));
        const uint32_t byte = mx_scale_byte(m, fit);
        const float divisor = mx_divisor(byte);
        uint32_t c[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = byte == 255u ? 0u : mx_codes8<TYPE>(x.v[4 * h + k].w, divisor);
        b.v[h] = make_uint4(c[0], c[1], c[2], c[3]);
        b.e |= byte << (8 * h);
    }
    return b;
}

// TYPE: of a's values, or ICQ_E2M1 where it is held.  MT, NT: 16 rows of a, of b to a wavefront.
template <int TYPE, int MT, int NT>
__global__ __launch_bounds__(64 * WAVES) void mx_few_kernel(Few f, int out_type, uint32_t first_block) {
    constexpr bool VALUES = TYPE != ICQ_E2M1;
    constexpr int AS = VALUES ? TYPE : ICQ_F32;                               // (a type to name where there are no values)
    __shared__ icq_f32x4 s_part[WAVES / 2][NT * MT][64];
    const Product &p = f.q.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = lane & 15, quarter = lane >> 4;
    const int part = wave % f.along;
    const int64_t n0 = ((int64_t)(first_block + blockIdx.x) * (WAVES / f.along) + wave / f.along) * (16 * NT);
    const int blocks = f.q.blocks;
    const uint8_t *row_b[NT], *scale_b[NT], *row_a[MT], *scale_a[MT];
    int64_t ra[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t r = min(n0 + 16 * j + at, p.N - 1);
        row_b[j] = p.b + r * p.ldb;
        scale_b[j] = f.q.eb + r * f.q.ld_eb;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        ra[i] = min((int64_t)(16 * i + at), p.M - 1);
        if (!VALUES) {
            row_a[i] = p.a + ra[i] * p.lda;
            scale_a[i] = f.q.ea + ra[i] * f.q.ld_ea;
        }
    }
    struct Operand { Blocks b[NT]; };
    Blocks a[MT];
    Raw<AS> raw[VALUES ? MT : 1];
    auto load_b = [&](Operand &o, int step) {
#pragma unroll
        for (int j = 0; j < NT; ++j) o.b[j] = held_blocks(row_b[j], scale_b[j], blocks, 8 * step + 2 * quarter);
    };
    auto load_a = [&](int step) {
        const int64_t c = (int64_t)step * 256 + 64 * quarter;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if constexpr (VALUES) {
#pragma unroll
                for (int k = 0; k < 8; ++k) raw[i].v[k] = read8<AS>(f.x, p.M, p.K, f.ldx, ra[i], c + 8 * k);
            } else {
                a[i] = held_blocks(row_a[i], scale_a[i], blocks, 8 * step + 2 * quarter);
                if (c + 64 > p.K)                                             // (zero in a: what b holds there does not matter)
#pragma unroll
                    for (int h = 0; h < 2; ++h) a[i].v[h] = first_codes(a[i].v[h], (int)min(max(p.K - c - 32 * h, (int64_t)0), (int64_t)32));
            }
        }
    };
    auto take_a = [&]() {
        if constexpr (VALUES)
#pragma unroll
            for (int i = 0; i < MT; ++i) a[i] = quantised<AS>(raw[i], f.fit);
    };
    icq_f32x4 acc[MT][NT] = {};
    auto multiply = [&](const Operand &o) {
        auto codes = [](const uint4 &v) {
            icq_i32x8 r = {(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
            return r;
        };
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes(o.b[j].v[0]), codes(a[i].v[0]), acc[i][j], 4, 4, 0, (int)o.b[j].e, 0, (int)a[i].e);
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes(o.b[j].v[1]), codes(a[i].v[1]), acc[i][j], 4, 4, 1, (int)o.b[j].e, 1, (int)a[i].e);
            }
    };
    Operand even, odd;
    const int end = min(p.kb, ((int)blockIdx.y + 1) * p.per), by = f.along;
    int step = blockIdx.y * p.per + part;
    if (step < end && n0 < p.N) {
        load_b(even, step);
        load_a(step);
        for (;;) {
            take_a();
            if (step + by < end) load_b(odd, step + by);
            multiply(even);
            if ((step += by) >= end) break;
            load_a(step);
            take_a();
            if (step + by < end) load_b(even, step + by);
            multiply(odd);
            if ((step += by) >= end) break;
            load_a(step);
        }
    }
    // the parts' sums: halves onto halves
    for (int h = f.along / 2; h > 0; h >>= 1) {
        const int place = wave / f.along * (f.along / 2);
        __syncthreads();
        if (part >= h && part < 2 * h) {
#pragma unroll
            for (int t = 0; t < NT * MT; ++t) s_part[place + part - h][t][lane] = acc[t % MT][t / MT];
        }
        __syncthreads();
        if (part < h) {
#pragma unroll
            for (int t = 0; t < NT * MT; ++t) acc[t % MT][t / MT] += s_part[place + part][t][lane];
        }
    }
    if (part != 0) return;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = 16 * i + at;
        if (m >= p.M) continue;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t n = n0 + 16 * j + 4 * quarter;
            if (p.splits > 1) store_part(p, blockIdx.y, m, n, acc[i][j]);
            else if (out_type == ICQ_F32) store4<ICQ_F32>(p, m, n, acc[i][j]);
            else if (out_type == ICQ_BF16) store4<ICQ_BF16>(p, m, n, acc[i][j]);
            else store4<ICQ_F16>(p, m, n, acc[i][j]);
        }
    }
}

template <int TYPE>
int launch(const Few &f, bool wide, int out_type, hipStream_t s) {
    const Product &p = f.q.p;
    auto go = [&](auto kernel, int nt) {
        const int64_t rows = (int64_t)16 * nt * (WAVES / f.along);
        const uint32_t blocks = (uint32_t)((p.N + rows - 1) / rows);
        for (uint32_t i = 0; i < blocks; i += ICQ_PRODUCT_BLOCKS)
            hipLaunchKernelGGL(kernel, dim3(std::min(blocks - i, ICQ_PRODUCT_BLOCKS), (uint32_t)p.splits), dim3(64 * WAVES), 0, s, f, out_type, i);
    };
    if (p.M > 16) go(mx_few_kernel<TYPE, 2, 1>, 1);
    else if (wide) go(mx_few_kernel<TYPE, 1, 4>, 4);
    else go(mx_few_kernel<TYPE, 1, 1>, 1);
    return icq_check_launch();
}

}  // namespace

int icq_launch_mx_few(const MxProduct &q, const icq_mx_plan &plan, const void *x, int a_type, int64_t ldx, bool fit, int out_type, hipStream_t s) {
    Few f;
    f.q = q;
    f.x = x; f.ldx = ldx; f.fit = fit; f.along = plan.along;
    if (a_type == ICQ_E2M1) return launch<ICQ_E2M1>(f, plan.wide, out_type, s);
    int rc = ICQ_OK;
    ICQ_FOR_TYPE(a_type, rc = launch<TYPE>(f, plan.wide, out_type, s))
    return rc;
}
