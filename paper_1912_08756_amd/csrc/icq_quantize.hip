// Values in 8-bit floating point with one scale per block of 128.
//
// A block is 128 consecutive values of a row (of a column, for the transposed output), or a 128 x 128 tile.  With a the
// largest finite magnitude of the block (at least 2^-100) and F the format's largest value,
//     s = a / F,  or  s = 2^ceil(log2(a / F)) for scales that are powers of two,
//     code = the format's value nearest to x * (1 / s), ties to even;
// the quotients and the product are single-precision operations rounded once each.  Infinities and NaN do not count for a and
// become what the format has for them (e4m3 has no infinity: NaN).
//
// Both kernels read every value once and are bound by memory (a copy of 1 GiB runs at 5.17 TB/s).  Rows alone need no more than the 16
// lanes that hold a block agreeing on its largest value: 8192 x 8192 bf16 42 us, 4.8 TB/s; f32 57 us, 5.8 TB/s.  Columns need
// a 128 x 128 tile in registers, whose codes turn round in the LDS so that either output is written in whole 128-byte pieces:
// 8192 x 16000 bf16 both ways 117 us, 4.6 TB/s; 10007 x 4096 f32 in 128 x 128 blocks both ways 49.5 us, 5.0 TB/s.
#include "icq_eight.h"

namespace {

struct Quantize {
    const void *x;
    int64_t rows, cols, ldx;
    uint8_t *codes, *codes_t;
    int64_t ld, ld_t;
    float *scales, *scales_t;
    int across, down;          // blocks of 128 along a row, along a column
    int pow2;
};

// Magnitude's bits for the largest-value search: 0 for infinities and NaN.
__device__ __forceinline__ uint32_t size_bits(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// Scale and its reciprocal from the bits of the largest magnitude.
template <int FORMAT>
__device__ __forceinline__ void block_scale(uint32_t amax, int pow2, float &s, float &inv) {
    constexpr uint32_t least = 27u << 23;              // 2^-100
    amax = amax > least ? amax : least;
    if (pow2) {                                        // F = 1.75 * 2^8 or 1.75 * 2^15
        const uint32_t e = (amax >> 23) - (FORMAT == ICQ_E4M3 ? 8u : 15u) + ((amax & 0x7fffffu) > 0x600000u ? 1u : 0u);
        s = __uint_as_float(e << 23);
        inv = __uint_as_float((254u - e) << 23);
    } else {
        s = __uint_as_float(amax) / (FORMAT == ICQ_E4M3 ? 448.0f : 57344.0f);
        inv = 1.0f / s;
    }
}

// Eight values of row r from column c on, zero where there are none.
template <int TYPE>
__device__ __forceinline__ void load8(const Quantize &a, int64_t r, int64_t c, float *x) {
    typedef IcqElem<TYPE> E;
    const typename E::raw *p = static_cast<const typename E::raw *>(a.x) + r * a.ldx + c;
    if (c + 8 <= a.cols) {
        uint4 v[8 / E::PER];
        __builtin_memcpy(v, p, sizeof v);              // (wherever the row starts: the memory pipe takes 16 bytes from any address)
#pragma unroll
        for (int h = 0; h < 8 / E::PER; ++h) E::unpack(v[h], x + h * E::PER);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c + i < a.cols ? E::get(p[i]) : 0.0f;
    }
}

template <int FORMAT>
__device__ __forceinline__ uint2 codes8(const float *x, float inv) {
    uint2 w;
    w.x = icq_codes2<FORMAT, false>(x[0] * inv, x[1] * inv, 0);
    w.x = icq_codes2<FORMAT, true>(x[2] * inv, x[3] * inv, w.x);
    w.y = icq_codes2<FORMAT, false>(x[4] * inv, x[5] * inv, 0);
    w.y = icq_codes2<FORMAT, true>(x[6] * inv, x[7] * inv, w.y);
    return w;
}

// Rows: 16 lanes per block of 128, eight values each.
template <int TYPE, int FORMAT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(Quantize a, int64_t first_row, uint32_t tasks) {
    const uint32_t t = blockIdx.x * 16u + threadIdx.x / 16u;
    if (t >= tasks) return;
    const uint32_t row = t / (uint32_t)a.across, block = t % (uint32_t)a.across;
    const int64_t r = first_row + row, c = (int64_t)block * 128 + (threadIdx.x & 15u) * 8;
    float x[8];
    load8<TYPE>(a, r, c, x);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, size_bits(x[i]));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d, 16));
    float s, inv;
    block_scale<FORMAT>(m, a.pow2, s, inv);
    if (c < ((a.cols + 15) & ~(int64_t)15)) *reinterpret_cast<uint2 *>(a.codes + r * a.ld + c) = codes8<FORMAT>(x, inv);
    if ((threadIdx.x & 15u) == 0) a.scales[r * a.across + block] = s;
}

// Magnitudes' bits of infinities and NaN replaced by zero.
template <int TYPE>
__device__ __forceinline__ uint32_t finite_only(uint32_t m) {
    if constexpr (TYPE == ICQ_F32) return m < 0x7f800000u ? m : 0u;
    else {
        constexpr uint32_t inf = TYPE == ICQ_F16 ? 0x7c00u : 0x7f80u;
        return ((m & 0xffffu) < inf ? m & 0xffffu : 0u) | ((m >> 16) < inf ? m & 0xffff0000u : 0u);
    }
}

// The largest of 16 neighbouring lanes, in all of them.
template <int TYPE>
__device__ __forceinline__ uint32_t largest_of_16(uint32_t m) {
    m = larger<TYPE>(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x128, 0xf, 0xf, true));      // rotations by 8, 4, 2, 1 lanes
    m = larger<TYPE>(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x124, 0xf, 0xf, true));
    m = larger<TYPE>(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x122, 0xf, 0xf, true));
    return larger<TYPE>(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x121, 0xf, 0xf, true));
}

// A 128 x 128 tile per block; thread (g, h) holds rows 4 h .. 4 h + 3 of columns 8 g .. 8 g + 7.
// TILE: one scale for the whole tile, else one per row and column of it, each worked out by one thread (by all that need it, with words
// compared one by one: 139 us at 8192 x 16000 against 118; 256 threads of 8 x 8 values each: the same 118, small tiles slower).
template <int TYPE, int FORMAT, bool TILE>
__global__ __launch_bounds__(512) void quantize_tile_kernel(Quantize a, uint32_t first_tile) {
    constexpr int WORDS = Eight<TYPE>::WORDS;
    __shared__ __attribute__((aligned(16))) uint32_t s_cols[8][128];          // largest magnitudes: of a wavefront's rows in each column,
    __shared__ __attribute__((aligned(16))) uint32_t s_rows[128];             // of each row
    __shared__ __attribute__((aligned(16))) float s_inv[256];                 // the columns' reciprocal scales, then the rows'
    __shared__ __attribute__((aligned(16))) uint8_t s_turn[128][128];         // column c's 8-byte piece p at place p ^ (c / 8)
    const int tid = threadIdx.x, g = tid & 15, h = tid >> 4, wave = tid >> 6, lane = tid & 63;
    const uint32_t tile = first_tile + blockIdx.x;
    const int bc = (int)(tile % (uint32_t)a.across), br = (int)(tile / (uint32_t)a.across);
    const int64_t r0 = (int64_t)br * 128 + 4 * h, c0 = (int64_t)bc * 128 + 8 * g;
    Eight<TYPE> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = read8<TYPE>(a.x, a.rows, a.cols, a.ldx, r0 + i, c0);
    uint32_t col[WORDS], row[4];
    const auto largest = [&](auto bits) {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) col[k] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            row[i] = 0;
#pragma unroll
            for (int k = 0; k < WORDS; ++k) {
                const uint32_t m = bits(v[i].w[k]);
                col[k] = larger<TYPE>(col[k], m);
                row[i] = larger<TYPE>(row[i], m);
            }
        }
    };
    largest([](uint32_t w) { return magnitude<TYPE>(w); });
    uint32_t odd = 0;
#pragma unroll
    for (int k = 0; k < WORDS; ++k) odd |= finite_only<TYPE>(col[k]) ^ col[k];
    if (odd) largest([](uint32_t w) { return finite_only<TYPE>(magnitude<TYPE>(w)); });
    const int64_t wide = (a.cols + 15) & ~(int64_t)15, tall = (a.rows + 15) & ~(int64_t)15;
    if constexpr (TILE) {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < WORDS; ++k) m = larger<TYPE>(m, col[k]);
        m = largest_of_16<TYPE>(m);
        m = larger<TYPE>(m, (uint32_t)__shfl_xor((int)m, 16, 64));
        m = larger<TYPE>(m, (uint32_t)__shfl_xor((int)m, 32, 64));
        if (TYPE != ICQ_F32) m = max(m & 0xffffu, m >> 16);
        if (lane == 0) s_rows[wave] = m;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t m = largest_of_16<TYPE>(row[i]);
            if (TYPE != ICQ_F32) m = max(m & 0xffffu, m >> 16);
            if (g == i) s_rows[4 * h + i] = m;
        }
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            uint32_t m = larger<TYPE>(col[k], (uint32_t)__shfl_xor((int)col[k], 16, 64));
            m = larger<TYPE>(m, (uint32_t)__shfl_xor((int)m, 32, 64));
            if (lane < 16) {
                if (TYPE == ICQ_F32) s_cols[wave][8 * g + k] = m;
                else *reinterpret_cast<uint2 *>(&s_cols[wave][8 * g + 2 * k]) = make_uint2(m & 0xffffu, m >> 16);
            }
        }
    }
    __syncthreads();
    float inv_r[4], inv_c[8];
    if constexpr (TILE) {
        uint32_t m = s_rows[0];
#pragma unroll
        for (int w = 1; w < 8; ++w) m = max(m, s_rows[w]);
        float s, inv;
        block_scale<FORMAT>(float_bits<TYPE>(m), a.pow2, s, inv);
        if (tid == 0) {
            if (a.codes) a.scales[(int64_t)br * a.across + bc] = s;
            if (a.codes_t) a.scales_t[(int64_t)bc * a.down + br] = s;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) inv_r[i & 3] = inv_c[i] = inv;
    } else {
        if (tid < 256) {
            const int at = tid & 127;
            uint32_t m = tid < 128 ? s_cols[0][at] : s_rows[at];
            if (tid < 128)
#pragma unroll
                for (int w = 1; w < 8; ++w) m = max(m, s_cols[w][at]);
            float s, inv;
            block_scale<FORMAT>(float_bits<TYPE>(m), a.pow2, s, inv);
            s_inv[tid] = inv;
            const int64_t r = (int64_t)br * 128 + at, c = (int64_t)bc * 128 + at;
            if (tid < 128) {
                if (a.codes_t && c < a.cols) a.scales_t[c * a.down + br] = s;
            } else if (a.codes && r < a.rows) {
                a.scales[r * a.across + bc] = s;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            inv_c[i] = s_inv[8 * g + i];
            if (i < 4) inv_r[i] = s_inv[128 + 4 * h + i];
        }
    }
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        values8<TYPE>(v[i], x[i]);
        if (a.codes && r0 + i < a.rows && c0 < wide) *reinterpret_cast<uint2 *>(a.codes + (r0 + i) * a.ld + c0) = codes8<FORMAT>(x[i], inv_r[i]);
    }
    if (!a.codes_t) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t w = icq_codes2<FORMAT, false>(x[0][j] * inv_c[j], x[1][j] * inv_c[j], 0);
        w = icq_codes2<FORMAT, true>(x[2][j] * inv_c[j], x[3][j] * inv_c[j], w);
        *reinterpret_cast<uint32_t *>(&s_turn[8 * g + j][8 * ((h >> 1) ^ g) + 4 * (h & 1)]) = w;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int at = u * 512 + tid, c = at >> 3, piece = (at & 7) * 16;
        const int64_t out = (int64_t)bc * 128 + c, from = (int64_t)br * 128 + piece;
        if (out < a.cols && from < tall) {
            const uint4 q = *reinterpret_cast<const uint4 *>(&s_turn[c][piece ^ ((c >> 4) << 4)]);
            *reinterpret_cast<uint4 *>(a.codes_t + out * a.ld_t + from) = (c & 8) ? make_uint4(q.z, q.w, q.x, q.y) : q;
        }
    }
}

// A launch counts less than 2^32 threads: 2^31 of them at a time.
constexpr int64_t ROW_TASKS = 1ll << 27, TILES = 1ll << 22;

template <int TYPE, int FORMAT>
int launch(const Quantize &a, int block_rows, hipStream_t s) {
    if (block_rows == 1 && !a.codes_t) {
        const int64_t step = ROW_TASKS / a.across;                    // (a.across is at most 2^24)
        for (int64_t r = 0; r < a.rows; r += step) {
            const uint32_t tasks = (uint32_t)((a.rows - r < step ? a.rows - r : step) * a.across);
            hipLaunchKernelGGL(HIP_KERNEL_NAME(quantize_rows_kernel<TYPE, FORMAT>), dim3((tasks + 15u) / 16u), dim3(256), 0, s, a, r, tasks);
        }
        return icq_check_launch();
    }
    const int64_t tiles = (int64_t)a.across * a.down;
    for (int64_t t = 0; t < tiles; t += TILES) {
        const dim3 grid((uint32_t)(tiles - t < TILES ? tiles - t : TILES));
        if (block_rows == 1) hipLaunchKernelGGL(HIP_KERNEL_NAME(quantize_tile_kernel<TYPE, FORMAT, false>), grid, dim3(512), 0, s, a, (uint32_t)t);
        else hipLaunchKernelGGL(HIP_KERNEL_NAME(quantize_tile_kernel<TYPE, FORMAT, true>), grid, dim3(512), 0, s, a, (uint32_t)t);
    }
    return icq_check_launch();
}

}  // namespace

ICQ_EXPORT int icq_block_quantize(const void *x, int x_type, int64_t rows, int64_t cols, int64_t ldx, int format, int scaling,
                                  int block_rows, uint8_t *codes, int64_t ld_codes, float *scales, uint8_t *codes_t,
                                  int64_t ld_codes_t, float *scales_t, void *stream) {
    const int size = icq_type_bytes(x_type);
    if (size == 0 || (format != ICQ_E4M3 && format != ICQ_E5M2) || (scaling != ICQ_SCALES_F32 && scaling != ICQ_SCALES_POW2) ||
        (block_rows != 1 && block_rows != ICQ_BLOCK) || rows < 0 || cols < 0 || rows > ICQ_MAX_EXTENT || cols > ICQ_MAX_EXTENT ||
        (!codes && !codes_t))
        return ICQ_ERR_ARG;
    if (codes && (!scales || ld_codes < cols || ld_codes % 16 != 0 || (uintptr_t)codes % 16 != 0)) return ICQ_ERR_ARG;
    if (codes_t && (!scales_t || ld_codes_t < rows || ld_codes_t % 16 != 0 || (uintptr_t)codes_t % 16 != 0)) return ICQ_ERR_ARG;
    if (rows == 0 || cols == 0) return ICQ_OK;
    if (!x || ldx < cols || (uintptr_t)x % size != 0) return ICQ_ERR_ARG;
    Quantize a;
    a.x = x; a.rows = rows; a.cols = cols; a.ldx = ldx;
    a.codes = codes; a.ld = ld_codes; a.scales = scales;
    a.codes_t = codes_t; a.ld_t = ld_codes_t; a.scales_t = scales_t;
    a.across = (int)((cols + 127) / 128);
    a.down = (int)((rows + 127) / 128);
    a.pow2 = scaling == ICQ_SCALES_POW2;
    if ((block_rows != 1 || codes_t) && (int64_t)a.across * a.down > 0x7fffffff) return ICQ_ERR_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    int rc = ICQ_OK;
    ICQ_FOR_TYPE(x_type, rc = format == ICQ_E4M3 ? launch<TYPE, ICQ_E4M3>(a, block_rows, s) : launch<TYPE, ICQ_E5M2>(a, block_rows, s))
    return rc;
}
