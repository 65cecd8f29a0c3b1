// Values in microscaled 4-bit floating point and back: blocks of 32 values with one scale, a power of two.
//
// With a the largest magnitude of a block (at least 2^-100), its scale s is 2^(floor(log2 a) - 2) or the least power of two with a <= 6 s; both
// are read off a's bits.  x / s is exact, and one conversion rounds it to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6, ties to
// even.  A block with an infinity or a NaN: its largest magnitude's bits are those of no number; scale 255, codes 0.
//
// All three kernels read and write once and are bound by memory (a copy of 1 GiB runs at 5.12 TB/s): rows 8192 x 8192 bf16 34 us, 5.0 TB/s; tiles
// 10007 x 4096 f32 in squares both ways 46 us, 4.5 TB/s, 16384 x 16384 bf16 by rows and columns 186 us, 4.4 TB/s; values 10007 x 4096 into bf16 17 us.
// Values are read past the caches and written past them, so that codes stay: 10007 x 4096 f32 to codes both ways and back 83 us, through the
// caches 104.
#include "icq_eight.h"
#include "icq_mx.h"

namespace {

// The larger of a lane's and its neighbour's, one and two lanes away: a block of 32 is four lanes' eight values.
template <int TYPE>
__device__ __forceinline__ uint32_t largest_of_4(uint32_t m) {
    m = larger<TYPE>(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, true));
    return larger<TYPE>(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, true));
}

// The float bits of the larger half, or of the word.
template <int TYPE>
__device__ __forceinline__ uint32_t one_of(uint32_t m) {
    if constexpr (TYPE == ICQ_F32) return m;
    else return float_bits<TYPE>(max(m & 0xffffu, m >> 16));
}

template <int TYPE>
__device__ __forceinline__ uint32_t largest8(const Eight<TYPE> &v) {
    uint32_t m = magnitude<TYPE>(v.w[0]);
#pragma unroll
    for (int k = 1; k < Eight<TYPE>::WORDS; ++k) m = larger<TYPE>(m, magnitude<TYPE>(v.w[k]));
    return m;
}

// Rows: 16 lanes per 128 values, eight each.
template <int TYPE>
__global__ __launch_bounds__(256) void mx_rows_kernel(MxQuantize a, int64_t first_row, uint32_t tasks) {
    const uint32_t t = blockIdx.x * 16u + threadIdx.x / 16u, at = threadIdx.x & 15u;
    if (t >= tasks) return;
    const uint32_t row = t / (uint32_t)a.across, group = t % (uint32_t)a.across;
    const int64_t r = first_row + row, c = (int64_t)group * 128 + at * 8;
    const Eight<TYPE> v = read8<TYPE, true>(a.x, a.rows, a.cols, a.ldx, r, c);
    const uint32_t byte = mx_scale_byte(one_of<TYPE>(largest_of_4<TYPE>(largest8(v))), a.fit);
    const uint32_t codes = byte == 255u ? 0u : mx_codes8<TYPE>(v.w, mx_divisor(byte));
    const int64_t wide = (a.cols + 31) & ~(int64_t)31;
    if (c < wide) *reinterpret_cast<uint32_t *>(a.codes + r * a.ld + c / 2) = codes;
    uint32_t scales = (c < wide ? byte : 0u) << (8u * (at >> 2));
    scales |= (uint32_t)__builtin_amdgcn_mov_dpp((int)scales, 0x124, 0xf, 0xf, true);          // the four blocks' bytes: lanes 4 apart, then 8
    scales |= (uint32_t)__builtin_amdgcn_mov_dpp((int)scales, 0x128, 0xf, 0xf, true);
    if (at == 0) *reinterpret_cast<uint32_t *>(a.scales + r * a.ld_s + group * 4) = scales;
}

// Tiles are taken four rows of them at a time, so that lines of the transposed codes, which two tiles one above the other share, are written whole too
// (16384 x 16384 bf16 both ways, 1, 2, 4, 8 rows: 223, 197, 186, 214 us).
constexpr uint32_t HIGH = 4;

// A 128 x 128 tile per block; a wavefront has 32 rows of it, lane (g, h) rows 8 h .. 8 h + 7 of them in columns 8 g .. 8 g + 7, so that a
// block along a row is four neighbouring lanes' and one down a column four lanes' 16 apart.
// SQUARE: one scale for each 32 x 32.
template <int TYPE, bool SQUARE>
__global__ __launch_bounds__(256) void mx_tile_kernel(MxQuantize a, uint32_t first_tile, uint32_t tiles) {
    constexpr int WORDS = Eight<TYPE>::WORDS;
    __shared__ __attribute__((aligned(16))) uint8_t s_turn[128 * 80];          // columns' 64 bytes of codes, 16 bytes apart: column 8 g + j at place 16 j + g
    __shared__ uint8_t s_rows[128 * 4], s_cols[128 * 4];                       // scales: of the tile's rows, of its columns
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane & 15, h = lane >> 4;
    // XCD blockIdx % 8 takes a contiguous share of the launch's tiles: neighbours' halves of a line of codes, and their scales, meet in one cache
    const uint32_t xcd = blockIdx.x % 8, q8 = tiles / 8, r8 = tiles % 8;
    const uint32_t tile = first_tile + xcd * q8 + min(xcd, r8) + blockIdx.x / 8;
    const uint32_t band = tile / (HIGH * (uint32_t)a.across), in = tile % (HIGH * (uint32_t)a.across), high = min(HIGH, (uint32_t)a.down - HIGH * band);
    const int bc = (int)(in / high), br = (int)(HIGH * band + in % high);
    const int64_t r0 = (int64_t)br * 128 + 32 * wave + 8 * h, c0 = (int64_t)bc * 128 + 8 * g;
    const int64_t wide = (a.cols + 31) & ~(int64_t)31, tall = (a.rows + 31) & ~(int64_t)31;
    Eight<TYPE> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = read8<TYPE, true>(a.x, a.rows, a.cols, a.ldx, r0 + i, c0);
    uint32_t rows[8], cols[8];                                                 // scale bytes of this lane's rows and columns
    if constexpr (SQUARE) {
        uint32_t m = largest8(v[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) m = larger<TYPE>(m, largest8(v[i]));
        m = largest_of_4<TYPE>(m);
        m = larger<TYPE>(m, (uint32_t)__shfl_xor((int)m, 16, 64));
        m = larger<TYPE>(m, (uint32_t)__shfl_xor((int)m, 32, 64));
        const uint32_t byte = mx_scale_byte(one_of<TYPE>(m), a.fit);
#pragma unroll
        for (int i = 0; i < 8; ++i) rows[i] = cols[i] = byte;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) rows[i] = mx_scale_byte(one_of<TYPE>(largest_of_4<TYPE>(largest8(v[i]))), a.fit);
        if (a.codes_t) {
#pragma unroll
            for (int k = 0; k < WORDS; ++k) {
                uint32_t m = magnitude<TYPE>(v[0].w[k]);
#pragma unroll
                for (int i = 1; i < 8; ++i) m = larger<TYPE>(m, magnitude<TYPE>(v[i].w[k]));
                m = larger<TYPE>(m, (uint32_t)__shfl_xor((int)m, 16, 64));
                m = larger<TYPE>(m, (uint32_t)__shfl_xor((int)m, 32, 64));
                if constexpr (TYPE == ICQ_F32) cols[k] = mx_scale_byte(m, a.fit);
                else {
                    cols[2 * k] = mx_scale_byte(float_bits<TYPE>(m & 0xffffu), a.fit);
                    cols[2 * k + 1] = mx_scale_byte(float_bits<TYPE>(m >> 16), a.fit);
                }
            }
        }
    }
    if (a.codes) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t codes = rows[i] == 255u ? 0u : mx_codes8<TYPE>(v[i].w, mx_divisor(rows[i]));
            if (r0 + i < a.rows && c0 < wide) *reinterpret_cast<uint32_t *>(a.codes + (r0 + i) * a.ld + c0 / 2) = codes;
            if ((g & 3) == 0) s_rows[(32 * wave + 8 * h + i) * 4 + (g >> 2)] = (uint8_t)(c0 < wide ? rows[i] : 0u);
        }
    }
    if (a.codes_t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t codes = 0u;
            const float divisor = mx_divisor(cols[j]);
            const auto pair = [&](int i, uint32_t *w) {                        // rows i and i + 1 of column j
                if constexpr (TYPE == ICQ_F32) { w[0] = v[i].w[j]; w[1] = v[i + 1].w[j]; }
                else w[0] = __builtin_amdgcn_perm(v[i + 1].w[j >> 1], v[i].w[j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
            };
            uint32_t w[2];
            pair(0, w); codes = mx_codes2<TYPE, 0>(w, divisor, codes);
            pair(2, w); codes = mx_codes2<TYPE, 1>(w, divisor, codes);
            pair(4, w); codes = mx_codes2<TYPE, 2>(w, divisor, codes);
            pair(6, w); codes = mx_codes2<TYPE, 3>(w, divisor, codes);
            *reinterpret_cast<uint32_t *>(s_turn + (16 * j + g) * 80 + wave * 16 + h * 4) = cols[j] == 255u ? 0u : codes;
            if (h == 0) s_cols[(8 * g + j) * 4 + wave] = (uint8_t)((int64_t)br * 128 + 32 * wave < tall ? cols[j] : 0u);
        }
    }
    __syncthreads();
    if (a.codes && tid < 128 && (int64_t)br * 128 + tid < a.rows)
        *reinterpret_cast<uint32_t *>(a.scales + ((int64_t)br * 128 + tid) * a.ld_s + bc * 4) = *reinterpret_cast<const uint32_t *>(s_rows + tid * 4);
    if (!a.codes_t) return;
    if (tid >= 128 && (int64_t)bc * 128 + tid - 128 < a.cols)
        *reinterpret_cast<uint32_t *>(a.scales_t + ((int64_t)bc * 128 + tid - 128) * a.ld_st + br * 4) = *reinterpret_cast<const uint32_t *>(s_cols + (tid - 128) * 4);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int at = u * 256 + tid, place = at >> 2, piece = at & 3;
        const int64_t c = (int64_t)bc * 128 + 8 * (place & 15) + (place >> 4), from = (int64_t)br * 128 + 32 * piece;
        if (c < a.cols && from < tall) *reinterpret_cast<uint4 *>(a.codes_t + c * a.ld_t + from / 2) = *reinterpret_cast<const uint4 *>(s_turn + place * 80 + piece * 16);
    }
}

struct MxValues {
    const uint8_t *codes, *scales;
    int64_t ld, ld_s, rows, cols;
    void *out;
    int64_t ldo;
    int across;                // groups of 128 along a row
};

// 16 lanes per 128 values, eight each.
template <int TYPE>
__global__ __launch_bounds__(256) void mx_values_kernel(MxValues a, int64_t first_row, uint32_t tasks) {
    typedef IcqElem<TYPE> E;
    typedef typename E::raw raw;
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const uint32_t t = blockIdx.x * 16u + threadIdx.x / 16u, at = threadIdx.x & 15u;
    if (t >= tasks) return;
    const uint32_t row = t / (uint32_t)a.across, group = t % (uint32_t)a.across;
    const int64_t r = first_row + row, c = (int64_t)group * 128 + at * 8;
    if (c >= a.cols) return;
    const uint32_t codes = *reinterpret_cast<const uint32_t *>(a.codes + r * a.ld + c / 2);
    const float scale = mx_scale(a.scales[r * a.ld_s + c / 32]);
    const f32x2 q[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3)};
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = q[i >> 1][i & 1] * scale;
    raw *to = static_cast<raw *>(a.out) + r * a.ldo + c;
    if (c + 8 <= a.cols) {
#pragma unroll
        for (int k = 0; k < 8 / E::PER; ++k) {
            const uint4 w = E::pack(x + k * E::PER);
            icq_u32x4 q;
            __builtin_memcpy(&q, &w, 16);
            __builtin_nontemporal_store(q, reinterpret_cast<icq_u32x4 *>(to) + k);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < a.cols) to[i] = E::put(x[i]);
    }
}

// A launch counts less than 2^32 threads: 2^31 of them at a time.
constexpr int64_t ROW_TASKS = 1ll << 27, TILES = 1ll << 23;

// go(first row, tasks) over rows of `across` groups of 128.
template <typename F>
void for_rows(int64_t rows, int across, F go) {
    const int64_t step = ROW_TASKS / across;                                   // (across is at most 2^24)
    for (int64_t r = 0; r < rows; r += step) go(r, (uint32_t)((rows - r < step ? rows - r : step) * across));
}

template <int TYPE>
int launch_tiles(const MxQuantize &a, bool square, hipStream_t s) {
    const int64_t tiles = (int64_t)a.across * a.down;
    for (int64_t t = 0; t < tiles; t += TILES) {
        const dim3 grid((uint32_t)(tiles - t < TILES ? tiles - t : TILES));
        if (square) hipLaunchKernelGGL(HIP_KERNEL_NAME(mx_tile_kernel<TYPE, true>), grid, dim3(256), 0, s, a, (uint32_t)t, grid.x);
        else hipLaunchKernelGGL(HIP_KERNEL_NAME(mx_tile_kernel<TYPE, false>), grid, dim3(256), 0, s, a, (uint32_t)t, grid.x);
    }
    return icq_check_launch();
}

bool rows_ok(const uint8_t *codes, int64_t ld, const uint8_t *scales, int64_t ld_s, int64_t cols) {
    return codes && scales && ld >= (cols + 1) / 2 && ld % 16 == 0 && (uintptr_t)codes % 16 == 0 && ld_s >= (cols + 31) / 32 && ld_s % 4 == 0 && (uintptr_t)scales % 4 == 0;
}

}  // namespace

int icq_launch_mx_rows(const MxQuantize &a, int x_type, hipStream_t s) {
    ICQ_FOR_TYPE(x_type, for_rows(a.rows, a.across, [&](int64_t r, uint32_t tasks) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(mx_rows_kernel<TYPE>), dim3((tasks + 15u) / 16u), dim3(256), 0, s, a, r, tasks);
    }))
    return icq_check_launch();
}

ICQ_EXPORT int icq_mx_quantize(const void *x, int x_type, int64_t rows, int64_t cols, int64_t ldx, int scaling, int block_rows, uint8_t *codes,
                               int64_t ld_codes, uint8_t *scales, int64_t ld_scales, uint8_t *codes_t, int64_t ld_codes_t, uint8_t *scales_t,
                               int64_t ld_scales_t, void *stream) {
    const int size = icq_type_bytes(x_type);
    if (size == 0 || (scaling != ICQ_MX_FLOOR && scaling != ICQ_MX_FIT) || (block_rows != 1 && block_rows != ICQ_MX_BLOCK) || rows < 0 || cols < 0 ||
        rows > ICQ_MAX_EXTENT || cols > ICQ_MAX_EXTENT)
        return ICQ_ERR_ARG;
    if (rows == 0 || cols == 0) return ICQ_OK;                                 // (addresses of nothing may be null)
    if (!codes && !codes_t) return ICQ_ERR_ARG;
    if ((codes && !rows_ok(codes, ld_codes, scales, ld_scales, cols)) || (codes_t && !rows_ok(codes_t, ld_codes_t, scales_t, ld_scales_t, rows))) return ICQ_ERR_ARG;
    if (!x || ldx < cols || (uintptr_t)x % size != 0) return ICQ_ERR_ARG;
    MxQuantize a;
    a.x = x; a.rows = rows; a.cols = cols; a.ldx = ldx;
    a.codes = codes; a.ld = ld_codes; a.scales = scales; a.ld_s = ld_scales;
    a.codes_t = codes_t; a.ld_t = ld_codes_t; a.scales_t = scales_t; a.ld_st = ld_scales_t;
    a.across = (int)((cols + 127) / 128);
    a.down = (int)((rows + 127) / 128);
    a.fit = scaling == ICQ_MX_FIT;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (block_rows == 1 && !codes_t) return icq_launch_mx_rows(a, x_type, s);
    if ((int64_t)a.across * a.down > 0x7fffffff) return ICQ_ERR_ARG;
    int rc = ICQ_OK;
    ICQ_FOR_TYPE(x_type, rc = launch_tiles<TYPE>(a, block_rows != 1, s))
    return rc;
}

ICQ_EXPORT int icq_mx_dequantize(const uint8_t *codes, int64_t ld_codes, const uint8_t *scales, int64_t ld_scales, int64_t rows, int64_t cols, void *out,
                                 int out_type, int64_t ldo, void *stream) {
    const int size = icq_type_bytes(out_type);
    if (size == 0 || rows < 0 || cols < 0 || rows > ICQ_MAX_EXTENT || cols > ICQ_MAX_EXTENT) return ICQ_ERR_ARG;
    if (rows == 0 || cols == 0) return ICQ_OK;
    if (!rows_ok(codes, ld_codes, scales, ld_scales, cols) || !out || ldo < cols || (uintptr_t)out % size != 0) return ICQ_ERR_ARG;
    MxValues a;
    a.codes = codes; a.ld = ld_codes; a.scales = scales; a.ld_s = ld_scales; a.rows = rows; a.cols = cols; a.out = out; a.ldo = ldo;
    a.across = (int)((cols + 127) / 128);
    hipStream_t s = static_cast<hipStream_t>(stream);
    ICQ_FOR_TYPE(out_type, for_rows(rows, a.across, [&](int64_t r, uint32_t tasks) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(mx_values_kernel<TYPE>), dim3((tasks + 15u) / 16u), dim3(256), 0, s, a, r, tasks);
    }))
    return icq_check_launch();
}
