// Tiles of products in the LDS: loads straight into it, results out of it.
#pragma once
#include "icq_matmul.h"

typedef float f32x16 __attribute__((ext_vector_type(16)));

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
// wait for loads of its own built-in; they have no destination registers, and the waits for them are those of loads_left(0).  The compiler does not look
// into the text: a vector memory instruction has to come five wait states after a vector instruction that writes one of its scalar registers
// (v_readfirstlane, or v_readlane where the compiler brings a spilled one back, right before the statement), so the text itself holds them.
__device__ __forceinline__ void load_to_lds(const i32x4 &base, uint32_t off, int by, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(base), "s"(by) : "memory", "m0");
}

// The same as load_to_lds for 4 bytes per lane, to `to` + 4 * lane.
__device__ __forceinline__ void load_word_to_lds(const i32x4 &base, uint32_t off, int by, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(base), "s"(by) : "memory", "m0");
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
