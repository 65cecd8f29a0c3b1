// Products of matrices in microscaled 4-bit floating point, in tiles of 256 x 256 (four wavefronts of 128 x 128), 128 x 128 (four of 64 x 64)
// or 64 x 64 (four of 32 x 32).
//
// A stage is 256 values of each row: 128 bytes of codes and eight scales, which go from memory straight into the LDS. A row's eight 16-byte
// pieces are permuted by its number, by the choice of each lane's address, so that 16 rows' pieces fall on all 64 banks. One piece is a
// lane's operand of a 32x32x64 instruction; its scale is a byte of a word that holds the lane's four of the stage.
// A stage has four steps of 64 values. A step's fragments are read beside the matrix instructions of the step before. The one barrier of a
// stage stands before its last step's: by then the next stage has arrived and this one's last fragments are in registers, so its place
// in the LDS takes the stage after the next.
//
// Bound by the matrix instructions and the clock that they leave at 8192 x 8192 x 8192: 264 us over the same memory again and again, 4170 TFLOP/s, 272 to 292
// over other memory each time, 3770 to 4040 (a large library product 308, 3565; random codes in registers alone 6770; matrix pipe 49 % of the cycles, wavefronts
// wait for 28 %), and by the results where rows are short: 4096 x 16384 x 960 into bf16 64 us over the same memory, 69 over other, 15 of them the
// results' way to memory and 7 their turn through the LDS; a kernel that does nothing but fill such a result takes 21.
// Why these tiles (same memory, other memory): a wavefront of 128 x 128 reads half the fragments from the LDS that one of 64 x 64 reads for a product, 8192^3
// 264 and 272 against 321 and 359 us; but 4096 x 960 results of 16384 products (64 wide tiles) take 95 us so, 52 in tiles of 128 x 128, two to a compute
// unit, 44 with four stages.  Blocks that go on to a next tile: 4096 x 16384 x 1024 59 against 66 us when that was taken, 61 now with the wait states in
// the loads' text.  Rows of codes that start on 128 bytes are read faster: 1024 values 61 us, 960 in rows of 480 bytes 64.
#include "icq_mx.h"
#include "icq_tiles.h"

#include <algorithm>
#include <type_traits>

namespace {

// Rows and columns of a wavefront's part in units of 32, wavefronts along m and n, stages in the LDS, blocks that share a compute unit.
template <int NI_, int NJ_, int WM_, int WN_, int DEPTH_, int SHARE_>
struct Shape {
    static constexpr int NI = NI_, NJ = NJ_, WM = WM_, WN = WN_, DEPTH = DEPTH_, SHARE = SHARE_, WAVES = WM * WN, THREADS = 64 * WAVES, T = 32 * NI * WM;
    static constexpr int PARTS = T / (8 * WAVES), LOADS = 2 * PARTS;          // of a wavefront for a stage's codes: eight rows each
    static constexpr int WORDS = 2 * T / 32 / WAVES;                          // of a wavefront for four stages' scales: half of 64 rows' each
    static constexpr int FIRST = LOADS / 2;                                   // requested in the step of the barrier, the others in the next: halves of a's and b's rows
    static constexpr bool ON = NI * NJ == 16;                                 // a block goes on to a next tile: with a compute unit to itself, nothing else would cover a tile's start and end
    static constexpr int STAGE = 2 * T * 128, SCALES = 2 * T * 32;            // bytes of a stage's codes, of four stages' scales
    static constexpr int LDS_BYTES = DEPTH * STAGE + 2 * SCALES;
    static_assert(32 * NJ * WN == T && T % 64 == 0 && WORDS >= 1 && (2 * T / 32) % WAVES == 0 && (DEPTH - 1) * LOADS < 64,
                  "square tiles; whole loads; countable ones");
    static_assert(DEPTH * STAGE / WAVES >= 32 * 32 * NJ * 4 && (!ON || (DEPTH == 2 && WAVES == 4 && PARTS % 2 == 0 && T * 32 >= 32 * 64 * 4)), "results fit the stages, or a half of one");
    static_assert(SHARE * LDS_BYTES <= 160 * 1024, "fits the LDS");
};
typedef Shape<4, 4, 2, 2, 2, 1> Wide;
typedef Shape<2, 2, 2, 2, 2, 2> Small;
typedef Shape<2, 2, 2, 2, 4, 1> Deep;
typedef Shape<1, 1, 2, 2, 4, 2> Little;

// 32 rows and 32 NJ columns of the result, whole rows at a time: in the accumulators a lane has four neighbours of one row and the lanes 32 rows, whose
// stores would be 8 or 16 bytes here and there (64 bytes, with registers exchanged between lanes, took 2 us more for a tile of 256 x 256 than this).  They
// go through the LDS in the result's type, with no branch around the accumulators (the compiler would move and spill them).  turn: 32 rows of 16-byte
// pieces, a row's permuted by its number.
template <int OUT, int NJ>
__device__ __forceinline__ void store_rows_as(uint4 *turn, const f32x16 *acc, void *out, int64_t ldo, int64_t M, int64_t N, int64_t m0, int64_t n0, int lane) {
    typedef IcqElem<OUT> Elem;
    constexpr int WIDTH = 32 * NJ, PER = Elem::PER, PIECES = WIDTH / PER, AT_ONCE = 64 / PIECES, TIMES = 32 / AT_ONCE, SIZE = 16 / PER;
    constexpr int SHIFT = PIECES >= 8 ? 0 : 1;                                // eight rows' pieces of a column fall on all banks that a write reaches at once
    const int at = lane & 31, half = lane >> 5;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < NJ; ++j)
        if constexpr (OUT == ICQ_F32) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const icq_f32x4 v = {acc[j][4 * g], acc[j][4 * g + 1], acc[j][4 * g + 2], acc[j][4 * g + 3]};
                *reinterpret_cast<icq_f32x4 *>(turn + at * PIECES + ((j * 8 + 2 * g + half) ^ (at >> SHIFT & (PIECES - 1)))) = v;
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {                                     // a lane's halves of two pieces of eight for one whole
                const auto first = __builtin_amdgcn_permlane32_swap(Elem::pack2(acc[j][8 * h], acc[j][8 * h + 1]), Elem::pack2(acc[j][8 * h + 4], acc[j][8 * h + 5]), false, false);
                const auto second = __builtin_amdgcn_permlane32_swap(Elem::pack2(acc[j][8 * h + 2], acc[j][8 * h + 3]), Elem::pack2(acc[j][8 * h + 6], acc[j][8 * h + 7]), false, false);
                turn[at * PIECES + ((j * 4 + 2 * h + half) ^ (at >> SHIFT & (PIECES - 1)))] = make_uint4(first[0], second[0], first[1], second[1]);
            }
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int c = lane % PIECES, r = lane / PIECES;
    uint4 x[TIMES];
#pragma unroll
    for (int t = 0; t < TIMES; ++t) x[t] = turn[(t * AT_ONCE + r) * PIECES + (c ^ ((t * AT_ONCE + r) >> SHIFT & (PIECES - 1)))];
    uint8_t *to = static_cast<uint8_t *>(out) + ((m0 + r) * ldo + n0 + c * PER) * SIZE;
    const int64_t step = AT_ONCE * ldo * SIZE;
    if (m0 + 32 <= M && n0 + WIDTH <= N) {
#pragma unroll
        for (int t = 0; t < TIMES; ++t) __builtin_memcpy(to + t * step, &x[t], 16);              // (to any address)
        return;
    }
    const int left = (int)max((int64_t)0, min((int64_t)PER, N - n0 - c * PER));
#pragma unroll
    for (int t = 0; t < TIMES; ++t) {
        if (m0 + t * AT_ONCE + r >= M) continue;
        if (left == PER) {
            __builtin_memcpy(to + t * step, &x[t], 16);
            continue;
        }
        const uint32_t w[4] = {x[t].x, x[t].y, x[t].z, x[t].w};
#pragma unroll
        for (int e = 0; e < PER - 1; ++e)
            if (e < left) {
                if constexpr (OUT == ICQ_F32) reinterpret_cast<uint32_t *>(to + t * step)[e] = w[e];
                else reinterpret_cast<uint16_t *>(to + t * step)[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
            }
    }
}

// Where the codes of a tile's rows lie, and this lane's places in them.
template <typename S>
struct Target {
    const uint8_t *a, *b;
    uint32_t off_a[S::PARTS], off_b[S::PARTS];
};

// What is left of a row in the last stage: nothing (the stage is whole), more than half of its 256 values, or half at most.
enum Tail { WHOLE, MORE, LESS };

// OUT: the result's type, or that of the parts.
// A block takes tiles blockIdx.x, + gridDim.x, ...: more than one only where S::ON, the contraction is not in parts and a row has 16 bytes of
// scales.  The requests go on into the next tile: when this one's results are stored, the next one's first stage has arrived and the second is under way.
template <typename S, Tail TAIL, int OUT>
__global__ __launch_bounds__(S::THREADS, S::WAVES * S::SHARE / 4) void mx_tiles_kernel(MxProduct q, int tiles_m, int tiles_n, uint32_t tiles, uint32_t first_tile) {
    constexpr int T = S::T, NI = S::NI, NJ = S::NJ, DEPTH = S::DEPTH, WAVES = S::WAVES, PARTS = S::PARTS, WORDS = S::WORDS, LOADS = S::LOADS, FIRST = S::FIRST;
    constexpr int N = NI * NJ, F = NI + NJ;                                   // matrix instructions, fragments of a step
    constexpr bool ON = S::ON, RAGGED = TAIL != WHOLE;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];          // stages' codes, then two places for four stages' scales
    const Product &p = q.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int k0 = blockIdx.y * p.per, last = min(p.kb, k0 + p.per) - 1;      // stages k0 .. last, one at least
    const int wm = (wave % S::WM) * 32 * NI, wn = (wave / S::WM) * 32 * NJ, at = lane & 31, half = lane >> 5;
    const int whole = (int)(p.K / 256), ragged = (int)(p.K % 256);            // stages along K, and values in one more

    // Loads: instruction u of a wavefront brings rows 8 (WAVES u + wave) .. + 7 of a, then of b; row r's piece c sits at place c ^ (r / 2 % 8).
    // Four stages' scales are two pieces of 16 bytes of a row: an instruction brings one of 64 rows (in rows of 32 bytes they would meet on the
    // same banks when read).
    const int piece = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
    auto place_of = [&](uint32_t id, int64_t &m0, int64_t &n0) {
        // XCD id % 8 takes a contiguous share of the tiles, eight tiles of m at a time
        const int total = tiles_m * tiles_n, q8 = total / 8, r8 = total % 8, xcd = id % 8, at8 = id / 8;
        const int tile = xcd * q8 + (xcd < r8 ? xcd : r8) + at8;
        const int group = tile / (8 * tiles_n), in = tile % (8 * tiles_n), high = min(8, tiles_m - group * 8);
        m0 = (int64_t)(group * 8 + in % high) * T;
        n0 = (int64_t)(in / high) * T;
    };
    Target<S> late_to, to;                                                    // of the requests: of the second part of a stage, of the first
    auto aim = [&](Target<S> &to, uint32_t id) {
        int64_t m0, n0;
        place_of(id, m0, n0);
        to.a = p.a + m0 * p.lda;
        to.b = p.b + n0 * p.ldb;
#pragma unroll
        for (int u = 0; u < PARTS; ++u) {
            const int r = 8 * (WAVES * u + wave) + (lane >> 3);
            to.off_a[u] = (uint32_t)(min((int64_t)r, p.M - 1 - m0) * p.lda) + piece * 16;
            to.off_b[u] = (uint32_t)(min((int64_t)r, p.N - 1 - n0) * p.ldb) + piece * 16;
        }
    };
    const int words = (q.blocks + 3) >> 2;                                    // of four scales in a row
    const uint32_t beyond = piece * 32 >= ragged ? piece * 16 : 0;
    // what takes a piece of stage kb beyond the row's end back into it
    auto back_of = [&](int kb) { return RAGGED && kb == whole ? beyond : 0u; };
    // request v of stage kb into place buf
    auto request = [&](const Target<S> &to, int v, int kb, int buf, uint32_t back) {
        const int u = v >> 1;
        load_to_lds(bytes_from((v & 1) ? to.b : to.a), ((v & 1) ? to.off_b[u] : to.off_a[u]) - back, kb * 128,
                    buf * S::STAGE + (v & 1) * T * 128 + (WAVES * u + wave) * 1024);
    };
    // A piece of 16 bytes that would reach beyond its row starts earlier: its words sit by so many further in their place.
    auto request_scales = [&](uint32_t id, int kb, int place) {
        int64_t m0, n0;
        place_of(id, m0, n0);
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            const int x = w * WAVES + wave, r = x % (2 * T / 64) * 64, second = x / (2 * T / 64);
            const bool of_a = r < T;
            const uint32_t off = (uint32_t)(of_a ? min((int64_t)(r + lane), p.M - 1 - m0) * q.ld_ea : min((int64_t)(r - T + lane), p.N - 1 - n0) * q.ld_eb);
            load_to_lds(bytes_from(of_a ? q.ea + m0 * q.ld_ea : q.eb + n0 * q.ld_eb), off, min(2 * kb + 4 * second, words - 4) * 4,
                        DEPTH * S::STAGE + place * S::SCALES + x * 1024);
        }
    };

    f32x16 acc[NI][NJ];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    };
    i32x4 f[2][F];                                                            // fragments of two steps: a's, then b's
    uint32_t sc[F], lo[F], hi[F];                                             // scales of the stage; of the next one as they are read
    const uint32_t pick = half ? 0x07050301u : 0x06040200u;
    const uint8_t *row_a = smem + (wm + at) * 128, *row_b = smem + (T + wn + at) * 128;
    // fragment v of step s of the stage in place buf
    auto read = [&](int v, int s, int buf) {
        const uint8_t *row = (v < NI ? row_a + v * 4096 : row_b + (v - NI) * 4096) + buf * S::STAGE;
        return *reinterpret_cast<const i32x4 *>(row + (((2 * s + half) ^ (at >> 1 & 7)) << 4));
    };
    // the scales of stage kb, whose group of four lies in `place`: two words of a piece, the second only if there is one
    auto read_scales = [&](int v, int kb, int place) {
        const int row = v < NI ? wm + v * 32 + at : T + wn + (v - NI) * 32 + at;
        const int pair = (kb - k0) >> 1, at_word = 2 * kb - max(0, min(pair * 4 + 2 * k0, words - 4));
        const uint8_t *w = smem + DEPTH * S::STAGE + place * S::SCALES + (pair & 1) * 2 * T * 16 + row * 16;
        if constexpr (TAIL == LESS) {                                         // (an odd number of words in a row)
            lo[v] = *reinterpret_cast<const uint32_t *>(w + min(at_word, 3) * 4);
            hi[v] = *reinterpret_cast<const uint32_t *>(w + min(at_word + 1, 3) * 4);
        } else {                                                              // (an even one: half the bank conflicts)
            const uint2 both = *reinterpret_cast<const uint2 *>(w + at_word * 4);
            lo[v] = both.x;
            hi[v] = both.y;
        }
    };
    auto take_scales = [&]() {
#pragma unroll
        for (int v = 0; v < F; ++v) sc[v] = __builtin_amdgcn_perm(hi[v], lo[v], pick);
    };
    auto multiply = [&](int i, int j, int s) {
        const i32x4 x = f[s & 1][NI + j], y = f[s & 1][i];
        const icq_i32x8 n = {x[0], x[1], x[2], x[3], 0, 0, 0, 0}, m = {y[0], y[1], y[2], y[3], 0, 0, 0, 0};
        const int en = (int)sc[NI + j], em = (int)sc[i];
        if (s == 0) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(n, m, acc[i][j], 4, 4, 0, en, 0, em);
        else if (s == 1) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(n, m, acc[i][j], 4, 4, 1, en, 1, em);
        else if (s == 2) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(n, m, acc[i][j], 4, 4, 2, en, 2, em);
        else acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(n, m, acc[i][j], 4, 4, 3, en, 3, em);
    };

    uint32_t tile = first_tile + blockIdx.x;
    aim(to, tile);
    late_to = to;
    if (words >= 4) request_scales(tile, k0, 0);
    else {                                                                    // rows of fewer than 16 bytes: one by one, all there are
        int64_t m0, n0;
        place_of(tile, m0, n0);
        for (int r = tid; r < 2 * T; r += S::THREADS) {
            const uint8_t *from = r < T ? q.ea + min(m0 + r, p.M - 1) * q.ld_ea : q.eb + min(n0 + r - T, p.N - 1) * q.ld_eb;
            for (int w = 0; w < words; ++w) *reinterpret_cast<uint32_t *>(smem + DEPTH * S::STAGE + r * 16 + w * 4) = *reinterpret_cast<const uint32_t *>(from + w * 4);
        }
    }
    // beyond the last tile's last stage that one is requested again: no branch in the loop
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
        const int kb = min(k0 + d, last);
        const uint32_t back = back_of(kb);
#pragma unroll
        for (int v = 0; v < LOADS; ++v)
            if (d < DEPTH - 1 || v < FIRST) request(to, v, kb, d, back);
    }
    __builtin_amdgcn_s_waitcnt(loads_left((DEPTH - 2) * LOADS + FIRST));
    __syncthreads();
#pragma unroll
    for (int v = 0; v < F; ++v) {
        f[0][v] = read(v, 0, 0);
        read_scales(v, k0, 0);
    }
    take_scales();
    int buf = 0, place = 0;                                                   // of the stage under way, of its four's scales
    // the stage under way is kb of `tile`; the requests in its time are of the stages kb + DEPTH - 1 and kb + DEPTH, counted on into the next tile
    for (;;) {
        const bool more = ON && tile + gridDim.x < tiles;
        clear();
        int kb = k0, end;
        do {                                                                  // stages up to `end`: their scales are in the LDS, their requests of one tile
            if ((kb - k0) % 4 == 0) {                                         // (nobody reads the other place any more: a barrier since at least)
                if (kb + 4 <= last) request_scales(tile, kb + 4, place ^ 1);
                else if (more) request_scales(tile + gridDim.x, k0, place ^ 1);
            }
            const int group_end = min(k0 + (kb - k0) / 4 * 4 + 3, last), turn = last + 1 - DEPTH;
            end = group_end;
            if (ON && more) {                                                 // from stage `turn` on, a stage's first requests are the next tile's, then all
                if (kb == turn) aim(to, tile + gridDim.x);
                if (kb == turn + 1) late_to = to;
                if (kb <= turn) end = min(end, kb < turn ? turn - 1 : turn);
            }
            const auto stage = [&](auto cut) {                                // cut: of the row's last values only, fewer than 256
                constexpr bool CUT = decltype(cut)::value;
                const int next_buf = (buf + 1) & (DEPTH - 1), last_buf = (buf + DEPTH - 1) & (DEPTH - 1);
                const auto of = [&](int k) { return k <= last ? k : more ? k - last - 1 + k0 : last; };
                const int late = of(kb + DEPTH - 1), later = of(kb + DEPTH), next = of(kb + 1);
                const uint32_t back_late = back_of(late), back_later = back_of(later);
                const int next_place = kb == group_end ? place ^ 1 : place;   // (the last of all: whatever lies there)
                if constexpr (CUT) {                                          // scales of no block become some number, codes of no value zero in a
                    uint32_t keep = 0;
#pragma unroll
                    for (int s = 0; s < 4; ++s)
                        if (2 * s + half < q.blocks - 8 * whole) keep |= 0xffu << (8 * s);
#pragma unroll
                    for (int v = 0; v < F; ++v) sc[v] = (sc[v] & keep) | (0x7f7f7f7fu & ~keep);
                }
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    if (s == 3) {
                        // the next stage is here, and the next four's scales after the last; later stages may not be
                        __builtin_amdgcn_s_waitcnt(loads_left((DEPTH - 2) * LOADS));
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
                        __builtin_amdgcn_s_barrier();
                    }
                    if constexpr (CUT) {
                        const uint4 tail = first_codes(make_uint4(~0u, ~0u, ~0u, ~0u), min(max(ragged - 64 * s - 32 * half, 0), 32));
                        const i32x4 mask = {(int)tail.x, (int)tail.y, (int)tail.z, (int)tail.w};
#pragma unroll
                        for (int i = 0; i < NI; ++i) f[s & 1][i] &= mask;
                    }
#pragma unroll
                    for (int t = 0; t < N; ++t) {
                        // requests and reads, spread over the step's matrix instructions
#pragma unroll
                        for (int v = 0; v < LOADS; ++v) {
                            if (s == 0 && v >= FIRST && (v - FIRST) * N / (LOADS - FIRST) == t) request(ON ? late_to : to, v, late, last_buf, back_late);
                            if (s == 3 && v < FIRST && v * N / FIRST == t) request(to, v, later, buf, back_later);
                        }
                        multiply(t / NJ, t / NJ % 2 ? NJ - 1 - t % NJ : t % NJ, s);              // (neighbours share an operand)
#pragma unroll
                        for (int v = 0; v < F; ++v)
                            if (v * N / F == t) {
                                if (s == 3) read_scales(v, next, next_place);
                                f[(s + 1) & 1][v] = s < 3 ? read(v, s + 1, buf) : read(v, 0, next_buf);
                            }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                take_scales();
                buf = next_buf;
                ++kb;
            };
            const int whole_end = RAGGED ? min(end, whole - 1) : end;
            while (kb <= whole_end) stage(std::false_type());
            if constexpr (RAGGED)
                if (kb <= end) stage(std::true_type());
            if (kb > group_end) place ^= 1;
        } while (kb <= last);
        void *out = p.splits > 1 ? static_cast<void *>(p.part + (int64_t)blockIdx.y * p.M * p.N) : p.out;
        const int64_t ldo = p.splits > 1 ? p.N : p.ldo;
        int64_t m0, n0;
        place_of(tile, m0, n0);
        m0 += wm;
        n0 += wn;
        if constexpr (ON) {
            // the last stage's place: of its halves of a's and of b's rows the first ones take requests, the second ones results
            constexpr int HALF = T * 64, AT_A_TIME = OUT == ICQ_F32 ? 2 : 4;
            uint4 *turn = reinterpret_cast<uint4 *>(smem + ((buf + DEPTH - 1) & (DEPTH - 1)) * S::STAGE + HALF + (wave & 1) * (HALF / 2) + (wave >> 1) * 2 * HALF);
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int j = 0; j < NJ; j += AT_A_TIME) {
#pragma unroll
                    for (int e = 0; e < AT_A_TIME; ++e) asm volatile("" : "+a"(acc[i][j + e]));  // (read here, not all of them before the first branch)
                    store_rows_as<OUT, AT_A_TIME>(turn, acc[i] + j, out, ldo, p.M, p.N, m0 + i * 32, n0 + j * 32, lane);
                }
            if (!more) break;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
            __builtin_amdgcn_s_barrier();
        } else {
            __builtin_amdgcn_s_waitcnt(loads_left(0));                        // (a wavefront's part of the stages takes its results)
            __syncthreads();
            uint4 *turn = reinterpret_cast<uint4 *>(smem + wave * (DEPTH * S::STAGE / WAVES));
#pragma unroll
            for (int i = 0; i < NI; ++i) store_rows_as<OUT, NJ>(turn, acc[i], out, ldo, p.M, p.N, m0 + i * 32, n0, lane);
            break;
        }
        tile += gridDim.x;
    }
    __builtin_amdgcn_s_waitcnt(loads_left(0));                                // (requests into the LDS end before it is another's)
}

template <typename S>
int launch(const MxProduct &q, int num_cu, int out_type, hipStream_t s) {
    const int tm = (int)((q.p.M + S::T - 1) / S::T), tn = (int)((q.p.N + S::T - 1) / S::T);
    const uint32_t tiles = (uint32_t)((int64_t)tm * tn);
    // one tile after another in as many blocks as there is room for (a multiple of 8: a block stays with its XCD), or a block for each
    const bool on = S::ON && q.p.splits == 1 && q.blocks > 12;
    const uint32_t room = (uint32_t)(num_cu * S::SHARE) & ~7u;
    const auto go = [&](auto kernel) {
        if (icq_allow_lds(reinterpret_cast<const void *>(kernel), S::LDS_BYTES, true) != hipSuccess) return ICQ_ERR_HIP;
        const auto launch = [&](uint32_t blocks, uint32_t end, uint32_t first) {
            hipLaunchKernelGGL(kernel, dim3(blocks, (uint32_t)q.p.splits), dim3(S::THREADS), S::LDS_BYTES, s, q, tm, tn, end, first);
        };
        if (on && room > 0 && tiles > room) launch(room, tiles, 0);
        else
            for (uint32_t i = 0; i < tiles; i += ICQ_PRODUCT_BLOCKS) launch(std::min(tiles - i, ICQ_PRODUCT_BLOCKS), 0, i);
        return icq_check_launch();
    };
    if (q.p.splits > 1) out_type = ICQ_F32;
    const int tail = (int)(q.p.K % 256);
    ICQ_FOR_TYPE(out_type, return tail == 0 ? go(mx_tiles_kernel<S, WHOLE, TYPE>) : tail > 128 ? go(mx_tiles_kernel<S, MORE, TYPE>) : go(mx_tiles_kernel<S, LESS, TYPE>))
}

}  // namespace

int icq_launch_mx_tiles(const MxProduct &q, icq_tiles tiles, int num_cu, int out_type, hipStream_t s) {
    return tiles == ICQ_TILES_WIDE ? launch<Wide>(q, num_cu, out_type, s) : tiles == ICQ_TILES_LITTLE ? launch<Little>(q, num_cu, out_type, s)
           : tiles == ICQ_TILES_DEEP ? launch<Deep>(q, num_cu, out_type, s) : launch<Small>(q, num_cu, out_type, s);
}
