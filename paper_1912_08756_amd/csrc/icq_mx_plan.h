// How icq_mx_matmul computes a product, by its sizes.  Host code, no HIP.
#pragma once
#include "icq_matmul_plan.h"

#include <algorithm>

constexpr int ICQ_MX_FEW_WAVES = 8;                // of a block of the kernel for few rows
constexpr int ICQ_MX_FEW_LDS = 160 * 1024;         // it may use
constexpr int ICQ_MX_FEW_STEPS = 600;              // of 256 values of one row of a that fit it (136 bytes each) beside two steps of b for each wavefront and the parts' sums
static_assert(ICQ_MX_FEW_STEPS * 136 + 16 + ICQ_MX_FEW_WAVES * (2 * (4096 + 256) + 1024) <= ICQ_MX_FEW_LDS, "a, steps of b, sums");

// Whether that kernel quantises a's values itself, in every block, `per` steps of 256 values of M rows: while that costs less than a launch of its own
// (values against held, 16384 x 4096, 16 steps, other memory each time: 1 row 10.7 - 10.3 us, 4 rows 12.2 - 10.6; through a launch 8 rows 14.1 - 11.2).
static inline bool icq_mx_few_quantises(int64_t M, int64_t per) { return per <= 32 && M * per <= 64; }

// The tiles' times, by a model of them, in us, fitted to 25000 times of every form and number of parts at 3500 random sizes (17 to 8192 rows of a, 256
// to 65536 of b, 96 to 16384 values, over the same memory again and again, and by its own measure: what it chooses takes 1 % longer than the best in the mean, 4 % in
// nine of ten cases): a launch, and for each round of the chip's compute units (of pairs, where two blocks share one) a start with an end and a stage of 256 values,
// or those of a last round that is not full.  They are for the choice, not forecasts: 16384 x 960 x 4096 into f32 is modelled with 36, takes 43 so, 46 over other
// memory each time and 49 to 53 in a training step.  There is no term for b's way from memory; 17, 32, 64 and 128 rows against 1000000 x 960 the choice was the
// best all the same: 157, 164, 191 and 249 us, the next best form 166, 180, 226 and 259 (16 rows, by the kernel for few, 115).
struct icq_mx_times {
    icq_tiles tiles;
    int T, share;              // rows and columns of a tile, blocks that share a compute unit
    double launch, round, stage, last_round, last_stage, more;
};
constexpr icq_mx_times ICQ_MX_TIMES[4] = {{ICQ_TILES_WIDE, 256, 1, 4.0, 7.8, 1.5, 6.0, 1.15, 0.0}, {ICQ_TILES_SMALL, 128, 2, 2.0, 4.1, 0.98, 1.3, 0.56, 2.8},
                                          {ICQ_TILES_DEEP, 128, 1, 2.0, 3.9, 0.48, 2.7, 0.44, 0.0}, {ICQ_TILES_LITTLE, 64, 2, 1.8, 2.6, 0.43, 1.2, 0.32, 0.7}};

static inline double icq_mx_tiles_us(const icq_mx_times &t, int64_t blocks, int64_t per, int num_cu) {
    const int64_t room = (int64_t)num_cu * t.share, left = blocks % room;
    const double whole = t.round + t.stage * per, share = (double)left / num_cu;
    double us = t.launch + blocks / room * whole;
    if (t.share == 2) return us + (left > num_cu ? whole : left > 0 ? t.last_round + t.more * share + t.last_stage * per : 0.0);
    return us + (left > 0 ? t.last_round + (t.round - t.last_round) * share + (t.last_stage + (t.stage - t.last_stage) * share) * per : 0.0);
}

// `few` rows of a: wavefronts of 32 rows of b or of 16, `along` of a block's share rows and take parts of the contraction.  Else tiles: of 256 x 256, of
// 128 x 128 with two stages in the LDS or four, or of 64 x 64.
struct icq_mx_plan {
    bool few, wide;
    int along;
    icq_tiles tiles;
    int splits, per;           // parts of the contraction between blocks, steps of 256 values in each
};

static inline icq_mx_plan icq_plan_mx(int64_t M, int64_t N, int64_t K, int num_cu) {
    const int64_t stages = (K + 255) / 256;
    icq_mx_plan best = {M <= 16, false, 1, ICQ_TILES_SMALL, 1, (int)stages};
    if (best.few) {
        best.wide = N >= 64 * (int64_t)num_cu;
        const int64_t groups = (N + (best.wide ? 32 : 16) - 1) / (best.wide ? 32 : 16);
        // four wavefronts to a row as far as there are steps, eight where there are few rows (1, 2, 4, 8 of them, in us: 8 x 1000000 x 960 116, 107, 105, 152;
        // 8 x 500000 x 2048 111, 110, 109, 106; 1 x 100000 x 8000 106, 96, 80, 79; 1 x 16384 x 4096 13.3, 8.7, 7.0, 7.0)
        while (best.along < 4 && 2 * best.along <= stages) best.along *= 2;
        if (8 <= stages && groups * best.along < 8 * (int64_t)num_cu) best.along = 8;
        // and as many blocks, while a wavefront keeps four steps; more where a does not fit the LDS
        const int64_t blocks = (groups * best.along + ICQ_MX_FEW_WAVES - 1) / ICQ_MX_FEW_WAVES, idle = num_cu / (blocks > 0 ? blocks : 1);
        const int64_t most = stages / (4 * best.along), fit = ICQ_MX_FEW_STEPS / M, n = std::max((stages + fit - 1) / fit, std::min(idle, most));
        if (n > 1) {
            best.per = (int)((stages + n - 1) / n);
            best.splits = (int)((stages + best.per - 1) / best.per);
        }
        return best;
    }
    double least = -1.0;
    for (int form = 0; form < 4; ++form) {
        const icq_mx_times &t = ICQ_MX_TIMES[form];
        const int64_t tiles = ((M + t.T - 1) / t.T) * ((N + t.T - 1) / t.T), room = (int64_t)num_cu * t.share;
        for (int splits = 1; splits <= 16 && (splits == 1 || stages >= 2 * splits); splits *= 2) {
            const int64_t per = (stages + splits - 1) / splits, parts = (stages + per - 1) / per, blocks = tiles * parts;
            if (t.tiles == ICQ_TILES_DEEP && blocks > room) continue;
            const double us = icq_mx_tiles_us(t, blocks, per, num_cu) + (parts > 1 ? 1.7 + 0.3 * parts + (double)parts * M * N * 8 / 4.8e6 : 0.0);
            if (least < 0.0 || us < least) {
                least = us;
                best.tiles = t.tiles;
                best.splits = (int)parts;
                best.per = (int)per;
            }
        }
    }
    return best;
}
