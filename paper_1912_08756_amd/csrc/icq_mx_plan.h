// How icq_mx_matmul computes a product, by its sizes.  Host code, no HIP.
#pragma once
#include "icq_matmul_plan.h"

constexpr int ICQ_MX_FEW_WAVES = 8;                // of a block of the kernel for few rows

// Whether that kernel quantises a's values itself, in every block, `per` steps of 256 values of M rows: 68 KB of the LDS at most, and while that costs
// less than a launch of its own (values against held, 16384 x 4096, 16 steps: 1 row 8.8 - 8.6, 4 rows 10.3 - 9.2, 8 rows 12.4 - 9.8, 16 rows 16.9 - 10.8; a launch
// about 2).
static inline bool icq_mx_few_quantises(int64_t M, int64_t per) { return per <= 32 && M * per <= 64; }

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
    // (N K large: the tiles' loads into the LDS read faster, 6.3 TB/s against 5.5: 1 x 65536 x 8192 45 against 50 us, 16 x 65536 x 8192 47 against 67;
    // 16 x 16384 x 4096 8.3 against 10.8, 1 x 16384 x 4096 8.3 against 8.6)
    const bool long_rows = K >= 4096 && N >= 64 * (int64_t)num_cu && (M >= 8 || N * K >= (int64_t)1 << 28);
    icq_mx_plan best = {M <= 16 && !long_rows, false, 1, ICQ_TILES_SMALL, 1, (int)stages};
    if (best.few) {
        best.wide = N >= 64 * (int64_t)num_cu;
        const int64_t groups = (N + (best.wide ? 32 : 16) - 1) / (best.wide ? 32 : 16);
        // four wavefronts to a row as far as there are steps, eight where there are few rows
        while (best.along < 4 && 2 * best.along <= stages) best.along *= 2;
        if (8 <= stages && groups * best.along < 8 * (int64_t)num_cu) best.along = 8;
        // and as many blocks, while a wavefront keeps four steps
        const int64_t blocks = (groups * best.along + ICQ_MX_FEW_WAVES - 1) / ICQ_MX_FEW_WAVES, idle = num_cu / (blocks > 0 ? blocks : 1);
        const int64_t most = stages / (4 * best.along), n = idle < most ? idle : most;
        if (n > 1) {
            best.per = (int)((stages + n - 1) / n);
            best.splits = (int)((stages + best.per - 1) / best.per);
        }
        return best;
    }
    double least = -1.0;
    for (int64_t T = 256; T >= 64; T /= 2) {
        const int64_t tiles = ((M + T - 1) / T) * ((N + T - 1) / T);
        for (int splits = 1; splits <= 16 && (splits == 1 || stages >= 2 * splits); splits *= 2) {
            const int64_t per = (stages + splits - 1) / splits, parts = (stages + per - 1) / per, blocks = tiles * parts;
            const int64_t rounds = blocks / (2 * num_cu), left = blocks % (2 * num_cu);
            const bool alone = blocks <= num_cu;
            const auto last = [&](double pair, double one) { return left > num_cu ? pair : left > 0 ? one : 0.0; };
            const double share = (double)left / num_cu;
            double us;
            if (T == 256) us = 1.5 * (blocks / num_cu) + (blocks % num_cu > 0 ? 1.1 + 0.4 * (blocks % num_cu) / num_cu : 0.0);
            else if (T == 128) us = 1.0 * rounds + last(1.0, 0.5 + 0.1 * share);
            else us = 0.45 * rounds + last(0.45, 0.3);
            us *= per;
            if (parts > 1) us += 2.5 + (double)parts * M * N * 8 / 4.4e6;
            if (least < 0.0 || us < least) {
                least = us;
                best.tiles = T == 256 ? ICQ_TILES_WIDE : T == 64 ? ICQ_TILES_LITTLE : alone ? ICQ_TILES_DEEP : ICQ_TILES_SMALL;
                best.splits = (int)parts;
                best.per = (int)per;
            }
        }
    }
    return best;
}
