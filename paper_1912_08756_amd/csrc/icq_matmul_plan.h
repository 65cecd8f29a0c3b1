// How icq_block_matmul computes a product, by its sizes.  Host code, no HIP.
#pragma once
#include <cstdint>

// Tiles of 256 x 256 (not into f32), of 128 x 128 with two stages in the LDS or four, or of 64 x 64.
enum icq_tiles { ICQ_TILES_WIDE, ICQ_TILES_SMALL, ICQ_TILES_DEEP, ICQ_TILES_LITTLE };

// Up to 16 rows; up to 32 where b has 16 rows for a compute unit or fewer (32 x 4096 x 4096: 10.5 us, in tiles 13; 32 x 16384 x 4096: 24,
// in tiles 14; 16 x 16384 x 4096: 14.4 here).
static inline bool icq_product_few_usable(int64_t M, int64_t N, int num_cu) { return M <= 16 || (M <= 32 && N <= 16 * (int64_t)num_cu); }

// 64 rows of b to a block instead of 16: a's rows are read a quarter as often.
static inline bool icq_product_few_wide(int64_t M, int64_t N, int num_cu) { return M <= 16 && N >= 64 * (int64_t)num_cu; }

constexpr int ICQ_PRODUCT_FEW_WAVES = 8;           // of a block, each with every eighth scale block

// Parts of the contraction: where the rows of b leave more than half of the chip idle, as long as a wavefront keeps four steps.
static inline int icq_product_few_splits(int64_t N, int64_t K, int num_cu) {
    const int64_t blocks = (N + 15) / 16, idle = num_cu / (blocks > 0 ? blocks : 1), most = (K + 127) / 128 / (4 * ICQ_PRODUCT_FEW_WAVES);
    const int64_t n = idle < most ? idle : most;
    return (int)(n < 1 ? 1 : n);
}

// How a product is computed: `few` rows; else in tiles, the contraction in `splits` parts.
struct icq_product_plan {
    bool few;
    icq_tiles tiles;
    int splits;
};

// Tiles: the plan of the least time by a model of it, in us, from times of every form and number of parts on 33 to 8192 rows: 4.5 for a
// launch with its first loads and last stores, and for a step (one scale block)
//     256 x 256: 1.8 for a round of the chip, 1.2 and more for a part of one;
//     128 x 128: 1.2 for two that share a compute unit, 0.5 to 0.6 for one by itself, the more of them the longer;
//     64 x 64:   0.45 for two that share a compute unit, 0.3 for one by itself;
// with the widened codes of a 32-bit result 1.9, 0.6 to 1.2, 0.66 and 0.45.  A split writes and reads its sums at 4.4 TB/s and costs a
// launch.  (1024 x 1024 x 4096 into bf16: 128 x 128 in 1, 2, 4, 8 parts 23.1, 19.4, 19.1, 29.0; 64 x 64 in 1, 2, 4 parts 14.1, 18.6, 20.0.)
static inline icq_product_plan icq_plan_product(int64_t M, int64_t N, int64_t K, bool exact, int num_cu) {
    icq_product_plan best = {icq_product_few_usable(M, N, num_cu), ICQ_TILES_SMALL, 1};
    if (best.few) {
        best.splits = icq_product_few_splits(N, K, num_cu);
        return best;
    }
    const int64_t kb = (K + 127) / 128;
    double least = -1.0;
    for (int64_t T = exact ? 128 : 256; T >= 64; T /= 2) {
        const int64_t tiles = ((M + T - 1) / T) * ((N + T - 1) / T);
        for (int splits = 1; splits <= 16 && (splits == 1 || kb >= 4 * splits); splits *= 2) {
            const int64_t blocks = tiles * splits, steps = (kb + splits - 1) / splits, rounds = blocks / (2 * num_cu), left = blocks % (2 * num_cu);
            const bool alone = blocks <= num_cu;
            // what a step of the last round adds: a pair's, a single tile's, nothing
            const auto last = [&](double pair, double one) { return left > num_cu ? pair : left > 0 ? one : 0.0; };
            const double share = (double)left / num_cu;
            double us;
            if (T == 256) us = 1.8 * (blocks / num_cu) + (blocks % num_cu > 0 ? 1.2 + 0.6 * (blocks % num_cu) / num_cu : 0.0);
            else if (T == 128) us = exact ? 1.9 * rounds + last(1.9, 0.6 + 0.6 * share) : 1.2 * rounds + last(1.2, 0.5 + 0.1 * share);
            else us = exact ? 0.66 * rounds + last(0.66, 0.45) : 0.45 * rounds + last(0.45, 0.3);
            us *= steps;
            if (splits > 1) us += 2.5 + (double)splits * M * N * 8 / 4.4e6;
            if (least < 0.0 || us < least) {
                least = us;
                best.tiles = T == 256 ? ICQ_TILES_WIDE : T == 64 ? ICQ_TILES_LITTLE : alone ? ICQ_TILES_DEEP : ICQ_TILES_SMALL;
                best.splits = splits;
            }
        }
    }
    return best;
}
