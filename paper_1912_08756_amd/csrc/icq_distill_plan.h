// How the distillation calls go over a row, by its length and the number of rows.  Host code, no HIP.
#pragma once
#include <cstdint>

// Slices per row: one where there is a row for every compute unit, else enough blocks for the chip, none shorter than 8192 elements.
// Loss and gradient together in one kernel (row_bytes: a row's, else 0): one slice from half as many rows on (200 rows of 131072 bf16:
// 46 us in slices, 34 whole; 64 rows: 21 and 33), and for rows of up to 64 KB.
static inline int icq_distill_splits(int64_t R, int64_t V, int num_cu, int64_t row_bytes) {
    if (R >= num_cu || (row_bytes > 0 && (2 * R >= num_cu || row_bytes <= 65536))) return 1;
    const int64_t want = (4ll * num_cu + R - 1) / (R > 0 ? R : 1), most = V / 8192;
    const int64_t n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n > 1024 ? 1024 : n);
}

// Loss and gradient of whole rows in one kernel: its threads and the 16-byte groups that each holds, by the row's length: up to 16, 32, 64 KB, and
// longer (4096 rows of 24000 bf16: 86 us by 256 threads, 100 by 512; of 131072: 473 and 431); a row by itself on a compute unit by 1024.
enum icq_row_form { ICQ_ROW_1024_4, ICQ_ROW_256_4, ICQ_ROW_256_8, ICQ_ROW_256_16, ICQ_ROW_LONG };

static inline icq_row_form icq_distill_row_form(int64_t R, int64_t bytes, int num_cu) {
    if (R <= num_cu && bytes > 256 * 4 * 16 && bytes <= 1024 * 4 * 16) return ICQ_ROW_1024_4;
    if (bytes <= 256 * 4 * 16) return ICQ_ROW_256_4;
    if (bytes <= 256 * 8 * 16) return ICQ_ROW_256_8;
    return bytes <= 256 * 16 * 16 ? ICQ_ROW_256_16 : ICQ_ROW_LONG;
}

// The sums alone.  Whole rows of 256 KB and more by 512 threads (300 x 300000 f32: 74 us against 99 by 256, 1024 x 131072 bf16 53 and 55; shorter
// ones lose by it: 777 x 50021 f16 26.5 and 25.2, 8192 x 4096 f32 61 and 39).
static inline int icq_distill_forward_threads(int splits, int64_t bytes) { return splits == 1 && bytes >= 262144 ? 512 : 256; }
