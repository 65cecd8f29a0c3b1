// Whether two matrices share memory.  Host code, no HIP.
#pragma once
#include <cstdint>

// Rows of `len` bytes every `lda` from address a and every `ldb` from b, `rows` of each; len <= lda, ldb.
static inline bool icq_rows_overlap(uintptr_t a, int64_t lda, uintptr_t b, int64_t ldb, int64_t rows, int64_t len) {
    if (rows <= 0 || len <= 0) return false;
    const __int128 x = a, y = b, end_x = x + (__int128)(rows - 1) * lda + len, end_y = y + (__int128)(rows - 1) * ldb + len;
    if (end_x <= y || end_y <= x) return false;
    // b's row i against the two of a's rows around its start: a row reaches no further; of equal distances every row meets the same
    const auto meets = [&](int64_t i) {
        const __int128 from = y + (__int128)i * ldb, off = from - x;
        const __int128 k = off >= 0 ? off / lda : -((-off + lda - 1) / lda);      // rounded down
        for (__int128 r = k; r <= k + 1; ++r)
            if (r >= 0 && r < rows && from < x + r * lda + len && x + r * lda < from + len) return true;
        return false;
    };
    if (lda == ldb) return meets(0) || meets(rows - 1);
    for (int64_t i = 0; i < rows; ++i)
        if (meets(i)) return true;
    return false;
}
