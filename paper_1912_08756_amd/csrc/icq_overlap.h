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

// Rows of `len` bytes every `ld` from an address on.
struct icq_extent {
    uintptr_t from;
    int64_t rows, ld, len;
};

static inline bool icq_extents_overlap(const icq_extent &a, const icq_extent &b) {
    if (a.rows <= 0 || b.rows <= 0 || a.len <= 0 || b.len <= 0) return false;
    const __int128 end_a = (__int128)a.from + (__int128)(a.rows - 1) * a.ld + a.len, end_b = (__int128)b.from + (__int128)(b.rows - 1) * b.ld + b.len;
    if (end_a <= (__int128)b.from || end_b <= (__int128)a.from) return false;
    if (a.rows > 1 && b.rows > 1 && a.ld == b.ld) {
        // parts of the same long rows, which meet in some row unless their places within a row are apart
        const icq_extent &x = a.from <= b.from ? a : b, &y = a.from <= b.from ? b : a;
        const int64_t d = (int64_t)((__int128)(y.from - x.from) % x.ld);
        return d < x.len || d + y.len > x.ld;
    }
    // each row of the one with fewer rows against the other's rows around its start and up to its end
    const icq_extent &x = a.rows <= b.rows ? b : a, &y = a.rows <= b.rows ? a : b;
    for (int64_t i = 0; i < y.rows; ++i) {
        const __int128 from = (__int128)y.from + (__int128)i * y.ld, off = from - (__int128)x.from;
        if (x.rows == 1) {
            if (off < x.len && off + y.len > 0) return true;
            continue;
        }
        __int128 k = off >= 0 ? off / x.ld : 0;                                // the last row of x that starts at or before it, or the first
        if (k >= x.rows) k = x.rows - 1;
        if (off < k * x.ld + x.len && off + y.len > k * x.ld) return true;
        if (k + 1 < x.rows && off + y.len > (k + 1) * x.ld && off < (k + 1) * x.ld + x.len) return true;
    }
    return false;
}
