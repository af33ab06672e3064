// Rows of strided tensors that are written in place: whether they are distinct.  Plain arithmetic on the host.
#pragma once

#include <utility>

namespace dig {

// Rows of a tensor: [b][l] starts b * sb + l * st elements from the first and holds `width`.
struct RowSet {
    int B, L;
    long long sb, st, width;
    // From the first element of the first row to behind the last of the last.
    __int128 extent() const { return (__int128)(B - 1) * sb + (__int128)(L - 1) * st + width; }
    // The usual layouts: whole rows behind one another, sequence by sequence or token by token.
    bool in_order() const
    {
        return (L == 1 || st >= width) && (B == 1 || sb >= width) &&
               (B == 1 || L == 1 || sb >= (__int128)(L - 1) * st + width || st >= (__int128)(B - 1) * sb + width);
    }
};
// Whether a row of `r` meets one of `width` elements that starts `off` elements behind another row of r's, or that row itself (not, where `same`:
// then they are the same rows).  Rows (db, dl) apart are off + db sb + dl st apart; one of the two is tried out, the other follows.
inline bool rows_meet(RowSet r, long long off, long long width, bool same)
{
    if (r.L < r.B) {
        std::swap(r.L, r.B);
        std::swap(r.sb, r.st);
    }
    for (int db = 1 - r.B; db < r.B; ++db) {
        const __int128 x = off + (__int128)db * r.sb, lo = -x - width + 1, hi = r.width - 1 - x;            // lo <= dl st <= hi
        if (r.st == 0) {
            if (lo <= 0 && hi >= 0 && !(same && db == 0 && r.L == 1)) return true;
            continue;
        }
        const __int128 up = r.L - 1;
        __int128 first = lo > 0 ? (lo + r.st - 1) / r.st : -(-lo / r.st), last = hi >= 0 ? hi / r.st : -((-hi + r.st - 1) / r.st);
        first = first < -up ? -up : first;
        last = last > up ? up : last;
        if (first > last || (same && db == 0 && first == 0 && last == 0)) continue;
        return true;
    }
    return false;
}
// Whether a row of `r` meets the `width` elements that start `off` elements behind the first row's start.
inline bool rows_meet_block(RowSet r, long long off, long long width)
{
    if (off >= r.extent() || off + (__int128)width <= 0) return false;
    if (r.L < r.B) {
        std::swap(r.L, r.B);
        std::swap(r.sb, r.st);
    }
    for (int b = 0; b < r.B; ++b) {
        const __int128 x = off - (__int128)b * r.sb, lo = x - r.width + 1, hi = x + width - 1;             // lo <= l st <= hi
        if (hi < 0 || lo > (__int128)(r.L - 1) * r.st) continue;
        if (lo <= 0 || r.st == 0 || (lo + r.st - 1) / r.st * r.st <= hi) return true;
    }
    return false;
}
// Whether rows that are written in place are distinct: those of one tensor, and of one and the other, which starts `off` elements further.
inline bool distinct(const RowSet &r) { return r.in_order() || !rows_meet(r, 0, r.width, true); }
inline bool apart(const RowSet &q, const RowSet &k, long long off)
{
    if (off >= q.extent() || -(__int128)off >= k.extent()) return true;
    const bool sb = q.B == 1 || q.sb == k.sb, st = q.L == 1 || q.st == k.st;
    if (sb && st) {
        // side by side in wider rows
        RowSet both = q;
        both.width = off >= q.width ? off + k.width : -off >= k.width ? q.width - off : 0;
        return (both.width > 0 && both.in_order()) || !rows_meet(q, off, k.width, false);
    }
    // strides that differ: whole sequences, or a token of all sequences, have to be apart
    if (sb) return !rows_meet({q.B, 1, q.sb, 0, (long long)(q.L - 1) * q.st + q.width}, off, (long long)(k.L - 1) * k.st + k.width, false);
    const __int128 qw = (__int128)(q.B - 1) * q.sb + q.width, kw = (__int128)(k.B - 1) * k.sb + k.width, most = 1ll << 62;
    return st && qw < most && kw < most && !rows_meet({1, q.L, 0, q.st, (long long)qw}, off, (long long)kw, false);
}

}  // namespace dig
