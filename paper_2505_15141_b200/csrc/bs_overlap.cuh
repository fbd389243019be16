// Whether two arrays of a call share memory (host only).
#pragma once

#include <stdint.h>

namespace bs {

// [T, H] rows of `row` bytes; strides in bytes.
struct Rows {
    const void* at;
    long long st, sh;
    long long T, H, row;
};
inline Rows rows_of(const void* at, long long st, long long sh, long long T, long long H, long long d, long long element) {
    return {at, T > 1 ? st * element : 0, H > 1 ? sh * element : 0, T, H, d * element};   // of one token or head no stride matters
}
inline bool same_rows(const Rows& a, const Rows& b) {
    return a.at == b.at && a.st == b.st && a.sh == b.sh && a.T == b.T && a.H == b.H && a.row == b.row;
}

// Heads that follow one another, and tokens that do, are one row.
inline Rows joined(Rows r) {
    if (r.H > 1 && r.sh == r.row) { r.row *= r.H; r.H = 1; r.sh = 0; }
    if (r.T > 1 && r.st == r.row) { r.row *= r.T; r.T = 1; r.st = 0; }
    if (r.H > 1 && r.T == 1 && r.sh == r.row) { r.row *= r.H; r.H = 1; r.sh = 0; }
    return r;
}

// True where a byte is in both.  Exact where the arrays lie apart, begin together, one of them has no gaps, or they have one token stride,
// as views of one buffer have; what is interleaved in other ways (more than 2^16 pairs of heads, token strides that differ) counts as
// apart.
inline bool rows_overlap(Rows a, Rows b) {
    typedef __int128 wide;
    if (a.T < 1 || a.H < 1 || b.T < 1 || b.H < 1) return false;
    auto lowest = [](const Rows& r) { return (wide)(uintptr_t)r.at + (r.st < 0 ? (wide)(r.T - 1) * r.st : 0) + (r.sh < 0 ? (wide)(r.H - 1) * r.sh : 0); };
    auto behind = [](const Rows& r) { return (wide)(uintptr_t)r.at + (r.st > 0 ? (wide)(r.T - 1) * r.st : 0) + (r.sh > 0 ? (wide)(r.H - 1) * r.sh : 0) + r.row; };
    if (behind(a) <= lowest(b) || behind(b) <= lowest(a)) return false;
    if (a.at == b.at) return true;
    a = joined(a);
    b = joined(b);
    if (a.T == 1) a.st = b.st;
    if (b.T == 1) b.st = a.st;
    if (a.st != b.st) return false;
    // row (t, h) of a and (u, g) of b share a byte where off + g b.sh - h a.sh - (t - u) st lies within a row's length
    const wide off = (wide)(uintptr_t)b.at - (wide)(uintptr_t)a.at, st = a.st < 0 ? -(wide)a.st : (wide)a.st;
    const wide len_a = (wide)(a.H - 1) * a.sh + a.row, len_b = (wide)(b.H - 1) * b.sh + b.row;
    if (a.sh >= 0 && b.sh >= 0 && len_a <= st && len_b <= st) {   // the usual case: a token's heads within the token stride
        wide place = off % st;
        if (place < 0) place += st;
        if (place >= len_a && place + len_b <= st) return false;
    }
    const wide least = a.st < 0 ? 1 - a.T : 1 - b.T, most = a.st < 0 ? b.T - 1 : a.T - 1;   // of (t - u), counted along |st|
    auto floor_div = [&](wide x) { return x / st - (x % st < 0 ? 1 : 0); };
    auto meet = [&](wide x) {                                     // -b.row < x - k st < a.row for some k
        if (st == 0) return x > -b.row && x < a.row;
        const wide from = floor_div(x - a.row) + 1, to = floor_div(x + b.row - 1);
        return (from > least ? from : least) <= (to < most ? to : most);
    };
    if (a.sh == b.sh) {
        for (long long h = 1 - a.H; h < b.H; ++h)
            if (meet(off + (wide)h * a.sh)) return true;
        return false;
    }
    if (a.H * b.H > 65536) return false;
    for (long long h = 0; h < a.H; ++h)
        for (long long g = 0; g < b.H; ++g)
            if (meet(off + (wide)g * b.sh - (wide)h * a.sh)) return true;
    return false;
}

}  // namespace bs
