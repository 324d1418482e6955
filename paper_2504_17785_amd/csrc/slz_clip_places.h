// Whether matrices in memory have bytes in common (slz_clip.hip); host code that needs no GPU.
#pragma once
#include <stdint.h>

// Memory of a matrix: from `begin` to `end`, rows of `row` bytes `step` apart (0: one run); row <= step, all of it below 2^51 bytes
struct clip_place { uintptr_t begin, end; uint64_t row, step; uint32_t out; };

// The least t >= 0 with l <= a t mod m <= r, or -1; 0 <= l <= r < m, 0 <= a < m.
// Euclid's steps: where no multiple of a lies in the range, a t = m y + (l .. r) asks for m y mod a in (-r .. -l) mod a.
static inline __int128 clip_first_in(uint64_t a, uint64_t m, uint64_t l, uint64_t r) {
    if (l == 0) return 0;
    if (a == 0) return -1;
    const uint64_t first = (l + a - 1) / a;
    if (first * a <= r) return first;                  // below m + a
    const __int128 y = clip_first_in(m % a, a, (a - r % a) % a, (a - l % a) % a);
    return y < 0 ? y : (l + (__int128)m * y + a - 1) / a;
}
// Of rows at different distances, a's beginning first: row i of a meets a row of b that begins within the `wide` bytes from lo + i a.step on, counted from b's first row
__attribute__((noinline)) static bool clip_rows_meet(const clip_place &a, const clip_place &b) {
    const auto rows = [](const clip_place &p) { return p.step ? (int64_t)((p.end - p.begin - p.row) / p.step) + 1 : 1; };
    const int64_t lo = (int64_t)(a.begin - b.begin) - (int64_t)b.row + 1, wide = (int64_t)(a.row + b.row) - 1, step = a.step ? (int64_t)a.step : 1, count = rows(a);
    // the first and the last i with lo + i step <= at <= lo + i step + wide - 1, or with one of the two
    const auto floor_of = [&](int64_t n) { return n >= 0 ? n / step : -((-n + step - 1) / step); };
    const auto last_before = [&](int64_t at) { return floor_of(at - lo); };                     // lo + i step <= at
    const auto first_behind = [&](int64_t at) { return floor_of(at - lo - wide) + 1; };         // at < lo + i step + wide
    const auto within = [&](int64_t first, int64_t last) { return (first > 0 ? first : 0) <= (last < count - 1 ? last : count - 1); };
    // b's first row and its last one
    const int64_t end = (rows(b) - 1) * (int64_t)b.step;
    if (within(first_behind(0), last_before(0)) || within(first_behind(end), last_before(end))) return true;
    // rows of a that begin and end between them: a multiple of b.step in one of the ranges
    int64_t first = last_before(0) + 1, last = first_behind(end) - 1;
    if (first < 0) first = 0;
    if (last > count - 1) last = count - 1;
    if (b.step == 0 || first > last) return false;
    if (wide >= (int64_t)b.step) return true;
    // distance from the range's begin to the next multiple, which falls by a.step from row to row
    const uint64_t m = b.step, by = a.step % m, from = (m - (uint64_t)(lo + first * step) % m) % m;
    if (from < (uint64_t)wide) return true;
    const __int128 t = clip_first_in(by, m, from - (uint64_t)wide + 1, from);
    return t >= 0 && t <= last - first;
}
// a begins where b does or before: whether an element belongs to both
static inline bool clip_meet(const clip_place &a, const clip_place &b) {
    if (b.begin >= a.end) return false;
    if (a.step != b.step) return clip_rows_meet(a, b);
    if (a.step == 0) return true;
    // as of ranges of one matrix's columns: a next row of a is there where b begins behind one's end
    const uint64_t at = (b.begin - a.begin) % a.step;
    return at < a.row || at + b.row > a.step;
}
