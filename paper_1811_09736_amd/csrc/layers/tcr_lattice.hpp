// Whether rows that a call writes stand in each other's place, whatever their strides (no HIP in here).
#pragma once
#include <stdint.h>

namespace tcr {
namespace layers {

// The least x >= 0 with low <= a x mod m <= high (0 <= a < m, 0 <= low <= high < m), or -1: Euclid's algorithm.  Of a x = m y + r with r in [low, high], where no multiple of a lies in
// [low, high] itself, y is the least with -m y mod a in [low mod a, high mod a].
inline __int128 first_multiple_in(__int128 a, __int128 m, __int128 low, __int128 high) {
    if (low == 0) return 0;
    if (a == 0) return -1;
    if (2 * a > m) return first_multiple_in(m - a, m, m - high, m - low);      // (a reflected; halves at least with every second step)
    const __int128 x = (low + a - 1) / a;
    if (a * x <= high) return x;
    const __int128 y = first_multiple_in((a - m % a) % a, a, low % a, high % a);
    return y < 0 ? -1 : (low + m * y + a - 1) / a;
}

// Of rows of `wide` elements at i * step0 + j * step1, i < count0, j < count1: whether any two of them share an element.
inline bool lattice_meets(uint64_t count0, int64_t step0, uint64_t count1, int64_t step1, uint64_t wide) {
    if (count0 == 0 || count1 == 0 || wide == 0) return false;
    __int128 large = step0 < 0 ? -(__int128)step0 : step0, small = step1 < 0 ? -(__int128)step1 : step1, many_large = count0, many_small = count1;
    const __int128 w = wide;
    if ((count0 > 1 && large < w) || (count1 > 1 && small < w)) return true;
    if (count0 == 1 || count1 == 1) return false;
    if (large < small) {
        __int128 t = large;
        large = small;
        small = t;
        t = many_large;
        many_large = many_small;
        many_small = t;
    }
    if (large >= (many_small - 1) * small + w) return false;       // (one within the other: what slices and transpositions of an array are)
    // The first i >= 1 for which i * large is less than w away from a multiple of `small`: i = x + 1 with (x large + from) mod small < 2 w - 1.
    const __int128 from = (large + w - 1) % small, room = 2 * w - 1;
    __int128 x = 0;
    if (from >= room && room < small) x = first_multiple_in(large % small, small, small - from, small - from + room - 1);
    if (x < 0 || x + 1 >= many_large) return false;
    return ((x + 1) * large - w) / small + 1 < many_small;         // (the first of the multiples that near)
}

}  // namespace layers
}  // namespace tcr
