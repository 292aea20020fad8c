// Checks on the arrays of a call that the host sides of the scan and the convolution share.
#pragma once
#include <exception>
#include <type_traits>

#include "tcr_lattice.hpp"
#include "tcr_shared.hpp"

namespace tcr {
namespace layers {

inline bool missing(const void* p, uintptr_t size) { return p == nullptr || !on_boundary(p, size); }

// Tokens of all sequences, at most 2^63.
template <typename SHAPE>
uint64_t total_tokens(const SHAPE& a) {
    if (a.offsets != nullptr || a.tokens == 0) return a.tokens;
    return a.sequences > (1ull << 63) / a.tokens ? 1ull << 63 : a.sequences * a.tokens;
}

// The memory of an array of rows: its bytes, where the rows fill them without gaps.
struct Extent {
    uintptr_t from, to;
    bool whole;
};
// Rows of `wide` elements of `size` bytes for every sequence, token and group (strides in this order).
template <typename SHAPE>
Extent extent(const SHAPE& a, const void* p, const int64_t* stride, uint64_t wide, uintptr_t size, uint64_t groups = 1) {
    const uint64_t counts[3] = {a.offsets != nullptr ? 1 : a.sequences, a.tokens, groups};
    __int128 reach = wide, all = wide;             // (strides may be anything)
    bool whole = true;
    for (int i = 0; i < 3; ++i) {
        if (counts[i] > 1 && stride[i] < 0) whole = false;
        if (counts[i] > 1) reach += (__int128)(counts[i] - 1) * stride[i];
        all *= counts[i];
    }
    const uintptr_t from = reinterpret_cast<uintptr_t>(p);
    whole = whole && reach == all;
    return {from, whole ? from + (uintptr_t)((__int128)size * all) : from + size * wide, whole};
}
// Whether two of them share memory for certain.  (Rows with gaps may stand in each other's; they are only looked at where they start.)
inline bool share(const Extent& a, const Extent& b) { return a.whole && b.whole ? a.from < b.to && b.from < a.to : a.from == b.from; }
// An array without gaps against it; either may be missing or empty.
inline bool share(const Extent& a, const void* p, uint64_t bytes) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(p);
    return p != nullptr && bytes != 0 && share(a, Extent{from, from + (uintptr_t)bytes, true});
}

// Whether rows of `wide` elements that a call writes share elements with each other.
template <typename SHAPE>
bool rows_meet(const SHAPE& a, const int64_t* stride, uint64_t wide) {
    return lattice_meets(a.offsets == nullptr ? a.sequences : 1, a.offsets == nullptr ? stride[0] : 0, a.tokens, stride[1], wide);
}

// Whether two arrays without gaps share memory, either of which may be missing.
inline bool arrays_share(const void* x, uint64_t x_bytes, const void* y, uint64_t y_bytes) {
    if (x == nullptr || y == nullptr) return false;
    const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
    return p == q || (p < q + y_bytes && q < p + x_bytes);
}

// No exception leaves the library.
template <typename F>
tcr_status guarded(F f) {
    try {
        return f();
    } catch (const std::exception&) {
        return TCR_ERR_WORKSPACE;
    }
}

}  // namespace layers
}  // namespace tcr
