// Where the sequences of a call's tokens begin and end, and the activations: what the kernels of the scan and of the convolution share.
#pragma once
#include "tcr_shared.hpp"

namespace tcr {
namespace layers {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
// 1 / (1 + exp(-x)): from 0 at minus infinity to 1.
__device__ __forceinline__ float sigmoid_of(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-x)); }

// Where the sequences of a span begin and end.  bound(i) never leaves the span, whatever the offsets hold.
struct Bounds {
    const uint64_t* offsets;
    uint32_t count, span;
    __device__ __forceinline__ uint32_t at(uint32_t i) const {
        const uint64_t o = offsets[i];
        return o < span ? (uint32_t)o : span;
    }
    // How many of the count + 1 bounds are at most t.
    __device__ __forceinline__ uint32_t upto(uint32_t t) const {
        uint32_t low = 0, high = count + 1;
        while (low < high) {
            const uint32_t mid = low + (high - low) / 2;
            if (at(mid) <= t) low = mid + 1;
            else high = mid;
        }
        return low;
    }
};

// The sequence that a token of a span stands in, and where the next bound is.
struct Place {
    uint32_t seq, next;                        // next: the first bound behind the token (none: ~0)
    uint32_t start;                            // the last bound that is not behind it (none: 0)
    bool inside;                               // whether it stands in a sequence at all
    __device__ __forceinline__ void find(const Bounds& b, uint32_t span_index, uint32_t t) {
        if (b.offsets == nullptr) {
            seq = span_index, start = 0, next = b.span, inside = true;
            return;
        }
        const uint32_t n = b.upto(t);
        inside = n >= 1 && n <= b.count;
        seq = n - 1;
        start = n >= 1 ? b.at(n - 1) : 0;
        next = n <= b.count ? b.at(n) : ~0u;
    }
    // Over the bound at t, and over empty sequences there.
    __device__ __forceinline__ void pass(const Bounds& b, uint32_t t) {
        do ++seq;
        while (seq < b.count && b.at(seq + 1) <= t);
        inside = seq < b.count;
        start = t;
        next = inside ? b.at(seq + 1) : ~0u;
    }
};

}  // namespace layers
}  // namespace tcr
