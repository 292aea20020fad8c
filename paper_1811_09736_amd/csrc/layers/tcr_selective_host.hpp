// The checks of the selective scan's calls, forwards and backwards.
#pragma once
#include "tcr_operands.hpp"
#include "tcr_selective.hpp"

namespace tcr {
namespace layers {

constexpr uint64_t kMostTokens = 1ull << 31;       // in all; keeps every token index in range
constexpr uint32_t kMostStates = 64, kMostChannels = 1u << 20;
constexpr uint64_t kMostBlocks = 0xffffffffu;      // workgroups of a launch

inline tcr_status check(const tcr_selective* a) {
    if (a == nullptr || a->dtype > TCR_F32 || a->channels == 0 || a->states == 0 || a->groups == 0 || a->channels % a->groups != 0 || a->softplus > 1)
        return TCR_ERR_INVALID_ARG;
    if (a->a == nullptr || !on_boundary(a->a, 4) || !on_boundary(a->skip, 4) || !on_boundary(a->dt_bias, 4) || !on_boundary(a->offsets, 8)) return TCR_ERR_INVALID_ARG;
    if (a->states > kMostStates || a->channels > kMostChannels || a->sequences >= kMostTokens || total_tokens(*a) >= kMostTokens) return TCR_ERR_UNSUPPORTED;
    return TCR_OK;
}

inline Operand operand(const void* p, const int64_t* stride, bool packed, int64_t group = 0) { return {p, packed ? 0 : stride[0], stride[1], group}; }

inline Selective arguments(const tcr_selective& a, const void* x, const void* dt, const void* b, const void* c, const void* gate) {
    const bool packed = a.offsets != nullptr;
    Selective s = {};
    s.x = operand(x, a.x_stride, packed);
    s.dt = operand(dt, a.dt_stride, packed);
    s.gate = operand(gate, a.gate_stride, packed);
    s.b = operand(b, a.b_stride, packed, a.b_stride[2]);
    s.c = operand(c, a.c_stride, packed, a.c_stride[2]);
    s.out_seq = packed ? 0 : a.o_stride[0];
    s.out_tok = a.o_stride[1];
    s.a = a.a;
    s.skip = a.skip;
    s.bias = a.dt_bias;
    s.offsets = a.offsets;
    s.sequences = a.sequences;
    s.span = (uint32_t)a.tokens;
    s.channels = a.channels;
    s.states = a.states;
    s.groups = a.groups;
    s.softplus = a.softplus;
    return s;
}

}  // namespace layers
}  // namespace tcr
