// Host side of linear attention with a decay for each head: checks, roles, which kernels run.
#include "tcr_attention.hpp"

#include <cmath>
#include <exception>

using namespace tcr;
using namespace tcr::layers;
using tcr::host::launched;
using tcr::host::partials_for;

namespace {

constexpr uint64_t kMostTokens = 1ull << 31;       // in all; keeps every grid and token index in range

bool supported(const tcr_attention& a) {
    const uint64_t total = a.offsets != nullptr || a.tokens == 0 ? a.tokens : (a.sequences > kMostTokens / a.tokens ? kMostTokens : a.sequences * a.tokens);
    return a.dk >= 8 && a.dk <= 256 && a.dk % 8 == 0 && a.dv >= 8 && a.dv <= 256 && a.dv % 8 == 0 && a.heads <= 65535 && total < kMostTokens &&
           a.sequences * (uint64_t)a.heads < (1ull << 26);
}

tcr_status check(const tcr_attention* a) {
    if (a == nullptr || (a->dtype != TCR_F16 && a->dtype != TCR_BF16)) return TCR_ERR_INVALID_ARG;
    if (a->heads == 0 || a->kv_heads == 0 || a->heads % a->kv_heads != 0 || a->dk == 0 || a->dv == 0) return TCR_ERR_INVALID_ARG;
    if (a->log_decay == nullptr || !on_boundary(a->log_decay, 4) || !on_boundary(a->offsets, 8)) return TCR_ERR_INVALID_ARG;
    if (!(std::fabs(a->scale) >= 1e-18f && std::fabs(a->scale) <= 1e18f)) return TCR_ERR_INVALID_ARG;
    return supported(*a) ? TCR_OK : TCR_ERR_UNSUPPORTED;
}

View view(const void* p, const int64_t stride[3], uint32_t group, bool packed) { return {p, packed ? 0 : stride[0], stride[1], stride[2], group}; }

Scan scan_of(const tcr_attention& a, const View& va, const View& vb, const View& vc, void* out, const int64_t out_stride[3], uint32_t dk, uint32_t dv) {
    Scan s = {};
    s.a = va;
    s.b = vb;
    s.c = vc;
    s.out = out;
    s.out_seq = a.offsets != nullptr ? 0 : out_stride[0];
    s.out_tok = out_stride[1];
    s.out_head = out_stride[2];
    s.st_row = dv;
    s.st_col = 1;
    s.log_decay = a.log_decay;
    s.offsets = a.offsets;
    s.sequences = a.sequences;
    s.tokens = a.tokens;
    s.total = a.offsets != nullptr ? a.tokens : a.sequences * a.tokens;
    s.out_scale = a.scale;
    s.init_mul = s.fin_mul = 1.0f;
    s.heads = a.heads;
    s.dk = dk;
    s.dv = dv;
    return s;
}

template <typename T, typename OUT>
tcr_status run(const Scan& a, hipStream_t stream) {
    const uint64_t pairs = a.sequences * a.heads;
    if (a.offsets != nullptr && a.total != 0) {
        attention_outside_kernel<OUT><<<dim3((unsigned)div_up(a.total, 64)), dim3(256), 0, stream>>>(a);
        const tcr_status st = launched("attention_outside_kernel");
        if (st != TCR_OK) return st;
    }
    if (pairs == 0) return TCR_OK;
    if (pairs * div_up(a.dv, 64) >= 1024)
        attention_step_kernel<T, 16, OUT><<<dim3((unsigned)(pairs * div_up(a.dv, 64))), dim3(kStepThreads), 0, stream>>>(a);
    else
        attention_step_kernel<T, 4, OUT><<<dim3((unsigned)(pairs * div_up(a.dv, 16))), dim3(kStepThreads), 0, stream>>>(a);
    return launched("attention_step_kernel");
}

// Out of the type of the inputs, or binary32 (`wide`).
tcr_status run(const Scan& a, uint32_t dtype, bool wide, hipStream_t stream) {
    if (dtype == TCR_F16) return wide ? run<_Float16, float>(a, stream) : run<_Float16, _Float16>(a, stream);
    return wide ? run<__bf16, float>(a, stream) : run<__bf16, __bf16>(a, stream);
}

tcr_status check_states(const void* a, const void* b) { return on_boundary(a, 16) && on_boundary(b, 16) ? TCR_OK : TCR_ERR_INVALID_ARG; }

bool odd(const void* p) { return p == nullptr || !on_boundary(p, 2); }

tcr_status forward(const tcr_attention* shape, const void* q, const void* k, const void* v, void* out, const float* state, float* final_state,
                   hipStream_t stream) {
    tcr_status st = check(shape);
    if (st != TCR_OK) return st;
    const bool any = shape->tokens != 0 && (shape->sequences != 0 || shape->offsets != nullptr);
    if ((any && (odd(q) || odd(k) || odd(v) || odd(out))) || check_states(state, final_state) != TCR_OK) return TCR_ERR_INVALID_ARG;
    const uint32_t group = shape->heads / shape->kv_heads;
    const bool packed = shape->offsets != nullptr;
    Scan s = scan_of(*shape, view(q, shape->q_stride, 1, packed), view(k, shape->k_stride, group, packed), view(v, shape->v_stride, group, packed), out,
                     shape->o_stride, shape->dk, shape->dv);
    s.init = state;
    s.fin = final_state;
    return run(s, shape->dtype, false, stream);
}

tcr_status backward(const tcr_attention* shape, const void* dout, const void* q, const void* k, const void* v, void* dq, void* dk, void* dv,
                    const float* state, const float* dfinal, float* dstate, hipStream_t stream) {
    tcr_status st = check(shape);
    if (st != TCR_OK) return st;
    const bool any = shape->tokens != 0 && (shape->sequences != 0 || shape->offsets != nullptr);
    if (any && (odd(dout) || odd(q) || odd(k) || odd(v) || odd(dq) || odd(dk) || odd(dv))) return TCR_ERR_INVALID_ARG;
    if (check_states(state, dfinal) != TCR_OK || check_states(dstate, nullptr) != TCR_OK) return TCR_ERR_INVALID_ARG;
    const tcr_attention& a = *shape;
    const uint32_t group = a.heads / a.kv_heads;
    const bool packed = a.offsets != nullptr;
    const View vq = view(q, a.q_stride, 1, packed), vk = view(k, a.k_stride, group, packed), vv = view(v, a.v_stride, group, packed),
               vo = view(dout, a.o_stride, 1, packed);
    auto contiguous = [&](int64_t (&stride)[3], uint32_t d) {
        stride[2] = d;
        stride[1] = (int64_t)a.heads * d;
        stride[0] = (int64_t)a.tokens * stride[1];
    };
    int64_t stride[3];

    // dq: the states of the forward pass, transposed
    contiguous(stride, a.dk);
    Scan s = scan_of(a, vo, vv, vk, dq, stride, a.dv, a.dk);
    s.init = state;
    s.st_row = 1;
    s.st_col = a.dv;
    st = run(s, a.dtype, false, stream);
    if (st != TCR_OK) return st;

    // dk and dv, from the last token to the first; of shared heads by way of each head's own in binary32
    float* part = nullptr;
    if (group > 1) {
        const uint64_t want = (packed ? a.tokens : a.sequences * a.tokens) * a.heads * (a.dk > a.dv ? a.dk : a.dv);
        uint64_t got = 0;
        st = partials_for(stream, want, &part, &got);
        if (st != TCR_OK) return st;
        if (got < want) return TCR_ERR_WORKSPACE;
    }
    auto pass = [&](const View& va, const View& vb, const View& vc, uint32_t rows, uint32_t cols, void* out, bool first) {
        contiguous(stride, cols);
        Scan r = scan_of(a, va, vb, vc, group > 1 ? part : out, stride, rows, cols);
        r.reverse = r.late = 1;
        r.init = dfinal;
        r.init_mul = 1.0f / a.scale;
        r.fin_mul = a.scale;
        if (first) {                     // R transposed: dv x dk
            r.st_row = 1;
            r.st_col = a.dv;
        } else {
            r.fin = dstate;
        }
        const tcr_status done = run(r, a.dtype, group > 1, stream);
        if (done != TCR_OK || group == 1) return done;
        const uint64_t count = r.total * a.kv_heads * cols;
        if (count == 0) return TCR_OK;
        const dim3 grid((unsigned)div_up(count, 256));
        if (a.dtype == TCR_F16) attention_shared_kernel<<<grid, dim3(256), 0, stream>>>(part, static_cast<_Float16*>(out), count, cols, group);
        else attention_shared_kernel<<<grid, dim3(256), 0, stream>>>(part, static_cast<__bf16*>(out), count, cols, group);
        return launched("attention_shared_kernel");
    };
    st = pass(vv, vo, vq, a.dv, a.dk, dk, true);
    if (st != TCR_OK) return st;
    return pass(vk, vq, vo, a.dk, a.dv, dv, false);
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

}  // namespace

extern "C" tcr_status tcr_linear_attention(const tcr_attention* shape, const void* q, const void* k, const void* v, void* out, const float* state,
                                           float* final_state, void* stream) {
    return guarded([&] {
        if (shape != nullptr && state != nullptr && state == final_state) return TCR_ERR_INVALID_ARG;
        return forward(shape, q, k, v, out, state, final_state, static_cast<hipStream_t>(stream));
    });
}

extern "C" tcr_status tcr_linear_attention_step(const tcr_attention* shape, const void* q, const void* k, const void* v, void* out, const float* state,
                                                float* new_state, void* stream) {
    return guarded([&] {
        if (shape != nullptr && (shape->tokens != 1 || shape->offsets != nullptr || state == nullptr || new_state == nullptr)) return TCR_ERR_INVALID_ARG;
        return forward(shape, q, k, v, out, state, new_state, static_cast<hipStream_t>(stream));
    });
}

extern "C" tcr_status tcr_linear_attention_backward(const tcr_attention* shape, const void* dout, const void* q, const void* k, const void* v, void* dq,
                                                    void* dk, void* dv, const float* state, const float* dfinal, float* dstate, void* stream) {
    return guarded([&] {
        if (dstate != nullptr && dstate == dfinal) return TCR_ERR_INVALID_ARG;
        return backward(shape, dout, q, k, v, dq, dk, dv, state, dfinal, dstate, static_cast<hipStream_t>(stream));
    });
}
