// Host side of the short causal convolution: checks and launch shapes.
#include "tcr_conv.hpp"
#include "tcr_operands.hpp"

using namespace tcr;
using namespace tcr::layers;
using tcr::host::launched;
using tcr::host::partials_for;

namespace {

constexpr uint64_t kMostTokens = 1ull << 31;
constexpr uint32_t kMostChannels = 1u << 20;

// Threads that a call is cut for, and tokens of a run at most (the W - 1 in front of it are loaded once more).
constexpr uint64_t kFillThreads = 1u << 18;
constexpr uint32_t kLongRun = 32, kShortRun = 4;
// Workgroups of the gradients: three for each compute unit, which with four taps in 16 bits are there at once (165 registers), each with runs as long as it takes.  8191 tokens x 4096 channels:
// 55 us, and 5 for the sums; with four workgroups, of which one waits for the others, 62 and 6.  (Four taps in binary32 take 180 registers and have two there at once, two taps in 16 bits
// would have four.  Runs of every sequence are rounded up by themselves, and workgroups by the slabs of channels, so that a few may be left for a second turn.  Neither was measured.)
constexpr uint64_t kGradBlocks = 768;

uint64_t spans_of(const Conv& a) { return a.offsets != nullptr ? 1 : a.sequences; }

void cut(Conv& a, int vec, uint64_t threads, uint64_t longest) {
    const uint64_t cols = div_up(a.channels, vec);
    a.lanes = 64;
    while (a.lanes > 1 && a.lanes / 2 >= cols) a.lanes /= 2;
    uint64_t run = div_up(spans_of(a) * a.span * cols, threads);
    if (run > longest) run = longest;
    a.run = run < kShortRun ? kShortRun : (uint32_t)run;
    a.runs = (uint32_t)div_up(a.span, a.run);
    if (a.runs == 0) a.runs = 1;
}

template <typename T, int W>
tcr_status run(Conv a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    cut(a, V, kFillThreads, kLongRun);
    const uint64_t slabs = div_up(div_up(a.channels, V), a.lanes), blocks = slabs * div_up(spans_of(a) * a.runs, kConvThreads / a.lanes);
    if (blocks == 0) return TCR_OK;
    if (blocks > 0xffffffffu) return TCR_ERR_UNSUPPORTED;
    if (a.channels % V == 0) conv_kernel<T, V, W, true><<<grid_of(blocks), kConvThreads, 0, s>>>(a);
    else conv_kernel<T, V, W, false><<<grid_of(blocks), kConvThreads, 0, s>>>(a);
    return launched("conv_kernel");
}

template <typename T, int W>
tcr_status step(Conv a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const uint64_t blocks = div_up(a.sequences * div_up(a.channels, V), kConvThreads);
    if (blocks == 0) return TCR_OK;
    if (a.channels % V == 0) conv_step_kernel<T, V, W, true><<<grid_of(blocks), kConvThreads, 0, s>>>(a);
    else conv_step_kernel<T, V, W, false><<<grid_of(blocks), kConvThreads, 0, s>>>(a);
    return launched("conv_step_kernel");
}

template <typename T, int W>
tcr_status gradients(ConvGrad g, T* dweight, T* dbias, hipStream_t s) {
    constexpr int V = 4;
    cut(g.c, V, kGradBlocks * kConvThreads, kMostTokens);
    const uint64_t slabs = div_up(div_up(g.c.channels, V), g.c.lanes), places = div_up(spans_of(g.c) * g.c.runs, kConvThreads / g.c.lanes);
    const uint64_t each = (uint64_t)(W + 1) * g.c.channels;
    uint64_t parts = div_up(kGradBlocks, slabs), got = 0;
    if (parts > places) parts = places != 0 ? places : 1;
    const tcr_status st = partials_for(s, parts * each, each, &g.part, &got);
    if (st != TCR_OK) return st;
    g.parts = (uint32_t)(got / each);
    if (g.c.channels % V == 0) conv_grad_kernel<T, V, W, true><<<grid_of(slabs * g.parts), kConvThreads, 0, s>>>(g);
    else conv_grad_kernel<T, V, W, false><<<grid_of(slabs * g.parts), kConvThreads, 0, s>>>(g);
    if (launched("conv_grad_kernel") != TCR_OK) return TCR_ERR_HIP;
    conv_parts_kernel<T, W><<<grid_of(div_up(each, 64)), kConvThreads, 0, s>>>(g.part, dweight, dbias, g.c.channels, g.parts);
    return launched("conv_parts_kernel");
}

template <typename F>
tcr_status by_width(uint32_t width, F f) {
    return width == 2 ? f(std::integral_constant<int, 2>()) : width == 3 ? f(std::integral_constant<int, 3>()) : f(std::integral_constant<int, 4>());
}
template <typename F>
tcr_status by_type(uint32_t dtype, F f) {
    return dtype == TCR_F16 ? f(_Float16()) : dtype == TCR_BF16 ? f(__bf16()) : f(float());
}

tcr_status check(const tcr_convolution* a) {
    if (a == nullptr || a->dtype > TCR_F32 || a->channels == 0 || a->width == 0 || a->activation > 1 || !on_boundary(a->offsets, 8)) return TCR_ERR_INVALID_ARG;
    if (a->width < 2 || a->width > 4 || a->channels > kMostChannels || a->sequences >= kMostTokens || total_tokens(*a) >= kMostTokens) return TCR_ERR_UNSUPPORTED;
    return TCR_OK;
}

Conv arguments(const tcr_convolution& a, const void* x, const void* weight, const void* bias, const void* state) {
    const bool packed = a.offsets != nullptr;
    Conv c = {};
    c.x = x;
    c.weight = weight;
    c.bias = bias;
    c.state = state;
    c.offsets = a.offsets;
    c.x_seq = packed ? 0 : a.x_stride[0];
    c.x_tok = a.x_stride[1];
    c.out_seq = packed ? 0 : a.o_stride[0];
    c.out_tok = a.o_stride[1];
    c.sequences = a.sequences;
    c.span = (uint32_t)a.tokens;
    c.channels = a.channels;
    c.act = a.activation;
    return c;
}

uintptr_t size_of(const tcr_convolution& a) { return a.dtype == TCR_F32 ? 4 : 2; }
uint64_t state_bytes(const tcr_convolution& a) { return a.sequences * (a.width - 1) * a.channels * size_of(a); }

tcr_status forward(const tcr_convolution* shape, const void* x, const void* weight, const void* bias, void* out, const void* state, void* last, bool one,
                   hipStream_t stream) {
    const tcr_status st = check(shape);
    if (st != TCR_OK) return st;
    const tcr_convolution& a = *shape;
    const uintptr_t size = size_of(a);
    if (missing(weight, size) || !on_boundary(bias, size) || !on_boundary(state, size) || !on_boundary(last, size)) return TCR_ERR_INVALID_ARG;
    if (total_tokens(a) != 0) {
        if (missing(x, size) || missing(out, size)) return TCR_ERR_INVALID_ARG;
        if (rows_meet(a, a.o_stride, a.channels)) return TCR_ERR_INVALID_ARG;
        // (the inputs in front of a run are another thread's, and so are the states)
        const Extent written = extent(a, out, a.o_stride, a.channels, size), read = extent(a, x, a.x_stride, a.channels, size);
        if (share(written, read) || share(written, state, state_bytes(a)) || share(written, last, state_bytes(a))) return TCR_ERR_INVALID_ARG;
        if (!one && share(read, last, state_bytes(a))) return TCR_ERR_INVALID_ARG;
    }
    if ((state != last || !one) && arrays_share(state, state_bytes(a), last, state_bytes(a))) return TCR_ERR_INVALID_ARG;
    Conv c = arguments(a, x, weight, bias, state);
    c.out = out;
    c.fin = last;
    return by_type(a.dtype, [&](auto t) {
        return by_width(a.width, [&](auto w) { return one ? step<decltype(t), w()>(c, stream) : run<decltype(t), w()>(c, stream); });
    });
}

tcr_status backward(const tcr_convolution* shape, const void* dout, const void* x, const void* weight, const void* bias, void* dx, void* dweight, void* dbias,
                    const void* state, const void* dfinal, void* dstate, hipStream_t stream) {
    const tcr_status st = check(shape);
    if (st != TCR_OK) return st;
    const tcr_convolution& a = *shape;
    const uintptr_t size = size_of(a);
    if (missing(weight, size) || missing(dweight, size) || !on_boundary(bias, size) || !on_boundary(dbias, size) || !on_boundary(state, size) ||
        !on_boundary(dfinal, size) || !on_boundary(dstate, size))
        return TCR_ERR_INVALID_ARG;
    const uint64_t total = total_tokens(a);
    if (total != 0) {
        if (missing(dout, size) || missing(x, size) || missing(dx, size)) return TCR_ERR_INVALID_ARG;
        const int64_t rows[2] = {(int64_t)(a.tokens * a.channels), (int64_t)a.channels};
        const Extent written = extent(a, dx, rows, a.channels, size);
        if (share(written, extent(a, x, a.x_stride, a.channels, size)) || share(written, extent(a, dout, a.o_stride, a.channels, size))) return TCR_ERR_INVALID_ARG;
    }
    if (arrays_share(dstate, state_bytes(a), state, state_bytes(a)) || arrays_share(dstate, state_bytes(a), dfinal, state_bytes(a))) return TCR_ERR_INVALID_ARG;
    ConvGrad g = {};
    g.c = arguments(a, x, weight, bias, state);
    g.c.out = const_cast<void*>(dout);
    g.dfinal = dfinal;
    g.dx = dx;
    g.dstate = dstate;
    return by_type(a.dtype, [&](auto t) {
        typedef decltype(t) T;
        return by_width(a.width, [&](auto w) { return gradients<T, w()>(g, static_cast<T*>(dweight), static_cast<T*>(dbias), stream); });
    });
}

}  // namespace

extern "C" tcr_status tcr_causal_conv(const tcr_convolution* shape, const void* x, const void* weight, const void* bias, void* out, const void* state,
                                      void* final_state, void* stream) {
    return guarded([&] { return forward(shape, x, weight, bias, out, state, final_state, false, static_cast<hipStream_t>(stream)); });
}

extern "C" tcr_status tcr_causal_conv_step(const tcr_convolution* shape, const void* x, const void* weight, const void* bias, void* out, const void* state,
                                           void* new_state, void* stream) {
    return guarded([&] {
        if (shape != nullptr && (shape->tokens != 1 || shape->offsets != nullptr || state == nullptr || new_state == nullptr)) return TCR_ERR_INVALID_ARG;
        return forward(shape, x, weight, bias, out, state, new_state, true, static_cast<hipStream_t>(stream));
    });
}

extern "C" tcr_status tcr_causal_conv_backward(const tcr_convolution* shape, const void* dout, const void* x, const void* weight, const void* bias, void* dx,
                                               void* dweight, void* dbias, const void* state, const void* dfinal, void* dstate, void* stream) {
    return guarded([&] { return backward(shape, dout, x, weight, bias, dx, dweight, dbias, state, dfinal, dstate, static_cast<hipStream_t>(stream)); });
}
