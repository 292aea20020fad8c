// Host side of the selective scan: checks, how it is cut, which kernels run.
#include "tcr_selective_host.hpp"

using namespace tcr;
using namespace tcr::layers;
using tcr::host::launched;
using tcr::host::partials_for;

namespace {

// Wavefronts that a scan is cut for -- four on each SIMD: 8192 tokens x 4096 channels x 16 states, bfloat16, 272 us, with two 325, with eight 274 -- and chunks of a sequence at
// most: each looks through the ones in front of it.  Four is what the output kernels' registers allow in 16 bits up to 16 states; with more states, and in binary32 from 8, three, with 64 two
// or one, and channels that do not divide 1024 workgroups leave a few over: the last ones start when others have ended.  (Only the case above was measured.)
constexpr uint64_t kFillWaves = 4096, kMostChunks = 64;

template <typename T, int K, int P>
tcr_status run(Selective s, hipStream_t stream) {
    constexpr uint32_t kStates = K * P, kChannels = Slab<P>::kChannels, kTile = 8 * P;
    const uint64_t spans = s.offsets != nullptr ? 1 : s.sequences;
    if (spans == 0) return TCR_OK;
    s.slabs = (uint32_t)div_up(s.channels / s.groups, kChannels);
    const uint64_t slabs = (uint64_t)s.slabs * s.groups, all = slabs * kChannels, each = spans * all * (kStates + 1);
    uint64_t chunks = div_up(kFillWaves / 4, spans * slabs);
    if (chunks > kMostChunks) chunks = kMostChunks;
    auto cut = [&] {
        s.length = (uint32_t)(div_up(div_up(s.span, chunks), kTile) * kTile);
        if (s.length == 0) s.length = kTile;
        s.per_span = (uint32_t)div_up(s.span, s.length);
        if (s.per_span == 0) s.per_span = 1;
    };
    cut();
    if (slabs * spans * s.per_span > kMostBlocks) return TCR_ERR_UNSUPPORTED;
    if (s.per_span > 1) {
        uint64_t got = 0;
        const tcr_status st = partials_for(stream, (s.per_span - 1) * each, 0, &s.ends, &got);
        if (st != TCR_OK) return st;
        if (got < (s.per_span - 1) * each) {
            chunks = got / each + 1;
            cut();
        }
        s.sums = s.ends + (s.per_span - 1) * spans * all * kStates;
    }
    if (s.per_span > 1) {
        const uint64_t blocks = slabs * spans * (s.per_span - 1);
        selective_kernel<T, K, P, false><<<grid_of(blocks), kScanThreads, 0, stream>>>(s, (uint32_t)blocks);
        if (launched("selective_kernel<states>") != TCR_OK) return TCR_ERR_HIP;
    }
    const uint64_t blocks = slabs * spans * s.per_span;
    selective_kernel<T, K, P, true><<<grid_of(blocks), kScanThreads, 0, stream>>>(s, (uint32_t)blocks);
    return launched("selective_kernel");
}

template <typename T>
tcr_status run(const Selective& s, hipStream_t stream) {
    if (s.states <= 4) return run<T, 4, 1>(s, stream);
    if (s.states <= 8) return run<T, 4, 2>(s, stream);
    if (s.states <= 16) return run<T, 4, 4>(s, stream);
    if (s.states <= 32) return run<T, 4, 8>(s, stream);
    return run<T, 4, 16>(s, stream);
}

// Wavefronts from which on a thread takes two sequences: those that fill the chip.  4096 channels x 16 states, one / two / four: 32 sequences 6.9 / 6.9 / 8.8 us,
// 256 sequences 43.5 / 34 / 36.5 us (143 MB).
constexpr uint64_t kStepWaves = 2048;

template <typename T, int P>
tcr_status step(const Selective& s, hipStream_t stream) {
    const uint32_t whole = s.states == 4 * P && on_boundary(s.state, 16) && on_boundary(s.fin, 16);
    const uint64_t slabs = div_up(s.channels, kScanThreads / P), blocks = s.sequences * slabs;
    if (blocks == 0) return TCR_OK;
    if (blocks > kMostBlocks) return TCR_ERR_UNSUPPORTED;
    if (blocks * (kScanThreads / 64) < kStepWaves) selective_step_kernel<T, P, 1><<<grid_of(blocks), kScanThreads, 0, stream>>>(s, whole);
    else selective_step_kernel<T, P, 2><<<grid_of(slabs * div_up(s.sequences, 2)), kScanThreads, 0, stream>>>(s, whole);
    return launched("selective_step_kernel");
}
template <typename T>
tcr_status step(const Selective& s, hipStream_t stream) {
    if (s.states <= 4) return step<T, 1>(s, stream);
    if (s.states <= 8) return step<T, 2>(s, stream);
    if (s.states <= 16) return step<T, 4>(s, stream);
    if (s.states <= 32) return step<T, 8>(s, stream);
    return step<T, 16>(s, stream);
}

tcr_status forward(const tcr_selective* shape, const void* x, const void* dt, const void* b, const void* c, const void* gate, void* out, const float* state,
                   float* last, bool one, hipStream_t stream) {
    const tcr_status st = check(shape);
    if (st != TCR_OK) return st;
    const tcr_selective& a = *shape;
    const uintptr_t size = a.dtype == TCR_F32 ? 4 : 2;
    if (!on_boundary(state, 4) || !on_boundary(last, 4)) return TCR_ERR_INVALID_ARG;
    const uint64_t bytes = 4 * a.sequences * (uint64_t)a.channels * a.states;
    if (total_tokens(a) != 0) {
        if (missing(x, size) || missing(dt, size) || missing(b, size) || missing(c, size) || missing(out, size) || !on_boundary(gate, size)) return TCR_ERR_INVALID_ARG;
        if (rows_meet(a, a.o_stride, a.channels)) return TCR_ERR_INVALID_ARG;
        // (other workgroups read what one has written out for: b and c, and in the states' kernel all of them)
        const Extent written = extent(a, out, a.o_stride, a.channels, size);
        if (share(written, state, bytes) || share(written, last, bytes)) return TCR_ERR_INVALID_ARG;
        for (const Extent& read : {extent(a, x, a.x_stride, a.channels, size), extent(a, dt, a.dt_stride, a.channels, size), extent(a, b, a.b_stride, a.states, size, a.groups),
                                   extent(a, c, a.c_stride, a.states, size, a.groups), extent(a, gate, a.gate_stride, a.channels, size)})
            if (read.from != 0 && (share(written, read) || (!one && share(read, last, bytes)))) return TCR_ERR_INVALID_ARG;
    }
    if ((state != last || !one) && arrays_share(state, bytes, last, bytes)) return TCR_ERR_INVALID_ARG;
    Selective s = arguments(a, x, dt, b, c, gate);
    s.out = out;
    s.state = state;
    s.fin = last;
    if (one) return a.dtype == TCR_F16 ? step<_Float16>(s, stream) : a.dtype == TCR_BF16 ? step<__bf16>(s, stream) : step<float>(s, stream);
    return a.dtype == TCR_F16 ? run<_Float16>(s, stream) : a.dtype == TCR_BF16 ? run<__bf16>(s, stream) : run<float>(s, stream);
}

}  // namespace

extern "C" tcr_status tcr_selective_scan(const tcr_selective* shape, const void* x, const void* dt, const void* b, const void* c, const void* gate, void* out,
                                         const float* state, float* final_state, void* stream) {
    return guarded([&] { return forward(shape, x, dt, b, c, gate, out, state, final_state, false, static_cast<hipStream_t>(stream)); });
}

extern "C" tcr_status tcr_selective_scan_step(const tcr_selective* shape, const void* x, const void* dt, const void* b, const void* c, const void* gate, void* out,
                                              const float* state, float* new_state, void* stream) {
    return guarded([&] {
        if (shape != nullptr && (shape->tokens != 1 || shape->offsets != nullptr || state == nullptr || new_state == nullptr)) return TCR_ERR_INVALID_ARG;
        return forward(shape, x, dt, b, c, gate, out, state, new_state, true, static_cast<hipStream_t>(stream));
    });
}
