// Host side of the selective scan's gradients: checks, workspace, launches.
#include "tcr_selective_grad.hpp"
#include "tcr_selective_host.hpp"

using namespace tcr;
using namespace tcr::layers;
using tcr::host::launched;
using tcr::host::partials_for;

namespace {

template <typename T, int P>
tcr_status run(SelectiveGrad g, hipStream_t stream) {
    constexpr uint64_t kStates = 4 * P, kChannels = Slab<P>::kChannels, kTile = kGradTile<P>;
    Selective& s = g.s;
    const uint64_t spans = s.offsets != nullptr ? 1 : s.sequences, tokens = spans * s.span;
    s.slabs = (uint32_t)div_up(s.channels / s.groups, kChannels);
    s.length = kTile;
    s.per_span = s.span != 0 ? (uint32_t)div_up(s.span, kTile) : 1;
    const uint64_t slabs = (uint64_t)s.slabs * s.groups, all = slabs * kChannels, chunks = spans * s.per_span;
    if (slabs * chunks > kMostBlocks) return TCR_ERR_UNSUPPORTED;
    // (all of it in front of the first launch: a call that lacks room has done nothing)
    const uint64_t sizes[] = {chunks * all * kStates, chunks * all * kStates, chunks * all, chunks * all * 2, slabs * tokens * 2 * kStates, chunks};
    uint64_t need = 0, got = 0;
    for (uint64_t n : sizes) need += n;
    float* room = nullptr;
    const tcr_status st = partials_for(stream, need, need, &room, &got);
    if (st != TCR_OK) return st;
    s.ends = room;
    g.back = s.ends + sizes[0];
    s.sums = g.back + sizes[1];
    g.means = s.sums + sizes[2];
    g.shares = g.means + sizes[3];
    g.closed = s.offsets != nullptr ? reinterpret_cast<uint32_t*>(g.shares + sizes[4]) : nullptr;
    const uint64_t blocks = slabs * chunks;
    if (blocks != 0) {
        if (s.per_span > 1) {
            selective_parts_kernel<T, P><<<grid_of(blocks), kScanThreads, 0, stream>>>(g, (uint32_t)blocks);
            if (launched("selective_parts_kernel") != TCR_OK) return TCR_ERR_HIP;
            dim3 columns = grid_of(div_up(spans * all * kStates, 64));
            columns.z = 2;
            selective_carry_kernel<kStates><<<columns, 64 * kCarryLines, 0, stream>>>(g, all);
            if (launched("selective_carry_kernel") != TCR_OK) return TCR_ERR_HIP;
        }
        selective_grad_kernel<T, P><<<grid_of(blocks), kScanThreads, 0, stream>>>(g, (uint32_t)blocks);
        if (launched("selective_grad_kernel") != TCR_OK) return TCR_ERR_HIP;
    }
    if (tokens != 0) {
        selective_shares_kernel<T, (int)kStates><<<grid_of(div_up(tokens * s.groups * 2 * kStates, kScanThreads)), kScanThreads, 0, stream>>>(g, tokens);
        if (launched("selective_shares_kernel") != TCR_OK) return TCR_ERR_HIP;
    }
    selective_means_kernel<(int)kStates><<<grid_of(div_up(all * (kStates + 2), 64)), 1024, 0, stream>>>(g, all, chunks);
    return launched("selective_means_kernel");
}

template <typename T>
tcr_status run(const SelectiveGrad& g, hipStream_t stream) {
    if (g.s.states <= 4) return run<T, 1>(g, stream);
    if (g.s.states <= 8) return run<T, 2>(g, stream);
    if (g.s.states <= 16) return run<T, 4>(g, stream);
    if (g.s.states <= 32) return run<T, 8>(g, stream);
    return run<T, 16>(g, stream);
}

tcr_status backward(const tcr_selective* shape, const void* dout, const void* x, const void* dt, const void* b, const void* c, const void* gate, void* dx,
                    void* ddt, float* da, void* db, void* dc, float* dskip, void* dgate, float* dbias, const float* state, const float* dfinal, float* dstate,
                    hipStream_t stream) {
    const tcr_status st = check(shape);
    if (st != TCR_OK) return st;
    const tcr_selective& a = *shape;
    const uintptr_t size = a.dtype == TCR_F32 ? 4 : 2;
    if (missing(da, 4) || !on_boundary(dskip, 4) || !on_boundary(dbias, 4) || !on_boundary(state, 4) || !on_boundary(dfinal, 4) || !on_boundary(dstate, 4))
        return TCR_ERR_INVALID_ARG;
    if ((dgate != nullptr) != (gate != nullptr)) return TCR_ERR_INVALID_ARG;
    const uint64_t states = 4 * a.sequences * (uint64_t)a.channels * a.states;
    if (arrays_share(dstate, states, state, states) || arrays_share(dstate, states, dfinal, states)) return TCR_ERR_INVALID_ARG;
    if (total_tokens(a) != 0) {
        for (const void* p : {dout, x, dt, b, c, (const void*)dx, (const void*)ddt, (const void*)db, (const void*)dc})
            if (missing(p, size)) return TCR_ERR_INVALID_ARG;
        if (!on_boundary(gate, size) || !on_boundary(dgate, size)) return TCR_ERR_INVALID_ARG;
    }
    SelectiveGrad g = {};
    g.s = arguments(a, x, dt, b, c, gate);
    g.s.out = const_cast<void*>(dout);
    g.s.state = state;
    g.dfinal = dfinal;
    g.dx = dx;
    g.ddt = ddt;
    g.db = db;
    g.dc = dc;
    g.dgate = dgate;
    g.da = da;
    g.dskip = dskip;
    g.dbias = dbias;
    g.dstate = dstate;
    return a.dtype == TCR_F16 ? run<_Float16>(g, stream) : a.dtype == TCR_BF16 ? run<__bf16>(g, stream) : run<float>(g, stream);
}

}  // namespace

extern "C" tcr_status tcr_selective_scan_backward(const tcr_selective* shape, const void* dout, const void* x, const void* dt, const void* b, const void* c,
                                                  const void* gate, void* dx, void* ddt, float* da, void* db, void* dc, float* dskip, void* dgate,
                                                  float* ddt_bias, const float* state, const float* dfinal, float* dstate, void* stream) {
    return guarded([&] {
        return backward(shape, dout, x, dt, b, c, gate, dx, ddt, da, db, dc, dskip, dgate, ddt_bias, state, dfinal, dstate, static_cast<hipStream_t>(stream));
    });
}
