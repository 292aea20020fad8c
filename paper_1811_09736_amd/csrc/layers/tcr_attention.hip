// Host side of linear attention with a decay for each head: checks, roles, which kernels run.
#include "tcr_attention.hpp"
#include "tcr_attention_chunk.hpp"

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

// Tokens of a sequence up to which its states go from token to token in registers, each token a pass over them, and not through a chunk's products, which take
// the same for 1 and for 32 tokens.  16 heads of 128 x 128, steps / chunk: 1 sequence, 4 tokens 6.9 / 9.1 us, 8 tokens 10.3 / 9.1;
// 256 sequences, 2 tokens 129 / 127, 4 tokens 177 / 129.
constexpr uint64_t kStepTokens = 2, kFewStepTokens = 4, kFewPairs = 32;
constexpr uint64_t kWholeChunks = 2;
// Blocks of a sequence up to which each adds up the states in front of it by itself, without a kernel for the carries.  16 heads of 128 x 128: 4 x 2048 tokens in
// 8 blocks each 62 us, with that kernel 70; 2048 tokens in 16 blocks 33.2 and 32.3.  States that are read transposed are read in pieces of 16 bytes: once, not for each block.
constexpr uint32_t kDirectBlocks = 8;
// Wavefronts that a launch is cut for: two on each SIMD, or four where blocks stay long, for whose states' bytes more of them make up.  16 heads of 128 x 128,
// two / four: 2 x 4096 tokens, blocks of 512 / 256 tokens 65 / 75 us; 8 x 2048 tokens, 1024 / 512 tokens 115 / 104; 32768 tokens, 2048 / 1024 tokens 235 / 225.
constexpr uint64_t kFillWaves = 2048, kLongChunks = 16;
// Floats of states between blocks that a call asks for at most.  Blocks are cut for the workgroups that fill the chip, each sequence into as many, so sequences and heads that
// come close to that number by themselves would get twice of it: batches of 256 x 256 states 128 MiB.
constexpr uint64_t kMostStates = (64ull << 20) / 4;

// Workgroups for a kernel whose workgroups take the place of others behind the last.
unsigned at_most(uint64_t blocks) { return (unsigned)(blocks < kGridRow ? blocks : kGridRow); }

template <typename T, typename OUT>
tcr_status run_steps(const Scan& a, hipStream_t stream) {
    if (a.offsets != nullptr && a.total != 0) {
        attention_outside_kernel<OUT><<<dim3(at_most(div_up(a.total, 64))), dim3(256), 0, stream>>>(a);
        if (launched("attention_outside_kernel") != TCR_OK) return TCR_ERR_HIP;
    }
    const uint64_t pairs = a.sequences * a.heads;
    if (pairs == 0) return TCR_OK;
    if (pairs * div_up(a.dv, 64) >= 1024)
        attention_step_kernel<T, 16, OUT><<<grid_of(pairs * div_up(a.dv, 64)), dim3(kStepThreads), 0, stream>>>(a);
    else
        attention_step_kernel<T, 4, OUT><<<dim3((unsigned)(pairs * div_up(a.dv, 16))), dim3(kStepThreads), 0, stream>>>(a);
    return launched("attention_step_kernel");
}

// The kernel that takes a pair of widths: rows and columns of S that a workgroup holds, tokens of a chunk, wavefronts.
struct ChunkShape {
    uint32_t rows, cols, chunk, waves;
};
ChunkShape chunk_shape(uint32_t dk, uint32_t dv) {
    if (dk > 128) return {256, 64, 32, 4};
    return {dk <= 64 ? 64u : 128u, dv <= 64 ? 64u : 128u, 64, dv <= 64 ? 4u : 8u};
}

// Memory for a call's states between blocks: the stream's workspace, or what the caller of run() sets aside.  `shared`: the states serve a second scan,
// which is `turned`: it finds them there, transposed.
struct Room {
    bool given = false, shared = false, turned = false;
    float* floats = nullptr;
    uint64_t count = 0;
};

// How a scan is cut: as many blocks as fill the chip, or as there are chunks or pairs of them; fewer where `most` floats, or kMostStates, do not hold their states.
// *need: the floats that these blocks want.
Blocks cut(const Scan& a, const ChunkShape& shape, uint64_t most, uint64_t* need) {
    if (most > kMostStates) most = kMostStates;
    const uint64_t slabs = div_up(a.dv, shape.cols), units = a.heads * slabs;
    const uint64_t spans = a.offsets != nullptr ? 1 : a.sequences;
    // (per block and unit a state, per block and head what is kept, two floats)
    const uint64_t each = units * shape.rows * shape.cols + 2 * a.heads;
    Blocks b = {};
    const uint64_t span = a.offsets != nullptr ? a.total : a.tokens;
    const uint64_t chunks = div_up(span, shape.chunk), pairs = div_up(chunks, 2);
    uint64_t per_span = div_up(2 * kFillWaves / shape.waves, units * spans);
    if (chunks < per_span * kLongChunks) per_span = div_up(kFillWaves / shape.waves, units * spans);
    // (the kernel for the states takes as long as a chunk or two: sequences of so many stay whole.  Of one chunk where each block adds up the others' states,
    // of two where that would be too many: 1024 tokens in 8 blocks of two chunks 24 us, in 16 of one 31.)
    const uint64_t most_blocks = chunks <= kWholeChunks ? 1 : chunks <= kDirectBlocks ? chunks : pairs;
    if (per_span > most_blocks) per_span = most_blocks;
    if (per_span > 1 && per_span * spans > most / each + 1) {
        per_span = (most / each + 1) / spans;
        if (per_span == 0) per_span = 1;
    }
    b.span = (uint32_t)span;
    b.length = (uint32_t)(div_up(div_up(span, per_span), shape.chunk) * shape.chunk);
    b.per_span = (uint32_t)div_up(span, b.length);
    b.count = (uint32_t)(b.per_span * spans);
    *need = b.per_span > 1 ? (b.count - 1) * each : 0;
    return b;
}

template <typename T, typename OUT, int DK, int W, int NT, int C>
tcr_status run_chunks(const Scan& a, const Room& given, hipStream_t stream) {
    const ChunkShape shape = {DK, 16 * W * NT, C, W};
    Room room = given;
    uint64_t need = 0;
    Blocks b = cut(a, shape, given.given ? given.count : ~0ull, &need);
    if (need != 0 && !given.given) {
        const tcr_status st = partials_for(stream, need, 0, &room.floats, &room.count);
        if (st != TCR_OK) return st;
        if (room.count < need) b = cut(a, shape, room.count, &need);
    }
    const uint64_t slabs = div_up(a.dv, shape.cols), units = a.heads * slabs, state_size = (uint64_t)DK * shape.cols;
    if (need != 0) {
        b.states = room.floats;
        b.keep = reinterpret_cast<Kept*>(room.floats + (b.count - 1) * units * state_size);
        b.turned = room.turned;
        b.direct = b.per_span <= kDirectBlocks && !room.shared;
        if (!room.turned) {
            attention_chunk_kernel<T, T, DK, W, NT, C, true><<<dim3((unsigned)((b.count - 1) * units)), dim3(64 * W), 0, stream>>>(a, b);
            if (launched("attention_chunk_kernel<states>") != TCR_OK) return TCR_ERR_HIP;
            if (!b.direct) attention_carry_kernel<<<dim3((unsigned)(units * state_size / 256)), dim3(256), 0, stream>>>(b, (uint32_t)slabs, state_size);
            if (launched("attention_carry_kernel") != TCR_OK) return TCR_ERR_HIP;
        }
    }
    attention_chunk_kernel<T, OUT, DK, W, NT, C, false><<<grid_of(b.count * units), dim3(64 * W), 0, stream>>>(a, b);
    return launched("attention_chunk_kernel");
}

// Whether chunks take a scan, or it goes token by token.  (Packed sequences: by their mean, as only the device knows more of their lengths.  A long one among many of one token
// goes the way of the others: 1000 tokens behind 1000 single ones, 16 heads of 128 x 128, take 2.7 ms token by token, 1.1 ms by chunks; 256 single tokens 0.11 and 0.53 ms.)
bool by_chunks(const Scan& a) {
    const uint64_t steps = a.sequences * a.heads <= kFewPairs ? kFewStepTokens : kStepTokens;
    if (a.sequences == 0 || a.total <= steps * a.sequences) return false;
    for (const View* v : {&a.a, &a.b, &a.c})
        if (v->tok < 0 || v->tok > (1 << 23)) return false;        // offsets inside a chunk are 31 bits and count upwards
    return a.out_tok >= 0 && a.out_tok <= (1 << 22);
}

template <typename T, typename OUT>
tcr_status run(const Scan& a, const Room& room, hipStream_t stream) {
    if (!by_chunks(a)) return run_steps<T, OUT>(a, stream);
    const ChunkShape shape = chunk_shape(a.dk, a.dv);
    if (shape.rows == 256) return run_chunks<T, OUT, 256, 4, 1, 32>(a, room, stream);
    if (shape.rows == 128) return shape.cols == 64 ? run_chunks<T, OUT, 128, 4, 1, 64>(a, room, stream) : run_chunks<T, OUT, 128, 8, 1, 64>(a, room, stream);
    return shape.cols == 64 ? run_chunks<T, OUT, 64, 4, 1, 64>(a, room, stream) : run_chunks<T, OUT, 64, 8, 1, 64>(a, room, stream);
}

// Out of the type of the inputs, or binary32 (`wide`).
tcr_status run(const Scan& a, uint32_t dtype, bool wide, hipStream_t stream, const Room& room = Room()) {
    if (dtype == TCR_F16) return wide ? run<_Float16, float>(a, room, stream) : run<_Float16, _Float16>(a, room, stream);
    return wide ? run<__bf16, float>(a, room, stream) : run<__bf16, __bf16>(a, room, stream);
}

tcr_status check_states(const void* a, const void* b) { return on_boundary(a, 16) && on_boundary(b, 16) ? TCR_OK : TCR_ERR_INVALID_ARG; }

// The memory of an array of rows: its bytes, where the rows fill them without gaps.
struct Extent {
    uintptr_t from, to;
    bool whole;
};
Extent extent(const tcr_attention& a, const void* p, const int64_t stride[3], uint64_t heads, uint64_t d) {
    const uint64_t counts[3] = {a.offsets != nullptr ? 1 : a.sequences, a.tokens, heads};
    __int128 reach = d, all = d;                   // (strides may be anything)
    bool whole = true;
    for (int i = 0; i < 3; ++i) {
        if (counts[i] > 1 && stride[i] < 0) whole = false;
        reach += (__int128)(counts[i] - 1) * stride[i];
        all *= counts[i];
    }
    const uintptr_t from = reinterpret_cast<uintptr_t>(p);
    whole = whole && reach == all;
    return {from, whole ? from + (uintptr_t)(2 * all) : from + 2 * d, whole};
}
// Whether two of them share memory for certain.  (Rows with gaps may stand in each other's; they are only looked at where they start.)
bool share(const Extent& a, const Extent& b) { return a.whole && b.whole ? a.from < b.to && b.from < a.to : a.from == b.from; }
// The same of two arrays of states.
bool states_share(const tcr_attention& a, const float* x, const float* y) {
    if (x == nullptr || y == nullptr) return false;
    const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y), bytes = 4 * a.sequences * a.heads * a.dk * a.dv;
    return x == y || (p < q + bytes && q < p + bytes);
}

bool odd(const void* p) { return p == nullptr || !on_boundary(p, 2); }

// step: final_state may be `state`
tcr_status forward(const tcr_attention* shape, const void* q, const void* k, const void* v, void* out, const float* state, float* final_state, bool step,
                   hipStream_t stream) {
    tcr_status st = check(shape);
    if (st != TCR_OK) return st;
    const bool any = shape->tokens != 0 && (shape->sequences != 0 || shape->offsets != nullptr);
    if ((any && (odd(q) || odd(k) || odd(v) || odd(out))) || check_states(state, final_state) != TCR_OK) return TCR_ERR_INVALID_ARG;
    // (other workgroups read the rows of q, k and v that one has written out for: those of other columns, of heads that share them, of blocks behind)
    if (any) {
        const Extent written = extent(*shape, out, shape->o_stride, shape->heads, shape->dv);
        if (share(written, extent(*shape, q, shape->q_stride, shape->heads, shape->dk)) || share(written, extent(*shape, k, shape->k_stride, shape->kv_heads, shape->dk)) ||
            share(written, extent(*shape, v, shape->v_stride, shape->kv_heads, shape->dv)))
            return TCR_ERR_INVALID_ARG;
    }
    if ((state != final_state || !step) && states_share(*shape, state, final_state)) return TCR_ERR_INVALID_ARG;
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
    if (check_states(state, dfinal) != TCR_OK || check_states(dstate, nullptr) != TCR_OK || states_share(*shape, dstate, dfinal)) return TCR_ERR_INVALID_ARG;
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

    // dk and dv, from the last token to the first
    auto reversed = [&](const View& va, const View& vb, const View& vc, uint32_t rows, uint32_t cols, void* out) {
        contiguous(stride, cols);
        Scan r = scan_of(a, va, vb, vc, out, stride, rows, cols);
        r.reverse = r.late = 1;
        r.init = dfinal;
        r.init_mul = 1.0f / a.scale;
        r.fin_mul = a.scale;
        return r;
    };
    Scan of_k = reversed(vv, vo, vq, a.dv, a.dk, dk), of_v = reversed(vk, vq, vo, a.dk, a.dv, dv);
    of_k.st_row = 1;                     // R transposed: dv x dk
    of_k.st_col = a.dv;
    of_v.fin = dstate;
    // The states between blocks are the same for both, transposed: where both are cut alike they are worked out once.
    // Gradients of shared keys and values go by way of each head's own in binary32, in front of the states in the workspace.
    const uint64_t part = group == 1 ? 0 : div_up(of_k.total * a.heads * (a.dk > a.dv ? a.dk : a.dv), 64) * 64;
    const ChunkShape shape_k = chunk_shape(of_k.dk, of_k.dv), shape_v = chunk_shape(of_v.dk, of_v.dv);
    auto need_of = [](const Scan& r) {
        uint64_t need = 0;
        if (by_chunks(r)) (void)cut(r, chunk_shape(r.dk, r.dv), ~0ull, &need);
        return need;
    };
    const uint64_t need_q = need_of(s), need_k = need_of(of_k), need_v = need_of(of_v);
    const uint64_t behind = part + (need_k > need_v ? need_k : need_v);
    // (all of it in front of the first launch: a call that lacks room has done nothing)
    uint64_t got = 0;
    Room room;
    room.given = true;
    st = partials_for(stream, need_q > behind ? need_q : behind, part, &room.floats, &got);
    if (st != TCR_OK) return st;
    room.count = got;
    st = run(s, a.dtype, false, stream, room);
    if (st != TCR_OK) return st;
    float* const floats = room.floats;
    room.floats += part;
    room.count = got - part;
    const bool alike = need_k != 0 && need_k == need_v && shape_k.rows == shape_v.rows && shape_k.cols == shape_v.cols && shape_k.chunk == shape_v.chunk &&
                       div_up(of_k.dv, shape_k.cols) == div_up(of_v.dv, shape_v.cols) && room.count >= need_k;
    for (Scan* r : {&of_v, &of_k}) {
        void* const out = r->out;
        if (group > 1) r->out = floats;
        room.shared = alike;
        room.turned = alike && r == &of_k;
        st = run(*r, a.dtype, group > 1, stream, room);
        if (st != TCR_OK) return st;
        const uint64_t count = r->total * a.kv_heads * r->dv;
        if (group == 1 || count == 0) continue;
        const dim3 grid(at_most(div_up(count, 256)));
        if (a.dtype == TCR_F16) attention_shared_kernel<<<grid, dim3(256), 0, stream>>>(floats, static_cast<_Float16*>(out), count, r->dv, group);
        else attention_shared_kernel<<<grid, dim3(256), 0, stream>>>(floats, static_cast<__bf16*>(out), count, r->dv, group);
        if (launched("attention_shared_kernel") != TCR_OK) return TCR_ERR_HIP;
    }
    return TCR_OK;
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
        return forward(shape, q, k, v, out, state, final_state, false, static_cast<hipStream_t>(stream));
    });
}

extern "C" tcr_status tcr_linear_attention_step(const tcr_attention* shape, const void* q, const void* k, const void* v, void* out, const float* state,
                                                float* new_state, void* stream) {
    return guarded([&] {
        if (shape != nullptr && (shape->tokens != 1 || shape->offsets != nullptr || state == nullptr || new_state == nullptr)) return TCR_ERR_INVALID_ARG;
        return forward(shape, q, k, v, out, state, new_state, true, static_cast<hipStream_t>(stream));
    });
}

extern "C" tcr_status tcr_linear_attention_backward(const tcr_attention* shape, const void* dout, const void* q, const void* k, const void* v, void* dq,
                                                    void* dk, void* dv, const float* state, const float* dfinal, float* dstate, void* stream) {
    return guarded([&] {
        return backward(shape, dout, q, k, v, dq, dk, dv, state, dfinal, dstate, static_cast<hipStream_t>(stream));
    });
}
