// Selective state space scan: a segmented scan whose factors depend on the data, `states` running values a channel.
//
//     d_t = softplus(dt_t + bias),   h_t[n] = exp(d_t a[n]) h_{t-1}[n] + d_t x_t b_t[n],   y_t = sum_n c_t[n] h_t[n] + skip x_t,
//     out_t = y_t, or y_t gate_t sigmoid(gate_t).
// a, skip, bias: by channel; b, c: by token, shared by the channels of a group.  Everything between loads and stores is binary32.
//
// A workgroup takes a slab of channels and a chunk of tokens, tile by tile.  P lanes hold a channel, each K of its states in registers for the
// whole chunk; what a token needs of its channel (d and d x) and of its group (b, c) stands in LDS as binary32, made once by whole vectors.
// What bounds it is the vector unit: an exponential (3.2 times a multiply-add), two multiplications and two multiply-adds for each state.
#pragma once
#include "tcr_places.hpp"

namespace tcr {
namespace layers {

constexpr int kScanThreads = 256;
constexpr int kTokens = 4;                     // whose sums over a channel's lanes are made together
constexpr int kTurn = 8;                       // tokens of a turn of the inner loop

struct Operand {                               // of the rows of a sequence's tokens; strides in elements
    const void* p;
    int64_t seq, tok, group;
};

struct Selective {
    Operand x, dt, gate, b, c;                 // gate.p: NULL for none
    void* out;
    int64_t out_seq, out_tok;
    const float *a, *skip, *bias, *state;      // skip, bias, state: NULL for none
    float* fin;                                // the states behind the last tokens; NULL: not wanted
    const uint64_t* offsets;
    uint64_t sequences;
    float *ends, *sums;                        // of every chunk: [chunk][padded channel][padded state] the state behind it from nothing, [chunk][padded channel] the sum of d
    uint32_t span, length, per_span;           // tokens of a span (a sequence, or all packed ones), of a chunk; chunks of a span
    uint32_t channels, states, groups, slabs;  // slabs of a group
    uint32_t softplus;
};

// log(1 + e) for e in [0, 1] as 2 atanh(s), s = e / (2 + e) <= 1/3, so that nothing is lost where e is small: 2 s + s^3 p(s^2) with the polynomial of degree 3 whose
// largest error, 5e-9 of the result (a tenth of a rounding), is the least on [0, 1/9].
__device__ __forceinline__ float log1p_unit(float e) {
    const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
    float v = __builtin_fmaf(0.28023902f, q, 0.27999245f);
    v = __builtin_fmaf(v, q, 0.40021693f);
    v = __builtin_fmaf(v, q, 0.66666413f);
    return __builtin_fmaf(s * q, v, s + s);
}
// (the median of x, 0 and infinity is the larger of x and 0 in one operation, and no NaN: a NaN comes by way of the logarithm)
__device__ __forceinline__ float softplus_of(float x) { return __builtin_amdgcn_fmed3f(x, 0.0f, __builtin_inff()) + log1p_unit(exp_of(-__builtin_fabsf(x))); }

// A value h carried over many tokens at once, whose steps sum to `sum`: 2^(sum rate) h + end.  Both may be in range where the factor is not, so it is applied in three equal parts:
// third_of is one of them.  Its limit of 2^127 keeps 0 at 0 and takes nothing else away: 2^381 h is beyond the range for every other h.
__device__ __forceinline__ float third_of(float sum, float third_rate) { return __builtin_amdgcn_exp2f(__builtin_fminf(sum * third_rate, 127.0f)); }
__device__ __forceinline__ float carried(float third, float h, float end) { return __builtin_fmaf(third, third * (third * h), end); }

// The states n0 .. n0 + K - 1 of a channel in an array [sequence][channel][state]; 0 where there is no array or no such state.
template <int K>
__device__ __forceinline__ void load_states(const float* states, uint64_t seq, const Selective& s, uint32_t ch, uint32_t n0, bool real, float (&h)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) h[k] = states != nullptr && real && n0 + k < s.states ? states[(seq * s.channels + ch) * s.states + n0 + k] : 0.0f;
}
template <int K>
__device__ __forceinline__ void store_states(float* states, uint64_t seq, const Selective& s, uint32_t ch, uint32_t n0, bool real, const float (&h)[K]) {
    if (states == nullptr || !real) return;
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (n0 + k < s.states) states[(seq * s.channels + ch) * s.states + n0 + k] = h[k];
}

// Sums of y[0 .. 3] over the P lanes of a channel (lane = part * (64 / P) + channel).  Lanes swap halves, so that each step has half as many values left:
// lane part p ends with the sum of token sum_token<P>(p, i) in y[i], i < sum_count<P>.
template <int P> constexpr int sum_count = P == 1 ? 4 : P == 2 ? 2 : 1;
template <int P>
__device__ __forceinline__ int sum_token(int lane, int i) {
    if (P == 1) return i;
    if (P == 2) return (lane >> 5) + 2 * i;
    return (lane >> 5) + 2 * ((lane >> 4) & 1);
}
__device__ __forceinline__ float swap_add32(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
    const uint32_t low = r[0], high = r[1];                // (a bit_cast of r[1] itself reads r[0])
    return __builtin_bit_cast(float, low) + __builtin_bit_cast(float, high);
}
__device__ __forceinline__ float swap_add16(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
    const uint32_t low = r[0], high = r[1];                // (a bit_cast of r[1] itself reads r[0])
    return __builtin_bit_cast(float, low) + __builtin_bit_cast(float, high);
}
template <int CTRL>
__device__ __forceinline__ float dpp_of(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
constexpr int kRor4 = 0x124, kRor8 = 0x128;
template <int P>
__device__ __forceinline__ void sum_parts(float (&y)[kTokens]) {
    if (P == 1) return;
    y[0] = swap_add32(y[0], y[1]);
    y[1] = swap_add32(y[2], y[3]);
    if (P == 2) return;
    y[0] = swap_add16(y[0], y[1]);
    if (P >= 8) y[0] += dpp_of<kRor8>(y[0]);
    if (P >= 16) y[0] += dpp_of<kRor4>(y[0]);
}
// The same of one value: every lane has the sum.
template <int P>
__device__ __forceinline__ float sum_one(float y) {
#pragma unroll
    for (int m = 32; m >= 64 / P; m >>= 1) y += __shfl_xor(y, m);
    return y;
}

// Eight floats of LDS, from a boundary of 16 bytes on.
__device__ __forceinline__ void put_vec(float* to, const float (&v)[kVec]) {
    *reinterpret_cast<f4v*>(to) = f4v{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f4v*>(to + 4) = f4v{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void get_vec(const float* from, float (&v)[kVec]) {
    const f4v a = *reinterpret_cast<const f4v*>(from), b = *reinterpret_cast<const f4v*>(from + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}

// How a workgroup stands in the grid: slab of channels fastest, so that neighbours read neighbouring columns of the same tokens.
template <int P>
struct Slab {
    static constexpr int kWide = 64 / P, kChannels = 4 * kWide;
    uint32_t chunk, span, group, first, end, padded;       // first, end: channels; padded: the slab's place among padded channels
    __device__ __forceinline__ Slab(const Selective& s, uint32_t chunks) {
        const uint32_t all = s.slabs * s.groups, each = s.channels / s.groups, block = workgroup();
        const uint32_t slab = block % all, rest = block / all;
        chunk = rest % chunks;
        span = rest / chunks;
        group = slab / s.slabs;
        first = group * each + (slab % s.slabs) * kChannels;
        end = (group + 1) * each;
        padded = slab * kChannels;
    }
};

// Of the wavefronts of a SIMD the one that is ahead waits: left to itself the oldest runs first, and the last ones alone at the end, when one wavefront by itself
// issues half as fast as two.  A step's priority is one less than that of the step in front of it, around four.  (8192 tokens x 4096 channels, the two kernels under rocprofv3: 168 + 124 us without, 156 + 116 with.)
__device__ __forceinline__ void keep_pace(uint32_t step) {
    switch (step & 3) {
        case 0: __builtin_amdgcn_s_setprio(3); break;
        case 1: __builtin_amdgcn_s_setprio(2); break;
        case 2: __builtin_amdgcn_s_setprio(1); break;
        default: __builtin_amdgcn_s_setprio(0);
    }
}

// OUT: outputs and last states; otherwise a chunk's state from nothing and its sum of d, for the chunks behind it.
template <typename T, int K, int P, bool OUT>
__global__ __launch_bounds__(kScanThreads) void selective_kernel(Selective s, uint32_t blocks) {
    constexpr int kWide = 64 / P, kChannels = 4 * kWide, kTile = 8 * P, kStates = K * P, kRow = kChannels / kVec;
    constexpr int kShared = kTile * kStates / kScanThreads > 0 ? kTile * kStates / kScanThreads : 1;
    static_assert(kTile * kRow == kScanThreads && kTile % kTurn == 0, "one vector of a tile for each thread, whole turns");
    __shared__ __attribute__((aligned(16))) float ds[kTile][kChannels], us[kTile][kChannels];          // d, d x; then y in the place of d
    __shared__ __attribute__((aligned(16))) float bs[kTile][kStates], cs[OUT ? kTile : 1][kStates];
    if (workgroup() >= blocks) return;
    const Slab<P> slab(s, OUT ? s.per_span : s.per_span - 1);
    const uint32_t tid = threadIdx.x, lane = tid & 63, wide = (tid >> 6) * kWide + lane % kWide, n0 = lane / kWide * K;
    const uint32_t ch = slab.first + wide;
    const bool real = ch < slab.end;
    const uint64_t spans = s.offsets != nullptr ? 1 : s.sequences, all = (uint64_t)s.slabs * s.groups * kChannels;
    const uint32_t t0 = slab.chunk * s.length, t1 = s.span - t0 < s.length ? s.span : t0 + s.length;
    const Bounds bounds = {s.offsets, (uint32_t)s.sequences, s.span};
    Place at;
    at.find(bounds, slab.span, t0);

    float rate[K], h[K], sum = 0.0f, total = 0.0f;         // sums of d: of a tile, of the chunk (in two levels: the factor over a chunk has the sum in its exponent)
#pragma unroll
    for (int k = 0; k < K; ++k) {
        rate[k] = real && n0 + k < s.states ? s.a[(uint64_t)ch * s.states + n0 + k] * kLog2e : 0.0f;
        h[k] = 0.0f;
    }
    if (at.inside && at.start == t0) load_states(s.state, at.seq, s, ch, n0, real, h);
    else if (OUT && at.inside) {
        // the state that the chunks in front leave, back to the one in which the sequence begins
        uint32_t i = at.start / s.length;
        const uint64_t one = spans * all, place = slab.span * all + slab.padded + wide;
        auto end_of = [&](uint32_t c, int k) { return s.ends[(c * one + place) * kStates + n0 + k]; };
#pragma unroll
        for (int k = 0; k < K; ++k) h[k] = end_of(i, k);
        for (++i; i < slab.chunk; ++i) {
            const float passed = s.sums[i * one + place];
#pragma unroll
            for (int k = 0; k < K; ++k) h[k] = carried(third_of(passed, rate[k] * (1.0f / 3.0f)), h[k], end_of(i, k));
        }
    }

    // what this thread puts into LDS: eight channels of one of a tile's tokens, and some of b and c
    const uint32_t my_token = tid / kRow, my_wide = tid % kRow * kVec, my_first = slab.first + my_wide, my_end = slab.end;
    const T* const x_row = static_cast<const T*>(s.x.p) + slab.span * s.x.seq;
    const T* const dt_row = static_cast<const T*>(s.dt.p) + slab.span * s.dt.seq;
    const T* const gate_row = static_cast<const T*>(s.gate.p) + slab.span * s.gate.seq;
    const T* const b_row = static_cast<const T*>(s.b.p) + slab.span * s.b.seq + slab.group * s.b.group;
    const T* const c_row = static_cast<const T*>(s.c.p) + slab.span * s.c.seq + slab.group * s.c.group;
    T* const out_row = static_cast<T*>(s.out) + slab.span * s.out_seq;
    const bool gated = OUT && s.gate.p != nullptr;
    float bias[kVec], skip[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        bias[i] = s.bias != nullptr && my_first + i < my_end ? s.bias[my_first + i] : 0.0f;
        skip[i] = OUT && s.skip != nullptr && my_first + i < my_end ? s.skip[my_first + i] : 0.0f;
    }
    const uint32_t begin = s.offsets != nullptr ? bounds.at(0) : 0, finish = s.offsets != nullptr ? bounds.at(bounds.count) : s.span;

    typedef typename Vec<T>::v vec;
    vec x_next = {}, dt_next = {}, gate_next = {};
    T b_next[kShared] = {}, c_next[kShared] = {};
    auto fetch = [&](uint32_t tile) {
        const uint32_t t = tile + my_token;
        const bool there = t < t1 && my_first < my_end;
        x_next = there ? load_raw(x_row + t * s.x.tok, my_first, my_end) : vec{};
        dt_next = there ? load_raw(dt_row + t * s.dt.tok, my_first, my_end) : vec{};
        if (gated) gate_next = there ? load_raw(gate_row + t * s.gate.tok, my_first, my_end) : vec{};
#pragma unroll
        for (int i = 0; i < kShared; ++i) {
            const uint32_t e = tid + i * kScanThreads, bt = tile + e / kStates, n = e % kStates;
            const bool any = e < kTile * kStates && bt < t1 && n < s.states;
            b_next[i] = any ? b_row[bt * s.b.tok + n] : (T)0.0f;
            if (OUT) c_next[i] = any ? c_row[bt * s.c.tok + n] : (T)0.0f;
        }
    };
    if (t0 < t1) fetch(t0);
    for (uint32_t tile = t0; tile < t1; tile += kTile) {
        keep_pace((tile - t0) / kTile);
        const vec x_now = x_next, gate_now = gate_next;
        // (whole vectors, and branches around whole vectors: a choice for each element costs as much as a state)
        float v[kVec], u[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = (float)dt_next[i] + bias[i];
        if (s.softplus)
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = softplus_of(v[i]);
        if (tile + kTile > t1) {               // behind the chunk: the states stay
            if (tile + my_token >= t1)
#pragma unroll
                for (int i = 0; i < kVec; ++i) v[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) u[i] = v[i] * (float)x_now[i];
        put_vec(ds[my_token] + my_wide, v);
        put_vec(us[my_token] + my_wide, u);
#pragma unroll
        for (int i = 0; i < kShared; ++i) {
            const uint32_t e = tid + i * kScanThreads;
            if (e >= kTile * kStates) break;
            bs[e / kStates][e % kStates] = (float)b_next[i];
            if (OUT) cs[e / kStates][e % kStates] = (float)c_next[i];
        }
        __syncthreads();
        if (tile + kTile < t1) fetch(tile + kTile);

        auto token = [&](uint32_t j) {
            const float d = ds[j][wide], du = us[j][wide];
            float y = 0.0f;
            if (!OUT) sum += d;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                h[k] = __builtin_fmaf(__builtin_amdgcn_exp2f(d * rate[k]), h[k], du * bs[j][n0 + k]);
                if (OUT) y = __builtin_fmaf(cs[j][n0 + k], h[k], y);
            }
            return y;
        };
        const uint32_t here = t1 - tile < kTile ? t1 - tile : kTile;
        for (uint32_t j = 0; j < here; j += kTurn) {
            const uint32_t t = tile + j;
            if (at.next >= t + kTurn || at.next >= t1) {
                float y[kTurn];
#pragma unroll
                for (int i = 0; i < kTurn; ++i) y[i] = token(j + i);
                if (OUT)
#pragma unroll
                    for (int q = 0; q < kTurn; q += kTokens) {
                        float four[kTokens] = {y[q], y[q + 1], y[q + 2], y[q + 3]};
                        sum_parts<P>(four);
#pragma unroll
                        for (int i = 0; i < sum_count<P>; ++i) ds[j + q + sum_token<P>(lane, i)][wide] = four[i];
                    }
                continue;
            }
            for (uint32_t i = 0; i < kTurn && t + i < t1; ++i) {
                if (at.next == t + i) {
                    if (OUT && at.inside) store_states(s.fin, at.seq, s, ch, n0, real, h);
                    at.pass(bounds, t + i);
                    if (at.inside) load_states(s.state, at.seq, s, ch, n0, real, h);
                }
                const float y = sum_one<P>(token(j + i));
                if (OUT && lane < kWide) ds[j + i][wide] = y;
            }
        }
        __syncthreads();
        if (!OUT) {
            total += sum;
            sum = 0.0f;
        }
        const uint32_t t = tile + my_token;
        if (OUT && t < t1 && my_first < my_end) {
            get_vec(ds[my_token] + my_wide, v);
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = __builtin_fmaf(skip[i], (float)x_now[i], v[i]);
            if (gated)
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float z = (float)gate_now[i];
                    v[i] *= z * sigmoid_of(z);
                }
            if (t < begin || t >= finish)
#pragma unroll
                for (int i = 0; i < kVec; ++i) v[i] = 0.0f;
            store_vec(out_row + t * s.out_tok, my_first, my_end, v);
        }
    }
    if constexpr (OUT) {
        if (at.inside && at.next == t1) store_states(s.fin, at.seq, s, ch, n0, real, h);
        if (s.offsets != nullptr && s.fin != nullptr)
            for (uint32_t e = slab.chunk; e < bounds.count; e += s.per_span)
                if (bounds.at(e + 1) <= bounds.at(e)) {
                    load_states(s.state, e, s, ch, n0, real, h);
                    store_states(s.fin, e, s, ch, n0, real, h);
                }
    } else {
        const uint64_t place = (slab.chunk * spans + slab.span) * all + slab.padded + wide;
#pragma unroll
        for (int k = 0; k < K; ++k) s.ends[place * kStates + n0 + k] = h[k];
        if (lane < kWide) s.sums[place] = total;
    }
}

// One token for every sequence: four states a lane, P lanes a channel, lane = channel * P + part as the states lie in memory; S sequences a thread, all loads first.
// Bound by the states' bytes, which pass the caches by: the next step finds none of them there (256 sequences x 4096 channels x 16 states 33 us, 4.3 TB/s; kept in the caches 42).
template <typename T, int P, int S>
__global__ __launch_bounds__(kScanThreads) void selective_step_kernel(Selective s, uint32_t whole) {
    constexpr int K = 4, kChannels = kScanThreads / P;
    const uint32_t slabs = (s.channels + kChannels - 1) / kChannels, block = workgroup();
    const uint64_t first = (uint64_t)(block / slabs) * S;
    if (first >= s.sequences) return;
    const uint32_t ch = block % slabs * kChannels + threadIdx.x / P, n0 = threadIdx.x % P * K;
    if (ch >= s.channels) return;                          // (all lanes of the channel)
    const uint32_t group = ch / (s.channels / s.groups);
    const bool writer = threadIdx.x % P == 0, gated = s.gate.p != nullptr;
    float h[S][K], bv[S][K], cv[S][K], x[S], raw[S], z[S], rate[K];
#pragma unroll
    for (int q = 0; q < S; ++q) {
        const uint64_t seq = first + q < s.sequences ? first + q : first;
        const T* const b = static_cast<const T*>(s.b.p) + seq * s.b.seq + group * s.b.group;
        const T* const c = static_cast<const T*>(s.c.p) + seq * s.c.seq + group * s.c.group;
        const uint64_t place = (seq * s.channels + ch) * s.states + n0;
        if (whole) {
            typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
            const f4v v = __builtin_nontemporal_load(reinterpret_cast<const f4v*>(s.state + place));
            const four bs = *reinterpret_cast<const four*>(b + n0), cs = *reinterpret_cast<const four*>(c + n0);
#pragma unroll
            for (int k = 0; k < K; ++k) h[q][k] = v[k], bv[q][k] = (float)bs[k], cv[q][k] = (float)cs[k];
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const bool any = n0 + k < s.states;
                h[q][k] = any ? s.state[place + k] : 0.0f;
                bv[q][k] = any ? (float)b[n0 + k] : 0.0f;
                cv[q][k] = any ? (float)c[n0 + k] : 0.0f;
            }
        }
        x[q] = (float)static_cast<const T*>(s.x.p)[seq * s.x.seq + ch];
        raw[q] = (float)static_cast<const T*>(s.dt.p)[seq * s.dt.seq + ch];
        z[q] = gated ? (float)static_cast<const T*>(s.gate.p)[seq * s.gate.seq + ch] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) rate[k] = n0 + k < s.states ? s.a[(uint64_t)ch * s.states + n0 + k] * kLog2e : 0.0f;
    const float bias = s.bias != nullptr ? s.bias[ch] : 0.0f, skip = s.skip != nullptr ? s.skip[ch] : 0.0f;
#pragma unroll
    for (int q = 0; q < S; ++q) {
        if (first + q >= s.sequences) break;
        const uint64_t seq = first + q, place = (seq * s.channels + ch) * s.states + n0;
        const float d = s.softplus ? softplus_of(raw[q] + bias) : raw[q] + bias, u = d * x[q];
        float y = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            h[q][k] = __builtin_fmaf(__builtin_amdgcn_exp2f(d * rate[k]), h[q][k], u * bv[q][k]);
            y = __builtin_fmaf(cv[q][k], h[q][k], y);
        }
#pragma unroll
        for (int m = 1; m < P; m <<= 1) y += __shfl_xor(y, m);
        if (whole) {
            __builtin_nontemporal_store(f4v{h[q][0], h[q][1], h[q][2], h[q][3]}, reinterpret_cast<f4v*>(s.fin + place));
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (n0 + k < s.states) s.fin[place + k] = h[q][k];
        }
        y = __builtin_fmaf(skip, x[q], y);
        if (gated) y *= z[q] * sigmoid_of(z[q]);
        if (writer) static_cast<T*>(s.out)[seq * s.out_seq + ch] = (T)y;
    }
}

}  // namespace layers
}  // namespace tcr
