// Gradients of the selective scan.  With dy_t = dout_t (gate_t sigmoid(gate_t)) and the gradient g_t of h_t,
//
//     g_t[n] = c_t[n] dy_t + exp(d_{t+1} a[n]) g_{t+1}[n]               (behind the last token: dfinal)
//     dc_t[n] = sum_channels dy_t h_t[n],   db_t[n] = sum_channels g_t[n] d_t x_t,   dgate_t = dout_t (y_t + skip x_t) silu'(gate_t)
//     dx_t = d_t sum_n g_t[n] b_t[n] + skip dy_t,   dd_t = x_t sum_n g_t[n] b_t[n] + sum_n g_t[n] a[n] exp(d_t a[n]) h_{t-1}[n]
//     da[n] = sum_t g_t[n] d_t exp(d_t a[n]) h_{t-1}[n],   dskip = sum_t dy_t x_t,   ddt_t = dd_t sigmoid(dt_t + bias),   dbias = sum_t ddt_t.
//
// Tokens are cut into chunks of one tile.  selective_parts_kernel goes over them once: a chunk's state from nothing and, with the product of the factors so far, what it
// hands back to the tokens in front of it (where factors may be above 1 once more, backwards).  selective_carry_kernel makes of these the states in front of every chunk and the gradients behind it.  selective_grad_kernel
// then does every chunk by itself: forwards once more with the states in front of each kTurn tokens kept in LDS, then turn by turn from the last to the first, the turn's
// states and factors in registers.  Sums over channels and over chunks pass through the workspace and are added up in the same order every time.
// What bounds it is the vector unit: two exponentials and about twenty operations for each state and token.
#pragma once
#include <type_traits>

#include "tcr_selective.hpp"

namespace tcr {
namespace layers {

struct SelectiveGrad {
    Selective s;                               // out: dout
    const float* dfinal;                       // NULL: none
    void *dx, *ddt, *db, *dc, *dgate;          // contiguous
    float *da, *dskip, *dbias, *dstate;        // dskip, dbias, dstate: NULL: not wanted
    float* back;                               // like s.ends: what a chunk hands back; then what comes back to it from behind
    float* means;                              // [chunk][2][padded channel] sums of dskip and dbias
    float* shares;                             // [slab][token][2][padded state] sums of db and dc
    uint32_t* closed;                          // [chunk] whether a bound lies in it, so that nothing passes through; NULL: none do
};

// Tokens of a chunk: a vector for each thread, but no more than leave room for two workgroups and more in LDS (32 states, 2048 tokens x 2048 channels: 64 tokens 356 us, 32 240).
template <int P> constexpr int kGradTile = P >= 8 ? 32 : 8 * P;

// The inputs of a tile, as each thread has loaded eight channels of a token, and as they stand in LDS.
template <typename T, int P>
struct GradTile {
    static constexpr int kTile = kGradTile<P>, kChannels = Slab<P>::kChannels, kStates = 4 * P, kRow = kChannels / kVec;
    typedef typename Vec<T>::v vec;
    uint32_t token, wide, first;               // this thread's
    bool there, inside;                        // inside: of a sequence
    vec x, gate, dout;
    float raw[kVec], d[kVec], dy[kVec];

    __device__ __forceinline__ void load(const SelectiveGrad& g, const Slab<P>& slab, uint32_t t0, uint32_t t1, uint32_t begin, uint32_t finish) {
        const Selective& s = g.s;
        const uint32_t tid = threadIdx.x;
        token = tid / kRow;
        wide = tid % kRow * kVec;
        first = slab.first + wide;
        const uint32_t t = t0 + token;
        there = token < kTile && t < t1 && first < slab.end;
        x = dout = gate = vec{};
        vec dt = {};
        if (there) {
            x = load_raw(static_cast<const T*>(s.x.p) + slab.span * s.x.seq + t * s.x.tok, first, slab.end);
            dt = load_raw(static_cast<const T*>(s.dt.p) + slab.span * s.dt.seq + t * s.dt.tok, first, slab.end);
            dout = load_raw(static_cast<const T*>(s.out) + slab.span * s.out_seq + t * s.out_tok, first, slab.end);
            if (s.gate.p != nullptr) gate = load_raw(static_cast<const T*>(s.gate.p) + slab.span * s.gate.seq + t * s.gate.tok, first, slab.end);
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) raw[i] = 0.0f;
        if (s.bias != nullptr && there) load_vec(s.bias, (uint64_t)first, (uint64_t)slab.end, raw);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            raw[i] += (float)dt[i];
            d[i] = raw[i];
            dy[i] = (float)dout[i];
        }
        if (s.softplus)
#pragma unroll
            for (int i = 0; i < kVec; ++i) d[i] = softplus_of(raw[i]);
        if (s.gate.p != nullptr)
#pragma unroll
            for (int i = 0; i < kVec; ++i) dy[i] *= (float)gate[i] * sigmoid_of((float)gate[i]);
        inside = there && t >= begin && t < finish;
    }
    __device__ __forceinline__ void put(const SelectiveGrad& g, const Slab<P>& slab, uint32_t t0, uint32_t t1, uint32_t begin, uint32_t finish, float (*ds)[kChannels],
                                        float (*us)[kChannels], float (*dys)[kChannels], float (*bs)[kStates], float (*cs)[kStates]) {
        const Selective& s = g.s;
        float u[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) u[i] = d[i] * (float)x[i];
        if (!inside)                           // outside of all sequences: nothing
#pragma unroll
            for (int i = 0; i < kVec; ++i) d[i] = u[i] = dy[i] = 0.0f;
        if (token < kTile) {
            put_vec(ds[token] + wide, d);
            put_vec(us[token] + wide, u);
            put_vec(dys[token] + wide, dy);
        }
        const T* const b = static_cast<const T*>(s.b.p) + slab.span * s.b.seq + slab.group * s.b.group;
        const T* const c = static_cast<const T*>(s.c.p) + slab.span * s.c.seq + slab.group * s.c.group;
        for (uint32_t e = threadIdx.x; e < kTile * kStates; e += kScanThreads) {
            const uint32_t bt = t0 + e / kStates, n = e % kStates;
            const bool any = bt < t1 && bt >= begin && bt < finish && n < s.states;
            bs[e / kStates][n] = any ? (float)b[bt * s.b.tok + n] : 0.0f;
            cs[e / kStates][n] = any ? (float)c[bt * s.c.tok + n] : 0.0f;
        }
    }
};

// Of every chunk: its state from nothing (from `state`, behind a sequence's beginning), what it hands back, its sum of d.
template <typename T, int P>
__global__ __launch_bounds__(kScanThreads) void selective_parts_kernel(SelectiveGrad g, uint32_t blocks) {
    typedef GradTile<T, P> Tile;
    constexpr int K = 4, kWide = 64 / P, kTile = Tile::kTile, kStates = Tile::kStates, kChannels = Tile::kChannels;
    __shared__ __attribute__((aligned(16))) float ds[kTile][kChannels], us[kTile][kChannels], dys[kTile][kChannels], bs[kTile][kStates], cs[kTile][kStates];
    __shared__ bool grown[4];
    if (workgroup() >= blocks) return;
    const Selective& s = g.s;
    const Slab<P> slab(s, s.per_span);
    const uint32_t lane = threadIdx.x & 63, wide = (threadIdx.x >> 6) * kWide + lane % kWide, n0 = lane / kWide * K, ch = slab.first + wide;
    const bool real = ch < slab.end;
    const uint32_t t0 = slab.chunk * kTile, t1 = s.span - t0 < kTile ? s.span : t0 + kTile;
    const Bounds bounds = {s.offsets, (uint32_t)s.sequences, s.span};
    const uint32_t begin = s.offsets != nullptr ? bounds.at(0) : 0, finish = s.offsets != nullptr ? bounds.at(bounds.count) : s.span;
    Place at;
    at.find(bounds, slab.span, t0);
    bool grows = false;
    {
        Tile tile;
        tile.load(g, slab, t0, t1, begin, finish);
        tile.put(g, slab, t0, t1, begin, finish, ds, us, dys, bs, cs);
        if (!s.softplus)
#pragma unroll
            for (int i = 0; i < kVec; ++i) grows |= tile.d[i] < 0.0f;
    }
    float rate[K], h[K], pass[K], back[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        rate[k] = real && n0 + k < s.states ? s.a[(uint64_t)ch * s.states + n0 + k] * kLog2e : 0.0f;
        grows |= rate[k] > 0.0f;
        h[k] = back[k] = 0.0f;
        pass[k] = 1.0f;
    }
    if (__any(grows) && lane == 0) grown[threadIdx.x >> 6] = true;
    else if (lane == 0) grown[threadIdx.x >> 6] = false;
    bool open = at.start != t0;                // whether what comes back from here reaches the tokens in front of the chunk
    if (at.inside && at.start == t0) load_states(s.state, at.seq, s, ch, n0, real, h);
    __syncthreads();
    // Where a factor may be above 1, products of factors leave the range though nothing that they carry does: what comes back is made by itself, from the last token to the first.
    // (Twice the exponentials.  Factors of at most 1 only vanish, and what they carry with them.)
    grows = grown[0] | grown[1] | grown[2] | grown[3];
    float sum = 0.0f;
    // BACK: with what comes back -- not from behind a bound, where another sequence may hold infinities or NaN that no factor of 0 would keep there.
    auto token = [&](auto with_back, uint32_t j) {
        constexpr bool BACK = decltype(with_back)::value;
        const float d = ds[j][wide], u = us[j][wide], dy = BACK ? dys[j][wide] : 0.0f;
        sum += d;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float a = __builtin_amdgcn_exp2f(d * rate[k]);
            h[k] = __builtin_fmaf(a, h[k], u * bs[j][n0 + k]);
            if (BACK) {
                pass[k] *= a;
                back[k] = __builtin_fmaf(pass[k], cs[j][n0 + k] * dy, back[k]);
            }
        }
    };
    auto leave = [&] {                         // the sequence ends here
        if (open && !grows && at.inside && g.dfinal != nullptr) {
            float after[K];
            load_states(g.dfinal, at.seq, s, ch, n0, real, after);
#pragma unroll
            for (int k = 0; k < K; ++k) back[k] = __builtin_fmaf(pass[k], after[k], back[k]);
        }
    };
    const uint32_t here = t1 - t0;
    for (uint32_t j = 0; j < here; j += kTokens) {
        const uint32_t t = t0 + j;
        if (at.next >= t + kTokens || at.next >= t1) {
            if (open && !grows)
#pragma unroll
                for (int i = 0; i < kTokens; ++i) token(std::true_type(), j + i);
            else
#pragma unroll
                for (int i = 0; i < kTokens; ++i) token(std::false_type(), j + i);
            continue;
        }
        for (uint32_t i = 0; i < kTokens && t + i < t1; ++i) {
            if (at.next == t + i) {
                leave();
                open = false;
                at.pass(bounds, t + i);
#pragma unroll
                for (int k = 0; k < K; ++k) h[k] = 0.0f;
                if (at.inside) load_states(s.state, at.seq, s, ch, n0, real, h);
            }
            if (open && !grows) token(std::true_type(), j + i);
            else token(std::false_type(), j + i);
        }
    }
    if (at.next == t1) leave();
    if (grows) {
        at.find(bounds, slab.span, t0);
        if (at.start != t0) {
            if (at.inside && at.next <= t1) load_states(g.dfinal, at.seq, s, ch, n0, real, back);
            for (uint32_t j = (at.next < t1 ? at.next : t1) - t0; j-- > 0;) {
                const float d = ds[j][wide], dy = dys[j][wide];
#pragma unroll
                for (int k = 0; k < K; ++k) back[k] = __builtin_amdgcn_exp2f(d * rate[k]) * __builtin_fmaf(cs[j][n0 + k], dy, back[k]);
            }
        }
    }
    const uint64_t spans = s.offsets != nullptr ? 1 : s.sequences, all = (uint64_t)s.slabs * s.groups * kChannels, id = slab.chunk * spans + slab.span;
    const uint64_t place = id * all + slab.padded + wide;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        s.ends[place * kStates + n0 + k] = h[k];
        g.back[place * kStates + n0 + k] = back[k];
    }
    if (lane < kWide) s.sums[place] = sum;
    if (g.closed != nullptr && threadIdx.x == 0) g.closed[id] = !open;
}

// From chunks' own results to what reaches them: s.ends[i] becomes the state in front of chunk i, g.back[i] the gradient behind it.  A column of threads for each padded
// channel and state, eight chunks a thread, a round of chunks for all of them: each thread makes one step of its eight, takes what the threads in front of it and the rounds before
// bring, and goes over its eight again.  Forwards in the first layer of workgroups, backwards in the second.  (64 chunks of 131072 columns 35 us, 134 MB read and
// written at 3.8 TB/s; 96 chunks of 8192 columns 13 us, with one thread a column from chunk to chunk 37.)
constexpr int kCarryLines = 8, kCarryChunks = 8;
template <int NP>
__global__ __launch_bounds__(64 * kCarryLines) void selective_carry_kernel(SelectiveGrad g, uint64_t all) {
    __shared__ float steps[2][kCarryLines][64], sums[2][kCarryLines][64];
    __shared__ bool closed[2][kCarryLines][64];
    const Selective& s = g.s;
    const uint64_t spans = s.offsets != nullptr ? 1 : s.sequences, one = all * NP;
    const uint32_t lane = threadIdx.x % 64, line = threadIdx.x / 64;
    const uint64_t at = (uint64_t)workgroup() * 64 + lane;
    const bool real = at < spans * one;
    const uint64_t span = real ? at / one : 0, rest = real ? at % one : 0, padded = rest / NP;
    const uint32_t n = rest % NP;
    // (the channel that stands there)
    const uint64_t each = s.channels / s.groups, group_wide = all / s.groups, in_group = padded % group_wide, ch = padded / group_wide * each + in_group;
    const float rate = in_group < each && n < s.states ? s.a[ch * s.states + n] * (kLog2e / 3.0f) : 0.0f;     // (a third)
    const bool backwards = blockIdx.z != 0;
    float* const values = backwards ? g.back : s.ends;
    float carry = 0.0f;
    uint32_t turn = 0;
    for (uint32_t base = 0; base < s.per_span; base += kCarryLines * kCarryChunks, turn ^= 1) {
        float v[kCarryChunks], keep[kCarryChunks];
        bool open[kCarryChunks];
        const uint32_t first = base + line * kCarryChunks;
        // (all loads first, the last chunk's again where there are fewer)
        auto id_of = [&](int i) {
            const uint32_t c = first + i < s.per_span ? first + i : s.per_span - 1;
            return (backwards ? s.per_span - 1 - c : c) * spans + span;
        };
#pragma unroll
        for (int i = 0; i < kCarryChunks; ++i) {
            const uint64_t id = id_of(i);
            v[i] = values[id * one + rest];
            keep[i] = s.sums[id * all + padded];
            open[i] = g.closed == nullptr || g.closed[id] == 0;
        }
        float step = 0.0f, sum = 0.0f;         // step: the sum of d
        bool shut = false;
#pragma unroll
        for (int i = 0; i < kCarryChunks; ++i) {
            if (first + i < s.per_span) step += keep[i];
            keep[i] = third_of(keep[i], rate);
            if (first + i >= s.per_span) break;
            sum = open[i] ? carried(keep[i], sum, v[i]) : v[i];
            shut |= !open[i];
        }
        steps[turn][line][lane] = third_of(step, rate);
        sums[turn][line][lane] = sum;
        closed[turn][line][lane] = shut;
        __syncthreads();
        float mine = carry;
        for (uint32_t l = 0; l < kCarryLines; ++l) {
            if (l == line) mine = carry;
            carry = closed[turn][l][lane] ? sums[turn][l][lane] : carried(steps[turn][l][lane], carry, sums[turn][l][lane]);
        }
#pragma unroll
        for (int i = 0; i < kCarryChunks; ++i) {
            if (first + i >= s.per_span) break;
            if (real) values[id_of(i) * one + rest] = mine;
            mine = open[i] ? carried(keep[i], mine, v[i]) : v[i];
        }
    }
}

// Sums over the 64 / P channels of a wavefront that stand side by side in the low bits of the lane, of eight values at once; each step leaves half as many to each lane.
// Lane l ends with the sum of value share_value<P>(l, i) in v[i], i < share_count<P>.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
#pragma clang fp contract(off)
    return x + dpp_of<CTRL>(x);                // (contracted with the product that x is, the lanes' exchange would be an operation of its own)
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141;
template <int P> constexpr int share_count = P == 16 ? 2 : 1;
template <int P>
__device__ __forceinline__ int share_value(int lane, int i) {
    const int b5 = lane >> 5 & 1, b4 = lane >> 4 & 1, b3 = lane >> 3 & 1, b2 = lane >> 2 & 1, b1 = lane >> 1 & 1, b0 = lane & 1;
    if (P == 1) return 4 * b5 + 2 * b4 + b3;
    if (P == 2) return 4 * b4 + 2 * b3 + b2;
    if (P == 4) return 4 * b3 + 2 * b2 + b1;
    if (P == 8) return 4 * b2 + 2 * b1 + b0;
    return 4 * b1 + 2 * b0 + i;
}
template <int CTRL, int COUNT>
__device__ __forceinline__ void halve(float* v, bool high) {
#pragma unroll
    for (int i = 0; i < COUNT / 2; ++i) {
        const float low = add_dpp<CTRL>(v[i]), up = add_dpp<CTRL>(v[i + COUNT / 2]);
        v[i] = high ? up : low;
    }
}
template <int P>
__device__ __forceinline__ void sum_shares(float (&v)[8], int lane) {
    if constexpr (P == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = swap_add32(v[i], v[i + 4]);
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = swap_add16(v[i], v[i + 2]);
        halve<kRor8, 2>(v, lane & 8);
        v[0] = add_dpp<kXor1>(add_dpp<kXor2>(add_dpp<kHalfMirror>(v[0])));
    } else if constexpr (P == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = swap_add16(v[i], v[i + 4]);
        halve<kRor8, 4>(v, lane & 8);
        halve<kHalfMirror, 2>(v, lane & 4);
        v[0] = add_dpp<kXor1>(add_dpp<kXor2>(v[0]));
    } else if constexpr (P == 4) {
        halve<kRor8, 8>(v, lane & 8);
        halve<kHalfMirror, 4>(v, lane & 4);
        halve<kXor2, 2>(v, lane & 2);
        v[0] = add_dpp<kXor1>(v[0]);
    } else if constexpr (P == 8) {
        halve<kHalfMirror, 8>(v, lane & 4);
        halve<kXor2, 4>(v, lane & 2);
        halve<kXor1, 2>(v, lane & 1);
    } else {
        halve<kXor2, 8>(v, lane & 2);
        halve<kXor1, 4>(v, lane & 1);
    }
}

template <typename T, int P>
__global__ __launch_bounds__(kScanThreads, P == 16 ? 2 : 3) void selective_grad_kernel(SelectiveGrad g, uint32_t blocks) {
    typedef GradTile<T, P> Tile;
    constexpr int K = 4, kWide = 64 / P, kTile = Tile::kTile, kStates = Tile::kStates, kChannels = Tile::kChannels, kTurns = kTile / kTurn;
    __shared__ __attribute__((aligned(16))) float ds[kTile][kChannels], us[kTile][kChannels];          // d, d x; then sum g b and sum g a exp(d a) h
    __shared__ __attribute__((aligned(16))) float dys[kTile][kChannels];                               // dy; then y
    __shared__ __attribute__((aligned(16))) float bs[kTile][kStates], cs[kTile][kStates];
    __shared__ float fronts[kTurns][K][kScanThreads];      // the states in front of each turn
    __shared__ float shares[2][4][kTurn][2 * kStates];     // a turn's sums of db and dc over each wavefront's channels
    if (workgroup() >= blocks) return;
    const Selective& s = g.s;
    const Slab<P> slab(s, s.per_span);
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wide = wave * kWide + lane % kWide, n0 = lane / kWide * K, ch = slab.first + wide;
    const bool real = ch < slab.end;
    const uint32_t t0 = slab.chunk * kTile, t1 = s.span - t0 < kTile ? s.span : t0 + kTile;
    const Bounds bounds = {s.offsets, (uint32_t)s.sequences, s.span};
    const uint32_t begin = s.offsets != nullptr ? bounds.at(0) : 0, finish = s.offsets != nullptr ? bounds.at(bounds.count) : s.span;
    const uint64_t spans = s.offsets != nullptr ? 1 : s.sequences, all = (uint64_t)s.slabs * s.groups * kChannels, id = slab.chunk * spans + slab.span;
    const uint64_t place = id * all + slab.padded + wide;
    {
        Tile tile;
        tile.load(g, slab, t0, t1, begin, finish);
        tile.put(g, slab, t0, t1, begin, finish, ds, us, dys, bs, cs);
    }
    float rate[K], h[K], back[K], da[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        rate[k] = real && n0 + k < s.states ? s.a[(uint64_t)ch * s.states + n0 + k] * kLog2e : 0.0f;
        h[k] = s.per_span > 1 ? s.ends[place * kStates + n0 + k] : 0.0f;
        back[k] = s.per_span > 1 ? g.back[place * kStates + n0 + k] : 0.0f;
        da[k] = 0.0f;
    }
    Place at;
    at.find(bounds, slab.span, t0);
    if (at.start == t0 || !at.inside) load_states(at.inside ? s.state : nullptr, at.seq, s, ch, n0, real, h);
    __syncthreads();

    // Turns with a sequence's first or last token in them go the longer way (of a sequence that is a span by itself: only where something is given or wanted there).
    const bool starts = s.offsets != nullptr || g.dstate != nullptr, stops = s.offsets != nullptr || g.dfinal != nullptr;
    uint32_t quiet = 0;
    auto enter = [&](uint32_t t) {             // forwards, at a bound
        at.pass(bounds, t);
        load_states(at.inside ? s.state : nullptr, at.seq, s, ch, n0, real, h);
    };
    for (uint32_t turn = 0; turn < kTurns; ++turn) {
        const uint32_t j = turn * kTurn, t = t0 + j;
#pragma unroll
        for (int k = 0; k < K; ++k) fronts[turn][k][tid] = h[k];
        if (t >= t1) break;
        if (at.next == t && turn != 0) {       // (the states in front of the turn are those behind the bound)
            enter(t);
#pragma unroll
            for (int k = 0; k < K; ++k) fronts[turn][k][tid] = h[k];
        }
        if ((at.start < t || !starts) && (at.next > t + kTurn || !stops)) quiet |= 1u << turn;
        if (turn + 1 == kTurns || t + kTurn >= t1) break;
        auto token = [&](uint32_t i) {
            const float d = ds[i][wide], u = us[i][wide];
#pragma unroll
            for (int k = 0; k < K; ++k) h[k] = __builtin_fmaf(__builtin_amdgcn_exp2f(d * rate[k]), h[k], u * bs[i][n0 + k]);
        };
        if (at.next >= t + kTurn) {
#pragma unroll
            for (int i = 0; i < kTurn; ++i) token(j + i);
        } else {
            for (uint32_t i = 0; i < kTurn; ++i) {
                if (at.next == t + i) enter(t + i);
                token(j + i);
            }
        }
    }

    // From the last turn to the first.  `at` is the place of the token at hand.
    const uint32_t turns = (t1 - t0 + kTurn - 1) / kTurn;
    at.find(bounds, slab.span, t1 - 1);
    auto turn_of = [&](auto plain, uint32_t turn) {
        constexpr bool kPlain = decltype(plain)::value;
        const uint32_t j = turn * kTurn, t = t0 + j;
        float a[kTurn][K], ah[kTurn][K];       // the factors, and what is left of the states in front
#pragma unroll
        for (int k = 0; k < K; ++k) h[k] = fronts[turn][k][tid];
        Place ahead = at;
        if (!kPlain) ahead.find(bounds, slab.span, t);
#pragma unroll
        for (int i = 0; i < kTurn; ++i) {
            if (!kPlain && i != 0 && ahead.next == t + i && t + i < t1) {
                ahead.pass(bounds, t + i);
                load_states(ahead.inside ? s.state : nullptr, ahead.seq, s, ch, n0, real, h);
            }
            const float d = ds[j + i][wide], u = us[j + i][wide];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                a[i][k] = __builtin_amdgcn_exp2f(d * rate[k]);
                ah[i][k] = a[i][k] * h[k];
                h[k] = __builtin_fmaf(u, bs[j + i][n0 + k], ah[i][k]);
            }
        }
#pragma unroll
        for (int half = kTurn / kTokens - 1; half >= 0; --half) {
            float ys[kTokens], gbs[kTokens], ws[kTokens];
#pragma unroll
            for (int m = kTokens - 1; m >= 0; --m) {
                const int i = half * kTokens + m;
                if (!kPlain && at.inside && at.next == t + i + 1) load_states(g.dfinal, at.seq, s, ch, n0, real, back);
                const float d = ds[j + i][wide], u = us[j + i][wide], dy = dys[j + i][wide];
                float y = 0.0f, gb = 0.0f, w = 0.0f, v[8];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const float b = bs[j + i][n0 + k], c = cs[j + i][n0 + k];
                    const float now = __builtin_fmaf(u, b, ah[i][k]), grad = __builtin_fmaf(c, dy, back[k]), through = grad * ah[i][k];
                    y = __builtin_fmaf(c, now, y);
                    gb = __builtin_fmaf(grad, b, gb);
                    w = __builtin_fmaf(through, rate[k], w);
                    da[k] = __builtin_fmaf(through, d, da[k]);
                    v[k] = grad * u;
                    v[4 + k] = dy * now;
                    back[k] = a[i][k] * grad;
                }
                if (!kPlain && at.start == t + i) {        // the place's first token: what is in front of it belongs to another sequence, or to none
                    if (at.inside) store_states(g.dstate, at.seq, s, ch, n0, real, back);
#pragma unroll
                    for (int k = 0; k < K; ++k) back[k] = 0.0f;
                    if (t + i != 0) at.find(bounds, slab.span, t + i - 1);
                }
                ys[m] = y;
                gbs[m] = gb;
                ws[m] = w;
                sum_shares<P>(v, lane);
                // (lanes with the same sum all write it: a branch here would part the tokens' operations)
#pragma unroll
                for (int e = 0; e < share_count<P>; ++e) {
                    const int value = share_value<P>(lane, e);
                    shares[turn & 1][wave][i][(value >> 2) * kStates + n0 + (value & 3)] = v[e];
                }
            }
            sum_parts<P>(ys);
            sum_parts<P>(gbs);
            sum_parts<P>(ws);
#pragma unroll
            for (int i = 0; i < sum_count<P>; ++i) {
                const uint32_t to = j + half * kTokens + sum_token<P>(lane, i);
                ds[to][wide] = gbs[i];
                us[to][wide] = ws[i];
                dys[to][wide] = ys[i];
            }
        }
    };
    const uint64_t tokens = (uint64_t)s.span * spans;
    for (uint32_t turn = turns; turn-- > 0;) {
        if (quiet >> turn & 1) turn_of(std::true_type(), turn);
        else turn_of(std::false_type(), turn);
        __syncthreads();
        for (uint32_t e = tid; e < kTurn * 2 * kStates; e += kScanThreads) {
            const uint32_t i = e / (2 * kStates), v = e % (2 * kStates), t = t0 + turn * kTurn + i;
            const auto& part = shares[turn & 1];
            const float sum = (part[0][i][v] + part[1][i][v]) + (part[2][i][v] + part[3][i][v]);
            if (t < t1) g.shares[(slab.padded / kChannels * tokens + slab.span * (uint64_t)s.span + t) * (2 * kStates) + v] = sum;
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) s.ends[place * kStates + n0 + k] = da[k];
    if (s.span == 0 && s.offsets == nullptr) {
        load_states(g.dfinal, slab.span, s, ch, n0, real, h);
        store_states(g.dstate, slab.span, s, ch, n0, real, h);
    }
    if (s.offsets != nullptr && g.dstate != nullptr)
        for (uint32_t e = slab.chunk; e < bounds.count; e += s.per_span)
            if (bounds.at(e + 1) <= bounds.at(e)) {
                load_states(g.dfinal, e, s, ch, n0, real, h);
                store_states(g.dstate, e, s, ch, n0, real, h);
            }

    // What is each token's and channel's own, by the threads that loaded it: loaded once more, as the registers are the turns' (two wavefronts on a SIMD with them
    // kept, three without).
    Tile tile;
    tile.load(g, slab, t0, t1, begin, finish);
    const uint32_t t = t0 + tile.token;
    const bool inside = tile.inside;
    if (tile.token < kTile) {
        float gb[kVec], w[kVec], y[kVec], skip[kVec], dx[kVec], ddt[kVec];
        get_vec(ds[tile.token] + tile.wide, gb);
        get_vec(us[tile.token] + tile.wide, w);
        get_vec(dys[tile.token] + tile.wide, y);
#pragma unroll
        for (int i = 0; i < kVec; ++i) skip[i] = 0.0f;
        if (s.skip != nullptr && tile.there) load_vec(s.skip, (uint64_t)tile.first, (uint64_t)slab.end, skip);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            dx[i] = __builtin_fmaf(gb[i], tile.d[i], skip[i] * tile.dy[i]);
            ddt[i] = __builtin_fmaf(gb[i], (float)tile.x[i], w[i] * (1.0f / kLog2e));
        }
        if (s.softplus)
#pragma unroll
            for (int i = 0; i < kVec; ++i) ddt[i] *= sigmoid_of(tile.raw[i]);
        if (!inside)
#pragma unroll
            for (int i = 0; i < kVec; ++i) dx[i] = ddt[i] = 0.0f;
        // (each thread overwrites what only it has read)
        float own[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) own[i] = inside ? tile.dy[i] * (float)tile.x[i] : 0.0f;
        put_vec(ds[tile.token] + tile.wide, own);
        put_vec(us[tile.token] + tile.wide, ddt);
        if (tile.there) {
            const uint64_t row = (slab.span * (uint64_t)s.span + t) * s.channels;
            store_vec(static_cast<T*>(g.dx) + row, tile.first, slab.end, dx);
            store_vec(static_cast<T*>(g.ddt) + row, tile.first, slab.end, ddt);
            if (g.dgate != nullptr) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float z = (float)tile.gate[i], f = sigmoid_of(z);
                    y[i] = (float)tile.dout[i] * __builtin_fmaf(skip[i], (float)tile.x[i], y[i]) * __builtin_fmaf(z * f, 1.0f - f, f);
                }
                if (!inside)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) y[i] = 0.0f;
                store_vec(static_cast<T*>(g.dgate) + row, tile.first, slab.end, y);
            }
        }
    }
    if (g.dskip == nullptr && g.dbias == nullptr) return;
    __syncthreads();
    for (uint32_t e = tid; e < 2 * kChannels; e += kScanThreads) {
        const float* const from = e < kChannels ? &ds[0][e] : &us[0][e - kChannels];
        float v = 0.0f;
        for (int j = 0; j < kTile; ++j) v += from[j * kChannels];
        g.means[(id * 2 + e / kChannels) * all + slab.padded + e % kChannels] = v;
    }
}

// db and dc: the sums over a group's slabs.
template <typename T, int NP>
__global__ __launch_bounds__(kScanThreads) void selective_shares_kernel(SelectiveGrad g, uint64_t tokens) {
    const Selective& s = g.s;
    const uint64_t at = (uint64_t)workgroup() * kScanThreads + threadIdx.x, n = at % (2 * NP), rest = at / (2 * NP), group = rest % s.groups, token = rest / s.groups;
    if (token >= tokens || n % NP >= s.states) return;
    const float* from = g.shares + ((uint64_t)group * s.slabs * tokens + token) * (2 * NP) + n;
    float v = 0.0f;
    for (uint32_t i = 0; i < s.slabs; ++i) v += from[i * tokens * (2 * NP)];
    static_cast<T*>(n < NP ? g.db : g.dc)[(token * s.groups + group) * s.states + n % NP] = (T)v;
}

// da, dskip and dbias: the sums over chunks.  64 columns a workgroup, sixteen lines of additions for each.
template <int NP>
__global__ __launch_bounds__(1024) void selective_means_kernel(SelectiveGrad g, uint64_t all, uint64_t chunks) {
    __shared__ float sums[16][64];
    const Selective& s = g.s;
    const uint64_t rates = all * NP, at = (uint64_t)workgroup() * 64 + threadIdx.x % 64;
    const uint32_t line = threadIdx.x / 64;
    float v = 0.0f;
    if (at < rates) {
        for (uint64_t c = line; c < chunks; c += 16) v += s.ends[c * rates + at];
    } else if (at < rates + 2 * all && (g.dskip != nullptr || g.dbias != nullptr)) {
        for (uint64_t c = line; c < chunks; c += 16) v += g.means[c * 2 * all + (at - rates)];
    }
    sums[line][threadIdx.x % 64] = v;
    __syncthreads();
    if (line != 0 || at >= rates + 2 * all) return;
    v = 0.0f;
    for (int i = 0; i < 16; ++i) v += sums[i][threadIdx.x];
    const uint64_t padded = at < rates ? at / NP : (at - rates) % all;
    const uint64_t each = s.channels / s.groups, group_wide = all / s.groups, in_group = padded % group_wide, ch = padded / group_wide * each + in_group;
    if (in_group >= each) return;
    if (at < rates) {
        if (at % NP < s.states) g.da[ch * s.states + at % NP] = v;
    } else if (at - rates < all) {
        if (g.dskip != nullptr) g.dskip[ch] = v;
    } else if (g.dbias != nullptr) {
        g.dbias[ch] = v;
    }
}

}  // namespace layers
}  // namespace tcr
