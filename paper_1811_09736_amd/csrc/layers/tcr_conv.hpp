// Short causal convolution of every channel with its own taps, W of them:
//
//     s_t = bias + sum_j w[j] x_{t-W+1+j},   y_t = s_t, or s_t sigmoid(s_t)
// where the W - 1 inputs in front of a sequence come from its state, or are 0.  A thread takes a few channels and a run of tokens and keeps the last W - 1
// inputs in registers: every input is loaded once, those in front of a run once more.  Bound by memory.
//
// Gradients, with ds_t = dout_t (y_t)':   dx_t = sum_m w[W-1-m] ds_{t+m} over the sequence's tokens,   dw[j] = sum_t ds_t x_{t-W+1+j},   dbias = sum_t ds_t.
// The run goes forwards all the same: what ds_t gives the W - 1 inputs in front waits in registers until the last of it has come.
#pragma once
#include "tcr_places.hpp"

namespace tcr {
namespace layers {

constexpr int kConvThreads = 256;

struct Conv {
    const void *x, *weight, *bias, *state;     // bias, state: NULL for none
    void *out, *fin;                           // fin: NULL: not wanted
    const uint64_t* offsets;
    int64_t x_seq, x_tok, out_seq, out_tok;
    uint64_t sequences;
    uint32_t span, run, runs, channels, act;   // tokens of a span and of a run, runs of a span
    uint32_t lanes;                            // of a run side by side (a power of two, 64 at most), each with some channels
};

struct ConvGrad {
    Conv c;                                    // out: dout
    const void* dfinal;                        // NULL: none
    void *dx, *dstate;                         // dstate: NULL: not wanted
    float* part;                               // [parts][W + 1][channels] sums of dw and dbias
    uint32_t parts;                            // workgroups of a slab; they take the runs in turns
};

template <typename T, int V> struct Some { typedef T v __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };

// V elements as they are in memory.  WHOLE: the number of columns is a multiple of V, so that no vector goes beyond the end and no branch parts a load from the next.
template <typename T, int V, bool WHOLE>
__device__ __forceinline__ typename Some<T, V>::v raw_some(const T* row, uint32_t col, uint32_t cols) {
    if (WHOLE || col + V <= cols) return *reinterpret_cast<const typename Some<T, V>::v*>(row + col);
    typename Some<T, V>::v x;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = col + i < cols ? row[col + i] : (T)0.0f;
    return x;
}
template <typename T, int V, bool WHOLE>
__device__ __forceinline__ void load_some(const T* row, uint32_t col, uint32_t cols, float (&v)[V]) {
    const typename Some<T, V>::v x = raw_some<T, V, WHOLE>(row, col, cols);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)x[i];
}
template <typename T, int V, bool WHOLE>
__device__ __forceinline__ void store_some(T* row, uint32_t col, uint32_t cols, const float (&v)[V]) {
    if (WHOLE || col + V <= cols) {
        typename Some<T, V>::v x;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (T)v[i];
        *reinterpret_cast<typename Some<T, V>::v*>(row + col) = x;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (col + i < cols) row[col + i] = (T)v[i];
    }
}

// The W - 1 inputs in front of token t of the sequence at `at`, the oldest first; those in front of the sequence from its state.
template <typename T, int V, int W, bool WHOLE>
__device__ __forceinline__ void load_front(const Conv& a, const T* x_row, const Place& at, uint32_t t, uint32_t col, float (&x)[W - 1][V]) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int64_t token = (int64_t)t - (W - 1) + j;
        if (at.inside && token >= (int64_t)at.start) load_some<T, V, WHOLE>(x_row + token * a.x_tok, col, a.channels, x[j]);
        else if (at.inside && a.state != nullptr)
            load_some<T, V, WHOLE>(static_cast<const T*>(a.state) + ((uint64_t)at.seq * (W - 1) + (W - 1 + token - at.start)) * a.channels, col, a.channels, x[j]);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) x[j][i] = 0.0f;
    }
}
// Rows of an array of states, [sequence][W - 1][channel].
template <typename T, int V, int W, bool WHOLE>
__device__ __forceinline__ void store_rows(void* states, uint64_t seq, const Conv& a, uint32_t col, const float (&x)[W - 1][V]) {
    if (states == nullptr) return;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) store_some<T, V, WHOLE>(static_cast<T*>(states) + (seq * (W - 1) + j) * a.channels, col, a.channels, x[j]);
}

// The taps of V channels, which lie behind one another: whole vectors where all of the channels are there.
template <typename T, int V, int W, bool WHOLE>
__device__ __forceinline__ void load_taps(const Conv& a, const T* weight, uint32_t col, float (&w)[W][V], float (&bias)[V]) {
    const T* const from = weight + (uint64_t)col * W;
    if (WHOLE || col + V <= a.channels) {
        float flat[V * W];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const typename Some<T, V>::v part = *reinterpret_cast<const typename Some<T, V>::v*>(from + j * V);
#pragma unroll
            for (int i = 0; i < V; ++i) flat[j * V + i] = (float)part[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][i] = flat[i * W + j];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][i] = col + i < a.channels ? (float)from[i * W + j] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) bias[i] = 0.0f;
    if (a.bias != nullptr) load_some<T, V, WHOLE>(static_cast<const T*>(a.bias), col, a.channels, bias);
}

// What a thread works at: channels from col on, tokens t0 .. t1 - 1 of a span.
struct Part {
    uint32_t col, run, span, t0, t1;
    // Slab `block % slabs` of the channels; runs by `place`, of the spans one after the other.
    template <int V>
    __device__ __forceinline__ uint32_t slabs(const Conv& a) {
        return ((a.channels + V - 1) / V + a.lanes - 1) / a.lanes;
    }
    template <int V>
    __device__ __forceinline__ uint64_t first(const Conv& a) {
        const uint32_t n = slabs<V>(a), block = workgroup();
        col = (block % n * a.lanes + threadIdx.x % a.lanes) * V;
        return (uint64_t)(block / n) * (kConvThreads / a.lanes) + threadIdx.x / a.lanes;
    }
    __device__ __forceinline__ bool set(const Conv& a, uint64_t place) {
        if (place >= (a.offsets != nullptr ? 1 : a.sequences) * a.runs || col >= a.channels) return false;
        run = (uint32_t)(place % a.runs);
        span = (uint32_t)(place / a.runs);
        t0 = run * a.run;
        t1 = a.span - t0 < a.run ? a.span : t0 + a.run;
        return true;
    }
};

template <typename T, int V, int W, bool WHOLE>
__global__ __launch_bounds__(kConvThreads) void conv_kernel(Conv a) {
    Part my;
    if (!my.set(a, my.first<V>(a))) return;
    const Bounds bounds = {a.offsets, (uint32_t)a.sequences, a.span};
    const T* const x_row = static_cast<const T*>(a.x) + my.span * a.x_seq;
    T* const out_row = static_cast<T*>(a.out) + my.span * a.out_seq;
    float w[W][V], bias[V], x[W][V];
    load_taps<T, V, W, WHOLE>(a, static_cast<const T*>(a.weight), my.col, w, bias);
    Place at;
    at.find(bounds, my.span, my.t0);
    {
        float front[W - 1][V];
        load_front<T, V, W, WHOLE>(a, x_row, at, my.t0, my.col, front);
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) x[j][i] = front[j][i];
    }
    constexpr int kAhead = 4;
    for (uint32_t t = my.t0; t < my.t1; t += kAhead) {
        typename Some<T, V>::v next[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) next[u] = raw_some<T, V, WHOLE>(x_row + (t + u < my.t1 ? t + u : my.t1 - 1) * a.x_tok, my.col, a.channels);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (t + u >= my.t1) break;
            if (at.next == t + u) {
                float front[W - 1][V];
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) front[j][i] = x[j][i];
                if (at.inside) store_rows<T, V, W, WHOLE>(a.fin, at.seq, a, my.col, front);
                at.pass(bounds, t + u);
                load_front<T, V, W, WHOLE>(a, x_row, at, t + u, my.col, front);
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) x[j][i] = front[j][i];
            }
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[W - 1][i] = (float)next[u][i];
                float s = bias[i];
#pragma unroll
                for (int j = 0; j < W; ++j) s = __builtin_fmaf(w[j][i], x[j][i], s);
                y[i] = s;
#pragma unroll
                for (int j = 0; j + 1 < W; ++j) x[j][i] = x[j + 1][i];
            }
            if (a.act)
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] *= sigmoid_of(y[i]);
            if (!at.inside)
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = 0.0f;
            store_some<T, V, WHOLE>(out_row + (t + u) * a.out_tok, my.col, a.channels, y);
        }
    }
    float front[W - 1][V];
    if (at.inside && at.next == my.t1) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) front[j][i] = x[j][i];
        store_rows<T, V, W, WHOLE>(a.fin, at.seq, a, my.col, front);
    }
    if (a.offsets != nullptr && a.fin != nullptr)
        for (uint32_t e = my.run; e < bounds.count; e += a.runs)
            if (bounds.at(e + 1) <= bounds.at(e)) {
                const Place empty = {e, 0, 0, true};
                load_front<T, V, W, WHOLE>(a, x_row, empty, 0, my.col, front);
                store_rows<T, V, W, WHOLE>(a.fin, e, a, my.col, front);
            }
}

// One token for every sequence.
template <typename T, int V, int W, bool WHOLE>
__global__ __launch_bounds__(kConvThreads) void conv_step_kernel(Conv a) {
    const uint32_t cols = (a.channels + V - 1) / V;
    const uint64_t place = (uint64_t)workgroup() * kConvThreads + threadIdx.x, seq = place / cols;
    const uint32_t col = (uint32_t)(place % cols) * V;
    if (seq >= a.sequences) return;
    float w[W][V], bias[V], x[W][V], rows[W - 1][V], y[V];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) load_some<T, V, WHOLE>(static_cast<const T*>(a.state) + (seq * (W - 1) + j) * a.channels, col, a.channels, x[j]);
    load_some<T, V, WHOLE>(static_cast<const T*>(a.x) + seq * a.x_seq, col, a.channels, x[W - 1]);
    load_taps<T, V, W, WHOLE>(a, static_cast<const T*>(a.weight), col, w, bias);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float s = bias[i];
#pragma unroll
        for (int j = 0; j < W; ++j) s = __builtin_fmaf(w[j][i], x[j][i], s);
        y[i] = a.act ? s * sigmoid_of(s) : s;
#pragma unroll
        for (int j = 0; j + 1 < W; ++j) rows[j][i] = x[j + 1][i];
    }
    store_some<T, V, WHOLE>(static_cast<T*>(a.out) + seq * a.out_seq, col, a.channels, y);
    store_rows<T, V, W, WHOLE>(a.fin, seq, a, col, rows);
}

template <typename T, int V, int W, bool WHOLE>
__global__ __launch_bounds__(kConvThreads) void conv_grad_kernel(ConvGrad g) {
    __shared__ float sums[kConvThreads * V];
    const Conv& a = g.c;
    Part my;
    const uint32_t slabs = my.slabs<V>(a);
    const uint64_t step = (uint64_t)g.parts * (kConvThreads / a.lanes);
    float dw[W + 1][V];                        // the last: of the bias
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) dw[j][i] = 0.0f;
    for (uint64_t place = my.first<V>(a); my.set(a, place); place += step) {
        const Bounds bounds = {a.offsets, (uint32_t)a.sequences, a.span};
        const T* const x_row = static_cast<const T*>(a.x) + my.span * a.x_seq;
        const T* const dout_row = static_cast<const T*>(a.out) + my.span * a.out_seq;
        T* const dx_row = static_cast<T*>(g.dx) + (uint64_t)my.span * a.span * a.channels;
        float w[W][V], bias[V], x[W - 1][V], wait[W - 1][V];               // wait[m]: of the input at t - (W - 1) + m
        load_taps<T, V, W, WHOLE>(a, static_cast<const T*>(a.weight), my.col, w, bias);
        Place at;
        at.find(bounds, my.span, my.t0);
        load_front<T, V, W, WHOLE>(a, x_row, at, my.t0, my.col, x);
        auto clear = [&] {
#pragma unroll
            for (int m = 0; m < W - 1; ++m)
#pragma unroll
                for (int i = 0; i < V; ++i) wait[m][i] = 0.0f;
        };
        // the gradient of the input at `token`: of the run's own, or of its own sequences' states
        auto put = [&](int64_t token, const float (&v)[V]) {
            if (!at.inside) return;
            if (token >= (int64_t)at.start) {
                if (token >= (int64_t)my.t0 && token < (int64_t)my.t1) store_some<T, V, WHOLE>(dx_row + token * a.channels, my.col, a.channels, v);
            } else if (g.dstate != nullptr && at.start >= my.t0 && (at.start < my.t1 || a.span == 0)) {
                store_some<T, V, WHOLE>(static_cast<T*>(g.dstate) + ((uint64_t)at.seq * (W - 1) + (W - 1 + token - at.start)) * a.channels, my.col, a.channels, v);
            }
        };
        // behind the last token of a sequence, at `end`: all that waits, and what comes from the state behind it
        auto finish = [&](uint32_t end) {
            if (!at.inside) return;
#pragma unroll
            for (int m = 0; m < W - 1; ++m) {
                if (g.dfinal != nullptr) {
                    float more[V];
                    load_some<T, V, WHOLE>(static_cast<const T*>(g.dfinal) + ((uint64_t)at.seq * (W - 1) + m) * a.channels, my.col, a.channels, more);
#pragma unroll
                    for (int i = 0; i < V; ++i) wait[m][i] += more[i];
                }
                put((int64_t)end - (W - 1) + m, wait[m]);
            }
        };
        clear();
        // one token: the slope, the sums (of the run's `own`), what it gives the inputs in front; `done` is the gradient of the input W - 1 tokens in front
        auto token = [&](const float (&now)[V], float (&ds)[V], bool own, float (&done)[V]) {
            if (a.act)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float s = bias[i];
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) s = __builtin_fmaf(w[j][i], x[j][i], s);
                    s = __builtin_fmaf(w[W - 1][i], now[i], s);
                    const float z = sigmoid_of(s);
                    ds[i] *= __builtin_fmaf(s * z, 1.0f - z, z);
                }
            if (own)
#pragma unroll
                for (int i = 0; i < V; ++i) {
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) dw[j][i] = __builtin_fmaf(ds[i], x[j][i], dw[j][i]);
                    dw[W - 1][i] = __builtin_fmaf(ds[i], now[i], dw[W - 1][i]);
                    dw[W][i] += ds[i];
                }
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int m = 0; m < W - 1; ++m) wait[m][i] = __builtin_fmaf(w[m][i], ds[i], wait[m][i]);
                done[i] = wait[0][i];
#pragma unroll
                for (int m = 0; m + 1 < W - 1; ++m) wait[m][i] = wait[m + 1][i];
                wait[W - 2][i] = w[W - 1][i] * ds[i];
#pragma unroll
                for (int j = 0; j + 1 < W - 1; ++j) x[j][i] = x[j + 1][i];
                x[W - 2][i] = now[i];
            }
        };
        // (and the W - 1 tokens behind the run, whose gradients go to the run's last inputs)
        const uint32_t last = my.t1 + (W - 1);
        for (uint32_t t = my.t0;;) {
            if (at.inside) {
                // as far as the sequence or the run goes: the loads of kAhead tokens ahead of their use
                constexpr uint32_t kAhead = 4;
                const uint32_t to = at.next < last ? at.next : last;
                for (; t < to; t += kAhead) {
                    typename Some<T, V>::v nows[kAhead], dss[kAhead];
#pragma unroll
                    for (uint32_t u = 0; u < kAhead; ++u) {
                        const uint32_t from = t + u < to ? t + u : to - 1;
                        nows[u] = raw_some<T, V, WHOLE>(x_row + from * a.x_tok, my.col, a.channels);
                        dss[u] = raw_some<T, V, WHOLE>(dout_row + from * a.out_tok, my.col, a.channels);
                    }
#pragma unroll
                    for (uint32_t u = 0; u < kAhead; ++u) {
                        if (t + u >= to) break;
                        float now[V], ds[V], done[V];
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            now[i] = (float)nows[u][i];
                            ds[i] = (float)dss[u][i];
                        }
                        token(now, ds, t + u < my.t1, done);
                        put((int64_t)(t + u) - (W - 1), done);
                    }
                }
                t = to;
                if (t != at.next) break;
                finish(t);
            } else {
                float none[V];
#pragma unroll
                for (int i = 0; i < V; ++i) none[i] = 0.0f;
                for (; t < my.t1 && t != at.next; ++t) store_some<T, V, WHOLE>(dx_row + (uint64_t)t * a.channels, my.col, a.channels, none);
            }
            if (t >= my.t1) break;
            at.pass(bounds, t);
            load_front<T, V, W, WHOLE>(a, x_row, at, t, my.col, x);
            clear();
        }
        if (a.offsets != nullptr && g.dstate != nullptr)
            for (uint32_t e = my.run; e < bounds.count; e += a.runs)
                if (bounds.at(e + 1) <= bounds.at(e)) {
                    Conv of = a;
                    of.state = g.dfinal;
                    const Place empty = {e, 0, 0, true};
                    load_front<T, V, W, WHOLE>(of, x_row, empty, 0, my.col, x);
                    store_rows<T, V, W, WHOLE>(g.dstate, e, a, my.col, x);
                }
    }
    // the sums of the workgroup's runs, always in the same order
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) sums[i * kConvThreads + threadIdx.x] = dw[j][i];
        __syncthreads();
        for (uint32_t o = threadIdx.x; o < a.lanes * V; o += kConvThreads) {
            const uint32_t lane = o % a.lanes, i = o / a.lanes, c = (workgroup() % slabs * a.lanes + lane) * V + i;
            float v = 0.0f;
            for (uint32_t r = lane; r < kConvThreads; r += a.lanes) v += sums[i * kConvThreads + r];
            if (c < a.channels) g.part[((uint64_t)(workgroup() / slabs) * (W + 1) + j) * a.channels + c] = v;
        }
    }
}

// dweight and dbias from the workgroups' sums: 64 columns of [W + 1][channels] a workgroup, four lines of additions for each.
template <typename T, int W>
__global__ __launch_bounds__(kConvThreads) void conv_parts_kernel(const float* part, T* dweight, T* dbias, uint32_t channels, uint32_t parts) {
    __shared__ float sums[kConvThreads];
    const uint64_t all = (uint64_t)channels * (W + 1), at = (uint64_t)workgroup() * 64 + threadIdx.x % 64;
    float v = 0.0f;
    if (at < all)
        for (uint32_t p = threadIdx.x / 64; p < parts; p += kConvThreads / 64) v += part[p * all + at];
    sums[threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.x >= 64 || at >= all) return;
    v = (sums[threadIdx.x] + sums[threadIdx.x + 64]) + (sums[threadIdx.x + 128] + sums[threadIdx.x + 192]);
    const uint32_t j = (uint32_t)(at / channels), c = (uint32_t)(at % channels);
    if (j < W) dweight[(uint64_t)c * W + j] = (T)v;
    else if (dbias != nullptr) dbias[c] = (T)v;
}

}  // namespace layers
}  // namespace tcr
