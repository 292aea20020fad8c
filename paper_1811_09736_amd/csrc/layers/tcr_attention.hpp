// Linear attention with a decay for each head, what its kernels share.
//
// One operation serves the forward pass, its gradients and single tokens: the decayed running sum of outer products
//     S_t = lambda S_{t-1} + b_t c_t^T,     out_t = scale * a_t^T S_t          (S: dk x dv, binary32)
// over each sequence.  With (a, b, c) =
//     (q, k, v)   it is the attention itself;
//     (dout, v, k) the gradient of q;
//     (v, dout, q) and (k, q, dout), from the last token to the first, those of k and v:
//         R_t = lambda R_{t+1} + scale q_t dout_t^T,  dk_t = R_t v_t,  dv_t = R_t^T k_t.
// The gradient of the last state enters R undecayed at the last token, and the gradient of the first state is R_0 decayed
// once more: `late`.
#pragma once
#include "tcr_shared.hpp"

namespace tcr {
namespace layers {

// Rows of one role: token t of sequence s and head h at p + s * seq + t * tok + (h / group) * head elements (packed sequences:
// t counts from the first token of all, seq is 0).
struct View {
    const void* p;
    int64_t seq, tok, head;
    uint32_t group;
};

struct Scan {
    View a, b, c;
    void* out;
    int64_t out_seq, out_tok, out_head;
    const float* init;          // states [sequences][heads], each dk x dv at strides st_row and st_col; nullptr: zeros
    float* fin;                 // nullptr: not wanted
    int64_t st_row, st_col;
    const float* log_decay;     // [heads]
    const uint64_t* offsets;    // nullptr: every sequence has `tokens` tokens
    uint64_t sequences, tokens, total;
    float out_scale, init_mul, fin_mul;
    uint32_t heads, dk, dv;
    uint32_t reverse, late;
};

// The natural logarithm of a head's decay; minus infinity (nothing is kept) as a number whose product with 0 is 0.  (NaN stays, and with it all that the head decays.)
__device__ __forceinline__ float decay_of(const Scan& a, uint32_t h) {
    const float d = a.log_decay[h];
    return d < -1e30f ? -1e30f : d;
}
// decay^steps
__device__ __forceinline__ float decayed(float log_decay, float steps) { return expf(log_decay * steps); }
// A state is multiplied by the same decay^steps chunk after chunk (token after token, block after block).  Near 1 the rounding of that one number, 2^-25, would add up over all
// that the state remembers, to 2e-5 of it after 512 chunks; so where log_decay * steps lies within kNearOne, decay^steps - 1 is worked out too, by its series (whose
// next term is 2^-29 of it there), and the sums below take what the rounding left out.
constexpr float kNearOne = 0.25f;
__device__ __forceinline__ bool near_one(float log_decay, float steps) { return fabsf(log_decay * steps) <= kNearOne; }
__device__ __forceinline__ float less_one(float log_decay, float steps) {
    const float x = log_decay * steps;
    float sum = 1.0f;
#pragma unroll
    for (int i = 7; i >= 2; --i) sum = fmaf(sum * x, 1.0f / (float)i, 1.0f);
    return sum * x;
}
// decay^steps as whole + rest, whole 1 or 0: S + (decay^steps - 1) S.
struct Kept {
    float whole, rest;
};
__device__ __forceinline__ Kept kept(float log_decay, float steps) {
    return near_one(log_decay, steps) ? Kept{1.0f, less_one(log_decay, steps)} : Kept{0.0f, decayed(log_decay, steps)};
}
__device__ __forceinline__ bool nothing(const Kept& k) { return k.whole == 0.0f && k.rest == 0.0f; }
// decay^steps x + y
__device__ __forceinline__ float kept_plus(const Kept& k, float x, float y) { return fmaf(k.whole, x, fmaf(k.rest, x, y)); }

// Tokens of sequence s: where they start and how many; whatever the offsets hold, inside [0, total).
struct Span {
    uint64_t first, count;
};
__device__ __forceinline__ Span span_of(const Scan& a, uint64_t s) {
    if (a.offsets == nullptr) return {s * a.tokens, a.tokens};
    const uint64_t o = a.offsets[s], e = a.offsets[s + 1];
    const uint64_t lo = o < a.total ? o : a.total, hi = e < a.total ? e : a.total;
    return {lo, hi > lo ? hi - lo : 0};
}
// Element offset of a sequence's token 0 in a view.
__device__ __forceinline__ int64_t base_of(const Scan& a, int64_t seq, int64_t tok, uint64_t s, uint64_t first) {
    return a.offsets == nullptr ? (int64_t)s * seq : (int64_t)first * tok;
}

// --------------------------------------------------------------------------------------------- token by token
// S in registers, one workgroup per sequence, head and slab of 4 * LANES columns: thread (row group, lane) holds 4 columns of
// every (256 / LANES)-th row.  A token costs the products with its own row elements and one sum over the rows, across
// lanes and then wavefronts.  For a single token the bound is the state's bytes, read once and written once:
// 256 sequences x 16 heads x 128 x 128 in 107 us, 5.07 TB/s, where a copy reaches 5.2 to 5.5.  Narrow slabs (16 columns) where there are few sequences: 1 sequence of 16 heads
// makes 128 workgroups, 4.5 us.
constexpr int kStepThreads = 256;

template <typename T, int LANES, typename OUT>
__global__ __launch_bounds__(kStepThreads) void attention_step_kernel(const Scan a) {
    constexpr int kRows = kStepThreads / LANES, kPasses = 256 / kRows, kWaves = kStepThreads / 64;
    __shared__ float sums[2][kWaves][4 * LANES];
    const uint32_t slabs = (a.dv + 4 * LANES - 1) / (4 * LANES);
    const uint32_t group = workgroup(), slab = group % slabs, h = group / slabs % a.heads;       // (fewer than 2^29 in all)
    const bool there = group / slabs / a.heads < a.sequences;         // (or a workgroup that nothing is left for)
    const uint64_t s = there ? group / slabs / a.heads : 0;
    const int lane = threadIdx.x % LANES, row0 = threadIdx.x / LANES, wave = threadIdx.x / 64;
    const uint32_t col = slab * 4 * LANES + lane * 4;
    const bool live = there && col < a.dv;
    Span span = span_of(a, s);
    if (!there) span.count = 0;
    const float log_decay = decay_of(a, h), lambda = decayed(log_decay, 1.0f);
    const Kept decay = kept(log_decay, 1.0f);
    const int64_t state = ((int64_t)s * a.heads + h) * a.dk * a.dv;

    f4v acc[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        acc[p] = f4v{0, 0, 0, 0};
        const uint32_t row = p * kRows + row0;
        if (a.init != nullptr && live && row < a.dk) {
            const float* from = a.init + state + (int64_t)row * a.st_row + (int64_t)col * a.st_col;
            if (a.st_col == 1) acc[p] = *reinterpret_cast<const f4v*>(from);
            else
                for (int i = 0; i < 4; ++i) acc[p][i] = from[i * a.st_col];
        }
    }
    const T* pa = static_cast<const T*>(a.a.p) + base_of(a, a.a.seq, a.a.tok, s, span.first) + (int64_t)(h / a.a.group) * a.a.head;
    const T* pb = static_cast<const T*>(a.b.p) + base_of(a, a.b.seq, a.b.tok, s, span.first) + (int64_t)(h / a.b.group) * a.b.head;
    const T* pc = static_cast<const T*>(a.c.p) + base_of(a, a.c.seq, a.c.tok, s, span.first) + (int64_t)(h / a.c.group) * a.c.head;
    OUT* po = static_cast<OUT*>(a.out) + base_of(a, a.out_seq, a.out_tok, s, span.first) + (int64_t)h * a.out_head;
    if (span.count != 0 && a.init_mul != 1.0f)
#pragma unroll
        for (int p = 0; p < kPasses; ++p) acc[p] *= a.init_mul;

    for (uint64_t i = 0; i < span.count; ++i) {
        const int64_t t = a.reverse ? (int64_t)(span.count - 1 - i) : (int64_t)i;
        const Kept now = a.late && i == 0 ? Kept{1.0f, 0.0f} : decay;
        f4v c = {0, 0, 0, 0}, o = {0, 0, 0, 0};
        if (live)
            for (int j = 0; j < 4; ++j) c[j] = (float)pc[t * a.c.tok + col + j];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const uint32_t row = p * kRows + row0;
            if (row < a.dk) {
                const float b = (float)pb[t * a.b.tok + row], q = (float)pa[t * a.a.tok + row];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    acc[p][j] = kept_plus(now, acc[p][j], b * c[j]);
                    o[j] = fmaf(q, acc[p][j], o[j]);
                }
            }
        }
#pragma unroll
        for (int x = LANES; x < 64; x <<= 1)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], x);
        // (two buffers: the next token's sums go to the other one, so one barrier a token is enough)
        float(*buffer)[4 * LANES] = sums[i & 1];
        if ((threadIdx.x & 63) < LANES) *reinterpret_cast<f4v*>(&buffer[wave][lane * 4]) = o;
        __syncthreads();
        if (threadIdx.x < 4 * LANES && slab * 4 * LANES + threadIdx.x < a.dv) {
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) total += buffer[w][threadIdx.x];
            po[t * a.out_tok + slab * 4 * LANES + threadIdx.x] = (OUT)(total * a.out_scale);
        }
    }
    if (a.fin != nullptr && live) {
        const float mul = span.count == 0 ? 1.0f : (a.late ? lambda * a.fin_mul : a.fin_mul);
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            const uint32_t row = p * kRows + row0;
            if (row >= a.dk) continue;
            float* to = a.fin + state + (int64_t)row * a.st_row + (int64_t)col * a.st_col;
            if (a.st_col == 1) *reinterpret_cast<f4v*>(to) = acc[p] * mul;
            else
                for (int i = 0; i < 4; ++i) to[i * a.st_col] = acc[p][i] * mul;
        }
    }
}

// Zeros in the rows of tokens that lie in no sequence.  One workgroup per 64 tokens, and every gridDim.x-th 64 behind them.
template <typename OUT>
__global__ __launch_bounds__(256) void attention_outside_kernel(const Scan a) {
    const uint64_t first = a.offsets[0], last = a.offsets[a.sequences];
    for (uint64_t from = (uint64_t)blockIdx.x * 64; from < a.total; from += (uint64_t)gridDim.x * 64)
        for (uint64_t t = from; t < a.total && t < from + 64; ++t) {
            if (t >= first && t < last) continue;
            OUT* out = static_cast<OUT*>(a.out) + (int64_t)t * a.out_tok;
            for (uint32_t i = threadIdx.x; i < a.heads * a.dv; i += 256) out[(int64_t)(i / a.dv) * a.out_head + i % a.dv] = (OUT)0.0f;
        }
}

// Gradients of shared keys and values: the sum over the heads that share them, in binary32, rounded once.
template <typename T>
__global__ __launch_bounds__(256) void attention_shared_kernel(const float* __restrict__ part, T* __restrict__ out, uint64_t count, uint32_t d,
                                                               uint32_t group) {
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (uint64_t)gridDim.x * 256) {         // (token, shared head, column)
        const float* from = part + i / d * group * d + i % d;
        float sum = 0.0f;
        for (uint32_t g = 0; g < group; ++g) sum += from[(uint64_t)g * d];
        out[i] = (T)sum;
    }
}

}  // namespace layers
}  // namespace tcr
