// Linear attention by chunks of C tokens on the matrix cores.  With i, j the tokens of a chunk and S the state in front of it,
//     out_i  = scale * ( sum_{j <= i} lambda^(i-j) (a_i . b_j) c_j  +  lambda^(i+1) a_i^T S )
//     S_next = lambda^C S + sum_j b_j (lambda^(C-1-j) c_j)^T
// i.e. a product with a triangular matrix inside the chunk and a carry between chunks: the scan of tiles that the library's scans
// are, with a matrix for the running sum.
//
// One workgroup of 4 wavefronts takes a block of consecutive tokens of one head, chunk after chunk, and a slab of 64 * NT columns
// of c; each wavefront holds its 16 * NT columns of S in accumulator registers all along.  The chunk's rows pass through
// LDS once; the next chunk's are loaded into registers meanwhile.  Where sequences and heads are too few to fill the chip, tokens are cut into
// several blocks: a first kernel (STATES) leaves the state that each block alone arrives at, a second adds up what
// reaches each block from the ones in front, and this one starts from there.
//
// Layouts.  v_mfma_f32_16x16x32: lane l = n + 16 g gives A[n][8g .. 8g+7] and B[8g .. 8g+7][n] and receives D[4g .. 4g+3][n].
//   scores    D = b a^T: a lane gets 4 consecutive j of one i, and stores them as a row of P for the others
//   S         D[dk][dv] = b^T c: operands by ds_read_b64_tr_b16, which reads 4 rows and returns columns
//   out       D = S^T a^T + c^T P^T: a lane gets 4 consecutive elements of one token's output.  S goes from accumulator to operand
//             without leaving its lane: the order of the 32 summands of a product is free as long as both operands have the same,
//             so the lane's 4 + 4 rows of two tiles are summands 8g .. 8g+7, and a is read in that order.
//
// Rounding.  The matrix cores take 16-bit operands.  a, b and c are theirs exactly; the derived ones would cost the results half of
// their precision if they were rounded: scores and S as a factor are given as two parts (high + low, 2 products), decayed c, whose sums are the
// binary32 states, as three bfloat16 or two binary16 parts.  binary16 holds neither large nor small values, so scores, S and c are
// brought near 2^14 by powers of two there.
#pragma once
#include "tcr_attention.hpp"

namespace tcr {
namespace layers {

constexpr int kChunkThreads = 256, kChunkWaves = 4;

// How the tokens are cut: spans (sequences, or all packed tokens) into blocks of `length` tokens, counted in the order of the scan.
struct Blocks {
    uint64_t span, length;
    uint32_t per_span, count;
    float* states;              // [heads][slabs][count - 1] of what a workgroup holds: the state behind each block but the last
    float* keep;                // [heads][count - 1]: what is left behind a block of a state in front of it
};

// A chunk: tokens of sequence s at rows low .. low + len - 1 of the views.
struct Chunk {
    uint64_t s;
    int64_t low;
    int len;
    bool begin, last;           // holds the first / last token of its sequence, in the order of the scan
};

struct Walk {
    uint64_t pos, end;          // in the order of the scan
    uint64_t s, lo, hi;         // the sequence at hand and its tokens in that order

    __device__ __forceinline__ bool find(const Scan& a) {
        const uint64_t token = a.reverse ? a.total - 1 - pos : pos;
        uint64_t from, to;
        if (a.offsets == nullptr) {
            s = token / a.tokens;
            from = s * a.tokens;
            to = from + a.tokens;
        } else {
            uint64_t low = 0, high = a.sequences;             // the last sequence that starts at or in front of the token
            while (high - low > 1) {
                const uint64_t mid = (low + high) / 2;
                if (a.offsets[mid] <= token) low = mid;
                else high = mid;
            }
            s = low;
            from = a.offsets[s];
            to = a.offsets[s + 1];
            to = to < a.total ? to : a.total;
            if (from > token || to <= token) return false;
        }
        lo = a.reverse ? a.total - to : from;
        hi = a.reverse ? a.total - from : to;
        return true;
    }
    template <int C>
    __device__ __forceinline__ bool next(const Scan& a, Chunk& c) {
        while (pos < end) {
            if (pos >= hi && !find(a)) {                       // (a token of no sequence)
                ++pos;
                hi = pos;
                continue;
            }
            uint64_t stop = pos + C;
            stop = stop < hi ? stop : hi;
            stop = stop < end ? stop : end;
            c.s = s;
            c.len = (int)(stop - pos);
            c.begin = pos == lo;
            c.last = stop == hi;
            const uint64_t first = a.reverse ? a.total - stop : pos;
            c.low = (int64_t)(a.offsets == nullptr ? first - s * a.tokens : first);
            pos = stop;
            return true;
        }
        return false;
    }
};

__device__ __forceinline__ f4v mfma(half8v a, half8v b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f4v mfma(bf8v a, bf8v b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Rows row .. row + 3 of columns col .. col + 15 of an LDS array, by the 16 lanes of a group: lane n gets column col + n of the four rows.
typedef short s4v __attribute__((ext_vector_type(4)));
template <typename T>
__device__ __forceinline__ s4v columns(const T* base, int stride, int row, int col, int n) {
    typedef __attribute__((address_space(3))) s4v lds_s4v;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(base + (row + (n >> 2)) * stride + col + (n & 3) * 4));
}
template <typename T>
__device__ __forceinline__ typename Bits<T>::v8 joined(s4v a, s4v b) {
    typedef short s8v __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(typename Bits<T>::v8, (s8v)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A value that is split into parts, as a binary32 number: left to itself the compiler may fuse its last multiplication with the rounding of the
// high part and not with the subtraction of that part, and in the rare case that these round apart the parts miss it by half a spacing.
__device__ __forceinline__ float settled(float x) {
    asm("" : "+v"(x));
    return x;
}
__device__ __forceinline__ float wave_largest(float x) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x = fmaxf(x, __shfl_xor(x, m));
    return x;
}
// The power of two that brings `largest` to [2^14, 2^15): what is split into binary16 parts then keeps 22 bits.
__device__ __forceinline__ float near_top(float largest) {
    const int e = (int)(__builtin_bit_cast(uint32_t, largest) >> 23);         // (not negative; 0 and subnormals: e = 0)
    int f = 127 + 14 + 127 - e;
    f = f > 187 ? 187 : (f < 67 ? 67 : f);                                    // 2^-60 .. 2^60: a product of two of them is one too
    return __builtin_bit_cast(float, (uint32_t)f << 23);
}
__device__ __forceinline__ float reciprocal_power(float f) { return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, f)); }

template <typename T, int DK, int NT, int C>
struct ChunkLds {
    // (rows 16 bytes beyond a multiple of 256: reads of 8 or 16 bytes from 16 rows meet no bank twice; 32 bytes: reads of columns)
    static constexpr int kStrideA = DK + 8, kStrideB = DK + 16, kStrideC = 64 * NT + 16, kStrideP = C + 16;
    alignas(16) T b[C * kStrideB];
    alignas(16) T c[C * kStrideC];
    float powers[C + 1];                     // lambda^0 .. lambda^C
};
template <typename T, int DK, int NT, int C>
struct ChunkLdsOut : ChunkLds<T, DK, NT, C> {
    alignas(16) T a[C * ChunkLds<T, DK, NT, C>::kStrideA];
    alignas(16) T p[2][C * ChunkLds<T, DK, NT, C>::kStrideP];
    float p_factor[C / 16];
};

template <typename T, typename OUT, int DK, int NT, int C, bool STATES>
__global__ __launch_bounds__(kChunkThreads, 2) void attention_chunk_kernel(const Scan a, const Blocks blocks) {
    typedef typename Bits<T>::v8 v8;
    constexpr bool kHalf = std::is_same<T, _Float16>::value;
    constexpr int CT = C / 16, KT = DK / 16, kParts = kHalf ? 2 : 3, kSlab = 64 * NT;
    typedef typename std::conditional<STATES, ChunkLds<T, DK, NT, C>, ChunkLdsOut<T, DK, NT, C>>::type Lds;
    constexpr int SA = Lds::kStrideA, SB = Lds::kStrideB, SC = Lds::kStrideC, SP = Lds::kStrideP;
    __shared__ __align__(16) Lds lds;

    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const uint32_t slabs = (a.dv + kSlab - 1) / kSlab;
    const uint32_t slab = blockIdx.x % slabs, h = blockIdx.x / slabs % a.heads, block = blockIdx.x / slabs / a.heads;
    const float log_decay = decay_of(a, h);
    constexpr int kHeld = KT * NT * 4;                              // floats of S a lane holds
    const int64_t state_size = (int64_t)kChunkThreads * kHeld;

    // the block's tokens, in the order of the scan
    Walk walk;
    walk.pos = block / blocks.per_span * blocks.span + block % blocks.per_span * blocks.length;
    {
        const uint64_t span_end = (block / blocks.per_span + 1) * blocks.span;
        walk.end = walk.pos + blocks.length;
        walk.end = walk.end < span_end ? walk.end : span_end;
        walk.s = walk.lo = walk.hi = 0;
    }
    const uint64_t block_start = walk.pos;
    if constexpr (STATES) {
        // only the sequence that goes on behind the block counts
        walk.pos = walk.end - 1;
        const bool some = walk.find(a);
        const uint64_t from = some && walk.lo > block_start ? walk.lo : block_start;
        if (slab == 0 && threadIdx.x == 0)
            blocks.keep[(uint64_t)h * (blocks.count - 1) + block] =
                some && walk.lo < block_start ? decayed(log_decay, (float)(walk.end - block_start)) : 0.0f;
        walk.pos = some ? from : walk.end;
    }

    for (int i = threadIdx.x; i <= C; i += kChunkThreads) lds.powers[i] = decayed(log_decay, (float)i);

    // Rows of the next chunk on their way, 16 bytes a lane.  Rows and columns beyond the ends read as 0 (an offset outside the buffer).
    constexpr int kVecs = DK / 8, kCVecs = kSlab / 8, kPassRows = kChunkThreads / kVecs, kPassRowsC = kChunkThreads / kCVecs;
    constexpr int kPasses = C / kPassRows, kPassesC = C / kPassRowsC;
    u4v ra[kPasses], rb[kPasses], rc[kPassesC];
    const int row = threadIdx.x / kVecs, col = threadIdx.x % kVecs * 8, row_c = threadIdx.x / kCVecs, col_c = threadIdx.x % kCVecs * 8;
    auto fetch = [&](const View& v, const Chunk& c, int r0, uint32_t column, bool inside, int step, u4v* to, auto passes) {
        const T* base = static_cast<const T*>(v.p) + (int64_t)(a.offsets == nullptr ? c.s : 0) * v.seq + c.low * v.tok + (int64_t)(h / v.group) * v.head;
        __amdgpu_buffer_rsrc_t buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, 0x7fffffff, 0x00020000);
        const uint32_t pitch = (uint32_t)v.tok * sizeof(T);
#pragma unroll
        for (int p = 0; p < decltype(passes)::value; ++p) {
            const int r = r0 + p * step;
            const uint32_t at = (uint32_t)(a.reverse ? c.len - 1 - r : r) * pitch + column * (uint32_t)sizeof(T);
            to[p] = __builtin_amdgcn_raw_buffer_load_b128(buffer, inside && r < c.len ? at : 0xfffffff0u, 0, 0);
        }
    };
    auto fetch_all = [&](const Chunk& c) {
        if constexpr (!STATES) fetch(a.a, c, row, col, (uint32_t)col < a.dk, kPassRows, ra, std::integral_constant<int, kPasses>());
        fetch(a.b, c, row, col, (uint32_t)col < a.dk, kPassRows, rb, std::integral_constant<int, kPasses>());
        fetch(a.c, c, row_c, slab * kSlab + col_c, slab * kSlab + col_c < a.dv, kPassRowsC, rc, std::integral_constant<int, kPassesC>());
    };

    f4v S[KT][NT];
    const uint32_t dv0 = slab * kSlab + w * 16 * NT + n;             // this lane's columns of S: dv0 + 16 nt; rows: 16 mt + 4 g + r
    auto from_states = [&](const float* from) {
#pragma unroll
        for (int mt = 0; mt < KT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[mt][nt] = *reinterpret_cast<const f4v*>(from + ((w * KT + mt) * NT + nt) * 256 + lane * 4);
    };
    auto clear = [&] {
#pragma unroll
        for (int mt = 0; mt < KT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[mt][nt] = f4v{0, 0, 0, 0};
    };
    float* const own_states = blocks.states + ((int64_t)(h * slabs + slab) * (blocks.count - 1) + block) * state_size;
    clear();
    if (!STATES && block % blocks.per_span != 0) from_states(own_states - state_size);       // (0 where a sequence starts with the block)

    // the diagonal's decays of the scores this wavefront computes: lambda^(n - 4g - r), 0 above the diagonal
    __syncthreads();
    float diagonal[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) diagonal[r] = n >= 4 * g + r ? lds.powers[n - 4 * g - r < 0 ? 0 : n - 4 * g - r] : 0.0f;

    Chunk now, ahead;
    bool more = walk.next<C>(a, now);
    if (more) fetch_all(now);
    while (more) {
        // ---- the chunk's rows into LDS (all reads of the last chunk's are done)
        if constexpr (!STATES)
#pragma unroll
            for (int p = 0; p < kPasses; ++p) *reinterpret_cast<u4v*>(&lds.a[(row + p * kPassRows) * SA + col]) = ra[p];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) *reinterpret_cast<u4v*>(&lds.b[(row + p * kPassRows) * SB + col]) = rb[p];
#pragma unroll
        for (int p = 0; p < kPassesC; ++p) *reinterpret_cast<u4v*>(&lds.c[(row_c + p * kPassRowsC) * SC + col_c]) = rc[p];
        __syncthreads();
        more = walk.next<C>(a, ahead);
        if (more) fetch_all(ahead);

        if (now.begin) {
            if (a.init != nullptr) {
                const float* from = a.init + ((int64_t)now.s * a.heads + h) * a.dk * a.dv;
#pragma unroll
                for (int mt = 0; mt < KT; ++mt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const uint32_t k = mt * 16 + 4 * g + r, v = dv0 + 16 * nt;
                            S[mt][nt][r] = k < a.dk && v < a.dv ? from[(int64_t)k * a.st_row + (int64_t)v * a.st_col] * a.init_mul : 0.0f;
                        }
            } else {
                clear();
            }
        }
        const int late = a.late && now.begin ? 1 : 0;

        f4v o[CT][NT];
        if constexpr (!STATES) {
            // ---- scores: tile row `it` by wavefront it
            for (int it = w; it < CT; it += kChunkWaves) {
                f4v s[CT];
#pragma unroll
                for (int jt = 0; jt < CT; ++jt) s[jt] = f4v{0, 0, 0, 0};
#pragma unroll
                for (int ks = 0; ks < DK / 32; ++ks) {
                    const v8 rows = *reinterpret_cast<const v8*>(&lds.a[(it * 16 + n) * SA + ks * 32 + 8 * g]);
#pragma unroll
                    for (int jt = 0; jt < CT; ++jt)
                        if (jt <= it) s[jt] = mfma(*reinterpret_cast<const v8*>(&lds.b[(jt * 16 + n) * SB + ks * 32 + 8 * g]), rows, s[jt]);
                }
                float largest = 0.0f;
#pragma unroll
                for (int jt = 0; jt < CT; ++jt) {
                    if (jt > it) continue;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        // (a score above the diagonal is dropped, whatever it is)
                        const float d = jt == it ? diagonal[r] : lds.powers[(it - jt) * 16 + n - 4 * g - r];
                        s[jt][r] = jt == it && n < 4 * g + r ? 0.0f : s[jt][r] * d;
                        if constexpr (kHalf) largest = fmaxf(largest, fabsf(s[jt][r]));
                    }
                }
                float factor = 1.0f;
                if constexpr (kHalf) {
                    factor = near_top(wave_largest(largest));
                    if (lane == 0) lds.p_factor[it] = factor;
                }
#pragma unroll
                for (int jt = 0; jt < CT; ++jt) {
                    if (jt > (it | 1)) continue;
                    T hi[4], lo[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = kHalf ? settled(s[jt][r] * factor) : s[jt][r];
                        hi[r] = (T)x;
                        lo[r] = (T)(x - (float)hi[r]);
                    }
                    typedef T v4 __attribute__((ext_vector_type(4)));
                    *reinterpret_cast<v4*>(&lds.p[0][(it * 16 + n) * SP + jt * 16 + 4 * g]) = v4{hi[0], hi[1], hi[2], hi[3]};
                    *reinterpret_cast<v4*>(&lds.p[1][(it * 16 + n) * SP + jt * 16 + 4 * g]) = v4{lo[0], lo[1], lo[2], lo[3]};
                }
            }
            // ---- what the state in front of the chunk gives
            float factor = 1.0f;
            if constexpr (kHalf) {
                float largest = 0.0f;
#pragma unroll
                for (int mt = 0; mt < KT; ++mt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) largest = fmaxf(largest, fabsf(S[mt][nt][r]));
                factor = near_top(wave_largest(largest));
            }
#pragma unroll
            for (int it = 0; it < CT; ++it)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) o[it][nt] = f4v{0, 0, 0, 0};
#pragma unroll
            for (int ks = 0; ks < DK / 32; ++ks) {
                v8 hi[NT], lo[NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const float x = kHalf ? settled(S[2 * ks + (r >> 2)][nt][r & 3] * factor) : S[2 * ks + (r >> 2)][nt][r & 3];
                        hi[nt][r] = (T)x;
                        lo[nt][r] = (T)(x - (float)hi[nt][r]);
                    }
#pragma unroll
                for (int it = 0; it < CT; ++it) {
                    const T* from = &lds.a[(it * 16 + n) * SA + ks * 32 + 4 * g];
                    const v8 rows = joined<T>(*reinterpret_cast<const s4v*>(from), *reinterpret_cast<const s4v*>(from + 16));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        o[it][nt] = mfma(hi[nt], rows, o[it][nt]);
                        o[it][nt] = mfma(lo[nt], rows, o[it][nt]);
                    }
                }
            }
            __syncthreads();                                                       // the scores are there
#pragma unroll
            for (int it = 0; it < CT; ++it) {
                float f = lds.powers[it * 16 + n + 1 - late];
                if constexpr (kHalf) f *= reciprocal_power(factor) * lds.p_factor[it];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) o[it][nt] *= f;
            }
        }

        // ---- c by columns: for out as it is, for S decayed to the chunk's end
        float largest_c = 0.0f;
        v8 cols[C / 32][NT];
#pragma unroll
        for (int ks = 0; ks < C / 32; ++ks)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int at = (w * NT + nt) * 16;
                cols[ks][nt] = joined<T>(columns(lds.c, SC, ks * 32 + 8 * g, at, n), columns(lds.c, SC, ks * 32 + 8 * g + 4, at, n));
                if constexpr (kHalf)
#pragma unroll
                    for (int r = 0; r < 8; ++r) largest_c = fmaxf(largest_c, fabsf((float)cols[ks][nt][r]));
            }
        if constexpr (!STATES) {
#pragma unroll
            for (int ks = 0; ks < C / 32; ++ks)
#pragma unroll
                for (int it = 2 * ks; it < CT; ++it)
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        const v8 scores = *reinterpret_cast<const v8*>(&lds.p[part][(it * 16 + n) * SP + ks * 32 + 8 * g]);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) o[it][nt] = mfma(cols[ks][nt], scores, o[it][nt]);
                    }
            OUT* out = static_cast<OUT*>(a.out) + (int64_t)(a.offsets == nullptr ? now.s : 0) * a.out_seq + now.low * a.out_tok + (int64_t)h * a.out_head;
#pragma unroll
            for (int it = 0; it < CT; ++it) {
                const int i = it * 16 + n;
                if (i >= now.len) continue;
                const float f = a.out_scale * (kHalf ? reciprocal_power(lds.p_factor[it]) : 1.0f);
                OUT* to = out + (int64_t)(a.reverse ? now.len - 1 - i : i) * a.out_tok;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint32_t v = slab * kSlab + (w * NT + nt) * 16 + 4 * g;
                    if (v >= a.dv) continue;
                    typedef OUT o4 __attribute__((ext_vector_type(4), aligned(sizeof(OUT))));
                    const f4v x = o[it][nt] * f;
                    *reinterpret_cast<o4*>(to + v) = o4{(OUT)x[0], (OUT)x[1], (OUT)x[2], (OUT)x[3]};
                }
            }
        }

        // ---- the state behind the chunk
        float factor_c = 1.0f;
        if constexpr (kHalf) {
            largest_c = wave_largest(largest_c);
            // (values that two parts hold to 22 bits as they are stay as they are)
            if (!(largest_c >= 0.125f && largest_c < 32768.0f)) factor_c = near_top(largest_c);
        }
        {
            const float f = lds.powers[now.len - late] * factor_c;
#pragma unroll
            for (int mt = 0; mt < KT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) S[mt][nt] *= f;
        }
#pragma unroll
        for (int ks = 0; ks < C / 32; ++ks) {
            v8 part[kParts][NT];
            float decays[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const int steps = now.len - 1 - (ks * 32 + 8 * g + r);
                decays[r] = lds.powers[steps < 0 ? 0 : steps] * factor_c;
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    float x = settled((float)cols[ks][nt][r] * decays[r]);
#pragma unroll
                    for (int p = 0; p < kParts; ++p) {
                        part[p][nt][r] = (T)x;
                        x -= (float)part[p][nt][r];
                    }
                }
#pragma unroll
            for (int mt = 0; mt < KT; ++mt) {
                const v8 rows = joined<T>(columns(lds.b, SB, ks * 32 + 8 * g, mt * 16, n), columns(lds.b, SB, ks * 32 + 8 * g + 4, mt * 16, n));
#pragma unroll
                for (int p = kParts - 1; p >= 0; --p)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) S[mt][nt] = mfma(rows, part[p][nt], S[mt][nt]);
            }
        }
        if (kHalf && factor_c != 1.0f) {
            const float f = reciprocal_power(factor_c);
#pragma unroll
            for (int mt = 0; mt < KT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) S[mt][nt] *= f;
        }
        if (!STATES && now.last && a.fin != nullptr) {
            float* to = a.fin + ((int64_t)now.s * a.heads + h) * a.dk * a.dv;
            const float mul = a.late ? lds.powers[1] * a.fin_mul : a.fin_mul;
#pragma unroll
            for (int mt = 0; mt < KT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t k = mt * 16 + 4 * g + r, v = dv0 + 16 * nt;
                        if (k < a.dk && v < a.dv) to[(int64_t)k * a.st_row + (int64_t)v * a.st_col] = S[mt][nt][r] * mul;
                    }
        }
        __syncthreads();                                                           // all reads of this chunk's rows are done
        now = ahead;
    }
    if constexpr (STATES) {
#pragma unroll
        for (int mt = 0; mt < KT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f4v*>(own_states + ((w * KT + mt) * NT + nt) * 256 + lane * 4) = S[mt][nt];
    }
}

// What reaches each block from the ones in front of it: running sums over the blocks, in place.
__global__ __launch_bounds__(256) void attention_carry_kernel(const Blocks blocks, uint32_t slabs, uint64_t state_size) {
    const uint64_t at = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 4, group = at / state_size;      // (head, slab); state_size: a multiple of 1024
    f4v* states = reinterpret_cast<f4v*>(blocks.states + group * (blocks.count - 1) * state_size + at % state_size);
    const float* keep = blocks.keep + group / slabs * (blocks.count - 1);
    f4v carry = {0, 0, 0, 0};
#pragma unroll 4
    for (uint32_t n = 0; n + 1 < blocks.count; ++n) {
        carry = states[n * (state_size / 4)] + carry * keep[n];
        states[n * (state_size / 4)] = carry;
    }
}

// Final states of sequences without tokens: the first ones.
__global__ __launch_bounds__(256) void attention_empty_kernel(const Scan a) {
    const uint64_t s = blockIdx.x / a.heads;
    if (span_of(a, s).count != 0) return;
    const uint64_t size = (uint64_t)a.dk * a.dv, from = (uint64_t)blockIdx.x * size;
    for (uint64_t i = threadIdx.x; i < size; i += 256) a.fin[from + i] = a.init != nullptr ? a.init[from + i] : 0.0f;
}

}  // namespace layers
}  // namespace tcr
