// Linear attention by chunks of C tokens on the matrix cores.  With i, j the tokens of a chunk and S the state in front of it,
//     out_i  = scale * ( sum_{j <= i} lambda^(i-j) (a_i . b_j) c_j  +  lambda^(i+1) a_i^T S )
//     S_next = lambda^C S + sum_j b_j (lambda^(C-1-j) c_j)^T
// i.e. a product with a triangular matrix inside the chunk and a carry between chunks: the scan of tiles that the library's scans
// are, with a matrix for the running sum.
//
// One workgroup of W wavefronts takes a block of consecutive tokens of one head, chunk after chunk, and a slab of 16 * W * NT columns
// of c; each wavefront holds its 16 * NT columns of S in accumulator registers all along.  The chunk's rows pass through
// LDS once; the next chunk's are loaded into registers meanwhile.  Where sequences and heads are too few to fill the chip, tokens are cut into
// several blocks: a first kernel (STATES) leaves the state that each block alone arrives at, a second adds up what
// reaches each block from the ones in front, and this one starts from there.
//
// MI355X, 32768 tokens, 16 heads of 128 x 128, bfloat16, 227 us: states 68, carries 16, this 143, 929 MB and 155 GFLOP (all parts) in all, which a copy and a large product would take
// 175 and 118 us for.  Two workgroups on a compute unit take 10 200 cycles for a chunk each: vector ALUs are busy for 46 %, LDS for 43 % (12 % in bank conflicts, see ChunkLds),
// matrix cores for 30 % of the time, in turn between barriers.
// Eight wavefronts of 16 columns on 128 registers beat four of 32 columns on 256 by 5 to 8 % although each of them reads all of a and b from LDS.
//
// Layouts.  v_mfma_f32_16x16x32: lane l = n + 16 g gives A[n][8g .. 8g+7] and B[8g .. 8g+7][n] and receives D[4g .. 4g+3][n].
//   scores    D = b a^T: a lane gets 4 consecutive j of one i, and stores them as a row of P for the others
//   S         D[dk][dv] = b^T c: operands by ds_read_b64_tr_b16, which reads 4 rows and returns columns
//   out       D = S^T a^T + c^T P^T: a lane gets 4 consecutive elements of one token's output.  S goes from accumulator to operand
//             without leaving its lane: the order of the 32 summands of a product is free as long as both operands have the same,
//             so the lane's 4 + 4 rows of two tiles are summands 8g .. 8g+7, and a is read in that order.  The tokens of b, c and P stand in
//             the same order (4g .. 4g+3 and 16 + 4g .. 16 + 4g+3 of 32): reads of columns then meet no bank twice.
//
// Rounding.  The matrix cores take 16-bit operands.  a, b and c are theirs exactly; the derived ones would cost the results half of
// their precision if they were rounded: scores and S as a factor are given as two parts (high + low, 2 products, off by 2^-17 of themselves in bfloat16 and
// 2^-20 in binary16 at most, for outputs that are rounded by up to 2^-8 and 2^-11), decayed c, whose sums are the binary32 states, as three bfloat16 or two binary16 parts (2^-21 at most).
// The gradients' states too, so that a gradient is the same whether the states' own is asked for or not (two bfloat16 parts for them: gradients of 4 x 2048 tokens, 16 heads of 128 x 128, 170 us instead of 181, 192 on another machine).
// binary16 holds neither large nor small values, so scores, S and c are brought near 2^14 by powers of two there.
#pragma once
#include "tcr_attention.hpp"

namespace tcr {
namespace layers {

// How the tokens are cut: spans (sequences, or all packed tokens) into blocks of `length` tokens, counted in the order of the scan.
struct Blocks {
    uint32_t span, length, per_span, count;
    float* states;              // [heads][slabs][count - 1] of what a workgroup holds: the state behind each block but the last
    Kept* keep;                 // [heads][count - 1]: what is left behind a block of a state in front of it (0: nothing reaches the next block)
    uint32_t turned;            // the states are transposed: those of a scan with b and c exchanged, cut alike
    uint32_t direct;            // a block adds up the states of the ones in front of it itself; otherwise they hold what reaches the next block
};

// A chunk: tokens of sequence s at rows low .. low + len - 1 of the views.
struct Chunk {
    uint32_t s, low;
    int len;
    bool begin, last;           // holds the first / last token of its sequence, in the order of the scan
};

// (What is the same for a whole wavefront is kept in scalar registers, which the compiler has to be told of loaded values.)
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ float uniform(float x) { return __builtin_bit_cast(float, uniform(__builtin_bit_cast(uint32_t, x))); }
template <typename P>
__device__ __forceinline__ P* uniform(P* p) {
    const uint64_t x = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<P*>((uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x));
}

// The chunks of a block, one after the other.
struct Walk {
    const uint64_t* offsets;
    uint32_t sequences, tokens, total, reverse;
    uint32_t pos, end;          // in the order of the scan
    uint32_t s, lo, hi;         // the sequence at hand and its tokens in that order

    __device__ __forceinline__ uint32_t cut(uint32_t i) const {
        const uint64_t o = offsets[i];
        return uniform(o < total ? (uint32_t)o : total);
    }
    // The sequence of the token at pos; false: it lies in none.
    __device__ __forceinline__ bool find() {
        const uint32_t token = reverse ? total - 1 - pos : pos;
        uint32_t from, to;
        if (offsets == nullptr) {
            s = token / tokens;
            from = s * tokens;
            to = from + tokens;
        } else {
            uint32_t low = 0, high = sequences;               // the last sequence that starts at or in front of the token
            while (high - low > 1) {
                const uint32_t mid = (low + high) / 2;
                if (cut(mid) <= token) low = mid;
                else high = mid;
            }
            s = low;
            from = cut(s);
            to = cut(s + 1);
            if (from > token || to <= token) return false;
        }
        lo = reverse ? total - to : from;
        hi = reverse ? total - from : to;
        return true;
    }
    // Where to go on from a token of no sequence: in front of all of them, behind them (offsets that decrease leave others: one by one).
    __device__ __forceinline__ uint32_t beyond() const {
        const uint32_t token = reverse ? total - 1 - pos : pos, first = cut(0), last = cut(sequences);
        if (token < first) return reverse || first >= end ? end : first;
        if (token >= last) return !reverse || total - last >= end ? end : total - last;
        return pos + 1;
    }
    template <int C>
    __device__ __forceinline__ bool next(Chunk& c) {
        while (pos < end) {
            if (pos >= hi && !find()) {
                pos = hi = beyond();
                continue;
            }
            uint32_t stop = end - pos < C ? end : pos + C;
            stop = stop < hi ? stop : hi;
            c.s = s;
            c.len = (int)(stop - pos);
            c.begin = pos == lo;
            c.last = stop == hi;
            c.low = (reverse ? total - stop : pos) - (offsets == nullptr ? s * tokens : 0);
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
// Two numbers as PARTS pairs of 16-bit ones whose sums they are.  binary16: every part but the last is cut off, not rounded (one instruction for
// the pair; what is cut off is the next part's), the last one rounded if `fine`.
template <typename T, int PARTS>
__device__ __forceinline__ void split(float a, float b, uint32_t (&parts)[PARTS], bool fine) {
    if constexpr (std::is_same<T, _Float16>::value) {
        a = settled(a);
        b = settled(b);
    }
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        if constexpr (std::is_same<T, _Float16>::value) {
            typedef __fp16 cut2 __attribute__((ext_vector_type(2)));
            typedef _Float16 pair __attribute__((ext_vector_type(2)));
            if (p + 1 < PARTS || !fine) {
                const pair h = __builtin_bit_cast(pair, (cut2)__builtin_amdgcn_cvt_pkrtz(a, b));
                parts[p] = __builtin_bit_cast(uint32_t, h);
                a -= (float)h[0];
                b -= (float)h[1];
            } else {
                parts[p] = __builtin_bit_cast(uint32_t, pair{(_Float16)a, (_Float16)b});
            }
        } else {
            typedef __bf16 pair __attribute__((ext_vector_type(2)));
            typedef float wide __attribute__((ext_vector_type(2)));
            parts[p] = __builtin_bit_cast(uint32_t, __builtin_convertvector(wide{a, b}, pair));
            a -= __builtin_bit_cast(float, parts[p] << 16);
            b -= __builtin_bit_cast(float, parts[p] & 0xffff0000u);
        }
    }
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

template <typename T, int DK, int COLS, int C>
struct ChunkLds {
    // (rows 16 bytes beyond a multiple of 128: reads of 8 or 16 bytes from 16 rows meet no bank twice; 32 bytes: reads of columns do not, those of rows meet the banks of rows n
    // and n + 8 twice -- of b and of the scores, a quarter of all LDS cycles)
    static constexpr int kStrideA = DK + 8, kStrideB = DK + 16, kStrideC = COLS + 16, kStrideP = C + 16;
    alignas(16) T b[C * kStrideB];
    alignas(16) T c[C * kStrideC];
    float beyond[C];                         // (what a look-up of steps behind a short chunk's end meets, for rows of zeros)
    float powers[C + 1];                     // lambda^0 .. lambda^C
    float missed[C + 1];                     // what their rounding left out, where lambda^C is near 1
};
template <typename T, int DK, int COLS, int C>
struct ChunkLdsOut : ChunkLds<T, DK, COLS, C> {
    alignas(16) T a[C * ChunkLds<T, DK, COLS, C>::kStrideA];
    alignas(16) T p[2][C * ChunkLds<T, DK, COLS, C>::kStrideP];
    float p_factor[C / 16][C / 32];          // of the scores of 16 rows and 32 columns
};

// What is loaded in front of this is asked for in front of it.  (Left to itself the compiler asks for each operand right where it is used, and waits for
// every one: a chunk took twice as long.)
__device__ __forceinline__ void loads_first() { __builtin_amdgcn_sched_barrier(0); }

// A range of memory of whose 2^31 bytes what lies outside reads as 0 and is not written: kOutside does, also with a scalar offset added.
constexpr uint32_t kOutside = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(uniform(p)), 0, 0x7fffffff, 0x00020000);
}

template <typename T, typename OUT, int DK, int W, int NT, int C, bool STATES>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(W / 2, W / 2))) void attention_chunk_kernel(const Scan a, const Blocks blocks) {
    typedef typename Bits<T>::v8 v8;
    constexpr bool kHalf = std::is_same<T, _Float16>::value;
    constexpr int CT = C / 16, KT = DK / 16, kParts = kHalf ? 2 : 3, kSlab = 16 * W * NT, KS = C / 32;
    constexpr int kChunkThreads = 64 * W;
    typedef typename std::conditional<STATES, ChunkLds<T, DK, kSlab, C>, ChunkLdsOut<T, DK, kSlab, C>>::type Lds;
    constexpr int SA = Lds::kStrideA, SB = Lds::kStrideB, SC = Lds::kStrideC, SP = Lds::kStrideP;
    __shared__ __align__(16) Lds lds;

    const int w = (int)uniform(threadIdx.x >> 6);
    int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const uint32_t slabs = (a.dv + kSlab - 1) / kSlab;
    const uint32_t group = workgroup(), slab = group % slabs, h = group / slabs % a.heads, block = group / slabs / a.heads;      // (fewer than 2^29 in all)
    const float log_decay = decay_of(a, h);
    constexpr int kHeld = KT * NT * 4;                              // floats of S a lane holds
    constexpr uint32_t kStateSize = kChunkThreads * kHeld;
    // a head's rows, and its states
    const T* const pa = static_cast<const T*>(a.a.p) + (int64_t)(h / a.a.group) * a.a.head;
    const T* const pb = static_cast<const T*>(a.b.p) + (int64_t)(h / a.b.group) * a.b.head;
    const T* const pc = static_cast<const T*>(a.c.p) + (int64_t)(h / a.c.group) * a.c.head + slab * kSlab;
    OUT* const po = static_cast<OUT*>(a.out) + (int64_t)h * a.out_head + slab * kSlab;
    const uint32_t state_floats = a.dk * a.dv, left = a.dv - slab * kSlab;        // (columns of c from this slab's first on)

    // the block's tokens, in the order of the scan
    Walk walk;
    walk.offsets = a.offsets;
    walk.sequences = (uint32_t)a.sequences;
    walk.tokens = (uint32_t)a.tokens;
    walk.total = (uint32_t)a.total;
    walk.reverse = a.reverse;
    const uint32_t span_first = block / blocks.per_span * blocks.span, in_span = block % blocks.per_span * blocks.length;
    const uint32_t block_start = span_first + in_span;
    walk.pos = block_start;
    walk.end = blocks.span - in_span < blocks.length ? span_first + blocks.span : block_start + blocks.length;
    // (a workgroup that nothing is left for, which only whole sequences' grids have, finds no token; an exit up there would part the loads of the arguments: 0.4 us a launch)
    if (block >= blocks.count) walk.end = block_start;
    walk.s = walk.lo = walk.hi = 0;
    if constexpr (STATES) {
        // only the sequence that goes on behind the block counts
        walk.pos = walk.end - 1;
        const bool some = walk.find();
        const uint32_t from = some && walk.lo > block_start ? walk.lo : block_start;
        if (slab == 0 && threadIdx.x == 0)
            blocks.keep[(uint64_t)h * (blocks.count - 1) + block] =
                some && walk.lo < block_start ? kept(log_decay, (float)(walk.end - block_start)) : Kept{0.0f, 0.0f};
        walk.pos = some ? from : walk.end;
    }

    const float* const powers = lds.beyond + C;                     // powers[-C .. C]

    // Rows of the next chunk on their way, 16 bytes a lane.  Rows and columns beyond the ends read as 0 (an offset outside the buffer).  A lane's
    // rows are `step` apart, so one offset serves all of its loads; backwards they count down from the last of C rows.
    constexpr int kVecs = DK / 8, kCVecs = kSlab / 8, kPassRows = kChunkThreads / kVecs, kPassRowsC = kChunkThreads / kCVecs;
    constexpr int kPasses = C / kPassRows, kPassesC = C / kPassRowsC;
    u4v ra[kPasses], rb[kPasses], rc[kPassesC];
    uint32_t row = threadIdx.x / kVecs, col = threadIdx.x % kVecs * 8, row_c = threadIdx.x / kCVecs, col_c = threadIdx.x % kCVecs * 8;
    const uint32_t tok_a = (uint32_t)a.a.tok, tok_b = (uint32_t)a.b.tok, tok_c = (uint32_t)a.c.tok, tok_o = (uint32_t)a.out_tok;
    const bool reverse = a.reverse != 0;
    auto fetch = [&](const T* head, int64_t seq, uint32_t tok, const Chunk& c, uint32_t r0, uint32_t column, bool inside, auto step, u4v* to, auto passes) {
        constexpr int kStep = decltype(step)::value, kCount = decltype(passes)::value;
        const int64_t first = (int64_t)c.low + (reverse ? c.len - C : 0);                    // (maybe in front of the array; no such row is read)
        const __amdgpu_buffer_rsrc_t buffer = buffer_at(head + ((int64_t)c.s * seq + first * (int64_t)tok));
        const uint32_t at = (__umul24(reverse ? C - 1 - (kCount - 1) * kStep - r0 : r0, tok) + column) * (uint32_t)sizeof(T);
        const uint32_t pitch = kStep * tok * (uint32_t)sizeof(T), rows = inside ? (uint32_t)c.len : 0u;
#pragma unroll
        for (int p = 0; p < kCount; ++p)
            to[p] = __builtin_amdgcn_raw_buffer_load_b128(buffer, r0 + p * kStep < rows ? at : kOutside, (reverse ? kCount - 1 - p : p) * pitch, 0);
    };
    auto fetch_all = [&](const Chunk& c) {
        const std::integral_constant<int, kPassRows> step;
        const std::integral_constant<int, kPasses> passes;
        if constexpr (!STATES) fetch(pa, a.a.seq, tok_a, c, row, col, col < a.dk, step, ra, passes);
        fetch(pb, a.b.seq, tok_b, c, row, col, col < a.dk, step, rb, passes);
        fetch(pc, a.c.seq, tok_c, c, row_c, col_c, col_c < left, std::integral_constant<int, kPassRowsC>(), rc, std::integral_constant<int, kPassesC>());
    };

    // S: rows 16 mt + 4 g + r, columns 16 (NT w + nt) + n of the slab
    f4v S[KT][NT];
    auto clear = [&] {
#pragma unroll
        for (int mt = 0; mt < KT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[mt][nt] = f4v{0, 0, 0, 0};
    };
    // element of S = f(element, byte offset in a state) for all of them
    auto each = [&](auto f) {
        uint32_t k0 = 4 * g, v0 = w * 16 * NT + n;
        const uint32_t st_row = (uint32_t)a.st_row, st_col = (uint32_t)a.st_col;
#pragma unroll
        for (int mt = 0; mt < KT; ++mt) {
            __builtin_amdgcn_sched_barrier(0);                      // (few offsets at a time)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t k = k0 + mt * 16 + r, v = v0 + 16 * nt;
                    S[mt][nt][r] = f(S[mt][nt][r], k < a.dk && v < left ? (k * st_row + (v + slab * kSlab) * st_col) * 4 : kOutside);
                }
        }
    };
    float* const own_states = blocks.states + ((int64_t)(h * slabs + slab) * (blocks.count - 1) + block) * kStateSize;
    clear();
    if (!STATES && block % blocks.per_span != 0) {                  // (not looked at where a sequence starts with the block)
        const uint32_t in_front = block / blocks.per_span * blocks.per_span, head_states = (blocks.count - 1) * slabs;
        for (uint32_t m = blocks.direct ? in_front : block - 1; m < block; ++m) {
            const Kept keep = m == in_front || !blocks.direct ? Kept{0.0f, 0.0f} : blocks.keep[(uint64_t)h * (blocks.count - 1) + m];
            const float* const from = blocks.states + ((int64_t)h * head_states + m) * kStateSize;
            f4v x[KT][NT];
#pragma unroll
            for (int mt = 0; mt < KT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    x[mt][nt] = f4v{0, 0, 0, 0};
                    if (!blocks.turned) {
                        x[mt][nt] = *reinterpret_cast<const f4v*>(from + (int64_t)slab * (blocks.count - 1) * kStateSize + ((w * KT + mt) * NT + nt) * 256 + lane * 4);
                    } else {
                        // (row k, column v of this S is row v, column k there)
                        const uint32_t v = slab * kSlab + (w * NT + nt) * 16 + n;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const uint32_t k = mt * 16 + 4 * g + r;
                            const float* there = from + (int64_t)(k / kSlab) * (blocks.count - 1) * kStateSize +
                                                 ((k % kSlab / (16 * NT) * KT + v / 16) * NT + k / 16 % NT) * 256 + (v % 16 / 4 * 16 + k % 16) * 4 + v % 4;
                            if (k < a.dk) x[mt][nt][r] = *there;
                        }
                    }
                }
            loads_first();                                          // (the state does not wait for what is kept of the ones in front)
            if (nothing(keep)) clear();                             // (NaN ends with its sequence)
#pragma unroll
            for (int mt = 0; mt < KT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[mt][nt][r] = kept_plus(keep, S[mt][nt][r], x[mt][nt][r]);
        }
    }

    if (!STATES && a.offsets != nullptr) {
        // zeros in the rows of the block's tokens that lie in no sequence
        const uint32_t from = a.reverse ? walk.total - walk.end : block_start, to = a.reverse ? walk.total - block_start : walk.end;
        const uint32_t first = walk.cut(0), last = walk.cut(walk.sequences);
        auto zeros = [&](uint32_t t, uint32_t end) {
            for (t += threadIdx.x / kSlab; t < end; t += kChunkThreads / kSlab)
                if (threadIdx.x % kSlab < left) po[(int64_t)t * a.out_tok + threadIdx.x % kSlab] = (OUT)0.0f;
        };
        zeros(from, to < first ? to : first);
        zeros(from > last ? from : last, to);
        // final states of sequences without tokens: the first ones
        if (block == 0 && slab == 0 && a.fin != nullptr)
            for (uint32_t s0 = 0; s0 < walk.sequences; s0 += 64) {
                uint64_t empty = __ballot(s0 + lane < walk.sequences && span_of(a, s0 + lane).count == 0);
                for (; empty != 0; empty &= empty - 1) {
                    const int64_t at = ((int64_t)(s0 + __builtin_ctzll(empty)) * a.heads + h) * state_floats;
                    for (uint32_t i = threadIdx.x * 4; i < state_floats; i += kChunkThreads * 4)
                        *reinterpret_cast<f4v*>(a.fin + at + i) = a.init != nullptr ? *reinterpret_cast<const f4v*>(a.init + at + i) : f4v{0, 0, 0, 0};
                }
            }
    }

    // (the chunk's first barrier stands in front of the first look-up)
    if (threadIdx.x <= C) {
        const float power = decayed(log_decay, (float)threadIdx.x);
        lds.powers[threadIdx.x] = power;
        lds.missed[threadIdx.x] = near_one(log_decay, (float)C) ? less_one(log_decay, (float)threadIdx.x) - (power - 1.0f) : 0.0f;
        if (threadIdx.x < C) lds.beyond[threadIdx.x] = 0.0f;
    }
    float missed = 0.0f;                                            // what the roundings of the state's decays have left out so far
    Chunk now, ahead;
    bool more = walk.next<C>(now);
    if (more) fetch_all(now);
    while (more) {
        // (addresses are worked out in every chunk: kept in registers all along they would push others to memory, and the wait for one of those
        // is a wait for the next chunk's rows too)
        uint32_t t = threadIdx.x;
        asm volatile("" : "+v"(t));
        lane = (int)(t & 63);
        n = lane & 15;
        g = lane >> 4;
        row = t / kVecs;
        col = t % kVecs * 8;
        row_c = t / kCVecs;
        col_c = t % kCVecs * 8;
        // ---- the chunk's rows into LDS (all reads of the last chunk's are done)
        if constexpr (!STATES)
#pragma unroll
            for (int p = 0; p < kPasses; ++p) *reinterpret_cast<u4v*>(&lds.a[(row + p * kPassRows) * SA + col]) = ra[p];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) *reinterpret_cast<u4v*>(&lds.b[(row + p * kPassRows) * SB + col]) = rb[p];
#pragma unroll
        for (int p = 0; p < kPassesC; ++p) *reinterpret_cast<u4v*>(&lds.c[(row_c + p * kPassRowsC) * SC + col_c]) = rc[p];
        __syncthreads();
        more = walk.next<C>(ahead);
        if (more) fetch_all(ahead);

        if (now.begin) {
            missed = 0.0f;
            if (a.init != nullptr) {
                const __amdgpu_buffer_rsrc_t from = buffer_at(a.init + ((int64_t)now.s * a.heads + h) * state_floats);
                each([&](float, uint32_t at) { return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from, at, 0, 0)) * a.init_mul; });
            } else {
                clear();
            }
        }
        const int late = a.late && now.begin ? 1 : 0;

        f4v o[CT][NT];
        if constexpr (!STATES) {
            // (binary16: `scale` comes in with the factors at the end)
            const float score_scale = kHalf ? 1.0f : a.out_scale;
            // ---- scores, 16 rows and 32 columns at a time, the rows by lanes
            for (int task = w; task < CT * KS; task += W) {
                const int it = task / KS, jp = task % KS * 2;                      // (column tiles jp and jp + 1)
                if (jp > it) continue;
                f4v s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
                const bool both = jp < it;
                constexpr int kAhead = W == 8 ? (kHalf ? 1 : 2) : 4;                             // (products' operands at once: as registers allow)
#pragma unroll
                for (int k0 = 0; k0 < DK / 32; k0 += kAhead) {
                    v8 rows[kAhead], by[2][kAhead];
#pragma unroll
                    for (int ks = 0; ks < kAhead; ++ks) {
                        if (k0 + ks >= DK / 32) continue;
                        const int at = (k0 + ks) * 32 + 8 * g;
                        rows[ks] = *reinterpret_cast<const v8*>(&lds.a[(it * 16 + n) * SA + at]);
                        by[0][ks] = *reinterpret_cast<const v8*>(&lds.b[(jp * 16 + n) * SB + at]);
                        by[1][ks] = *reinterpret_cast<const v8*>(&lds.b[(jp * 16 + 16 + n) * SB + at]);
                    }
                    loads_first();
#pragma unroll
                    for (int ks = 0; ks < kAhead; ++ks) {
                        if (k0 + ks >= DK / 32) continue;
                        s[0] = mfma(by[0][ks], rows[ks], s[0]);
                        if (both) s[1] = mfma(by[1][ks], rows[ks], s[1]);
                    }
                }
                float largest = 0.0f;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        // (a score above the diagonal is dropped, whatever it is)
                        const int steps = (it - jp - t) * 16 + n - 4 * g - r;
                        s[t][r] = steps < 0 ? 0.0f : s[t][r] * (powers[steps] * score_scale);
                        if constexpr (kHalf) largest = fmaxf(largest, fabsf(s[t][r]));
                    }
                float factor = 1.0f;
                if constexpr (kHalf) {
                    factor = near_top(wave_largest(largest));
                    if (lane == 0) lds.p_factor[it][jp / 2] = factor;
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    uint32_t x[2], y[2];
                    split<T, 2>(s[t][0] * factor, s[t][1] * factor, x, false);
                    split<T, 2>(s[t][2] * factor, s[t][3] * factor, y, false);
                    const int at = (it * 16 + n) * SP + jp * 16 + 8 * g + 4 * t;
                    *reinterpret_cast<u2v*>(&lds.p[0][at]) = u2v{x[0], y[0]};
                    *reinterpret_cast<u2v*>(&lds.p[1][at]) = u2v{x[1], y[1]};
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
                v8 rows[CT];
#pragma unroll
                for (int it = 0; it < CT; ++it) {
                    const T* from = &lds.a[(it * 16 + n) * SA + ks * 32 + 4 * g];
                    rows[it] = joined<T>(*reinterpret_cast<const s4v*>(from), *reinterpret_cast<const s4v*>(from + 16));
                }
                if (!(kHalf && W == 8)) loads_first();
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    u4v parts[2];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const f4v x = S[2 * ks + (r >> 1)][nt];
                        const int e = (r & 1) * 2;
                        uint32_t y[2];
                        split<T, 2>(kHalf ? x[e] * factor : x[e], kHalf ? x[e + 1] * factor : x[e + 1], y, false);
                        parts[0][r] = y[0];
                        parts[1][r] = y[1];
                    }
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int it = 0; it < CT; ++it) o[it][nt] = mfma(__builtin_bit_cast(v8, parts[p]), rows[it], o[it][nt]);
                }
            }
            __syncthreads();                                                       // the scores are there
#pragma unroll
            for (int it = 0; it < CT; ++it) {
                float f = lds.powers[it * 16 + n + 1 - late] * score_scale;
                if constexpr (kHalf) f *= reciprocal_power(factor) * lds.p_factor[it][0];
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
                cols[ks][nt] = joined<T>(columns(lds.c, SC, ks * 32 + 4 * g, at, n), columns(lds.c, SC, ks * 32 + 16 + 4 * g, at, n));
                if constexpr (kHalf)
#pragma unroll
                    for (int r = 0; r < 8; ++r) largest_c = fmaxf(largest_c, fabsf((float)cols[ks][nt][r]));
            }
        float factor_c = 1.0f;
        if constexpr (kHalf) {
            // (here, and not where it is used: a factor is the same for a wavefront, the largest value of each lane would take up a vector register meanwhile.  Also where
            // the largest is at home in binary16: two parts hold 21 bits of what lies within 2^18 of the top, and of smaller values none that lie below 2^-25)
            factor_c = uniform(near_top(wave_largest(largest_c)));
        }
        if constexpr (!STATES) {
            constexpr bool kNextToo = W != 8;                                      // (as registers allow)
            v8 scores[2][CT];                                                      // one part of 32 columns, and the next on its way
            auto read_scores = [&](int at) {
#pragma unroll
                for (int it = at / 2 * 2; it < CT; ++it)
                    scores[at & 1][it] = *reinterpret_cast<const v8*>(&lds.p[at & 1][(it * 16 + n) * SP + at / 2 * 32 + 8 * g]);
            };
            if (kNextToo) read_scores(0);
#pragma unroll
            for (int at = 0; at < 2 * KS; ++at) {
                const int ks = at / 2;
                if (!kNextToo) read_scores(at);
                else if (at + 1 < 2 * KS) read_scores(at + 1);
                loads_first();
#pragma unroll
                for (int it = 2 * ks; it < CT; ++it) {
                    if (kHalf && ks > 0 && (at & 1) == 0) {                        // from the factor of the columns in front to these
                        const float f = lds.p_factor[it][ks] * reciprocal_power(lds.p_factor[it][ks - 1]);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) o[it][nt] *= f;
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) o[it][nt] = mfma(cols[ks][nt], scores[at & 1][it], o[it][nt]);
                }
            }
            // (rows 16 it + n; backwards from the last of C, as above)
            const int64_t first = (int64_t)now.low + (reverse ? now.len - C : 0);
            const __amdgpu_buffer_rsrc_t out = buffer_at(po + ((int64_t)now.s * a.out_seq + first * (int64_t)tok_o));
            const uint32_t pitch = 16 * tok_o * (uint32_t)sizeof(OUT);
            const uint32_t at_row = __umul24((uint32_t)(reverse ? 15 - n : n), tok_o);
#pragma unroll
            for (int it = 0; it < CT; ++it) {
                const float f = kHalf ? a.out_scale * reciprocal_power(lds.p_factor[it][it / 2]) : 1.0f;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint32_t v = (w * NT + nt) * 16 + 4 * g;
                    // (the tile's offset is added here and not given as the store's scalar one: 16-byte stores of that form, binary32 outputs, lost their first
                    // elements in a few lanes: the registers of a store of more than 8 bytes must not be written right behind it, and the compiler keeps that
                    // distance for the form without a scalar offset only)
                    const uint32_t behind = (reverse ? CT - 1 - it : it) * pitch;
                    const uint32_t at = it * 16 + n < now.len && v < left ? (at_row + v) * (uint32_t)sizeof(OUT) + behind : kOutside;
                    typedef OUT o4 __attribute__((ext_vector_type(4)));
                    const f4v x = kHalf ? o[it][nt] * f : o[it][nt];
                    const o4 y = {(OUT)x[0], (OUT)x[1], (OUT)x[2], (OUT)x[3]};
                    if constexpr (sizeof(OUT) == 2) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2v, y), out, at, 0, 0);
                    else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4v, y), out, at, 0, 0);
                }
            }
        }

        // ---- the state behind the chunk
        // (what the chunk adds is summed apart and comes to S at once: one rounding of its size a chunk, and not one for each product.  The decay is rounded so
        // that it makes up for what the roundings of the ones before it have left out: its own is the same in every chunk)
        if (STATES || (now.last ? a.fin != nullptr : more)) {                      // (a state that nothing follows is not worked out)
            const int steps = now.len - late;
            const float power = lds.powers[steps], owed = lds.missed[steps] + missed, decay = power + owed;
            missed = uniform(owed - (decay - power));
            // (a chunk of up to 32 tokens takes the second half's rows of zeros along, 0.5 us: a branch around them sends 12 registers and more to memory)
            constexpr int kBatch = W == 8 ? 2 : 4;                                 // (as registers allow)
            constexpr int kSteps = KT / kBatch * KS;
            v8 rows[2][kBatch];                                                    // of these 32 tokens and kBatch * 16 rows of S, and the next on their way
            auto read_rows = [&](int i) {
#pragma unroll
                for (int m = 0; m < kBatch; ++m) {
                    const int from = i % KS * 32 + 4 * g, at = (i / KS * kBatch + m) * 16;
                    rows[i & 1][m] = joined<T>(columns(lds.b, SB, from, at, n), columns(lds.b, SB, from + 16, at, n));
                }
            };
            u4v part[KS][kParts][NT];
            if (W != 8) read_rows(0);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                float decays[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    decays[r] = powers[now.len - 1 - (ks * 32 + (r >> 2) * 16 + 4 * g + (r & 3))];
                    if constexpr (kHalf) decays[r] *= factor_c;
                }
                loads_first();
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        uint32_t y[kParts];
                        split<T, kParts>((float)cols[ks][nt][2 * r] * decays[2 * r], (float)cols[ks][nt][2 * r + 1] * decays[2 * r + 1], y, true);
#pragma unroll
                        for (int p = 0; p < kParts; ++p) part[ks][p][nt][r] = y[p];
                    }
                loads_first();
            }
            if (W == 8) read_rows(0);
            f4v add[kBatch][NT];
            // (negated twice: an instruction with a negated operand keeps S in its place, without one the sum goes to the place of `add` and 32 registers do not fit)
            const float minus = settled(-decay), back = reciprocal_power(factor_c);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int ks = i % KS, m0 = i / KS * kBatch;
                if (i + 1 < kSteps) read_rows(i + 1);
                loads_first();
#pragma unroll
                for (int p = kParts - 1; p >= 0; --p)
#pragma unroll
                    for (int m = 0; m < kBatch; ++m)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            add[m][nt] = mfma(rows[i & 1][m], __builtin_bit_cast(v8, part[ks][p][nt]), ks == 0 && p == kParts - 1 ? f4v{0, 0, 0, 0} : add[m][nt]);
                if (ks == KS - 1)
#pragma unroll
                    for (int m = 0; m < kBatch; ++m)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int r = 0; r < 4; ++r) S[m0 + m][nt][r] = fmaf(-S[m0 + m][nt][r], minus, kHalf ? add[m][nt][r] * back : add[m][nt][r]);
            }
        }
        if (!STATES && now.last && a.fin != nullptr) {
            const __amdgpu_buffer_rsrc_t to = buffer_at(a.fin + ((int64_t)now.s * a.heads + h) * state_floats);
            const float mul = a.late ? lds.powers[1] * a.fin_mul : a.fin_mul;
            each([&](float x, uint32_t at) {
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x * mul), to, at, 0, 0);
                return x;
            });
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

// What reaches each block from the ones in front of it: running sums over the blocks, in place.  A lane an element: the bytes are few, and it
// is the wavefronts that keep enough of them on their way.
__global__ __launch_bounds__(256) void attention_carry_kernel(const Blocks blocks, uint32_t slabs, uint64_t state_size) {
    const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x, group = at / state_size;      // (head, slab); state_size: a multiple of 256
    float* states = blocks.states + group * (blocks.count - 1) * state_size + at % state_size;
    const Kept* keep = blocks.keep + group / slabs * (blocks.count - 1);
    float carry = 0.0f;
    constexpr uint32_t kAtOnce = 16;         // the loads of many blocks at once, then their sums
    const uint32_t end = blocks.count - 1;
    for (uint32_t n0 = 0; n0 < end; n0 += kAtOnce) {
        float own[kAtOnce];
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) own[i] = states[(n0 + i < end ? n0 + i : end - 1) * state_size];
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i)
            if (n0 + i < end) {
                carry = nothing(keep[n0 + i]) ? own[i] : kept_plus(keep[n0 + i], carry, own[i]);       // (NaN ends with its sequence)
                states[(n0 + i) * state_size] = carry;
            }
    }
}

}  // namespace layers
}  // namespace tcr
