// The Euclidean norm of many tensors together, and their scaling to a largest norm.
//
//     norm = sqrt(sum of all squares),   factor = min(1, limit / (norm + eps)),   out = factor g.
// Two passes over the data: sums of squares in binary64, one for each workgroup, always of the same pieces in the same order (squares of binary32 and bfloat16 values
// neither overflow nor vanish there, and what it costs stays behind the loads: 33 T multiply-adds a second beside at most 2.5 T elements);
// then every workgroup adds those sums up for itself -- of many sums one workgroup does in front -- and scales.  Bound by memory.
// The tensors' places travel in the kernel's arguments, kClipTensors a launch: as many as 4 KiB hold.
#pragma once
#include "tcr_shared.hpp"

namespace tcr {
namespace layers {

constexpr int kClipThreads = 256, kClipTensors = 143, kClipItems = 4, kFoldThreads = 1024;
// Workgroups, and sums, of a call at most; of how many sums every scaling workgroup makes the norm itself.  (1e8 binary32 elements: 261 us, with 2048 workgroups 296.)
constexpr uint32_t kClipParts = 8192, kClipFew = 256;
constexpr uint32_t kClipPiece = kClipThreads * kVec * kClipItems;          // elements that a workgroup takes at a time

struct ClipTable {
    const void* from[kClipTensors];
    void* to[kClipTensors];                    // may be `from`
    uint64_t count[kClipTensors];              // times four, and the type
    uint32_t first[kClipTensors];              // of its pieces
    uint32_t tensors, pieces;
};
struct ClipLimit {
    float limit, eps;
    float* norm;                               // written by workgroup 0; NULL: not here
};

static_assert(sizeof(ClipTable) + sizeof(ClipLimit) + 16 <= 4096, "kernel arguments");

// The tensor that a piece belongs to.
__device__ __forceinline__ uint32_t tensor_of(const ClipTable& t, uint32_t piece) {
    uint32_t low = 0, high = t.tensors;        // the last whose first piece is at most `piece`: none has none
    while (high - low > 1) {
        const uint32_t mid = (low + high) / 2;
        if (t.first[mid] <= piece) low = mid;
        else high = mid;
    }
    return low;
}

template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* room) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) v += room[w];
    return v;
}

template <typename T>
__device__ __forceinline__ double squares(const T* from, uint64_t count, uint64_t base) {
    double v[2] = {};
    typename Vec<T>::v x[kClipItems];
#pragma unroll
    for (int i = 0; i < kClipItems; ++i) {
        const uint64_t at = base + (uint64_t)(i * kClipThreads + threadIdx.x) * kVec;
        x[i] = at < count ? load_raw(from, at, count) : typename Vec<T>::v{};
    }
#pragma unroll
    for (int i = 0; i < kClipItems; ++i)
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
            const double d = (double)(float)x[i][k];
            v[k & 1] = __builtin_fma(d, d, v[k & 1]);
        }
    return v[0] + v[1];
}

__global__ __launch_bounds__(kClipThreads) void clip_squares_kernel(ClipTable t, double* sums) {
    __shared__ double room[kClipThreads / 64];
    double v = 0.0;
    for (uint32_t piece = blockIdx.x; piece < t.pieces; piece += gridDim.x) {
        const uint32_t i = tensor_of(t, piece), type = t.count[i] & 3;
        const uint64_t base = (uint64_t)(piece - t.first[i]) * kClipPiece, count = t.count[i] >> 2;
        if (type == TCR_F32) v += squares(static_cast<const float*>(t.from[i]), count, base);
        else if (type == TCR_F16) v += squares(static_cast<const _Float16*>(t.from[i]), count, base);
        else v += squares(static_cast<const __bf16*>(t.from[i]), count, base);
    }
    v = block_sum<kClipThreads>(v, room);
    if (threadIdx.x == 0) sums[blockIdx.x] = v;
}

template <int THREADS>
__device__ __forceinline__ double total_of(const double* sums, uint32_t parts, double* room) {
    double v = 0.0;
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < parts; i += THREADS) v += sums[i];
    return block_sum<THREADS>(v, room);
}

// One sum of all of them (total: NULL: not wanted; may be `sums`, all of which is read in front of it), and the norm (NULL: likewise).
__global__ __launch_bounds__(kFoldThreads) void clip_norm_kernel(const double* sums, uint32_t parts, double* total, float* norm) {
    __shared__ double room[kFoldThreads / 64];
    const double v = total_of<kFoldThreads>(sums, parts, room);
    if (threadIdx.x != 0) return;
    if (total != nullptr) *total = v;
    if (norm != nullptr) *norm = (float)__builtin_sqrt(v);
}

template <typename T>
__device__ __forceinline__ void scaled(const T* from, T* to, uint64_t count, uint64_t base, float factor) {
    typename Vec<T>::v x[kClipItems];
#pragma unroll
    for (int i = 0; i < kClipItems; ++i) {
        const uint64_t at = base + (uint64_t)(i * kClipThreads + threadIdx.x) * kVec;
        if (at < count) x[i] = load_raw(from, at, count);
    }
#pragma unroll
    for (int i = 0; i < kClipItems; ++i) {
        const uint64_t at = base + (uint64_t)(i * kClipThreads + threadIdx.x) * kVec;
        float v[kVec];
#pragma unroll
        for (int k = 0; k < kVec; ++k) v[k] = (float)x[i][k] * factor;
        if (at < count) store_vec(to, at, count, v);
    }
}

__global__ __launch_bounds__(kClipThreads) void clip_scale_kernel(ClipTable t, ClipLimit limit, const double* sums, uint32_t parts) {
    __shared__ double room[kClipThreads / 64];
    const double norm = __builtin_sqrt(total_of<kClipThreads>(sums, parts, room));
    if (limit.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *limit.norm = (float)norm;
    // (a norm that is NaN makes all of it NaN)
    const double ratio = (double)limit.limit / (norm + (double)limit.eps);
    const float factor = ratio >= 1.0 ? 1.0f : (float)ratio;
    for (uint32_t piece = blockIdx.x; piece < t.pieces; piece += gridDim.x) {
        const uint32_t i = tensor_of(t, piece), type = t.count[i] & 3;
        if (factor == 1.0f && t.from[i] == t.to[i]) continue;  // nothing changes
        const uint64_t base = (uint64_t)(piece - t.first[i]) * kClipPiece, count = t.count[i] >> 2;
        if (type == TCR_F32) scaled(static_cast<const float*>(t.from[i]), static_cast<float*>(t.to[i]), count, base, factor);
        else if (type == TCR_F16) scaled(static_cast<const _Float16*>(t.from[i]), static_cast<_Float16*>(t.to[i]), count, base, factor);
        else scaled(static_cast<const __bf16*>(t.from[i]), static_cast<__bf16*>(t.to[i]), count, base, factor);
    }
}

}  // namespace layers
}  // namespace tcr
