// The Euclidean norm of many tensors together, and their scaling to a largest norm.
//
//     norm = sqrt(sum of all squares),   factor = min(1, limit / (norm + eps)),   out = factor g.
// Two passes over the data: sums of squares in binary64, one for each workgroup, always of the same pieces in the same order (squares of binary32 and bfloat16 values
// neither overflow nor vanish there, and what it costs stays behind the loads: 33 T multiply-adds a second beside at most 2.5 T elements);
// then every workgroup adds those sums up for itself and scales.  Bound by memory.
// The tensors' places travel in the kernel's arguments, kClipTensors a launch.
#pragma once
#include "tcr_shared.hpp"

namespace tcr {
namespace layers {

constexpr int kClipThreads = 256, kClipTensors = 120, kClipItems = 8;
constexpr uint32_t kClipParts = 2048;          // workgroups, and sums, at most
constexpr uint32_t kClipPiece = kClipThreads * kVec * kClipItems;          // elements that a workgroup takes at a time

struct ClipTensor {
    const void* from;
    void* to;                                  // may be `from`
    uint64_t count;
    uint32_t first, dtype;                     // the first of its pieces
};
struct ClipTable {
    uint32_t tensors, pieces;
    ClipTensor tensor[kClipTensors];
};
static_assert(sizeof(ClipTable) <= 3900, "kernel arguments");

struct ClipLimit {
    float limit, eps;
    float* norm;                               // written by workgroup 0; NULL: not here
};

// The tensor that a piece belongs to.
__device__ __forceinline__ uint32_t tensor_of(const ClipTable& t, uint32_t piece) {
    uint32_t low = 0, high = t.tensors;        // the last whose first piece is at most `piece`: none has none
    while (high - low > 1) {
        const uint32_t mid = (low + high) / 2;
        if (t.tensor[mid].first <= piece) low = mid;
        else high = mid;
    }
    return low;
}

__device__ __forceinline__ double block_sum(double v, double* room) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    return (room[0] + room[1]) + (room[2] + room[3]);
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
    __shared__ double room[4];
    double v = 0.0;
    for (uint32_t piece = blockIdx.x; piece < t.pieces; piece += gridDim.x) {
        const ClipTensor& a = t.tensor[tensor_of(t, piece)];
        const uint64_t base = (uint64_t)(piece - a.first) * kClipPiece;
        if (a.dtype == TCR_F32) v += squares(static_cast<const float*>(a.from), a.count, base);
        else if (a.dtype == TCR_F16) v += squares(static_cast<const _Float16*>(a.from), a.count, base);
        else v += squares(static_cast<const __bf16*>(a.from), a.count, base);
    }
    v = block_sum(v, room);
    if (threadIdx.x == 0) sums[blockIdx.x] = v;
}

__device__ __forceinline__ double norm_of(const double* sums, uint32_t parts, double* room) {
    double v = 0.0;
    for (uint32_t i = threadIdx.x; i < parts; i += kClipThreads) v += sums[i];
    return __builtin_sqrt(block_sum(v, room));
}

__global__ __launch_bounds__(kClipThreads) void clip_norm_kernel(const double* sums, uint32_t parts, float* norm) {
    __shared__ double room[4];
    const double v = norm_of(sums, parts, room);
    if (threadIdx.x == 0) *norm = (float)v;
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
    __shared__ double room[4];
    const double norm = norm_of(sums, parts, room);
    if (limit.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *limit.norm = (float)norm;
    // (a norm that is NaN makes all of it NaN)
    const double ratio = (double)limit.limit / (norm + (double)limit.eps);
    const float factor = ratio >= 1.0 ? 1.0f : (float)ratio;
    for (uint32_t piece = blockIdx.x; piece < t.pieces; piece += gridDim.x) {
        const ClipTensor& a = t.tensor[tensor_of(t, piece)];
        if (factor == 1.0f && a.from == a.to) continue;        // nothing changes
        const uint64_t base = (uint64_t)(piece - a.first) * kClipPiece;
        if (a.dtype == TCR_F32) scaled(static_cast<const float*>(a.from), static_cast<float*>(a.to), a.count, base, factor);
        else if (a.dtype == TCR_F16) scaled(static_cast<const _Float16*>(a.from), static_cast<_Float16*>(a.to), a.count, base, factor);
        else scaled(static_cast<const __bf16*>(a.from), static_cast<__bf16*>(a.to), a.count, base, factor);
    }
}

}  // namespace layers
}  // namespace tcr
