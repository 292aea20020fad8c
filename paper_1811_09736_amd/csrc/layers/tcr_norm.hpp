// Root-mean-square norm with the residual's addition: one pass, the row in registers between its sum of squares and its use.
//
//     s = x + r,   rstd = 1 / sqrt(mean s^2 + eps),   y = s rstd w
// and y in the type of x, or in 8 bits with a scale for each row or each group of columns:
//     scale = max |y| / M (M = 448 for e4m3, 127 for whole numbers; at least 2^-126),   code = y / scale, the binary32 quotient rounded to nearest even.
// Everything between the loads and the stores is binary32; s is stored rounded to the type of x, y comes from the sum before
// that rounding.
//
// Gradients, with g = dy w:   dx = rstd (g - s rstd^2 mean(g s)) + ds,   dw = sum over rows of dy s rstd.
#pragma once
#include "tcr_shared.hpp"

namespace tcr {
namespace layers {

constexpr float kSmallestScale = 1.17549435e-38f;

enum NormOut { kNormSame = 0, kNormE4M3 = 1, kNormI8 = 2 };

struct Norm {
    const void *x, *residual, *weight;
    void *out, *total;
    float *scales, *rstd;
    uint64_t rows, cols;
    int64_t x_stride, r_stride;
    float eps;
    uint32_t group;                            // columns per scale; 0: the row
    uint32_t weight_wide;                      // weight in binary32 beside inputs of 16 bits
};

struct NormGrad {
    const void *dout, *total, *weight, *dtotal;
    const float* rstd;
    void *dx, *dweight;
    float* part;                               // [parts][cols] sums of dweight
    uint64_t rows, cols;
    int64_t dout_stride, total_stride, dtotal_stride;
    uint32_t weight_wide, parts;
};

template <typename T>
__device__ __forceinline__ void load_weight(const void* w, uint32_t wide, uint64_t col, uint64_t cols, float (&v)[kVec]) {
    if (wide) load_vec(static_cast<const float*>(w), col, cols, v);
    else load_vec(static_cast<const T*>(w), col, cols, v);
}

// The larger magnitude; NaN, whose bits are the largest, stays.
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
template <int LANES>
__device__ __forceinline__ uint32_t lanes_largest(uint32_t x) {
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) x = larger(x, (uint32_t)__shfl_xor((int)x, m));
    return x;
}
// The sum (maximum) over what holds a row: LANES lanes of a wavefront (<= 64), or all wavefronts of the workgroup (0).  `room` is free again
// only after the next barrier.
template <int LANES>
__device__ __forceinline__ float row_sum(float x, float* room) {
#pragma unroll
    for (int m = 1; m < (LANES == 0 ? 64 : LANES); m <<= 1) x += __shfl_xor(x, m);
    if constexpr (LANES == 0) {
        if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.0f;
        for (uint32_t w = 0; w < blockDim.x / 64; ++w) x += room[w];
    }
    return x;
}
template <int LANES>
__device__ __forceinline__ uint32_t row_largest(uint32_t x, uint32_t* room) {
    x = lanes_largest<LANES == 0 ? 64 : LANES>(x);
    if constexpr (LANES == 0) {
        if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0;
        for (uint32_t w = 0; w < blockDim.x / 64; ++w) x = larger(x, room[w]);
    }
    return x;
}
// The largest magnitude of a group of columns, which 4, 8 or 16 lanes hold (a row starts on a group; lanes beyond its end hold zeros; fewer
// lanes than a group's hold a whole row).
template <int LANES>
__device__ __forceinline__ uint32_t group_largest(uint32_t x, uint32_t group) {
    x = lanes_largest<4>(x);
    if (group >= 64) x = larger(x, (uint32_t)__shfl_xor((int)x, 4));
    if (group >= 128 && LANES != 8) x = larger(x, (uint32_t)__shfl_xor((int)x, 8));
    return x;
}

template <int OUT>
__device__ __forceinline__ float scale_of(uint32_t largest) {
    const float top = __builtin_bit_cast(float, largest) / (OUT == kNormE4M3 ? 448.0f : 127.0f);
    return top < kSmallestScale ? kSmallestScale : top;          // (NaN stays)
}
// The binary32 quotients of eight values and a scale: the product with the rounded reciprocal, and what it leaves of the value by one more multiply-add.  (8191 x 5120 in 8
// bits 56.9 us, true divisions 59.0, the product alone 56.7, which misses the quotient's last bit and with it one code in a thousand where inputs of few bits put
// quotients on the middle between two codes.)  Scales whose remainders or reciprocals leave the normal range: true divisions.
__device__ __forceinline__ void quotients(const float (&y)[kVec], float scale, float (&q)[kVec]) {
    if (scale >= 0x1p-80f && scale <= 0x1p120f) {
        const float inverse = 1.0f / scale;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            q[i] = y[i] * inverse;
            q[i] = fmaf(fmaf(-q[i], scale, y[i]), inverse, q[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) q[i] = y[i] / scale;
    }
}
// Eight codes.  |y / scale| is at most M but for a rounding, so nothing has to be cut off.  NaN becomes NaN, or 0 as a whole number.
template <int OUT>
__device__ __forceinline__ u2v codes_of(const float (&y)[kVec], float scale) {
    float q[kVec];
    quotients(y, scale, q);
    u2v c;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const float a = q[4 * half], b = q[4 * half + 1], d = q[4 * half + 2], e = q[4 * half + 3];
        if constexpr (OUT == kNormE4M3) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
            c[half] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(d, e, w, true);
        } else {
            auto whole = [](float v) { return (uint32_t)(uint8_t)(int8_t)(v == v ? (int)rintf(v) : 0); };
            c[half] = whole(a) | whole(b) << 8 | whole(d) << 16 | whole(e) << 24;
        }
    }
    return c;
}
__device__ __forceinline__ void store_codes(uint8_t* row, uint64_t col, uint64_t cols, u2v c) {
    if (col + kVec <= cols) {
        typedef uint32_t pair __attribute__((ext_vector_type(2), aligned(1)));
        *reinterpret_cast<pair*>(row + col) = c;
    } else {
        for (int i = 0; i < kVec; ++i)
            if (col + i < cols) row[col + i] = (uint8_t)(c[i >> 2] >> (8 * (i & 3)));
    }
}

// ITEMS vectors per lane; LANES lanes per row and 256 / LANES rows per workgroup, or (0) a row per workgroup, of as many wavefronts as hold it.
// MI355X: 16384 x 4096 bfloat16 with the residual, 537 MB, in 93.5 us, 5.7 TB/s, where a copy reaches 5.2 to 5.5.
constexpr int kNormThreads = 256, kMostWaves = 16;
template <typename T, int OUT, int LANES, int ITEMS>
__global__ __launch_bounds__(LANES == 0 ? kMostWaves * 64 : kNormThreads) void norm_kernel(const Norm a) {
    __shared__ float sums[kMostWaves];
    __shared__ uint32_t most[kMostWaves];
    const uint32_t lanes = LANES == 0 ? blockDim.x : LANES, lane = LANES == 0 ? threadIdx.x : threadIdx.x % LANES;
    const uint64_t row = LANES == 0 ? workgroup() : (uint64_t)workgroup() * (kNormThreads / (LANES == 0 ? 1 : LANES)) + threadIdx.x / (LANES == 0 ? 1 : LANES);
    if (row >= a.rows) return;                            // (whole groups of lanes, in kernels without barriers, or whole workgroups)
    const uint64_t cols = a.cols;
    const T* x = static_cast<const T*>(a.x) + (int64_t)row * a.x_stride;
    const T* r = a.residual != nullptr ? static_cast<const T*>(a.residual) + (int64_t)row * a.r_stride : nullptr;

    typename Vec<T>::v first[ITEMS], second[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) first[i] = load_raw(x, ((uint64_t)i * lanes + lane) * kVec, cols);
    if (r != nullptr) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) second[i] = load_raw(r, ((uint64_t)i * lanes + lane) * kVec, cols);
    }
    float s[ITEMS][kVec], square = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            s[i][j] = (float)first[i][j];
            if (r != nullptr) s[i][j] += (float)second[i][j];
            square = fmaf(s[i][j], s[i][j], square);
        }
    const float rstd = 1.0f / sqrtf(row_sum<LANES>(square, sums) / (float)cols + a.eps);
    if (a.rstd != nullptr && lane == 0) a.rstd[row] = rstd;
    if (a.total != nullptr) {
        T* total = static_cast<T*>(a.total) + row * cols;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) store_vec(total, ((uint64_t)i * lanes + lane) * kVec, cols, s[i]);
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint64_t col = ((uint64_t)i * lanes + lane) * kVec;
        float w[kVec];
        load_weight<T>(a.weight, a.weight_wide, col, cols, w);
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            s[i][j] = s[i][j] * rstd * w[j];
            if constexpr (OUT != kNormSame) top = larger(top, magnitude(s[i][j]));
        }
        if constexpr (OUT == kNormSame) {
            store_vec(static_cast<T*>(a.out) + row * cols, col, cols, s[i]);
        } else if (a.group != 0) {
            const float scale = scale_of<OUT>(group_largest<LANES>(top, a.group));
            if (col < cols) {
                store_codes(static_cast<uint8_t*>(a.out) + row * cols, col, cols, codes_of<OUT>(s[i], scale));
                if (col % a.group == 0) a.scales[row * ((cols + a.group - 1) / a.group) + col / a.group] = scale;
            }
            top = 0;
        }
    }
    if constexpr (OUT != kNormSame) {
        if (a.group == 0) {
            const float scale = scale_of<OUT>(row_largest<LANES>(top, most));
            if (lane == 0) a.scales[row] = scale;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const uint64_t col = ((uint64_t)i * lanes + lane) * kVec;
                if (col < cols) store_codes(static_cast<uint8_t*>(a.out) + row * cols, col, cols, codes_of<OUT>(s[i], scale));
            }
        }
    }
}

// Rows that no registers hold: the row is read again for each use (from a cache, mostly).
constexpr int kLongWaves = kMostWaves;
template <typename T, int OUT>
__global__ __launch_bounds__(kLongWaves * 64) void norm_long_kernel(const Norm a) {
    constexpr uint64_t kStep = kLongWaves * 64 * kVec;
    __shared__ float sums[kLongWaves];
    __shared__ uint32_t most[kLongWaves];
    const uint64_t row = workgroup(), cols = a.cols;
    if (row >= a.rows) return;                            // (whole workgroups)
    const T* x = static_cast<const T*>(a.x) + (int64_t)row * a.x_stride;
    const T* r = a.residual != nullptr ? static_cast<const T*>(a.residual) + (int64_t)row * a.r_stride : nullptr;
    auto sum_at = [&](uint64_t col, float(&s)[kVec]) {
        load_vec(x, col, cols, s);
        if (r == nullptr) return;
        float add[kVec];
        load_vec(r, col, cols, add);
#pragma unroll
        for (int j = 0; j < kVec; ++j) s[j] += add[j];
    };
    float square = 0.0f, s[kVec], w[kVec];
    for (uint64_t col = threadIdx.x * kVec; col < cols; col += kStep) {
        sum_at(col, s);
#pragma unroll
        for (int j = 0; j < kVec; ++j) square = fmaf(s[j], s[j], square);
    }
    const float rstd = 1.0f / sqrtf(row_sum<0>(square, sums) / (float)cols + a.eps);
    if (a.rstd != nullptr && threadIdx.x == 0) a.rstd[row] = rstd;
    float scale = 1.0f;
    if constexpr (OUT != kNormSame) {
        if (a.group == 0) {
            uint32_t top = 0;
            for (uint64_t col = threadIdx.x * kVec; col < cols; col += kStep) {
                sum_at(col, s);
                load_weight<T>(a.weight, a.weight_wide, col, cols, w);
#pragma unroll
                for (int j = 0; j < kVec; ++j) top = larger(top, magnitude(s[j] * rstd * w[j]));
            }
            scale = scale_of<OUT>(row_largest<0>(top, most));
            if (threadIdx.x == 0) a.scales[row] = scale;
        }
    }
    // (all lanes of a wavefront take every step: a group's lanes have to be there together.  `total` may be `residual`: each
    // lane reads its columns for the last time right before it writes them.)
    for (uint64_t first = 0; first < cols; first += kStep) {
        const uint64_t col = first + threadIdx.x * kVec;
        sum_at(col, s);
        if (a.total != nullptr) store_vec(static_cast<T*>(a.total) + row * cols, col, cols, s);
        load_weight<T>(a.weight, a.weight_wide, col, cols, w);
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            s[j] = s[j] * rstd * w[j];
            if constexpr (OUT != kNormSame) top = larger(top, magnitude(s[j]));
        }
        if constexpr (OUT == kNormSame) {
            store_vec(static_cast<T*>(a.out) + row * cols, col, cols, s);
        } else {
            if (a.group != 0) {
                scale = scale_of<OUT>(group_largest<0>(top, a.group));
                if (col < cols && col % a.group == 0) a.scales[row * ((cols + a.group - 1) / a.group) + col / a.group] = scale;
            }
            if (col < cols) store_codes(static_cast<uint8_t*>(a.out) + row * cols, col, cols, codes_of<OUT>(s, scale));
        }
    }
}

// Gradients: a row per wavefront and four per workgroup (LANES == 64), or a row per workgroup (0); each takes every parts-th of them, the next
// row's loads on their way meanwhile, and keeps its sums of dweight in registers.  MI355X: 16384 x 4096 bfloat16, 537 MB, in 98 us and 5 for the parts, 5.2 TB/s
// (166 without the loads ahead, with four wavefronts of 16 columns a lane).
template <typename T, int LANES, int ITEMS>
__global__ __launch_bounds__(LANES == 0 ? kMostWaves * 64 : kNormThreads) void norm_grad_kernel(const NormGrad a) {
    static_assert(LANES == 0 || LANES == 64, "");
    constexpr uint32_t kRowsAtOnce = LANES == 0 ? 1 : kNormThreads / 64;
    __shared__ float sums[2][kMostWaves];
    __shared__ float parts[LANES == 0 ? 1 : kRowsAtOnce][LANES == 0 ? 1 : 64 * kVec * ITEMS];
    const uint32_t lanes = LANES == 0 ? blockDim.x : LANES, lane = LANES == 0 ? threadIdx.x : threadIdx.x % 64, in_group = LANES == 0 ? 0 : threadIdx.x / 64;
    const uint64_t cols = a.cols;
    typedef typename Vec<T>::v vec;
    float dw[ITEMS][kVec] = {};
    vec dy[ITEMS], total[ITEMS], more[ITEMS];
    auto load = [&](uint64_t row) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint64_t col = ((uint64_t)i * lanes + lane) * kVec;
            dy[i] = load_raw(static_cast<const T*>(a.dout) + (int64_t)row * a.dout_stride, col, cols);
            total[i] = load_raw(static_cast<const T*>(a.total) + (int64_t)row * a.total_stride, col, cols);
            if (a.dtotal != nullptr) more[i] = load_raw(static_cast<const T*>(a.dtotal) + (int64_t)row * a.dtotal_stride, col, cols);
        }
    };
    constexpr bool kAhead = ITEMS == 1 || LANES == 64;    // (two vectors a lane leave no registers for the next row's in a workgroup of 16 wavefronts)
    const uint64_t step = (uint64_t)a.parts * kRowsAtOnce;
    uint64_t row = (uint64_t)blockIdx.x * kRowsAtOnce + in_group;
    if (kAhead && row < a.rows) load(row);
    for (int turn = 0; row < a.rows; turn ^= 1) {
        if (!kAhead) load(row);
        const float rstd = a.rstd[row];
        float g[ITEMS][kVec], s[ITEMS][kVec], add[ITEMS][kVec], dot = 0.0f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                g[i][j] = (float)dy[i][j];
                s[i][j] = (float)total[i][j];
                add[i][j] = a.dtotal != nullptr ? (float)more[i][j] : 0.0f;
            }
        const uint64_t next = row + step;
        if (kAhead && next < a.rows) load(next);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint64_t col = ((uint64_t)i * lanes + lane) * kVec;
            float w[kVec];
            load_weight<T>(a.weight, a.weight_wide, col, cols, w);
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                dw[i][j] = fmaf(g[i][j] * rstd, s[i][j], dw[i][j]);
                g[i][j] *= w[j];
                dot = fmaf(g[i][j], s[i][j], dot);
            }
        }
        // (two places for the sums: a wavefront that is a row ahead writes to the other one)
        const float c = row_sum<LANES>(dot, sums[turn]) / (float)cols * rstd * rstd;
        T* dx = static_cast<T*>(a.dx) + row * cols;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
            for (int j = 0; j < kVec; ++j) g[i][j] = fmaf(rstd, g[i][j] - s[i][j] * c, add[i][j]);
            store_vec(dx, ((uint64_t)i * lanes + lane) * kVec, cols, g[i]);
        }
        row = next;
    }
    if constexpr (LANES == 0) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) store_vec(a.part + (uint64_t)blockIdx.x * cols, ((uint64_t)i * lanes + lane) * kVec, cols, dw[i]);
    } else {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int j = 0; j < kVec; ++j) parts[in_group][(i * 64 + lane) * kVec + j] = dw[i][j];
        __syncthreads();
        for (uint32_t col = threadIdx.x; col < cols; col += kNormThreads) {
            float sum = 0.0f;
#pragma unroll
            for (uint32_t r = 0; r < kRowsAtOnce; ++r) sum += parts[r][col];
            a.part[(uint64_t)blockIdx.x * cols + col] = sum;
        }
    }
}

// The same for rows that no registers hold: dx here, dweight in norm_weight_kernel.
template <typename T>
__global__ __launch_bounds__(kLongWaves * 64) void norm_grad_long_kernel(const NormGrad a) {
    constexpr uint64_t kStep = kLongWaves * 64 * kVec;
    __shared__ float sums[kLongWaves];
    const uint64_t row = workgroup(), cols = a.cols;
    if (row >= a.rows) return;                            // (whole workgroups)
    const T* dy = static_cast<const T*>(a.dout) + (int64_t)row * a.dout_stride;
    const T* total = static_cast<const T*>(a.total) + (int64_t)row * a.total_stride;
    const T* more = a.dtotal != nullptr ? static_cast<const T*>(a.dtotal) + (int64_t)row * a.dtotal_stride : nullptr;
    const float rstd = a.rstd[row];
    float g[kVec], s[kVec], w[kVec], dot = 0.0f;
    auto load = [&](uint64_t col) {
        load_vec(dy, col, cols, g);
        load_vec(total, col, cols, s);
        load_weight<T>(a.weight, a.weight_wide, col, cols, w);
#pragma unroll
        for (int j = 0; j < kVec; ++j) g[j] *= w[j];
    };
    for (uint64_t col = threadIdx.x * kVec; col < cols; col += kStep) {
        load(col);
#pragma unroll
        for (int j = 0; j < kVec; ++j) dot = fmaf(g[j], s[j], dot);
    }
    const float c = row_sum<0>(dot, sums) / (float)cols * rstd * rstd;
    for (uint64_t col = threadIdx.x * kVec; col < cols; col += kStep) {
        load(col);
        float add[kVec] = {};
        if (more != nullptr) load_vec(more, col, cols, add);
#pragma unroll
        for (int j = 0; j < kVec; ++j) g[j] = fmaf(rstd, g[j] - s[j] * c, add[j]);
        store_vec(static_cast<T*>(a.dx) + row * cols, col, cols, g);
    }
}

// Sums of dweight over every parts-th row, for 512 columns a workgroup (rows that no registers hold).
template <typename T>
__global__ __launch_bounds__(64) void norm_weight_kernel(const NormGrad a) {
    const uint64_t tiles = (a.cols + 64 * kVec - 1) / (64 * kVec), col = (blockIdx.x % tiles * 64 + threadIdx.x) * kVec;
    const uint32_t part = (uint32_t)(blockIdx.x / tiles);
    float dw[kVec] = {};
    for (uint64_t row = part; row < a.rows; row += a.parts) {
        float g[kVec], s[kVec];
        load_vec(static_cast<const T*>(a.dout) + (int64_t)row * a.dout_stride, col, a.cols, g);
        load_vec(static_cast<const T*>(a.total) + (int64_t)row * a.total_stride, col, a.cols, s);
#pragma unroll
        for (int j = 0; j < kVec; ++j) dw[j] = fmaf(g[j] * a.rstd[row], s[j], dw[j]);
    }
    store_vec(a.part + (uint64_t)part * a.cols, col, a.cols, dw);
}

// dweight from the parts: 64 columns a workgroup, the parts among its 16 wavefronts.
template <typename OUT>
__global__ __launch_bounds__(1024) void norm_parts_kernel(const float* __restrict__ part, OUT* __restrict__ dweight, uint64_t cols, uint32_t parts) {
    __shared__ float sums[16][64];
    const uint64_t col = (uint64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int wave = threadIdx.x >> 6;
    float sum = 0.0f;
    if (col < cols) {
#pragma unroll 16
        for (uint32_t p = wave; p < parts; p += 16) sum += part[(uint64_t)p * cols + col];
    }
    sums[wave][threadIdx.x & 63] = sum;
    __syncthreads();
    if (wave == 0 && col < cols) {
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 16; ++w) sum += sums[w][threadIdx.x];
        dweight[col] = (OUT)sum;
    }
}

}  // namespace layers
}  // namespace tcr
