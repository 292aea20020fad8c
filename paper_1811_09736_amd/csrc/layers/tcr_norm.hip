// Host side of the root-mean-square norm: checks and launch shapes.
#include "tcr_norm.hpp"

#include <exception>

using namespace tcr;
using namespace tcr::layers;
using tcr::host::launched;
using tcr::host::partials_for;

namespace {

constexpr uint64_t kMostRows = 1ull << 31, kMostCols = 1ull << 24;

// Lanes of 8 columns for a row of up to 512, several rows a workgroup; then a workgroup of as many wavefronts as hold the row, up to 8 of them with 8 columns
// a lane, then with 16.  (5120 columns: 5 wavefronts of 16 a lane 57.0 us for 8191 rows in 8 bits, 10 of 8 a lane 68; 4096: 4 of 16 96.5 us for 16384 rows, 8 of 8 93.9.)
template <typename T, int OUT>
tcr_status run(const Norm& a, hipStream_t s) {
    const unsigned waves = (unsigned)div_up(a.cols, 64 * kVec);
    auto rows = [&](unsigned lanes) { return grid_of(div_up(a.rows, kNormThreads / lanes)); };
    if (a.cols <= 64) norm_kernel<T, OUT, 8, 1><<<rows(8), kNormThreads, 0, s>>>(a);
    else if (a.cols <= 128) norm_kernel<T, OUT, 16, 1><<<rows(16), kNormThreads, 0, s>>>(a);
    else if (a.cols <= 256) norm_kernel<T, OUT, 32, 1><<<rows(32), kNormThreads, 0, s>>>(a);
    else if (a.cols <= 512) norm_kernel<T, OUT, 64, 1><<<rows(64), kNormThreads, 0, s>>>(a);
    else if (waves <= 8) norm_kernel<T, OUT, 0, 1><<<grid_of(a.rows), waves * 64, 0, s>>>(a);
    else if (waves <= 2 * kMostWaves) norm_kernel<T, OUT, 0, 2><<<grid_of(a.rows), (waves + 1) / 2 * 64, 0, s>>>(a);
    else norm_long_kernel<T, OUT><<<grid_of(a.rows), kLongWaves * 64, 0, s>>>(a);
    return launched("norm_kernel");
}

template <typename T>
tcr_status run(const Norm& a, uint32_t codes, hipStream_t s) {
    return codes == TCR_E4M3 ? run<T, kNormE4M3>(a, s) : codes == TCR_I8 ? run<T, kNormI8>(a, s) : run<T, kNormSame>(a, s);
}

bool off(const void* p, uintptr_t size) { return p == nullptr || !on_boundary(p, size); }

// codes: TCR_E4M3 or TCR_I8, or the dtype itself
tcr_status forward(const Norm& a, uint32_t dtype, uint32_t weight_dtype, uint32_t codes, hipStream_t s) {
    if (dtype > TCR_F32 || (weight_dtype != dtype && weight_dtype != TCR_F32) || a.cols == 0) return TCR_ERR_INVALID_ARG;
    if (!(a.eps >= 0.0f)) return TCR_ERR_INVALID_ARG;
    if (a.rows == 0) return TCR_OK;
    const uintptr_t size = dtype == TCR_F32 ? 4 : 2;
    if (off(a.x, size) || off(a.weight, weight_dtype == TCR_F32 ? 4 : 2) || off(a.out, codes == dtype ? size : 1)) return TCR_ERR_INVALID_ARG;
    if (!on_boundary(a.residual, size) || !on_boundary(a.total, size) || !on_boundary(a.rstd, 4)) return TCR_ERR_INVALID_ARG;
    if (a.rows >= kMostRows || a.cols > kMostCols) return TCR_ERR_UNSUPPORTED;
    return dtype == TCR_F16 ? run<_Float16>(a, codes, s) : dtype == TCR_BF16 ? run<__bf16>(a, codes, s) : run<float>(a, codes, s);
}

template <typename T>
tcr_status backward(NormGrad a, hipStream_t s) {
    // Rows of up to 1024 columns a wavefront each, four a workgroup, without barriers (32768 x 1024: 61 us, two wavefronts a row 71); up to 4096 columns 8 a lane with
    // the next row's loads ahead (16384 x 4096: 102 us, 16 a lane without 108); then 16 a lane (8191 x 5120: 79 us, 8 a lane 99).
    // As many parts as keep the chip busy, 16 wavefronts on each compute unit (twice as many: 5 to 10 % slower), or as there is room for.
    const unsigned waves = (unsigned)div_up(a.cols, 64 * kVec), items = waves <= 8 && waves != 2 ? 1 : 2, block = (waves + items - 1) / items * 64;
    const uint64_t rows_at_once = waves <= 2 ? kNormThreads / 64 : 1, units = div_up(a.rows, rows_at_once), held = waves <= 2 * kMostWaves ? div_up(4096, waves) : 1024;
    uint64_t parts = held > 1024 ? 1024 : (held < 256 ? 256 : held), got = 0;
    if (parts > units) parts = units != 0 ? units : 1;
    const tcr_status st = partials_for(s, parts * a.cols, a.cols, &a.part, &got);
    if (st != TCR_OK) return st;
    parts = got / a.cols;
    a.parts = (uint32_t)parts;
    const dim3 grid((unsigned)parts);
    if (waves == 1) norm_grad_kernel<T, 64, 1><<<grid, kNormThreads, 0, s>>>(a);
    else if (waves == 2) norm_grad_kernel<T, 64, 2><<<grid, kNormThreads, 0, s>>>(a);
    else if (items == 1) norm_grad_kernel<T, 0, 1><<<grid, block, 0, s>>>(a);
    else if (waves <= 2 * kMostWaves) norm_grad_kernel<T, 0, 2><<<grid, block, 0, s>>>(a);
    else {
        if (a.rows != 0) norm_grad_long_kernel<T><<<grid_of(a.rows), kLongWaves * 64, 0, s>>>(a);
        norm_weight_kernel<T><<<dim3((unsigned)(parts * div_up(a.cols, 64 * kVec))), 64, 0, s>>>(a);
    }
    if (launched("norm_grad_kernel") != TCR_OK) return TCR_ERR_HIP;
    const dim3 columns((unsigned)div_up(a.cols, 64));
    if (a.weight_wide) norm_parts_kernel<<<columns, 1024, 0, s>>>(a.part, static_cast<float*>(a.dweight), a.cols, a.parts);
    else norm_parts_kernel<<<columns, 1024, 0, s>>>(a.part, static_cast<T*>(a.dweight), a.cols, a.parts);
    return launched("norm_parts_kernel");
}

template <typename F>
tcr_status guarded(F f) {
    try {
        return f();
    } catch (const std::exception&) {
        return TCR_ERR_WORKSPACE;
    }
}

}  // namespace

extern "C" tcr_status tcr_rms_norm(const void* x, const void* residual, const void* weight, void* out, void* total, float* rstd, uint64_t rows,
                                   uint64_t cols, int64_t x_stride, int64_t residual_stride, float eps, uint32_t dtype, uint32_t weight_dtype,
                                   void* stream) {
    return guarded([&] {
        const Norm a = {x, residual, weight, out, total, nullptr, rstd, rows, cols, x_stride, residual_stride, eps, 0, weight_dtype != dtype};
        return forward(a, dtype, weight_dtype, dtype, static_cast<hipStream_t>(stream));
    });
}

extern "C" tcr_status tcr_rms_norm_quantized(const void* x, const void* residual, const void* weight, void* codes, float* scales, void* total,
                                             uint64_t rows, uint64_t cols, int64_t x_stride, int64_t residual_stride, float eps, uint32_t dtype,
                                             uint32_t weight_dtype, uint32_t code_type, uint32_t group, void* stream) {
    return guarded([&] {
        if (code_type != TCR_E4M3 && code_type != TCR_I8) return TCR_ERR_INVALID_ARG;
        if (rows != 0 && off(scales, 4)) return TCR_ERR_INVALID_ARG;
        if (group != 0 && group != 32 && group != 64 && group != 128) return TCR_ERR_UNSUPPORTED;
        const Norm a = {x, residual, weight, codes, total, scales, nullptr, rows, cols, x_stride, residual_stride, eps, group, weight_dtype != dtype};
        return forward(a, dtype, weight_dtype, code_type, static_cast<hipStream_t>(stream));
    });
}

extern "C" tcr_status tcr_rms_norm_backward(const void* dout, const void* total, const void* weight, const float* rstd, const void* dtotal, void* dx,
                                            void* dweight, uint64_t rows, uint64_t cols, int64_t dout_stride, int64_t total_stride,
                                            int64_t dtotal_stride, uint32_t dtype, uint32_t weight_dtype, void* stream) {
    return guarded([&] {
        if (dtype > TCR_F32 || (weight_dtype != dtype && weight_dtype != TCR_F32) || cols == 0) return TCR_ERR_INVALID_ARG;
        const uintptr_t size = dtype == TCR_F32 ? 4 : 2, wsize = weight_dtype == TCR_F32 ? 4 : 2;
        if (off(weight, wsize) || off(dweight, wsize)) return TCR_ERR_INVALID_ARG;
        if (rows != 0 && (off(dout, size) || off(total, size) || off(rstd, 4) || off(dx, size) || !on_boundary(dtotal, size)))
            return TCR_ERR_INVALID_ARG;
        if (rows >= kMostRows || cols > kMostCols) return TCR_ERR_UNSUPPORTED;
        const NormGrad a = {dout, total, weight, dtotal, rstd, dx, dweight, nullptr, rows, cols, dout_stride, total_stride, dtotal_stride,
                            weight_dtype != dtype, 0};
        hipStream_t s = static_cast<hipStream_t>(stream);
        return dtype == TCR_F16 ? backward<_Float16>(a, s) : dtype == TCR_BF16 ? backward<__bf16>(a, s) : backward<float>(a, s);
    });
}
