// Host side of the norm over many tensors and of the clipping: checks, tables, launches.
#include "tcr_clip.hpp"
#include "tcr_operands.hpp"

#include <algorithm>
#include <vector>

using namespace tcr;
using namespace tcr::layers;
using tcr::host::launched;
using tcr::host::partials_for;

namespace {

constexpr uint64_t kMostElements = 1ull << 40;     // of a tensor and of all: pieces stay in 32 bits

uint64_t size_of(uint32_t dtype) { return dtype == TCR_F32 ? 4 : 2; }

tcr_status check(const tcr_tensor* tensors, uint64_t count, const float* norm) {
    if ((count != 0 && tensors == nullptr) || missing(norm, 4)) return TCR_ERR_INVALID_ARG;
    if (count > (1u << 24)) return TCR_ERR_UNSUPPORTED;
    uint64_t all = 0;
    for (uint64_t i = 0; i < count; ++i) {
        const tcr_tensor& t = tensors[i];
        if (t.dtype > TCR_F32 || (t.count != 0 && missing(t.data, size_of(t.dtype)))) return TCR_ERR_INVALID_ARG;
        if (t.count > kMostElements || (all += t.count) > kMostElements) return TCR_ERR_UNSUPPORTED;
    }
    return TCR_OK;
}

// Launch tables over the tensors that hold anything, and the workgroups of each.
struct Launches {
    std::vector<ClipTable> tables;
    std::vector<uint32_t> blocks;
    uint32_t parts = 0;
};
Launches tables_of(const tcr_tensor* tensors, void* const* out, uint64_t count) {
    Launches got;
    uint64_t pieces = 0;
    for (uint64_t i = 0; i < count; ++i) {
        const tcr_tensor& t = tensors[i];
        if (t.count == 0) continue;
        if (got.tables.empty() || got.tables.back().tensors == kClipTensors) {
            got.tables.emplace_back();
            got.tables.back().tensors = got.tables.back().pieces = 0;
        }
        ClipTable& table = got.tables.back();
        const uint32_t at = table.tensors++;
        table.from[at] = t.data;
        table.to[at] = out != nullptr ? out[i] : t.data;
        table.count[at] = t.count << 2 | t.dtype;
        table.first[at] = table.pieces;
        const uint32_t here = (uint32_t)div_up(t.count, kClipPiece);
        table.pieces += here;
        pieces += here;
    }
    // (all launches together have kClipParts sums at most, or one each: one, and a share of the others)
    const uint64_t launches = got.tables.size(), more = launches < kClipParts ? kClipParts - launches : 0;
    for (const ClipTable& t : got.tables) {
        const uint64_t share = pieces <= kClipParts ? t.pieces : 1 + (uint64_t)(t.pieces - 1) * more / (pieces - launches + (more == 0));
        got.blocks.push_back((uint32_t)share);
        got.parts += (uint32_t)share;
    }
    return got;
}

tcr_status sums_of(const Launches& l, double** sums, hipStream_t stream) {
    uint64_t got = 0;
    float* room = nullptr;
    const uint64_t need = 2 * (uint64_t)l.parts;
    const tcr_status st = partials_for(stream, need, need, &room, &got);
    if (st != TCR_OK) return st;
    *sums = reinterpret_cast<double*>(room);
    uint32_t at = 0;
    for (size_t i = 0; i < l.tables.size(); ++i) {
        clip_squares_kernel<<<dim3(l.blocks[i]), kClipThreads, 0, stream>>>(l.tables[i], *sums + at);
        if (launched("clip_squares_kernel") != TCR_OK) return TCR_ERR_HIP;
        at += l.blocks[i];
    }
    return TCR_OK;
}

tcr_status norm_kernel(const Launches& l, const double* sums, float* norm, hipStream_t stream) {
    clip_norm_kernel<<<dim3(1), kFoldThreads, 0, stream>>>(sums, l.parts, nullptr, norm);
    return launched("clip_norm_kernel");
}

// Whether what is written stands in the place of anything but its own tensor, or twice.
bool overlapping(const tcr_tensor* tensors, void* const* out, uint64_t count, const float* norm) {
    struct Range {
        uintptr_t from, to;
        uint64_t index;
    };
    std::vector<Range> written;
    auto range = [&](const void* p, uint64_t i) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        return Range{at, at + (uintptr_t)(tensors[i].count * size_of(tensors[i].dtype)), i};
    };
    for (uint64_t i = 0; i < count; ++i)
        if (tensors[i].count != 0) written.push_back(range(out != nullptr ? out[i] : tensors[i].data, i));
    const uintptr_t n = reinterpret_cast<uintptr_t>(norm);
    written.push_back({n, n + 4, count});
    std::sort(written.begin(), written.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    for (size_t i = 0; i + 1 < written.size(); ++i)
        if (written[i].to > written[i + 1].from) return true;
    if (out == nullptr) return false;
    for (uint64_t i = 0; i < count; ++i) {
        if (tensors[i].count == 0) continue;
        const Range r = range(tensors[i].data, i);
        // the ranges are apart and in order: those that end behind r.from, as far as they begin in front of r.to
        auto w = std::lower_bound(written.begin(), written.end(), r.from, [](const Range& a, uintptr_t from) { return a.to <= from; });
        for (; w != written.end() && w->from < r.to; ++w)
            if (w->index != i || w->from != r.from) return true;
    }
    return false;
}

}  // namespace

extern "C" tcr_status tcr_gradient_norm(const tcr_tensor* tensors, uint64_t count, float* norm, void* stream) {
    return guarded([&] {
        tcr_status st = check(tensors, count, norm);
        if (st != TCR_OK) return st;
        const Launches l = tables_of(tensors, nullptr, count);
        double* sums = nullptr;
        st = sums_of(l, &sums, static_cast<hipStream_t>(stream));
        return st != TCR_OK ? st : norm_kernel(l, sums, norm, static_cast<hipStream_t>(stream));
    });
}

extern "C" tcr_status tcr_clip_gradients(const tcr_tensor* tensors, void* const* out, uint64_t count, float max_norm, float eps, float* norm, void* stream) {
    return guarded([&] {
        tcr_status st = check(tensors, count, norm);
        if (st != TCR_OK) return st;
        if (!(max_norm >= 0.0f) || !(eps >= 0.0f)) return TCR_ERR_INVALID_ARG;
        if (out != nullptr)
            for (uint64_t i = 0; i < count; ++i)
                if (tensors[i].count != 0 && missing(out[i], size_of(tensors[i].dtype))) return TCR_ERR_INVALID_ARG;
        if (overlapping(tensors, out, count, norm)) return TCR_ERR_INVALID_ARG;
        const Launches l = tables_of(tensors, out, count);
        double* sums = nullptr;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        st = sums_of(l, &sums, s);
        if (st != TCR_OK) return st;
        if (l.tables.empty()) return norm_kernel(l, sums, norm, s);
        uint32_t parts = l.parts;
        if (parts > kClipFew) {
            clip_norm_kernel<<<dim3(1), kFoldThreads, 0, s>>>(sums, parts, sums, norm);
            if (launched("clip_norm_kernel") != TCR_OK) return TCR_ERR_HIP;
            parts = 1;
        }
        for (size_t i = 0; i < l.tables.size(); ++i) {
            const ClipLimit limit = {max_norm, eps, i == 0 && parts == l.parts ? norm : nullptr};
            const uint32_t blocks = std::min(l.tables[i].pieces, kClipParts);
            clip_scale_kernel<<<dim3(blocks), kClipThreads, 0, s>>>(l.tables[i], limit, sums, parts);
            if (launched("clip_scale_kernel") != TCR_OK) return TCR_ERR_HIP;
        }
        return TCR_OK;
    });
}
