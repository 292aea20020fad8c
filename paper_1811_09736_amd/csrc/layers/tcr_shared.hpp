// What the operators in this directory use of the library's host side (defined in tcr_api.hip): the workspace of a stream and
// the text of the last HIP error; and the checks and loads that they share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../../include/tcr.h"

namespace tcr {
namespace host {

// Room for `want` floats in the workspace that calls on `stream` use (a multiple of 256 bytes, aligned to 256 bytes), or for
// fewer where it cannot be grown -- the caller's buffer, a stream that is being recorded: *got says how many, at most `want`.
// The memory belongs to the calls on the stream in their order, as all of the workspace does.  With room for fewer than `least` the call cannot go on: what it
// returns then (a caller's buffer: TCR_ERR_WORKSPACE, a stream that is being recorded: TCR_ERR_UNSUPPORTED).
tcr_status partials_for(hipStream_t stream, uint64_t want, uint64_t least, float** room, uint64_t* got);

// TCR_OK, or TCR_ERR_HIP with the error's text kept for tcr_last_hip_error.
tcr_status launched(const char* what);

}  // namespace host

namespace layers {

typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));

inline bool on_boundary(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline uint64_t div_up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// A grid has fewer than 2^32 threads in each of its dimensions; of more, HIP starts what is left of the number modulo 2^32 and reports no error.  Workgroups that need more stand
// in rows of kGridRow; those of the last row that nothing is left for end at once.
constexpr uint32_t kGridRow = (1u << 22) - 1;    // (of up to 1024 threads each)
inline dim3 grid_of(uint64_t blocks) { return blocks <= kGridRow ? dim3((unsigned)blocks) : dim3(kGridRow, (unsigned)div_up(blocks, kGridRow)); }
__device__ __forceinline__ uint32_t workgroup() { return blockIdx.y * kGridRow + blockIdx.x; }

template <typename T> struct Bits;
template <> struct Bits<_Float16> { typedef half8v v8; };
template <> struct Bits<__bf16> { typedef bf8v v8; };

}  // namespace layers
}  // namespace tcr
