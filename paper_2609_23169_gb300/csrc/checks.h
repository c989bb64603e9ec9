// Small host checks shared by the entry points.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ultratex.h"

namespace ut {

inline bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool at4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline ut_status status_of(cudaError_t e) { return e == cudaSuccess ? UT_OK : UT_ERR_CUDA; }

}  // namespace ut
