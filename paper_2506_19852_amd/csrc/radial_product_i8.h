// What the parts of the 8-bit integer products share: sizes, checks, and the entry points behind the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "radial_layer_common.h"

namespace radial {

constexpr int kCodeGroup = 128;                // codes of a row are kept in whole groups of this many
constexpr int32_t kMostCodeRows = 1 << 29;
constexpr int32_t kMostCodeCols = 1 << 23;
constexpr int32_t kExactCols = 131071;         // products of up to 2^14 each, summed below 2^31
inline int64_t code_groups(int64_t n) { return (n + kCodeGroup - 1) / kCodeGroup; }

inline int check_matrix(const void* p, int32_t type, int64_t stride, int64_t cols, const char* name) {
  if ((uintptr_t)p % size_of(type)) return fail(RADIAL_ESHAPE, "%s is not aligned to its elements", name);
  if (stride < cols) return fail(RADIAL_ESHAPE, "the stride of %s must not be below its columns", name);
  return RADIAL_OK;
}
inline int check_workspace(const void* workspace, size_t bytes, size_t needed) {
  if (!workspace || bytes < needed) return fail(RADIAL_EINVAL, "workspace is NULL or too small: %zu bytes needed, %zu given", needed, workspace ? bytes : (size_t)0);
  if ((uintptr_t)workspace & 255u) return fail(RADIAL_ESHAPE, "workspace is not 256-byte aligned");
  return RADIAL_OK;
}

size_t quantize_i8_workspace(int32_t rows, int32_t cols);
int quantize_i8(int32_t rows, int32_t cols, const void* x, int32_t type, int64_t stride, int8_t* codes, float* scales, int8_t* codes_t, float* scales_t,
                float* sums_t, bool accumulate, void* workspace, hipStream_t stream);

}  // namespace radial
