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

// ---- codes ----------------------------------------------------------------------------------------

constexpr float kLargestCode = 127.f;
constexpr float kSmallestCodeScale = 1.17549435e-38f;  // 2^-126
constexpr uint32_t kInfinityBits = 0x7f800000u;

// Largest magnitudes are compared as bits: a NaN is above infinity, infinity above all others, so that neither is lost.
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

template <int kControl>
__device__ __forceinline__ uint32_t max_dpp_bits(uint32_t x) {
  constexpr int kAll = 0xf;
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kControl, kAll, kAll, true));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max_dpp_bits<kSwapOnes>(x);
  x = max_dpp_bits<kSwapTwos>(x);
  x = max_dpp_bits<kHalfRowMirror>(x);
  x = max_dpp_bits<kRowMirror>(x);
  const auto rows = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max((uint32_t)rows[0], (uint32_t)rows[1]);
  const auto halves = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max((uint32_t)halves[0], (uint32_t)halves[1]);
}

// x / scale to the nearest whole number, in the low byte.  The quotient as a float32 value is the product with the inverse, and what it leaves, once
// more (off by half a unit and 2^-46 of the value); adding 1.5 * 2^23 rounds it to whole, ties to even.
struct Code {
  float scale, inverse;
  Code() = default;
  __device__ __forceinline__ explicit Code(uint32_t largest) {
    const float amax = __builtin_bit_cast(float, largest);
    scale = largest < kInfinityBits ? fmaxf(amax / kLargestCode, kSmallestCodeScale) : __builtin_nanf("");
    inverse = 1.f / scale;
  }
  __device__ __forceinline__ uint32_t operator()(float x) const {
    const float q = x * inverse;
    const float quotient = __builtin_fmaf(__builtin_fmaf(-q, scale, x), inverse, q);
    return __builtin_bit_cast(uint32_t, quotient + 12582912.f);
  }
  // Four codes, all 0 where the scale is NaN.
  __device__ __forceinline__ uint32_t four(float a, float b, float c, float d) const {
    constexpr uint32_t kLowBytes = 0x0c0c0400u, kLowHalves = 0x05040100u;
    const uint32_t ab = __builtin_amdgcn_perm((*this)(b), (*this)(a), kLowBytes), cd = __builtin_amdgcn_perm((*this)(d), (*this)(c), kLowBytes);
    const uint32_t all = __builtin_amdgcn_perm(cd, ab, kLowHalves);
    return scale == scale ? all : 0u;
  }
};

// ---- between the sources --------------------------------------------------------------------------

// A matrix to quantise: codes and scales of its rows, of its columns (codes_t), sums of its columns; pitches in bytes, 0: the columns rounded up to whole groups.
struct QuantI8 {
  const void* x;
  int64_t stride;
  int32_t rows, cols;
  int8_t *codes, *codes_t;
  int64_t pitch, pitch_t;
  float *scales, *scales_t, *sums_t;
  bool accumulate;
};
size_t quantize_i8_workspace(int32_t rows, int32_t cols);
// One or two matrices of one type, each with a workspace of its own; of two, the columns of both are wanted.
int quantize_i8(const QuantI8* q, int count, int32_t type, char* const* workspace, hipStream_t stream);

// Bytes from a row of codes to the next in a workspace: an odd number of groups, so that the rows of a tile do not meet in a few of the memory's channels
// (32 768 x 5120 x 5120: 687 us with the activations' rows 41 groups apart, 704 with 40).
inline int64_t odd_pitch(int64_t cols) { return (code_groups(cols) | 1) * kCodeGroup; }

}  // namespace radial
