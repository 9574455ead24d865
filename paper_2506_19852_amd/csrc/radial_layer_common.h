// What the layer operators (norms, rotary positions, 8-bit products) share: eight elements at a time, sums over lanes.  gfx950 only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "radial_internal.h"
#include "radial_layer.h"
#include "radial_tile.h"

namespace radial {

inline bool is_type(int32_t t) { return t == RADIAL_BF16 || t == RADIAL_F32; }
// Threads that a launch may have in its first dimension.
constexpr int64_t kMostThreads = (1LL << 32) - 1024;
inline int size_of(int32_t type) { return type == RADIAL_F32 ? 4 : 2; }

// ---- elements ---------------------------------------------------------------------------------

// Eight consecutive elements as they lie in memory, 16-byte aligned.
template <class T>
struct Eight;
template <>
struct Eight<__bf16> {
  u32x4 raw;
  __device__ __forceinline__ void load(const __bf16* p) { raw = *(const u32x4*)p; }
  __device__ __forceinline__ void clear() { raw = u32x4{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, raw[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, raw[i] & 0xffff0000u);
    }
  }
  __device__ static __forceinline__ void store(__bf16* p, const float (&v)[8]) {
    *(u32x4*)p = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
  }
};
template <>
struct Eight<float> {
  f32x4 lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = *(const f32x4*)p;
    hi = *(const f32x4*)(p + 4);
  }
  __device__ __forceinline__ void clear() { lo = hi = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = lo[i];
      v[4 + i] = hi[i];
    }
  }
  __device__ static __forceinline__ void store(float* p, const float (&v)[8]) {
    *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
};

// ---- sums over lanes ----------------------------------------------------------------------------

template <int kControl>
__device__ __forceinline__ float add_dpp(float x) {
  constexpr int kAll = 0xf;
  return x + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), kControl, kAll, kAll, true));
}
template <int kControl>
__device__ __forceinline__ float max_dpp(float x) {
  constexpr int kAll = 0xf;
  return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), kControl, kAll, kAll, true)));
}
constexpr int kSwapOnes = 0xb1, kSwapTwos = 0x4e;       // quad_perm [1,0,3,2], [2,3,0,1]
constexpr int kHalfRowMirror = 0x141, kRowMirror = 0x140;  // once all four, all eight lanes hold the same, a mirror swaps fours, eights

// The sum over each L neighbouring lanes, the same bits in all of them: in registers (the data-parallel moves within rows of 16 lanes, then the
// swaps of rows and halves), no LDS.
template <int L>
__device__ __forceinline__ float lane_sum(float x) {
  static_assert(L == 16 || L == 32 || L == 64, "whole rows of lanes");
  x = add_dpp<kSwapOnes>(x);
  x = add_dpp<kSwapTwos>(x);
  x = add_dpp<kHalfRowMirror>(x);
  x = add_dpp<kRowMirror>(x);
  if constexpr (L >= 32) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto sw = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t first = sw[0], second = sw[1];
    x = __builtin_bit_cast(float, first) + __builtin_bit_cast(float, second);
  }
  if constexpr (L == 64) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t first = sw[0], second = sw[1];
    x = __builtin_bit_cast(float, first) + __builtin_bit_cast(float, second);
  }
  return x;
}

}  // namespace radial
