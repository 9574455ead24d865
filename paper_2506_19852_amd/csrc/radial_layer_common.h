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

// Sixteen bytes at the address of any element: one access, as the memory unit takes any alignment (a wave's lines are then one more).  Against single
// elements, norms of 32 760 x 5121 took 306 us instead of 395, their gradients 565 (739); of 4 x 24 544 x 108, whose rows then are 16 lanes' as aligned
// ones are, 27 (60); a product of 12 837 x 2470 x 1009 with its quantisation 59 (74); half turns of 39 pairs, 2 x 22 500 x 40 heads x 80, 265 (278).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef f32x2 f32x2_any __attribute__((aligned(4)));

// Eight consecutive elements as they lie in memory.  load and store want 16-byte alignment; load_any takes any element's address; load_some and store_some the
// first `count` from there (the others are zero, and are not touched).  set rounds eight values to T, set_pair elements 2 i and
// 2 i + 1 where `on`, and put writes them as they lie: elements that were loaded and not set keep their bits, a NaN's among them.  A row's last eight, where they are fewer, are better read as the eight that
// end with the row and moved down by drop() when they are used: a load whose value is put together from single elements is waited for.
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
  __device__ __forceinline__ void set(const float (&v)[8]) {
    raw = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
  }
  __device__ __forceinline__ void set_pair(int i, bool on, float a, float b) {
    const uint32_t two = pack_bf16(a, b);
    raw[i] = on ? two : raw[i];
  }
  __device__ __forceinline__ void put(__bf16* p) const { *(u32x4*)p = raw; }
  __device__ static __forceinline__ void store(__bf16* p, const float (&v)[8]) {
    Eight<__bf16> e;
    e.set(v);
    e.put(p);
  }
  __device__ __forceinline__ void load_any(const __bf16* p) { raw = *(const u32x4_any*)p; }
  // Element i <- element i + n, zero behind; 0 <= n < 8.
  __device__ __forceinline__ void drop(int n) {
    if (n & 4) raw = u32x4{raw[2], raw[3], 0u, 0u};
    if (n & 2) raw = u32x4{raw[1], raw[2], raw[3], 0u};
    if (n & 1) raw = u32x4{raw[0] >> 16 | raw[1] << 16, raw[1] >> 16 | raw[2] << 16, raw[2] >> 16 | raw[3] << 16, raw[3] >> 16};
  }
  __device__ __forceinline__ void load_some(const __bf16* p, int count) {
    if (count >= 8) return load_any(p);
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = i < count ? ((const uint16_t*)p)[i] : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = e[2 * i] | e[2 * i + 1] << 16;
  }
  __device__ static __forceinline__ void store_some(__bf16* p, const float (&v)[8], int count) {
    Eight<__bf16> e;
    e.set(v);
    e.put_some(p, count);
  }
  __device__ __forceinline__ void put_some(__bf16* p, int count) const {
    if (count >= 8) {
      *(u32x4_any*)p = raw;
      return;
    }
    if (count <= 0) return;
    // four, two, one
    if (count & 4) *(u32x2_any*)p = u32x2{raw[0], raw[1]};
    const uint32_t two = count & 4 ? raw[2] : raw[0], three = count & 4 ? raw[3] : raw[1];
    if (count & 2) *(u32_any*)(p + (count & 4)) = two;
    if (count & 1) *(uint16_t*)(p + (count & 6)) = (uint16_t)(count & 2 ? three : two);
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
  __device__ __forceinline__ void set(const float (&v)[8]) {
    lo = f32x4{v[0], v[1], v[2], v[3]};
    hi = f32x4{v[4], v[5], v[6], v[7]};
  }
  __device__ __forceinline__ void set_pair(int i, bool on, float a, float b) {
    f32x4& half = i < 2 ? lo : hi;
    const int at = 2 * (i & 1);
    half[at] = on ? a : half[at];
    half[at + 1] = on ? b : half[at + 1];
  }
  __device__ __forceinline__ void put(float* p) const {
    *(f32x4*)p = lo;
    *(f32x4*)(p + 4) = hi;
  }
  __device__ static __forceinline__ void store(float* p, const float (&v)[8]) {
    Eight<float> e;
    e.set(v);
    e.put(p);
  }
  __device__ __forceinline__ void load_any(const float* p) {
    lo = *(const f32x4_any*)p;
    hi = *(const f32x4_any*)(p + 4);
  }
  __device__ __forceinline__ void drop(int n) {
    if (n & 4) {
      lo = hi;
      hi = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (n & 2) {
      lo = f32x4{lo[2], lo[3], hi[0], hi[1]};
      hi = f32x4{hi[2], hi[3], 0.f, 0.f};
    }
    if (n & 1) {
      lo = f32x4{lo[1], lo[2], lo[3], hi[0]};
      hi = f32x4{hi[1], hi[2], hi[3], 0.f};
    }
  }
  __device__ __forceinline__ void load_some(const float* p, int count) {
    if (count >= 8) return load_any(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = i < count ? p[i] : 0.f;
      hi[i] = 4 + i < count ? p[4 + i] : 0.f;
    }
  }
  __device__ static __forceinline__ void store_some(float* p, const float (&v)[8], int count) {
    Eight<float> e;
    e.set(v);
    e.put_some(p, count);
  }
  __device__ __forceinline__ void put_some(float* p, int count) const {
    if (count >= 8) {
      *(f32x4_any*)p = lo;
      *(f32x4_any*)(p + 4) = hi;
      return;
    }
    if (count <= 0) return;
    if (count & 4) *(f32x4_any*)p = lo;
    Eight<float> rest = *this;  // moved by drop(), which leaves it in registers; choosing elements by a condition put them into scratch memory
    rest.drop(count & 4);
    if (count & 2) *(f32x2_any*)(p + (count & 4)) = f32x2{rest.lo[0], rest.lo[1]};
    rest.drop(count & 2);
    if (count & 1) p[count & 6] = rest.lo[0];
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
