// What a tuning step does with the gradients, for gfx950: their common norm, and AdamW over many tensors in one launch, with states in float32 or in E4M3
// codes with a scale for each 128 values.  Both are bound by memory: 28 bytes a value with float32 weights, gradients and states, 14 with states
// in 8 bits and bf16 gradients.
//
// A table on the device names the tensors and, for every piece of 4096 values of one of them, which it is: a workgroup takes one piece, so that one launch
// serves tensors of any number and size.
#include <math.h>

#include "radial_layer_common.h"

namespace radial {
namespace {

constexpr int kBlock = 128;             // values that share a scale
constexpr int kPiece = 4096;            // values of a workgroup
constexpr int kMostPieces = 1 << 23;    // the launch's threads stay below 2^32
constexpr int kNormGroups = 2048;       // workgroups of the norm at most: eight a compute unit
constexpr float kLargest = 448.f;       // of E4M3
constexpr float kMostFloat = 3.402823466e38f;
constexpr float kSmallestLargest = 0x1p-100f;  // blocks of smaller values are zeros: 448 / amax stays in range

struct Tensor {
  void* weight;
  __bf16* copy;
  const void* grad;
  void *first, *second;
  float *first_scales, *second_scales;
  int64_t n;
  float decay;
  int32_t kind;
};
// bits of kind
constexpr int kWeightF32 = 1, kGradF32 = 2, kCodes = 4;

struct Piece {
  int32_t tensor, index;
};

// Values of a piece that begins at value `at`.
__device__ __forceinline__ int32_t left_of(const Tensor& t, int64_t at) { return (int32_t)(t.n - at < kPiece ? t.n - at : kPiece); }

// The table: `count` tensors, then `pieces` pieces.
inline size_t table_bytes_of(int64_t count, int64_t pieces) { return (size_t)count * sizeof(Tensor) + (size_t)pieces * sizeof(Piece); }
__host__ __device__ __forceinline__ const Piece* pieces_of_table(const void* table, int32_t count) { return (const Piece*)((const Tensor*)table + count); }

// ---- table ------------------------------------------------------------------------------------------

constexpr int kTensorsAtOnce = 32;  // arguments of a launch, 2.4 KB
struct TableArgs {
  void* table;
  int32_t count, first;
  int32_t piece0[kTensorsAtOnce];
  Tensor tensors[kTensorsAtOnce];
};
static_assert(sizeof(TableArgs) <= 4096, "arguments of a launch");

__global__ void __launch_bounds__(256) write_table_kernel(TableArgs a) {
  const int32_t i = blockIdx.x;
  const Tensor t = a.tensors[i];
  if (threadIdx.x == 0) ((Tensor*)a.table)[a.first + i] = t;
  Piece* pieces = (Piece*)pieces_of_table(a.table, a.count) + a.piece0[i];
  const int32_t count = (int32_t)((t.n + kPiece - 1) / kPiece);
  for (int32_t p = threadIdx.x; p < count; p += 256) pieces[p] = Piece{a.first + i, p};
}

// ---- four values at a time --------------------------------------------------------------------------

// The four values from p + at, of which `count` are inside the tensor (kWhole: all).
typedef uint32_t u32_byte_any __attribute__((aligned(1)));
template <bool kWhole>
__device__ __forceinline__ f32x4 load_four(const float* p, uint32_t at, int32_t count) {
  p += at;
  if (kWhole || count >= 4) return *(const f32x4_any*)p;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < count) v[e] = p[e];
  return v;
}
template <bool kWhole>
__device__ __forceinline__ f32x4 load_four(const __bf16* p, uint32_t at, int32_t count) {
  p += at;
  if (kWhole || count >= 4) {
    const u32x2 r = *(const u32x2_any*)p;
    return f32x4{__builtin_bit_cast(float, r[0] << 16), __builtin_bit_cast(float, r[0] & 0xffff0000u), __builtin_bit_cast(float, r[1] << 16),
                 __builtin_bit_cast(float, r[1] & 0xffff0000u)};
  }
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < count) v[e] = (float)p[e];
  return v;
}
template <bool kWhole>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, uint32_t at, int32_t count) {
  p += at;
  if (kWhole || count >= 4) return *(const u32_byte_any*)p;
  uint32_t v = 0;
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < count) v |= (uint32_t)p[e] << 8 * e;
  return v;
}
template <bool kWhole>
__device__ __forceinline__ void store_four(float* p, uint32_t at, f32x4 v, int32_t count) {
  p += at;
  if (kWhole || count >= 4) {
    *(f32x4_any*)p = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < count) p[e] = v[e];
}
template <bool kWhole>
__device__ __forceinline__ void store_four(__bf16* p, uint32_t at, f32x4 v, int32_t count) {
  p += at;
  if (kWhole || count >= 4) {
    *(u32x2_any*)p = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < count) p[e] = (__bf16)v[e];
}
template <bool kWhole>
__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t at, uint32_t v, int32_t count) {
  p += at;
  if (kWhole || count >= 4) {
    *(u32_byte_any*)p = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < count) p[e] = (uint8_t)(v >> 8 * e);
}

// ---- norm -------------------------------------------------------------------------------------------

// Squares and sums in 64 bits: a float32 square passes its range from 2^64 on, and 10^8 of them lose three digits.  Each workgroup writes its sum; a second launch adds
// them up in order.
template <class T>
__device__ __forceinline__ double squares_of_piece(const T* g, int32_t count) {
  Eight<T> v[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int32_t at = (j * 256 + (int)threadIdx.x) * 8;
    v[j].load_some(g + at, count - at);
  }
  double sum = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float x[8];
    v[j].get(x);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fma((double)x[e], (double)x[e], sum);
  }
  return sum;
}

__device__ __forceinline__ double block_sum(double x) {
  __shared__ double of_wave[4];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = x;
  __syncthreads();
  return (of_wave[0] + of_wave[1]) + (of_wave[2] + of_wave[3]);
}

__global__ void __launch_bounds__(256) grad_squares_kernel(const void* table, int32_t count, int32_t pieces, double* sums) {
  const Piece* all = pieces_of_table(table, count);
  double sum = 0;
  for (int32_t p = blockIdx.x; p < pieces; p += gridDim.x) {
    const Piece piece = all[p];
    const Tensor& t = ((const Tensor*)table)[piece.tensor];
    const int64_t at = (int64_t)piece.index * kPiece;
    const int32_t left = left_of(t, at);
    sum += t.kind & kGradF32 ? squares_of_piece((const float*)t.grad + at, left) : squares_of_piece((const __bf16*)t.grad + at, left);
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(256) finish_norm_kernel(const double* sums, int32_t count, float scale, float max_norm, float* norm) {
  double sum = 0;
  for (int32_t i = threadIdx.x; i < count; i += 256) sum += sums[i];
  sum = block_sum(sum);
  if (threadIdx.x) return;
  const double length = (double)scale * sqrt(sum);
  norm[0] = (float)length;
  norm[1] = !(sum <= 1.7976931348623157e308) ? __builtin_nanf("") : length > (double)max_norm ? (float)((double)scale * ((double)max_norm / length)) : scale;
}

// ---- step -------------------------------------------------------------------------------------------

struct StepArgs {
  const void* table;
  int32_t count;
  float lr, beta1, of_grad1, beta2, of_grad2, eps, by_first, by_second;
  double lr_wide;
  float log_beta1, log_beta2;
  int64_t step;
  uint64_t seed;
  const float* factor;
  const float* lr_at;
  const int64_t* step_at;
};

__host__ __device__ __forceinline__ uint32_t mixed(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9E3779B1u;
  x ^= x >> 15;
  x *= 0x6A09E667u;
  return x ^ x >> 16;
}

// The largest of each 32 neighbouring lanes, in all of them.
__device__ __forceinline__ float max_of_32(float x) {
  x = max_dpp<kSwapOnes>(x);
  x = max_dpp<kSwapTwos>(x);
  x = max_dpp<kHalfRowMirror>(x);
  x = max_dpp<kRowMirror>(x);
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto sw = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t first = sw[0], second = sw[1];
  return fmaxf(__builtin_bit_cast(float, first), __builtin_bit_cast(float, second));
}

__device__ __forceinline__ f32x4 decode_four(uint32_t codes, float scale) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  return f32x4{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
}
__device__ __forceinline__ uint32_t nearest_codes(f32x4 y) {
  int v = 0;  // v_cvt_pk_fp8_f32 rounds to nearest even
  v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], v, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], v, true);
  return (uint32_t)v;
}
// Towards zero or one code further, by sixteen random bits.  Times 2^-120 E4M3's smallest normal number is float32's, so that the codes are the upper bits of the
// product, subnormal ones too, and a carry moves on into the exponent.
__device__ __forceinline__ uint32_t random_code(float y, uint32_t bits16) {
  const uint32_t u = __builtin_bit_cast(uint32_t, y), magnitude = __builtin_bit_cast(uint32_t, fabsf(y) * 0x1p-120f);
  const uint32_t code = min((magnitude + (bits16 << 4)) >> 20, 0x7eu);
  return (y == y ? code : 0x7fu) | (u >> 31) << 7;
}

// Quotients and roots without the steps of the library functions that cover operands which do not occur here: 60 instructions a value where those took 85, and 105 million bf16 weights with bf16
// gradients and states in 8 bits 196 us instead of 297.  The three below are rounded to nearest, for every significand and with the instruction's result off by a unit either way, so that the codes
// are those of float32 arithmetic; the weights' quotient is the product with v_rcp_f32's inverse, a unit off, which only moves the update by 2^-23 of itself.
//
// a / 448: product with the inverse, and what it leaves once more.
__device__ __forceinline__ float over_448(float a) {
  constexpr float kInverse = 1.f / kLargest;
  const float q = a * kInverse;
  return __builtin_fmaf(__builtin_fmaf(-q, kLargest, a), kInverse, q);
}
// 448 / a for a from 2^-100 on, as (448 2^-9) / (a 2^-9), so that the inverse is a normal number.
__device__ __forceinline__ float of_448(float a) {
  constexpr float kScaled = kLargest * 0x1p-9f;
  const float t = a * 0x1p-9f, first = __builtin_amdgcn_rcpf(t), r = __builtin_fmaf(__builtin_fmaf(-t, first, 1.f), first, first), q = kScaled * r;
  return __builtin_fmaf(__builtin_fmaf(-q, t, kScaled), r, q);
}
// sqrt(v), rounded to nearest: v / sqrt(v) and 1 / (2 sqrt(v)), both corrected once by what their product leaves of 1/2, and the root by what its square leaves of v.  Where that would leave the
// normal numbers, below 2^-96, 2^64 v takes v's place (kSmall: it may be; a wave without such a value does without the choice, and 105 million bf16 weights took 196 us instead of 198, rounded at
// random 234 instead of 242).  NaN for an infinite v, whose code in the state is that of NaN; what divides by the root takes NaN for infinity, now and when the code is read again: m over it is 0, as it
// is with states in float32.  (A NaN in v without one in m has no other origin.)
constexpr float kSmallSquare = 0x1p-96f;
template <bool kSmall>
__device__ __forceinline__ float root_of(float v) {
  const bool small = kSmall && v < kSmallSquare;
  const float x = small ? v * 0x1p64f : v, y = __builtin_amdgcn_rsqf(kSmall ? fmaxf(x, 0x1p-126f) : x), s = x * y, half = 0.5f * y;
  const float left = __builtin_fmaf(-half, s, 0.5f), root = __builtin_fmaf(s, left, s);
  const float nearest = __builtin_fmaf(__builtin_fmaf(-root, root, x), __builtin_fmaf(half, left, half), root);
  return small ? nearest * 0x1p-32f : nearest;
}

// Codes and scale of a block's values: 32 lanes, four each.
template <bool kPositive, bool kRandom>
__device__ __forceinline__ uint32_t encode_four(f32x4 v, const uint32_t (&bits)[4], float& scale) {
  float largest = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
  largest = max_of_32(largest);
  const bool any = largest >= kSmallestLargest;
  scale = any ? over_448(largest) : 0.f;
  const float inverse = any ? of_448(largest) : 0.f;
  if (largest == __builtin_inff()) scale = largest;  // and the codes are those of NaN
  f32x4 y = {v[0] * inverse, v[1] * inverse, v[2] * inverse, v[3] * inverse};
  if constexpr (kRandom) {
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float one = y[e];  // (the bits of y[e] itself are those of y[0]: a bit cast of a vector's element takes the vector's address)
      uint32_t code = random_code(one, kPositive ? bits[e] >> 16 : bits[e] & 0xffffu);
      if (kPositive) code = max(code, min(__builtin_bit_cast(uint32_t, one), 1u));  // a positive value keeps a positive code
      codes |= code << 8 * e;
    }
    return codes;
  }
  if (kPositive) {
    // a positive value keeps a positive code: it is the smallest code's value at least; 0 stays 0 and NaN NaN.  (From the smallest root, 2^-74.5, beside the largest, 2^64, y is 2^-129.7: positive.)
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = y[e] > 0.f ? fmaxf(y[e], 0x1p-9f) : y[e];
  }
  return nearest_codes(y);
}

// The step of a workgroup's piece: a wave takes 1024 neighbouring values, a lane four of every 256 (so that 32 lanes are one block of 128).  Products
// and sums are rounded one by one, as the formula is written: a state's codes then do not depend on how a compiler joins them.
template <class W, class G, bool kCoded, bool kRandom, bool kWhole>
__device__ __forceinline__ void step_piece(const StepArgs& a, const Tensor& t, Piece piece, int32_t left, float factor, float by_decay, float by_first, float by_second, int64_t step) {
#pragma clang fp contract(off)
  const int64_t first = (int64_t)piece.index * kPiece;
  const uint32_t lane_at = (threadIdx.x >> 6) * 1024 + (threadIdx.x & 63) * 4;
  W* weight = (W*)t.weight + first;
  const G* grad = (const G*)t.grad + first;
  uint8_t *m_coded = (uint8_t*)t.first + first, *v_coded = (uint8_t*)t.second + first;
  float *m_wide = (float*)t.first + first, *v_wide = (float*)t.second + first;
  float *m_scales = t.first_scales + first / kBlock, *v_scales = t.second_scales + first / kBlock;
  f32x4 w[4], g[4], m[4], v[4];
  uint32_t m_codes[4], v_codes[4];
  float m_scale[4], v_scale[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t at = lane_at + j * 256;
    const int32_t count = left - (int32_t)at;
    g[j] = load_four<kWhole>(grad, at, count);
    w[j] = load_four<kWhole>(weight, at, count);
    if constexpr (kCoded) {
      m_codes[j] = load_codes<kWhole>(m_coded, at, count);
      v_codes[j] = load_codes<kWhole>(v_coded, at, count);
      m_scale[j] = kWhole || count > 0 ? m_scales[at / kBlock] : 0.f;
      v_scale[j] = kWhole || count > 0 ? v_scales[at / kBlock] : 0.f;
    } else {
      m[j] = load_four<kWhole>(m_wide, at, count);
      v[j] = load_four<kWhole>(v_wide, at, count);
    }
  }
  uint32_t key = 0;
  if constexpr (kRandom) {
    key = mixed(mixed(mixed((uint32_t)a.seed) ^ (uint32_t)(a.seed >> 32)) ^ (uint32_t)step);
    key = mixed(key ^ (uint32_t)piece.tensor);
    const uint32_t far = (uint32_t)(first >> 32);
    if (far) key = mixed(key ^ far);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t at = lane_at + j * 256;
    const int32_t count = left - (int32_t)at;
    const bool some = kWhole || count > 0;
    if constexpr (kCoded) {
      m[j] = decode_four(m_codes[j], m_scale[j]);
      v[j] = decode_four(v_codes[j], v_scale[j]);
      v[j] = v[j] * v[j];
    }
    f32x4 root;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = g[j][e] * factor;
      m[j][e] = m[j][e] * a.beta1 + x * a.of_grad1;
      v[j][e] = v[j][e] * a.beta2 + x * x * a.of_grad2;
    }
    if constexpr (!kCoded) {
#pragma unroll
      for (int e = 0; e < 4; ++e) root[e] = sqrtf(v[j][e]);
    } else if (__builtin_amdgcn_ballot_w64(fminf(fminf(v[j][0], v[j][1]), fminf(v[j][2], v[j][3])) < kSmallSquare)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) root[e] = root_of<true>(v[j][e]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) root[e] = root_of<false>(v[j][e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float divisor = root[e] * by_second + a.eps;
      if constexpr (kCoded) divisor = fminf(divisor, __builtin_inff());  // a root that is NaN counts as infinite
      // the decay joins the update before either meets the weight: as a factor 1 - lr decay of float32 it would be a multiple of 2^-24, 19 % too much at 1e-7 and nothing at 1e-8.  (An infinite
      // weight stays one: its decay is that of the largest number.)
      const float inside = __builtin_amdgcn_fmed3f(w[j][e], -kMostFloat, kMostFloat);
      w[j][e] = w[j][e] - __builtin_fmaf(by_decay, inside, by_first * (m[j][e] * __builtin_amdgcn_rcpf(divisor)));
    }
    if (some) {
      store_four<kWhole>(weight, at, w[j], count);
      if (t.copy) store_four<kWhole>(t.copy + first, at, w[j], count);
    }
    if constexpr (kCoded) {
      uint32_t bits[4] = {};
      if constexpr (kRandom) {
#pragma unroll
        for (int e = 0; e < 4; ++e) bits[e] = mixed(key ^ ((uint32_t)first + at + e));
      }
      if (!kWhole && count < 4) {
        // what lies behind the tensor counts for nothing in its block
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e >= count) m[j][e] = root[e] = 0.f;
      }
      float ms, vs;
      const uint32_t mc = encode_four<false, kRandom>(m[j], bits, ms), vc = encode_four<true, kRandom>(root, bits, vs);
      if (some) {
        store_codes<kWhole>(m_coded, at, mc, count);
        store_codes<kWhole>(v_coded, at, vc, count);
        if ((threadIdx.x & 31) == 0) {
          m_scales[at / kBlock] = ms;
          v_scales[at / kBlock] = vs;
        }
      }
    } else if (some) {
      store_four<kWhole>(m_wide, at, m[j], count);
      store_four<kWhole>(v_wide, at, v[j], count);
    }
  }
}

template <class W_, class G_, bool kCoded_, bool kRandomly_>
struct step_of {
  using W = W_;
  using G = G_;
  static constexpr bool kCoded = kCoded_, kRandomly = kRandomly_;
};

template <bool kRandom>
__global__ void __launch_bounds__(256) adamw_step_kernel(StepArgs a) {
  const Piece piece = pieces_of_table(a.table, a.count)[blockIdx.x];
  const Tensor t = ((const Tensor*)a.table)[piece.tensor];
  const float factor = a.factor ? *a.factor : 1.f;
  if (!(fabsf(factor) < __builtin_inff())) return;
  int64_t step = a.step_at ? *a.step_at : a.step;
  step = step > 1 ? step : 1;  // of the corrections and of the random bits
  float lr = a.lr, by_first = a.by_first, by_second = a.by_second, by_decay;
  if (a.lr_at || a.step_at) {
    // from the device: 1 - beta^t as -(e^(t log beta) - 1), which keeps its digits where beta^t is near 1
    if (a.lr_at) lr = *a.lr_at;
    const float counted = (float)step;
    by_first = lr / (a.beta1 > 0.f ? -expm1f(counted * a.log_beta1) : 1.f);
    by_second = 1.f / sqrtf(a.beta2 > 0.f ? -expm1f(counted * a.log_beta2) : 1.f);
    by_decay = lr * t.decay;
  } else {
    by_decay = (float)(a.lr_wide * (double)t.decay);
  }
  const int32_t left = left_of(t, (int64_t)piece.index * kPiece);
  auto go = [&](auto types) __attribute__((always_inline)) {
    using S = decltype(types);
    if (left == kPiece) step_piece<typename S::W, typename S::G, S::kCoded, S::kRandomly, true>(a, t, piece, left, factor, by_decay, by_first, by_second, step);
    else step_piece<typename S::W, typename S::G, S::kCoded, S::kRandomly, false>(a, t, piece, left, factor, by_decay, by_first, by_second, step);
  };
  switch (t.kind) {
    case 0: return go(step_of<__bf16, __bf16, false, false>{});
    case 1: return go(step_of<float, __bf16, false, false>{});
    case 2: return go(step_of<__bf16, float, false, false>{});
    case 3: return go(step_of<float, float, false, false>{});
    case 4: return go(step_of<__bf16, __bf16, true, kRandom>{});
    case 5: return go(step_of<float, __bf16, true, kRandom>{});
    case 6: return go(step_of<__bf16, float, true, kRandom>{});
    default: return go(step_of<float, float, true, kRandom>{});
  }
}

// ---- host ---------------------------------------------------------------------------------------------

int check_tensor(const radial_adamw_tensor& t, int32_t i) {
  if (t.n < 0 || t.n >= 1LL << 40) return fail(RADIAL_EINVAL, "tensor %d: n must be >= 0 and below 2^40 (got %lld)", i, (long long)t.n);
  if (!is_type(t.weight_type) || !is_type(t.grad_type)) return fail(RADIAL_EINVAL, "tensor %d: types must be RADIAL_BF16 or RADIAL_F32", i);
  if (!(t.decay >= 0.0 && t.decay <= 3.4028234663852886e38)) return fail(RADIAL_EINVAL, "tensor %d: decay must be >= 0 and finite", i);
  if (!t.first_scales != !t.second_scales) return fail(RADIAL_EINVAL, "tensor %d: first_scales and second_scales go together", i);
  if (t.n && (!t.weight || !t.grad || !t.first || !t.second)) return fail(RADIAL_EINVAL, "tensor %d: weight, grad, first or second is NULL", i);
  const uintptr_t states = t.first_scales ? 1 : 4;
  if ((uintptr_t)t.weight % size_of(t.weight_type) || (uintptr_t)t.grad % size_of(t.grad_type) || (uintptr_t)t.copy & 1u || (uintptr_t)t.first % states ||
      (uintptr_t)t.second % states || ((uintptr_t)t.first_scales | (uintptr_t)t.second_scales) & 3u)
    return fail(RADIAL_ESHAPE, "tensor %d: a pointer is not aligned to its elements", i);
  return RADIAL_OK;
}
int64_t pieces_of_tensor(const radial_adamw_tensor& t) { return (t.n + kPiece - 1) / kPiece; }

int check_plan(const radial_adamw_plan_info* plan, const void* table, size_t table_bytes) {
  if (!plan) return fail(RADIAL_EINVAL, "plan is NULL");
  if (plan->count < 1 || plan->pieces < 0 || plan->pieces > kMostPieces || plan->table_bytes != table_bytes_of(plan->count, plan->pieces))
    return fail(RADIAL_EINVAL, "plan is not one of radial_adamw_plan");
  if (!table || table_bytes < plan->table_bytes)
    return fail(RADIAL_EINVAL, "table is NULL or too small: %zu bytes needed, %zu given", plan->table_bytes, table ? table_bytes : (size_t)0);
  if ((uintptr_t)table & 15u) return fail(RADIAL_ESHAPE, "table is not 16-byte aligned");
  return RADIAL_OK;
}
int32_t norm_groups(int32_t pieces) { return pieces < 1 ? 1 : pieces < kNormGroups ? pieces : kNormGroups; }

}  // namespace
}  // namespace radial

using namespace radial;

extern "C" int radial_adamw_plan(const radial_adamw_tensor* tensors, int32_t count, radial_adamw_plan_info* plan) {
  if (!tensors || !plan) return fail(RADIAL_EINVAL, "tensors or plan is NULL");
  if (count < 1) return fail(RADIAL_EINVAL, "count must be >= 1");
  int64_t pieces = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (int rc = check_tensor(tensors[i], i)) return rc;
    pieces += pieces_of_tensor(tensors[i]);
    if (pieces > kMostPieces) return fail(RADIAL_ESHAPE, "more than 2^23 pieces of 4096 values are too many for one launch");
  }
  plan->count = count;
  plan->pieces = (int32_t)pieces;
  plan->table_bytes = table_bytes_of(count, pieces);
  return RADIAL_OK;
}

extern "C" int radial_adamw_table(const radial_adamw_tensor* tensors, const radial_adamw_plan_info* plan, void* table, size_t table_bytes, void* hip_stream) {
  if (!tensors) return fail(RADIAL_EINVAL, "tensors is NULL");
  if (int rc = check_plan(plan, table, table_bytes)) return rc;
  radial_adamw_plan_info of_tensors;
  if (int rc = radial_adamw_plan(tensors, plan->count, &of_tensors)) return rc;
  if (of_tensors.pieces != plan->pieces) return fail(RADIAL_EINVAL, "plan is not that of the tensors");
  int32_t piece = 0;
  for (int32_t first = 0; first < plan->count; first += kTensorsAtOnce) {
    const int32_t some = plan->count - first < kTensorsAtOnce ? plan->count - first : kTensorsAtOnce;
    TableArgs a = {};
    a.table = table; a.count = plan->count; a.first = first;
    for (int32_t i = 0; i < some; ++i) {
      const radial_adamw_tensor& t = tensors[first + i];
      const int32_t kind = (t.weight_type == RADIAL_F32 ? kWeightF32 : 0) | (t.grad_type == RADIAL_F32 ? kGradF32 : 0) | (t.first_scales ? kCodes : 0);
      a.tensors[i] = Tensor{t.weight, (__bf16*)t.copy, t.grad, t.first, t.second, t.first_scales, t.second_scales, t.n, (float)t.decay, kind};
      a.piece0[i] = piece;
      piece += (int32_t)pieces_of_tensor(t);
    }
    write_table_kernel<<<dim3((unsigned)some), dim3(256), 0, (hipStream_t)hip_stream>>>(a);
    RADIAL_HIP_TRY(hipGetLastError());
  }
  return RADIAL_OK;
}

extern "C" size_t radial_grad_norm_workspace(const radial_adamw_plan_info* plan) {
  return !plan || plan->count < 1 || plan->pieces < 0 || plan->pieces > kMostPieces ? 0 : (size_t)norm_groups(plan->pieces) * sizeof(double);
}

extern "C" int radial_grad_norm(const radial_adamw_plan_info* plan, const void* table, size_t table_bytes, float scale, float max_norm, float* norm,
                                void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_plan(plan, table, table_bytes)) return rc;
  if (!(scale > 0.f && scale <= 3.4028234663852886e38f)) return fail(RADIAL_EINVAL, "scale must be > 0 and finite");
  if (!(max_norm > 0.f)) return fail(RADIAL_EINVAL, "max_norm must be > 0");
  if (!norm) return fail(RADIAL_EINVAL, "norm is NULL");
  if ((uintptr_t)norm & 3u) return fail(RADIAL_ESHAPE, "norm is not aligned to its elements");
  const size_t needed = radial_grad_norm_workspace(plan);
  if (!workspace || workspace_bytes < needed) return fail(RADIAL_EINVAL, "workspace is NULL or too small: %zu bytes needed, %zu given", needed, workspace ? workspace_bytes : (size_t)0);
  if ((uintptr_t)workspace & 7u) return fail(RADIAL_ESHAPE, "workspace is not 8-byte aligned");
  hipStream_t stream = (hipStream_t)hip_stream;
  const int32_t groups = norm_groups(plan->pieces);
  grad_squares_kernel<<<dim3((unsigned)groups), dim3(256), 0, stream>>>(table, plan->count, plan->pieces, (double*)workspace);
  RADIAL_HIP_TRY(hipGetLastError());
  finish_norm_kernel<<<dim3(1), dim3(256), 0, stream>>>((const double*)workspace, groups, scale, max_norm, norm);
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}

extern "C" int radial_adamw_step(const radial_adamw_params* params, const radial_adamw_plan_info* plan, const void* table, size_t table_bytes,
                                 void* hip_stream) {
  if (!params) return fail(RADIAL_EINVAL, "params is NULL");
  const radial_adamw_params& p = *params;
  constexpr double kMost = 3.4028234663852886e38;
  if (!(p.lr >= 0.0 && p.lr <= kMost)) return fail(RADIAL_EINVAL, "lr must be >= 0 and finite");
  if (!(p.beta1 >= 0.0 && p.beta1 < 1.0) || !(p.beta2 >= 0.0 && p.beta2 < 1.0)) return fail(RADIAL_EINVAL, "beta1 and beta2 must be >= 0 and below 1");
  if (!((float)p.eps >= 1.17549435e-38f && p.eps <= kMost)) return fail(RADIAL_EINVAL, "eps must be a normal positive number of float32");
  if (p.step < 1 && !p.step_at) return fail(RADIAL_EINVAL, "step must be >= 1");
  if (p.rounding != RADIAL_ROUND_NEAREST && p.rounding != RADIAL_ROUND_RANDOM)
    return fail(RADIAL_EINVAL, "rounding must be RADIAL_ROUND_NEAREST or RADIAL_ROUND_RANDOM (got %d)", p.rounding);
  if (((uintptr_t)p.factor | (uintptr_t)p.lr_at) & 3u || (uintptr_t)p.step_at & 7u) return fail(RADIAL_ESHAPE, "factor, lr_at or step_at is not aligned to its element");
  if (int rc = check_plan(plan, table, table_bytes)) return rc;
  if (!plan->pieces) return RADIAL_OK;
  const double step = (double)(p.step < 1 ? 1 : p.step);
  StepArgs a = {};
  a.table = table; a.count = plan->count;
  a.lr = (float)p.lr; a.lr_wide = p.lr; a.eps = (float)p.eps;
  a.beta1 = (float)p.beta1; a.of_grad1 = (float)(1.0 - p.beta1);
  a.beta2 = (float)p.beta2; a.of_grad2 = (float)(1.0 - p.beta2);
  a.by_first = (float)(p.lr / (1.0 - pow(p.beta1, step)));
  a.by_second = (float)(1.0 / sqrt(1.0 - pow(p.beta2, step)));
  a.log_beta1 = p.beta1 > 0.0 ? (float)log(p.beta1) : 0.f;
  a.log_beta2 = p.beta2 > 0.0 ? (float)log(p.beta2) : 0.f;
  a.step = p.step; a.seed = p.seed; a.factor = p.factor; a.lr_at = p.lr_at; a.step_at = p.step_at;
  const dim3 grid((unsigned)plan->pieces), threads(256);
  if (p.rounding == RADIAL_ROUND_RANDOM) adamw_step_kernel<true><<<grid, threads, 0, (hipStream_t)hip_stream>>>(a);
  else adamw_step_kernel<false><<<grid, threads, 0, (hipStream_t)hip_stream>>>(a);
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}
