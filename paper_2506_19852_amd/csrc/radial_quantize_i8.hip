// Codes of 8-bit integers for gfx950: a matrix with one float32 scale for each row, by rows, and by columns as the rows of its transpose.
#include <math.h>

#include "radial_layer_common.h"
#include "radial_product_i8.h"

namespace radial {
namespace {

constexpr float kLargest = 127.f;
constexpr float kSmallestScale = 1.17549435e-38f;  // 2^-126
constexpr uint32_t kInfinity = 0x7f800000u;

struct QuantArgs {
  const void* x;
  int64_t stride;
  int32_t rows, cols;
  int32_t row_tiles, col_tiles;  // of 128
  int8_t *codes, *codes_t;
  float *scales, *scales_t, *sums_t;
  int32_t accumulate;
  int32_t slabs;           // parts of the rows whose columns are looked over by themselves
  uint32_t* largest;       // [slabs, cols]: bits of the largest magnitude
  float* sums;             // [slabs, cols]
};

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
  __device__ __forceinline__ explicit Code(uint32_t largest) {
    const float amax = __builtin_bit_cast(float, largest);
    scale = largest < kInfinity ? fmaxf(amax / kLargest, kSmallestScale) : __builtin_nanf("");
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

// Codes along the rows: a wave takes a row, a lane eight columns of every 512.  kPieces pieces of 512 stay in registers between the largest magnitude
// and the codes; longer rows (kPieces 0) are read twice.
template <class T, int kPieces>
__global__ void __launch_bounds__(256) quantize_rows_i8_kernel(QuantArgs a) {
  const int32_t lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.rows) return;
  const T* x = (const T*)a.x + row * a.stride;
  const int32_t padded = a.col_tiles * kCodeGroup;
  int8_t* codes = a.codes + (int64_t)row * padded;
  constexpr int kHeld = kPieces ? kPieces : 1;
  Eight<T> held[kHeld];
  uint32_t largest = 0;
  auto look = [&](const Eight<T>& e) __attribute__((always_inline)) {
    float v[8];
    e.get(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(v[i]));
  };
  if constexpr (kPieces > 0) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const int32_t c = p * 512 + lane * 8;
      held[p].load_some(x + c, a.cols - c);
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p) look(held[p]);
  } else {
    for (int32_t c = lane * 8; c < a.cols; c += 512) {
      held[0].load_some(x + c, a.cols - c);
      look(held[0]);
    }
  }
  const Code code(wave_max(largest));
  auto put = [&](const Eight<T>& e, int32_t c) __attribute__((always_inline)) {
    float v[8];
    e.get(v);
    if (c < padded) *(u32x2*)(codes + c) = u32x2{code.four(v[0], v[1], v[2], v[3]), code.four(v[4], v[5], v[6], v[7])};
  };
  if constexpr (kPieces > 0) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) put(held[p], p * 512 + lane * 8);
  } else {
    for (int32_t c = lane * 8; c < padded; c += 512) {
      held[0].load_some(x + c, a.cols - c);
      put(held[0], c);
    }
  }
  if (lane == 0) a.scales[row] = code.scale;
}

// Largest magnitudes and sums of the columns of a slab of rows: a wave takes every fourth row, a lane eight of 512 columns.
template <class T>
__global__ void __launch_bounds__(256) look_over_columns_kernel(QuantArgs a) {
  __shared__ uint32_t of_wave[4][512];
  __shared__ float sum_of_wave[4][512];
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t tiles = (a.cols + 511) / 512, slab = blockIdx.x / tiles, c = blockIdx.x % tiles * 512 + lane * 8;
  const int32_t first = (int32_t)((int64_t)a.rows * slab / a.slabs), last = (int32_t)((int64_t)a.rows * (slab + 1) / a.slabs);
  uint32_t largest[8] = {};
  float sum[8] = {};
  const T* x = (const T*)a.x + c;
  for (int32_t r = first + wave; r < last; r += 16) {
    Eight<T> e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int32_t row = r + 4 * i;
      e[i].load_some(x + (int64_t)min(row, last - 1) * a.stride, row < last ? a.cols - c : 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[8];
      e[i].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        largest[j] = max(largest[j], magnitude(v[j]));
        sum[j] += v[j];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    of_wave[wave][lane * 8 + j] = largest[j];
    sum_of_wave[wave][lane * 8 + j] = sum[j];
  }
  __syncthreads();
  const int32_t c0 = blockIdx.x % tiles * 512;
  for (int32_t i = threadIdx.x; i < 512 && c0 + i < a.cols; i += 256) {
    const int64_t at = (int64_t)slab * a.cols + c0 + i;
    a.largest[at] = max(max(of_wave[0][i], of_wave[1][i]), max(of_wave[2][i], of_wave[3][i]));
    a.sums[at] = (sum_of_wave[0][i] + sum_of_wave[1][i]) + (sum_of_wave[2][i] + sum_of_wave[3][i]);
  }
}

// The slabs' magnitudes and sums put together: scales of the transpose's rows, sums of the columns.
__global__ void __launch_bounds__(256) join_slabs_kernel(QuantArgs a) {
  __shared__ uint32_t largest_of[4][64];
  __shared__ float sum_of[4][64];
  const int32_t lane = threadIdx.x & 63, part = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  uint32_t largest = 0;
  float sum = 0.f;
  for (int32_t s = part; s < a.slabs && c < a.cols; s += 4) {
    largest = max(largest, a.largest[(int64_t)s * a.cols + c]);
    sum += a.sums[(int64_t)s * a.cols + c];
  }
  largest_of[part][lane] = largest;
  sum_of[part][lane] = sum;
  __syncthreads();
  if (part || c >= a.cols) return;
  const Code code(max(max(largest_of[0][lane], largest_of[1][lane]), max(largest_of[2][lane], largest_of[3][lane])));
  if (a.scales_t) a.scales_t[c] = code.scale;
  if (a.sums_t) {
    const float all = (sum_of[0][lane] + sum_of[1][lane]) + (sum_of[2][lane] + sum_of[3][lane]);
    a.sums_t[c] = a.accumulate ? a.sums_t[c] + all : all;
  }
}

// Codes along the columns, by tiles of 128 x 128: a thread holds eight rows of eight columns; its codes pass through LDS in pieces of eight rows, exchanged by
// column so that the pieces of one write lie in different banks.
template <class T>
__global__ void __launch_bounds__(256) quantize_columns_i8_kernel(QuantArgs a) {
  __shared__ __align__(16) u32x2 turned[kCodeGroup * 16];
  const int32_t row0 = blockIdx.x / a.col_tiles * kCodeGroup, col0 = blockIdx.x % a.col_tiles * kCodeGroup;
  const int32_t tr = threadIdx.x >> 4, tc = threadIdx.x & 15;
  const int32_t r0 = row0 + tr * 8, c0 = col0 + tc * 8;
  float v[8][8];
  {
    Eight<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      raw[i].load_some((const T*)a.x + (int64_t)min(r0 + i, a.rows - 1) * a.stride + c0, r0 + i < a.rows ? a.cols - c0 : 0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i].get(v[i]);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int32_t c = tc * 8 + j;
    const float scale = a.scales_t[min(col0 + c, a.cols - 1)];
    Code code(0);
    code.scale = scale;
    code.inverse = 1.f / scale;
    turned[c * 16 + (tr ^ tc)] = u32x2{code.four(v[0][j], v[1][j], v[2][j], v[3][j]), code.four(v[4][j], v[5][j], v[6][j], v[7][j])};
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int32_t c = i * 32 + (threadIdx.x >> 3), piece = threadIdx.x & 7;
    const u32x2 lo = turned[c * 16 + ((2 * piece) ^ (c >> 3))], hi = turned[c * 16 + ((2 * piece + 1) ^ (c >> 3))];
    if (col0 + c < a.cols) *(u32x4*)(a.codes_t + ((int64_t)(col0 + c) * a.row_tiles + row0 / kCodeGroup) * kCodeGroup + piece * 16) = u32x4{lo[0], lo[1], hi[0], hi[1]};
  }
}

// Slabs of the rows: workgroups of 512 columns that fill the chip twice over, of 16 rows at least.
inline int32_t slabs_of(int32_t rows, int32_t cols) {
  const int64_t tiles = ((int64_t)cols + 511) / 512, most = ((int64_t)rows + 15) / 16;
  const int64_t wanted = (1024 + tiles - 1) / tiles;
  return (int32_t)(wanted < most ? wanted : most);
}

template <class T>
int launch_quantize(const QuantArgs& a, hipStream_t stream) {
  const dim3 threads(256);
  const int64_t tiles = (int64_t)a.row_tiles * a.col_tiles;
  if (tiles > kMostThreads / 256) return fail(RADIAL_ESHAPE, "x is too large for one launch");
  if (a.codes) {
    if (((int64_t)a.rows + 3) / 4 > kMostThreads / 256) return fail(RADIAL_ESHAPE, "x is too large for one launch");
    const dim3 grid((unsigned)(((int64_t)a.rows + 3) / 4));
    const int64_t pieces = ((int64_t)a.col_tiles * kCodeGroup + 511) / 512;
    if (pieces <= 1) quantize_rows_i8_kernel<T, 1><<<grid, threads, 0, stream>>>(a);
    else if (pieces <= 2) quantize_rows_i8_kernel<T, 2><<<grid, threads, 0, stream>>>(a);
    else if (pieces <= 4) quantize_rows_i8_kernel<T, 4><<<grid, threads, 0, stream>>>(a);
    else if (pieces <= 6) quantize_rows_i8_kernel<T, 6><<<grid, threads, 0, stream>>>(a);
    else if (pieces <= 10) quantize_rows_i8_kernel<T, 10><<<grid, threads, 0, stream>>>(a);
    else if (pieces <= 16) quantize_rows_i8_kernel<T, 16><<<grid, threads, 0, stream>>>(a);
    else quantize_rows_i8_kernel<T, 0><<<grid, threads, 0, stream>>>(a);
    RADIAL_HIP_TRY(hipGetLastError());
  }
  if (a.codes_t || a.sums_t) {
    look_over_columns_kernel<T><<<dim3((unsigned)((((int64_t)a.cols + 511) / 512) * a.slabs)), threads, 0, stream>>>(a);
    RADIAL_HIP_TRY(hipGetLastError());
    join_slabs_kernel<<<dim3((unsigned)(((int64_t)a.cols + 63) / 64)), threads, 0, stream>>>(a);
    RADIAL_HIP_TRY(hipGetLastError());
  }
  if (a.codes_t) {
    quantize_columns_i8_kernel<T><<<dim3((unsigned)tiles), threads, 0, stream>>>(a);
    RADIAL_HIP_TRY(hipGetLastError());
  }
  return RADIAL_OK;
}

}  // namespace

size_t quantize_i8_workspace(int32_t rows, int32_t cols) { return (size_t)slabs_of(rows, cols) * cols * 8; }

int quantize_i8(int32_t rows, int32_t cols, const void* x, int32_t type, int64_t stride, int8_t* codes, float* scales, int8_t* codes_t, float* scales_t,
                float* sums_t, bool accumulate, void* workspace, hipStream_t stream) {
  QuantArgs a = {};
  a.x = x; a.stride = stride; a.rows = rows; a.cols = cols;
  a.codes = codes; a.scales = scales; a.codes_t = codes_t; a.scales_t = scales_t; a.sums_t = sums_t; a.accumulate = accumulate;
  a.row_tiles = (int32_t)code_groups(rows);
  a.col_tiles = (int32_t)code_groups(cols);
  a.slabs = slabs_of(rows, cols);
  a.largest = (uint32_t*)workspace;
  a.sums = (float*)workspace + (int64_t)a.slabs * cols;
  return type == RADIAL_F32 ? launch_quantize<float>(a, stream) : launch_quantize<__bf16>(a, stream);
}

}  // namespace radial

using namespace radial;

extern "C" size_t radial_quantize_rows_i8_workspace(int32_t rows, int32_t cols) {
  return rows < 1 || cols < 1 || rows > kMostCodeRows || cols > kMostCodeRows ? 0 : quantize_i8_workspace(rows, cols);
}

extern "C" int radial_quantize_rows_i8(int32_t rows, int32_t cols, const void* x, int32_t type, int64_t stride, int8_t* codes, float* scales,
                                       int8_t* codes_t, float* scales_t, float* sums_t, int32_t accumulate, void* workspace, size_t workspace_bytes,
                                       void* hip_stream) {
  if (rows < 1 || cols < 1) return fail(RADIAL_EINVAL, "rows and cols must be >= 1");
  if (!x) return fail(RADIAL_EINVAL, "x is NULL");
  if (!is_type(type)) return fail(RADIAL_EINVAL, "type must be RADIAL_BF16 or RADIAL_F32 (got %d)", type);
  if (!codes != !scales || !codes_t != !scales_t) return fail(RADIAL_EINVAL, "codes and scales go together");
  if (!codes && !codes_t && !sums_t) return fail(RADIAL_EINVAL, "none of codes, codes_t and sums_t is given");
  if (rows > kMostCodeRows || cols > kMostCodeRows) return fail(RADIAL_ESHAPE, "rows and cols must be at most 2^29: x is too large for one launch");
  if (int rc = check_matrix(x, type, stride, cols, "x")) return rc;
  if (((uintptr_t)codes | (uintptr_t)codes_t) & 15u) return fail(RADIAL_ESHAPE, "codes are not 16-byte aligned");
  if (((uintptr_t)scales | (uintptr_t)scales_t | (uintptr_t)sums_t) & 3u) return fail(RADIAL_ESHAPE, "scales or sums_t are not aligned to their elements");
  if (codes_t || sums_t) {
    if (int rc = check_workspace(workspace, workspace_bytes, quantize_i8_workspace(rows, cols))) return rc;
  }
  return quantize_i8(rows, cols, x, type, stride, codes, scales, codes_t, scales_t, sums_t, accumulate != 0, workspace, (hipStream_t)hip_stream);
}
