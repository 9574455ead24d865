// Codes of 8-bit integers for gfx950: a matrix with one float32 scale for each row, by rows, and by columns as the rows of its transpose.  Bound by memory: a row's scale needs all of
// the row, which stays in registers (32 760 x 5120 in bf16 91 us, 5.5 TB/s); a column's needs all of the column, so that columns take two passes over the matrix, the second
// from the last-level cache as far as it goes (14 040 x 5120: columns 60 us, rows and columns 79; 5120 x 5120 28 and 39).  Within the gradients of a projection of that size the two
// passes over both matrices take some 190 us, the first from a cold cache.
#include <math.h>

#include "radial_layer_common.h"
#include "radial_product_i8.h"

namespace radial {
namespace {

// One matrix and what is wanted of it.  Columns need two passes over it: one for the largest magnitudes, one for the codes.
struct Job {
  const void* x;
  int64_t stride;
  int32_t rows, cols;
  int32_t row_tiles, col_tiles;       // of 128
  int8_t *codes, *codes_t;
  int64_t pitch, pitch_t;             // bytes from a row of codes to the next
  float *scales, *scales_t, *sums_t;
  int32_t accumulate;
  int32_t wide_tiles, slabs, strips;  // the first pass: 512 columns x a slab of the rows; the second: 128 columns x a strip of the row tiles
  uint32_t* of_rows;                  // [wide_tiles, rows]: bits of the largest magnitude of a row's 512 columns
  uint32_t* of_cols;                  // [slabs, cols]: of a column's rows of a slab
  float* sums;                        // [slabs, cols]
};
struct Jobs {
  Job job[2];
  int32_t first_of_second;  // workgroup
};

// Codes along the rows: kTeam waves take a row, a lane eight columns of every 512 kTeam.  kPieces pieces stay in registers between the largest magnitude
// and the codes; longer rows (kPieces 0) are read twice.  Few rows take four waves each (512 x 4096: 4.5 us, with one 5.2).
template <class T, int kPieces, int kTeam>
__global__ void __launch_bounds__(256) quantize_rows_i8_kernel(Job a) {
  __shared__ uint32_t of_wave[4];
  constexpr int kStep = 512 * kTeam;
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = kTeam == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= a.rows) return;  // kTeam 4: there is a row for each workgroup
  const int32_t at = lane * 8 + (kTeam == 1 ? 0 : wave * 512);
  const T* x = (const T*)a.x + row * a.stride;
  const int32_t padded = a.col_tiles * kCodeGroup;
  int8_t* codes = a.codes + row * a.pitch;
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
      const int32_t c = p * kStep + at;
      held[p].load_some(x + c, a.cols - c);
    }
#pragma unroll
    for (int p = 0; p < kPieces; ++p) look(held[p]);
  } else {
    for (int32_t c = at; c < a.cols; c += kStep) {
      held[0].load_some(x + c, a.cols - c);
      look(held[0]);
    }
  }
  largest = wave_max(largest);
  if constexpr (kTeam > 1) {
    if (lane == 0) of_wave[wave] = largest;
    __syncthreads();
    largest = max(max(of_wave[0], of_wave[1]), max(of_wave[2], of_wave[3]));
  }
  const Code code(largest);
  auto put = [&](const Eight<T>& e, int32_t c) __attribute__((always_inline)) {
    float v[8];
    e.get(v);
    if (c < padded) *(u32x2*)(codes + c) = u32x2{code.four(v[0], v[1], v[2], v[3]), code.four(v[4], v[5], v[6], v[7])};
  };
  if constexpr (kPieces > 0) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) put(held[p], p * kStep + at);
  } else {
    for (int32_t c = at; c < padded; c += kStep) {
      held[0].load_some(x + c, a.cols - c);
      put(held[0], c);
    }
  }
  if (lane == 0 && (kTeam == 1 || wave == 0)) a.scales[row] = code.scale;
}

// First pass: largest magnitudes and sums of the columns of a slab of rows, and of each row of the 512 columns, where they are wanted: a wave takes every fourth row, a
// lane eight columns.
constexpr int kLookWaves = 4, kAtOnce = 8;  // waves of a workgroup, rows of a wave under way
template <class T>
__global__ void __launch_bounds__(64 * kLookWaves) look_over_kernel(Jobs jobs) {
  __shared__ uint32_t of_wave[kLookWaves][512];
  __shared__ float sum_of_wave[kLookWaves][512];
  const bool second = (int32_t)blockIdx.x >= jobs.first_of_second;
  const Job& a = jobs.job[second];
  const int32_t id = blockIdx.x - (second ? jobs.first_of_second : 0);
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t slab = id / a.wide_tiles, tile = id % a.wide_tiles, c = tile * 512 + lane * 8;
  const int32_t first = (int32_t)((int64_t)a.rows * slab / a.slabs), last = (int32_t)((int64_t)a.rows * (slab + 1) / a.slabs);
  uint32_t largest[8] = {};
  float sum[8] = {};
  const T* x = (const T*)a.x + c;
  for (int32_t r = first + wave; r < last; r += kLookWaves * kAtOnce) {
    Eight<T> e[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int32_t row = r + kLookWaves * i;
      e[i].load_some(x + (int64_t)min(row, last - 1) * a.stride, row < last ? a.cols - c : 0);
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      float v[8];
      e[i].get(v);
      uint32_t of_row = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t m = magnitude(v[j]);
        largest[j] = max(largest[j], m);
        of_row = max(of_row, m);
        sum[j] += v[j];
      }
      if (a.codes) {
        const int32_t row = r + kLookWaves * i;
        of_row = wave_max(of_row);
        if (lane == 0 && row < last) a.of_rows[(int64_t)tile * a.rows + row] = of_row;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    of_wave[wave][lane * 8 + j] = largest[j];
    sum_of_wave[wave][lane * 8 + j] = sum[j];
  }
  __syncthreads();
  for (int32_t i = threadIdx.x; i < 512 && tile * 512 + i < a.cols; i += 64 * kLookWaves) {
    const int64_t at = (int64_t)slab * a.cols + tile * 512 + i;
    uint32_t all = 0;
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kLookWaves; ++w) {
      all = max(all, of_wave[w][i]);
      total += sum_of_wave[w][i];
    }
    a.of_cols[at] = all;
    if (a.sums_t) a.sums[at] = total;
  }
}

// The largest of `count` values `step` apart, eight asked for at a time (the last one again behind the end).
__device__ __forceinline__ uint32_t largest_of(const uint32_t* p, int64_t step, int32_t count) {
  uint32_t largest = 0;
  for (int32_t i = 0; i < count; i += 8) {
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = p[min(i + j, count - 1) * step];
#pragma unroll
    for (int j = 0; j < 8; ++j) largest = max(largest, v[j]);
  }
  return largest;
}
// The sum of a column over every `step`th slab from `first` on, in order, eight asked for at a time.
__device__ __forceinline__ float sum_of(const Job& a, int32_t c, int32_t first, int32_t step) {
  float all = 0.f;
  for (int32_t s = first; s < a.slabs; s += 8 * step) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = a.sums[(int64_t)min(s + j * step, a.slabs - 1) * a.cols + c];
#pragma unroll
    for (int j = 0; j < 8; ++j) all += s + j * step < a.slabs ? v[j] : 0.f;
  }
  return all;
}
__device__ __forceinline__ void put_sum(const Job& a, int32_t c, float sum) { a.sums_t[c] = a.accumulate ? a.sums_t[c] + sum : sum; }
__global__ void __launch_bounds__(64) put_sums_kernel(Job a) {
  const int32_t c = blockIdx.x * 64 + threadIdx.x;
  if (c < a.cols) put_sum(a, c, sum_of(a, c, 0, 1));
}

// Second pass, by tiles of 128 x 128, a strip of them one below the other for each workgroup: the largest magnitudes of its rows and columns are put together, then a
// thread holds eight rows of eight columns.  Codes along the rows go out as they are; those of the transpose pass through LDS in pieces of eight rows, exchanged by
// column so that the pieces of one write lie in different banks.
template <class T>
__global__ void __launch_bounds__(256) quantize_tiles_i8_kernel(Jobs jobs) {
  __shared__ __align__(16) u32x2 turned[kCodeGroup * 16];
  __shared__ uint32_t half[2][kCodeGroup];
  __shared__ float half_sum[2][kCodeGroup];
  __shared__ Code of_col[kCodeGroup], of_row[kCodeGroup];
  const bool second = (int32_t)blockIdx.x >= jobs.first_of_second;
  const Job& a = jobs.job[second];
  const int32_t id = blockIdx.x - (second ? jobs.first_of_second : 0);
  const int32_t col0 = id % a.col_tiles * kCodeGroup, strip = id / a.col_tiles;
  const int32_t first = (int32_t)((int64_t)a.row_tiles * strip / a.strips), last = (int32_t)((int64_t)a.row_tiles * (strip + 1) / a.strips);
  const int32_t tr = threadIdx.x >> 4, tc = threadIdx.x & 15, c0 = col0 + tc * 8;
  {
    const int32_t c = threadIdx.x & 127, part = threadIdx.x >> 7;
    const bool sums = a.sums_t && strip == 0 && col0 + c < a.cols;
    if (sums) half_sum[part][c] = sum_of(a, col0 + c, part, 2);
    half[part][c] = col0 + c < a.cols ? largest_of(a.of_cols + (int64_t)part * a.cols + col0 + c, 2 * (int64_t)a.cols, (a.slabs + 1 - part) / 2) : 0u;
    __syncthreads();
    if (part == 0) {
      const Code code(max(half[0][c], half[1][c]));
      of_col[c] = code;
      if (strip == 0 && col0 + c < a.cols) {
        a.scales_t[col0 + c] = code.scale;
        if (sums) put_sum(a, col0 + c, half_sum[0][c] + half_sum[1][c]);
      }
    }
    __syncthreads();
  }
  Code mine[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) mine[j] = of_col[tc * 8 + j];
  for (int32_t tile = first; tile < last; ++tile) {
    const int32_t row0 = tile * kCodeGroup, r0 = row0 + tr * 8;
    float v[8][8];
    {
      Eight<T> raw[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) raw[i].load_some((const T*)a.x + (int64_t)min(r0 + i, a.rows - 1) * a.stride + c0, r0 + i < a.rows ? a.cols - c0 : 0);
#pragma unroll
      for (int i = 0; i < 8; ++i) raw[i].get(v[i]);
    }
    if (a.codes) {
      if (threadIdx.x < kCodeGroup) {
        const uint32_t largest = row0 + (int32_t)threadIdx.x < a.rows ? largest_of(a.of_rows + row0 + threadIdx.x, a.rows, a.wide_tiles) : 0u;
        const Code code(largest);
        of_row[threadIdx.x] = code;
        if (col0 == 0 && row0 + (int32_t)threadIdx.x < a.rows) a.scales[row0 + threadIdx.x] = code.scale;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Code code = of_row[tr * 8 + i];
        if (r0 + i < a.rows)
          *(u32x2*)(a.codes + (int64_t)(r0 + i) * a.pitch + c0) = u32x2{code.four(v[i][0], v[i][1], v[i][2], v[i][3]), code.four(v[i][4], v[i][5], v[i][6], v[i][7])};
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const Code& code = mine[j];
      turned[(tc * 8 + j) * 16 + (tr ^ tc)] = u32x2{code.four(v[0][j], v[1][j], v[2][j], v[3][j]), code.four(v[4][j], v[5][j], v[6][j], v[7][j])};
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int32_t c = i * 32 + (threadIdx.x >> 3), piece = threadIdx.x & 7;
      const u32x2 lo = turned[c * 16 + ((2 * piece) ^ (c >> 3))], hi = turned[c * 16 + ((2 * piece + 1) ^ (c >> 3))];
      if (col0 + c < a.cols) *(u32x4*)(a.codes_t + (int64_t)(col0 + c) * a.pitch_t + row0 + piece * 16) = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    __syncthreads();
  }
}

inline int32_t at_most(int64_t wanted, int64_t most) { return (int32_t)(wanted < most ? wanted : most); }
// Slabs of the first pass: up to two workgroups for each compute unit, of 32 rows at least (the second pass reads a value of each slab).  (14 040 x 5120: 520 workgroups, eight too many,
// cost 4 us; three for each are alike.)
inline int32_t slabs_of(int32_t rows, int32_t cols) {
  const int64_t tiles = ((int64_t)cols + 511) / 512;
  return at_most(tiles < 512 ? 512 / tiles : 1, ((int64_t)rows + 31) / 32);
}
// Strips of the second: up to three workgroups for each compute unit, which all fit at once, as long as there are tiles.  (14 040 x 5120: columns 64 us, with both orientations 84;
// with 1040 workgroups, one round and a third, 67 and 90; 32 760 x 5120 both 228 and 251.)
inline int32_t strips_of(int32_t rows, int32_t cols) { return at_most(code_groups(cols) < 768 ? 768 / code_groups(cols) : 1, code_groups(rows)); }

template <class T>
int launch_rows(const Job& a, hipStream_t stream) {
  const bool few = a.rows <= 2048;  // two rounds of four waves a row on the chip's compute units
  const int64_t groups = few ? a.rows : ((int64_t)a.rows + 3) / 4;
  if (groups > kMostThreads / 256) return fail(RADIAL_ESHAPE, "x is too large for one launch");
  const dim3 grid((unsigned)groups), threads(256);
  const int64_t pieces = ((int64_t)a.col_tiles * kCodeGroup + (few ? 2047 : 511)) / (few ? 2048 : 512);
  if (few) {
    if (pieces <= 1) quantize_rows_i8_kernel<T, 1, 4><<<grid, threads, 0, stream>>>(a);
    else if (pieces <= 3) quantize_rows_i8_kernel<T, 3, 4><<<grid, threads, 0, stream>>>(a);
    else quantize_rows_i8_kernel<T, 0, 4><<<grid, threads, 0, stream>>>(a);
  } else if (pieces <= 2) {
    quantize_rows_i8_kernel<T, 2, 1><<<grid, threads, 0, stream>>>(a);
  } else if (pieces <= 4) {
    quantize_rows_i8_kernel<T, 4, 1><<<grid, threads, 0, stream>>>(a);
  } else if (pieces <= 6) {
    quantize_rows_i8_kernel<T, 6, 1><<<grid, threads, 0, stream>>>(a);
  } else if (pieces <= 10) {
    quantize_rows_i8_kernel<T, 10, 1><<<grid, threads, 0, stream>>>(a);
  } else if (pieces <= 16) {
    quantize_rows_i8_kernel<T, 16, 1><<<grid, threads, 0, stream>>>(a);
  } else {
    quantize_rows_i8_kernel<T, 0, 1><<<grid, threads, 0, stream>>>(a);
  }
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}

// One or two matrices whose columns are wanted, in two launches.
template <class T>
int launch_passes(const Job* job, int count, hipStream_t stream) {
  Jobs jobs = {};
  int64_t looks = 0, tiles = 0;
  for (int i = 0; i < count; ++i) {
    jobs.job[i] = job[i];
    if (i == 1) jobs.first_of_second = (int32_t)looks;
    looks += (int64_t)job[i].wide_tiles * job[i].slabs;
  }
  if (count == 1) jobs.first_of_second = 0x7fffffff;
  if (looks > kMostThreads / (64 * kLookWaves)) return fail(RADIAL_ESHAPE, "x is too large for one launch");
  for (int i = 0; i < count; ++i) tiles += (int64_t)job[i].col_tiles * job[i].strips;
  if (tiles > kMostThreads / 256) return fail(RADIAL_ESHAPE, "x is too large for one launch");
  look_over_kernel<T><<<dim3((unsigned)looks), dim3(64 * kLookWaves), 0, stream>>>(jobs);
  RADIAL_HIP_TRY(hipGetLastError());
  if (!job[0].codes_t) {
    put_sums_kernel<<<dim3((unsigned)(((int64_t)job[0].cols + 63) / 64)), dim3(64), 0, stream>>>(job[0]);
  } else {
    if (count == 2) jobs.first_of_second = job[0].col_tiles * job[0].strips;
    quantize_tiles_i8_kernel<T><<<dim3((unsigned)tiles), dim3(256), 0, stream>>>(jobs);
  }
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}

Job job_of(const QuantI8& q, char* workspace) {
  Job a = {};
  a.x = q.x; a.stride = q.stride; a.rows = q.rows; a.cols = q.cols;
  a.codes = q.codes; a.scales = q.scales; a.codes_t = q.codes_t; a.scales_t = q.scales_t; a.sums_t = q.sums_t; a.accumulate = q.accumulate;
  a.row_tiles = (int32_t)code_groups(q.rows);
  a.col_tiles = (int32_t)code_groups(q.cols);
  a.pitch = q.pitch ? q.pitch : (int64_t)a.col_tiles * kCodeGroup;
  a.pitch_t = q.pitch_t ? q.pitch_t : (int64_t)a.row_tiles * kCodeGroup;
  a.wide_tiles = (int32_t)(((int64_t)q.cols + 511) / 512);
  a.slabs = slabs_of(q.rows, q.cols);
  a.strips = strips_of(q.rows, q.cols);
  a.of_cols = (uint32_t*)workspace;
  a.sums = (float*)(a.of_cols + (int64_t)a.slabs * q.cols);
  a.of_rows = (uint32_t*)(a.sums + (int64_t)a.slabs * q.cols);
  return a;
}

// Two matrices share their launches up to this many bytes.  Beyond, each goes through both passes before the next, so that the second pass finds what the first has
// read in the last-level cache: two of 14 040 x 5120 in bf16 168 us, in shared launches 180 (both as first built); 1001 x 333 and 1001 x 2049 24 us, one after the other 33.
constexpr int64_t kShared = 128LL << 20;

template <class T>
int quantize(const QuantI8* q, int count, char* const* workspace, hipStream_t stream) {
  Job job[2];
  int64_t bytes = 0;
  for (int i = 0; i < count; ++i) {
    job[i] = job_of(q[i], workspace[i]);
    bytes += (int64_t)q[i].rows * q[i].cols * (int64_t)sizeof(T);
  }
  // codes along the rows come with the transpose's in its second pass, which holds the values anyway; without a transpose in one launch of their own
  Job& a = job[0];
  if (a.codes && !a.codes_t) {
    if (int rc = launch_rows<T>(a, stream)) return rc;
    a.codes = nullptr;
  }
  if (!a.codes_t && !a.sums_t) return RADIAL_OK;
  if (bytes <= kShared) return launch_passes<T>(job, count, stream);
  for (int i = 0; i < count; ++i) {
    if (int rc = launch_passes<T>(job + i, 1, stream)) return rc;
  }
  return RADIAL_OK;
}

}  // namespace

size_t quantize_i8_workspace(int32_t rows, int32_t cols) {
  return ((size_t)slabs_of(rows, cols) * cols * 2 + (size_t)(((int64_t)cols + 511) / 512) * rows) * 4;
}

int quantize_i8(const QuantI8* q, int count, int32_t type, char* const* workspace, hipStream_t stream) {
  return type == RADIAL_F32 ? quantize<float>(q, count, workspace, stream) : quantize<__bf16>(q, count, workspace, stream);
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
  QuantI8 q = {};
  q.x = x; q.stride = stride; q.rows = rows; q.cols = cols; q.codes = codes; q.scales = scales; q.codes_t = codes_t; q.scales_t = scales_t;
  q.sums_t = sums_t; q.accumulate = accumulate != 0;
  char* parts[1] = {(char*)workspace};
  return quantize_i8(&q, 1, type, parts, (hipStream_t)hip_stream);
}
