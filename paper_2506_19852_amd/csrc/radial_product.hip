// 8-bit products for gfx950: matrices as E4M3 codes with a float32 scale for each 128 columns of a row, or for each block of 128 x 128, made by
// quantize_groups_kernel, and their product
//     C[m, n] = sum over groups g of  sa[g, m] sb[g, n] (A_g[m, :] . B_g[n, :]).
// One group is the depth of one v_mfma_f32_16x16x128_f8f6f4, so a group's sum comes out of the matrix pipe whole and is scaled in float32.
// The tile is computed transposed (matrix A operand = rows of B, B operand = rows of A): a lane then holds one row m of C and four
// neighbouring columns n, so that sa is one value per lane and with blocks sa sb is one factor for all of a lane's sums.
#include <math.h>

#include <type_traits>

#include "radial_layer_common.h"
#include "radial_product_rule.h"

namespace radial {
namespace {

constexpr int kGroup = 128;
constexpr float kLargest = 448.f;                  // of E4M3
constexpr float kSmallestScale = 1.17549435e-38f;  // 2^-126

// ---- codes and scales -----------------------------------------------------------------------------

struct QuantArgs {
  const void* x;
  int64_t stride;
  int32_t rows, cols;
  uint8_t *codes, *codes_t;
  float *scales, *scales_t;
  int32_t col_tiles, row_tiles;
};

// x / scale as float32: the product with the inverse, and what it leaves, once more; off by half a unit and 2^-46 of the value.  (A division
// proper takes some ten instructions.)  Infinite scales give NaN.
struct Quotient {
  float scale, inverse;
  __device__ __forceinline__ explicit Quotient(float amax) {
    scale = fmaxf(amax / kLargest, kSmallestScale);
    inverse = 1.f / scale;
  }
  __device__ __forceinline__ float operator()(float x) const {
    const float q = x * inverse;
    return __builtin_fmaf(__builtin_fmaf(-q, scale, x), inverse, q);
  }
};

__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
  int v = 0;  // v_cvt_pk_fp8_f32 rounds to nearest even; no quotient rounds beyond 448
  v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, v, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  return (uint32_t)v;
}

// The bytes of eight codes that belong to the first `count`: beside an infinity the quotients of what lies behind the matrix are NaN, not zero.  Matrices of
// whole tiles (kWhole) do without (32 760 x 5120 by rows: 92.8 us, 97.8 with it, 14 040 x 5120 in both orientations 68.0, 68.9).
__device__ __forceinline__ u32x2 first_codes(int32_t count) {
  const uint32_t n[2] = {(uint32_t)max(0, min(count, 4)), (uint32_t)max(0, min(count - 4, 4))};
  return u32x2{n[0] == 4 ? ~0u : (1u << 8 * n[0]) - 1, n[1] == 4 ? ~0u : (1u << 8 * n[1]) - 1};
}

// One workgroup per 128 x 128 tile; a thread holds eight rows of eight columns.  Codes along the rows go out as they are (16 lanes, 128 bytes); those of the
// transpose pass through LDS in pieces of eight rows, exchanged by column so that the pieces of one write lie in different banks.
template <class T, bool kBlocks, bool kRows, bool kCols, bool kWhole>
__global__ void __launch_bounds__(256) quantize_groups_kernel(QuantArgs a) {
  __shared__ float wave_amax[4][kGroup];
  __shared__ __align__(16) u32x2 turned[kCols ? kGroup * 16 : 1];
  const int32_t row0 = blockIdx.x / a.col_tiles * kGroup, col0 = blockIdx.x % a.col_tiles * kGroup;
  const int32_t tr = threadIdx.x >> 4, tc = threadIdx.x & 15, wave = threadIdx.x >> 6;
  const int32_t r0 = row0 + tr * 8, c0 = col0 + tc * 8;
  float v[8][8];
  {
    Eight<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      raw[i].load_some((const T*)a.x + (int64_t)(r0 + i) * a.stride + c0, r0 + i < a.rows ? a.cols - c0 : 0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i].get(v[i]);
  }
  float of_row[8], of_col[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    of_row[i] = of_col[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      of_row[i] = fmaxf(of_row[i], fabsf(v[i][j]));
      of_col[i] = fmaxf(of_col[i], fabsf(v[j][i]));
    }
  }
  if constexpr (kBlocks || kRows) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      of_row[i] = max_dpp<kSwapOnes>(of_row[i]);
      of_row[i] = max_dpp<kSwapTwos>(of_row[i]);
      of_row[i] = max_dpp<kHalfRowMirror>(of_row[i]);
      of_row[i] = max_dpp<kRowMirror>(of_row[i]);
    }
  }
  if constexpr (kBlocks) {
    float amax = of_row[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) amax = fmaxf(amax, of_row[i]);
    if (tc == 0) wave_amax[0][tr] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) amax = fmaxf(amax, wave_amax[0][i]);
#pragma unroll
    for (int i = 0; i < 8; ++i) of_row[i] = of_col[i] = amax;
  } else if constexpr (kCols) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      of_col[i] = fmaxf(of_col[i], __shfl_xor(of_col[i], 16));
      of_col[i] = fmaxf(of_col[i], __shfl_xor(of_col[i], 32));
    }
    if ((threadIdx.x & 63) < 16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) wave_amax[wave][tc * 8 + i] = of_col[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i)
      of_col[i] = fmaxf(fmaxf(wave_amax[0][tc * 8 + i], wave_amax[1][tc * 8 + i]), fmaxf(wave_amax[2][tc * 8 + i], wave_amax[3][tc * 8 + i]));
  }

  const int32_t row_tile = row0 / kGroup, col_tile = col0 / kGroup;
  u32x2 along[8];  // codes of a row's eight columns (blocks: the transpose's codes are these)
  if constexpr (kRows) {
    const u32x2 of_matrix = kWhole ? u32x2{~0u, ~0u} : first_codes(a.cols - c0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Quotient q(of_row[i]);
      along[i] = u32x2{four_codes(q(v[i][0]), q(v[i][1]), q(v[i][2]), q(v[i][3])), four_codes(q(v[i][4]), q(v[i][5]), q(v[i][6]), q(v[i][7]))} & of_matrix;
      if (r0 + i < a.rows) {
        *(u32x2*)(a.codes + ((int64_t)(r0 + i) * a.col_tiles + col_tile) * kGroup + tc * 8) = along[i];
        if (!kBlocks && tc == 0) a.scales[(int64_t)col_tile * a.rows + r0 + i] = q.scale;
        if (kBlocks && threadIdx.x == 0 && i == 0) a.scales[(int64_t)col_tile * a.row_tiles + row_tile] = q.scale;
      }
    }
  }
  if constexpr (kCols) {
    const u32x2 of_matrix = kWhole ? u32x2{~0u, ~0u} : first_codes(a.rows - r0);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const Quotient q(of_col[j]);
      const int32_t c = tc * 8 + j;
      turned[c * 16 + (tr ^ tc)] =
          u32x2{four_codes(q(v[0][j]), q(v[1][j]), q(v[2][j]), q(v[3][j])), four_codes(q(v[4][j]), q(v[5][j]), q(v[6][j]), q(v[7][j]))} & of_matrix;
      if (!kBlocks && tr == 0 && col0 + c < a.cols) a.scales_t[(int64_t)row_tile * a.cols + col0 + c] = q.scale;
      if (kBlocks && threadIdx.x == 0 && j == 0) a.scales_t[(int64_t)row_tile * a.col_tiles + col_tile] = q.scale;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int32_t c = i * 32 + (threadIdx.x >> 3), piece = threadIdx.x & 7;
      const u32x2 lo = turned[c * 16 + ((2 * piece) ^ (c >> 3))], hi = turned[c * 16 + ((2 * piece + 1) ^ (c >> 3))];
      if (col0 + c < a.cols) *(u32x4*)(a.codes_t + ((int64_t)(col0 + c) * a.row_tiles + row_tile) * kGroup + piece * 16) = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  }
}

// Groups along the rows alone need no tile: a thread holds one row's eight columns.  Against eight rows a thread, as above, 2 x 5120 took 2.4 us instead
// of 4.9, 1237 x 1000 2.6 (6.3), 32 760 x 5120 93 (100): 5.4 TB/s.
template <class T, bool kWhole>
__global__ void __launch_bounds__(256) quantize_rows_kernel(QuantArgs a) {
  const int32_t tc = threadIdx.x & 15, col_tile = blockIdx.x % a.col_tiles;
  const int32_t row = blockIdx.x / a.col_tiles * 16 + (threadIdx.x >> 4), c0 = col_tile * kGroup + tc * 8;
  const bool live = row < a.rows;
  const T* p = (const T*)a.x + (int64_t)(live ? row : 0) * a.stride + c0;
  float v[8];
  Eight<T> raw;
  raw.load_some(p, a.cols - c0);
  raw.get(v);
  float amax = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(v[j]));
  amax = max_dpp<kSwapOnes>(amax);
  amax = max_dpp<kSwapTwos>(amax);
  amax = max_dpp<kHalfRowMirror>(amax);
  amax = max_dpp<kRowMirror>(amax);
  const Quotient q(amax);
  if (!live) return;
  u32x2 codes = {four_codes(q(v[0]), q(v[1]), q(v[2]), q(v[3])), four_codes(q(v[4]), q(v[5]), q(v[6]), q(v[7]))};
  if (!kWhole) codes &= first_codes(a.cols - c0);
  *(u32x2*)(a.codes + ((int64_t)row * a.col_tiles + col_tile) * kGroup + tc * 8) = codes;
  if (tc == 0) a.scales[(int64_t)col_tile * a.rows + row] = q.scale;
}

template <class T, bool kWhole>
int launch_quantize(const QuantArgs& a, bool blocks, hipStream_t stream) {
  const bool rows_alone = a.codes && !a.codes_t && !blocks;
  const int64_t grid = rows_alone ? ((int64_t)a.rows + 15) / 16 * a.col_tiles : (int64_t)a.row_tiles * a.col_tiles;
  if (grid > kMostThreads / 256) return fail(RADIAL_ESHAPE, "x is too large for one launch");
  const dim3 blocks_of_grid((unsigned)grid), threads(256);
  if (rows_alone) quantize_rows_kernel<T, kWhole><<<blocks_of_grid, threads, 0, stream>>>(a);
  else if (blocks && a.codes && a.codes_t) quantize_groups_kernel<T, true, true, true, kWhole><<<blocks_of_grid, threads, 0, stream>>>(a);
  else if (blocks && a.codes) quantize_groups_kernel<T, true, true, false, kWhole><<<blocks_of_grid, threads, 0, stream>>>(a);
  else if (blocks) quantize_groups_kernel<T, true, false, true, kWhole><<<blocks_of_grid, threads, 0, stream>>>(a);
  else if (a.codes) quantize_groups_kernel<T, false, true, true, kWhole><<<blocks_of_grid, threads, 0, stream>>>(a);
  else quantize_groups_kernel<T, false, false, true, kWhole><<<blocks_of_grid, threads, 0, stream>>>(a);
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}
template <class T>
int launch_quantize(const QuantArgs& a, bool blocks, hipStream_t stream) {
  const bool whole = a.cols % kGroup == 0 && (!a.codes_t || a.rows % kGroup == 0);
  return whole ? launch_quantize<T, true>(a, blocks, stream) : launch_quantize<T, false>(a, blocks, stream);
}

// ---- product ----------------------------------------------------------------------------------------

struct ProductArgs {
  const uint8_t *a, *b;
  const float *sa, *sb;
  __bf16* out;
  int64_t out_stride;
  int32_t M, N, groups;
  int64_t sa_stride;  // scales of A from one group to the next
  int32_t b_blocks;  // 128-row blocks of B
};

__device__ __forceinline__ i32x8 sixteen_rows(const uint8_t* row) {
  const u32x4 lo = *(const u32x4*)row, hi = *(const u32x4*)(row + 16);
  return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// D[16 x 16] = A[16 x 128] B[128 x 16] of E4M3 codes: lane l supplies bytes 32 (l/16) .. + 31 of row l%16 on either side and
// holds column l%16, rows 4 (l/16) .. + 3.  The pipe adds eight neighbouring products at a time and drops what is below 2^-13 of the largest
// (a product of 2^-13 arrives beside 1, one of 2^-14 does not; eight places away both do).  So does the instruction of 32 codes, at which 32 760 x 5120 x 5120 took 980 us
// instead of 748; the bf16 instruction is exact to float32 but takes twice the matrix time and wants its codes unpacked.  Against float64 the results of that product are
// off by 1.65577e-3 of their norm, their rounding to bf16 alone by 1.65561e-3.
__device__ __forceinline__ f32x4 product16(i32x8 a, i32x8 b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);  // formats 0: E4M3; no block exponents
}

// Up to 16 rows: bound by reading B (2 x 30 720 x 5120: 27.7-30.1 us, 5.2-5.7 TB/s; 2 x 5120 x 5120: 8.9 us, 3 TB/s, five groups a wave).  Few results: by how
// long the groups take one after the other.  A workgroup of 8 waves takes 16 x 16 of C, each wave every 8th group, straight from memory (a lane's 32 bytes of a row, four lanes a line); the parts meet in
// LDS.  Four groups of a wave at a time, or 16 waves, were slower by 0.7 us and more.
constexpr int kParts = 8;
template <bool kBlocks>
__global__ void __launch_bounds__(64 * kParts) product_pieces_kernel(ProductArgs a) {
  __shared__ f32x4 parts[kParts][64];
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t m0, n0;
  tile_of(blockIdx.x, (a.M + 15) / 16, (a.N + 15) / 16, m0, n0);
  m0 *= 16;
  n0 *= 16;
  const int32_t m = m0 + (lane & 15), row = min(m, a.M - 1);
  const int64_t bytes = (int64_t)a.groups * kGroup;
  const uint8_t* b_row = a.b + min(n0 + (lane & 15), a.N - 1) * bytes + (lane >> 4) * 32;
  const uint8_t* a_row = a.a + row * bytes + (lane >> 4) * 32;
  int32_t n[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) n[e] = n0 + 4 * (lane >> 4) + e;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int32_t g = wave; g < a.groups; g += kParts) {
    const f32x4 d = product16(sixteen_rows(b_row + (int64_t)g * kGroup), sixteen_rows(a_row + (int64_t)g * kGroup));
    const float sa = a.sa[(int64_t)g * a.sa_stride + row];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float sb = kBlocks ? a.sb[(int64_t)g * a.b_blocks + n0 / kGroup] : a.sb[(int64_t)g * a.N + min(n[e], a.N - 1)];
      sum[e] = __builtin_fmaf(d[e], sa * sb, sum[e]);
    }
  }
  parts[wave][lane] = sum;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int w = 1; w < kParts; ++w) sum += parts[w][lane];
  if (m >= a.M) return;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n[e] < a.N) a.out[m * a.out_stride + n[e]] = (__bf16)sum[e];
}

// Many rows: a workgroup takes a tile of 16 kMTiles kWavesM x 64 kWavesN, stage by stage of one group (128 bytes of every row), which copies put into
// LDS kStages - 1 stages ahead, straight from memory; a wave takes 16 kMTiles rows of 64 columns.  It holds the four fragments of its columns
// and walks the fragments of its rows: four matrix instructions each, whose sums are scaled and added while the next ones run.  kSplit parts of the
// workgroup's waves take the groups in turn and add up their sums at the end.
// 256 x 256 tiles, eight waves, two a SIMD: 32 760 x 5120 x 5120 with blocks 740-815 us over boxes (2.1-2.3 PFLOP/s) once some 30 launches have let the board settle
// its clock, 1.7-1.8 GHz (what bounds it is the power; the launches before take 750 to 1035), 8192^3 427-504 us (2.2-2.6).  With groups on both sides, one
// product more per sum, 824-915 us.  32 x 32 x 64 matrix instructions, half
// the operand reads, were 14 % slower (their two halves of a group depend on each other), workgroups that stay and fetch the next tile's first stage early 2 %.
template <int kWavesM, int kWavesN, int kMTiles, int kStages, int kSplit>
struct TileShape {
  static constexpr int kWaves = kWavesM * kWavesN;  // of one part of the groups
  static constexpr int kTileM = 16 * kMTiles * kWavesM, kTileN = 64 * kWavesN;
  static constexpr int kCodes = (kTileM + kTileN) * kGroup;                              // bytes of a stage: rows of A, then of B, 128 each
  static constexpr int kCopies = kCodes / 1024 / kWaves;                                 // of a wave
  static constexpr int kScaleCopies = ((kTileM + kTileN) / 64 + kWaves - 1) / kWaves;    // of a wave, 64 scales each; what is left over copies more
  static constexpr int kStage = kCodes + kScaleCopies * kWaves * 256;                    // and the rows' scales
  static constexpr int kRing = kStages * kStage;                                         // of one part
  static constexpr int kMerge = (kSplit - 1) * kWaves * kMTiles * 4096;                  // sums of the other parts
  static constexpr int kLds = kSplit * kRing > kMerge ? kSplit * kRing : kMerge;
  static constexpr int kAhead = kStages - 1;                                             // stages between a copy and its use
  static constexpr int kInFlight = (kStages - 2) * (kCopies + kScaleCopies);             // copies of a wave that may be under way when a stage begins
  static_assert(kCodes % (1024 * kWaves) == 0 && kTileM % 64 == 0 && kLds <= 160 * 1024 && kInFlight <= 63, "whole copies, counted");
};

// Until at most kLeft copies of this wave are under way.
template <int kLeft>
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLeft) : "memory"); }

template <int kWavesM, int kWavesN, int kMTiles, int kStages, int kSplit, bool kBlocks>
__global__ void __launch_bounds__(64 * kWavesM * kWavesN * kSplit) product_tile_kernel(ProductArgs a) {
  using S = TileShape<kWavesM, kWavesN, kMTiles, kStages, kSplit>;
  extern __shared__ __align__(1024) char lds[];
  const int lane = threadIdx.x & 63, wave_of_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = kSplit == 1 ? 0 : wave_of_all / S::kWaves, wave = wave_of_all - part * S::kWaves;
  int32_t m0, n0;
  {
    const int32_t tiles_m = (a.M + S::kTileM - 1) / S::kTileM, tiles_n = (a.N + S::kTileN - 1) / S::kTileN;
    tile_of(blockIdx.x, tiles_m, tiles_n, m0, n0);
    m0 *= S::kTileM;
    n0 *= S::kTileN;
  }
  const int64_t bytes = (int64_t)a.groups * kGroup;
  const uint8_t* a_base = a.a + m0 * bytes;
  const uint8_t* b_base = a.b + n0 * bytes;
  const uint32_t lds0 = lds_address(lds) + part * S::kRing;

  // This wave's copies: 8 rows of 128 bytes each; a lane's source row and piece are those that belong at its place.  Rows beyond the matrix
  // repeat its last one.
  uint32_t from[S::kCopies], scale_from[S::kScaleCopies];
#pragma unroll
  for (int i = 0; i < S::kCopies; ++i) {
    const int copy = wave * S::kCopies + i;
    const bool of_a = copy * 8 < S::kTileM;
    const int place = (of_a ? copy : copy - S::kTileM / 8) * 64 + lane, line = place >> 4;
    const int source = (place & 15) ^ (of_a ? exchange_of<false>(line) : exchange_of<true>(line));
    const int32_t r = min(line * 2 + (source >> 3), (of_a ? a.M - m0 : a.N - n0) - 1);
    from[i] = (uint32_t)r * (uint32_t)bytes + (source & 7) * 16;
  }
#pragma unroll
  for (int i = 0; i < S::kScaleCopies; ++i) {
    const int first = (wave * S::kScaleCopies + i) * 64;
    // scales of blocks are no copies: those of A once more
    scale_from[i] = 4u * (uint32_t)(first < S::kTileM || kBlocks ? min(m0 + first + lane, a.M - 1) : min(n0 + first - S::kTileM + lane, a.N - 1));
  }
  // Stage j of the part is group j kSplit + part.
  constexpr uint64_t kAll = ~0ull;
  auto copy_codes = [&](int32_t j, uint32_t stage, int i, uint64_t lanes, bool all) __attribute__((always_inline)) {
    const int copy = wave * S::kCopies + i;
    const uint8_t* base = (copy * 8 < S::kTileM ? a_base : b_base) + (int64_t)(j * kSplit + part) * kGroup;
    if (all) copy16_to_lds_sv(base, from[i], lds0 + stage + copy * 1024);
    else copy16_to_lds_sv_masked(base, from[i], lds0 + stage + copy * 1024, lanes);
  };
  auto copy_scales = [&](int32_t j, uint32_t stage, uint64_t lanes) __attribute__((always_inline)) {
    const int64_t g = j * kSplit + part;
#pragma unroll
    for (int i = 0; i < S::kScaleCopies; ++i) {
      const int first = (wave * S::kScaleCopies + i) * 64;
      const float* base = first < S::kTileM || kBlocks ? a.sa + g * a.sa_stride : a.sb + g * a.N;
      copy4_to_lds_sv_masked(base, scale_from[i], lds0 + stage + S::kCodes + first * 4, lanes);
    }
  };

  const int wm = wave / kWavesN, wn = wave % kWavesN;
  const int l16 = lane & 15, q = lane >> 4;
  f32x4 sum[kMTiles][4];
#pragma unroll
  for (int i = 0; i < kMTiles; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int32_t mine = (a.groups - part + kSplit - 1) / kSplit;  // stages of this part
  for (int32_t j = 0; j < S::kAhead && j < mine; ++j) {
    copy_scales(j, j * S::kStage, kAll);
#pragma unroll
    for (int i = 0; i < S::kCopies; ++i) copy_codes(j, j * S::kStage, i, kAll, true);
  }

  // A lane's 32 bytes of a row are pieces q and q + 4, the same on both sides (which bytes make up a lane's part does not matter): a read is served 16
  // lanes at a time, lanes 0 .. 3, 12 .. 15, 20 .. 27 first, and neighbouring pieces of those rows lie in different banks.  With pieces 2 q and 2 q + 1
  // they met two by two: 0.31 of 1.78 million cycles at 32 760 x 5120 x 5120.
  uint32_t a_at[2], b_at[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    a_at[h] = lds0 + wm * kMTiles * 16 * kGroup + code_piece<false>(l16, q + 4 * h);
    b_at[h] = lds0 + (S::kTileM + wn * 64) * kGroup + code_piece<true>((l16 >> 2) * 16 + (l16 & 3), q + 4 * h);
  }
  const uint32_t a_scale_at = lds0 + S::kCodes + (wm * kMTiles * 16 + l16) * 4;
  const uint32_t b_scale_at = lds0 + S::kCodes + (S::kTileM + wn * 64 + q * 16) * 4;
  using Lds = __attribute__((address_space(3))) const char*;
  auto fragment = [&](const Lds (&at)[2], int distance) __attribute__((always_inline)) -> i32x8 {
    using Piece = __attribute__((address_space(3))) const u32x4*;
    const u32x4 lo = *(Piece)(at[0] + distance), hi = *(Piece)(at[1] + distance);
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  // The wave's columns are of one block; its scale is a scalar, asked for one stage ahead.  (A vector load would wait for the copies, which come before it.)
  using Scalars = const float __attribute__((address_space(4)))*;
  const Scalars block_scales = (Scalars)(a.sb + min((n0 + wn * 64) / kGroup, a.b_blocks - 1));
  auto block_scale = [&](int32_t g) __attribute__((always_inline)) { return block_scales[(int64_t)g * a.b_blocks]; };
  float next_block = kBlocks ? block_scale(min(part, a.groups - 1)) : 0.f;
  uint32_t stage = 0, free = S::kAhead * S::kStage;  // where the stage's codes lie, and where those of the stage kAhead later go
  // `copies`: there is a stage to copy (1), there is none (0), or `lanes` says so, all or none (2).
  auto walk = [&](int32_t j, auto copies_, uint64_t lanes) __attribute__((always_inline)) {
    constexpr int copies = decltype(copies_)::value;
    const Lds at_a[2] = {lds_pointer<const char>(a_at[0] + stage), lds_pointer<const char>(a_at[1] + stage)};
    const Lds at_b[2] = {lds_pointer<const char>(b_at[0] + stage), lds_pointer<const char>(b_at[1] + stage)};
    const auto* a_scales = lds_pointer<const float>(a_scale_at + stage);
    const auto* b_scales = lds_pointer<const f32x4>(b_scale_at + stage);
    if (copies) copy_scales(j + S::kAhead, free, copies == 1 ? kAll : lanes);
    // Row 4 i + j of fragment t is column 16 i + 4 t + j of the wave's 64: a lane's sums of the four are 16 neighbouring columns.
    i32x8 columns[4];
    f32x4 sb[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      columns[t] = fragment(at_b, t * 4 * kGroup);
      if (!kBlocks) sb[t] = b_scales[t];
    }
    const float of_block = next_block;
    if (kBlocks) next_block = block_scale(min((j + 1) * kSplit + part, a.groups - 1));
    // The sums of one row fragment are added between the matrix instructions of the next: each has the time of three to come out of the pipe.
    i32x8 rows = fragment(at_a, 0);
    float factor = a_scales[0], before = 0.f;
    f32x4 d[4];
#pragma unroll
    for (int i = 0; i <= kMTiles; ++i) {
      i32x8 next;
      float next_factor = 0.f;
      if (i + 1 < kMTiles) {
        next = fragment(at_a, (i + 1) * 16 * kGroup);
        next_factor = a_scales[(i + 1) * 16];
      }
      // copies in the first half of a stage (spread over all of it the last ones came late: 867 instead of 838 us; all in the first quarter: 908)
      if (copies && i < kMTiles) {
#pragma unroll
        for (int c = 2 * i * S::kCopies / kMTiles; c < 2 * (i + 1) * S::kCopies / kMTiles && c < S::kCopies; ++c) copy_codes(j + S::kAhead, free, c, lanes, copies == 1);
      }
      if (kBlocks) factor *= of_block;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (i > 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[i - 1][t][e] = __builtin_fmaf(d[t][e], kBlocks ? before : before * sb[t][e], sum[i - 1][t][e]);
        }
        if (i < kMTiles) d[t] = product16(columns[t], rows);
        __builtin_amdgcn_sched_barrier(0);
      }
      before = factor;
      rows = next;
      factor = next_factor;
    }
    stage = stage + S::kStage == S::kRing ? 0 : stage + S::kStage;
    free = free + S::kStage == S::kRing ? 0 : free + S::kStage;
  };
  // Copies come in order: once only those of the kAhead - 1 stages behind are under way, this stage's are done.  The last stages, where
  // some parts have one less, wait for all.
  int32_t j = 0;
  for (; (j + S::kAhead) * kSplit + kSplit - 1 < a.groups; ++j) {
    wait_copies<S::kInFlight>();
    __syncthreads();
    walk(j, std::integral_constant<int, 1>(), kAll);
  }
  for (; j * kSplit < a.groups; ++j) {
    wait_copies<0>();
    __syncthreads();
    if (kSplit == 1) walk(j, std::integral_constant<int, 0>(), 0ull);
    else if (j < mine) walk(j, std::integral_constant<int, kSplit == 1 ? 0 : 2>(), j + S::kAhead < mine ? kAll : 0ull);
  }

#pragma unroll
  for (int i = 0; i < kMTiles; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(sum[i][j]));  // the last sums are added here, not where they are stored, which would hold both parts of each
  if constexpr (kSplit > 1) {
    // the other parts' sums, in order
    __syncthreads();
    auto place = [&](int of_part, int i, int t) { return lds_cast<f32x4>(lds + (((of_part - 1) * S::kWaves + wave) * kMTiles * 4 + i * 4 + t) * 1024 + lane * 16); };
    if (part > 0) {
#pragma unroll
      for (int i = 0; i < kMTiles; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) *place(part, i, t) = sum[i][t];
    }
    __syncthreads();
    if (part > 0) return;
    for (int from_part = 1; from_part < kSplit; ++from_part)
#pragma unroll
      for (int i = 0; i < kMTiles; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) sum[i][t] += *place(from_part, i, t);
  }
#pragma unroll
  for (int i = 0; i < kMTiles; ++i) {
    uint32_t pair[8];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      pair[2 * t] = pack_bf16(sum[i][t][0], sum[i][t][1]);
      pair[2 * t + 1] = pack_bf16(sum[i][t][2], sum[i][t][3]);
    }
    // 16 neighbouring columns of a lane, wherever they lie (by way of LDS, to store whole rows of a tile, single elements were slower)
    const int32_t m = m0 + (wm * kMTiles + i) * 16 + l16, n = n0 + wn * 64 + q * 16;
    if (m >= a.M) continue;
    __bf16* out = a.out + m * a.out_stride + n;
    if (n + 16 <= a.N) {
      *(u32x4_any*)out = u32x4{pair[0], pair[1], pair[2], pair[3]};
      *(u32x4_any*)(out + 8) = u32x4{pair[4], pair[5], pair[6], pair[7]};
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (n + e < a.N) ((uint16_t*)out)[e] = (uint16_t)(pair[e / 2] >> (e % 2 * 16));
    }
  }
}

template <int kWavesM, int kWavesN, int kMTiles, int kStages, int kSplit, bool kBlocks>
int launch_tiles(const ProductArgs& a, hipStream_t stream) {
  using S = TileShape<kWavesM, kWavesN, kMTiles, kStages, kSplit>;
  const int64_t tiles = ((int64_t)a.M + S::kTileM - 1) / S::kTileM * (((int64_t)a.N + S::kTileN - 1) / S::kTileN);
  if (tiles > kMostThreads / (64 * S::kWaves * kSplit)) return fail(RADIAL_ESHAPE, "M*N is too large for one launch");
  if constexpr (S::kLds > 65536) {
    static DeviceOnce configured;
    if (int rc = allow_dynamic_lds(configured, (const void*)product_tile_kernel<kWavesM, kWavesN, kMTiles, kStages, kSplit, kBlocks>, S::kLds)) return rc;
  }
  product_tile_kernel<kWavesM, kWavesN, kMTiles, kStages, kSplit, kBlocks><<<dim3((unsigned)tiles), dim3(64 * S::kWaves * kSplit), S::kLds, stream>>>(a);
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}

template <bool kBlocks>
int launch_form(int form, const ProductArgs& a, hipStream_t stream) {
  switch (form) {
    case 0: return launch_tiles<2, 4, 8, 2, 1, kBlocks>(a, stream);
    case 1: return launch_tiles<2, 4, 6, 2, 1, kBlocks>(a, stream);
    case 2: return launch_tiles<2, 2, 4, 2, 1, kBlocks>(a, stream);
    case 3: return launch_tiles<2, 2, 4, 2, 2, kBlocks>(a, stream);
    case 4: return launch_tiles<2, 2, 2, 3, 1, kBlocks>(a, stream);
    case 5: return launch_tiles<2, 2, 2, 3, 2, kBlocks>(a, stream);
    case 6: return launch_tiles<2, 1, 2, 2, 2, kBlocks>(a, stream);
    default: return launch_tiles<2, 1, 2, 2, 4, kBlocks>(a, stream);
  }
}

template <bool kBlocks>
int launch_product(const ProductArgs& a, hipStream_t stream) {
  if (takes_pieces(a.M, a.N)) {
    const int64_t tiles = pieces_of(a.M) * pieces_of(a.N);
    if (tiles > kMostThreads / (64 * kParts)) return fail(RADIAL_ESHAPE, "N is too large for one launch");
    product_pieces_kernel<kBlocks><<<dim3((unsigned)tiles), dim3(64 * kParts), 0, stream>>>(a);
    RADIAL_HIP_TRY(hipGetLastError());
    return RADIAL_OK;
  }
  const ProductPlan plan = plan_product(a.M, a.N, a.groups);
  ProductArgs part = a;
  part.M = plan.rows;
  if (int rc = launch_form<kBlocks>(plan.form, part, stream)) return rc;
  if (plan.rows == a.M) return RADIAL_OK;
  part.M = a.M - plan.rows;
  part.a += (int64_t)plan.rows * a.groups * kGroup;
  part.sa += plan.rows;
  part.out += plan.rows * a.out_stride;
  return launch_form<kBlocks>(plan.rest, part, stream);
}

}  // namespace
}  // namespace radial

using namespace radial;

extern "C" int radial_quantize_groups_fp8(int32_t rows, int32_t cols, const void* x, int32_t type, int64_t stride, int32_t grouping, uint8_t* codes,
                                          float* scales, uint8_t* codes_t, float* scales_t, void* hip_stream) {
  if (rows < 1 || cols < 1) return fail(RADIAL_EINVAL, "rows and cols must be >= 1");
  if (!x) return fail(RADIAL_EINVAL, "x is NULL");
  if (!is_type(type)) return fail(RADIAL_EINVAL, "type must be RADIAL_BF16 or RADIAL_F32 (got %d)", type);
  if (grouping != RADIAL_GROUPS && grouping != RADIAL_BLOCKS) return fail(RADIAL_EINVAL, "grouping must be RADIAL_GROUPS or RADIAL_BLOCKS (got %d)", grouping);
  if (!codes != !scales || !codes_t != !scales_t) return fail(RADIAL_EINVAL, "codes and scales go together");
  if (!codes && !codes_t) return fail(RADIAL_EINVAL, "neither codes nor codes_t is given");
  if ((uintptr_t)x % size_of(type)) return fail(RADIAL_ESHAPE, "x is not aligned to its elements");
  if (stride < cols) return fail(RADIAL_ESHAPE, "stride must not be below cols");
  if (((uintptr_t)codes | (uintptr_t)codes_t) & 15u) return fail(RADIAL_ESHAPE, "codes are not 16-byte aligned");
  if (((uintptr_t)scales | (uintptr_t)scales_t) & 3u) return fail(RADIAL_ESHAPE, "scales are not aligned to their elements");
  if (rows > 0x7fffffff - kGroup || cols > 0x7fffffff - kGroup) return fail(RADIAL_ESHAPE, "x is too large for one launch");
  QuantArgs a = {};
  a.x = x; a.stride = stride; a.rows = rows; a.cols = cols;
  a.codes = codes; a.scales = scales; a.codes_t = codes_t; a.scales_t = scales_t;
  a.row_tiles = (int32_t)(((int64_t)rows + kGroup - 1) / kGroup);
  a.col_tiles = (int32_t)(((int64_t)cols + kGroup - 1) / kGroup);
  const bool blocks = grouping == RADIAL_BLOCKS;
  return type == RADIAL_F32 ? launch_quantize<float>(a, blocks, (hipStream_t)hip_stream) : launch_quantize<__bf16>(a, blocks, (hipStream_t)hip_stream);
}

extern "C" int radial_product_fp8(int32_t M, int32_t N, int32_t K, const uint8_t* a_codes, const float* a_scales, const uint8_t* b_codes,
                                  const float* b_scales, int32_t b_grouping, void* out, int64_t out_stride, void* hip_stream) {
  if (M < 1 || N < 1 || K < 1) return fail(RADIAL_EINVAL, "M, N, K must be >= 1");
  if (!a_codes || !a_scales || !b_codes || !b_scales || !out) return fail(RADIAL_EINVAL, "codes, scales or out is NULL");
  if (b_grouping != RADIAL_GROUPS && b_grouping != RADIAL_BLOCKS) return fail(RADIAL_EINVAL, "b_grouping must be RADIAL_GROUPS or RADIAL_BLOCKS (got %d)", b_grouping);
  if (((uintptr_t)a_codes | (uintptr_t)b_codes) & 15u) return fail(RADIAL_ESHAPE, "codes are not 16-byte aligned");
  if (((uintptr_t)a_scales | (uintptr_t)b_scales) & 3u) return fail(RADIAL_ESHAPE, "scales are not aligned to their elements");
  if ((uintptr_t)out & 1u) return fail(RADIAL_ESHAPE, "out is not aligned to its elements");
  if (out_stride < N) return fail(RADIAL_ESHAPE, "out_stride must not be below N");
  if (M > 1 << 29 || N > 1 << 29 || K > 1 << 23) return fail(RADIAL_ESHAPE, "M and N must be at most 2^29 and K 2^23: larger ones are too large for one launch");
  ProductArgs a = {};
  a.a = a_codes; a.b = b_codes; a.sa = a_scales; a.sb = b_scales;
  a.out = (__bf16*)out; a.out_stride = out_stride;
  a.M = M; a.N = N; a.sa_stride = M;
  a.groups = (K + kGroup - 1) / kGroup;
  a.b_blocks = (N + kGroup - 1) / kGroup;
  hipStream_t stream = (hipStream_t)hip_stream;
  const bool blocks = b_grouping == RADIAL_BLOCKS;
  return blocks ? launch_product<true>(a, stream) : launch_product<false>(a, stream);
}
