// Products of 8-bit integers for gfx950:
//     C[m, n] = sa[m] sb[n] (A[m, :] . B[n, :]) + bias[n],
// A and B int8 codes with a scale for each row, summed exactly in 32 bits by v_mfma_i32_16x16x64_i8.  The tile is computed transposed (matrix A operand = rows
// of B, B operand = rows of A): a lane then holds one row m of C and, by the order in which it reads B's rows, sixteen neighbouring columns n.
#include <type_traits>

#include "radial_product_i8.h"
#include "radial_product_i8_rule.h"

namespace radial {
namespace {

typedef int32_t i32x4v __attribute__((ext_vector_type(4)));

struct ProductArgs {
  const int8_t *a, *b;
  const float *sa, *sb, *bias;
  void* out;
  int64_t out_stride;
  int64_t a_row, a_group, b_row, b_group;  // bytes from a row, a group of a row to the next
  int32_t M, N, groups;
  int32_t out_type, accumulate;
};

// D[16 x 16] += A[16 x 64] B[64 x 16]: lane l supplies 16 bytes of row l%16 on either side, the part l/16 of the 64, and holds column l%16, rows 4 (l/16) .. + 3.
__device__ __forceinline__ i32x4v multiply(u32x4 a, u32x4 b, i32x4v c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4v, a), __builtin_bit_cast(i32x4v, b), c, 0, 0, 0);
}

__device__ __forceinline__ float result(int32_t sum, float scale, float bias) { return __builtin_fmaf((float)sum, scale, bias); }

// Some consecutive results of a row, `count` of kCount inside the matrix.
template <int kCount>
__device__ __forceinline__ void put(const ProductArgs& a, int32_t m, int32_t n, const float (&y)[kCount], int32_t count) {
  const int64_t at = m * a.out_stride + n;
  if (a.out_type == RADIAL_F32) {
    float* out = (float*)a.out + at;
    if (count >= kCount) {
#pragma unroll
      for (int i = 0; i < kCount; i += 4) {
        f32x4 v = {y[i], y[i + 1], y[i + 2], y[i + 3]};
        if (a.accumulate) v += *(const f32x4_any*)(out + i);
        *(f32x4_any*)(out + i) = v;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kCount; ++i)
        if (i < count) out[i] = a.accumulate ? out[i] + y[i] : y[i];
    }
  } else {
    __bf16* out = (__bf16*)a.out + at;
    if (count >= kCount) {
#pragma unroll
      for (int i = 0; i < kCount; i += 4) {
        if constexpr (kCount % 8 == 0) {
          if (i % 8 == 0) *(u32x4_any*)(out + i) = u32x4{pack_bf16(y[i], y[i + 1]), pack_bf16(y[i + 2], y[i + 3]), pack_bf16(y[i + 4], y[i + 5]), pack_bf16(y[i + 6], y[i + 7])};
        } else {
          *(u32x2_any*)(out + i) = u32x2{pack_bf16(y[i], y[i + 1]), pack_bf16(y[i + 2], y[i + 3])};
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kCount; ++i)
        if (i < count) out[i] = (__bf16)y[i];
    }
  }
}

// A wave's float32 results of one row fragment, 16 rows of 64 columns that are all inside: lane l has row l%16, columns 16 (l/16) .. + 15.  Pieces of 16 bytes change lanes, so that
// each store writes 64 neighbouring bytes of a row and not every fourth piece of it: the gradients of 14 040 x 5120 x 5120 take 848 us instead of 859, 1237 x 1961 x 1001
// 13.4 instead of 14.4.  (bf16 results, which are every second piece, gained nothing from the like.)
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
  const auto sw = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  const uint32_t first = sw[0], second = sw[1];
  a = first;
  b = second;
}
__device__ __forceinline__ void swap_rows(uint32_t& a, uint32_t& b) {
  const auto sw = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  const uint32_t first = sw[0], second = sw[1];
  a = first;
  b = second;
}
__device__ __forceinline__ void put_fragment(const ProductArgs& a, int32_t m, int32_t n_of_wave, int32_t q, const float (&y)[16]) {
  uint32_t piece[4][4];  // piece t of a lane: columns 16 q + 4 t on; after the swaps columns 16 t + 4 q on
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) piece[t][e] = __builtin_bit_cast(uint32_t, y[4 * t + e]);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    swap_halves(piece[0][e], piece[2][e]);
    swap_halves(piece[1][e], piece[3][e]);
    swap_rows(piece[0][e], piece[1][e]);
    swap_rows(piece[2][e], piece[3][e]);
  }
  if (m >= a.M) return;
  float* out = (float*)a.out + m * a.out_stride + n_of_wave + 4 * q;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    f32x4 v = __builtin_bit_cast(f32x4, u32x4{piece[t][0], piece[t][1], piece[t][2], piece[t][3]});
    if (a.accumulate) v += *(const f32x4_any*)(out + 16 * t);
    *(f32x4_any*)(out + 16 * t) = v;
  }
}

// Few rows, or few results: a workgroup of 8 waves takes 16 x 16 of C, each wave every 8th group, straight from memory (a lane's 32 bytes of a row, four
// lanes a line); the parts meet in LDS.  (1 x 5120 x 5120 7.7 us; two or four times the rows for a workgroup were slower: 64 x 5120 x 5120 22 to 24 us, in tiles of 32 x 64 8.5.)
constexpr int kParts = 8;

// The sums of the parts, scaled: wave 0 holds them, column n0 + 4 (lane / 16) on, row m.
__device__ __forceinline__ void join_parts(const ProductArgs& a, i32x4v (&parts)[kParts][64], i32x4v sum, int32_t m, int32_t n0, float sa) {
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  parts[wave][lane] = sum;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int w = 1; w < kParts; ++w) sum += parts[w][lane];
  const int32_t n = n0 + 4 * (lane >> 4);
  if (m >= a.M) return;
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = result(sum[e], sa * a.sb[min(n + e, a.N - 1)], a.bias ? a.bias[min(n + e, a.N - 1)] : 0.f);
  put(a, m, n, y, a.N - n);
}

__global__ void __launch_bounds__(64 * kParts) product_i8_pieces_kernel(ProductArgs a) {
  __shared__ i32x4v parts[kParts][64];
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t m0, n0;
  tile_of(blockIdx.x, (a.M + 15) / 16, (a.N + 15) / 16, m0, n0);
  m0 *= 16;
  n0 *= 16;
  const int32_t m = m0 + (lane & 15), row = min(m, a.M - 1);
  const int8_t* b_row = a.b + min(n0 + (lane & 15), a.N - 1) * a.b_row + (lane >> 4) * 32;
  const int8_t* a_row = a.a + row * a.a_row + (lane >> 4) * 32;
  i32x4v sum = {0, 0, 0, 0};
  for (int32_t g = wave; g < a.groups; g += kParts) {
    const int8_t *b = b_row + g * a.b_group, *of_a = a_row + g * a.a_group;
    sum = multiply(*(const u32x4*)b, *(const u32x4*)of_a, sum);
    sum = multiply(*(const u32x4*)(b + 16), *(const u32x4*)(of_a + 16), sum);
  }
  join_parts(a, parts, sum, m, n0, a.sa[row]);
}

// A projection of up to 4 rows of up to 8192 columns in one launch: every workgroup quantises the rows for itself, into LDS, while the first groups of its weights are under
// way, and goes on as above.  Bound by reading W: 2 x 5120 x 5120 8.2 us, 3.2 TB/s, of which a launch is three to four (in two launches 4.8 + 8.6).
constexpr int kFewRows = 4, kFewCols = 8192, kUnderWay = 5;
template <class T, int kRows>
__global__ void __launch_bounds__(64 * kParts) linear_i8_few_kernel(ProductArgs a, const T* x, int64_t stride, int32_t cols) {
  constexpr int kPieces = kFewCols / (64 * kParts * 8);  // of eight columns of a thread
  __shared__ i32x4v parts[kParts][64];
  __shared__ __align__(16) int8_t codes[kRows][kFewCols];
  __shared__ uint32_t of_wave[kRows][kParts];
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n0 = blockIdx.x * 16;
  const int8_t* b_row = a.b + min(n0 + (lane & 15), a.N - 1) * a.b_row + (lane >> 4) * 32;
  Eight<T> held[kRows][kPieces];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const int32_t c = (p * 64 * kParts + (int32_t)threadIdx.x) * 8;
      held[r][p].load_some(x + min(r, a.M - 1) * stride + c, cols - c);
    }
  u32x4 under_way[kUnderWay][2];
#pragma unroll
  for (int i = 0; i < kUnderWay; ++i) {
    const int8_t* b = b_row + min(wave + i * kParts, a.groups - 1) * a.b_group;
    under_way[i][0] = *(const u32x4*)b;
    under_way[i][1] = *(const u32x4*)(b + 16);
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    uint32_t largest = 0;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      float v[8];
      held[r][p].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) largest = max(largest, magnitude(v[j]));
    }
    largest = wave_max(largest);
    if (lane == 0) of_wave[r][wave] = largest;
  }
  __syncthreads();
  const int32_t mine = min(lane & 15, kRows - 1);
  float sa = 0.f;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    uint32_t largest = 0;
#pragma unroll
    for (int w = 0; w < kParts; ++w) largest = max(largest, of_wave[r][w]);
    const Code code(largest);
    if (r == mine) sa = code.scale;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      float v[8];
      held[r][p].get(v);
      *(u32x2*)&codes[r][(p * 64 * kParts + threadIdx.x) * 8] = u32x2{code.four(v[0], v[1], v[2], v[3]), code.four(v[4], v[5], v[6], v[7])};
    }
  }
  __syncthreads();
  i32x4v sum = {0, 0, 0, 0};
  auto add = [&](int32_t g, const u32x4 (&column)[2]) __attribute__((always_inline)) {
    const int8_t* of_a = &codes[mine][g * kCodeGroup + (lane >> 4) * 32];
    sum = multiply(column[0], *(const u32x4*)of_a, sum);
    sum = multiply(column[1], *(const u32x4*)(of_a + 16), sum);
  };
#pragma unroll
  for (int i = 0; i < kUnderWay; ++i)
    if (wave + i * kParts < a.groups) add(wave + i * kParts, under_way[i]);
  for (int32_t g = wave + kUnderWay * kParts; g < a.groups; g += kParts) {
    const int8_t* b = b_row + g * a.b_group;
    const u32x4 column[2] = {*(const u32x4*)b, *(const u32x4*)(b + 16)};
    add(g, column);
  }
  join_parts(a, parts, sum, lane & 15, n0, sa);
}

// Many rows: a workgroup takes a tile of 16 kMTiles kWavesM x 64 kWavesN, stage by stage of one group (128 bytes of every row), which copies put into LDS
// kStages - 1 stages ahead, straight from memory.  kSplit parts of the workgroup's waves take the groups in turn and add up their sums at the end.
// 256 x 256 tiles, eight waves, two a SIMD: 32 760 x 5120 x 5120 660-690 us from board to board (2.5-2.6 POP/s; a large library product of whole numbers without scales takes 733-755), 8192^3 400
// (2.75).  At 32 760 rows the matrix pipes are busy 54 % of the cycles at 2.2 GHz; with codes of zeros it takes 550 and 8192^3 318 (3.46 POP/s, 69 %): the board's power, then the reads of A from
// beyond the last-level cache (a quarter of A's memory: 640).  What does not change the time: fragments read a stage ahead through rings of four and five
// stages of 64 bytes (717 beside 700), four waves of 128 x 128 with a third fewer reads from LDS (750), A in blocks of 128 columns (708 beside 704).  Asking for lines of A three stages ahead
// costs 50 us; tiles of 128 x 256, two workgroups a unit, 831.
template <int kWavesM, int kWavesN, int kMTiles, int kStages, int kSplit>
struct TileShape {
  static constexpr int kWaves = kWavesM * kWavesN;  // of one part of the groups
  static constexpr int kTileM = 16 * kMTiles * kWavesM, kTileN = 64 * kWavesN;
  static constexpr int kNTiles = 4;
  static constexpr int kStage = (kTileM + kTileN) * kCodeGroup;                  // bytes of a stage: rows of A, then of B, 128 each
  static constexpr int kCopies = kStage / 1024 / kWaves;                         // of a wave
  static constexpr int kRing = kStages * kStage;                                 // of one part
  static constexpr int kMerge = (kSplit - 1) * kWaves * kMTiles * kNTiles * 1024;  // sums of the other parts
  static constexpr int kLds = kSplit * kRing > kMerge ? kSplit * kRing : kMerge;
  static constexpr int kAhead = kStages - 1;                                     // stages between a copy and its use
  static constexpr int kInFlight = (kStages - 2) * kCopies;                      // copies of a wave that may be under way when a stage begins
  static_assert(kStage % (1024 * kWaves) == 0 && kLds <= 160 * 1024 && kInFlight <= 63, "whole copies, counted");
};

// Until at most kLeft copies of this wave are under way.
template <int kLeft>
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLeft) : "memory"); }

template <int kWavesM, int kWavesN, int kMTiles, int kStages, int kSplit>
__global__ void __launch_bounds__(64 * kWavesM * kWavesN * kSplit) __attribute__((amdgpu_waves_per_eu(2))) product_i8_tile_kernel(ProductArgs a) {
  using S = TileShape<kWavesM, kWavesN, kMTiles, kStages, kSplit>;
  extern __shared__ __align__(1024) char lds[];
  const int lane = threadIdx.x & 63, wave_of_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = kSplit == 1 ? 0 : wave_of_all / S::kWaves, wave = wave_of_all - part * S::kWaves;
  int32_t m0, n0;
  tile_of<kBandI8>(blockIdx.x, (a.M + S::kTileM - 1) / S::kTileM, (a.N + S::kTileN - 1) / S::kTileN, m0, n0);
  m0 *= S::kTileM;
  n0 *= S::kTileN;
  const int8_t* a_base = a.a + m0 * a.a_row;
  const int8_t* b_base = a.b + n0 * a.b_row;
  const uint32_t lds0 = lds_address(lds) + part * S::kRing;

  // This wave's copies: 8 rows of 128 bytes each; a lane's source row and piece are those that belong at its place.  Rows beyond the matrix
  // repeat its last one.
  uint32_t from[S::kCopies];
#pragma unroll
  for (int i = 0; i < S::kCopies; ++i) {
    const int copy = wave * S::kCopies + i;
    const bool of_a = copy * 8 < S::kTileM;
    const int place = (of_a ? copy : copy - S::kTileM / 8) * 64 + lane, line = place >> 4;
    const int source = (place & 15) ^ (of_a ? exchange_of<false>(line) : exchange_of<true>(line));
    const int32_t r = min(line * 2 + (source >> 3), (of_a ? a.M - m0 : a.N - n0) - 1);
    from[i] = (uint32_t)r * (uint32_t)(of_a ? a.a_row : a.b_row) + (source & 7) * 16;
  }
  // Stage j of the part is group j kSplit + part.
  constexpr uint64_t kAll = ~0ull;
  auto copy_codes = [&](int32_t j, uint32_t stage, int i, uint64_t lanes, bool all) __attribute__((always_inline)) {
    const int copy = wave * S::kCopies + i;
    const int8_t* base = copy * 8 < S::kTileM ? a_base + (j * kSplit + part) * a.a_group : b_base + (j * kSplit + part) * a.b_group;
    if (all) copy16_to_lds_sv(base, from[i], lds0 + stage + copy * 1024);
    else copy16_to_lds_sv_masked(base, from[i], lds0 + stage + copy * 1024, lanes);
  };

  const int wm = wave / kWavesN, wn = wave % kWavesN;
  const int l16 = lane & 15, q = lane >> 4;
  i32x4v sum[kMTiles][S::kNTiles];
#pragma unroll
  for (int i = 0; i < kMTiles; ++i)
#pragma unroll
    for (int j = 0; j < S::kNTiles; ++j) sum[i][j] = i32x4v{0, 0, 0, 0};

  const int32_t mine = (a.groups - part + kSplit - 1) / kSplit;  // stages of this part
  for (int32_t j = 0; j < S::kAhead && j < mine; ++j) {
#pragma unroll
    for (int i = 0; i < S::kCopies; ++i) copy_codes(j, j * S::kStage, i, kAll, true);
  }

  // A lane's 32 bytes of a row are pieces q and q + 4, the same on both sides (which bytes make up a lane's part does not matter): neighbouring
  // pieces of the 16 rows that are read together lie in different banks.
  uint32_t a_at[2], b_at[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    a_at[h] = lds0 + wm * kMTiles * 16 * kCodeGroup + code_piece<false>(l16, q + 4 * h);
    b_at[h] = lds0 + (S::kTileM + wn * 64) * kCodeGroup + code_piece<true>((l16 >> 2) * 16 + (l16 & 3), q + 4 * h);
  }
  auto piece = [&](uint32_t at, int distance) __attribute__((always_inline)) -> u32x4 { return *lds_pointer<const u32x4>(at + distance); };
  uint32_t stage = 0, free = S::kAhead * S::kStage;  // where the stage's codes lie, and where those of the stage kAhead later go
  // `copies`: there is a stage to copy (1), there is none (0), or `lanes` says so, all or none (2).
  auto walk = [&](int32_t j, auto copies_, uint64_t lanes) __attribute__((always_inline)) {
    constexpr int copies = decltype(copies_)::value;
    // Row 4 i + j of fragment t is column 16 i + 4 t + j of 64: a lane's sums of four fragments are 16 neighbouring columns.
    u32x4 columns[S::kNTiles][2], rows[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      rows[h] = piece(a_at[h] + stage, 0);
#pragma unroll
      for (int t = 0; t < S::kNTiles; ++t) columns[t][h] = piece(b_at[h] + stage, t * 4 * kCodeGroup);
    }
#pragma unroll
    for (int i = 0; i < kMTiles; ++i) {
      u32x4 next[2];
      if (i + 1 < kMTiles) {
#pragma unroll
        for (int h = 0; h < 2; ++h) next[h] = piece(a_at[h] + stage, (i + 1) * 16 * kCodeGroup);
      }
      if (copies) {
#pragma unroll
        for (int c = 2 * i * S::kCopies / kMTiles; c < 2 * (i + 1) * S::kCopies / kMTiles && c < S::kCopies; ++c) copy_codes(j + S::kAhead, free, c, lanes, copies == 1);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < S::kNTiles; ++t) sum[i][t] = multiply(columns[t][h], rows[h], sum[i][t]);
      __builtin_amdgcn_sched_barrier(0);
      rows[0] = next[0];
      rows[1] = next[1];
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

  if constexpr (kSplit > 1) {
    // the other parts' sums
    __syncthreads();
    auto place = [&](int of_part, int i, int t) { return lds_cast<i32x4v>(lds + (((of_part - 1) * S::kWaves + wave) * kMTiles * S::kNTiles + i * S::kNTiles + t) * 1024 + lane * 16); };
    if (part > 0) {
#pragma unroll
      for (int i = 0; i < kMTiles; ++i)
#pragma unroll
        for (int t = 0; t < S::kNTiles; ++t) *place(part, i, t) = sum[i][t];
    }
    __syncthreads();
    if (part > 0) return;
    for (int from_part = 1; from_part < kSplit; ++from_part)
#pragma unroll
      for (int i = 0; i < kMTiles; ++i)
#pragma unroll
        for (int t = 0; t < S::kNTiles; ++t) sum[i][t] += *place(from_part, i, t);
  }
  const int32_t n = n0 + wn * 64 + q * 16;
  const bool whole = a.out_type == RADIAL_F32 && n0 + wn * 64 + 64 <= a.N;
  float sb[16], bias[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int32_t at = min(n + e, a.N - 1);
    sb[e] = a.sb[at];
    bias[e] = a.bias ? a.bias[at] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < kMTiles; ++i) {
    const int32_t m = m0 + (wm * kMTiles + i) * 16 + l16;
    const float sa = a.sa[min(m, a.M - 1)];
    float y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = result(sum[i][e >> 2][e & 3], sa * sb[e], bias[e]);
    if (whole) put_fragment(a, m, n0 + wn * 64, q, y);
    else if (m < a.M) put(a, m, n, y, a.N - n);
  }
}

template <int kWavesM, int kWavesN, int kMTiles, int kStages, int kSplit>
int launch_tiles(const ProductArgs& a, hipStream_t stream) {
  using S = TileShape<kWavesM, kWavesN, kMTiles, kStages, kSplit>;
  const int64_t tiles = ((int64_t)a.M + S::kTileM - 1) / S::kTileM * (((int64_t)a.N + S::kTileN - 1) / S::kTileN);
  if (tiles > kMostThreads / (64 * S::kWaves * kSplit)) return fail(RADIAL_ESHAPE, "M*N is too large for one launch");
  if constexpr (S::kLds > 65536) {
    static DeviceOnce configured;
    if (int rc = allow_dynamic_lds(configured, (const void*)product_i8_tile_kernel<kWavesM, kWavesN, kMTiles, kStages, kSplit>, S::kLds)) return rc;
  }
  product_i8_tile_kernel<kWavesM, kWavesN, kMTiles, kStages, kSplit><<<dim3((unsigned)tiles), dim3(64 * S::kWaves * kSplit), S::kLds, stream>>>(a);
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}

int launch_form(int form, const ProductArgs& a, hipStream_t stream) {
  switch (form) {
    case 0: return launch_tiles<2, 4, 8, 2, 1>(a, stream);
    case 1: return launch_tiles<2, 4, 6, 2, 1>(a, stream);
    case 2: return launch_tiles<4, 2, 2, 2, 1>(a, stream);
    case 3: return launch_tiles<4, 2, 2, 3, 1>(a, stream);
    case 4: return launch_tiles<2, 2, 3, 3, 1>(a, stream);
    case 5: return launch_tiles<4, 2, 1, 3, 1>(a, stream);
    case 6: return launch_tiles<4, 1, 1, 3, 1>(a, stream);
    case 7: return launch_tiles<4, 1, 1, 3, 2>(a, stream);
    case 8: return launch_tiles<2, 1, 1, 3, 2>(a, stream);
    default: return launch_tiles<2, 1, 1, 3, 4>(a, stream);
  }
}

// One sum of whole numbers.
int launch_product(const ProductArgs& a, hipStream_t stream) {
  if (takes_pieces_i8(a.M, a.N)) {
    const int64_t tiles = pieces_of(a.M) * pieces_of(a.N);
    if (tiles > kMostThreads / (64 * kParts)) return fail(RADIAL_ESHAPE, "N is too large for one launch");
    product_i8_pieces_kernel<<<dim3((unsigned)tiles), dim3(64 * kParts), 0, stream>>>(a);
    RADIAL_HIP_TRY(hipGetLastError());
    return RADIAL_OK;
  }
  const ProductPlan plan = plan_product_i8(a.M, a.N, a.groups);
  ProductArgs part = a;
  part.M = plan.rows;
  if (int rc = launch_form(plan.form, part, stream)) return rc;
  if (plan.rows == a.M) return RADIAL_OK;
  part.M = a.M - plan.rows;
  part.a += plan.rows * a.a_row;
  part.sa += plan.rows;
  part.out = (char*)part.out + plan.rows * a.out_stride * size_of(a.out_type);
  return launch_form(plan.rest, part, stream);
}

int product_i8(int32_t M, int32_t N, int32_t K, const int8_t* a_codes, int64_t a_pitch, const float* a_scales, const int8_t* b_codes, int64_t b_pitch,
               const float* b_scales, const float* bias, void* out, int32_t out_type, int64_t out_stride, bool accumulate, hipStream_t stream) {
  ProductArgs a = {};
  a.a = a_codes; a.b = b_codes; a.sa = a_scales; a.sb = b_scales; a.bias = bias;
  a.out = out; a.out_type = out_type; a.out_stride = out_stride; a.accumulate = accumulate;
  a.M = M; a.N = N;
  int32_t groups = (int32_t)code_groups(K);
  a.a_row = a_pitch;
  a.b_row = b_pitch;
  a.a_group = a.b_group = kCodeGroup;
  if (K <= kExactCols) {
    a.groups = groups;
    return launch_product(a, stream);
  }
  for (constexpr int32_t kMost = kExactCols / kCodeGroup; groups > 0; groups -= a.groups) {
    a.groups = groups < kMost ? groups : kMost;
    if (int rc = launch_product(a, stream)) return rc;
    a.a += a.groups * a.a_group;
    a.b += a.groups * a.b_group;
    a.bias = nullptr;
    a.accumulate = 1;
  }
  return RADIAL_OK;
}

template <class T>
int launch_few(const ProductArgs& a, const void* x, int64_t stride, int32_t cols, hipStream_t stream) {
  const dim3 grid((unsigned)pieces_of(a.N)), threads(64 * kParts);
  if (pieces_of(a.N) > kMostThreads / (64 * kParts)) return fail(RADIAL_ESHAPE, "N is too large for one launch");
  if (a.M == 1) linear_i8_few_kernel<T, 1><<<grid, threads, 0, stream>>>(a, (const T*)x, stride, cols);
  else if (a.M == 2) linear_i8_few_kernel<T, 2><<<grid, threads, 0, stream>>>(a, (const T*)x, stride, cols);
  else linear_i8_few_kernel<T, kFewRows><<<grid, threads, 0, stream>>>(a, (const T*)x, stride, cols);
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}

int check_sizes(int32_t M, int32_t N, int32_t K) {
  if (M < 1 || N < 1 || K < 1) return fail(RADIAL_EINVAL, "M, N, K must be >= 1");
  if (M > kMostCodeRows || N > kMostCodeRows || K > kMostCodeCols)
    return fail(RADIAL_ESHAPE, "M and N must be at most 2^29 and K 2^23: larger ones are too large for one launch");
  return RADIAL_OK;
}
int check_codes(const void* codes, const void* scales, const char* name) {
  if (!codes || !scales) return fail(RADIAL_EINVAL, "%s codes or scales are NULL", name);
  if ((uintptr_t)codes & 15u) return fail(RADIAL_ESHAPE, "%s codes are not 16-byte aligned", name);
  if ((uintptr_t)scales & 3u) return fail(RADIAL_ESHAPE, "%s scales are not aligned to their elements", name);
  return RADIAL_OK;
}
int check_out(const void* out, int32_t type, int64_t stride, int64_t cols, int64_t depth, bool accumulate, const char* name) {
  if (!out) return fail(RADIAL_EINVAL, "%s is NULL", name);
  if (!is_type(type)) return fail(RADIAL_EINVAL, "the type of %s must be RADIAL_BF16 or RADIAL_F32 (got %d)", name, type);
  if (accumulate && type != RADIAL_F32) return fail(RADIAL_EINVAL, "%s has to be float32 to be added to", name);
  if (depth > kExactCols && type != RADIAL_F32)
    return fail(RADIAL_EUNSUPPORTED, "sums of more than 131071 products are taken in parts: %s has to be float32", name);
  return check_matrix(out, type, stride, cols, name);
}
int check_floats(const void* p, const char* name) {
  return (uintptr_t)p & 3u ? fail(RADIAL_ESHAPE, "%s is not aligned to its elements", name) : RADIAL_OK;
}

// Parts of a workspace, each 256-byte aligned.
struct Parts {
  char* at;
  size_t used = 0;
  template <class T>
  T* take(int64_t count) {
    T* p = (T*)(at + used);
    used += ((size_t)count * sizeof(T) + 255) / 256 * 256;
    return p;
  }
};
struct FwdParts {
  int8_t* codes;
  float* scales;
  FwdParts(Parts& p, int32_t M, int32_t K) : codes(p.take<int8_t>(M * odd_pitch(K))), scales(p.take<float>(M)) {}
};
struct BwdParts {
  int8_t *dy, *dy_t, *x_t;
  float *dy_scales, *dy_t_scales, *x_t_scales;
  char* quantise[2];  // workspaces of the quantiser, for dy and x
  BwdParts(Parts& p, int32_t M, int32_t N, int32_t K) {
    dy = p.take<int8_t>(M * odd_pitch(N));
    dy_t = p.take<int8_t>(N * odd_pitch(M));
    x_t = p.take<int8_t>(K * odd_pitch(M));
    dy_scales = p.take<float>(M);
    dy_t_scales = p.take<float>(N);
    x_t_scales = p.take<float>(K);
    quantise[0] = p.take<char>((int64_t)quantize_i8_workspace(M, N));
    quantise[1] = p.take<char>((int64_t)quantize_i8_workspace(M, K));
  }
};

}  // namespace
}  // namespace radial

using namespace radial;

extern "C" int radial_product_i8(int32_t M, int32_t N, int32_t K, const int8_t* a_codes, const float* a_scales, const int8_t* b_codes,
                                 const float* b_scales, const float* bias, void* out, int32_t out_type, int64_t out_stride, int32_t accumulate,
                                 void* hip_stream) {
  if (int rc = check_sizes(M, N, K)) return rc;
  if (int rc = check_codes(a_codes, a_scales, "a")) return rc;
  if (int rc = check_codes(b_codes, b_scales, "b")) return rc;
  if (int rc = check_out(out, out_type, out_stride, N, K, accumulate != 0, "out")) return rc;
  if (int rc = check_floats(bias, "bias")) return rc;
  const int64_t pitch = code_groups(K) * kCodeGroup;
  return product_i8(M, N, K, a_codes, pitch, a_scales, b_codes, pitch, b_scales, bias, out, out_type, out_stride, accumulate != 0, (hipStream_t)hip_stream);
}

extern "C" size_t radial_linear_i8_fwd_workspace(int32_t M, int32_t N, int32_t K) {
  if (M < 1 || N < 1 || K < 1 || M > kMostCodeRows || N > kMostCodeRows || K > kMostCodeCols) return 0;
  Parts p = {nullptr};
  FwdParts(p, M, K);
  return p.used;
}

extern "C" int radial_linear_i8_fwd(int32_t M, int32_t N, int32_t K, const void* x, int32_t type, int64_t x_stride, const int8_t* w_codes,
                                    const float* w_scales, const float* bias, void* y, int32_t y_type, int64_t y_stride, void* workspace,
                                    size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_sizes(M, N, K)) return rc;
  if (!x) return fail(RADIAL_EINVAL, "x is NULL");
  if (!is_type(type)) return fail(RADIAL_EINVAL, "type must be RADIAL_BF16 or RADIAL_F32 (got %d)", type);
  if (int rc = check_matrix(x, type, x_stride, K, "x")) return rc;
  if (int rc = check_codes(w_codes, w_scales, "w")) return rc;
  if (int rc = check_out(y, y_type, y_stride, N, K, false, "y")) return rc;
  if (int rc = check_floats(bias, "bias")) return rc;
  if (int rc = check_workspace(workspace, workspace_bytes, radial_linear_i8_fwd_workspace(M, N, K))) return rc;
  hipStream_t stream = (hipStream_t)hip_stream;
  if (M <= kFewRows && K <= kFewCols) {
    ProductArgs a = {};
    a.b = w_codes; a.sb = w_scales; a.bias = bias; a.b_row = code_groups(K) * kCodeGroup; a.b_group = kCodeGroup;
    a.out = y; a.out_type = y_type; a.out_stride = y_stride;
    a.M = M; a.N = N; a.groups = (int32_t)code_groups(K);
    return type == RADIAL_F32 ? launch_few<float>(a, x, x_stride, K, stream) : launch_few<__bf16>(a, x, x_stride, K, stream);
  }
  Parts p = {(char*)workspace};
  const FwdParts of(p, M, K);
  QuantI8 q = {};
  q.x = x; q.stride = x_stride; q.rows = M; q.cols = K; q.codes = of.codes; q.pitch = odd_pitch(K); q.scales = of.scales;
  char* none[1] = {nullptr};
  if (int rc = quantize_i8(&q, 1, type, none, stream)) return rc;
  return product_i8(M, N, K, of.codes, odd_pitch(K), of.scales, w_codes, code_groups(K) * kCodeGroup, w_scales, bias, y, y_type, y_stride, false, stream);
}

extern "C" size_t radial_linear_i8_bwd_workspace(int32_t M, int32_t N, int32_t K) {
  if (M < 1 || N < 1 || K < 1 || M > kMostCodeCols || N > kMostCodeCols || K > kMostCodeRows) return 0;
  Parts p = {nullptr};
  BwdParts(p, M, N, K);
  return p.used;
}

extern "C" int radial_linear_i8_bwd(int32_t M, int32_t N, int32_t K, const void* dy, int32_t type, int64_t dy_stride, const void* x,
                                    int64_t x_stride, const int8_t* wt_codes, const float* wt_scales, void* dx, int32_t dx_type, int64_t dx_stride,
                                    void* dw, int32_t dw_type, int64_t dw_stride, float* dbias, int32_t accumulate, void* workspace,
                                    size_t workspace_bytes, void* hip_stream) {
  if (M < 1 || N < 1 || K < 1) return fail(RADIAL_EINVAL, "M, N, K must be >= 1");
  if (M > kMostCodeCols || N > kMostCodeCols || K > kMostCodeRows)
    return fail(RADIAL_ESHAPE, "M and N must be at most 2^23 and K 2^29: larger ones are too large for one launch");
  if (!dy) return fail(RADIAL_EINVAL, "dy is NULL");
  if (!is_type(type)) return fail(RADIAL_EINVAL, "type must be RADIAL_BF16 or RADIAL_F32 (got %d)", type);
  if (int rc = check_matrix(dy, type, dy_stride, N, "dy")) return rc;
  if (!dx && !dw && !dbias) return fail(RADIAL_EINVAL, "none of dx, dw and dbias is given");
  const bool add = accumulate != 0;
  if (dx) {
    if (int rc = check_codes(wt_codes, wt_scales, "wt")) return rc;
    if (int rc = check_out(dx, dx_type, dx_stride, K, N, false, "dx")) return rc;
  }
  if (dw) {
    if (!x) return fail(RADIAL_EINVAL, "x is NULL");
    if (int rc = check_matrix(x, type, x_stride, K, "x")) return rc;
    if (int rc = check_out(dw, dw_type, dw_stride, K, M, add, "dw")) return rc;
  }
  if (int rc = check_floats(dbias, "dbias")) return rc;
  if (int rc = check_workspace(workspace, workspace_bytes, radial_linear_i8_bwd_workspace(M, N, K))) return rc;
  hipStream_t stream = (hipStream_t)hip_stream;
  Parts p = {(char*)workspace};
  const BwdParts of(p, M, N, K);
  QuantI8 q[2] = {};
  q[0].x = dy; q[0].stride = dy_stride; q[0].rows = M; q[0].cols = N; q[0].sums_t = dbias; q[0].accumulate = add;
  if (dx) q[0].codes = of.dy, q[0].pitch = odd_pitch(N), q[0].scales = of.dy_scales;
  if (dw) q[0].codes_t = of.dy_t, q[0].pitch_t = odd_pitch(M), q[0].scales_t = of.dy_t_scales;
  q[1].x = x; q[1].stride = x_stride; q[1].rows = M; q[1].cols = K; q[1].codes_t = of.x_t; q[1].pitch_t = odd_pitch(M); q[1].scales_t = of.x_t_scales;
  if (int rc = quantize_i8(q, dw ? 2 : 1, type, of.quantise, stream)) return rc;
  if (dx) {
    if (int rc = product_i8(M, K, N, of.dy, odd_pitch(N), of.dy_scales, wt_codes, code_groups(N) * kCodeGroup, wt_scales, nullptr, dx, dx_type, dx_stride, false, stream)) return rc;
  }
  if (!dw) return RADIAL_OK;
  return product_i8(N, K, M, of.dy_t, odd_pitch(M), of.dy_t_scales, of.x_t, odd_pitch(M), of.x_t_scales, nullptr, dw, dw_type, dw_stride, add, stream);
}
