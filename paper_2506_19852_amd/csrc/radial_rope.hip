// Rotary positions for gfx950: the table of turns, and queries and keys turned by it (or, for the gradient, back).
//     (u, v) -> (u c - v s, u s + v c),   c, s = magnitude cos, sin of position * frequency of the pair;   gradient: s -> -s
//
// Bound by memory: every element is read and written once.  The table is kept by axis (of a 480p clip 21 x 8 + 30 x 28 + 52 x 28 turns, 20 KiB),
// so it stays in the caches whatever the number of tokens, and a lane loads its turns once for all heads it takes.  q and k of 32 760 tokens x 40 heads x 128
// in bf16, token-major in and head-major out: 247 us, 5.4 TB/s, what a large copy reaches.
#include <math.h>

#include "radial_layer_common.h"

namespace radial {
namespace {

constexpr int kMaxAxes = 3;
constexpr int kMaxHeadDim = 1024;

// ---- table ----------------------------------------------------------------------------------------

struct TableArgs {
  float* table;
  int32_t axes, size[kMaxAxes], dims[kMaxAxes], scaling[kMaxAxes], original[kMaxAxes];
  double factor[kMaxAxes], theta, fast, slow, magnitude;
  int64_t turns;  // of all axes
};

// One thread per turn.  In 64 bits: at position 10^6 a float32 angle would be off by 0.06.
__global__ void __launch_bounds__(256) rope_table_kernel(TableArgs a) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.turns; i += (int64_t)gridDim.x * 256) {
    int64_t at = i;
    int axis = 0;
    for (; axis + 1 < a.axes && at >= (int64_t)a.size[axis] * (a.dims[axis] / 2); ++axis) at -= (int64_t)a.size[axis] * (a.dims[axis] / 2);
    const int32_t pairs = a.dims[axis] / 2;
    const int64_t position = at / pairs;
    const double share = (double)(at % pairs) / pairs;  // 2 j / dims
    double theta = a.theta;
    if (a.scaling[axis] == RADIAL_ROPE_SCALE_BASE && pairs > 1) theta *= pow(a.factor[axis], (double)pairs / (pairs - 1));
    double f = pow(theta, -share);
    if (a.scaling[axis] == RADIAL_ROPE_SCALE_LINEAR) f /= a.factor[axis];
    if (a.scaling[axis] == RADIAL_ROPE_SCALE_PARTS) {
      const double turns = a.original[axis] * f / (2.0 * M_PI);
      const double keep = fmin(1.0, fmax(0.0, (turns - a.slow) / (a.fast - a.slow)));
      f *= keep + (1.0 - keep) / a.factor[axis];
    }
    double s, c;
    sincos((double)position * f, &s, &c);
    a.table[2 * i] = (float)(a.magnitude * c);
    a.table[2 * i + 1] = (float)(a.magnitude * s);
  }
}

// ---- turns ----------------------------------------------------------------------------------------

struct HeadsArg {
  const char* in;
  char* out;
  int64_t isb, ish, isn, osb, osh, osn;  // strides in elements
};

struct RopeArgs {
  HeadsArg x[2];          // q, k
  int32_t heads[2];
  const float* table;
  const int32_t* positions;
  int32_t first;
  int32_t B, N, D;
  int32_t size1, size2;   // positions of the second and third axis (1 without)
  int32_t total;          // positions of the grid
  int32_t pair_end[2];    // pairs of the first axis, of the first two
  int32_t pairs;          // of all axes
  int32_t axis_pairs[3];
  int64_t axis_at[3];     // floats before the axis in the table
  int32_t units;          // pieces of a head that a lane takes
  int32_t heads_each;     // heads a lane takes
  float sign;             // +1 forward, -1 gradient
};

// Where a token lies on each axis; on = false: it is copied.
struct Place {
  int64_t row[3];  // floats from the table's start to the token's turns on the axis
  bool on;
};

__device__ __forceinline__ Place place_of(const RopeArgs& a, int32_t b, int32_t n) {
  Place p;
  const int64_t index = a.positions ? (int64_t)a.positions[(int64_t)b * a.N + n] : (int64_t)a.first + n;
  p.on = index >= 0 && index < a.total;
  const uint32_t i = p.on ? (uint32_t)index : 0u;
  const uint32_t two = i / (uint32_t)a.size2, at2 = i - two * (uint32_t)a.size2;
  const uint32_t at0 = two / (uint32_t)a.size1, at1 = two - at0 * (uint32_t)a.size1;
  p.row[0] = a.axis_at[0] + (int64_t)at0 * a.axis_pairs[0] * 2;
  p.row[1] = a.axis_at[1] + (int64_t)at1 * a.axis_pairs[1] * 2;
  p.row[2] = a.axis_at[2] + (int64_t)at2 * a.axis_pairs[2] * 2;
  return p;
}

// Turn of a pair: cos and sin.
__device__ __forceinline__ f32x2 turn_of(const RopeArgs& a, const Place& p, int32_t pair) {
  const int axis = (pair >= a.pair_end[0]) + (pair >= a.pair_end[1]);
  const int32_t base = axis == 0 ? 0 : a.pair_end[axis - 1];
  const int64_t row = axis == 0 ? p.row[0] : axis == 1 ? p.row[1] : p.row[2];
  const f32x2 t = *(const f32x2*)(a.table + row + 2 * (pair - base));
  return f32x2{t[0], t[1] * a.sign};
}

enum class Pieces {
  kInterleaved,  // eight dimensions in a row: four pairs
  kHalf,         // eight pairs, dimensions 8u .. and R/2 + 8u ..; behind them eight dimensions that stay
  kHalfAny,      // the same where R/2 is no multiple of eight: the last of the pairs, and of the dimensions that stay, may be fewer, at any address
};

// Waves of a SIMD.  Whole pieces of halves read two places of a head each: 40 + 40 bf16 heads of 32 760 tokens took 284 us with five waves, 290 with the six that
// their registers allow.
constexpr int most_waves(Pieces pieces) { return pieces == Pieces::kHalf ? 5 : 8; }

// One thread per token and piece of a head; heads heads_each at a time.  Turns are rounded once, at the end.
template <class T, Pieces kPieces>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, most_waves(kPieces)))) rope_kernel(RopeArgs a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (int64_t)a.B * a.N * a.units) return;
  const int32_t unit = (int32_t)(id % a.units);
  const int64_t token = id / a.units;
  const int32_t b = (int32_t)(token / a.N), n = (int32_t)(token % a.N);
  const Place place = place_of(a, b, n);
  const int32_t rotated = 2 * a.pairs;

  constexpr bool kAny = kPieces == Pieces::kHalfAny;
  constexpr int kPairs = kPieces == Pieces::kInterleaved ? 4 : 8;
  const int32_t pair0 = unit * kPairs;
  const bool stays = kPieces != Pieces::kInterleaved && pair0 >= a.pairs;  // a piece behind the pairs
  // Pairs of the piece that turn.  The rest is copied as it lies in memory: turned by 1 and 0 it would carry an infinity from one of a pair to the other,
  // and a signalling bf16 NaN that passes through float32 comes back quiet.
  const int32_t turning = place.on ? max(0, min(kPairs, a.pairs - pair0)) : 0;
  f32x2 turn[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) turn[i] = i < turning ? turn_of(a, place, pair0 + i) : f32x2{1.f, 0.f};
  // dimensions of the piece's first and second part
  int32_t one, two = 0, count = 8;  // count: dimensions of either
  if (kPieces == Pieces::kInterleaved) one = 8 * unit;
  else if (stays) one = rotated + 8 * (unit - (a.pairs + 7) / 8);
  else { one = pair0; two = a.pairs + pair0; }
  if (kAny) count = min(8, stays ? a.D - one : a.pairs - pair0);

  const int32_t all = a.heads[0] + a.heads[1];
  const int32_t h0 = blockIdx.y * a.heads_each, h1 = min(h0 + a.heads_each, all);
  constexpr int kAtOnce = 4;
  for (int32_t h = h0; h < h1; h += kAtOnce) {
    const T* in[kAtOnce];
    T* out[kAtOnce];
    Eight<T> lo[kAtOnce], hi[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int32_t head = min(h + j, h1 - 1);
      const int which = head >= a.heads[0];
      const HeadsArg& x = a.x[which];
      const int32_t hh = head - (which ? a.heads[0] : 0);
      in[j] = (const T*)x.in + b * x.isb + hh * x.ish + n * x.isn;
      out[j] = (T*)x.out + b * x.osb + hh * x.osh + n * x.osn;
      if (h + j >= h1) continue;
      if constexpr (kAny) {
        const int32_t whole = stays ? a.D - rotated : a.pairs, back = whole < 8 ? 0 : 8 - count;
        if (whole < 8) {
          lo[j].load_some(in[j] + one, count);
          hi[j].load_some(in[j] + two, stays ? 0 : count);
        } else {
          lo[j].load_any(in[j] + one - back);
          if (!stays) hi[j].load_any(in[j] + two - back);
        }
      } else {
        lo[j].load(in[j] + one);
        if (kPieces == Pieces::kHalf && !stays) hi[j].load(in[j] + two);
      }
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      if (h + j >= h1) continue;
      if constexpr (kPieces == Pieces::kInterleaved) {
        float v[8];
        lo[j].get(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = v[2 * i], y = v[2 * i + 1];
          lo[j].set_pair(i, i < turning, x * turn[i][0] - y * turn[i][1], x * turn[i][1] + y * turn[i][0]);
        }
        lo[j].put(out[j] + one);
      } else {
        if (kAny && count < 8 && (stays ? a.D - rotated : a.pairs) >= 8) {
          lo[j].drop(8 - count);
          if (!stays) hi[j].drop(8 - count);
        }
        if (stays) {
          if (kAny) lo[j].put_some(out[j] + one, count);
          else lo[j].put(out[j] + one);
        } else {
          float u[8], v[8];
          lo[j].get(u);
          hi[j].get(v);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float x = u[i], y = v[i];
            u[i] = x * turn[i][0] - y * turn[i][1];
            v[i] = x * turn[i][1] + y * turn[i][0];
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            lo[j].set_pair(i, turning, u[2 * i], u[2 * i + 1]);
            hi[j].set_pair(i, turning, v[2 * i], v[2 * i + 1]);
          }
          if (kAny) {
            lo[j].put_some(out[j] + one, count);
            hi[j].put_some(out[j] + two, count);
          } else {
            lo[j].put(out[j] + one);
            hi[j].put(out[j] + two);
          }
        }
      }
    }
  }
}

// ---- checks ---------------------------------------------------------------------------------------

int check_params(const radial_rope_params* p) {
  if (!p) return fail(RADIAL_EINVAL, "params is NULL");
  if (p->axes < 1 || p->axes > kMaxAxes) return fail(RADIAL_EINVAL, "axes must be 1 to 3 (got %d)", p->axes);
  if (p->layout != RADIAL_ROPE_INTERLEAVED && p->layout != RADIAL_ROPE_HALF) return fail(RADIAL_EINVAL, "unknown layout %d", p->layout);
  int64_t total = 1, rotated = 0;
  for (int i = 0; i < p->axes; ++i) {
    if (p->size[i] < 1) return fail(RADIAL_EINVAL, "size[%d] must be >= 1", i);
    total *= p->size[i];
    if (total > 0x7fffffffLL) return fail(RADIAL_EINVAL, "the grid must have below 2^31 positions");
    if (p->dims[i] < 2 || p->dims[i] % 2 || p->dims[i] > kMaxHeadDim) return fail(RADIAL_EINVAL, "dims[%d] must be even, 2 to %d", i, kMaxHeadDim);
    rotated += p->dims[i];
    if (p->scaling[i] < RADIAL_ROPE_SCALE_NONE || p->scaling[i] > RADIAL_ROPE_SCALE_PARTS) return fail(RADIAL_EINVAL, "unknown scaling[%d] %d", i, p->scaling[i]);
    if (p->scaling[i] != RADIAL_ROPE_SCALE_NONE && (!(p->factor[i] > 0.0) || !isfinite(p->factor[i]))) return fail(RADIAL_EINVAL, "factor[%d] must be positive and finite", i);
    if (p->scaling[i] == RADIAL_ROPE_SCALE_PARTS) {
      if (p->original[i] < 1) return fail(RADIAL_EINVAL, "original[%d] must be >= 1", i);
      if (!(p->slow >= 0.0) || !(p->fast > p->slow) || !isfinite(p->fast)) return fail(RADIAL_EINVAL, "fast must be finite and above slow, slow not negative");
    }
  }
  if (rotated > kMaxHeadDim) return fail(RADIAL_EINVAL, "the axes turn %lld dimensions, at most %d are supported", (long long)rotated, kMaxHeadDim);
  if (!(p->theta > 0.0) || !isfinite(p->theta)) return fail(RADIAL_EINVAL, "theta must be positive and finite");
  if (!isfinite(p->magnitude)) return fail(RADIAL_EINVAL, "magnitude must be finite");
  return RADIAL_OK;
}

int64_t turns_of(const radial_rope_params& p) {
  int64_t n = 0;
  for (int i = 0; i < p.axes; ++i) n += (int64_t)p.size[i] * (p.dims[i] / 2);
  return n;
}

int check_heads(const char* name, const radial_tensor& t, int32_t D) {
  if (!t.ptr) return fail(RADIAL_EINVAL, "%s.ptr is NULL", name);
  if ((uintptr_t)t.ptr & 15u) return fail(RADIAL_ESHAPE, "%s.ptr is not 16-byte aligned", name);
  if (t.stride_n < D || (t.stride_n & 7) || (t.stride_h & 7) || (t.stride_b & 7) || t.stride_h < 0 || t.stride_b < 0)
    return fail(RADIAL_ESHAPE, "%s strides must be non-negative multiples of 8 elements with stride_n >= D", name);
  return RADIAL_OK;
}

HeadsArg heads_arg(const radial_tensor& in, const radial_tensor& out) {
  return HeadsArg{(const char*)in.ptr, (char*)out.ptr, in.stride_b, in.stride_h, in.stride_n, out.stride_b, out.stride_h, out.stride_n};
}

template <class T>
void launch(const RopeArgs& a, Pieces pieces, dim3 grid, hipStream_t stream) {
  if (pieces == Pieces::kInterleaved) rope_kernel<T, Pieces::kInterleaved><<<grid, dim3(256), 0, stream>>>(a);
  else if (pieces == Pieces::kHalf) rope_kernel<T, Pieces::kHalf><<<grid, dim3(256), 0, stream>>>(a);
  else rope_kernel<T, Pieces::kHalfAny><<<grid, dim3(256), 0, stream>>>(a);
}

int check_table(const radial_rope_params& p, const float* table, size_t bytes) {
  if (!table) return fail(RADIAL_EINVAL, "table is NULL");
  if ((uintptr_t)table & 15u) return fail(RADIAL_ESHAPE, "table is not 16-byte aligned");
  const size_t need = (size_t)turns_of(p) * 2 * sizeof(float);
  return bytes >= need ? RADIAL_OK : fail(RADIAL_ESHAPE, "table holds %zu bytes, %zu needed", bytes, need);
}

int turn(const radial_rope_params* params, const float* table, size_t table_bytes, int32_t B, int32_t N, int32_t D, int32_t q_heads, radial_tensor q,
         radial_tensor q_out, int32_t k_heads, radial_tensor k, radial_tensor k_out, int32_t type, const int32_t* positions, int32_t first,
         bool gradient, void* hip_stream) {
  if (int rc = check_params(params)) return rc;
  const radial_rope_params& p = *params;
  if (int rc = check_table(p, table, table_bytes)) return rc;
  if (B < 1 || N < 1 || q_heads < 1) return fail(RADIAL_EINVAL, "B, N, q_heads must be >= 1");
  if (D < 8 || D % 8 || D > kMaxHeadDim) return fail(RADIAL_EUNSUPPORTED, "head dimension must be a multiple of 8 up to %d (got %d)", kMaxHeadDim, D);
  if (!is_type(type)) return fail(RADIAL_EINVAL, "type must be RADIAL_BF16 or RADIAL_F32 (got %d)", type);
  if (int rc = check_heads(gradient ? "dq_out" : "q", q, D)) return rc;
  if (int rc = check_heads(gradient ? "dq" : "q_out", q_out, D)) return rc;
  if (k.ptr || k_out.ptr || k_heads) {
    if (k_heads < 1) return fail(RADIAL_EINVAL, "k_heads must be >= 1 where there are keys");
    if (int rc = check_heads(gradient ? "dk_out" : "k", k, D)) return rc;
    if (int rc = check_heads(gradient ? "dk" : "k_out", k_out, D)) return rc;
  }
  if (!positions && first < 0) return fail(RADIAL_EINVAL, "first must not be negative");
  if (positions && ((uintptr_t)positions & 3u)) return fail(RADIAL_ESHAPE, "positions is not aligned to its elements");

  RopeArgs a = {};
  a.x[0] = heads_arg(q, q_out);
  if (k_heads) a.x[1] = heads_arg(k, k_out);
  a.heads[0] = q_heads; a.heads[1] = k_heads;
  a.table = table; a.positions = positions; a.first = first;
  a.B = B; a.N = N; a.D = D;
  a.size1 = p.axes > 1 ? p.size[1] : 1;
  a.size2 = p.axes > 2 ? p.size[2] : 1;
  a.total = p.size[0] * a.size1 * a.size2;
  int64_t at = 0;
  for (int i = 0; i < kMaxAxes; ++i) {
    a.axis_pairs[i] = i < p.axes ? p.dims[i] / 2 : 0;
    a.axis_at[i] = at;
    if (i < p.axes) at += (int64_t)p.size[i] * p.dims[i];
    a.pairs += a.axis_pairs[i];
    if (i < 2) a.pair_end[i] = a.pairs;
  }
  if (2 * a.pairs > D) return fail(RADIAL_ESHAPE, "the axes turn %d dimensions, the heads have %d", 2 * a.pairs, D);
  a.sign = gradient ? -1.f : 1.f;
  const Pieces pieces = p.layout == RADIAL_ROPE_INTERLEAVED ? Pieces::kInterleaved : a.pairs % 8 == 0 ? Pieces::kHalf : Pieces::kHalfAny;
  a.units = pieces == Pieces::kInterleaved ? D / 8 : (a.pairs + 7) / 8 + (D - 2 * a.pairs + 7) / 8;
  const int64_t heads = (int64_t)q_heads + k_heads;
  if ((int64_t)B * N > kMostThreads / a.units) return fail(RADIAL_ESHAPE, "B*N*D is too large for one launch");
  const int64_t lanes = (int64_t)B * N * a.units;
  a.heads_each = 8;
  const int64_t groups = (lanes + 255) / 256;
  // few tokens: heads over more lanes, until there are some for every compute unit
  while (a.heads_each > 1 && groups * ((heads + a.heads_each - 1) / a.heads_each) < 1024) a.heads_each /= 2;
  const int64_t parts = (heads + a.heads_each - 1) / a.heads_each;
  if (parts > 65535) return fail(RADIAL_ESHAPE, "too many heads for one launch");
  const dim3 grid((unsigned)groups, (unsigned)parts);
  if (type == RADIAL_F32) launch<float>(a, pieces, grid, (hipStream_t)hip_stream);
  else launch<__bf16>(a, pieces, grid, (hipStream_t)hip_stream);
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}

}  // namespace
}  // namespace radial

using namespace radial;

extern "C" size_t radial_rope_table_bytes(const radial_rope_params* params) {
  return check_params(params) == RADIAL_OK ? (size_t)turns_of(*params) * 2 * sizeof(float) : 0;
}

extern "C" int radial_rope_table(const radial_rope_params* params, float* table, size_t table_bytes, void* hip_stream) {
  if (int rc = check_params(params)) return rc;
  const radial_rope_params& p = *params;
  if (int rc = check_table(p, table, table_bytes)) return rc;
  TableArgs a = {};
  a.table = table;
  a.axes = p.axes;
  for (int i = 0; i < p.axes; ++i) {
    a.size[i] = p.size[i]; a.dims[i] = p.dims[i]; a.scaling[i] = p.scaling[i]; a.original[i] = p.original[i]; a.factor[i] = p.factor[i];
  }
  a.theta = p.theta; a.fast = p.fast; a.slow = p.slow; a.magnitude = p.magnitude;
  a.turns = turns_of(p);
  const int64_t grid = (a.turns + 255) / 256;
  rope_table_kernel<<<dim3((unsigned)(grid < 65536 ? grid : 65536)), dim3(256), 0, (hipStream_t)hip_stream>>>(a);
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}

extern "C" int radial_rope_fwd(const radial_rope_params* params, const float* table, size_t table_bytes, int32_t B, int32_t N, int32_t D, int32_t q_heads, radial_tensor q,
                               radial_tensor q_out, int32_t k_heads, radial_tensor k, radial_tensor k_out, int32_t type, const int32_t* positions,
                               int32_t first, void* hip_stream) {
  return turn(params, table, table_bytes, B, N, D, q_heads, q, q_out, k_heads, k, k_out, type, positions, first, false, hip_stream);
}

extern "C" int radial_rope_bwd(const radial_rope_params* params, const float* table, size_t table_bytes, int32_t B, int32_t N, int32_t D, int32_t q_heads, radial_tensor dq_out,
                               radial_tensor dq, int32_t k_heads, radial_tensor dk_out, radial_tensor dk, int32_t type, const int32_t* positions,
                               int32_t first, void* hip_stream) {
  return turn(params, table, table_bytes, B, N, D, q_heads, dq_out, dq, k_heads, dk_out, dk, type, positions, first, true, hip_stream);
}
