// Gated residual and norms for gfx950, forward and backward.  For a token (row) of C channels, with a conditioning row shared by `group` tokens:
//     u = N_post(y) w_post,   r = a x + g u,   z = N_pre(r) w (1 + s) + t
//     N(v) = (v - mean) / sqrt(var + eps)   or   v / sqrt(mean(v^2) + eps)
// and, with n = N_pre(r), m = N_post(y), 1/size the two norms' factors, and D the whole gradient of r:
//     d = dz w (1 + s),   D = dr + (d - mean(d) - n mean(d n)) / size,   dx = a D      (mean(d) for layer norms only)
//     e = D g w_post,     dy = (e - mean(e) - m mean(e m)) / size_y                    (dy = e without a norm)
//     P = sum dz n, T = sum dz, Q = sum D m over a group's tokens:
//     ds = P w,  dt = T,  dg = Q w_post,  dw = sum over groups P (1 + s),  dw_post = sum over groups Q g.
//
// Both passes are bound by memory up to 8192 channels: each tensor is read or written once and a row stays in registers between its statistics and its results.
// A team of lanes takes a row: 16, 32 or 64 lanes with eight channels each up to 512 channels, from there all waves of the workgroup.  A thread
// has the same channels in all rows of its workgroup, so that it loads the conditioning row once and keeps the sums over tokens in registers; a
// workgroup's rows are of one group.  The backward writes a workgroup's sums to the workspace, where a second kernel adds them up
// in a fixed order (no atomics).  32 760 x 5120 in bf16, residual and layer norm: forward 251-267 us (5.0-5.3 TB/s, what a large copy reaches), backward
// 408-413 us (4.9 TB/s), with a second norm 261 and 418; 20 475 x 8192, the same bytes, 259 and 418.
//
// From 8193 to 16 384 channels a thread has 32 of them, and the gradients' sums, conditioning and rows do not fit its 256 registers: 470 to 640 bytes of a lane's values
// (550 to 800 where rows are not aligned) go through scratch memory for every token.  The gradients of 20 455 x 8200 take 1597 us against a copy's 380,
// of 13 650 x 12 288 1208, of 10 237 x 16 384 1057 (bf16; float32 2676, 2028, 1984 against 760).  The forward fits but for float32 branches (up to 100 bytes): 285, 273, 274 us of 253
// (650, 593, 585 of 506).  Gradients of float32 rows of more than 4096 channels keep eight bytes there, which costs nothing (813-818 us of 760 at 8192).
#include <float.h>
#include <math.h>

#include "radial_layer_common.h"

namespace radial {
namespace {

constexpr int kMaxChannels = 16384;

struct RowsArg {
  char* ptr;
  int64_t sb, sn;  // elements
};

struct NormArgs {
  RowsArg x, y, r, z;        // forward; backward: r, y read, z = dz
  RowsArg dr, dx, dy;        // backward
  const float *gate, *post_weight, *weight, *scale, *shift;
  float* partial;            // backward: [groups][chunks][3][C] sums P, T, Q of a workgroup's rows
  int32_t N, C, group, groups_of_batch;
  int32_t chunks, rows;      // workgroups that share a group, tokens of each
  int32_t post, pre;
  float eps, residual_scale;
  int64_t mod_stride;
  int32_t wants;             // backward: bits of the sums that are wanted: 1 P, 2 T, 4 Q
};

// Where the waves of a team that is the whole workgroup meet: up to four values of each, zero where there is no wave.  `turn` alternates between two
// places, so that one barrier does for each meeting (who writes a place again has passed the barrier of the meeting between, behind all
// reads of it).
constexpr int kMaxWaves = 8;
struct Meeting {
  f32x4 place[2][kMaxWaves];
};

// The channels of a thread: 8 V of them, eight in a row, V times, a team's width apart.  kVec: rows are 16-byte aligned and of whole eights;
// otherwise they start anywhere and the last eight may be fewer.
template <bool kVec, int V>
struct Channels {
  int32_t first, width, C;
  __device__ __forceinline__ int32_t at(int v, int e) const { return (v * width + first) * 8 + e; }
  __device__ __forceinline__ bool has(int v, int e) const { return at(v, kVec ? 0 : e) < C; }
  __device__ __forceinline__ int32_t count() const {
    int32_t n = 0;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) n += has(v, e);
    return n;
  }
};

// A thread's channels of a row, as they lie in memory.
template <class T, bool kVec, int V>
struct Held {
  Eight<T> piece[V];
  __device__ __forceinline__ void load(const T* row, const Channels<kVec, V>& ch) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (kVec) {
        if (ch.has(v, 0)) piece[v].load(row + ch.at(v, 0));
        else piece[v].clear();
      } else if (ch.C < 8) {
        piece[v].load_some(row + ch.at(v, 0), ch.C - ch.at(v, 0));
      } else {
        if (ch.has(v, 0)) piece[v].load_any(row + min(ch.at(v, 0), ch.C - 8));
        else piece[v].clear();
      }
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int v = 0; v < V; ++v) piece[v].clear();
  }
  __device__ __forceinline__ void get(float (&out)[8 * V], const Channels<kVec, V>& ch) const {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float e8[8];
      Eight<T> eight = piece[v];
      if (!kVec && ch.C >= 8 && ch.has(v, 0) && ch.at(v, 8) > ch.C) eight.drop(ch.at(v, 8) - ch.C);
      eight.get(e8);
#pragma unroll
      for (int e = 0; e < 8; ++e) out[8 * v + e] = e8[e];
    }
  }
};

template <class T, bool kVec, int V>
__device__ __forceinline__ void store_row(T* row, const float (&val)[8 * V], const Channels<kVec, V>& ch) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float e8[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) e8[e] = val[8 * v + e];
    if constexpr (kVec) {
      if (ch.has(v, 0)) Eight<T>::store(row + ch.at(v, 0), e8);
    } else {
      Eight<T>::store_some(row + ch.at(v, 0), e8, ch.C - ch.at(v, 0));
    }
  }
}

// A conditioning row or a weight, `missing` where it is not given.
template <bool kVec, int V>
__device__ __forceinline__ void load_mod(float (&out)[8 * V], const float* row, float missing, const Channels<kVec, V>& ch) {
  if (row) {
    Held<float, kVec, V> h;
    h.load(row, ch);
    h.get(out, ch);
  } else {
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) out[i] = missing;
  }
}

// Rows of a team and its sums.  kWide: the team is the workgroup; otherwise L lanes.  kFast: fewer instructions and waits for more registers (what the
// waves left is read at once, channels are masked an eight at a time): the gradients at 5120 channels, where only eight waves fit a compute unit
// anyway, took 443 us instead of 482; the forward, which loses a wave of four by it, 276 instead of 256, the gradients at 1536 channels 175 instead of 154.
template <bool kWide, int L, bool kFast>
struct Team {
  static constexpr bool kExchanges = kWide, kEights = kFast;
  Meeting* meet;
  int32_t turn, wave, waves;
  float of_C;  // 1 / channels of a row
  __device__ __forceinline__ float lanes(float x) const { return lane_sum<kWide ? 64 : L>(x); }
  // Every wave's values to every wave: add(values) for one after the other.
  template <class Add>
  __device__ __forceinline__ void each(Add&& add) const {
    if constexpr (kFast) {
      f32x4 all[kMaxWaves];
#pragma unroll
      for (int w = 0; w < kMaxWaves; ++w) all[w] = meet->place[turn][w];
#pragma unroll
      for (int w = 0; w < kMaxWaves; ++w) add(all[w]);
    } else {
#pragma unroll 1
      for (int w = 0; w < waves; ++w) add(meet->place[turn][w]);
    }
  }
  __device__ __forceinline__ void exchange(f32x4 mine) {
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) meet->place[turn][wave] = mine;
    __syncthreads();
  }
};

// Mean and 1/size of the row, from `val` (zero beyond the channels).  A layer norm's variance is taken about the mean of the wave's own channels and then
// moved to the row's (sum (v - m)^2 = sum (v - m_w)^2 + n_w (m_w - m)^2 per wave): no cancellation where the mean is large, and one exchange instead of two.
template <int E>
__device__ __forceinline__ float sum_of(const float (&val)[E]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) s += val[i];
  return s;
}
// Masked one by one, or (kEights: vectors) an eight at a time.
template <bool kVec, int V, bool kEights>
__device__ __forceinline__ float squares_about(const float (&val)[8 * V], float mean, const Channels<kVec, V>& ch) {
  float s = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float of_eight = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = kEights || ch.has(v, e) ? val[8 * v + e] - mean : 0.f;
      if (kEights) of_eight = __builtin_fmaf(d, d, of_eight);
      else s = __builtin_fmaf(d, d, s);
    }
    if (kEights) s += ch.has(v, 0) ? of_eight : 0.f;
  }
  return s;
}

template <bool kVec, int V, class T>
__device__ __forceinline__ void statistics(const float (&val)[8 * V], int32_t kind, float eps, T& team, const Channels<kVec, V>& ch, float own_count,
                                           float of_own, float& mean, float& inverse) {
  mean = 0.f;
  float about = 0.f;
  if (kind == RADIAL_NORM_LAYER) about = team.lanes(sum_of(val)) * of_own;
  float squares = team.lanes(squares_about<kVec, V, T::kEights>(val, about, ch));
  if constexpr (T::kExchanges) {
    team.exchange(f32x4{about * own_count, squares, own_count, about});
    squares = 0.f;
    team.each([&](f32x4 theirs) {
      mean += theirs[0];
      squares += theirs[1];
    });
    mean *= team.of_C;
    if (kind == RADIAL_NORM_LAYER)
      team.each([&](f32x4 theirs) {
        const float d = theirs[3] - mean;
        squares = __builtin_fmaf(theirs[2] * d, d, squares);
      });
  } else {
    mean = about;
  }
  inverse = __builtin_amdgcn_rsqf(squares * team.of_C + eps);  // to one unit; eps is a normal number
}

// v <- (v - mean) inverse, zero where there is no channel.
template <bool kVec, int V, bool kEights>
__device__ __forceinline__ void normalise(float (&val)[8 * V], float mean, float inverse, const Channels<kVec, V>& ch) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float factor = !kEights || ch.has(v, 0) ? inverse : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) val[8 * v + e] = kEights || ch.has(v, e) ? (val[8 * v + e] - mean) * factor : 0.f;
  }
}

// Two sums over the row at once.
template <class T>
__device__ __forceinline__ void two_sums(float& a, float& b, T& team) {
  a = team.lanes(a);
  b = team.lanes(b);
  if constexpr (T::kExchanges) {
    team.exchange(f32x4{a, b, 0.f, 0.f});
    a = b = 0.f;
    team.each([&](f32x4 theirs) {
      a += theirs[0];
      b += theirs[1];
    });
  }
}

// What a workgroup works on.
template <bool kVec, int V, bool kWide, int L, bool kFast>
struct Share {
  Channels<kVec, V> ch;
  Team<kWide, L, kFast> team;
  int32_t teams, first, last;  // rows first, first + teams, ... below last, of batch b
  int32_t b, group;            // group: b * groups_of_batch + g
  float own_count, of_own;     // channels of this wave (wide) or of the row, and 1 / them
  __device__ __forceinline__ Share(const NormArgs& a, Meeting* meet) {
    group = blockIdx.x / a.chunks;
    const int32_t chunk = blockIdx.x % a.chunks;
    b = group / a.groups_of_batch;
    const int32_t g = group % a.groups_of_batch;
    const int64_t begin = (int64_t)g * a.group + (int64_t)chunk * a.rows;
    const int64_t end = min(min(begin + a.rows, (int64_t)(g + 1) * a.group), (int64_t)a.N);
    teams = kWide ? 1 : blockDim.x / L;
    first = (int32_t)min(begin, (int64_t)a.N) + (kWide ? 0 : threadIdx.x / L);
    last = (int32_t)max(end, (int64_t)0);
    ch.first = kWide ? threadIdx.x : threadIdx.x % L;
    ch.width = kWide ? blockDim.x : L;
    ch.C = a.C;
    team.meet = meet;
    if (kWide) {
      if (threadIdx.x < 2 * kMaxWaves) meet->place[threadIdx.x / kMaxWaves][threadIdx.x % kMaxWaves] = f32x4{0.f, 0.f, 0.f, 0.f};
      __syncthreads();
    }
    team.turn = 0;
    team.wave = threadIdx.x >> 6;
    team.waves = (blockDim.x + 63) >> 6;
    team.of_C = 1.f / (float)a.C;
    own_count = team.lanes((float)ch.count());
    of_own = 1.f / fmaxf(own_count, 1.f);
  }
};

template <class T>
__device__ __forceinline__ T* row_of(const RowsArg& t, int32_t b, int32_t n) {
  return (T*)t.ptr + (int64_t)b * t.sb + (int64_t)n * t.sn;
}

template <class XT, class YT, bool kVec, int V, bool kWide, int L>
__global__ void __launch_bounds__(kWide ? 512 : 256) norm_fwd_kernel(NormArgs a) {
  __shared__ Meeting meet;
  Share<kVec, V, kWide, L, false> s(a, &meet);
  constexpr int E = 8 * V;
  const int64_t mod = (int64_t)s.group * a.mod_stride;
  float gate[E], factor[E], shift[E];
  {
    float w[E];
    load_mod<kVec, V>(gate, a.gate ? a.gate + mod : nullptr, 1.f, s.ch);
    load_mod<kVec, V>(w, a.post_weight, 1.f, s.ch);
#pragma unroll
    for (int i = 0; i < E; ++i) gate[i] *= w[i];
    load_mod<kVec, V>(factor, a.scale ? a.scale + mod : nullptr, 0.f, s.ch);
    load_mod<kVec, V>(w, a.weight, 1.f, s.ch);
#pragma unroll
    for (int i = 0; i < E; ++i) factor[i] = (1.f + factor[i]) * w[i];
    load_mod<kVec, V>(shift, a.shift ? a.shift + mod : nullptr, 0.f, s.ch);
  }
  // The next row is fetched while one is worked on.
  Held<XT, kVec, V> x, next_x;
  Held<YT, kVec, V> y, next_y;
  auto fetch = [&](int32_t n) __attribute__((always_inline)) {
    if (n >= s.last) return;
    next_x.load(row_of<XT>(a.x, s.b, n), s.ch);
    if (a.y.ptr) next_y.load(row_of<YT>(a.y, s.b, n), s.ch);
  };
  next_x.clear();
  next_y.clear();
  fetch(s.first);
  // Teams of a wave end together: a team without a row left works on its last one again and stores nothing.
  for (int32_t n = s.first; kWide ? n < s.last : __any(n < s.last); n += s.teams) {
    const bool live = kWide || n < s.last;
    x = next_x;
    y = next_y;
    fetch(n + s.teams);
    float r[E];
    x.get(r, s.ch);
    if (a.y.ptr) {
      float u[E];
      y.get(u, s.ch);
      if (a.post != RADIAL_NORM_NONE) {
        float mean, inverse;
        statistics<kVec, V>(u, a.post, a.eps, s.team, s.ch, s.own_count, s.of_own, mean, inverse);
#pragma unroll
        for (int i = 0; i < E; ++i) u[i] = (u[i] - mean) * inverse;
      }
#pragma unroll
      for (int i = 0; i < E; ++i) r[i] = s.ch.has(i / 8, i % 8) ? a.residual_scale * r[i] + gate[i] * u[i] : 0.f;
      if (live) store_row<XT, kVec, V>(row_of<XT>(a.r, s.b, n), r, s.ch);
    }
    if (a.pre != RADIAL_NORM_NONE) {
      float mean, inverse;
      statistics<kVec, V>(r, a.pre, a.eps, s.team, s.ch, s.own_count, s.of_own, mean, inverse);
#pragma unroll
      for (int i = 0; i < E; ++i) r[i] = (r[i] - mean) * inverse * factor[i] + shift[i];
      if (live) store_row<YT, kVec, V>(row_of<YT>(a.z, s.b, n), r, s.ch);
    }
  }
}

template <class XT, class YT, bool kVec, int V, bool kWide, int L>
__global__ void __launch_bounds__(kWide ? 512 : 256) norm_bwd_kernel(NormArgs a) {
  __shared__ Meeting meet;
  __shared__ float merged[kWide ? 1 : 3][kWide ? 1 : 256 * 8];
  constexpr bool kFast = kVec && kWide && V == 2;
  Share<kVec, V, kWide, L, kFast> s(a, &meet);
  constexpr int E = 8 * V;
  const int64_t mod = (int64_t)s.group * a.mod_stride;
  const bool has_y = a.y.ptr != nullptr, has_z = a.z.ptr != nullptr;
  float gate[E], factor[E];
  {
    float w[E];
    load_mod<kVec, V>(gate, a.gate ? a.gate + mod : nullptr, 1.f, s.ch);
    load_mod<kVec, V>(w, a.post_weight, 1.f, s.ch);
#pragma unroll
    for (int i = 0; i < E; ++i) gate[i] = s.ch.has(i / 8, i % 8) ? gate[i] * w[i] : 0.f;
    load_mod<kVec, V>(factor, a.scale ? a.scale + mod : nullptr, 0.f, s.ch);
    load_mod<kVec, V>(w, a.weight, 1.f, s.ch);
#pragma unroll
    for (int i = 0; i < E; ++i) factor[i] = (1.f + factor[i]) * w[i];
  }
  float P[E], T[E], Q[E];
#pragma unroll
  for (int i = 0; i < E; ++i) P[i] = T[i] = Q[i] = 0.f;
  // The next row is fetched while one is worked on, where registers allow it.
  constexpr int kAhead = V < 4 ? 1 : 0;
  struct Row {
    Held<XT, kVec, V> r, dr;
    Held<YT, kVec, V> y, dz;
  } held[kAhead + 1];
  auto fetch = [&](int32_t n, Row& to) __attribute__((always_inline)) {
    if (n >= s.last) return;
    if (has_z) {
      to.r.load(row_of<XT>(a.r, s.b, n), s.ch);
      to.dz.load(row_of<YT>(a.z, s.b, n), s.ch);
    }
    if (a.dr.ptr) to.dr.load(row_of<XT>(a.dr, s.b, n), s.ch);
    if (has_y) to.y.load(row_of<YT>(a.y, s.b, n), s.ch);
  };
#pragma unroll
  for (int i = 0; i <= kAhead; ++i) {
    held[i].r.clear();
    held[i].dr.clear();
    held[i].y.clear();
    held[i].dz.clear();
    if (i > 0) fetch(s.first + (i - 1) * s.teams, held[i]);
  }
  for (int32_t row = s.first; kWide ? row < s.last : __any(row < s.last); row += s.teams) {
    const bool live = kWide || row < s.last;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) held[i] = held[i + 1];
    fetch(row + kAhead * s.teams, held[kAhead]);
    const Row& now = held[0];
    float D[E];
    if (a.dr.ptr) {
      now.dr.get(D, s.ch);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) D[i] = 0.f;
    }
    if (has_z) {
      float n[E], d[E];
      now.r.get(n, s.ch);
      now.dz.get(d, s.ch);
      float mean, inverse;
      statistics<kVec, V>(n, a.pre, a.eps, s.team, s.ch, s.own_count, s.of_own, mean, inverse);
      float along = 0.f, flat = 0.f;
      normalise<kVec, V, kFast>(n, mean, inverse, s.ch);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if (live) {
          P[i] += d[i] * n[i];
          T[i] += d[i];
        }
        d[i] *= factor[i];
        flat += d[i];
        along += d[i] * n[i];
      }
      two_sums(flat, along, s.team);
      flat = a.pre == RADIAL_NORM_LAYER ? flat * s.team.of_C : 0.f;
      along *= s.team.of_C;
#pragma unroll
      for (int i = 0; i < E; ++i) D[i] += inverse * (d[i] - flat - n[i] * along);
    }
    {
      float dx[E];
#pragma unroll
      for (int i = 0; i < E; ++i) dx[i] = a.residual_scale * D[i];
      if (live) store_row<XT, kVec, V>(row_of<XT>(a.dx, s.b, row), dx, s.ch);
    }
    if (has_y) {
      float m[E];
      now.y.get(m, s.ch);
      float inverse = 1.f;
      if (a.post != RADIAL_NORM_NONE) {
        float mean;
        statistics<kVec, V>(m, a.post, a.eps, s.team, s.ch, s.own_count, s.of_own, mean, inverse);
        normalise<kVec, V, kFast>(m, mean, inverse, s.ch);
      }
      // where there is no channel m is 0, and so is gate
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if (live) Q[i] += D[i] * m[i];
        D[i] *= gate[i];
      }
      if (a.post != RADIAL_NORM_NONE) {
        float along = 0.f, flat = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          flat += D[i];
          along += D[i] * m[i];
        }
        two_sums(flat, along, s.team);
        flat = a.post == RADIAL_NORM_LAYER ? flat * s.team.of_C : 0.f;
        along *= s.team.of_C;
#pragma unroll
        for (int i = 0; i < E; ++i) D[i] = inverse * (D[i] - flat - m[i] * along);
      }
      if (live) store_row<YT, kVec, V>(row_of<YT>(a.dy, s.b, row), D, s.ch);
    }
  }
  if (!a.wants) return;
  float* out = a.partial + (int64_t)blockIdx.x * 3 * a.C;
  if constexpr (kWide) {
    if (a.wants & 1) store_row<float, kVec, V>(out, P, s.ch);
    if (a.wants & 2) store_row<float, kVec, V>(out + a.C, T, s.ch);
    if (a.wants & 4) store_row<float, kVec, V>(out + 2 * (int64_t)a.C, Q, s.ch);
  } else {
    // the teams' sums meet in LDS: [team][lane * 8 + element]
    const int32_t at = threadIdx.x * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      merged[0][at + i] = P[i];
      merged[1][at + i] = T[i];
      merged[2][at + i] = Q[i];
    }
    __syncthreads();
    for (int32_t c = threadIdx.x; c < a.C; c += blockDim.x) {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        if (!(a.wants >> k & 1)) continue;
        float sum = 0.f;
        for (int t = 0; t < s.teams; ++t) sum += merged[k][t * L * 8 + c];
        out[(int64_t)k * a.C + c] = sum;
      }
    }
  }
}

struct GradArgs {
  const float* partial;  // [groups][chunks][3][C]
  float* of_group;       // [groups][2][C]: P and Q of each group, where another kernel adds them up, or null
  const float *gate, *post_weight, *weight, *scale;
  float *dgate, *dscale, *dshift, *dpost_weight, *dweight;
  int32_t C, chunks, groups, wants;
  int64_t mod_stride, dmod_stride;
};

constexpr int kGradColumns = 16, kGradSlices = 64;  // a wave: 16 channels, four slices
constexpr int kFewGroups = 16;
constexpr int64_t kMostInY = 65535;

// The sum over a wave's four slices, in all of them.
__device__ __forceinline__ float over_four(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// The gradients of a group's conditioning from its sums k: P, T, Q.
__device__ __forceinline__ void store_grad(const GradArgs& a, int64_t group, int32_t c, int32_t k, float total) {
  const int64_t mod = group * a.dmod_stride + c;
  if (k == 0 && a.dscale) a.dscale[mod] = a.weight ? total * a.weight[c] : total;
  if (k == 1) a.dshift[mod] = total;
  if (k == 2 && a.dgate) a.dgate[mod] = a.post_weight ? total * a.post_weight[c] : total;
}

// Up to 16 groups: 16 channels of all of them, each group with its share of 64 slices, which add up its workgroups' sums; then the slices' sums, and the gradients
// of the weights.  (With 64 channels and 16 slices the gradients of 2 x 1237 x 1000 took 41 us instead of 26.)
__global__ void __launch_bounds__(kGradColumns * kGradSlices) norm_grad_kernel(GradArgs a) {
  __shared__ float sums[3][kGradSlices / 4][kGradColumns], of_groups[3][kFewGroups][kGradColumns];
  const int32_t lane = threadIdx.x, slice = threadIdx.y;
  const int32_t c = blockIdx.x * kGradColumns + lane;
  int32_t slices = kGradSlices;  // of a group
  while (slices * a.groups > kGradSlices) slices /= 2;
  const int64_t group = slice / slices;
  float sum[3] = {0.f, 0.f, 0.f};
  if (c < a.C && group < a.groups) {
    const float* p = a.partial + group * a.chunks * 3 * a.C + c;
    const int64_t step = 3 * (int64_t)a.C;
#pragma unroll
    for (int k = 0; k < 3; ++k, p += a.C) {
      if (!(a.wants >> k & 1)) continue;
#pragma unroll 8
      for (int32_t i = slice % slices; i < a.chunks; i += slices) sum[k] += p[i * step];
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    sum[k] = over_four(sum[k]);
    if (slice % 4 == k) sums[k][slice / 4][lane] = sum[k];
  }
  __syncthreads();
  // slice k of each group's adds up P, T or Q
  const int32_t k = slice % slices;
  if (k < 3 && c < a.C && group < a.groups && (a.wants >> k & 1)) {
    float total = 0.f;
#pragma unroll 4
    for (int i = 0; i < slices / 4; ++i) total += sums[k][slice / slices * (slices / 4) + i][lane];
    store_grad(a, group, c, k, total);
    if (k == 0 && a.scale) total *= 1.f + a.scale[group * a.mod_stride + c];
    if (k == 2 && a.gate) total *= a.gate[group * a.mod_stride + c];
    of_groups[k][group][lane] = total;
  }
  __syncthreads();
  if (slice > 2 || !(a.wants >> slice & 1) || c >= a.C) return;
  float total = 0.f;
  for (int g = 0; g < a.groups; ++g) total += of_groups[slice][g][lane];
  if (slice == 0 && a.dweight) a.dweight[c] = total;
  if (slice == 2 && a.dpost_weight) a.dpost_weight[c] = total;
}

// More groups, each with few sums: a wave for 64 channels of a group, or the four of a workgroup.  (With 1024 threads for
// each group and 16 channels the gradients of 32 760 x 5120 in groups of 1560 took 454 us instead of 427, of 4 x 1000 x 1536 in groups of 20 116 (32), of 2 859 (60).)
__global__ void __launch_bounds__(256) norm_grad_many_kernel(GradArgs a, int32_t waves_of_group) {
  __shared__ float sums[3][4][64];
  const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t c = blockIdx.x * 64 + lane, first = wave % waves_of_group;
  const int64_t group = (blockIdx.y + (int64_t)blockIdx.z * kMostInY) * (4 / waves_of_group) + wave / waves_of_group;
  const bool live = c < a.C && group < a.groups;
  float sum[3] = {0.f, 0.f, 0.f};
  if (live) {
    const float* p = a.partial + group * a.chunks * 3 * a.C + c;
    for (int32_t i = first; i < a.chunks; i += waves_of_group) {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (a.wants >> k & 1) sum[k] += p[(i * 3 + k) * (int64_t)a.C];
    }
  }
  if (waves_of_group > 1) {
#pragma unroll
    for (int k = 0; k < 3; ++k) sums[k][wave][lane] = sum[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) sum[k] = (sums[k][0][lane] + sums[k][1][lane]) + (sums[k][2][lane] + sums[k][3][lane]);
  }
  if (!live || first) return;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (!(a.wants >> k & 1)) continue;
    store_grad(a, group, c, k, sum[k]);
    if (a.of_group && k != 1) a.of_group[(group * 2 + (k == 2)) * a.C + c] = sum[k];
  }
}

// dw and dw_post: sums over the groups, each times its conditioning.
__global__ void __launch_bounds__(kGradColumns * kGradSlices) norm_weight_grad_kernel(GradArgs a) {
  __shared__ float sums[2][kGradSlices / 4][kGradColumns];
  const int32_t lane = threadIdx.x, slice = threadIdx.y;
  const int32_t c = blockIdx.x * kGradColumns + lane;
  float dw = 0.f, dw_post = 0.f;
  if (c < a.C) {
    for (int64_t g = slice; g < a.groups; g += kGradSlices) {
      if (a.dweight) dw += a.of_group[g * 2 * a.C + c] * (a.scale ? 1.f + a.scale[g * a.mod_stride + c] : 1.f);
      if (a.dpost_weight) dw_post += a.of_group[(g * 2 + 1) * a.C + c] * (a.gate ? a.gate[g * a.mod_stride + c] : 1.f);
    }
  }
  dw = over_four(dw);
  dw_post = over_four(dw_post);
  if (slice % 4 == 0) sums[0][slice / 4][lane] = dw;
  if (slice % 4 == 1) sums[1][slice / 4][lane] = dw_post;
  __syncthreads();
  if (slice > 1 || c >= a.C) return;
  float total = 0.f;
#pragma unroll
  for (int i = 0; i < kGradSlices / 4; ++i) total += sums[slice][i][lane];
  if (slice == 0 && a.dweight) a.dweight[c] = total;
  if (slice == 1 && a.dpost_weight) a.dpost_weight[c] = total;
}

// ---- launches -----------------------------------------------------------------------------------

// How a call is laid out; goes by the sizes alone, so that the workspace does too.
struct Layout {
  int32_t groups_of_batch;
  int64_t groups;
  int32_t chunks, rows;
};

constexpr int32_t kNarrow = 512;  // channels up to which a row is a wave's or less

// Channels of a thread of a wide team, in eights.
int eights_of(int32_t C) { return C <= 4096 ? 1 : C <= 8192 ? 2 : 4; }

// `rounds` times the workgroups that run at a time, by the waves that fit a compute unit, shared out over the groups; a workgroup has `least` rows or
// more for each of its teams, since each loads the conditioning and, backward, writes its sums, but for fewer than 256 teams' worth of rows, where
// what counts is how many rows come one after the other.
Layout make_layout(const radial_norm_params& p, int32_t waves_of_unit, int32_t rounds, int32_t least) {
  Layout l;
  l.groups_of_batch = (int32_t)(((int64_t)p.N + p.group - 1) / p.group);
  l.groups = (int64_t)p.B * l.groups_of_batch;
  const int32_t of_group = p.group < p.N ? p.group : p.N;
  const int32_t V = eights_of(p.C);
  const int32_t waves = p.C <= kNarrow ? 4 : (p.C + 512 * V - 1) / (512 * V);
  const int32_t teams = p.C <= 128 ? 16 : p.C <= 256 ? 8 : p.C <= kNarrow ? 4 : 1;
  // Where there is one round all of it has to fit at once: five waves are two on one of the unit's four SIMDs, so that two workgroups of them fit, not three
  // (gradients of 32 760 x 5120 values in rows of 2304: 246 us instead of 281, without a branch 185 (232); with rounds enough the forward is better with three).
  const int32_t fit = rounds == 1 && waves > 4 ? waves_of_unit / 4 / ((waves + 3) / 4) : waves_of_unit / waves;
  const int64_t workgroups = (int64_t)256 * rounds * (fit > 1 ? fit : 1);
  int64_t chunks = workgroups / l.groups;
  const int64_t rows_of_team = ((int64_t)p.B * p.N / teams + 255) / 256;
  if (rows_of_team < least) least = rows_of_team < 1 ? 1 : (int32_t)rows_of_team;
  const int64_t most = ((int64_t)of_group + least * teams - 1) / (least * teams);
  if (chunks > most) chunks = most;
  if (chunks < 1) chunks = 1;
  l.rows = (int32_t)((of_group + chunks - 1) / chunks);
  l.chunks = (int32_t)(((int64_t)of_group + l.rows - 1) / l.rows);
  return l;
}

Layout fwd_layout(const radial_norm_params& p) { return make_layout(p, 16, 8, 1); }
Layout bwd_layout(const radial_norm_params& p) { return make_layout(p, p.C <= 4096 ? 16 : 8, 1, 4); }

bool aligned(const void* ptr, int64_t sb, int64_t sn, int size) {
  return ((uintptr_t)ptr & 15u) == 0 && sb * size % 16 == 0 && sn * size % 16 == 0;
}

template <class XT, class YT, bool kVec, int V, bool kWide, int L>
int launch_one(const NormArgs& a, bool backward, int64_t grid, hipStream_t stream) {
  int threads = 256;
  if (kWide) threads = ((a.C + 8 * V - 1) / (8 * V) + 63) / 64 * 64;
  if (backward) {
    norm_bwd_kernel<XT, YT, kVec, V, kWide, L><<<dim3((unsigned)grid), dim3(threads), 0, stream>>>(a);
  } else {
    norm_fwd_kernel<XT, YT, kVec, V, kWide, L><<<dim3((unsigned)grid), dim3(threads), 0, stream>>>(a);
  }
  RADIAL_HIP_TRY(hipGetLastError());
  return RADIAL_OK;
}

template <class XT, class YT, bool kVec>
int launch_types(const NormArgs& a, bool backward, int64_t grid, hipStream_t stream) {
  const int eights = eights_of(a.C);
  if (a.C <= 128) return launch_one<XT, YT, kVec, 1, false, 16>(a, backward, grid, stream);
  if (a.C <= 256) return launch_one<XT, YT, kVec, 1, false, 32>(a, backward, grid, stream);
  if (a.C <= kNarrow) return launch_one<XT, YT, kVec, 1, false, 64>(a, backward, grid, stream);
  if (eights == 1) return launch_one<XT, YT, kVec, 1, true, 64>(a, backward, grid, stream);
  if (eights == 2) return launch_one<XT, YT, kVec, 2, true, 64>(a, backward, grid, stream);
  return launch_one<XT, YT, kVec, 4, true, 64>(a, backward, grid, stream);
}

template <bool kVec>
int launch_rows(const NormArgs& a, int32_t x_type, int32_t y_type, bool backward, int64_t grid, hipStream_t stream) {
  if (x_type == RADIAL_F32)
    return y_type == RADIAL_F32 ? launch_types<float, float, kVec>(a, backward, grid, stream) : launch_types<float, __bf16, kVec>(a, backward, grid, stream);
  return y_type == RADIAL_F32 ? launch_types<__bf16, float, kVec>(a, backward, grid, stream) : launch_types<__bf16, __bf16, kVec>(a, backward, grid, stream);
}

int launch(const NormArgs& a, int32_t x_type, int32_t y_type, bool vec, bool backward, int64_t grid, hipStream_t stream) {
  return vec ? launch_rows<true>(a, x_type, y_type, backward, grid, stream) : launch_rows<false>(a, x_type, y_type, backward, grid, stream);
}

// ---- checks -------------------------------------------------------------------------------------

bool is_norm(int32_t kind) { return kind == RADIAL_NORM_LAYER || kind == RADIAL_NORM_RMS; }

int check_params(const radial_norm_params* p) {
  if (!p) return fail(RADIAL_EINVAL, "params is NULL");
  if (p->B < 1 || p->N < 1 || p->C < 1 || p->group < 1) return fail(RADIAL_EINVAL, "B, N, C, group must be >= 1");
  // a workgroup's teams step over its last row by up to 32 before they stop
  if ((int64_t)p->B * p->N > 0x7fffffffLL - 1024) return fail(RADIAL_EINVAL, "B*N must be below 2^31 - 1024");
  if (p->C > kMaxChannels) return fail(RADIAL_EUNSUPPORTED, "C must be at most %d (got %d)", kMaxChannels, p->C);
  if (p->post != RADIAL_NORM_NONE && !is_norm(p->post)) return fail(RADIAL_EINVAL, "post must be a RADIAL_NORM_ value (got %d)", p->post);
  if (p->pre != RADIAL_NORM_NONE && !is_norm(p->pre)) return fail(RADIAL_EINVAL, "pre must be a RADIAL_NORM_ value (got %d)", p->pre);
  if (!(p->eps >= FLT_MIN) || !isfinite(p->eps)) return fail(RADIAL_EINVAL, "eps must be positive, normal and finite");
  if (!isfinite(p->residual_scale)) return fail(RADIAL_EINVAL, "residual_scale must be finite");
  return RADIAL_OK;
}

int check_rows(const char* name, const radial_rows& t, const radial_norm_params& p) {
  if (!t.ptr) return fail(RADIAL_EINVAL, "%s.ptr is NULL", name);
  if (!is_type(t.type)) return fail(RADIAL_EINVAL, "%s.type must be RADIAL_BF16 or RADIAL_F32 (got %d)", name, t.type);
  if ((uintptr_t)t.ptr % size_of(t.type)) return fail(RADIAL_ESHAPE, "%s.ptr is not aligned to its elements", name);
  if ((p.N > 1 && t.stride_n < p.C) || t.stride_n < 0 || t.stride_b < 0)
    return fail(RADIAL_ESHAPE, "%s strides must not be negative, and stride_n not below C", name);
  return RADIAL_OK;
}

int check_mod(const char* name, const float* mod, int64_t stride, const radial_norm_params& p) {
  if (!mod) return RADIAL_OK;
  if ((uintptr_t)mod & 3u) return fail(RADIAL_ESHAPE, "%s is not aligned to its elements", name);
  if (stride < p.C) return fail(RADIAL_ESHAPE, "the stride of %s must not be below C", name);
  return RADIAL_OK;
}

int same_type(const char* x, int32_t of_x, const char* y, int32_t of_y) {
  return of_x == of_y ? RADIAL_OK : fail(RADIAL_EINVAL, "%s and %s must have one type", x, y);
}

RowsArg arg(const radial_rows& t) { return RowsArg{(char*)t.ptr, t.stride_b, t.stride_n}; }

NormArgs common_args(const radial_norm_params& p, const Layout& l) {
  NormArgs a = {};
  a.N = p.N; a.C = p.C; a.group = p.group; a.groups_of_batch = l.groups_of_batch;
  a.chunks = l.chunks; a.rows = l.rows;
  a.post = p.post; a.pre = p.pre;
  a.eps = p.eps; a.residual_scale = p.residual_scale;
  a.mod_stride = p.mod_stride;
  return a;
}

int check_grid(const Layout& l) {
  return l.groups * l.chunks <= kMostThreads / 512 ? RADIAL_OK : fail(RADIAL_ESHAPE, "too many groups for one launch");
}

}  // namespace
}  // namespace radial

using namespace radial;

extern "C" int radial_norm_fwd(const radial_norm_params* params, radial_rows x, radial_rows y, const float* gate, const float* post_weight,
                               const float* weight, const float* scale, const float* shift, radial_rows r, radial_rows z, void* hip_stream) {
  if (int rc = check_params(params)) return rc;
  const radial_norm_params& p = *params;
  if (int rc = check_rows("x", x, p)) return rc;
  const bool has_y = y.ptr != nullptr, has_z = p.pre != RADIAL_NORM_NONE;
  if (has_y) {
    if (int rc = check_rows("y", y, p)) return rc;
    if (int rc = check_rows("r", r, p)) return rc;
    if (int rc = same_type("x", x.type, "r", r.type)) return rc;
  } else if (r.ptr || gate || post_weight || p.post != RADIAL_NORM_NONE || p.residual_scale != 1.f) {
    return fail(RADIAL_EINVAL, "without y there is no r, gate, post norm or residual_scale");
  }
  if (has_z) {
    if (int rc = check_rows("z", z, p)) return rc;
    if (has_y)
      if (int rc = same_type("y", y.type, "z", z.type)) return rc;
  } else if (z.ptr || weight || scale || shift) {
    return fail(RADIAL_EINVAL, "z, weight, scale and shift need a norm (pre)");
  }
  if (!has_y && !has_z) return fail(RADIAL_EINVAL, "neither y nor z is given");
  if (post_weight && p.post == RADIAL_NORM_NONE) return fail(RADIAL_EINVAL, "post_weight needs a norm (post)");
  const struct { const char* name; const float* ptr; int64_t stride; } mods[] = {
      {"gate", gate, p.mod_stride}, {"scale", scale, p.mod_stride}, {"shift", shift, p.mod_stride}, {"post_weight", post_weight, p.C}, {"weight", weight, p.C}};
  for (const auto& m : mods)
    if (int rc = check_mod(m.name, m.ptr, m.stride, p)) return rc;
  const Layout l = fwd_layout(p);
  if (int rc = check_grid(l)) return rc;
  NormArgs a = common_args(p, l);
  a.x = arg(x);
  if (has_y) { a.y = arg(y); a.r = arg(r); }
  if (has_z) a.z = arg(z);
  a.gate = gate; a.post_weight = post_weight; a.weight = weight; a.scale = scale; a.shift = shift;
  bool vec = p.C % 8 == 0 && p.mod_stride % 4 == 0;
  for (const radial_rows* t : {&x, &y, &r, &z})
    if (t->ptr) vec = vec && aligned(t->ptr, t->stride_b, t->stride_n, size_of(t->type));
  for (const auto& m : mods) vec = vec && ((uintptr_t)m.ptr & 15u) == 0;
  return launch(a, x.type, has_y ? y.type : z.type, vec, false, l.groups * l.chunks, (hipStream_t)hip_stream);
}

extern "C" size_t radial_norm_bwd_workspace(const radial_norm_params* params) {
  if (check_params(params) != RADIAL_OK) return 0;
  const Layout l = bwd_layout(*params);
  if (check_grid(l) != RADIAL_OK) return 0;
  // the workgroups' sums, then the groups'
  const size_t raw = ((size_t)l.groups * l.chunks * 3 + (size_t)l.groups * 2) * params->C * sizeof(float);
  return (raw + 255) & ~(size_t)255;
}

extern "C" int radial_norm_bwd(const radial_norm_params* params, radial_rows r, radial_rows y, radial_rows dz, radial_rows dr, const float* gate,
                               const float* post_weight, const float* weight, const float* scale, radial_rows dx, radial_rows dy, float* dgate,
                               float* dscale, float* dshift, float* dpost_weight, float* dweight, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_params(params)) return rc;
  const radial_norm_params& p = *params;
  const bool has_y = y.ptr != nullptr, has_z = p.pre != RADIAL_NORM_NONE;
  if (int rc = check_rows("dx", dx, p)) return rc;
  if (dr.ptr) {
    if (int rc = check_rows("dr", dr, p)) return rc;
    if (int rc = same_type("dr", dr.type, "dx", dx.type)) return rc;
  }
  if (has_z) {
    if (int rc = check_rows("r", r, p)) return rc;
    if (int rc = check_rows("dz", dz, p)) return rc;
    if (int rc = same_type("r", r.type, "dx", dx.type)) return rc;
  } else if (dz.ptr || weight || scale || dscale || dshift || dweight) {
    return fail(RADIAL_EINVAL, "dz, weight, scale and their gradients need a norm (pre)");
  } else if (!dr.ptr) {
    return fail(RADIAL_EINVAL, "dr.ptr is NULL, and there is no dz");
  }
  if (has_y) {
    if (int rc = check_rows("y", y, p)) return rc;
    if (int rc = check_rows("dy", dy, p)) return rc;
    if (int rc = same_type("y", y.type, "dy", dy.type)) return rc;
    if (has_z)
      if (int rc = same_type("y", y.type, "dz", dz.type)) return rc;
  } else if (dy.ptr || gate || post_weight || dgate || dpost_weight || p.post != RADIAL_NORM_NONE || p.residual_scale != 1.f) {
    return fail(RADIAL_EINVAL, "without y there is no dy, gate, post norm or residual_scale");
  }
  if (!has_y && !has_z) return fail(RADIAL_EINVAL, "neither y nor dz is given");
  if ((post_weight || dpost_weight) && p.post == RADIAL_NORM_NONE) return fail(RADIAL_EINVAL, "post_weight needs a norm (post)");
  const struct { const char* name; const float* ptr; int64_t stride; } mods[] = {
      {"gate", gate, p.mod_stride}, {"scale", scale, p.mod_stride}, {"post_weight", post_weight, p.C}, {"weight", weight, p.C},
      {"dgate", dgate, p.dmod_stride}, {"dscale", dscale, p.dmod_stride}, {"dshift", dshift, p.dmod_stride}, {"dpost_weight", dpost_weight, p.C}, {"dweight", dweight, p.C}};
  for (const auto& m : mods)
    if (int rc = check_mod(m.name, m.ptr, m.stride, p)) return rc;
  const size_t need = radial_norm_bwd_workspace(params);
  if (!need) return fail(RADIAL_ESHAPE, "too many groups for one launch");
  if (!workspace || ((uintptr_t)workspace & 255u)) return fail(RADIAL_ESHAPE, "workspace must be a 256-byte aligned device pointer");
  if (workspace_bytes < need) return fail(RADIAL_ESHAPE, "workspace holds %zu bytes, %zu needed", workspace_bytes, need);

  const Layout l = bwd_layout(p);
  NormArgs a = common_args(p, l);
  if (has_z) { a.r = arg(r); a.z = arg(dz); }
  if (has_y) { a.y = arg(y); a.dy = arg(dy); }
  if (dr.ptr) a.dr = arg(dr);
  a.dx = arg(dx);
  a.gate = gate; a.post_weight = post_weight; a.weight = weight; a.scale = scale;
  a.partial = (float*)workspace;
  a.wants = (dscale || dweight ? 1 : 0) | (dshift ? 2 : 0) | (dgate || dpost_weight ? 4 : 0);
  bool vec = p.C % 8 == 0 && p.mod_stride % 4 == 0;
  for (const radial_rows* t : {&r, &y, &dz, &dr, &dx, &dy})
    if (t->ptr) vec = vec && aligned(t->ptr, t->stride_b, t->stride_n, size_of(t->type));
  for (int i = 0; i < 4; ++i) vec = vec && ((uintptr_t)mods[i].ptr & 15u) == 0;
  if (int rc = launch(a, dx.type, has_y ? y.type : dz.type, vec, true, l.groups * l.chunks, (hipStream_t)hip_stream)) return rc;
  if (!a.wants) return RADIAL_OK;

  GradArgs g = {};
  g.partial = a.partial;
  const bool few = l.groups <= kFewGroups;
  g.of_group = (dweight || dpost_weight) && !few ? a.partial + (size_t)l.groups * l.chunks * 3 * p.C : nullptr;
  g.gate = gate; g.post_weight = post_weight; g.weight = weight; g.scale = scale;
  g.dgate = dgate; g.dscale = dscale; g.dshift = dshift; g.dpost_weight = dpost_weight; g.dweight = dweight;
  g.C = p.C; g.chunks = l.chunks; g.groups = (int32_t)l.groups; g.wants = a.wants;
  g.mod_stride = p.mod_stride; g.dmod_stride = p.dmod_stride;
  const unsigned columns = (unsigned)((p.C + kGradColumns - 1) / kGradColumns);
  const dim3 block(kGradColumns, kGradSlices);
  if (few) {
    norm_grad_kernel<<<dim3(columns), block, 0, (hipStream_t)hip_stream>>>(g);
  } else {
    const int32_t waves_of_group = l.chunks > 8 ? 4 : 1;
    const int64_t rows = (l.groups * waves_of_group + 3) / 4;
    const unsigned in_y = (unsigned)(rows < kMostInY ? rows : kMostInY), in_z = (unsigned)((rows + kMostInY - 1) / kMostInY);
    norm_grad_many_kernel<<<dim3((unsigned)((p.C + 63) / 64), in_y, in_z), dim3(256), 0, (hipStream_t)hip_stream>>>(g, waves_of_group);
  }
  RADIAL_HIP_TRY(hipGetLastError());
  if (g.of_group) {
    norm_weight_grad_kernel<<<dim3(columns), block, 0, (hipStream_t)hip_stream>>>(g);
    RADIAL_HIP_TRY(hipGetLastError());
  }
  return RADIAL_OK;
}
