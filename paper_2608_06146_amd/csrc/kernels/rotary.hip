// Head norms and rotary positions: rows of Q and K before the attention
// (forward), their gradients (backward), and a decode step's rows on their way
// into the paged caches (append).
//
//   y = w x / sqrt(mean x^2 + eps)  (or x),  z = scale R(pos * inv_freq) y
//   dy = scale R(-angle) dz,  g = w dy,  dw = sum dy x rho,
//   dx = rho (g - x rho^2 mean(g x)),  rho = 1 / sqrt(mean x^2 + eps)
//
// All of it is bound by memory: every element is read once and written once.
// A row of one head is shared by eight lanes (a group).  A lane holds D / 8
// dimensions in units of 16 bytes, chosen so that the lanes of a group access
// neighbouring units (whole 128-byte lines) and both members of a pair are in
// one lane; only where a lane has a single unit (bf16, D = 64, halves) the
// members are in lanes four apart, which exchange their values.
//
// A workgroup takes a tile of rows of one tensor (q or k).  Its lanes compute
// the cosines and sines of the tile's rows once, a pair each, into LDS; its
// groups then take the tile's (row, head) pairs in order, neighbours reading
// neighbouring heads, with the rows of the next ones in flight.
//
// Angles: a position times the pair's 64-bit fraction of a turn, modulo 2^64,
// is the angle in turns; its leading 32 bits are split into a quadrant and an
// angle within +-pi/4, whose sine and cosine are Taylor sums (to x^9 and x^10:
// remainders below 2e-9).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../rotary.hpp"
#include "device_common.hpp"
#include "e4m3.hpp"

namespace padoc {
namespace {

constexpr int kThreads = 256;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

constexpr int kLanes = 8;                    // of a group
constexpr int kGroups = kThreads / kLanes;   // of a workgroup, and rows of a tile at most
template <int D>
constexpr int kElems = D / kLanes;           // elements of a lane
// Elements of a 16-byte unit, the size of a lane's memory accesses, and units
// of a lane.
template <typename T>
constexpr int kUnit = 16 / (int)sizeof(T);
template <typename T, int D>
constexpr int kUnits = kElems<D> / kUnit<T>;

// A 16-byte unit at an address aligned to one element.
template <typename T>
struct Unit;
template <>
struct Unit<__bf16> {
  typedef u32x4 type __attribute__((aligned(2)));
};
template <>
struct Unit<float> {
  typedef u32x4 type __attribute__((aligned(4)));
};

// Rows are stored past the caches (non-temporal), and loaded so (STREAM) by
// calls that read and write more than 128 MiB, half of what the last-level cache
// holds; of shorter calls the producer's rows are likely still there.  Measured
// with inputs and outputs in turn: 43,067 rows of 18 heads of 128 (bf16) 69.3 us
// (5.7 TB/s), with plain loads 72.0, plain stores 74.0, both plain 78.2; their
// backward 111.4, 116.2, 119.1 and 120.6; 5,437 rows of 32 heads of 64 (fp32, 89
// MB) 15.0 with plain loads, 17.2 past the caches.
constexpr int64_t kStreamBytes = 128 << 20;
template <bool STREAM, typename T>
__device__ __forceinline__ u32x4 load_unit(const T* p) {
  const auto q = reinterpret_cast<const typename Unit<T>::type*>(p);
  return STREAM ? __builtin_nontemporal_load(q) : *q;
}

// A lane's elements of a head as they were loaded: its units in turn.
template <typename T, int D>
struct Raw {
  u32x4 u[kUnits<T, D>];
  template <bool STREAM>
  __device__ __forceinline__ void load(const T* p, const int (&at)[kUnits<T, D>]) {
#pragma unroll
    for (int i = 0; i < kUnits<T, D>; ++i) u[i] = load_unit<STREAM>(p + at[i]);
  }
  __device__ __forceinline__ float elem(int i) const {
    const uint32_t w = u[i / kUnit<T>][i % kUnit<T> * (int)sizeof(T) / 4];
    return __uint_as_float(sizeof(T) == 4 ? w : i % 2 ? w & 0xffff0000u : w << 16);
  }
  __device__ __forceinline__ void get(float (&x)[kElems<D>]) const {
#pragma unroll
    for (int i = 0; i < kElems<D>; ++i) x[i] = elem(i);
  }
};

// One unit's elements, rounded to nearest-even once, here (NaN stays NaN).
__device__ __forceinline__ u32x4 pack_unit(const __bf16*, const float* x) {
  const bf16x8 b = __builtin_convertvector((f32x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}), bf16x8);
  u32x4 u;
  __builtin_memcpy(&u, &b, 16);
  return u;
}
__device__ __forceinline__ u32x4 pack_unit(const float*, const float* x) {
  u32x4 u;
  __builtin_memcpy(&u, x, 16);
  return u;
}
template <typename T, int N, int E>
__device__ __forceinline__ void store_row(T* p, const int (&at)[N], const float (&x)[E]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    __builtin_nontemporal_store(pack_unit(p, x + i * kUnit<T>), reinterpret_cast<typename Unit<T>::type*>(p + at[i]));
}

// Sum over the eight lanes of a group, in every one of them.
__device__ __forceinline__ float group_sum(float v) {
  v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xf, 0xf, true));   // lane ^ 1
  v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xf, 0xf, true));   // lane ^ 2
  v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xf, 0xf, true));  // 7 - lane
  return v;
}

template <int CTRL>
__device__ __forceinline__ double from_lane(double v) {
  return __hiloint2double(__builtin_amdgcn_mov_dpp(__double2hiint(v), CTRL, 0xf, 0xf, true),
                          __builtin_amdgcn_mov_dpp(__double2loint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ double group_sum(double v) {
  v += from_lane<0xB1>(v);
  v += from_lane<0x4E>(v);
  v += from_lane<0x141>(v);
  return v;
}

// The value of lane ^ 4: from four lanes on for the lower half of a group (banks
// 0 and 2 of a row of 16 lanes), from four lanes back for the upper.
__device__ __forceinline__ float other_half(float v) {
  const int x = __float_as_int(v);
  int r = __builtin_amdgcn_update_dpp(0, x, 0x104, 0xf, 0x5, false);
  r = __builtin_amdgcn_update_dpp(r, x, 0x114, 0xf, 0xa, false);
  return __int_as_float(r);
}
__device__ __forceinline__ double other_half(double v) {
  return __hiloint2double(__float_as_int(other_half(__int_as_float(__double2hiint(v)))),
                          __float_as_int(other_half(__int_as_float(__double2loint(v)))));
}

// Sine and cosine of `phase` turns / 2^32.
__device__ __forceinline__ void sincos_turns(uint32_t phase, float& s, float& c) {
  const uint32_t quadrant = (phase + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(phase - (quadrant << 30)) * 1.46291807926715968105e-9f;  // 2 pi / 2^32
  const float y = x * x;
  const float sx = x + x * y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880))));
  const float cx = 1.f + y * (-1.f / 2 + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320 + y * (-1.f / 3628800)))));
  s = quadrant & 1 ? cx : sx;
  c = quadrant & 1 ? sx : cx;
  if (quadrant & 2) s = -s;
  if ((quadrant + 1) & 2) c = -c;
}

// The same in 64 bits, of 2^64, off by less than 2^-36 (of this phase's: a turn's
// own rounding, below 2^-64, goes times the position): the last terms of the series are
// 2^-14 and less and stay in fp32.
__device__ __forceinline__ void sincos_turns(uint64_t phase, double& s, double& c) {
  const uint32_t quadrant = (uint32_t)((phase + 0x2000000000000000ull) >> 62);
  const double x = (double)(int64_t)(phase - ((uint64_t)quadrant << 62)) * 3.40612158008655459e-19;  // 2 pi / 2^64
  const double y = x * x;
  const float yf = (float)y;
  const float s7 = -1.f / 5040 + yf * (1.f / 362880 + yf * (-1.f / 39916800));
  const float c8 = 1.f / 40320 + yf * (-1.f / 3628800 + yf * (1.f / 479001600));
  const double sx = fma(x * y, fma(y, fma(y, (double)s7, 1. / 120), -1. / 6), x);
  const double cx = fma(y, fma(y, fma(y, fma(y, (double)c8, -1. / 720), 1. / 24), -0.5), 1.);
  s = quadrant & 1 ? cx : sx;
  c = quadrant & 1 ? sx : cx;
  if (quadrant & 2) s = -s;
  if ((quadrant + 1) & 2) c = -c;
}

// A lane's place in its group: which units it holds.  A slot is what holds whole
// pairs: a unit (pairs of neighbours), or units k and k + n (halves; n = units
// of half the rotated dimensions), where behind the n rotated slots k stands for
// two of the other units.  Lane l has slots l, l + 8, ... (split: lanes l and l + 4
// share slot l, a unit each).  Pair m of a lane has elements first(m) and
// second(m).
template <typename T, int D, bool PAIRS>
struct Place {
  static constexpr int E = kUnit<T>, N = kUnits<T, D>;
  static constexpr bool kSplit = !PAIRS && N == 1;
  static constexpr int kSlotLanes = kSplit ? kLanes / 2 : kLanes;
  static constexpr int kPairsPerSlot = PAIRS ? E / 2 : E;
  static constexpr int kSlots = PAIRS ? N : kSplit ? 1 : N / 2;
  int at[N];
  int turned;  // slots 0 .. turned-1 are rotated
  __device__ __forceinline__ Place(int pairs) {
    const int lane = threadIdx.x % kLanes;
    const int n = pairs / kPairsPerSlot;  // rotated slots of the group
    turned = 0;
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      const int k = i * kSlotLanes + lane % kSlotLanes;
      turned += k < n;
      if (PAIRS) {
        at[i] = k * E;
      } else {
        const int a = (k < n ? k : n + k) * E, b = (k < n ? k + n : D / 2 / E + k) * E;
        if (kSplit) {
          at[0] = lane < kSlotLanes ? a : b;
        } else {
          at[2 * i % N] = a;
          at[(2 * i + 1) % N] = b;
        }
      }
    }
  }
  static constexpr int first(int m) { return PAIRS ? 2 * m : kSplit ? m : m / E * (2 * E) + m % E; }
  static constexpr int second(int m) { return PAIRS ? 2 * m + 1 : m / E * (2 * E) + E + m % E; }
  // (Slot) lane and place in the lane of a pair.
  static __device__ __forceinline__ int lane_of(int pair) { return pair / kPairsPerSlot % kSlotLanes; }
  static __device__ __forceinline__ int index_of(int pair) {
    return pair / kPairsPerSlot / kSlotLanes * kPairsPerSlot + pair % kPairsPerSlot;
  }
};

// Cosines and sines of a tile's rows: per row and two pairs of a lane, the lanes'
// 16 bytes side by side.
template <typename T, int D, bool PAIRS, typename F = float>
struct AngleTable {
  typedef Place<T, D, PAIRS> P;
  typedef F F4 __attribute__((ext_vector_type(4)));
  F4 at[kGroups][P::kSlots * P::kPairsPerSlot / 2][P::kSlotLanes];
  static_assert(sizeof(at) == kGroups * D * sizeof(F), "D / 2 pairs a row");

  // Fill rows [0, n): thread t takes pair t % (D / 2) of rows t / (D / 2), ...;
  // scaled, the sine negated for the inverse rotation.
  __device__ __forceinline__ void fill(const RotaryParams& p, const int32_t* pos, int64_t stride, int64_t row0, int n) {
    constexpr int kPairs = D / 2;
    const int pair = threadIdx.x % kPairs;
    if (pair >= p.pairs) return;
    const uint64_t turn = p.table.turn[pair];
    pos += p.table.axis[pair] * stride + row0;
    const int m = P::index_of(pair);
    F* dst = reinterpret_cast<F*>(&at[0][m / 2][P::lane_of(pair)]) + m % 2 * 2;
    for (int r = threadIdx.x / kPairs; r < n; r += kThreads / kPairs) {
      F s, c;
      const uint64_t phase = (uint64_t)(int64_t)pos[r] * turn;
      if constexpr (sizeof(F) == 8)
        sincos_turns(phase, s, c);
      else
        sincos_turns((uint32_t)(phase >> 32), s, c);
      dst[r * D] = c * p.scale;
      dst[r * D + 1] = p.inverse ? -s * p.scale : s * p.scale;
    }
  }
};

// Rotate a lane's pairs by the angles of a row of the table.  (Split: every lane
// of the group calls it with its one unit.)
template <typename T, int D, bool PAIRS>
__device__ __forceinline__ void turn(float (&x)[kElems<D>], const AngleTable<T, D, PAIRS>& table, int row,
                                     const Place<T, D, PAIRS>& pl) {
  typedef Place<T, D, PAIRS> P;
  float y[kElems<D>];
  if (P::kSplit) {
#pragma unroll
    for (int i = 0; i < kElems<D>; ++i) y[i] = other_half(x[i]);
  }
#pragma unroll
  for (int slot = 0; slot < P::kSlots; ++slot) {
    if (slot >= pl.turned) break;
#pragma unroll
    for (int i = 0; i < P::kPairsPerSlot / 2; ++i) {
      const int m0 = slot * P::kPairsPerSlot + 2 * i;
      const f32x4 t = table.at[row][m0 / 2][threadIdx.x % P::kSlotLanes];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int a = P::first(m0 + j);
        const float c = t[2 * j], s = t[2 * j + 1], ya = x[a];
        if (P::kSplit) {
          x[a] = ya * c + y[a] * (threadIdx.x % kLanes < P::kSlotLanes ? -s : s);
        } else {
          const int b = P::second(m0 + j) % kElems<D>;
          const float yb = x[b];
          x[a] = ya * c - yb * s;
          x[b] = yb * c + ya * s;
        }
      }
    }
  }
}

template <int D>
__device__ __forceinline__ float rms_scale(const float (&x)[kElems<D>], float eps) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kElems<D>; ++i) s += x[i] * x[i];
  return __builtin_amdgcn_rsqf(group_sum(s) * (1.f / D) + eps);
}

template <typename T>
__device__ __forceinline__ const T* head_row(const padoc_heads& x, int64_t row, int h) {
  return static_cast<const T*>(x.data) + row * x.row_stride + h * x.head_stride;
}

// Rows that a lane has in flight at once.  Measured, 18 heads of 128: 43,067 rows
// in bf16 69.9 us (74.4 with 4), 20,000 in fp32 67.5 (71.1).
constexpr int kAhead = 2;

// A tile of one tensor (q's or k's) as a workgroup sees it.
struct Tile {
  padoc_heads in, out, x;
  const void* w;
  int heads, h0;   // heads of the tile, from h0 on
  int64_t row0;
  int rows;
};

// Tile `b` of the launch; q's tiles come first.
__device__ __forceinline__ Tile tile_of(const RotaryParams& p, int64_t b) {
  Tile t;
  const bool is_q = b < p.tiles_q.items;
  const TileGrid& g = is_q ? p.tiles_q : p.tiles_k;
  if (!is_q) b -= p.tiles_q.items;
  const int64_t block = b / g.head_runs;
  t.h0 = (int)(b - block * g.head_runs) * g.heads;
  t.heads = min(g.heads, (is_q ? p.Hq : p.Hkv) - t.h0);
  t.row0 = block * g.rows;
  t.rows = (int)min((int64_t)g.rows, (int64_t)(is_q ? p.n_q : p.n) - t.row0);
  t.in = is_q ? p.q : p.k;
  t.out = is_q ? p.qo : p.ko;
  t.x = is_q ? p.xq : p.xk;
  t.w = is_q ? p.wq : p.wk;
  return t;
}

// A group's place among the (row, head) pairs of a tile, which the workgroup's
// groups take in turn.
struct Cursor {
  int row, h;
  __device__ __forceinline__ Cursor(const Tile& t, int group) : row(group / t.heads), h(group - row * t.heads) {}
  // To the place `groups` pairs on: dr rows and dh heads (groups = dr * heads + dh).
  __device__ __forceinline__ void next(const Tile& t, int dr, int dh) {
    row += dr;
    h += dh;
    if (h >= t.heads) {
      h -= t.heads;
      ++row;
    }
  }
  template <typename T>
  __device__ __forceinline__ T* at(const padoc_heads& x, const Tile& t) const {
    return static_cast<T*>(x.data) + (t.row0 + row) * x.row_stride + (t.h0 + h) * x.head_stride;
  }
};

// Rows of a tile: norm, rotation, and `put(row, head, values)`.  The first
// rows are asked for before the angles are computed, the others kAhead turns
// before theirs.
template <bool STREAM, typename T, int D, bool PAIRS, class Put>
__device__ __forceinline__ void turn_tile(const RotaryParams& p, const Tile& t, const int32_t* pos, int64_t pos_stride,
                                          AngleTable<T, D, PAIRS>& table, const Place<T, D, PAIRS>& pl, Put put) {
  constexpr int U = kAhead;
  const int dr = kGroups / t.heads, dh = kGroups - dr * t.heads;
  Cursor ahead(t, threadIdx.x / kLanes), at = ahead;
  Raw<T, D> raw[U], rw;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (ahead.row < t.rows) raw[u].template load<STREAM>(ahead.at<const T>(t.in, t), pl.at);
    ahead.next(t, dr, dh);
  }
  if (t.w) rw.template load<false>(static_cast<const T*>(t.w), pl.at);
  table.fill(p, pos, pos_stride, t.row0, t.rows);
  __syncthreads();
  float wt[kElems<D>];
  if (t.w) rw.get(wt);
  while (at.row < t.rows) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (at.row >= t.rows) break;
      float x[kElems<D>];
      raw[u].get(x);
      if (ahead.row < t.rows) raw[u].template load<STREAM>(ahead.at<const T>(t.in, t), pl.at);
      ahead.next(t, dr, dh);
      if (t.w) {
        const float rho = rms_scale<D>(x, p.eps);
#pragma unroll
        for (int i = 0; i < kElems<D>; ++i) x[i] *= rho * wt[i];
      }
      turn(x, table, at.row, pl);
      put(at, x);
      at.next(t, dr, dh);
    }
  }
  __syncthreads();
}

// Forward (and, with `inverse`, the backward of a rotation without norms).
template <typename T, int D, bool PAIRS, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotary_fwd_kernel(const RotaryParams p) {
  __shared__ AngleTable<T, D, PAIRS> table;
  const Place<T, D, PAIRS> pl(p.pairs);
  for (int64_t b = blockIdx.x; b < p.items; b += gridDim.x) {
    const Tile t = tile_of(p, b);
    turn_tile<STREAM>(p, t, p.pos, p.pos_stride, table, pl, [&](const Cursor& c, const float (&x)[kElems<D>]) {
      store_row(c.at<T>(t.out, t), pl.at, x);
    });
  }
}

// Workgroups of the backward for a compute unit: its launch bound, and how many
// items a unit gets of a long call.  (Its registers would let more run at once:
// 84 of them in bf16, d = 128, so five.)  Measured with items for 2, 3, 4 and 5
// workgroups a unit, 18 heads: 43,067 rows of 128 in bf16 120.7, 112.4, 117.9 and
// 117.9 us; 40,000 of 64 in bf16 78.8, 60.5, 59.2 and 59.5; 20,000 of 128 in fp32
// 115.0, 106.8, 110.5 and 110.5.
constexpr int bwd_per_unit(int D, bool bf16) { return D == 64 ? 4 : bf16 ? 3 : 2; }

// Backward: dx of an item's tiles, and the weight's gradient over them (fp32):
// in acc, lane by lane, then over the lanes that hold the same dimensions of a
// wavefront and over the four wavefronts through LDS, into part[item][D].  The
// tiles of an item lie as many rows apart as all items take at once, so that
// what the chip reads at a time is one stretch of memory.
template <typename T, int D, bool PAIRS, bool STREAM>
__global__ __launch_bounds__(kThreads, bwd_per_unit(D, sizeof(T) == 2)) void rotary_bwd_kernel(const RotaryParams p) {
  constexpr int U = sizeof(T) == 2 ? 2 : 1;  // rows of each tensor in flight
  __shared__ AngleTable<T, D, PAIRS> table;
  __shared__ float sums[kThreads / 64][D];
  const Place<T, D, PAIRS> pl(p.pairs);
  for (int64_t b = blockIdx.x; b < p.items; b += gridDim.x) {
    Tile t = tile_of(p, b);
    const int dr = kGroups / t.heads, dh = kGroups - dr * t.heads;
    float acc[kElems<D>] = {}, wt[kElems<D>];
    if (t.w) {
      Raw<T, D> rw;
      rw.template load<false>(static_cast<const T*>(t.w), pl.at);
      rw.get(wt);
    }
    const TileGrid& grid = b < p.tiles_q.items ? p.tiles_q : p.tiles_k;
    const int64_t apart = grid.items / grid.head_runs * grid.rows;
    for (; t.row0 < p.n; t.row0 += apart) {
      t.rows = (int)min((int64_t)grid.rows, p.n - t.row0);
      Cursor ahead(t, threadIdx.x / kLanes), at = ahead;
      Raw<T, D> rg[U], rx[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (ahead.row < t.rows) {
          rg[u].template load<STREAM>(ahead.at<const T>(t.in, t), pl.at);
          if (t.w) rx[u].template load<STREAM>(ahead.at<const T>(t.x, t), pl.at);
        }
        ahead.next(t, dr, dh);
      }
      table.fill(p, p.pos, p.pos_stride, t.row0, t.rows);
      __syncthreads();
      while (at.row < t.rows) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (at.row >= t.rows) break;
          float g[kElems<D>], x[kElems<D>];
          rg[u].get(g);
          if (t.w) rx[u].get(x);
          if (ahead.row < t.rows) {
            rg[u].template load<STREAM>(ahead.at<const T>(t.in, t), pl.at);
            if (t.w) rx[u].template load<STREAM>(ahead.at<const T>(t.x, t), pl.at);
          }
          ahead.next(t, dr, dh);
          turn(g, table, at.row, pl);
          if (t.w) {
            const float rho = rms_scale<D>(x, p.eps);
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < kElems<D>; ++i) {
              x[i] *= rho;
              acc[i] += g[i] * x[i];
              g[i] *= wt[i];
              dot += g[i] * x[i];
            }
            const float mean = group_sum(dot) * (1.f / D);
#pragma unroll
            for (int i = 0; i < kElems<D>; ++i) g[i] = rho * (g[i] - x[i] * mean);
          }
          store_row(at.at<T>(t.out, t), pl.at, g);
          at.next(t, dr, dh);
        }
      }
      __syncthreads();
    }
    if (!p.part) continue;
#pragma unroll
    for (int i = 0; i < kElems<D>; ++i) {
      float v = acc[i];
#pragma unroll
      for (int m = kLanes; m < 64; m *= 2) v += __shfl_xor(v, m);
      if (threadIdx.x % 64 < kLanes) sums[threadIdx.x / 64][pl.at[i / kUnit<T>] + i % kUnit<T>] = v;
    }
    __syncthreads();
    if (threadIdx.x < D) {
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < kThreads / 64; ++k) v += sums[k][threadIdx.x];
      p.part[b * D + threadIdx.x] = v;
    }
    __syncthreads();
  }
}

// Sums of the items' parts in a fixed order, in 64 bits: 16 columns of one
// tensor a workgroup (q's, then k's), 64 of its rows side by side.
__global__ __launch_bounds__(1024) void rotary_bwd_sum_kernel(const float* __restrict__ part, int64_t n_q, int64_t n_k,
                                                              int D, float* dwq, float* dwk) {
  __shared__ double sums[16][16];
  const int col = threadIdx.x % 16, r0 = threadIdx.x / 16;
  const bool is_q = (int)blockIdx.x * 16 < D;
  const int at = blockIdx.x * 16 + col - (is_q ? 0 : D);
  float* dw = is_q ? dwq : dwk;
  if (!dw) return;
  const float* src = part + (is_q ? 0 : n_q * D) + at;
  const int64_t n = is_q ? n_q : n_k;
  double v = 0;
#pragma unroll 8
  for (int64_t r = r0; r < n; r += 64) v += src[r * D];
  v += __shfl_xor(v, 16);
  v += __shfl_xor(v, 32);
  if (threadIdx.x % 64 < 16) sums[threadIdx.x / 64][col] = v;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  v = 0;
#pragma unroll
  for (int r = 0; r < 16; ++r) v += sums[r][col];
  dw[at] = (float)v;
}

__device__ __forceinline__ bool slot_of(const RotaryParams& p, int64_t row, int32_t& blk, int32_t& slot) {
  blk = p.slots[2 * row];
  slot = p.slots[2 * row + 1];
  return blk >= 0 && blk < p.n_blocks && slot >= 0 && slot < kBlock;
}

// V rows into the d-major cache: ROWS consecutive new rows of one head a
// workgroup.  A run of rows that go to consecutive slots of one half of a block
// (eight tokens) is written together: for each dimension one 16-byte store
// (bf16) where the half is whole, else its elements one by one.  A run belongs
// to the workgroup that its first row is in, so the rows are staged with the
// seven after them; two runs are written side by side, so that both halves of a
// block leave as 32 contiguous bytes a dimension.
template <typename T, int D, int ROWS>
struct VTile {
  static constexpr int kRows = ROWS + 7;
  static constexpr int kStride = D + 4 / (int)sizeof(T);  // bf16: two runs eight rows apart lie in other banks
  T tile[kRows * kStride];
  int64_t place[kRows + 1];  // slot of row first - 1 + i, counted through the pool; -2: none
  int32_t runs[ROWS];        // first row | length << 8
  int32_t n_runs;
};

template <bool STREAM, typename T, int D, int ROWS>
__device__ __forceinline__ void append_v(const RotaryParams& p, int64_t item, VTile<T, D, ROWS>& m) {
  constexpr int kRows = VTile<T, D, ROWS>::kRows, kStride = VTile<T, D, ROWS>::kStride;
  constexpr int E = kUnit<T>;
  T* tile = m.tile;
  int64_t* place = m.place;
  int32_t* runs = m.runs;
  const int64_t tiles = ((int64_t)p.n + ROWS - 1) / ROWS;
  const int h = (int)(item / tiles);
  const int64_t first = (item - h * tiles) * ROWS;
  const int tid = threadIdx.x;
  if (tid <= kRows) {
    const int64_t row = first - 1 + tid;
    int32_t blk, slot;
    const bool ok = row >= 0 && row < p.n && slot_of(p, row, blk, slot);
    place[tid] = ok ? (int64_t)blk * kBlock + slot : -2;
  }
#pragma unroll 4
  for (int u = tid; u < kRows * D / E; u += kThreads) {
    const int r = u / (D / E), c = u % (D / E) * E;
    if (first + r < p.n) {
      const u32x4 x = load_unit<STREAM>(head_row<T>(p.v, first + r, h) + c);
      T y[E];
      __builtin_memcpy(y, &x, 16);
#pragma unroll
      for (int e = 0; e < E; e += 4 / (int)sizeof(T))
        __builtin_memcpy(&tile[r * kStride + c + e], &y[e], 4);
    }
  }
  __syncthreads();
  if (tid < 64) {
    const int64_t s = tid < ROWS ? place[tid + 1] : -2;
    const bool leads = s >= 0 && (s % 8 == 0 || place[tid] != s - 1);
    int len = 1;
    while (leads && len < 8 - (int)(s % 8) && place[tid + 1 + len] == s + len) ++len;
    const uint64_t all = __ballot(leads);
    if (leads) runs[__popcll(all & ((1ull << tid) - 1))] = tid | len << 8;
    if (tid == 0) m.n_runs = __popcll(all);
  }
  __syncthreads();
  const int lane = tid % 64, n = m.n_runs;
  for (int step = tid / 64; step < (n + 1) / 2 * (D / 32); step += kThreads / 64) {
    const int run = step / (D / 32) * 2 + lane % 2;
    if (run >= n) continue;
    const int c = step % (D / 32) * 32 + lane / 2;
    const int r = runs[run] & 255, len = runs[run] >> 8;
    const int64_t s = place[r + 1];
    T* dst = static_cast<T*>(p.v_cache) + ((s / kBlock * p.Hkv + h) * D + c) * kBlock + s % kBlock;
    const T* src = tile + r * kStride + c;
    if (len == 8) {
      T y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = src[i * kStride];
      __builtin_memcpy(__builtin_assume_aligned(dst, 16), y, sizeof(y));
    } else {
      for (int i = 0; i < len; ++i) dst[i] = src[i * kStride];
    }
  }
  __syncthreads();
}

// Append: items of four roles, one after the other: v's rows into the V cache,
// tiles of q's rows into q_out, tiles of k's rows into their slots of the K
// cache, block-table patches.
template <typename T, int D, bool PAIRS, int ROWS, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotary_append_kernel(const RotaryParams p) {
  __shared__ union Shared {
    AngleTable<T, D, PAIRS> table;
    VTile<T, D, ROWS> v;
    __device__ Shared() {}
  } shared;
  const Place<T, D, PAIRS> pl(p.pairs);
  for (int64_t b = blockIdx.x; b < p.items; b += gridDim.x) {
    if (b < p.items_v) {
      append_v<STREAM>(p, b, shared.v);
      continue;
    }
    const int64_t i = b - p.items_v, n_q = p.tiles_q.items, n_turned = n_q + p.tiles_k.items;
    if (i >= n_turned) {
      const int64_t e = (i - n_turned) * kThreads + threadIdx.x;
      if (e < p.n_patch) p.block_table[p.patch[2 * e]] = p.patch[2 * e + 1];
      continue;
    }
    const Tile t = tile_of(p, i);
    const bool is_q = i < n_q;
    T* cache = static_cast<T*>(p.k_cache);
    turn_tile<STREAM>(p, t, is_q ? p.q_pos : p.pos, is_q ? p.q_pos_stride : p.pos_stride, shared.table, pl,
              [&](const Cursor& c, const float (&x)[kElems<D>]) {
      if (is_q) {
        store_row(c.at<T>(t.out, t), pl.at, x);
        return;
      }
      int32_t blk, slot;
      if (!slot_of(p, t.row0 + c.row, blk, slot)) return;
      // (16 bytes of a line each: plain stores, which the L2 puts together)
#pragma unroll
      for (int u = 0; u < kUnits<T, D>; ++u) {
        T* dst = cache + paged_k_offset<D>(blk, t.h0 + c.h, p.Hkv, slot, pl.at[u] / 8) + pl.at[u] % 8;
        *reinterpret_cast<u32x4*>(dst) = pack_unit(dst, x + u * kUnit<T>);
      }
    });
  }
}

// Maximum over the eight lanes of a group, in every one of them.
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true));
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));
}

// The codes of a row that a group holds, and its scale byte.
template <int N>
__device__ __forceinline__ uint32_t quantize_row(const float (&x)[N], uint32_t (&codes)[N / 4], uint32_t nan_codes) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) a = max(a, __float_as_uint(x[i]) & 0x7fffffffu);
  const uint32_t b = e4m3::scale_byte(group_max(a));
  const float r = e4m3::inverse_scale(b);
#pragma unroll
  for (int i = 0; i < N; i += 4)
    codes[i / 4] = b == e4m3::kNan ? nan_codes : e4m3::codes4(x[i], x[i + 1], x[i + 2], x[i + 3], r);
  return b;
}

// z rounded to fp32 to odd: where fp32 does not hold it, towards zero with the last bit
// set, so that a second rounding, to a code, and a comparison see it as they would z.
__device__ __forceinline__ float round_to_odd(double z) {
  const uint32_t lo = (uint32_t)__double2loint(z);
  const uint32_t odd = (lo & 0x1fffffffu) ? 0x20000000u : 0u;
  return (float)__hiloint2double(__double2hiint(z), (int)((lo & 0xe0000000u) | odd));
}

// A tile of K's rows for an 8-bit cache, normed and rotated in 64 bits, off by some
// 2^-36 + 2 pi |pos| 2^-64 of scale (|y_a| + |y_b|) of a pair (up to position 2^25 the first
// is the larger): a code has four significant bits, and fp32's errors in z (1.2 units of 2^-24
// of it, 1.9 with v_rsq_f32's own) would move a value in some 2^20 across the border
// between two of them, which then differs by a sixteenth; so is one in some 2^32, or in
// 2^26 at the farthest positions.  K has few of a call's rows,
// and q's, which go past memory meanwhile, hide them (K in fp32: 41.7 us where this took 47.7).
template <bool STREAM, typename T, int D, bool PAIRS, class Put>
__device__ __forceinline__ void turn_tile_wide(const RotaryParams& p, const Tile& t, const int32_t* pos, int64_t pos_stride,
                                               AngleTable<T, D, PAIRS, double>& table, const Place<T, D, PAIRS>& pl, Put put) {
  typedef Place<T, D, PAIRS> P;
  const int dr = kGroups / t.heads, dh = kGroups - dr * t.heads;
  Cursor at(t, threadIdx.x / kLanes);
  Raw<T, D> raw, rw{};
  if (at.row < t.rows) raw.template load<STREAM>(at.at<const T>(t.in, t), pl.at);
  if (t.w) rw.template load<false>(static_cast<const T*>(t.w), pl.at);
  table.fill(p, pos, pos_stride, t.row0, t.rows);
  __syncthreads();
  while (at.row < t.rows) {
    float x[kElems<D>];
    raw.get(x);
    const Cursor here = at;
    at.next(t, dr, dh);
    if (at.row < t.rows) raw.template load<STREAM>(at.at<const T>(t.in, t), pl.at);
    double rho = 1.;
    if (t.w) {
      double s = 0.;
#pragma unroll
      for (int i = 0; i < kElems<D>; ++i) s += (double)x[i] * (double)x[i];
      const double v = group_sum(s) * (1. / D) + (double)p.eps;
      rho = __builtin_amdgcn_rsq(v);
      const double e = fma(-v * rho, rho, 1.);  // (NaN where v is 0 or infinite: the root is exact)
      rho = e == e ? fma(0.5 * rho, e, rho) : rho;
    }
    // (Else the compiler keeps every element and weight in 64 bits as well.)
#pragma unroll
    for (int i = 0; i < kElems<D>; ++i) asm("" : "+v"(x[i]));
#pragma unroll
    for (int i = 0; i < kUnits<T, D>; ++i) asm("" : "+v"(rw.u[i]));
    auto normed = [&](int i) { return t.w ? (double)x[i] * (rho * (double)rw.elem(i)) : (double)x[i]; };
#pragma unroll
    for (int m0 = 0; m0 < P::kSlots * P::kPairsPerSlot; m0 += 2) {
      const bool turned = m0 / P::kPairsPerSlot < pl.turned;
      const auto cs = table.at[here.row][m0 / 2][threadIdx.x % P::kSlotLanes];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const double c = cs[2 * j], s = cs[2 * j + 1];
        const int a = P::first(m0 + j), b = P::second(m0 + j) % kElems<D>;
        const double ya = normed(a);
        if (P::kSplit) {
          const double yb = other_half(ya);
          x[a] = round_to_odd(!turned ? ya : ya * c + yb * (threadIdx.x % kLanes < P::kSlotLanes ? -s : s));
        } else {
          const double yb = normed(b);
          x[a] = round_to_odd(turned ? ya * c - yb * s : ya);
          x[b] = round_to_odd(turned ? yb * c + ya * s : yb);
        }
      }
      __builtin_amdgcn_sched_barrier(0);  // (its values are done with before the next ones)
    }
    put(here, x);
  }
  __syncthreads();
}

// V's codes of one row and head, byte by byte (d-major V).
template <typename T, int D, bool PAIRS>
__device__ __forceinline__ void store_bytes(uint8_t* dst, const Place<T, D, PAIRS>& pl, const uint32_t (&codes)[kElems<D> / 4]) {
  constexpr int E = kUnit<T>;
#pragma unroll
  for (int i = 0; i < kElems<D>; ++i) dst[(pl.at[i / E] + i % E) * kBlock] = (uint8_t)(codes[i / 4] >> (8 * (i % 4)));
}

// V rows of a prefill into an 8-bit cache: ROWS consecutive new rows of one head
// a workgroup, whose codes are staged.  Sixteen rows that fill a block are written
// together, 16 bytes for each dimension, by the workgroup that their first row is
// in (so the fifteen rows after its own are staged too); the others byte by byte.
template <int D, int ROWS>
struct VCodes {
  static constexpr int kAround = kBlock - 1;  // rows before and after that a whole block can reach
  static constexpr int kRows = ROWS + kAround;
  static constexpr int kStride = D + 4;  // codes and the scale
  uint8_t tile[kRows * kStride];
  int64_t place[kRows + kAround];  // slot of row first - kAround + i, counted through the pool; -2: none
  bool whole[kRows];               // whether row first - kAround + i is the first of a whole block
  int32_t runs[ROWS];              // own rows that are
  int32_t n_runs;
};

template <bool STREAM, typename T, int D, bool PAIRS, int ROWS>
__device__ __forceinline__ void append_v_e4m3(const RotaryParams& p, const Place<T, D, PAIRS>& pl, int64_t item,
                                              VCodes<D, ROWS>& m) {
  using M = VCodes<D, ROWS>;
  constexpr int kRows = M::kRows, kStride = M::kStride, kAround = M::kAround;
  constexpr int E = kUnit<T>, kTurns = (kRows + kGroups - 1) / kGroups;
  static_assert(ROWS == 64 && kRows + kAround <= kThreads, "whole blocks among the own rows are listed by one wavefront");
  const int64_t tiles = ((int64_t)p.n + ROWS - 1) / ROWS;
  const int h = (int)(item / tiles);
  const int64_t first = (item - h * tiles) * ROWS;
  const int tid = threadIdx.x, group = tid / kLanes;
  if (tid < kRows + kAround) {
    const int64_t row = first - kAround + tid;
    int32_t blk, slot;
    const bool ok = row >= 0 && row < p.n && slot_of(p, row, blk, slot);
    m.place[tid] = ok ? (int64_t)blk * kBlock + slot : -2;
  }
  auto in = [&](int r) { return r < kRows && first + r < p.n; };  // (a group's lanes together)
  Raw<T, D> raw[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i)
    if (in(i * kGroups + group)) raw[i].template load<STREAM>(head_row<T>(p.v, first + i * kGroups + group, h), pl.at);
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    __builtin_amdgcn_sched_barrier(0);  // (a turn's values at a time)
    const int r = i * kGroups + group;
    if (!in(r)) continue;
    float x[kElems<D>];
    raw[i].get(x);
    uint32_t codes[kElems<D> / 4];
    const uint32_t scale = quantize_row(x, codes, 0);
    if (tid % kLanes == 0) m.tile[r * kStride + D] = (uint8_t)scale;
#pragma unroll
    for (int u = 0; u < kUnits<T, D>; ++u)
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<uint32_t*>(&m.tile[r * kStride + pl.at[u] + e]) = codes[(u * E + e) / 4];
  }
  __syncthreads();
  if (tid < kRows) {  // the own rows, then those before
    const int i = tid < ROWS ? kAround + tid : tid - ROWS;
    const int64_t s = m.place[i];
    bool whole = s >= 0 && s % kBlock == 0;
#pragma unroll
    for (int j = 1; j < kBlock; ++j) whole = whole && m.place[i + j] == s + j;
    m.whole[i] = whole;
    if (tid < ROWS) {
      const uint64_t all = __ballot(whole);
      if (whole) m.runs[__popcll(all & ((1ull << tid) - 1))] = tid;
      if (tid == 0) m.n_runs = __popcll(all);
    }
  }
  __syncthreads();
  const int lane = tid % 64, n = m.n_runs;
  for (int step = tid / 64; step < n * (D / 64); step += kThreads / 64) {
    const int c = step % (D / 64) * 64 + lane;
    const int r = m.runs[step / (D / 64)];
    const int64_t s = m.place[r + kAround];
    const uint8_t* src = m.tile + r * kStride + c;
    u32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      y[i] = (uint32_t)src[4 * i * kStride] | (uint32_t)src[(4 * i + 1) * kStride] << 8 |
             (uint32_t)src[(4 * i + 2) * kStride] << 16 | (uint32_t)src[(4 * i + 3) * kStride] << 24;
    *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(p.v_cache) + e4m3::codes_at<D>(s / kBlock, h, p.Hkv) + c * kBlock) = y;
  }
#pragma unroll
  for (int i = 0; i < ROWS / kGroups; ++i) {
    const int r = i * kGroups + group;
    const int64_t s = m.place[r + kAround];
    if (s < 0) continue;
    const int slot = (int)(s % kBlock), lead = r + kAround - slot;
    if (!(m.whole[lead] && m.place[lead] == s - slot)) {
      uint32_t codes[kElems<D> / 4];
#pragma unroll
      for (int u = 0; u < kUnits<T, D>; ++u)
#pragma unroll
        for (int e = 0; e < E; e += 4)
          codes[(u * E + e) / 4] = *reinterpret_cast<const uint32_t*>(&m.tile[r * kStride + pl.at[u] + e]);
      store_bytes<T, D>(static_cast<uint8_t*>(p.v_cache) + e4m3::codes_at<D>(s / kBlock, h, p.Hkv) + slot, pl, codes);
    }
    if (tid % kLanes == 0) p.scales[e4m3::scales_at(s / kBlock, h, p.Hkv) + kBlock + slot] = m.tile[r * kStride + D];
  }
  __syncthreads();
}

// Append into an 8-bit cache: items of four roles, as above.  ROWS == 0: v's
// tiles are cut like k's, a group takes a row of one head, and its lanes leave a
// byte per dimension (d-major V).  A workgroup makes one item (a loop over items
// would keep what one role needs in registers for the others: 128 of them and spills
// where 96 do).  Bound by memory: 20,456 rows of 16 + 2 + 2 heads of 128 in bf16, in 8
// runs, take 40.5 us (4.92 TB/s; a copy reaches 5.1 to 5.3), with the loop 47.7, with V
// byte by byte some 11 more; 5,439 rows of 28 + 4 + 4 heads of 64 in fp32 16.3.
template <typename T, int D, bool PAIRS, int ROWS, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotary_append_e4m3_kernel(const RotaryParams p) {
  __shared__ union Shared {
    AngleTable<T, D, PAIRS> table;
    AngleTable<T, D, PAIRS, double> wide;
    VCodes<D, 64> v;
    __device__ Shared() {}
  } shared;
  constexpr int E = kUnit<T>;
  const Place<T, D, PAIRS> pl(p.pairs);
  const int64_t b = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (b >= p.items) return;
  if (b < p.items_v) {
    if constexpr (ROWS > 0) {
      append_v_e4m3<STREAM>(p, pl, b, shared.v);
    } else {
      Tile t = tile_of(p, b + p.tiles_q.items);  // (k's tile of the same rows and heads)
      t.in = p.v;
      const int dr = kGroups / t.heads, dh = kGroups - dr * t.heads;
      for (Cursor c(t, threadIdx.x / kLanes); c.row < t.rows; c.next(t, dr, dh)) {
        Raw<T, D> raw;
        raw.template load<STREAM>(c.at<const T>(t.in, t), pl.at);
        float x[kElems<D>];
        raw.get(x);
        uint32_t codes[kElems<D> / 4];
        const uint32_t scale = quantize_row(x, codes, 0);
        int32_t blk, slot;
        if (!slot_of(p, t.row0 + c.row, blk, slot)) continue;
        const int h = t.h0 + c.h;
        uint8_t* dst = static_cast<uint8_t*>(p.v_cache) + e4m3::codes_at<D>(blk, h, p.Hkv) + slot;
        store_bytes<T, D>(dst, pl, codes);
        if (threadIdx.x % kLanes == 0) p.scales[e4m3::scales_at(blk, h, p.Hkv) + kBlock + slot] = (uint8_t)scale;
      }
    }
    return;
  }
  const int64_t i = b - p.items_v, n_q = p.tiles_q.items, n_turned = n_q + p.tiles_k.items;
  if (i >= n_turned) {
    const int64_t e = (i - n_turned) * kThreads + threadIdx.x;
    if (e < p.n_patch) p.block_table[p.patch[2 * e]] = p.patch[2 * e + 1];
    return;
  }
  // (k's tiles before q's: they wait longer for each row, and q's fill the time)
  const Tile t = tile_of(p, i < n_turned - n_q ? i + n_q : i - (n_turned - n_q));
  if (i >= n_turned - n_q) {
    turn_tile<STREAM>(p, t, p.q_pos, p.q_pos_stride, shared.table, pl, [&](const Cursor& c, const float (&x)[kElems<D>]) {
      store_row(c.at<T>(t.out, t), pl.at, x);
    });
    return;
  }
  turn_tile_wide<STREAM>(p, t, p.pos, p.pos_stride, shared.wide, pl, [&](const Cursor& c, const float (&x)[kElems<D>]) {
    uint32_t codes[kElems<D> / 4];
    const uint32_t scale = quantize_row(x, codes, e4m3::kNanCodes);
    int32_t blk, slot;
    if (!slot_of(p, t.row0 + c.row, blk, slot)) return;
    const int h = t.h0 + c.h;
    uint8_t* dst = static_cast<uint8_t*>(p.k_cache) + e4m3::codes_at<D>(blk, h, p.Hkv);
#pragma unroll
    for (int u = 0; u < kUnits<T, D>; ++u)
      __builtin_memcpy(__builtin_assume_aligned(dst + e4m3::k_at(slot, pl.at[u]), E), &codes[u * E / 4], E);
    if (threadIdx.x % kLanes == 0) p.scales[e4m3::scales_at(blk, h, p.Hkv) + slot] = (uint8_t)scale;
  });
}

constexpr int64_t kMaxGrid = 1 << 20;  // workgroups of a launch: the rest by strides

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of n rows of H heads (of H_all that the launch turns): as many turns a
// group (up to max_turns) as leave the chip about that many workgroups, so that
// a short call is spread over the chip.
TileGrid tile_grid(int64_t n, int H, int H_all, int max_turns, int64_t workgroups) {
  TileGrid g{};
  if (n == 0 || H == 0) return g;
  const int64_t turns = std::min<int64_t>(max_turns, ceil_div(n * H_all, kGroups * workgroups));
  g.heads = (int32_t)std::min<int64_t>(H, kGroups * turns);
  g.head_runs = (int32_t)ceil_div(H, g.heads);
  g.rows = (int32_t)std::max<int64_t>(1, std::min<int64_t>({kGroups * turns / g.heads, kGroups, n}));
  g.items = ceil_div(n, g.rows) * g.head_runs;
  return g;
}

template <template <typename, int, bool> class Call>
hipError_t dispatch(const RotaryParams& p, int D, bool bf16, bool pairs, dim3 grid, hipStream_t s) {
  if (bf16) {
    if (D == 64)
      pairs ? Call<__bf16, 64, true>::go(p, grid, s) : Call<__bf16, 64, false>::go(p, grid, s);
    else
      pairs ? Call<__bf16, 128, true>::go(p, grid, s) : Call<__bf16, 128, false>::go(p, grid, s);
  } else {
    if (D == 64)
      pairs ? Call<float, 64, true>::go(p, grid, s) : Call<float, 64, false>::go(p, grid, s);
    else
      pairs ? Call<float, 128, true>::go(p, grid, s) : Call<float, 128, false>::go(p, grid, s);
  }
  return hipGetLastError();
}

template <bool STREAM>
struct Fwd {
  template <typename T, int D, bool PAIRS>
  struct Call {
    static void go(const RotaryParams& p, dim3 grid, hipStream_t s) {
      hipLaunchKernelGGL((rotary_fwd_kernel<T, D, PAIRS, STREAM>), grid, dim3(kThreads), 0, s, p);
    }
  };
};
template <bool STREAM>
struct Bwd {
  template <typename T, int D, bool PAIRS>
  struct Call {
    static void go(const RotaryParams& p, dim3 grid, hipStream_t s) {
      hipLaunchKernelGGL((rotary_bwd_kernel<T, D, PAIRS, STREAM>), grid, dim3(kThreads), 0, s, p);
    }
  };
};
template <int ROWS, bool STREAM>
struct Append {
  template <typename T, int D, bool PAIRS>
  struct Call {
    static void go(const RotaryParams& p, dim3 grid, hipStream_t s) {
      hipLaunchKernelGGL((rotary_append_kernel<T, D, PAIRS, ROWS, STREAM>), grid, dim3(kThreads), 0, s, p);
    }
  };
};

template <int ROWS, bool STREAM>
struct AppendE4m3 {
  template <typename T, int D, bool PAIRS>
  struct Call {
    static void go(const RotaryParams& p, dim3 grid, hipStream_t s) {
      hipLaunchKernelGGL((rotary_append_e4m3_kernel<T, D, PAIRS, ROWS, STREAM>), grid, dim3(kThreads), 0, s, p);
    }
  };
};

// Whether a call that moves `rows` rows of a head goes past the caches.
bool streams(int64_t rows, int D, bool bf16) { return rows * D * (bf16 ? 2 : 4) > kStreamBytes; }

dim3 grid_of(int64_t items) { return dim3((unsigned)std::min(items, kMaxGrid)); }

// The backward's items.  A short call is cut into about 384 tiles, an item each
// (the sums at their ends then weigh less than in more of them), a long one into
// as many items as above, each of them some tiles, with their D sums left once.
// Measured for 384, 512, 768 and 1,024 tiles, 18 heads of 128 in bf16: 3,479 rows
// 18.3, 18.1, 16.3 and 21.0 us a call, 8,000 26.3, 26.3, 27.6 and 27.1; 3,479 in
// fp32 24.4, 25.4, 24.6 and 25.3.
constexpr int kComputeUnits = 256;
void bwd_grids(int64_t n, int Hq, int Hkv, int D, bool bf16, TileGrid& q, TileGrid& k) {
  q = tile_grid(n, Hq, Hq + Hkv, 8, kComputeUnits * 3 / 2);
  k = tile_grid(n, Hkv, Hq + Hkv, 8, kComputeUnits * 3 / 2);
  const int64_t held = kComputeUnits * bwd_per_unit(D, bf16);
  const int64_t passes = ceil_div(q.items + k.items, held);
  for (TileGrid* g : {&q, &k})
    if (g->items > 0) g->items = ceil_div(g->items / g->head_runs, passes) * g->head_runs;
}

}  // namespace

size_t rotary_bwd_parts(int64_t n, int Hq, int Hkv, int D, bool bf16) {
  TileGrid q, k;
  bwd_grids(n, Hq, Hkv, D, bf16, q, k);
  return (size_t)(q.items + k.items);
}

hipError_t launch_rotary_fwd(RotaryParams p, int D, bool bf16, bool pairs, hipStream_t s) {
  p.n_q = p.n;
  p.tiles_q = tile_grid(p.n, p.Hq, p.Hq + p.Hkv, 4, 4 * kComputeUnits);
  p.tiles_k = tile_grid(p.n, p.Hkv, p.Hq + p.Hkv, 4, 4 * kComputeUnits);
  p.items = p.tiles_q.items + p.tiles_k.items;
  if (p.items == 0) return hipSuccess;
  return streams((int64_t)p.n * (p.Hq + p.Hkv) * 2, D, bf16)
             ? dispatch<Fwd<true>::Call>(p, D, bf16, pairs, grid_of(p.items), s)
             : dispatch<Fwd<false>::Call>(p, D, bf16, pairs, grid_of(p.items), s);
}

hipError_t launch_rotary_bwd(RotaryParams p, int D, bool bf16, bool pairs, float* dwq, float* dwk, hipStream_t s) {
  p.n_q = p.n;
  bwd_grids(p.n, p.Hq, p.Hkv, D, bf16, p.tiles_q, p.tiles_k);
  p.items = p.tiles_q.items + p.tiles_k.items;
  if (p.items > 0) {
    const hipError_t e = streams((int64_t)p.n * (p.Hq + p.Hkv) * 3, D, bf16)
                             ? dispatch<Bwd<true>::Call>(p, D, bf16, pairs, grid_of(p.items), s)
                             : dispatch<Bwd<false>::Call>(p, D, bf16, pairs, grid_of(p.items), s);
    if (e != hipSuccess) return e;
  }
  if (dwq || dwk)
    hipLaunchKernelGGL(rotary_bwd_sum_kernel, dim3(2 * D / 16), dim3(1024), 0, s, p.part, p.tiles_q.items,
                       p.tiles_k.items, D, dwq, dwk);
  return hipGetLastError();
}

hipError_t launch_rotary_append(RotaryParams p, int D, bool bf16, bool pairs, hipStream_t s) {
  p.tiles_q = tile_grid(p.n_q, p.Hq, p.Hq + p.Hkv, 4, 4 * kComputeUnits);
  p.tiles_k = tile_grid(p.n, p.Hkv, p.Hq + p.Hkv, 4, 4 * kComputeUnits);
  // V rows of a workgroup: 64 of many (a prefill's runs, whole), 8 of few (a
  // decode step's scattered rows, spread over the chip).  Where the rows lie is
  // known on the device alone, so the count decides, about where the two cross for
  // scattered rows.  Measured, bf16, d = 128, 2 KV heads, us a call in eights and
  // in 64s: scattered, 1,600 rows 10.6 and 16.2, 2,400 12.9 and 17.1, 3,200 15.9
  // and 17.8, 4,000 20.8 and 18.8, 5,000 25.4 and 22.0; in eight runs, 1,600 rows
  // 10.5 and 9.5, 2,400 10.5 and 9.4, 3,200 12.0 and 9.8, 4,000 13.3 and 10.4,
  // 20,000 53.4 and 41.8.
  const bool tall = (int64_t)p.n * p.Hkv >= 6144;
  p.items_v = ceil_div(p.n, tall ? 64 : 8) * p.Hkv;
  p.items = p.items_v + p.tiles_q.items + p.tiles_k.items + ceil_div(p.n_patch, kThreads);
  if (p.items == 0) return hipSuccess;
  const dim3 grid = grid_of(p.items);
  if (!tall) return dispatch<Append<8, false>::Call>(p, D, bf16, pairs, grid, s);
  return streams(((int64_t)p.n_q * p.Hq + (int64_t)p.n * p.Hkv * 2) * 2, D, bf16)
             ? dispatch<Append<64, true>::Call>(p, D, bf16, pairs, grid, s)
             : dispatch<Append<64, false>::Call>(p, D, bf16, pairs, grid, s);
}

// Rows (of all heads) from which V's go in tiles of 64 rows.  As above, the
// count decides, as the kernel does not know scattered rows (a token a stream) from runs
// before it has read the slots: above the threshold scattered ones lose 1.3 to 2.0 us by it,
// runs win 0.6 to 3.5.  Measured without queries, us a call byte by byte and in tiles, in
// runs and scattered: 2 heads of 128 in bf16, 2,400 rows 6.7 and 6.2, 9.4 and 11.2;
// 3,200 rows 6.7 and 6.1, 10.6 and 12.6; 6,400 rows 9.1 and 6.3, 15.4 and 16.7; 8 heads,
// 400 rows 6.2 and 6.2, 6.9 and 10.2; 800 rows 9.6 and 6.1, 10.3 and 12.2; 4 heads of
// 64 in fp32, 1,600 rows 5.1 and 5.1, 7.0 and 8.0.
constexpr int64_t kTallE4m3 = 6144;

hipError_t launch_rotary_append_e4m3(RotaryParams p, int D, bool bf16, bool pairs, hipStream_t s) {
  p.tiles_q = tile_grid(p.n_q, p.Hq, p.Hq + p.Hkv, 4, 4 * kComputeUnits);
  p.tiles_k = tile_grid(p.n, p.Hkv, p.Hq + p.Hkv, 4, 4 * kComputeUnits);
  const bool tall = (int64_t)p.n * p.Hkv >= kTallE4m3;
  p.items_v = tall ? ceil_div(p.n, 64) * p.Hkv : p.tiles_k.items;
  p.items = p.items_v + p.tiles_q.items + p.tiles_k.items + ceil_div(p.n_patch, kThreads);
  if (p.items == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min(p.items, kMaxGrid), (unsigned)ceil_div(p.items, kMaxGrid));  // (an item a workgroup)
  if (!tall) return dispatch<AppendE4m3<0, false>::Call>(p, D, bf16, pairs, grid, s);
  return streams((int64_t)p.n_q * p.Hq * 2 + (int64_t)p.n * p.Hkv * 3, D, bf16)
             ? dispatch<AppendE4m3<64, true>::Call>(p, D, bf16, pairs, grid, s)
             : dispatch<AppendE4m3<64, false>::Call>(p, D, bf16, pairs, grid, s);
}

}  // namespace padoc
