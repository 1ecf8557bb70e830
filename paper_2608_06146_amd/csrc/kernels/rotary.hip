// Head norms and rotary positions: rows of Q and K before the attention
// (forward), their gradients (backward), and a decode step's rows on their way
// into the paged caches (append).
//
//   y = w x / sqrt(mean x^2 + eps)  (or x),  z = scale R(pos * inv_freq) y
//   dy = scale R(-angle) dz,  g = w dy,  dw = sum dy x rho,
//   dx = rho (g - x rho^2 mean(g x)),  rho = 1 / sqrt(mean x^2 + eps)
//
// All of it is bound by memory: every element is read once and written once.
// A row of one head is shared by D / 16 lanes (a group).  Lane l of a group
// holds 16 dimensions: the eight pairs 8l .. 8l+7, so that a rotation stays
// inside a lane and its memory accesses are 16 bytes each; where only the
// leading dimensions are rotated, the lanes behind them hold the rest.  A group
// takes several heads of one row one after the other: it computes the row's
// eight cosines and sines per lane once.
//
// Angles: a position times the pair's 64-bit fraction of a turn, modulo 2^64,
// is the angle in turns; its leading 32 bits are split into a quadrant and an
// angle within +-pi/4, whose sine and cosine are Taylor sums (to x^9 and x^10:
// remainders below 2e-9).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../rotary.hpp"
#include "device_common.hpp"

namespace padoc {
namespace {

constexpr int kThreads = 256;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// Eight elements at an address aligned to one element.
__device__ __forceinline__ void load8(const __bf16* p, float* x) {
  typedef u32x4 unit __attribute__((aligned(2)));
  const u32x4 u = *reinterpret_cast<const unit*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float* x) {
  typedef f32x4 unit __attribute__((aligned(4)));
  const f32x4 a = reinterpret_cast<const unit*>(p)[0], b = reinterpret_cast<const unit*>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = a[i];
    x[4 + i] = b[i];
  }
}
// Rounded to nearest-even once, here (NaN stays NaN).
__device__ __forceinline__ void store8(__bf16* p, const float* x) {
  typedef u32x4 unit __attribute__((aligned(2)));
  const bf16x8 b = __builtin_convertvector((f32x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}), bf16x8);
  u32x4 u;
  __builtin_memcpy(&u, &b, 16);
  *reinterpret_cast<unit*>(p) = u;
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  typedef f32x4 unit __attribute__((aligned(4)));
  reinterpret_cast<unit*>(p)[0] = f32x4{x[0], x[1], x[2], x[3]};
  reinterpret_cast<unit*>(p)[1] = f32x4{x[4], x[5], x[6], x[7]};
}

// A lane's 16 values of a head: its two chunks, one after the other.
template <typename T>
__device__ __forceinline__ void load16v(const T* p, const int (&at)[2], float (&x)[16]) {
  load8(p + at[0], x);
  load8(p + at[1], x + 8);
}
template <typename T>
__device__ __forceinline__ void store16v(T* p, const int (&at)[2], const float (&x)[16]) {
  store8(p + at[0], x);
  store8(p + at[1], x + 8);
}

// Sum over the L (4 or 8) lanes of a group, in every one of them.
template <int L>
__device__ __forceinline__ float group_sum(float v) {
  v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xf, 0xf, true));  // lane ^ 1
  v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xf, 0xf, true));  // lane ^ 2
  if (L == 8) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xf, 0xf, true));  // 7 - lane
  return v;
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

// A lane's place in its group: element offsets of its two 8-element chunks,
// and whether it holds rotated pairs.
template <int D, bool PAIRS>
struct Place {
  int at[2];
  int first_pair;
  bool turned;
  __device__ __forceinline__ Place(int lane, int pairs) {
    first_pair = 8 * lane;
    turned = first_pair < pairs;
    if (PAIRS || !turned) {  // neighbouring chunks (behind the rotated ones: the same in both styles)
      at[0] = 16 * lane;
      at[1] = 16 * lane + 8;
    } else {
      at[0] = 8 * lane;
      at[1] = 8 * lane + pairs;
    }
  }
};

struct Angles {
  float c[8], s[8];
};

// Cosines and sines of a lane's pairs for a row (scaled; the sine negated for
// the inverse rotation).
__device__ __forceinline__ Angles angles(const RotaryParams& p, const int32_t* pos, int64_t stride, int64_t row,
                                         int first_pair, bool turned) {
  Angles a;
  if (!turned) return a;
  int32_t at[kMaxAxes];
#pragma unroll
  for (int x = 0; x < kMaxAxes; ++x) at[x] = x < p.n_axes ? pos[x * stride + row] : 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int ax = p.table.axis[first_pair + j];
    const int32_t m = ax == 0 ? at[0] : ax == 1 ? at[1] : ax == 2 ? at[2] : at[3];
    float s, c;
    sincos_turns((uint32_t)((uint64_t)(int64_t)m * p.table.turn[first_pair + j] >> 32), s, c);
    a.c[j] = c * p.scale;
    a.s[j] = p.inverse ? -s * p.scale : s * p.scale;
  }
  return a;
}

// Rotate a lane's pairs.
template <bool PAIRS>
__device__ __forceinline__ void turn(float (&x)[16], const Angles& t) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int a = PAIRS ? 2 * j : j, b = PAIRS ? 2 * j + 1 : 8 + j;
    const float ya = x[a], yb = x[b];
    x[a] = ya * t.c[j] - yb * t.s[j];
    x[b] = yb * t.c[j] + ya * t.s[j];
  }
}

template <int D>
__device__ __forceinline__ float rms_scale(const float (&x)[16], float eps) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += x[i] * x[i];
  return __builtin_amdgcn_rsqf(group_sum<D / 16>(s) * (1.f / D) + eps);
}

template <typename T>
__device__ __forceinline__ const T* head_row(const padoc_heads& x, int64_t row, int h) {
  return static_cast<const T*>(x.data) + row * x.row_stride + h * x.head_stride;
}

// Heads [h0, h1) of a row of one tensor: norm, rotation, and `put(h, values)`.
template <typename T, int D, bool PAIRS, class Put>
__device__ __forceinline__ void turn_heads(const padoc_heads& in, const void* w, int64_t row, int h0, int h1,
                                           const Place<D, PAIRS>& pl, const Angles& t, float eps, Put put) {
  float wt[16];
  if (w) load16v(static_cast<const T*>(w), pl.at, wt);
  for (int h = h0; h < h1; ++h) {
    float x[16];
    load16v(head_row<T>(in, row, h), pl.at, x);
    if (w) {
      const float rho = rms_scale<D>(x, eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] *= rho * wt[i];
    }
    if (pl.turned) turn<PAIRS>(x, t);
    put(h, x);
  }
}

// Forward (and, with `inverse`, the backward of a rotation without norms).
// blockIdx.x, + gridDim.x, ...: kThreads / L rows, a group each; blockIdx.y: a
// run of heads, q's before k's.
template <typename T, int D, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rotary_fwd_kernel(const RotaryParams p) {
  constexpr int L = D / 16, R = kThreads / L;
  const Place<D, PAIRS> pl(threadIdx.x % L, p.pairs);
  const int h0 = blockIdx.y * p.heads_per_group, h1 = min(h0 + p.heads_per_group, p.Hq + p.Hkv);
  for (int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L; row < p.n; row += (int64_t)gridDim.x * R) {
    const Angles t = angles(p, p.pos, p.pos_stride, row, pl.first_pair, pl.turned);
    turn_heads<T, D, PAIRS>(p.q, p.wq, row, h0, min(h1, p.Hq), pl, t, p.eps, [&](int h, const float (&x)[16]) {
      store16v(const_cast<T*>(head_row<T>(p.qo, row, h)), pl.at, x);
    });
    turn_heads<T, D, PAIRS>(p.k, p.wk, row, max(h0 - p.Hq, 0), h1 - p.Hq, pl, t, p.eps, [&](int h, const float (&x)[16]) {
      store16v(const_cast<T*>(head_row<T>(p.ko, row, h)), pl.at, x);
    });
  }
}

// Backward of heads [h0, h1) of a row: dx, and the weight's gradient added up
// in acc.
template <typename T, int D, bool PAIRS>
__device__ __forceinline__ void turn_heads_bwd(const padoc_heads& dz, const padoc_heads& xin, const padoc_heads& out,
                                               const void* w, int64_t row, int h0, int h1, const Place<D, PAIRS>& pl,
                                               const Angles& t, float eps, float (&acc)[16]) {
  float wt[16];
  if (w) load16v(static_cast<const T*>(w), pl.at, wt);
  for (int h = h0; h < h1; ++h) {
    float g[16];
    load16v(head_row<T>(dz, row, h), pl.at, g);
    if (pl.turned) turn<PAIRS>(g, t);
    if (w) {
      float x[16];
      load16v(head_row<T>(xin, row, h), pl.at, x);
      const float rho = rms_scale<D>(x, eps);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[i] *= rho;
        acc[i] += g[i] * x[i];
        g[i] *= wt[i];
        dot += g[i] * x[i];
      }
      const float mean = group_sum<D / 16>(dot) * (1.f / D);
#pragma unroll
      for (int i = 0; i < 16; ++i) g[i] = rho * (g[i] - x[i] * mean);
    }
    store16v(const_cast<T*>(head_row<T>(out, row, h)), pl.at, g);
  }
}

// A workgroup takes rows blockIdx.x, + gridDim.x, ... in units of kThreads / L.
// Its sums of the weights' gradients (fp32, over its rows and heads) go to
// part[workgroup][q, k][D]: lanes of equal l over the wavefront, then the four
// wavefronts through LDS.
template <typename T, int D, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rotary_bwd_kernel(const RotaryParams p) {
  constexpr int L = D / 16, R = kThreads / L;
  const Place<D, PAIRS> pl(threadIdx.x % L, p.pairs);
  const int h0 = blockIdx.y * p.heads_per_group, h1 = min(h0 + p.heads_per_group, p.Hq + p.Hkv);
  float acc[2][16] = {};
  for (int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L; row < p.n; row += (int64_t)gridDim.x * R) {
    const Angles t = angles(p, p.pos, p.pos_stride, row, pl.first_pair, pl.turned);
    turn_heads_bwd<T, D, PAIRS>(p.q, p.xq, p.qo, p.wq, row, h0, min(h1, p.Hq), pl, t, p.eps, acc[0]);
    turn_heads_bwd<T, D, PAIRS>(p.k, p.xk, p.ko, p.wk, row, max(h0 - p.Hq, 0), h1 - p.Hq, pl, t, p.eps, acc[1]);
  }
  if (!p.part) return;
  __shared__ float sums[kThreads / 64][2][D];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = acc[w][i];
#pragma unroll
      for (int m = L; m < 64; m *= 2) v += __shfl_xor(v, m);
      if (threadIdx.x % 64 < L) sums[threadIdx.x / 64][w][pl.at[i / 8] + i % 8] = v;
    }
  __syncthreads();
  float* part = p.part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (2 * D);
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kThreads / 64; ++k) v += sums[k][i / D][i % D];
    part[i] = v;
  }
}

// Sums of the workgroups' parts in a fixed order: 16 columns of [q, k][D] a
// workgroup, 64 of its rows side by side.
__global__ __launch_bounds__(1024) void rotary_bwd_sum_kernel(const float* __restrict__ part, int n_part, int D,
                                                              float* dwq, float* dwk) {
  __shared__ float sums[64][17];
  const int col = threadIdx.x % 16, r0 = threadIdx.x / 16;
  const int at = blockIdx.x * 16 + col;
  float v = 0.f;
  for (int r = r0; r < n_part; r += 64) v += part[(int64_t)r * (2 * D) + at];
  sums[r0][col] = v;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  v = 0.f;
  for (int r = 0; r < 64; ++r) v += sums[r][col];
  float* dw = at < D ? dwq : dwk;
  if (dw) dw[at < D ? at : at - D] = v;
}

__device__ __forceinline__ bool slot_of(const RotaryParams& p, int64_t row, int32_t& blk, int32_t& slot) {
  blk = p.slots[2 * row];
  slot = p.slots[2 * row + 1];
  return blk >= 0 && blk < p.n_blocks && slot >= 0 && slot < kBlock;
}

// Append: items of four roles, one after the other: q's rows into q_out, k's
// rows into their slots of the K cache (kThreads / L rows and a run of heads
// each), v's rows into the V cache (one (row, head) of D elements per 64
// lanes), block-table patches.
template <typename T, int D, bool PAIRS>
__device__ __forceinline__ void append_item(const RotaryParams& p, int64_t b) {
  constexpr int L = D / 16, R = kThreads / L;
  const int lane = threadIdx.x % L;
  const int hp = p.heads_per_group;
  if (b < p.items_q) {
    const int runs = (p.Hq + hp - 1) / hp;
    const int64_t row = b / runs * R + threadIdx.x / L;
    if (row >= p.n_q) return;
    const Place<D, PAIRS> pl(lane, p.pairs);
    const Angles t = angles(p, p.q_pos, p.q_pos_stride, row, pl.first_pair, pl.turned);
    const int h0 = (int)(b % runs) * hp;
    turn_heads<T, D, PAIRS>(p.q, p.wq, row, h0, min(h0 + hp, p.Hq), pl, t, p.eps, [&](int h, const float (&x)[16]) {
      store16v(const_cast<T*>(head_row<T>(p.qo, row, h)), pl.at, x);
    });
    return;
  }
  b -= p.items_q;
  int32_t blk, slot;
  if (b < p.items_k) {
    const int runs = (p.Hkv + hp - 1) / hp;
    const int64_t row = b / runs * R + threadIdx.x / L;
    if (row >= p.n || !slot_of(p, row, blk, slot)) return;
    const Place<D, PAIRS> pl(lane, p.pairs);
    const Angles t = angles(p, p.pos, p.pos_stride, row, pl.first_pair, pl.turned);
    const int h0 = (int)(b % runs) * hp;
    T* cache = static_cast<T*>(p.k_cache);
    turn_heads<T, D, PAIRS>(p.k, p.wk, row, h0, min(h0 + hp, p.Hkv), pl, t, p.eps, [&](int h, const float (&x)[16]) {
      store8(cache + paged_k_offset<D>(blk, h, p.Hkv, slot, pl.at[0] / 8), x);
      store8(cache + paged_k_offset<D>(blk, h, p.Hkv, slot, pl.at[1] / 8), x + 8);
    });
    return;
  }
  b -= p.items_k;
  if (b < p.items_v) {
    const int64_t item = b * (kThreads / 64) + threadIdx.x / 64;
    const int64_t row = item / p.Hkv;
    if (row >= p.n || !slot_of(p, row, blk, slot)) return;
    const int h = (int)(item - row * p.Hkv);
    const T* src = head_row<T>(p.v, row, h);
    T* dst = static_cast<T*>(p.v_cache) + ((int64_t)blk * p.Hkv + h) * (D * kBlock) + slot;
    for (int c = threadIdx.x % 64; c < D; c += 64) dst[c * kBlock] = src[c];
    return;
  }
  const int64_t i = (b - p.items_v) * kThreads + threadIdx.x;
  if (i < p.n_patch) p.block_table[p.patch[2 * i]] = p.patch[2 * i + 1];
}

template <typename T, int D, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rotary_append_kernel(const RotaryParams p) {
  for (int64_t b = blockIdx.x; b < p.items; b += gridDim.x) append_item<T, D, PAIRS>(p, b);
}

constexpr int64_t kMaxGrid = 1 << 20;  // workgroups of a launch: the rest by strides

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Heads of a row that a group takes: as many as leave the chip about `groups`
// groups, so that a short call spreads its heads over more of them and a long
// one computes its cosines once per row.
int heads_per_group(int64_t n, int H, int64_t groups) {
  return (int)std::min<int64_t>(H, std::max<int64_t>(1, n * H / groups));
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

template <typename T, int D, bool PAIRS>
struct Fwd {
  static void go(const RotaryParams& p, dim3 grid, hipStream_t s) {
    hipLaunchKernelGGL((rotary_fwd_kernel<T, D, PAIRS>), grid, dim3(kThreads), 0, s, p);
  }
};
template <typename T, int D, bool PAIRS>
struct Bwd {
  static void go(const RotaryParams& p, dim3 grid, hipStream_t s) {
    hipLaunchKernelGGL((rotary_bwd_kernel<T, D, PAIRS>), grid, dim3(kThreads), 0, s, p);
  }
};
template <typename T, int D, bool PAIRS>
struct Append {
  static void go(const RotaryParams& p, dim3 grid, hipStream_t s) {
    hipLaunchKernelGGL((rotary_append_kernel<T, D, PAIRS>), grid, dim3(kThreads), 0, s, p);
  }
};

}  // namespace

BwdGrid rotary_bwd_grid(int64_t n, int Hq, int Hkv, int D) {
  BwdGrid g{};
  const int H = Hq + Hkv;
  if (n == 0 || H == 0) return g;
  g.heads_per_group = heads_per_group(n, H, 16384);
  g.y = (int32_t)ceil_div(H, g.heads_per_group);
  g.x = (int32_t)std::min<int64_t>(ceil_div(n, kThreads / (D / 16)), std::max<int64_t>(1, 1024 / g.y));
  return g;
}

hipError_t launch_rotary_fwd(RotaryParams p, int D, bool bf16, bool pairs, hipStream_t s) {
  const int H = p.Hq + p.Hkv;
  if (p.n == 0 || H == 0) return hipSuccess;
  p.heads_per_group = heads_per_group(p.n, H, 16384);
  const unsigned y = (unsigned)ceil_div(H, p.heads_per_group);
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(p.n, kThreads / (D / 16)), std::max<int64_t>(1, kMaxGrid / y)), y);
  return dispatch<Fwd>(p, D, bf16, pairs, grid, s);
}

hipError_t launch_rotary_bwd(RotaryParams p, int D, bool bf16, bool pairs, float* dwq, float* dwk, hipStream_t s) {
  const BwdGrid g = rotary_bwd_grid(p.n, p.Hq, p.Hkv, D);
  if (g.x > 0) {
    p.heads_per_group = g.heads_per_group;
    const hipError_t e = dispatch<Bwd>(p, D, bf16, pairs, dim3((unsigned)g.x, (unsigned)g.y), s);
    if (e != hipSuccess) return e;
  }
  if (dwq || dwk)
    hipLaunchKernelGGL(rotary_bwd_sum_kernel, dim3(2 * D / 16), dim3(1024), 0, s, p.part, g.x * g.y, D, dwq, dwk);
  return hipGetLastError();
}

hipError_t launch_rotary_append(RotaryParams p, int D, bool bf16, bool pairs, hipStream_t s) {
  const int R = kThreads / (D / 16);
  p.heads_per_group = heads_per_group(std::max(p.n, p.n_q), p.Hq + p.Hkv, 16384);
  const int hp = std::max(1, p.heads_per_group);
  p.heads_per_group = hp;
  p.items_q = p.Hq ? ceil_div(p.n_q, R) * ceil_div(p.Hq, hp) : 0;
  p.items_k = p.Hkv ? ceil_div(p.n, R) * ceil_div(p.Hkv, hp) : 0;
  p.items_v = ceil_div((int64_t)p.n * p.Hkv, kThreads / 64);
  p.items = p.items_q + p.items_k + p.items_v + ceil_div(p.n_patch, kThreads);
  if (p.items == 0) return hipSuccess;
  return dispatch<Append>(p, D, bf16, pairs, dim3((unsigned)std::min(p.items, kMaxGrid)), s);
}

}  // namespace padoc
