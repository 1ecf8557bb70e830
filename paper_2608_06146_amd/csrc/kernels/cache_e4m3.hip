// Blocks of bf16 / fp32 caches to blocks of 8-bit caches and back.
//
//   a = max |x_i| of a row, e = smallest exponent with a <= 448 * 2^e,
//   codes = e4m3(x * 2^-e); back: codes * 2^e
//
// A copy with a maximum in between, bound by memory: every element is read
// once (16 bytes a lane) and written once.  A (block, head) pair has 16 rows of K
// and of V.  To codes: a wavefront a pair, the maxima by swaps of lanes (with a
// workgroup a pair and maxima by LDS atomics, 16,384 blocks of two heads of 128
// in bf16 took 134 us; 69 so: 5.85 TB/s).  Back: a workgroup a pair, small pairs
// side by side (8,192 blocks of four heads of 64 to fp32: 48 us, 7.05 TB/s).
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <algorithm>

#include "../rotary.hpp"
#include "e4m3.hpp"

namespace padoc {
namespace {

using e4m3::u32x4;

constexpr int kThreads = 256;

template <typename T, int D>
struct Geom {
  static constexpr int E = 16 / (int)sizeof(T);     // elements of a 16-byte unit
  static constexpr int kUnits = kBlock * D / E;     // units of a (block, head) and tensor: 128 .. 512
  static constexpr int kLanes = kUnits < kThreads ? kUnits : kThreads;  // threads that share a pair
  static constexpr int kShare = kThreads / kLanes;  // pairs side by side
  static constexpr int kPer = kUnits / kLanes;      // units per thread and tensor
};

template <typename T, int E>
__device__ __forceinline__ void unpack(const u32x4& u, float (&x)[E]) {
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const uint32_t w = u[i * (int)sizeof(T) / 4];
    x[i] = __uint_as_float(sizeof(T) == 4 ? w : i % 2 ? w & 0xffff0000u : w << 16);
  }
}
template <typename T, int E>
__device__ __forceinline__ u32x4 pack(const float (&x)[E]) {  // (values that are exact in T, or NaN)
  u32x4 u;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    u[i] = sizeof(T) == 4 ? __float_as_uint(x[i]) : (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1 < E ? 2 * i + 1 : 0]) & 0xffff0000u);
  return u;
}

// Source and destination block of item `pair`, and its head; false: left out.
__device__ __forceinline__ bool blocks_of(const CastParams& p, int64_t item, int64_t& from, int64_t& to, int& head) {
  const int64_t i = item / p.Hkv;
  head = (int)(item - i * p.Hkv);
  from = p.pairs ? p.pairs[2 * i] : i;
  to = p.pairs ? p.pairs[2 * i + 1] : i;
  return from >= 0 && from < p.src_blocks && to >= 0 && to < p.dst_blocks;
}

// Token (K) and first dim of K unit u of the source layout.
template <typename T, int D>
__device__ __forceinline__ void k_unit(int u, int& token, int& dim) {
  constexpr int P = 8 / Geom<T, D>::E;  // units of an 8-dim piece
  token = kslot(u / P % kBlock);
  dim = u / P / kBlock * 8 + u % P * Geom<T, D>::E;
}

// Maxima over lanes.  A lane row is 16 lanes; swap16 / swap32 exchange odd rows
// of a with even rows of b / the high half of a with the low half of b.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
constexpr int kXor1 = 0xB1, kRor2 = 0x122, kRor4 = 0x124, kRor8 = 0x128;

// Largest magnitudes of the elements of a V unit's tokens: two to a word (bf16)
// or one (fp32).
template <typename T>
struct Top {
  static constexpr uint32_t kMask = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    if constexpr (sizeof(T) == 4)
      return max(a, b);
    else
      return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
  }
};

// A wavefront takes a (block, head) pair: its lanes hold the whole pair in
// registers, a lane always units of one token of K, and of the same tokens of V.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void quantize_kernel(const CastParams p, int64_t items) {
  using G = Geom<T, D>;
  using M = Top<T>;
  constexpr int kPer = G::kUnits / 64;  // units a lane and tensor
  constexpr int H = kBlock / G::E;      // units of a V row
  const int lane = threadIdx.x & 63;
  const int64_t step = (int64_t)gridDim.x * (kThreads / 64);
  for (int64_t item = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); item < items; item += step) {
    int64_t from = 0, to = 0;
    int head = 0;
    if (!blocks_of(p, item, from, to, head)) continue;
    const u32x4* ks = static_cast<const u32x4*>(p.k) + (from * p.Hkv + head) * G::kUnits + lane;
    const u32x4* vs = static_cast<const u32x4*>(p.v) + (from * p.Hkv + head) * G::kUnits + lane;
    u32x4 kx[kPer], vx[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) kx[i] = __builtin_nontemporal_load(ks + i * 64);
#pragma unroll
    for (int i = 0; i < kPer; ++i) vx[i] = __builtin_nontemporal_load(vs + i * 64);
    uint8_t* kd = p.k_codes + e4m3::codes_at<D>(to, head, p.Hkv);
    uint8_t* vd = p.v_codes + e4m3::codes_at<D>(to, head, p.Hkv);
    uint8_t* sd = p.scales + e4m3::scales_at(to, head, p.Hkv);

    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      float x[G::E];
      unpack<T>(kx[i], x);
#pragma unroll
      for (int e = 0; e < G::E; ++e) a = max(a, __float_as_uint(x[e]) & 0x7fffffffu);
    }
    {  // the lanes of a token: l, l + 32, and l + 16 (bf16) or l ^ 1 (fp32)
      const auto h = __builtin_amdgcn_permlane32_swap(a, a, false, false);
      a = max(h[0], h[1]);
      if constexpr (sizeof(T) == 4) {
        a = max(a, dpp<kXor1>(a));
      } else {
        const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
        a = max(r[0], r[1]);
      }
    }
    const uint32_t kb = e4m3::scale_byte(a);
    const float kr = e4m3::inverse_scale(kb);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      float x[G::E];
      unpack<T>(kx[i], x);
      int token, dim;
      k_unit<T, D>(lane + i * 64, token, dim);
      uint32_t c[G::E / 4];
#pragma unroll
      for (int e = 0; e < G::E; e += 4)
        c[e / 4] = kb == e4m3::kNan ? e4m3::kNanCodes : e4m3::codes4(x[e], x[e + 1], x[e + 2], x[e + 3], kr);
      __builtin_memcpy(__builtin_assume_aligned(kd + e4m3::k_at(token, dim), G::E), c, G::E);
      if (i == 0 && dim == 0) sd[token] = (uint8_t)kb;
    }

    // V: the lane's words over its units, then lane row r gets word r of all of
    // them, its lanes of the same tokens (every H-th) that of the row.
    uint32_t m[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = M::larger(m[j], vx[i][j] & M::kMask);
    const auto h0 = __builtin_amdgcn_permlane32_swap(m[0], m[2], false, false);
    const auto h1 = __builtin_amdgcn_permlane32_swap(m[1], m[3], false, false);
    const auto hr = __builtin_amdgcn_permlane16_swap(M::larger(h0[0], h0[1]), M::larger(h1[0], h1[1]), false, false);
    uint32_t t = M::larger(hr[0], hr[1]);
    t = M::larger(t, dpp<kRor8>(t));
    t = M::larger(t, dpp<kRor4>(t));
    if constexpr (H == 2) t = M::larger(t, dpp<kRor2>(t));
    // Scale bytes of word r, and 2^-e (its upper half, which holds all of it).
    const uint32_t b0 = e4m3::scale_byte(sizeof(T) == 4 ? t : t << 16), b1 = e4m3::scale_byte(sizeof(T) == 4 ? t : t & 0xffff0000u);
    const bool nan = b0 == e4m3::kNan || b1 == e4m3::kNan;
    const int w0 = lane % H * G::E + (lane >> 4) * (G::E / 4);  // first token of the lane's word r
    if (lane % 16 < H) {
      sd[kBlock + w0] = (uint8_t)b0;
      if constexpr (sizeof(T) == 2) sd[kBlock + w0 + 1] = (uint8_t)b1;
    }
    const uint32_t r0 = __float_as_uint(e4m3::inverse_scale(b0)), r1 = __float_as_uint(e4m3::inverse_scale(b1));
    const uint32_t inv = sizeof(T) == 4 ? r0 : (r0 >> 16) | r1;
    auto spread = [](uint32_t v, uint32_t (&out)[4]) {  // word r of lane row r to every row
      const auto q = __builtin_amdgcn_permlane16_swap(v, v, false, false);
      const auto e = __builtin_amdgcn_permlane32_swap(q[0], q[0], false, false);
      const auto o = __builtin_amdgcn_permlane32_swap(q[1], q[1], false, false);
      out[0] = e[0], out[1] = o[0], out[2] = e[1], out[3] = o[1];
    };
    u32x4 iv;
    {
      uint32_t o[4];
      spread(inv, o);
      iv = u32x4{o[0], o[1], o[2], o[3]};
    }
    if (__any(nan)) {  // elements of rows that are NaN: zeros
      uint32_t o[4];
      spread((b0 == e4m3::kNan ? (sizeof(T) == 4 ? 0xffffffffu : 0xffffu) : 0u) |
                 (sizeof(T) == 2 && b1 == e4m3::kNan ? 0xffff0000u : 0u), o);
#pragma unroll
      for (int i = 0; i < kPer; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) vx[i][j] &= ~o[j];
    }
    float r[G::E];
    unpack<T>(iv, r);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      float x[G::E];
      unpack<T>(vx[i], x);
      uint32_t c[G::E / 4];
#pragma unroll
      for (int e = 0; e < G::E; e += 4)
        c[e / 4] = e4m3::codes4(x[e] * r[e], x[e + 1] * r[e + 1], x[e + 2] * r[e + 2], x[e + 3] * r[e + 3], 1.f);
      __builtin_memcpy(__builtin_assume_aligned(vd + (lane + i * 64) * G::E, G::E), c, G::E);
    }
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(const CastParams p, int64_t items) {
  using G = Geom<T, D>;
  const int who = threadIdx.x / G::kLanes, u0 = threadIdx.x % G::kLanes;
  for (int64_t base = (int64_t)blockIdx.x * G::kShare; base < items; base += (int64_t)gridDim.x * G::kShare) {
    int64_t from = 0, to = 0;
    int head = 0;
    if (base + who >= items || !blocks_of(p, base + who, from, to, head)) continue;
    const uint8_t* kc = p.k_codes + e4m3::codes_at<D>(from, head, p.Hkv);
    const uint8_t* vc = p.v_codes + e4m3::codes_at<D>(from, head, p.Hkv);
    const uint8_t* sc = p.scales + e4m3::scales_at(from, head, p.Hkv);
    u32x4* kd = static_cast<u32x4*>(p.k_out) + (to * p.Hkv + head) * G::kUnits;
    u32x4* vd = static_cast<u32x4*>(p.v_out) + (to * p.Hkv + head) * G::kUnits;
#pragma unroll
    for (int i = 0; i < G::kPer; ++i) {
      const int u = u0 + i * G::kLanes;
      int token, dim;
      k_unit<T, D>(u, token, dim);
      float x[G::E], y[4];
      const uint32_t b = sc[token];
#pragma unroll
      for (int e = 0; e < G::E; e += 4) {
        e4m3::values4(*reinterpret_cast<const uint32_t*>(kc + e4m3::k_at(token, dim + e)), y);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[e + j] = b == e4m3::kNan ? __uint_as_float(0x7fc00000u) : y[j] * e4m3::scale_value(b);
      }
      __builtin_nontemporal_store(pack<T>(x), kd + u);
      constexpr int H = kBlock / G::E;
      const int t0 = u % H * G::E;
#pragma unroll
      for (int e = 0; e < G::E; e += 4) {
        e4m3::values4(*reinterpret_cast<const uint32_t*>(vc + u / H * kBlock + t0 + e), y);
        const uint32_t w = *reinterpret_cast<const uint32_t*>(sc + kBlock + t0 + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t c = (w >> (8 * j)) & 255u;
          x[e + j] = c == e4m3::kNan ? __uint_as_float(0x7fc00000u) : y[j] * e4m3::scale_value(c);
        }
      }
      __builtin_nontemporal_store(pack<T>(x), vd + u);
    }
  }
}

template <typename T, int D>
void launch(const CastParams& p, bool back, hipStream_t s) {
  const int64_t items = p.n_pairs * p.Hkv;
  const int64_t share = back ? Geom<T, D>::kShare : kThreads / 64;  // pairs of a workgroup
  const dim3 grid((unsigned)std::min<int64_t>((items + share - 1) / share, 1 << 20));
  if (back)
    hipLaunchKernelGGL((dequantize_kernel<T, D>), grid, dim3(kThreads), 0, s, p, items);
  else
    hipLaunchKernelGGL((quantize_kernel<T, D>), grid, dim3(kThreads), 0, s, p, items);
}

}  // namespace

// back: codes to values.
hipError_t launch_cast_blocks(const CastParams& p, int D, bool bf16, bool back, hipStream_t s) {
  if (p.n_pairs == 0) return hipSuccess;
  if (bf16)
    D == 64 ? launch<__bf16, 64>(p, back, s) : launch<__bf16, 128>(p, back, s);
  else
    D == 64 ? launch<float, 64>(p, back, s) : launch<float, 128>(p, back, s);
  return hipGetLastError();
}

}  // namespace padoc
