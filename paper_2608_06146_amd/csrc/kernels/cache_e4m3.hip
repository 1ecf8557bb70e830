// Blocks of bf16 / fp32 caches to blocks of 8-bit caches and back.
//
//   a = max |x_i| of a row, e = smallest exponent with a <= 448 * 2^e,
//   codes = e4m3(x * 2^-e); back: codes * 2^e
//
// A copy with a maximum in between, bound by memory: every element is read
// once (16 bytes a lane) and written once.  A workgroup takes the 16 rows of K
// and of V of one (block, head) pair at a time; small pairs side by side.
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

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void quantize_kernel(const CastParams p, int64_t items) {
  using G = Geom<T, D>;
  __shared__ uint32_t top[G::kShare][2][kBlock];  // largest magnitudes of the rows, as fp32 bits
  const int who = threadIdx.x / G::kLanes, u0 = threadIdx.x % G::kLanes;
  for (int64_t base = (int64_t)blockIdx.x * G::kShare; base < items; base += (int64_t)gridDim.x * G::kShare) {
    int64_t from = 0, to = 0;
    int head = 0;
    const bool on = base + who < items && blocks_of(p, base + who, from, to, head);
    if (u0 < 2 * kBlock) top[who][u0 / kBlock][u0 % kBlock] = 0;
    __syncthreads();
    u32x4 kx[G::kPer], vx[G::kPer];
    if (on) {
      const u32x4* ks = static_cast<const u32x4*>(p.k) + (from * p.Hkv + head) * G::kUnits;
      const u32x4* vs = static_cast<const u32x4*>(p.v) + (from * p.Hkv + head) * G::kUnits;
#pragma unroll
      for (int i = 0; i < G::kPer; ++i) {
        kx[i] = __builtin_nontemporal_load(ks + u0 + i * G::kLanes);
        vx[i] = __builtin_nontemporal_load(vs + u0 + i * G::kLanes);
      }
#pragma unroll
      for (int i = 0; i < G::kPer; ++i) {
        float x[G::E];
        unpack<T>(kx[i], x);
        uint32_t a = 0;
#pragma unroll
        for (int e = 0; e < G::E; ++e) a = max(a, __float_as_uint(x[e]) & 0x7fffffffu);
        int token, dim;
        k_unit<T, D>(u0 + i * G::kLanes, token, dim);
        atomicMax(&top[who][0][token], a);
        unpack<T>(vx[i], x);
        const int t0 = (u0 + i * G::kLanes) % (kBlock / G::E) * G::E;
#pragma unroll
        for (int e = 0; e < G::E; ++e) atomicMax(&top[who][1][t0 + e], __float_as_uint(x[e]) & 0x7fffffffu);
      }
    }
    __syncthreads();
    if (on) {
      uint8_t* kd = p.k_codes + e4m3::codes_at<D>(to, head, p.Hkv);
      uint8_t* vd = p.v_codes + e4m3::codes_at<D>(to, head, p.Hkv);
      if (u0 < 2 * kBlock)
        p.scales[e4m3::scales_at(to, head, p.Hkv) + u0] = (uint8_t)e4m3::scale_byte(top[who][u0 / kBlock][u0 % kBlock]);
#pragma unroll
      for (int i = 0; i < G::kPer; ++i) {
        const int u = u0 + i * G::kLanes;
        float x[G::E];
        unpack<T>(kx[i], x);
        int token, dim;
        k_unit<T, D>(u, token, dim);
        const uint32_t b = e4m3::scale_byte(top[who][0][token]);
        const float r = e4m3::inverse_scale(b);
        uint32_t* to_k = reinterpret_cast<uint32_t*>(kd + e4m3::k_at(token, dim));
#pragma unroll
        for (int e = 0; e < G::E; e += 4)
          to_k[e / 4] = b == e4m3::kNan ? e4m3::kNanCodes : e4m3::codes4(x[e], x[e + 1], x[e + 2], x[e + 3], r);
        unpack<T>(vx[i], x);
        constexpr int H = kBlock / G::E;
        const int t0 = u % H * G::E;
#pragma unroll
        for (int e = 0; e < G::E; ++e) {
          const uint32_t c = e4m3::scale_byte(top[who][1][t0 + e]);
          x[e] = c == e4m3::kNan ? 0.f : x[e] * e4m3::inverse_scale(c);
        }
        uint32_t* to_v = reinterpret_cast<uint32_t*>(vd + u / H * kBlock + t0);
#pragma unroll
        for (int e = 0; e < G::E; e += 4) to_v[e / 4] = e4m3::codes4(x[e], x[e + 1], x[e + 2], x[e + 3], 1.f);
      }
    }
    __syncthreads();
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
  const dim3 grid((unsigned)std::min<int64_t>((items + Geom<T, D>::kShare - 1) / Geom<T, D>::kShare, 1 << 20));
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
