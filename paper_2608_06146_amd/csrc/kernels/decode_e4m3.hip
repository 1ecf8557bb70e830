// One decode step over an 8-bit paged cache with bf16 queries: the schedule of
// the bf16 step (decode_step.hip) on e4m3 codes.
//
//   S = scale * q.(c_k 2^e_k),  P = softmax(S),  O = sum_j (P_j 2^e_j) c_v
//
// Codes become bf16 values on their way into the matrix products (a code has
// four significant bits, so that nothing is rounded).  K's scale goes into the
// conversion; V's, one for each key, into the probabilities before they are
// rounded to bf16.
#include "device_common.hpp"
#include "e4m3.hpp"
#include "fwd_item.hpp"

namespace padoc {
namespace {

using e4m3::bf16x8_t;
using e4m3::u32x4;
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;  // keys of a step: four blocks

__device__ __forceinline__ u32x4 load16_nt(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}

// Private work item `item` (at most 16 columns) on one wavefront, whose lane
// index is `lane`: keys in steps of 64, from HBM straight into
// v_mfma_f32_16x16x32_bf16 operands (lane l: row / column n = l%16, group
// g = l/16 with eight consecutive elements of the contraction).
//   S^T = K Q^T    four 16-key M blocks; row m of block T holds token
//                  4T + m%4 of cache block m/4, so that a lane's 16 scores are
//                  the 16 tokens of cache block g, in order; a lane's 16 codes
//                  (a 16-dim piece of a token) are two operands
//   O^T += V^T P^T the lane's 16 codes of a V row are the tokens of cache block
//                  g, two operands of eight
// Two register sets hold the codes of two steps, refilled after their last use.
constexpr int kSets = 2;

template <int D>
__device__ __forceinline__ void wave_item(const TileParams& p, int item, int lane) {
  constexpr int NP = D / 64;   // 16-dim pieces per lane and token
  constexpr int NDM = D / 16;  // 16-row blocks of O^T
  const WorkRec w = load_scalar(p.work + item);
  const int n = lane & 15, g = lane >> 4;
  const int G = p.G, kvh = w.kvh, Hkv = p.Hkv;
  const int col = w.col0 + n;
  const int t = col / G;
  const bool valid = n < w.ncol && t < w.ntok;
  const int32_t qrow = valid ? p.toks[w.tok_begin + t] : 0;
  const int32_t hq = kvh * G + (col - t * G);
  const uint8_t* Kc = static_cast<const uint8_t*>(p.k);
  const uint8_t* Vc = static_cast<const uint8_t*>(p.v);

  // Q fragments: dims 16 (g + 4 j) + 8 h .. +7.
  bf16x8_t bq[NP][2];
  const uint16_t* qp = static_cast<const uint16_t*>(p.q) + ((int64_t)qrow * p.Hq + hq) * D + 16 * g;
#pragma unroll
  for (int j = 0; j < NP; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint4 z = valid ? *reinterpret_cast<const uint4*>(qp + 64 * j + 8 * h) : make_uint4(0, 0, 0, 0);
      bq[j][h] = *reinterpret_cast<const bf16x8_t*>(&z);
    }

  struct Cursor {
    int ri, st;
    RangeRec R;
    int ok, unused;
  };
  auto advance = [&](Cursor& c) __attribute__((always_inline)) {
    if (++c.st * kStep >= c.R.n_keys) {
      c.st = 0;
      if (++c.ri < w.rng_count)
        c.R = load_scalar(p.ranges + w.rng_begin + c.ri);
      else
        c.ok = 0;
    }
  };
  Cursor C{0, 0, load_scalar(p.ranges + w.rng_begin), 1, 0};
  Cursor L = C;

  u32x4 kf[kSets][4][NP];  // [set][M block][piece]
  u32x4 vf[kSets][NDM];    // [set][16-row d block]
  u32x4 ks[kSets], vs[kSets];  // scales of the K tokens (cache block n/4) and of the V tokens (block g)
  int32_t id0, id1, id2, id3;  // ids of the load cursor's blocks, requested ahead

  // Blocks past the range's end take the step's first; past the item's last
  // step block 0 is read over and over (every step issues the same loads, so
  // that the compiler's waits for a set stay exact) and never used.
  auto fetch_ids = [&](const Cursor& c) __attribute__((always_inline)) {
    const int kb = c.st * kStep;
    const int32_t* b = p.block_table + c.R.kv_start + (kb >> 4);
    id0 = load_scalar(b);
    id1 = load_scalar(b + (kb + 16 < c.R.n_keys ? 1 : 0));
    id2 = load_scalar(b + (kb + 32 < c.R.n_keys ? 2 : 0));
    id3 = load_scalar(b + (kb + 48 < c.R.n_keys ? 3 : 0));
  };
  auto pick = [&](int i, bool real) __attribute__((always_inline)) -> int64_t {
    const int lo = (i & 1) ? id1 : id0, hi = (i & 1) ? id3 : id2;
    return real ? ((i & 2) ? hi : lo) : 0;
  };
  int64_t vblk[kSets];
  auto load_k = [&](int X, bool real) __attribute__((always_inline)) {
    const int64_t blk = pick(n >> 2, real);
    vblk[X] = pick(g, real);
    const uint8_t* kp = Kc + e4m3::codes_at<D>(blk, kvh, Hkv) + g * (kBlock * 16) + (n & 3) * 16;
#pragma unroll
    for (int T = 0; T < 4; ++T)
#pragma unroll
      for (int j = 0; j < NP; ++j) kf[X][T][j] = load16_nt(kp + 4 * T * 16 + 4 * j * (kBlock * 16));
    ks[X] = *reinterpret_cast<const u32x4*>(p.scales + e4m3::scales_at(blk, kvh, Hkv));
  };
  auto load_v = [&](int X) __attribute__((always_inline)) {
    const uint8_t* vp = Vc + e4m3::codes_at<D>(vblk[X], kvh, Hkv) + n * kBlock;
#pragma unroll
    for (int dm = 0; dm < NDM; ++dm) vf[X][dm] = load16_nt(vp + dm * 16 * kBlock);
    vs[X] = *reinterpret_cast<const u32x4*>(p.scales + e4m3::scales_at(vblk[X], kvh, Hkv) + kBlock);
  };

  float m_run = -INFINITY, l_part = 0.f;
  f32x4_t acc[NDM];
#pragma unroll
  for (int dm = 0; dm < NDM; ++dm) acc[dm] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  int lim = 0;
  auto load_lim = [&]() __attribute__((always_inline)) {
    lim = C.R.lim_off < 0 ? C.R.n_keys : valid ? p.lims[C.R.lim_off + t] : 0;
  };
  load_lim();
  const float sl2 = p.scale_log2;

  fetch_ids(L);
  load_k(0, true);
  load_v(0);
  advance(L);
#pragma unroll
  for (int X = 1; X < kSets; ++X) {
    const bool real = L.ok;
    fetch_ids(L);
    load_k(X, real);
    load_v(X);
    advance(L);
  }
  fetch_ids(L);

  auto step = [&](auto xc) __attribute__((always_inline)) -> bool {
    constexpr int X = decltype(xc)::value;
    const int kb = C.st * kStep;
    f32x4_t S[4];
#pragma unroll
    for (int T = 0; T < 4; ++T) {
      S[T] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const float sk = e4m3::scale_value((ks[X][T] >> (8 * (n & 3))) & 255u);
#pragma unroll
      for (int j = 0; j < NP; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          S[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e4m3::values8(kf[X][T][j][2 * h], kf[X][T][j][2 * h + 1], sk),
                                                         bq[j][h], S[T], 0, 0, 0);
    }
    const bool more = L.ok;
    load_k(X, more);  // set X's K is consumed
    // A V row that is NaN: the scores of its token are (where a column sees it);
    // no scale is infinite, so that probabilities of 0 stay 0.
    if (__any(e4m3::has_nan(vs[X][0]) || e4m3::has_nan(vs[X][1]) || e4m3::has_nan(vs[X][2]) || e4m3::has_nan(vs[X][3]))) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e4m3::byte_of(vs[X], e) == e4m3::kNan) {
          S[e / 4][e % 4] = __uint_as_float(0x7fc00000u);
          vs[X][e / 4] &= ~(255u << (8 * (e % 4)));
        }
    }
    if (kb + kStep > C.R.min_lim) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (kb + 16 * g + e >= lim) S[e / 4][e % 4] = -INFINITY;
    }
    float mx = S[0][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, S[e / 4][e % 4]);
    mx = max_lane_halves(max_lane_rows(mx));
    const float m_new = fmaxf(m_run, mx * sl2);
    const float m_sub = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = fast_exp2(m_run - m_sub);
    m_run = m_new;
    float ls = 0.f;
    bf16x8_t pb[2];
    const int keep = C.R.n_keys - (kb + 16 * g);  // tokens of the lane's V block that exist
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = fast_exp2(fmaf(S[e / 4][e % 4], sl2, -m_sub));
      ls += x;
      pb[e / 8][e % 8] = (__bf16)(x * e4m3::scale_value(e4m3::byte_of(vs[X], e)));
    }
    l_part = fmaf(l_part, alpha, ls);
#pragma unroll
    for (int dm = 0; dm < NDM; ++dm) {
      acc[dm] *= alpha;
      u32x4 v = vf[X][dm];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = keep - 4 * i;
        v[i] = k >= 4 ? v[i] : k <= 0 ? 0u : v[i] & (0xffffffffu >> (8 * (4 - k)));
      }
      acc[dm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e4m3::values8(v[0], v[1], 1.f), pb[0], acc[dm], 0, 0, 0);
      acc[dm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e4m3::values8(v[2], v[3], 1.f), pb[1], acc[dm], 0, 0, 0);
    }
    load_v(X);
    advance(L);
    fetch_ids(L);
    const int ri_before = C.ri;
    advance(C);
    if (!C.ok) return false;
    if (C.ri != ri_before) load_lim();
    return true;
  };
  for (bool go = true; go;)
    tile::static_for<kSets>([&](auto xc) __attribute__((always_inline)) {
      if (go) go = step(xc);
    });

  float lt = l_part + __shfl_xor(l_part, 16);
  lt += __shfl_xor(lt, 32);
  if (!valid) return;
  const int64_t slot = (int64_t)w.out_base + col;
  float* op = p.part_o + slot * D + 4 * g;
#pragma unroll
  for (int dm = 0; dm < NDM; ++dm)
    *reinterpret_cast<float4*>(op + dm * 16) = make_float4(acc[dm][0], acc[dm][1], acc[dm][2], acc[dm][3]);
  if (g == 0) {
    p.part_ml[2 * slot] = m_run;
    p.part_ml[2 * slot + 1] = lt;
  }
}

// As decode_step_kernel: shared tile items on the first workgroups, then every
// wavefront takes private items from its XCD's queue.
constexpr int kQueues = kPrivateQueues;

__device__ __forceinline__ int take_private(int* ctr, int lane) {
  int v = 0;
  if (lane == 0) v = atomicAdd(ctr, 1);
  return __builtin_amdgcn_readfirstlane(v);
}

template <int D>
__global__ __launch_bounds__(tile::kThreads) void decode_e4m3_kernel(TileParams p, int n_shared, int n_private,
                                                                     int n_groups, int* next) {
  const int b = blockIdx.x;
  if (b < n_shared) tile::fwd_item<D, true, true>(p, b);
  if (n_private <= 0) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int q = b % kQueues;
  const int n_q = (n_private - q + kQueues - 1) / kQueues;
  const int end = n_shared + n_groups;
  const int b0 = n_shared + (q - n_shared % kQueues + kQueues) % kQueues;
  const int n_first = b0 < end ? ((end - 1 - b0) / kQueues + 1) * tile::kWaves : 0;
  int* ctr = next + q * 64;
  int k = b >= n_shared ? ((b - b0) / kQueues) * tile::kWaves + wave : n_first + take_private(ctr, lane);
  while (k < n_q) {
    wave_item<D>(p, n_shared + q + kQueues * k, lane);
    k = n_first + take_private(ctr, lane);
  }
}

}  // namespace

// n_groups, next: as launch_decode_step_bf16.
hipError_t launch_decode_e4m3(const TileParams& p, int n_shared, int n_private, int n_groups, int* next, int D,
                              hipStream_t stream) {
  const int n_blocks = n_shared + n_groups;
  if (n_blocks <= 0) return hipSuccess;
  const dim3 grid(n_blocks), block(tile::kThreads);
  if (D == 64)
    hipLaunchKernelGGL((decode_e4m3_kernel<64>), grid, block, 0, stream, p, n_shared, n_private, n_groups, next);
  else
    hipLaunchKernelGGL((decode_e4m3_kernel<128>), grid, block, 0, stream, p, n_shared, n_private, n_groups, next);
  return hipGetLastError();
}

}  // namespace padoc
