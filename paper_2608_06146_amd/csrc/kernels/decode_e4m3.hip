// One decode step over an 8-bit paged cache with bf16 queries: the schedule of
// the bf16 step (decode_step.hip) on e4m3 codes.
//
//   S = scale * q.(c_k 2^e_k),  P = softmax(S),  O = sum_j (P_j 2^e_j) c_v
//
// Codes become bf16 values on their way into the matrix products (a code has
// four significant bits, so that nothing is rounded).  K's scale goes into the
// conversion; V's, one for each key, into the probabilities before they are
// rounded to bf16 (private items) or into the conversion too (shared ones).  That
// rounding, 2^-8 of a probability at most, is the price of bf16 matrix products
// (fp32 ones reach a tenth of their rate); with it O is off by 1.8e-3 (rms), by its own
// last rounding alone 1.63e-3.  Row sums add the probabilities before that
// rounding, in fp32.
//
// Bound by HBM for the private keys (from half of the units 4.5 TB/s, from all 6.0)
// and by the tile items' vector and matrix work for the shared ones.  64 pages (1,600
// queries, 2,800 shared and 24 x up to 1,024 private keys a page, 511 MB): the kernel
// 122 us, with the schedule's copy and the combine 131; the kernel on private keys alone
// (16 + 16 shared ones a page) 86, on shared ones alone (a private key a branch) 113 to
// 115; on bf16 caches 190 and 199.  Where shared keys are all, the codes
// save nothing (dense step, 128 queries on 9,098 keys: 102 us, bf16 103).
#include <type_traits>

#include "device_common.hpp"
#include "e4m3.hpp"
#include "fwd_item.hpp"

namespace padoc {
namespace {

using e4m3::bf16x8_t;
using e4m3::u32x4;
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kStep = 32;  // keys of a step: two blocks
constexpr int kSets = 2;   // steps in flight

__device__ __forceinline__ u32x4 load16_nt(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}
__device__ __forceinline__ u32x2 load_pair(const uint8_t* p) {  // four bytes, and four eight bytes on
  const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
  return u32x2{w[0], w[2]};
}

// Private work item `item` (at most 16 columns) on one wavefront, whose lane
// index is `lane`: keys in steps of 32, from HBM straight into
// v_mfma_f32_16x16x32_bf16 operands (lane l: row / column n = l%16, group
// g = l/16 with eight consecutive elements of the contraction).
//   S^T = K Q^T    two 16-key M blocks; row m of block T holds token 8T + m%8 of
//                  cache block m/8 (eight tokens of a 16-dim piece are a line of
//                  128 bytes, whole in one load), so that a lane's scores are
//                  tokens 8T + 4 (g%2) .. +3 of cache block g/2; a lane's 16 codes
//                  (a piece of a token) are two operands
//   O^T += V^T P^T a lane loads the 16 tokens of a V row: of row block 2e where g
//                  is even, of 2e + 1 where it is odd.  Two lane swaps exchange
//                  words, so that it has its scores' tokens of both rows.
// Two register sets hold the codes of two steps, refilled after their last use.
// Fewer bytes in flight are better here: a read of 420 MB in random 2 KB pieces
// took 62 us (6.5 TB/s) with 8 KB sets and 68 with 16 KB sets, two a wavefront,
// eight wavefronts a unit; and one pipeline over all items of a wavefront, whose
// loads never pause, took 5 us more than a pause between items (99.5 for 94.7: calls
// on a resident schedule, private keys alone, with 9 of combine).  With half lines
// (tokens 0 .. 3 and 8 .. 11 in one load) instead of whole ones: 106 for 95.
template <int D>
__device__ __forceinline__ void wave_item(const TileParamsE4m3& p, int item, int lane) {
  constexpr int NP = D / 64;   // 16-dim pieces per lane and token
  constexpr int NDM = D / 16;  // 16-row blocks of O^T
  const WorkRec w = load_scalar(p.work + item);
  // (as private_item: such an item's first loads wait for one record, not three)
  const bool direct = w.direct[0] >= 0;
  const int n = lane & 15, g = lane >> 4;
  const int G = p.G, kvh = w.kvh, Hkv = p.Hkv;
  const int col = w.col0 + n;
  const int t = col / G;
  const bool valid = n < w.ncol && t < w.ntok;
  const int32_t qrow = !valid ? 0 : direct ? w.direct[2] : p.toks[w.tok_begin + t];
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
  RangeRec R0;
  int n_steps = 0;
  if (direct) {
    R0.kv_start = w.direct[0];
    R0.n_keys = R0.min_lim = w.direct[1];
    R0.lim_off = -1;
    R0.seg = R0.key_begin = R0.reserved = 0;
    n_steps = (R0.n_keys + kStep - 1) / kStep;
  } else {
    R0 = load_scalar(p.ranges + w.rng_begin);
    for (int r = 0; r < w.rng_count; ++r)
      n_steps += (load_scalar(p.ranges + w.rng_begin + r).n_keys + kStep - 1) / kStep;
  }
  n_steps = __builtin_amdgcn_readfirstlane(n_steps);
  Cursor C{0, 0, R0, 1, 0};
  Cursor L = C;

  u32x4 kf[kSets][2][NP];    // [set][M block][piece]
  u32x4 vf[kSets][NDM / 2];  // [set][pair of 16-row blocks]
  u32x2 ks[kSets], vs[kSets];  // scales of eight K tokens of cache block n/8, of the lane's eight V tokens
  int32_t id0, id1;          // ids of the load cursor's blocks, requested ahead

  // A block past the range's end takes the step's first; past the item's last
  // step block 0 is read over and over (every step issues the same loads, so
  // that the compiler's waits for a set stay exact) and never used.
  auto fetch_ids = [&](const Cursor& c) __attribute__((always_inline)) {
    const int kb = c.st * kStep;
    const int32_t* b = p.block_table + c.R.kv_start + (kb >> 4);
    id0 = load_scalar(b);
    id1 = load_scalar(b + (kb + 16 < c.R.n_keys ? 1 : 0));
  };
  int64_t vblk[kSets];
  auto load_k = [&](int X, bool real) __attribute__((always_inline)) {
    const int64_t blk = real ? (n >= 8 ? id1 : id0) : 0;
    vblk[X] = real ? (g >= 2 ? id1 : id0) : 0;
    const uint8_t* kp = Kc + e4m3::codes_at<D>(blk, kvh, Hkv) + g * (kBlock * 16) + (n & 7) * 16;
#pragma unroll
    for (int T = 0; T < 2; ++T)
#pragma unroll
      for (int j = 0; j < NP; ++j) kf[X][T][j] = load16_nt(kp + 8 * T * 16 + 4 * j * (kBlock * 16));
    ks[X] = load_pair(p.scales + e4m3::scales_at(blk, kvh, Hkv) + 4 * ((n >> 2) & 1));
  };
  auto load_v = [&](int X) __attribute__((always_inline)) {
    const uint8_t* vp = Vc + e4m3::codes_at<D>(vblk[X], kvh, Hkv) + (16 * (g & 1) + n) * kBlock;
#pragma unroll
    for (int e = 0; e < NDM / 2; ++e) vf[X][e] = load16_nt(vp + e * 32 * kBlock);
    vs[X] = load_pair(p.scales + e4m3::scales_at(vblk[X], kvh, Hkv) + kBlock + 4 * (g & 1));
  };

  float m_run = -INFINITY, l_part = 0.f;
  f32x4_t acc[NDM];
#pragma unroll
  for (int dm = 0; dm < NDM; ++dm) acc[dm] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // This column's limit in the compute cursor's range (scalar loads, picked per
  // lane: a vector load here would have the compiler wait for every load in flight).
  int lim = 0;
  const int t_lo = w.col0 / G, t_hi = min(w.ntok - 1, (w.col0 + kPrivateCols - 1) / G);
  auto load_lim = [&]() __attribute__((always_inline)) {
    if (C.R.lim_off < 0) {
      lim = C.R.n_keys;
      return;
    }
    int v = 0;
    for (int i = t_lo; i <= t_hi; ++i) {
      const int32_t li = load_scalar(p.lims + C.R.lim_off + i);
      v = t == i ? li : v;
    }
    lim = valid ? v : 0;
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

  auto step = [&](auto xc) __attribute__((always_inline)) {
    constexpr int X = decltype(xc)::value;
    const int kb = C.st * kStep, first = kb + 16 * (g >> 1) + 4 * (g & 1);  // (of the lane's tokens)
    f32x4_t S[2];
#pragma unroll
    for (int T = 0; T < 2; ++T) {
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
    if (__any(e4m3::has_nan(vs[X][0]) || e4m3::has_nan(vs[X][1]))) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t m = 255u << (8 * (e & 3));
        if ((vs[X][e / 4] & m) == m) {
          S[e / 4][e % 4] = __uint_as_float(0x7fc00000u);
          vs[X][e / 4] &= ~m;
        }
      }
    }
    if (kb + kStep > C.R.min_lim) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (first + 8 * (e / 4) + e % 4 >= lim) S[e / 4][e % 4] = -INFINITY;
    }
    float mx = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])),
                     fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
    mx = max_lane_halves(max_lane_rows(mx));
    const float m_new = fmaxf(m_run, mx * sl2);
    const float m_sub = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = fast_exp2(m_run - m_sub);
    m_run = m_new;
    float ls = 0.f;
    bf16x8_t pb;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = fast_exp2(fmaf(S[e / 4][e % 4], sl2, -m_sub));
      ls += x;
      pb[e] = (__bf16)(x * e4m3::scale_value((vs[X][e / 4] >> (8 * (e & 3))) & 255u));
    }
    l_part = fmaf(l_part, alpha, ls);
    u32x2 v[NDM];  // codes of the lane's eight tokens of row blocks 0 .. NDM-1
#pragma unroll
    for (int e = 0; e < NDM / 2; ++e)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(vf[X][e][2 * i], vf[X][e][2 * i + 1], false, false);
        v[2 * e][i] = r[0];
        v[2 * e + 1][i] = r[1];
      }
    if (kb + kStep > C.R.n_keys) {  // tokens past the range's end: their P is 0, but slots may hold anything
      const int keep = C.R.n_keys - first;
      uint32_t m[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k = keep - 8 * i;
        m[i] = k >= 4 ? 0xffffffffu : k <= 0 ? 0u : 0xffffffffu >> (8 * (4 - k));
      }
#pragma unroll
      for (int dm = 0; dm < NDM; ++dm)
#pragma unroll
        for (int i = 0; i < 2; ++i) v[dm][i] &= m[i];
    }
#pragma unroll
    for (int dm = 0; dm < NDM; ++dm) {
      acc[dm] *= alpha;
      acc[dm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e4m3::values8(v[dm][0], v[dm][1], 1.f), pb, acc[dm], 0, 0, 0);
    }
    load_v(X);  // set X's V is consumed
    advance(L);
    fetch_ids(L);
    const int ri_before = C.ri;
    advance(C);
    if (C.ok && C.ri != ri_before) load_lim();
  };
  // Two steps a turn, counted ahead: left from within, the loop would have a path
  // (for the compiler) from a step to itself, with half of the loads in flight,
  // and its waits would allow no more.
  static_assert(kSets == 2, "the loop names both sets");
  for (; n_steps >= 2; n_steps -= 2) {
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
  }
  if (n_steps > 0) step(std::integral_constant<int, 0>{});

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
__global__ __launch_bounds__(tile::kThreads) void decode_e4m3_kernel(TileParamsE4m3 p, int n_shared,
                                                                     int n_private, int n_groups, int* next) {
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
hipError_t launch_decode_e4m3(const TileParamsE4m3& p, int n_shared, int n_private, int n_groups, int* next, int D,
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
