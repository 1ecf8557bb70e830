// Rotary handles, and what the entry points around them refuse.  No HIP calls.
#include "rotary.hpp"

#include <algorithm>
#include <cmath>
#include <limits>
#include <new>
#include <numeric>
#include <vector>

using padoc::clear_error;
using padoc::set_error;

namespace padoc {
namespace {

constexpr int64_t kI32Max = std::numeric_limits<int32_t>::max();
constexpr int32_t kMaxHeads = 4096;
constexpr int64_t kMaxStride = int64_t(1) << 40;  // elements

// Elements from the first to one past the last of n rows of H heads, or -1
// when that does not fit.
int64_t extent(const padoc_heads& x, int64_t n, int32_t H, int32_t D) {
  int64_t a = 0, b = 0, e = 0;
  if (__builtin_mul_overflow(x.row_stride, n - 1, &a) || __builtin_mul_overflow(x.head_stride, (int64_t)H - 1, &b) ||
      __builtin_add_overflow(a, b, &e) || __builtin_add_overflow(e, (int64_t)D, &e) || e > (int64_t(1) << 58))
    return -1;
  return e;
}

padoc_status check_heads(const char* name, const padoc_heads& x, int64_t n, int32_t H, int32_t D, size_t esz,
                         bool written) {
  if (n == 0 || H == 0) return PADOC_OK;
  if (!x.data) return set_error(PADOC_ERR_ARG, "%s is null", name);
  if ((uintptr_t)x.data & (esz - 1)) return set_error(PADOC_ERR_ARG, "%s is not aligned to its element size", name);
  if (x.row_stride < 0 || x.head_stride < 0 || x.row_stride > kMaxStride || x.head_stride > kMaxStride)
    return set_error(PADOC_ERR_BOUNDS, "%s: strides (%lld, %lld) outside [0, 2^40]", name, (long long)x.row_stride,
                     (long long)x.head_stride);
  if (extent(x, n, H, D) < 0) return set_error(PADOC_ERR_BOUNDS, "%s: its last row overflows the address", name);
  if (!written) return PADOC_OK;
  // rows of whole heads, or heads of whole rows, or (one of each) anything
  const int64_t heads = (H - 1) * x.head_stride + D, rows = (n - 1) * x.row_stride + D;
  const bool apart = (H == 1 || x.head_stride >= D) && (n == 1 || x.row_stride >= D) &&
                     (n == 1 || x.row_stride >= heads || H == 1 || x.head_stride >= rows);
  if (!apart)
    return set_error(PADOC_ERR_BOUNDS, "%s: heads of strides (%lld, %lld) overlap and cannot be written", name,
                     (long long)x.row_stride, (long long)x.head_stride);
  return PADOC_OK;
}

// Rows of a call's tensor: n rows of H heads.
struct Rows {
  const char* name;
  const padoc_heads& at;
  int64_t n;
  int32_t H;
};

// Whether `out` may be written while `in` is read or written: apart, or (where
// `same` allows it) the same rows, which their one reader writes.
padoc_status check_apart(const Rows& in, const Rows& out, int32_t D, size_t esz, bool same) {
  if (in.n == 0 || in.H == 0 || out.n == 0 || out.H == 0) return PADOC_OK;
  const bool strides = in.n == 1 || in.at.row_stride == out.at.row_stride;
  if (same && in.at.data == out.at.data && strides && (in.H == 1 || in.at.head_stride == out.at.head_stride))
    return PADOC_OK;
  const uintptr_t a = (uintptr_t)in.at.data, b = (uintptr_t)out.at.data;
  const uintptr_t an = (uintptr_t)extent(in.at, in.n, in.H, D) * esz;
  const uintptr_t bn = (uintptr_t)extent(out.at, out.n, out.H, D) * esz;
  if (a + an <= b || b + bn <= a) return PADOC_OK;
  const auto clear = [&](int64_t step, int64_t in_span, int64_t out_span) {  // each within a step, beside the other
    const int64_t delta = ((int64_t)(b - a) % step + step) % step;
    return in_span <= delta && delta + out_span <= step;
  };
  // slices of the same rows side by side, or of the same heads where rows lie within heads
  for (int by_head = 0; by_head < 2; ++by_head) {
    const auto count = [&](const Rows& x) { return by_head ? (int64_t)x.H : x.n; };
    const auto stride = [&](const Rows& x) { return (by_head ? x.at.head_stride : x.at.row_stride) * (int64_t)esz; };
    const auto span = [&](const Rows& x) {
      return (by_head ? (x.n - 1) * x.at.row_stride : (x.H - 1) * x.at.head_stride) * (int64_t)esz + D * (int64_t)esz;
    };
    if (count(in) > 1 && count(out) > 1 && stride(in) == stride(out) && stride(in) > 0 &&
        clear(stride(in), span(in), span(out)))
      return PADOC_OK;
  }
  // heads side by side ([n, H, 3, D] with q, k and v of a head together): every
  // row and head lies a multiple of `step` elements from its tensor's start
  int64_t step = 0;
  for (const Rows* x : {&in, &out}) {
    if (x->n > 1) step = std::gcd(step, x->at.row_stride);
    if (x->H > 1) step = std::gcd(step, x->at.head_stride);
  }
  if (step > 0 && clear(step * (int64_t)esz, D * (int64_t)esz, D * (int64_t)esz)) return PADOC_OK;
  return set_error(PADOC_ERR_ARG, "%s overlaps %s%s", out.name, in.name, same ? " without being the same rows" : "");
}

padoc_status check_pos(const char* name, const padoc_rotary* r, const int32_t* pos, int64_t stride, int64_t n) {
  if (n == 0) return PADOC_OK;
  if (!pos) return set_error(PADOC_ERR_ARG, "%s is null", name);
  if ((uintptr_t)pos & 3) return set_error(PADOC_ERR_ARG, "%s is not aligned to its element size", name);
  if (stride < 0 || stride > kMaxStride || (r->n_axes > 1 && stride != 0 && stride < n))
    return set_error(PADOC_ERR_BOUNDS, "%s: axis stride %lld is neither 0 nor at least the %lld rows", name,
                     (long long)stride, (long long)n);
  return PADOC_OK;
}

padoc_status check_weight(const char* name, const void* w, size_t esz) {
  if ((uintptr_t)w & (esz - 1)) return set_error(PADOC_ERR_ARG, "%s is not aligned to its element size", name);
  return PADOC_OK;
}

padoc_status check_sizes(int64_t n, int32_t Hq, int32_t Hkv) {
  if (n < 0) return set_error(PADOC_ERR_ARG, "%lld rows are negative", (long long)n);
  if (n > kI32Max) return set_error(PADOC_ERR_BOUNDS, "%lld rows exceed 2^31-1", (long long)n);
  if (Hq < 0 || Hkv < 0 || Hq > kMaxHeads || Hkv > kMaxHeads)
    return set_error(PADOC_ERR_SHAPE, "head counts (Hq=%d, Hkv=%d) outside [0, %d]", Hq, Hkv, kMaxHeads);
  return PADOC_OK;
}

// The host copy of a call's block pairs: ids in range, no destination twice, and
// (`within` one cache) no block both source and destination.
padoc_status check_pairs_host(const int32_t* pairs_host, int64_t n_pairs, int64_t src_blocks, int64_t dst_blocks,
                              bool within) {
  if (!pairs_host) return PADOC_OK;
  try {
    std::vector<int32_t> src((size_t)n_pairs), dst((size_t)n_pairs);
    for (int64_t i = 0; i < n_pairs; ++i) {
      src[i] = pairs_host[2 * i];
      dst[i] = pairs_host[2 * i + 1];
      if (src[i] < 0 || src[i] >= src_blocks || dst[i] < 0 || dst[i] >= dst_blocks)
        return set_error(PADOC_ERR_BOUNDS, "pair %lld: blocks (%d, %d) outside [0, %lld) and [0, %lld)", (long long)i,
                         src[i], dst[i], (long long)src_blocks, (long long)dst_blocks);
    }
    std::sort(dst.begin(), dst.end());
    const auto twice = std::adjacent_find(dst.begin(), dst.end());
    if (twice != dst.end()) return set_error(PADOC_ERR_BOUNDS, "block %d is a destination twice", *twice);
    if (within) {
      std::sort(src.begin(), src.end());
      for (int32_t b : src)
        if (std::binary_search(dst.begin(), dst.end(), b))
          return set_error(PADOC_ERR_BOUNDS, "block %d is a source and a destination", b);
    }
  } catch (const std::bad_alloc&) {
    return set_error(PADOC_ERR_ARG, "out of host memory");
  }
  return PADOC_OK;
}

// Sizes of a call on blocks.
padoc_status check_block_sizes(int64_t src_blocks, int64_t dst_blocks, int64_t n_pairs, int32_t Hkv, int32_t D) {
  if (D != 64 && D != 128) return set_error(PADOC_ERR_SHAPE, "head_dim=%d is not 64 or 128", D);
  if (Hkv < 1 || Hkv > kMaxHeads) return set_error(PADOC_ERR_SHAPE, "Hkv=%d outside [1, %d]", Hkv, kMaxHeads);
  if (n_pairs < 0) return set_error(PADOC_ERR_ARG, "n_pairs = %lld is negative", (long long)n_pairs);
  if (n_pairs > kI32Max) return set_error(PADOC_ERR_BOUNDS, "%lld pairs exceed 2^31-1", (long long)n_pairs);
  if (src_blocks < 0 || src_blocks > kI32Max || dst_blocks < 0 || dst_blocks > kI32Max)
    return set_error(PADOC_ERR_ARG, "block counts (%lld, %lld) must be in [0, 2^31-1]", (long long)src_blocks,
                     (long long)dst_blocks);
  return PADOC_OK;
}

// Device memory of a call: `bytes` bytes from `p` on.
struct Span {
  const char* name;
  const void* p;
  int64_t bytes;
};
padoc_status check_spans(const Span* s, int n) {
  for (int i = 0; i < n; ++i) {
    if (!s[i].p) return set_error(PADOC_ERR_ARG, "%s is null", s[i].name);
    if ((uintptr_t)s[i].p & 15) return set_error(PADOC_ERR_ARG, "%s must be 16-byte aligned", s[i].name);
    for (int j = 0; j < i; ++j)
      if ((uintptr_t)s[i].p < (uintptr_t)s[j].p + (uintptr_t)s[j].bytes &&
          (uintptr_t)s[j].p < (uintptr_t)s[i].p + (uintptr_t)s[i].bytes)
        return set_error(PADOC_ERR_ARG, "%s overlaps %s", s[i].name, s[j].name);
  }
  return PADOC_OK;
}

#define PADOC_TRY(expr)                     \
  do {                                      \
    const padoc_status st_ = (expr);        \
    if (st_ != PADOC_OK) return st_;        \
  } while (0)

}  // namespace

padoc_status check_rotary_fwd(const padoc_rotary* r, const padoc_rotary_fwd_args* a) {
  if (!r) return set_error(PADOC_ERR_ARG, "rotary is null");
  if (!a) return set_error(PADOC_ERR_ARG, "args is null");
  const int64_t n = a->n_rows;
  const int32_t Hq = a->num_heads_q, Hkv = a->num_heads_kv;
  const size_t e = r->esize();
  PADOC_TRY(check_sizes(n, Hq, Hkv));
  if (Hq + Hkv > 0) PADOC_TRY(check_pos("pos", r, a->pos, a->pos_stride, n));
  PADOC_TRY(check_heads("q", a->q, n, Hq, r->D, e, false));
  PADOC_TRY(check_heads("k", a->k, n, Hkv, r->D, e, false));
  PADOC_TRY(check_heads("q_out", a->q_out, n, Hq, r->D, e, true));
  PADOC_TRY(check_heads("k_out", a->k_out, n, Hkv, r->D, e, true));
  const Rows q{"q", a->q, n, Hq}, k{"k", a->k, n, Hkv};
  const Rows q_out{"q_out", a->q_out, n, Hq}, k_out{"k_out", a->k_out, n, Hkv};
  PADOC_TRY(check_apart(q, q_out, r->D, e, true));
  PADOC_TRY(check_apart(k, k_out, r->D, e, true));
  PADOC_TRY(check_apart(k, q_out, r->D, e, false));
  PADOC_TRY(check_apart(q, k_out, r->D, e, false));
  PADOC_TRY(check_apart(q_out, k_out, r->D, e, false));
  PADOC_TRY(check_weight("q_weight", a->q_weight, e));
  PADOC_TRY(check_weight("k_weight", a->k_weight, e));
  return PADOC_OK;
}

padoc_status check_rotary_bwd(const padoc_rotary* r, const padoc_rotary_bwd_args* a) {
  if (!r) return set_error(PADOC_ERR_ARG, "rotary is null");
  if (!a) return set_error(PADOC_ERR_ARG, "args is null");
  const int64_t n = a->n_rows;
  const int32_t Hq = a->num_heads_q, Hkv = a->num_heads_kv;
  const size_t e = r->esize();
  PADOC_TRY(check_sizes(n, Hq, Hkv));
  if (Hq + Hkv > 0) PADOC_TRY(check_pos("pos", r, a->pos, a->pos_stride, n));
  if ((a->dq_weight && !a->q_weight) || (a->dk_weight && !a->k_weight))
    return set_error(PADOC_ERR_ARG, "a weight's gradient is asked for without the weight");
  if (((uintptr_t)a->dq_weight | (uintptr_t)a->dk_weight) & 3)
    return set_error(PADOC_ERR_ARG, "dq_weight / dk_weight must be 4-byte aligned");
  if (a->dq_weight && a->dq_weight == a->dk_weight)
    return set_error(PADOC_ERR_ARG, "dq_weight and dk_weight are the same buffer");
  PADOC_TRY(check_heads("dq_out", a->dq_out, n, Hq, r->D, e, false));
  PADOC_TRY(check_heads("dk_out", a->dk_out, n, Hkv, r->D, e, false));
  PADOC_TRY(check_heads("dq", a->dq, n, Hq, r->D, e, true));
  PADOC_TRY(check_heads("dk", a->dk, n, Hkv, r->D, e, true));
  const Rows dq_out{"dq_out", a->dq_out, n, Hq}, dk_out{"dk_out", a->dk_out, n, Hkv};
  const Rows dq{"dq", a->dq, n, Hq}, dk{"dk", a->dk, n, Hkv};
  PADOC_TRY(check_apart(dq_out, dq, r->D, e, true));
  PADOC_TRY(check_apart(dk_out, dk, r->D, e, true));
  PADOC_TRY(check_apart(dk_out, dq, r->D, e, false));
  PADOC_TRY(check_apart(dq_out, dk, r->D, e, false));
  PADOC_TRY(check_apart(dq, dk, r->D, e, false));
  if (a->q_weight) {
    const Rows q{"q", a->q, n, Hq};
    PADOC_TRY(check_heads("q", a->q, n, Hq, r->D, e, false));
    PADOC_TRY(check_apart(q, dq, r->D, e, true));
    PADOC_TRY(check_apart(q, dk, r->D, e, false));
  }
  if (a->k_weight) {
    const Rows k{"k", a->k, n, Hkv};
    PADOC_TRY(check_heads("k", a->k, n, Hkv, r->D, e, false));
    PADOC_TRY(check_apart(k, dk, r->D, e, true));
    PADOC_TRY(check_apart(k, dq, r->D, e, false));
  }
  PADOC_TRY(check_weight("q_weight", a->q_weight, e));
  PADOC_TRY(check_weight("k_weight", a->k_weight, e));
  return PADOC_OK;
}

padoc_status check_rotary_append(const padoc_rotary* r, const padoc_rotary_append_args* a, bool session) {
  if (!r) return set_error(PADOC_ERR_ARG, "rotary is null");
  if (!a) return set_error(PADOC_ERR_ARG, "args is null");
  const int32_t Hq = a->num_heads_q, Hkv = a->num_heads_kv;
  const size_t e = r->esize();
  PADOC_TRY(check_sizes(a->n_q, Hq, Hkv));
  PADOC_TRY(check_sizes(a->n_new, Hq, Hkv));
  const bool any_q = a->n_q > 0 && Hq > 0, any_k = a->n_new > 0 && Hkv > 0;
  if (any_k || (any_q && !a->q_pos)) PADOC_TRY(check_pos("pos", r, a->pos, a->pos_stride, a->n_new));
  if (any_q && a->q_pos) PADOC_TRY(check_pos("q_pos", r, a->q_pos, a->q_pos_stride, a->n_q));
  if (any_q && !a->q_pos && a->n_q != a->n_new)
    return set_error(PADOC_ERR_ARG, "%lld query rows and %lld new rows need q_pos", (long long)a->n_q,
                     (long long)a->n_new);
  PADOC_TRY(check_heads("q", a->q, a->n_q, Hq, r->D, e, false));
  PADOC_TRY(check_heads("q_out", a->q_out, a->n_q, Hq, r->D, e, true));
  PADOC_TRY(check_heads("k", a->k, a->n_new, Hkv, r->D, e, false));
  PADOC_TRY(check_heads("v", a->v, a->n_new, Hkv, r->D, e, false));
  const Rows q_out{"q_out", a->q_out, a->n_q, Hq};
  PADOC_TRY(check_apart(Rows{"q", a->q, a->n_q, Hq}, q_out, r->D, e, true));
  PADOC_TRY(check_apart(Rows{"k", a->k, a->n_new, Hkv}, q_out, r->D, e, false));
  PADOC_TRY(check_apart(Rows{"v", a->v, a->n_new, Hkv}, q_out, r->D, e, false));
  PADOC_TRY(check_weight("q_weight", a->q_weight, e));
  PADOC_TRY(check_weight("k_weight", a->k_weight, e));
  if (session) {
    if (a->slots || a->k_cache || a->v_cache || a->num_blocks)
      return set_error(PADOC_ERR_ARG, "slots, k_cache, v_cache and num_blocks are the session's and must be 0");
    return PADOC_OK;
  }
  if (a->num_blocks < 0 || a->num_blocks > kI32Max)
    return set_error(PADOC_ERR_ARG, "num_blocks=%lld must be in [0, 2^31-1]", (long long)a->num_blocks);
  if (any_k) {
    if (!a->slots || !a->k_cache || !a->v_cache) return set_error(PADOC_ERR_ARG, "slots or a cache is null");
    if ((uintptr_t)a->slots & 3) return set_error(PADOC_ERR_ARG, "slots must be 4-byte aligned");
    if (((uintptr_t)a->k_cache | (uintptr_t)a->v_cache) & 15)
      return set_error(PADOC_ERR_ARG, "the caches must be 16-byte aligned");
    if (a->k_cache == a->v_cache) return set_error(PADOC_ERR_ARG, "k_cache and v_cache are the same buffer");
  }
  return PADOC_OK;
}

padoc_status check_copy_blocks(const void* k_src, const void* v_src, int64_t src_blocks, const void* k_dst,
                               const void* v_dst, int64_t dst_blocks, const int32_t* pairs, int64_t n_pairs,
                               const int32_t* pairs_host, int32_t Hkv, int32_t D, padoc_dtype dtype) {
  if (dtype != PADOC_F32 && dtype != PADOC_BF16)
    return set_error(PADOC_ERR_DTYPE, "dtype %d is not PADOC_F32 or PADOC_BF16", (int)dtype);
  PADOC_TRY(check_block_sizes(src_blocks, dst_blocks, n_pairs, Hkv, D));
  if (n_pairs == 0) return PADOC_OK;
  if (!k_src || !v_src || !k_dst || !v_dst || !pairs) return set_error(PADOC_ERR_ARG, "null buffer pointer");
  if (((uintptr_t)k_src | (uintptr_t)v_src | (uintptr_t)k_dst | (uintptr_t)v_dst) & 15)
    return set_error(PADOC_ERR_ARG, "the caches must be 16-byte aligned");
  if ((uintptr_t)pairs & 3) return set_error(PADOC_ERR_ARG, "pairs must be 4-byte aligned");
  if (k_src == v_src || k_dst == v_dst || k_src == v_dst || v_src == k_dst)
    return set_error(PADOC_ERR_ARG, "K and V caches must be distinct buffers");
  if ((k_src == k_dst) != (v_src == v_dst))
    return set_error(PADOC_ERR_ARG, "K and V must both be copied within their cache, or both to another");
  const int64_t block = (int64_t)Hkv * 16 * D * (dtype == PADOC_BF16 ? 2 : 4);
  if (k_src != k_dst) {
    const uintptr_t sn = (uintptr_t)(src_blocks * block), dn = (uintptr_t)(dst_blocks * block);
    for (const void* s : {k_src, v_src})
      for (const void* d : {k_dst, v_dst})
        if ((uintptr_t)s < (uintptr_t)d + dn && (uintptr_t)d < (uintptr_t)s + sn)
          return set_error(PADOC_ERR_ARG, "source and destination caches overlap without being the same");
  }
  return check_pairs_host(pairs_host, n_pairs, src_blocks, dst_blocks, k_src == k_dst);
}

padoc_status check_copy_blocks_e4m3(const padoc_cache_e4m3* src, const padoc_cache_e4m3* dst, const int32_t* pairs,
                                    int64_t n_pairs, const int32_t* pairs_host, int32_t Hkv, int32_t D) {
  if (!src || !dst) return set_error(PADOC_ERR_ARG, "src or dst is null");
  PADOC_TRY(check_block_sizes(src->num_blocks, dst->num_blocks, n_pairs, Hkv, D));
  if (n_pairs == 0) return PADOC_OK;
  if (!pairs) return set_error(PADOC_ERR_ARG, "pairs is null");
  if ((uintptr_t)pairs & 3) return set_error(PADOC_ERR_ARG, "pairs must be 4-byte aligned");
  const int64_t codes = (int64_t)Hkv * 16 * D, bytes = (int64_t)Hkv * 32;
  const Span spans[6] = {{"k of src", src->k, src->num_blocks * codes}, {"v of src", src->v, src->num_blocks * codes},
                         {"scales of src", src->scales, src->num_blocks * bytes},
                         {"k of dst", dst->k, dst->num_blocks * codes}, {"v of dst", dst->v, dst->num_blocks * codes},
                         {"scales of dst", dst->scales, dst->num_blocks * bytes}};
  const bool within = src->k == dst->k && src->v == dst->v && src->scales == dst->scales;
  PADOC_TRY(check_spans(spans, within ? 3 : 6));
  if (within && src->num_blocks != dst->num_blocks)
    return set_error(PADOC_ERR_ARG, "one cache with two block counts (%lld, %lld)", (long long)src->num_blocks,
                     (long long)dst->num_blocks);
  return check_pairs_host(pairs_host, n_pairs, src->num_blocks, dst->num_blocks, within);
}

padoc_status check_cast_blocks(const void* k, const void* v, int64_t blocks, const padoc_cache_e4m3* cache,
                               int64_t dst_blocks, int64_t src_blocks, const int32_t* pairs, int64_t n_pairs,
                               const int32_t* pairs_host, int32_t Hkv, int32_t D, padoc_dtype dtype, bool back) {
  if (!cache) return set_error(PADOC_ERR_ARG, "%s is null", back ? "src" : "dst");
  if (dtype != PADOC_F32 && dtype != PADOC_BF16)
    return set_error(PADOC_ERR_DTYPE, "dtype %d is not PADOC_F32 or PADOC_BF16", (int)dtype);
  PADOC_TRY(check_block_sizes(src_blocks, dst_blocks, n_pairs, Hkv, D));
  if (!pairs && n_pairs > std::min(src_blocks, dst_blocks))
    return set_error(PADOC_ERR_BOUNDS, "%lld blocks without pairs, of caches of %lld and %lld", (long long)n_pairs,
                     (long long)src_blocks, (long long)dst_blocks);
  if (!pairs && pairs_host) return set_error(PADOC_ERR_ARG, "pairs_host without pairs");
  if (n_pairs == 0) return PADOC_OK;
  if ((uintptr_t)pairs & 3) return set_error(PADOC_ERR_ARG, "pairs must be 4-byte aligned");
  const int64_t codes = (int64_t)Hkv * 16 * D, values = codes * (dtype == PADOC_BF16 ? 2 : 4);
  const Span spans[5] = {{back ? "k_dst" : "k_src", k, blocks * values}, {back ? "v_dst" : "v_src", v, blocks * values},
                         {"k of the 8-bit cache", cache->k, cache->num_blocks * codes},
                         {"v of the 8-bit cache", cache->v, cache->num_blocks * codes},
                         {"scales of the 8-bit cache", cache->scales, cache->num_blocks * Hkv * 32}};
  PADOC_TRY(check_spans(spans, 5));
  return check_pairs_host(pairs_host, n_pairs, src_blocks, dst_blocks, false);
}

padoc_status check_rotary_append_e4m3(const padoc_rotary* r, const padoc_rotary_append_args* a,
                                      const padoc_cache_e4m3* cache) {
  if (!a) return set_error(PADOC_ERR_ARG, "args is null");
  if (!cache) return set_error(PADOC_ERR_ARG, "cache is null");
  if (a->k_cache || a->v_cache || a->num_blocks)
    return set_error(PADOC_ERR_ARG, "k_cache, v_cache and num_blocks are the 8-bit cache's and must be 0");
  padoc_rotary_append_args rows = *a;
  rows.k_cache = cache->k;
  rows.v_cache = cache->v;
  rows.num_blocks = cache->num_blocks;
  PADOC_TRY(check_rotary_append(r, &rows, /*session=*/false));
  if (a->n_new == 0 || a->num_heads_kv == 0) return PADOC_OK;
  const int64_t codes = (int64_t)a->num_heads_kv * 16 * r->D;
  const Span spans[3] = {{"k of the cache", cache->k, cache->num_blocks * codes},
                         {"v of the cache", cache->v, cache->num_blocks * codes},
                         {"scales of the cache", cache->scales, cache->num_blocks * a->num_heads_kv * 32}};
  return check_spans(spans, 3);
}

}  // namespace padoc

extern "C" padoc_status padoc_rotary_create(const padoc_rotary_desc* d, padoc_rotary** out) {
  clear_error();
  if (!out) return set_error(PADOC_ERR_ARG, "out is null");
  *out = nullptr;
  if (!d) return set_error(PADOC_ERR_ARG, "desc is null");
  if (d->dtype != PADOC_F32 && d->dtype != PADOC_BF16)
    return set_error(PADOC_ERR_DTYPE, "dtype %d is not PADOC_F32 or PADOC_BF16", (int)d->dtype);
  if (d->head_dim != 64 && d->head_dim != 128)
    return set_error(PADOC_ERR_SHAPE, "head_dim=%d is not 64 or 128", d->head_dim);
  if (d->rotary_dim < 16 || d->rotary_dim > d->head_dim || d->rotary_dim % 16)
    return set_error(PADOC_ERR_SHAPE, "rotary_dim=%d is not a multiple of 16 in [16, head_dim=%d]", d->rotary_dim,
                     d->head_dim);
  if (d->n_axes < 1 || d->n_axes > padoc::kMaxAxes)
    return set_error(PADOC_ERR_SHAPE, "n_axes=%d outside [1, %d]", d->n_axes, padoc::kMaxAxes);
  if (d->style != PADOC_ROTARY_HALVES && d->style != PADOC_ROTARY_PAIRS)
    return set_error(PADOC_ERR_ARG, "style %d is not PADOC_ROTARY_HALVES or PADOC_ROTARY_PAIRS", d->style);
  if (!std::isfinite(d->scale)) return set_error(PADOC_ERR_ARG, "scale must be finite");
  if (!std::isfinite(d->norm_eps) || d->norm_eps < 0.f)
    return set_error(PADOC_ERR_ARG, "norm_eps must be finite and not negative");
  if (!d->inv_freq && (!std::isfinite(d->base) || d->base <= 0.0))
    return set_error(PADOC_ERR_ARG, "base must be positive and finite");
  const int32_t pairs = d->rotary_dim / 2;
  for (int32_t i = 0; i < pairs; ++i) {
    if (d->axis && (d->axis[i] < 0 || d->axis[i] >= d->n_axes))
      return set_error(PADOC_ERR_BOUNDS, "axis[%d]=%d outside [0, n_axes=%d)", i, d->axis[i], d->n_axes);
    if (d->inv_freq && !std::isfinite(d->inv_freq[i]))
      return set_error(PADOC_ERR_ARG, "inv_freq[%d] is not finite", i);
  }
  if (!d->inv_freq && !std::isfinite(std::pow(d->base, -2.0 * (pairs - 1) / d->rotary_dim)))
    return set_error(PADOC_ERR_ARG, "base %g gives frequencies that are not finite", d->base);
  padoc_rotary* r = new (std::nothrow) padoc_rotary();
  if (!r) return set_error(PADOC_ERR_ARG, "out of host memory");
  r->D = d->head_dim;
  r->pairs = pairs;
  r->n_axes = d->n_axes;
  r->style = d->style;
  r->scale = d->scale;
  r->eps = d->norm_eps;
  r->dtype = d->dtype;
  for (int32_t i = 0; i < pairs; ++i) {
    const double f = d->inv_freq ? d->inv_freq[i] : std::pow(d->base, -2.0 * i / d->rotary_dim);
    // Whole turns per position change nothing (positions are whole numbers);
    // the rest, in [-1/2, 1/2], as a fraction of 2^64.  The long double's 64
    // bits of fraction leave an error below 2^-64 turns, 2^-33 at any position.
    const long double turns = (long double)f / 6.283185307179586476925286766559005768L;
    const long double rest = turns - std::rint(turns);
    r->table.turn[i] = (uint64_t)(__int128)std::rint(rest * 18446744073709551616.0L);
    r->table.axis[i] = (uint8_t)(d->axis ? d->axis[i] : 0);
  }
  *out = r;
  return PADOC_OK;
}

extern "C" void padoc_rotary_destroy(padoc_rotary* r) { delete r; }
