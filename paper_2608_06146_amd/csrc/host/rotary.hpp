// Rotary handle and the argument checks of its entry points.  Host only.
#pragma once

#include "../rotary.hpp"
#include "plan.hpp"

struct padoc_rotary {
  padoc::RotaryTable table{};
  int32_t D = 0, pairs = 0, n_axes = 1, style = 0;
  float scale = 1.f, eps = 0.f;
  padoc_dtype dtype = PADOC_BF16;
  size_t esize() const { return dtype == PADOC_BF16 ? 2 : 4; }
};

namespace padoc {

padoc_status check_rotary_fwd(const padoc_rotary* r, const padoc_rotary_fwd_args* a);
padoc_status check_rotary_bwd(const padoc_rotary* r, const padoc_rotary_bwd_args* a);
// `session`: slots and caches come from the session (must be unset in `a`).
padoc_status check_rotary_append(const padoc_rotary* r, const padoc_rotary_append_args* a, bool session);
padoc_status check_copy_blocks(const void* k_src, const void* v_src, int64_t src_blocks, const void* k_dst,
                               const void* v_dst, int64_t dst_blocks, const int32_t* pairs, int64_t n_pairs,
                               const int32_t* pairs_host, int32_t Hkv, int32_t D, padoc_dtype dtype);

}  // namespace padoc
