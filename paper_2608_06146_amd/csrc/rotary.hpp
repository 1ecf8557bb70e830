// Kernel parameter blocks of the rotary and block-copy kernels, shared by the
// entry points and the kernels.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "padoc_attn.h"

namespace padoc {

constexpr int kMaxAxes = 4;
constexpr int kMaxPairs = 64;  // rotary_dim / 2

// Per pair: turns per position as a fraction of 2^64 (a position times it,
// modulo 2^64, is the angle in turns, whatever the position), and its axis.
// Passed to the kernels by value, so a handle owns no device memory.
struct RotaryTable {
  uint64_t turn[kMaxPairs];
  uint8_t axis[kMaxPairs];
};

// How the rows of one tensor are cut into tiles, one workgroup each.
struct TileGrid {
  int32_t rows;       // rows of a tile
  int32_t heads;      // heads of a tile
  int32_t head_runs;  // tiles side by side over the heads
  int64_t items;      // workgroups (backward: each takes every (items / head_runs)-th tile)
};

struct RotaryParams {
  RotaryTable table;
  const int32_t* pos;  // [n_axes][stride]
  int64_t pos_stride;
  int32_t pairs;  // rotary_dim / 2
  float scale, eps;
  int32_t inverse;  // rotate by the negative angle
  int32_t n, n_q;   // rows of k (and v), of q
  int32_t Hq, Hkv;
  TileGrid tiles_q, tiles_k;
  int64_t items;       // workgroup items of all kinds
  padoc_heads q, k;    // in: rows, or (inverse, backward) gradients of the outputs
  padoc_heads qo, ko;  // out
  const void* wq;
  const void* wk;
  // backward with weights
  padoc_heads xq, xk;  // the forward's rows
  float* part;         // [items of q, then of k][D] sums of the weights' gradients, or null
  // append
  const int32_t* q_pos;
  int64_t q_pos_stride;
  padoc_heads v;
  const int32_t* slots;
  void* k_cache;
  void* v_cache;
  uint8_t* scales;       // 8-bit caches (k_cache and v_cache hold codes)
  int64_t n_blocks;
  const int32_t* patch;  // (entry, block id) pairs of the block table
  int64_t n_patch;
  int32_t* block_table;
  int64_t items_v;
};

struct CopyParams {
  const void* k_src;
  const void* v_src;
  void* k_dst;
  void* v_dst;
  const int32_t* pairs;
  int64_t n_pairs, src_blocks, dst_blocks;
  int64_t units;  // 16-byte units of a block, per tensor
  // 8-bit caches: scales, and 16-byte units of a block's
  const void* s_src;
  void* s_dst;
  int64_t s_units;
};

// Blocks between caches of values and 8-bit caches (one way or the other).
struct CastParams {
  const void* k;  // values in
  const void* v;
  void* k_out;    // values out
  void* v_out;
  uint8_t* k_codes;
  uint8_t* v_codes;
  uint8_t* scales;
  const int32_t* pairs;  // null: block i to block i
  int64_t n_pairs, src_blocks, dst_blocks;
  int32_t Hkv;
};

// Items of a backward: each leaves D sums in the workspace.
size_t rotary_bwd_parts(int64_t n, int Hq, int Hkv, int D, bool bf16);

}  // namespace padoc
