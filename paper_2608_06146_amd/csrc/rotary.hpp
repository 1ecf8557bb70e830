// Kernel parameter blocks of the rotary and block-copy kernels, shared by the
// entry points and the kernels.
#pragma once

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

struct RotaryParams {
  RotaryTable table;
  const int32_t* pos;  // [n_axes][stride]
  int64_t pos_stride;
  int32_t n_axes, pairs;  // pairs: rotary_dim / 2
  float scale, eps;
  int32_t inverse;  // rotate by the negative angle
  int32_t n, Hq, Hkv;
  int32_t heads_per_group;  // heads of a row that one lane group takes
  padoc_heads q, k;    // in: rows, or (inverse, backward) gradients of the outputs
  padoc_heads qo, ko;  // out
  const void* wq;
  const void* wk;
  // backward with weights
  padoc_heads xq, xk;  // the forward's rows
  float* part;         // [blocks][2][D] sums of the weights' gradients, or null
  // append
  const int32_t* q_pos;
  int64_t q_pos_stride;
  int32_t n_q;
  padoc_heads v;
  const int32_t* slots;
  void* k_cache;
  void* v_cache;
  int64_t n_blocks;
  const int32_t* patch;  // (entry, block id) pairs of the block table
  int64_t n_patch;
  int32_t* block_table;
  int64_t items_q, items_k, items_v, items;  // workgroup items of each role, and all
};

struct CopyParams {
  const void* k_src;
  const void* v_src;
  void* k_dst;
  void* v_dst;
  const int32_t* pairs;
  int64_t n_pairs, src_blocks, dst_blocks;
  int64_t units;  // 16-byte units of a block, per tensor
};

// Grid of the backward's kernel over rows and heads: the partial sums it
// leaves are counted by the host before any launch.
struct BwdGrid {
  int32_t x, y, heads_per_group;
};
BwdGrid rotary_bwd_grid(int64_t n, int Hq, int Hkv, int D);

}  // namespace padoc
