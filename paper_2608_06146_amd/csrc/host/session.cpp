// Decode session, host side: stream tree, block pool, block-table regions
// and the per-step schedule (App. E, the masked parallel decoding loop).
// No HIP calls: the launch lives with the other entry points that enqueue
// device work.
#include "session.hpp"

#include <algorithm>
#include <cstring>
#include <limits>
#include <memory>
#include <new>

using padoc::clear_error;
using padoc::set_error;

namespace {

constexpr int32_t kBlk = 16;     // tokens per paged block
constexpr int32_t kMinCls = 2;   // smallest block-table region: 4 entries (64 tokens)
constexpr int64_t kI32Max = std::numeric_limits<int32_t>::max();

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

int32_t class_for(int64_t entries) {
  int32_t c = kMinCls;
  while ((int64_t(1) << c) < entries) ++c;
  return c;
}

bool alloc_region(padoc_session* s, int32_t cls, int64_t& off) {
  if (cls >= (int32_t)s->free_regions.size()) s->free_regions.resize(cls + 1);
  auto& fl = s->free_regions[cls];
  if (!fl.empty()) {
    off = fl.back();
    fl.pop_back();
    return true;
  }
  const int64_t n = int64_t(1) << cls;
  if (s->bt_top + n > s->desc.block_table_capacity) return false;
  off = s->bt_top;
  s->bt_top += n;
  return true;
}

void free_region(padoc_session* s, int32_t cls, int64_t off) {
  s->free_regions[cls].push_back(off);
  std::fill(s->bt_host.begin() + off, s->bt_host.begin() + off + (int64_t(1) << cls), -1);
}

void erase_sorted(std::vector<int32_t>& v, int32_t id) {
  auto it = std::lower_bound(v.begin(), v.end(), id);
  if (it != v.end() && *it == id) v.erase(it);
}

int32_t take_block(padoc_session* s) {
  const int32_t b = s->free_blocks.back();
  s->free_blocks.pop_back();
  s->block_refs[b] = 1;
  return b;
}

void drop_block(padoc_session* s, int32_t b) {
  if (--s->block_refs[b] == 0) s->free_blocks.push_back(b);
}

// Copy block src to dst in the next launch, after the copies before it that
// write src or dst or read dst.  `grow` was called for it.
void add_copy(padoc_session* s, int32_t src, int32_t dst) {
  const int32_t phase = std::max({0, s->write_phase[src] + 1, s->write_phase[dst] + 1, s->read_phase[dst] + 1});
  s->write_phase[dst] = phase;
  s->read_phase[src] = std::max(s->read_phase[src], phase);
  s->pending_copies.push_back({src, dst, phase});
}

template <class V>
void grow(V& v, size_t more) {  // room for `more` entries, at least doubling
  if (v.capacity() - v.size() < more) v.reserve(std::max(v.size() + more, 2 * v.size()));
}

// Whether a step that appends to stream x has to copy its last block first,
// when `copied` other streams of the step already do.
bool shares_last_block(const padoc_session* s, const padoc_session::Stream& x, int32_t copied) {
  return x.len % kBlk != 0 && s->block_refs[x.blocks.back()] - copied > 1;
}

// Release `id` and then its ancestors while they are closed and have no kept
// child: blocks back to the pool, region back to its free list.
void release_upwards(padoc_session* s, int32_t id) {
  while (id >= 0) {
    padoc_session::Stream& x = s->st[id];
    if (x.open || !x.kept || x.kept_children > 0) return;
    x.kept = false;
    for (auto it = x.blocks.rbegin(); it != x.blocks.rend(); ++it) drop_block(s, *it);
    x.blocks.clear();
    x.blocks.shrink_to_fit();
    if (x.cls >= 0) free_region(s, x.cls, x.bt_off);
    x.cls = -1;
    erase_sorted(s->kept_ids, id);
    if (x.parent >= 0) --s->st[x.parent].kept_children;
    id = x.parent;
  }
}

padoc_status check_session(const padoc_session* s) {
  if (!s) return set_error(PADOC_ERR_ARG, "session is null");
  return PADOC_OK;
}

padoc_status check_unprepared(const padoc_session* s) {
  if (s->prepared)
    return set_error(PADOC_ERR_MODE, "a prepared step has not been launched or committed");
  return PADOC_OK;
}

// The pending copies by phase, into copy_ptr and copy_pairs (which have room).
void order_copies(padoc_session* s) {
  std::stable_sort(s->pending_copies.begin(), s->pending_copies.end(),
                   [](const padoc_session::Copy& a, const padoc_session::Copy& b) { return a.phase < b.phase; });
  s->copy_ptr.clear();
  s->copy_pairs.clear();
  int32_t phase = -1;
  for (const padoc_session::Copy& c : s->pending_copies) {
    for (; phase < c.phase; ++phase) s->copy_ptr.push_back((int32_t)(s->copy_pairs.size() / 2));
    s->copy_pairs.push_back(c.src);
    s->copy_pairs.push_back(c.dst);
    s->write_phase[c.src] = s->write_phase[c.dst] = s->read_phase[c.src] = s->read_phase[c.dst] = -1;
  }
  s->copy_ptr.push_back((int32_t)(s->copy_pairs.size() / 2));
  s->pending_copies.clear();
}

// The step's tree: every kept stream in id order with its length after the
// step (lengths as they stand when n_new is null); a stream moving to a new
// block-table region (moving_to >= 0) is placed there.
void fill_tree(padoc_session* s, const int32_t* n_new, const int32_t* n_query, std::vector<padoc_segment>& seg,
               std::vector<int32_t>& seg_id) {
  seg.clear();
  seg_id.clear();
  int64_t q = 0;
  size_t row = 0;
  for (int32_t id : s->kept_ids) {
    padoc_session::Stream& x = s->st[id];
    padoc_segment g{};
    g.parent = x.parent >= 0 ? s->st[x.parent].index : -1;  // kept parents come first
    g.fork = x.fork;
    g.len = x.len;
    g.q_len = 0;
    g.kv_off = x.moving_to >= 0 ? x.moving_to : (x.cls >= 0 ? x.bt_off : 0);
    g.q_off = q;
    if (row < s->open_ids.size() && s->open_ids[row] == id) {
      if (n_new) {
        g.len += n_new[row];
        g.q_len = n_query[row];
        q += n_query[row];
      }
      ++row;
    }
    x.index = (int32_t)seg.size();
    seg.push_back(g);
    seg_id.push_back(id);
  }
}

}  // namespace

namespace padoc {
void session_free_host(padoc_session* s) { delete s; }
}  // namespace padoc

extern "C" padoc_status padoc_session_create(const padoc_session_desc* d, padoc_session** out) {
  clear_error();
  if (!out) return set_error(PADOC_ERR_ARG, "out is null");
  *out = nullptr;
  if (!d) return set_error(PADOC_ERR_ARG, "desc is null");
  if (d->dtype != PADOC_F32 && d->dtype != PADOC_BF16)
    return set_error(PADOC_ERR_DTYPE, "dtype %d is not PADOC_F32 or PADOC_BF16", (int)d->dtype);
  if (d->num_blocks < 0 || d->num_blocks > kI32Max)
    return set_error(PADOC_ERR_ARG, "num_blocks=%lld must be in [0, 2^31-1]", (long long)d->num_blocks);
  if (d->block_table_capacity < 0 || d->block_table_capacity > kI32Max)
    return set_error(PADOC_ERR_ARG, "block_table_capacity=%lld must be in [0, 2^31-1]",
                     (long long)d->block_table_capacity);
  // Head counts, head_dim, scale and schedule knobs are checked by a probe
  // plan of an empty tree (the same checks every step's plan passes).
  padoc_tree_desc probe{};
  probe.num_heads_q = d->num_heads_q;
  probe.num_heads_kv = d->num_heads_kv;
  probe.head_dim = d->head_dim;
  probe.softmax_scale = d->softmax_scale;
  probe.dtype = d->dtype;
  probe.block_size = kBlk;
  probe.num_kv_rows = d->num_blocks;
  probe.block_table_len = d->block_table_capacity;
  probe.max_chunk_keys = d->max_chunk_keys;
  probe.target_workgroups = d->target_workgroups;
  try {
    std::unique_ptr<padoc_session> s(new padoc_session());
    padoc_status st = padoc::build_plan(&probe, s->plan);
    if (st != PADOC_OK) return st;
    s->desc = *d;
    s->free_blocks.resize((size_t)d->num_blocks);
    for (int64_t i = 0; i < d->num_blocks; ++i) s->free_blocks[(size_t)i] = (int32_t)(d->num_blocks - 1 - i);
    s->bt_host.assign((size_t)d->block_table_capacity, -1);
    s->block_refs.assign((size_t)d->num_blocks, 0);
    s->write_phase.assign((size_t)d->num_blocks, -1);
    s->read_phase.assign((size_t)d->num_blocks, -1);
    s->taken.assign((size_t)d->num_blocks, 0);
    *out = s.release();
  } catch (const std::bad_alloc&) {
    return set_error(PADOC_ERR_ARG, "out of host memory creating the session");
  }
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_open(padoc_session* s, int32_t parent, int32_t fork, int32_t* id) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  if ((st = check_unprepared(s)) != PADOC_OK) return st;
  if (!id) return set_error(PADOC_ERR_ARG, "id is null");
  if (parent < -1 || parent >= (int32_t)s->st.size())
    return set_error(PADOC_ERR_ARG, "parent %d is not a stream of this session", parent);
  if (parent >= 0 && !s->st[parent].kept)
    return set_error(PADOC_ERR_ARG, "parent %d has been released", parent);
  if (parent < 0 ? fork != 0 : (fork < 0 || fork > s->st[parent].len))
    return set_error(PADOC_ERR_TREE, "fork %d outside [0, %d] (parent %d)", fork,
                     parent < 0 ? 0 : s->st[parent].len, parent);
  if ((int64_t)s->st.size() >= kI32Max) return set_error(PADOC_ERR_ARG, "too many streams");
  try {
    padoc_session::Stream x;
    x.parent = parent;
    x.fork = fork;
    const int32_t nid = (int32_t)s->st.size();
    s->st.push_back(std::move(x));
    s->open_ids.push_back(nid);
    s->kept_ids.push_back(nid);
    if (parent >= 0) ++s->st[parent].kept_children;
    *id = nid;
  } catch (const std::bad_alloc&) {
    return set_error(PADOC_ERR_ARG, "out of host memory");
  }
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_close(padoc_session* s, int32_t id) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  if ((st = check_unprepared(s)) != PADOC_OK) return st;
  if (id < 0 || id >= (int32_t)s->st.size() || !s->st[id].open)
    return set_error(PADOC_ERR_ARG, "stream %d is not open", id);
  s->st[id].open = false;
  erase_sorted(s->open_ids, id);
  release_upwards(s, id);
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_clone(padoc_session* s, int32_t id, int32_t len, int32_t* new_id) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  if ((st = check_unprepared(s)) != PADOC_OK) return st;
  if (!new_id) return set_error(PADOC_ERR_ARG, "new_id is null");
  if (id < 0 || id >= (int32_t)s->st.size() || !s->st[id].kept)
    return set_error(PADOC_ERR_ARG, "stream %d is not a kept stream of this session", id);
  if (len < 0 || len > s->st[id].len)
    return set_error(PADOC_ERR_TREE, "len %d outside [0, %d] (stream %d)", len, s->st[id].len, id);
  if ((int64_t)s->st.size() >= kI32Max) return set_error(PADOC_ERR_ARG, "too many streams");
  const int64_t nb = ceil_div(len, kBlk);
  try {
    const padoc_session::Stream& from = s->st[id];
    padoc_session::Stream x;
    x.parent = from.parent;
    x.fork = from.fork;
    x.len = len;
    x.blocks.assign(from.blocks.begin(), from.blocks.begin() + nb);
    grow(s->st, 1);  // from here on nothing throws
    grow(s->open_ids, 1);
    grow(s->kept_ids, 1);
    grow(s->pending_entries, (size_t)nb);
    if (nb > 0) {
      const int32_t cls = class_for(nb);
      if (!alloc_region(s, cls, x.bt_off))
        return set_error(PADOC_ERR_BOUNDS, "the block table (%lld entries) cannot hold the clone",
                         (long long)s->desc.block_table_capacity);
      x.cls = cls;
    }
    for (int64_t j = 0; j < nb; ++j) {
      ++s->block_refs[x.blocks[(size_t)j]];
      s->bt_host[(size_t)(x.bt_off + j)] = x.blocks[(size_t)j];
      s->pending_entries.push_back(x.bt_off + j);
    }
    const int32_t nid = (int32_t)s->st.size();
    if (x.parent >= 0) ++s->st[x.parent].kept_children;
    s->st.push_back(std::move(x));
    s->open_ids.push_back(nid);
    s->kept_ids.push_back(nid);
    *new_id = nid;
  } catch (const std::bad_alloc&) {
    return set_error(PADOC_ERR_ARG, "out of host memory");
  }
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_truncate(padoc_session* s, int32_t id, int32_t len) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  if ((st = check_unprepared(s)) != PADOC_OK) return st;
  if (id < 0 || id >= (int32_t)s->st.size() || !s->st[id].open)
    return set_error(PADOC_ERR_ARG, "stream %d is not open", id);
  padoc_session::Stream& x = s->st[id];
  if (len < 0 || len > x.len) return set_error(PADOC_ERR_TREE, "len %d outside [0, %d] (stream %d)", len, x.len, id);
  if (x.kept_children > 0)
    for (int32_t c : s->kept_ids)
      if (s->st[c].parent == id && s->st[c].fork > len)
        return set_error(PADOC_ERR_TREE, "stream %d sees %d tokens of stream %d, more than %d", c, s->st[c].fork, id,
                         len);
  const size_t nb = (size_t)ceil_div(len, kBlk);
  for (size_t j = x.blocks.size(); j > nb; --j) {
    drop_block(s, x.blocks[j - 1]);  // (free_blocks has held every block of the pool: no allocation)
    s->bt_host[(size_t)x.bt_off + j - 1] = -1;
  }
  x.blocks.resize(nb);
  x.len = len;
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_compact(padoc_session* s, int32_t max_moves, int32_t* n_moves) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  if ((st = check_unprepared(s)) != PADOC_OK) return st;
  if (max_moves < 0) return set_error(PADOC_ERR_ARG, "max_moves = %d is negative", max_moves);
  try {
    const int32_t n = (int32_t)s->desc.num_blocks;
    const int32_t used = n - (int32_t)s->free_blocks.size();
    // The moves: the i-th largest kept id to the i-th smallest free one.
    std::vector<int32_t> to((size_t)n, -1);
    std::vector<std::pair<int32_t, int32_t>> moves;
    for (int32_t dst = 0, src = n - 1; max_moves == 0 || (int32_t)moves.size() < max_moves; ++dst, --src) {
      while (dst < used && s->block_refs[dst] > 0) ++dst;
      if (dst >= used) break;
      while (s->block_refs[src] == 0) --src;  // (a free id below `used` leaves a kept one behind it)
      moves.push_back({src, dst});
      to[src] = dst;
    }
    int64_t entries = 0;
    for (int32_t id : s->kept_ids)
      for (int32_t b : s->st[id].blocks) entries += to[b] >= 0;
    grow(s->pending_entries, (size_t)entries);  // from here on nothing throws
    grow(s->pending_copies, moves.size());
    for (const auto& m : moves) {
      add_copy(s, m.first, m.second);
      s->block_refs[m.second] = s->block_refs[m.first];
      s->block_refs[m.first] = 0;
    }
    if (!moves.empty())
      for (int32_t id : s->kept_ids) {
        padoc_session::Stream& x = s->st[id];
        for (size_t j = 0; j < x.blocks.size(); ++j) {
          if (to[x.blocks[j]] < 0) continue;
          x.blocks[j] = to[x.blocks[j]];
          const int64_t e = x.bt_off + (int64_t)j;
          s->bt_host[(size_t)e] = x.blocks[j];
          s->pending_entries.push_back(e);
        }
      }
    s->free_blocks.clear();
    for (int32_t b = n - 1; b >= 0; --b)
      if (s->block_refs[b] == 0) s->free_blocks.push_back(b);
    if (n_moves) *n_moves = (int32_t)moves.size();
  } catch (const std::bad_alloc&) {
    return set_error(PADOC_ERR_ARG, "out of host memory");
  }
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_resize(padoc_session* s, int64_t num_blocks, void* k_cache, void* v_cache) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  if ((st = check_unprepared(s)) != PADOC_OK) return st;
  if (num_blocks < 0 || num_blocks > kI32Max)
    return set_error(PADOC_ERR_ARG, "num_blocks=%lld must be in [0, 2^31-1]", (long long)num_blocks);
  if (!s->pending_copies.empty())
    return set_error(PADOC_ERR_MODE, "block copies wait for the launch of a step");
  // (caches of no blocks may have no address)
  const bool emptied = s->desc.num_blocks == 0 && s->desc.block_table;
  const auto fits = [&](const void* now, const void* was) {
    return now ? was || emptied : !was || num_blocks == 0;
  };
  if (!fits(k_cache, s->desc.k_cache) || !fits(v_cache, s->desc.v_cache))
    return set_error(PADOC_ERR_ARG, "a session has device caches or none, from its creation on");
  const int64_t old = s->desc.num_blocks;
  for (int64_t b = num_blocks; b < old; ++b)
    if (s->block_refs[(size_t)b] > 0)
      return set_error(PADOC_ERR_BOUNDS, "block %lld is in use, behind the %lld blocks of the new pool", (long long)b,
                       (long long)num_blocks);
  try {
    std::vector<int32_t> free_blocks;
    free_blocks.reserve((size_t)num_blocks);
    for (int64_t b = num_blocks - 1; b >= old; --b) free_blocks.push_back((int32_t)b);  // taken last
    for (int32_t b : s->free_blocks)
      if (b < num_blocks) free_blocks.push_back(b);
    const size_t n = (size_t)num_blocks;
    for (std::vector<int32_t>* v : {&s->block_refs, &s->write_phase, &s->read_phase, &s->taken}) v->reserve(n);
    s->block_refs.resize(n, 0);
    s->write_phase.resize(n, -1);
    s->read_phase.resize(n, -1);
    s->taken.resize(n, 0);
    s->free_blocks.swap(free_blocks);
    s->desc.num_blocks = num_blocks;
    s->desc.k_cache = k_cache;
    s->desc.v_cache = v_cache;
  } catch (const std::bad_alloc&) {
    return set_error(PADOC_ERR_ARG, "out of host memory");
  }
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_copies(const padoc_session* s, int32_t* n_phases, const int32_t** phase_ptr,
                                             const int32_t** pairs) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  if (!n_phases || !phase_ptr || !pairs) return set_error(PADOC_ERR_ARG, "null pointer");
  *n_phases = s->prepared ? (int32_t)s->copy_ptr.size() - 1 : 0;
  *phase_ptr = s->prepared ? s->copy_ptr.data() : nullptr;
  *pairs = s->prepared ? s->copy_pairs.data() : nullptr;
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_select(const padoc_session* s, int32_t max_rows, const int64_t* priority,
                                             int32_t* n_new, int32_t* n_query) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  const size_t R = s->open_ids.size();
  if (R > 0 && (!n_new || !n_query)) return set_error(PADOC_ERR_ARG, "null pointer");
  if (max_rows < 0) return set_error(PADOC_ERR_ARG, "max_rows = %d is negative", max_rows);
  try {
    std::vector<int32_t> order(R);
    for (size_t i = 0; i < R; ++i) order[i] = (int32_t)i;
    const size_t take = max_rows == 0 ? R : std::min(R, (size_t)max_rows);
    // rows are in ascending stream id, so without priorities the first
    // `take` rows are the oldest streams; with them, the largest priority
    // first, equal priorities by ascending id
    if (priority && take < R)
      std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return priority[a] > priority[b]; });
    for (size_t i = 0; i < R; ++i) n_new[i] = n_query[i] = 0;
    for (size_t i = 0; i < take; ++i) n_new[order[i]] = n_query[order[i]] = 1;
  } catch (const std::bad_alloc&) {
    return set_error(PADOC_ERR_ARG, "out of host memory");
  }
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_prepare(padoc_session* s, const int32_t* n_new_in, const int32_t* n_query_in,
                                              int32_t* n_kv_rows, int32_t* n_q_rows, size_t* workspace_bytes) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  if ((st = check_unprepared(s)) != PADOC_OK) return st;
  const size_t R = s->open_ids.size();
  try {
    std::vector<int32_t> ones;
    if (!n_new_in || !n_query_in) ones.assign(R, 1);
    const int32_t* n_new = n_new_in ? n_new_in : ones.data();
    const int32_t* n_query = n_query_in ? n_query_in : ones.data();
    int64_t total_new = 0, total_q = 0, need_blocks = 0, n_shared = 0;
    for (size_t i = 0; i < R; ++i) {
      const padoc_session::Stream& x = s->st[s->open_ids[i]];
      if (n_new[i] < 0 || n_query[i] < 0 || n_query[i] > n_new[i])
        return set_error(PADOC_ERR_ARG, "row %zu: need 0 <= n_query (%d) <= n_new (%d)", i, n_query[i], n_new[i]);
      if ((int64_t)x.len + n_new[i] > kI32Max) return set_error(PADOC_ERR_BOUNDS, "stream length exceeds 2^31-1");
      total_new += n_new[i];
      total_q += n_query[i];
      need_blocks += ceil_div((int64_t)x.len + n_new[i], kBlk) - (int64_t)x.blocks.size();
    }
    // Streams that append to a block others hold copy it, all but the last of
    // a block's holders.
    for (size_t i = 0; i < R; ++i) {
      const padoc_session::Stream& x = s->st[s->open_ids[i]];
      if (n_new[i] > 0 && x.len % kBlk != 0 && shares_last_block(s, x, s->taken[x.blocks.back()])) {
        ++s->taken[x.blocks.back()];
        ++n_shared;
      }
    }
    if (n_shared > 0)
      for (size_t i = 0; i < R; ++i) {
        const padoc_session::Stream& x = s->st[s->open_ids[i]];
        if (!x.blocks.empty()) s->taken[x.blocks.back()] = 0;
      }
    need_blocks += n_shared;
    if (total_new > kI32Max || total_q > kI32Max) return set_error(PADOC_ERR_BOUNDS, "step exceeds 2^31-1 rows");
    if (need_blocks > (int64_t)s->free_blocks.size())
      return set_error(PADOC_ERR_BOUNDS, "the step needs %lld blocks, the pool has %zu free", (long long)need_blocks,
                       s->free_blocks.size());
    // Region moves (tentative until the plan is built).
    struct Move {
      int32_t id, cls;
      int64_t off;
    };
    std::vector<Move> moves;
    auto undo = [&] {
      for (const Move& m : moves) {
        s->free_regions[m.cls].push_back(m.off);
        s->st[m.id].moving_to = -1;
      }
    };
    for (size_t i = 0; i < R; ++i) {
      const int32_t id = s->open_ids[i];
      const padoc_session::Stream& x = s->st[id];
      const int64_t nb = ceil_div((int64_t)x.len + n_new[i], kBlk);
      if (nb == 0 || (x.cls >= 0 && (int64_t(1) << x.cls) >= nb)) continue;
      Move m{id, class_for(nb), 0};
      if (!alloc_region(s, m.cls, m.off)) {
        undo();
        return set_error(PADOC_ERR_BOUNDS, "the block table (%lld entries) cannot hold the step",
                         (long long)s->desc.block_table_capacity);
      }
      moves.push_back(m);
      s->st[id].moving_to = m.off;
    }
    // The step's schedule.
    fill_tree(s, n_new, n_query, s->seg, s->seg_id);
    padoc_tree_desc d{};
    d.n_seg = (int32_t)s->seg.size();
    d.seg = s->seg.data();
    d.num_heads_q = s->desc.num_heads_q;
    d.num_heads_kv = s->desc.num_heads_kv;
    d.head_dim = s->desc.head_dim;
    d.softmax_scale = s->desc.softmax_scale;
    d.dtype = s->desc.dtype;
    d.block_size = kBlk;
    d.num_kv_rows = s->desc.num_blocks;
    d.num_q_rows = total_q;
    d.block_table_len = s->desc.block_table_capacity;
    d.max_chunk_keys = s->desc.max_chunk_keys;
    d.target_workgroups = s->desc.target_workgroups;
    st = padoc::build_plan(&d, s->plan);
    if (st != PADOC_OK) {
      undo();
      return st;
    }
    // Commit: blocks, regions, patches, slots of the new rows.
    s->new_slot.resize((size_t)total_new * 2);
    grow(s->pending_copies, (size_t)n_shared);
    grow(s->pending_entries, (size_t)n_shared);
    s->copy_ptr.reserve(s->pending_copies.size() + (size_t)n_shared + 1);
    s->copy_pairs.reserve(2 * (s->pending_copies.size() + (size_t)n_shared));
    s->patch.clear();
    s->row_id.assign(s->open_ids.begin(), s->open_ids.end());
    s->row_n_new.assign(n_new, n_new + R);
    s->new_off.resize(R + 1);
    s->q_off.resize(R + 1);
    s->new_off[0] = s->q_off[0] = 0;
    for (size_t i = 0; i < R; ++i) {
      s->new_off[i + 1] = s->new_off[i] + n_new[i];
      s->q_off[i + 1] = s->q_off[i] + n_query[i];
    }
    for (size_t i = 0; n_shared > 0 && i < R; ++i) {
      padoc_session::Stream& x = s->st[s->open_ids[i]];
      if (n_new[i] == 0 || x.len % kBlk == 0 || !shares_last_block(s, x, 0)) continue;
      const int32_t b = take_block(s);
      add_copy(s, x.blocks.back(), b);
      --s->block_refs[x.blocks.back()];
      x.blocks.back() = b;
      if (x.moving_to < 0) {  // (a moving stream's entries are all written below)
        const int64_t e = x.bt_off + (int64_t)x.blocks.size() - 1;
        s->bt_host[(size_t)e] = b;
        s->pending_entries.push_back(e);
      }
    }
    for (const Move& m : moves) {
      padoc_session::Stream& x = s->st[m.id];
      x.moving_to = -1;
      if (x.cls >= 0) free_region(s, x.cls, x.bt_off);
      x.cls = m.cls;
      x.bt_off = m.off;
      for (size_t j = 0; j < x.blocks.size(); ++j) {
        s->bt_host[(size_t)x.bt_off + j] = x.blocks[j];
        s->patch.push_back((int32_t)(x.bt_off + (int64_t)j));
        s->patch.push_back(x.blocks[j]);
      }
    }
    for (size_t i = 0; i < R; ++i) {
      padoc_session::Stream& x = s->st[s->open_ids[i]];
      const int64_t nb = ceil_div((int64_t)x.len + n_new[i], kBlk);
      while ((int64_t)x.blocks.size() < nb) {
        const int32_t b = take_block(s);
        const int64_t e = x.bt_off + (int64_t)x.blocks.size();
        x.blocks.push_back(b);
        s->bt_host[(size_t)e] = b;
        s->patch.push_back((int32_t)e);
        s->patch.push_back(b);
      }
      int32_t* sl = s->new_slot.data() + 2 * (size_t)s->new_off[i];
      for (int32_t j = 0; j < n_new[i]; ++j) {
        const int32_t pos = x.len + j;
        sl[2 * j] = x.blocks[pos / kBlk];
        sl[2 * j + 1] = pos % kBlk;
      }
      x.len += n_new[i];
    }
    // Entries that clones, compactions and copies left to write, each once,
    // as they are now (free ones stay); what this step patches above is not
    // among them, or the same.
    if (!s->pending_entries.empty()) {
      std::sort(s->pending_entries.begin(), s->pending_entries.end());
      s->pending_entries.erase(std::unique(s->pending_entries.begin(), s->pending_entries.end()),
                               s->pending_entries.end());
      for (int64_t e : s->pending_entries)
        if (s->bt_host[(size_t)e] >= 0) {
          s->patch.push_back((int32_t)e);
          s->patch.push_back(s->bt_host[(size_t)e]);
        }
      s->pending_entries.clear();
    }
    order_copies(s);
    s->off_patch = align256((size_t)total_new * 8);
    s->off_copy = align256(s->off_patch + s->patch.size() * 4);
    s->rec_bytes = s->off_copy + s->copy_pairs.size() * 4;
    s->ws_records = align256(s->rec_bytes);
    s->ws_bytes = s->ws_records + s->plan.ws_bytes;
    s->prepared = true;
    if (n_kv_rows) *n_kv_rows = (int32_t)total_new;
    if (n_q_rows) *n_q_rows = (int32_t)total_q;
    if (workspace_bytes) *workspace_bytes = s->ws_bytes;
  } catch (const std::bad_alloc&) {
    return set_error(PADOC_ERR_ARG, "out of host memory preparing the step");
  }
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_commit(padoc_session* s) {
  clear_error();
  padoc_status st = check_session(s);
  if (st != PADOC_OK) return st;
  if (!s->prepared) return set_error(PADOC_ERR_MODE, "no step is prepared");
  s->prepared = false;
  return PADOC_OK;
}

extern "C" padoc_status padoc_session_view_get(const padoc_session* cs, padoc_session_view* v) {
  clear_error();
  padoc_status st = check_session(cs);
  if (st != PADOC_OK) return st;
  if (!v) return set_error(PADOC_ERR_ARG, "view is null");
  padoc_session* s = const_cast<padoc_session*>(cs);
  std::memset(v, 0, sizeof(*v));
  if (!s->prepared) {
    try {
      fill_tree(s, nullptr, nullptr, s->seg, s->seg_id);
      s->row_id.assign(s->open_ids.begin(), s->open_ids.end());
    } catch (const std::bad_alloc&) {
      return set_error(PADOC_ERR_ARG, "out of host memory");
    }
  }
  v->n_seg = (int32_t)s->seg.size();
  v->seg = s->seg.data();
  v->seg_id = s->seg_id.data();
  v->n_rows = (int32_t)s->row_id.size();
  v->row_id = s->row_id.data();
  if (s->prepared) {
    v->new_off = s->new_off.data();
    v->q_off = s->q_off.data();
    v->new_slot = s->new_slot.data();
    v->n_patch = (int32_t)(s->patch.size() / 2);
    v->patch = s->patch.data();
    v->plan = &s->plan;
    v->workspace_bytes = s->ws_bytes;
  }
  v->block_table = s->bt_host.data();
  v->free_blocks = (int64_t)s->free_blocks.size();
  return PADOC_OK;
}
