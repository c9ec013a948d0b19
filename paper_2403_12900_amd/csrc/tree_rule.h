// Host side of the drafted-tree operators: what a call's batch must satisfy,
// the relations between its token rows, and the rules that size the launches.
// Pure C++ (no HIP): the device library and the host test library share it.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <string>

#include "host_state.h"

namespace sprk {

constexpr int kTreeReqs = SPR_MAX_TREE_REQUESTS;
constexpr int kTreeNodes = SPR_MAX_TREE_NODES;
constexpr int kTreeRows = SPR_MAX_TREE_ROWS;
constexpr int kTreeMaxLen = 1 << 30;  // positions stay far from the 32-bit limit
static_assert(kTreeNodes == 64, "ancestor sets are 64-bit masks");
static_assert(kTreeRows == spr::kMaxRows, "a tree step is one decode pass");

// The trees of one call.  Row r = row0[i] + j is node j of request i.
struct TreeInfo {
  int n = 0, rows = 0, max_nodes = 0, max_levels = 0, max_children = 0;
  int slot[kTreeReqs], len[kTreeReqs], nodes[kTreeReqs], levels[kTreeReqs];
  int row0[kTreeReqs + 1];
  int children[kTreeReqs];       // most children of one of its nodes
  int8_t parent[kTreeRows];      // node, -1 for a root
  uint8_t depth[kTreeRows];
  uint8_t rank[kTreeRows];       // earlier children of the same parent
  uint8_t kids[kTreeRows];       // children of the node
  uint64_t anc[kTreeRows];       // bit a: node a is the row's node or an ancestor of it
};

// Checks a batch and derives its relations.  what: the caller's name, for the
// message.  with_cache: slots and lens are read, against n_slots table rows
// of max_blocks blocks.
inline spr_status parse_tree(const spr_tree_batch* b, bool with_cache, int n_slots, int max_blocks,
                             const char* what, TreeInfo* t, std::string* err) {
  const auto bad = [&](const std::string& m) {
    *err = std::string(what) + ": " + m;
    return SPR_ERR_INVALID_ARG;
  };
  if (b == nullptr || b->n_nodes == nullptr || b->parents == nullptr ||
      (with_cache && (b->slots == nullptr || b->lens == nullptr)))
    return bad("batch and its arrays must not be null");
  if (b->n < 1 || b->n > kTreeReqs) return bad("n must be in [1, SPR_MAX_TREE_REQUESTS]");
  t->n = b->n;
  t->rows = t->max_nodes = t->max_levels = t->max_children = 0;
  for (int i = 0; i < b->n; ++i) {
    const int nn = b->n_nodes[i];
    if (nn < 1 || nn > kTreeNodes) return bad("n_nodes must be in [1, SPR_MAX_TREE_NODES]");
    const int r0 = t->rows;
    if (r0 + nn > kTreeRows) return bad("more than SPR_MAX_TREE_ROWS nodes in all");
    t->row0[i] = r0;
    t->nodes[i] = nn;
    t->slot[i] = t->len[i] = 0;
    if (with_cache) {
      const int s = b->slots[i];
      if (s < 0 || s >= n_slots) return bad("slot id out of range");
      for (int k = 0; k < i; ++k)
        if (t->slot[k] == s) return bad("slot listed twice");
      if (b->lens[i] < 0 || b->lens[i] > kTreeMaxLen) return bad("lens must be in [0, 2^30]");
      if (static_cast<int64_t>(b->lens[i]) + nn > static_cast<int64_t>(max_blocks) * spr::kKvBlock)
        return bad("lens + n_nodes exceeds the slot's block-table row");
      t->slot[i] = s;
      t->len[i] = b->lens[i];
    }
    int levels = 1, most = 0;
    for (int j = 0; j < nn; ++j) {
      const int p = b->parents[r0 + j];
      if (j == 0 ? p != -1 : (p < 0 || p >= j)) return bad("parents must be -1 for node 0 and in [0, j) for node j");
      const int r = r0 + j;
      t->parent[r] = static_cast<int8_t>(p);
      t->kids[r] = t->rank[r] = t->depth[r] = 0;
      t->anc[r] = uint64_t{1} << j;
      if (j > 0) {
        t->anc[r] |= t->anc[r0 + p];
        t->depth[r] = static_cast<uint8_t>(t->depth[r0 + p] + 1);
        t->rank[r] = t->kids[r0 + p]++;
        levels = std::max(levels, t->depth[r] + 1);
        most = std::max<int>(most, t->kids[r0 + p]);
      }
    }
    t->levels[i] = levels;
    t->children[i] = most;
    t->rows += nn;
    t->max_nodes = std::max(t->max_nodes, nn);
    t->max_levels = std::max(t->max_levels, levels);
    t->max_children = std::max(t->max_children, most);
  }
  t->row0[t->n] = t->rows;
  return SPR_OK;
}

// Columns that one work-group of the attention kernel takes: 16 or 32 where
// that holds the widest request (its four waves then share out the blocks),
// else 64 or 128 (16 or 32 columns per wave), as far as `most`.
inline int tree_cols_per_group(const TreeInfo& t, int G, int most) {
  const int cols = t.max_nodes * G;
  int cw = 16;
  while (cw < cols && cw < most) cw *= 2;
  return cw;
}

// Work items of one attention launch: per request its column groups, each in
// KV splits of bps blocks.
struct TreeSplit {
  int bps = 1;
  // In launch order, the requests with the longest splits first, so that the
  // last work-groups to start are short ones: the request, its column groups,
  // the first of them and its first work item.
  uint8_t order[kTreeReqs], ncg[kTreeReqs], cg0[kTreeReqs];
  int item0[kTreeReqs + 1];
};

// Splits hold `least` blocks (a step of every wave that walks blocks) until
// the launch has more than its share of resident work-groups (`slots`) takes
// at once; they grow further while the partials exceed `floats` or a request
// has more than kTreeSplits.
constexpr int kTreeSplits = 32;
inline TreeSplit tree_split(const TreeInfo& t, int G, int Hkv, int hd, int cw, int least, int slots, size_t floats) {
  TreeSplit s;
  const auto blocks_of = [&](int i) { return (t.len[i] + t.nodes[i] + 15) / 16; };
  for (int i = 0; i < t.n; ++i) s.order[i] = static_cast<uint8_t>(i);
  std::stable_sort(s.order, s.order + t.n, [&](int i, int j) { return blocks_of(i) > blocks_of(j); });
  int64_t blocks = 0;
  int cg = 0;
  for (int r = 0; r < t.n; ++r) {
    const int i = s.order[r];
    s.ncg[r] = static_cast<uint8_t>((t.nodes[i] * G + cw - 1) / cw);
    s.cg0[r] = static_cast<uint8_t>(cg);
    cg += s.ncg[r];
    blocks += static_cast<int64_t>(s.ncg[r]) * blocks_of(i);
  }
  const int64_t per = static_cast<int64_t>(Hkv) * cw * (hd + 4);
  int64_t bps = std::max<int64_t>(1, (blocks * Hkv + slots - 1) / slots);
  // Rounding every request up to whole splits can leave more work-groups than
  // stay resident; splits up to twice as long that fit them into one round are
  // taken, but not longer ones (16 requests of 64 columns, 100 to 1500
  // positions, calls in a row: 56 us, without this 61.5).
  const auto groups = [&](int64_t w) {
    int64_t n = 0;
    for (int r = 0; r < t.n; ++r) n += (blocks_of(s.order[r]) + w - 1) / w * s.ncg[r];
    return n * Hkv;
  };
  for (int k = 0; k <= 8; ++k) {
    const int64_t whole = (bps + bps * k / 8 + least - 1) / least * least;
    if (groups(whole) <= slots) {
      bps = whole;
      break;
    }
  }
  for (;; bps += std::max<int64_t>(least, bps / 8)) {
    bps = (bps + least - 1) / least * least;
    int64_t items = 0, most = 1;
    for (int r = 0; r < t.n; ++r) {
      const int64_t ns = (blocks_of(s.order[r]) + bps - 1) / bps;
      s.item0[r] = static_cast<int>(items);
      items += ns * s.ncg[r];
      most = std::max(most, ns);
    }
    s.item0[t.n] = static_cast<int>(items);
    if (most == 1 || (most <= kTreeSplits && items * per <= static_cast<int64_t>(floats))) break;
  }
  s.bps = static_cast<int>(bps);
  return s;
}

// Checks a view; layer in [0, n_layers) (0 where all layers are meant).
inline spr_status check_view(const spr_kv_view* v, int layer, const char* what, std::string* err) {
  const auto bad = [&](const std::string& m) {
    *err = std::string(what) + ": " + m;
    return SPR_ERR_INVALID_ARG;
  };
  if (v == nullptr || v->k == nullptr || v->v == nullptr || v->block_table == nullptr)
    return bad("the view and its pointers must not be null");
  if ((reinterpret_cast<uintptr_t>(v->k) | reinterpret_cast<uintptr_t>(v->v)) & 15)
    return bad("k and v must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(v->block_table) & 3) return bad("the block table must be 4-byte aligned");
  if (v->kv_dtype != SPR_F32 && v->kv_dtype != SPR_BF16) return bad("unknown kv_dtype");
  if (v->head_dim != 64 && v->head_dim != 128) return bad("head_dim must be 64 or 128");
  if (v->n_kv_heads < 1 || v->n_kv_heads > 512) return bad("n_kv_heads must be in [1, 512]");
  if (v->n_layers < 1 || v->n_blocks < 1 || v->n_slots < 1 || v->max_blocks < 1)
    return bad("n_layers, n_blocks, n_slots and max_blocks must be >= 1");
  if (layer < 0 || layer >= v->n_layers) return bad("layer must be in [0, n_layers)");
  return SPR_OK;
}

// Whether two sets of `rows` rows of `width` bytes share a byte; rows of a set
// do not overlap each other (stride >= width > 0).
inline bool rows_overlap(uint64_t a, int64_t a_stride, uint64_t b, int64_t b_stride, int64_t width, int rows) {
  const int64_t off = static_cast<int64_t>(b - a);  // of b's first row
  for (int r = 0; r < rows; ++r) {
    // Row k of b starts at off + k b_stride; the last that starts before a's row r ends.
    const int64_t end = r * a_stride + width - 1 - off;
    if (end < 0) continue;
    const int64_t k = std::min<int64_t>(end / b_stride, rows - 1);
    if (off + k * b_stride + width > r * a_stride) return true;
  }
  return false;
}

// Temperatures (host, or null: 1) are finite and >= 0; random numbers may be
// missing only where every request is greedy.
inline spr_status check_temperatures(int n, const float* temperature, const float* accept, const float* sample,
                                     const char* what, std::string* err) {
  bool drawn = temperature == nullptr;
  for (int i = 0; i < n && temperature != nullptr; ++i) {
    const float v = temperature[i];
    if (!(v >= 0.f && v <= 3.402823466e38f)) {
      *err = std::string(what) + ": temperatures must be finite and >= 0";
      return SPR_ERR_INVALID_ARG;
    }
    drawn |= v > 0.f;
  }
  if (drawn && (accept == nullptr || sample == nullptr)) {
    *err = std::string(what) + ": accept and sample must not be null where a temperature is above 0";
    return SPR_ERR_INVALID_ARG;
  }
  return SPR_OK;
}

}  // namespace sprk
