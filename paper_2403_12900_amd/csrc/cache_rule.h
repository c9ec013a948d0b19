// Host side of the 4-bit cache's operators: what a call's arguments must
// satisfy, and the rules that size the launches.  Pure C++ (no HIP): the
// device library and the host test library share it.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <string>
#include <vector>

#include "host_state.h"

namespace sprk {

constexpr int kCacheReqs = SPR_MAX_CACHE_REQUESTS;
constexpr int kCacheMaxRows = SPR_MAX_CACHE_ROWS;
constexpr int kCacheMaxLen = 1 << 30;  // positions stay far from the 32-bit limit

// First number among a[0..n) that repeats an earlier one, or -1.
inline int first_repeat(const int32_t* a, int n) {
  if (n <= 16) {
    for (int i = 1; i < n; ++i)
      for (int k = 0; k < i; ++k)
        if (a[k] == a[i]) return i;
    return -1;
  }
  std::vector<int32_t> s(a, a + n);
  std::sort(s.begin(), s.end());
  const auto at = std::adjacent_find(s.begin(), s.end());
  if (at == s.end()) return -1;
  return static_cast<int>(std::find(std::find(a, a + n, *at) + 1, a + n, *at) - a);
}

struct CacheInfo {
  int n = 0, rows = 0, max_rows = 0;
  int slot[kCacheReqs], len[kCacheReqs], n_rows[kCacheReqs], row0[kCacheReqs + 1];
};

// Checks a batch against a view's table.  what: the caller's name.
inline spr_status parse_cache(const spr_cache_batch* b, int n_slots, int max_blocks, const char* what, CacheInfo* t,
                              std::string* err) {
  const auto bad = [&](const char* m) {
    *err = std::string(what) + ": " + m;
    return SPR_ERR_INVALID_ARG;
  };
  if (b == nullptr || b->slots == nullptr || b->lens == nullptr || b->rows == nullptr)
    return bad("batch and its arrays must not be null");
  if (b->n < 1 || b->n > kCacheReqs) return bad("n must be in [1, SPR_MAX_CACHE_REQUESTS]");
  t->n = b->n;
  t->rows = t->max_rows = 0;
  for (int i = 0; i < b->n; ++i) {
    const int s = b->slots[i], len = b->lens[i], rows = b->rows[i];
    if (s < 0 || s >= n_slots) return bad("slot id out of range");
    if (len < 0 || len > kCacheMaxLen) return bad("lens must be in [0, 2^30]");
    if (rows < 1) return bad("rows must be >= 1");
    if (rows > kCacheMaxRows - t->rows) return bad("more than SPR_MAX_CACHE_ROWS rows in all");
    if (static_cast<int64_t>(len) + rows > static_cast<int64_t>(max_blocks) * spr::kKvBlock)
      return bad("lens + rows exceeds the slot's block-table row");
    t->slot[i] = s;
    t->len[i] = len;
    t->n_rows[i] = rows;
    t->row0[i] = t->rows;
    t->rows += rows;
    t->max_rows = std::max(t->max_rows, rows);
  }
  t->row0[t->n] = t->rows;
  if (first_repeat(t->slot, t->n) >= 0) return bad("slot listed twice");
  return SPR_OK;
}

inline spr_status check_kv4_view(const spr_kv4_view* v, int layer, const char* what, std::string* err) {
  const auto bad = [&](const char* m) {
    *err = std::string(what) + ": " + m;
    return SPR_ERR_INVALID_ARG;
  };
  if (v == nullptr || v->data == nullptr || v->block_table == nullptr)
    return bad("the view and its pointers must not be null");
  if (reinterpret_cast<uintptr_t>(v->data) & 15) return bad("data must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(v->block_table) & 3) return bad("the block table must be 4-byte aligned");
  if (v->head_dim != 64 && v->head_dim != 128) return bad("head_dim must be 64 or 128");
  if (v->n_kv_heads < 1 || v->n_kv_heads > 512) return bad("n_kv_heads must be in [1, 512]");
  if (v->n_layers < 1 || v->n_blocks < 1 || v->n_slots < 1 || v->max_blocks < 1)
    return bad("n_layers, n_blocks, n_slots and max_blocks must be >= 1");
  if (layer < 0 || layer >= v->n_layers) return bad("layer must be in [0, n_layers)");
  return SPR_OK;
}

inline spr_status check_rotary(const spr_rotary* r, int head_dim, const char* what, std::string* err) {
  const auto bad = [&](const char* m) {
    *err = std::string(what) + ": " + m;
    return SPR_ERR_INVALID_ARG;
  };
  if (r->dims < 2 || r->dims > head_dim || r->dims % 2 != 0)
    return bad("rotary dims must be even and in [2, head_dim]");
  if (r->pairs != 0 && r->pairs != 1) return bad("rotary pairs must be 0 or 1");
  if (!std::isfinite(r->amplitude)) return bad("the rotary amplitude must be finite");
  for (int k = 0; k < r->dims / 2; ++k)
    if (!std::isfinite(r->turns[k])) return bad("rotary frequencies must be finite");
  return SPR_OK;
}

inline spr_status make_rotary(int dims, int pairs, double base, double factor, double original, double low, double high,
                              double amplitude, spr_rotary* out, std::string* err) {
  const auto bad = [&](const char* m) {
    *err = std::string("rotary_init: ") + m;
    return SPR_ERR_INVALID_ARG;
  };
  if (out == nullptr) return bad("out must not be null");
  if (dims < 2 || dims > 128 || dims % 2 != 0) return bad("dims must be even and in [2, 128]");
  if (pairs != 0 && pairs != 1) return bad("pairs must be 0 or 1");
  if (!(base > 0 && std::isfinite(base))) return bad("base must be positive and finite");
  if (!(factor >= 1 && std::isfinite(factor))) return bad("factor must be finite and >= 1");
  if (!std::isfinite(amplitude)) return bad("amplitude must be finite");
  if (factor > 1 && !(original > 0 && std::isfinite(original) && std::isfinite(low) && std::isfinite(high) && high > low))
    return bad("original must be positive and high above low, all finite");
  const double turn = 2 * 3.14159265358979323846;
  *out = spr_rotary{};
  out->dims = dims;
  out->pairs = pairs;
  out->amplitude = amplitude;
  for (int k = 0; k < dims / 2; ++k) {
    double w = std::pow(base, -2.0 * k / dims);
    if (factor > 1) {
      const double keep = std::min(1.0, std::max(0.0, (original * w / turn - low) / (high - low)));
      w *= keep + (1 - keep) / factor;
    }
    if (!std::isfinite(w)) return bad("base is too small: a frequency is not finite");
    out->turns[k] = w / turn;
  }
  return SPR_OK;
}

inline spr_status check_pages(const spr_pages* p, const char* what, std::string* err) {
  const auto bad = [&](const char* m) {
    *err = std::string(what) + ": " + m;
    return SPR_ERR_INVALID_ARG;
  };
  if (p == nullptr || p->k == nullptr || p->block_table == nullptr) return bad("the pages and their pointers must not be null");
  if ((reinterpret_cast<uintptr_t>(p->k) | reinterpret_cast<uintptr_t>(p->v)) & 15) return bad("pools must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(p->block_table) & 3) return bad("the block table must be 4-byte aligned");
  if (p->n_layers < 1 || p->n_blocks < 1 || p->n_slots < 1 || p->max_blocks < 1)
    return bad("n_layers, n_blocks, n_slots and max_blocks must be >= 1");
  if (p->block_bytes < 16 || p->block_bytes % 16 != 0 || p->block_bytes > (int64_t{1} << 30))
    return bad("block_bytes must be a multiple of 16 in [16, 2^30]");
  return SPR_OK;
}

// Pieces of 16 bytes that a thread of a fork or a move copies, all in flight (a
// work-group has 256 times as many, of one block in one layer of one pool), moves of
// one launch, and table entries of one of its work-groups.
constexpr int kForkDeep = 1, kMoveDeep = 4, kMoves = 384, kTableEntries = 1024;
// Work-groups of a launch: its threads are counted in 32 bits.
constexpr int64_t kMostGroups = (int64_t{1} << 24) - 1;

// Work-groups that copy one block in every layer.
inline int64_t page_items(const spr_pages& p, int deep) {
  return (p.v != nullptr ? 2 : 1) * int64_t{p.n_layers} * ((p.block_bytes / 16 + 256 * deep - 1) / (256 * deep));
}
// Work-groups that look through the block table.
inline int64_t table_groups(const spr_pages& p) {
  return (static_cast<int64_t>(p.n_slots) * p.max_blocks + kTableEntries - 1) / kTableEntries;
}

// The forks of one call, those that copy the same block side by side.
struct ForkPlan {
  int n = 0, groups = 0;
  int source[kCacheReqs], target[kCacheReqs], len[kCacheReqs], fresh[kCacheReqs];
  int first[kCacheReqs + 1];  // of each group; forks from first[groups] on copy nothing
};

inline spr_status plan_fork(const spr_pages* p, int n, const int32_t* source, const int32_t* target, const int32_t* lens,
                            const int32_t* fresh, ForkPlan* f, std::string* err) {
  const auto bad = [&](const char* m) {
    *err = std::string("cache_fork: ") + m;
    return SPR_ERR_INVALID_ARG;
  };
  if (source == nullptr || target == nullptr || lens == nullptr || fresh == nullptr)
    return bad("source, target, lens and fresh must not be null");
  if (n < 1 || n > kCacheReqs) return bad("n must be in [1, SPR_MAX_CACHE_REQUESTS]");
  const int64_t most = static_cast<int64_t>(p->max_blocks) * spr::kKvBlock;
  int order[kCacheReqs], ids[kCacheReqs], copies = 0;
  for (int i = 0; i < n; ++i) {
    if (source[i] < 0 || source[i] >= p->n_slots || target[i] < 0 || target[i] >= p->n_slots) return bad("slot id out of range");
    if (lens[i] < 0 || lens[i] > most) return bad("lens must be in [0, 16 * max_blocks]");
    order[i] = i;
    if (lens[i] % spr::kKvBlock == 0) continue;
    if (fresh[i] < 0 || fresh[i] >= p->n_blocks) return bad("fresh block out of range");
    ids[copies++] = fresh[i];
  }
  if (first_repeat(target, n) >= 0) return bad("target listed twice");
  if (first_repeat(ids, copies) >= 0) return bad("fresh block listed twice");
  std::vector<int32_t> t(target, target + n);
  std::sort(t.begin(), t.end());
  for (int i = 0; i < n; ++i)
    if (std::binary_search(t.begin(), t.end(), source[i])) return bad("a target is also a source");
  // Sorted by source and block; forks that copy nothing at the end.
  const auto key = [&](int i) {
    return lens[i] % spr::kKvBlock == 0 ? INT64_MAX : (static_cast<int64_t>(source[i]) << 32) + lens[i] / spr::kKvBlock;
  };
  std::stable_sort(order, order + n, [&](int a, int b) { return key(a) < key(b); });
  f->n = n;
  f->groups = 0;
  for (int k = 0; k < n; ++k) {
    const int i = order[k];
    if (k < copies && (k == 0 || key(i) != key(order[k - 1]))) f->first[f->groups++] = k;
    f->source[k] = source[i];
    f->target[k] = target[i];
    f->len[k] = lens[i];
    f->fresh[k] = lens[i] % spr::kKvBlock == 0 ? -1 : fresh[i];
  }
  f->first[f->groups] = copies;
  if (n + f->groups * page_items(*p, kForkDeep) > kMostGroups) return bad("the blocks are too large for one call");
  return SPR_OK;
}

// The moves of one call in ascending order of src.
inline spr_status plan_move(const spr_pages* p, int n, const int32_t* src, const int32_t* dst,
                            std::vector<std::pair<int32_t, int32_t>>* moves, std::string* err) {
  const auto bad = [&](const char* m) {
    *err = std::string("cache_move: ") + m;
    return SPR_ERR_INVALID_ARG;
  };
  if (src == nullptr || dst == nullptr) return bad("src and dst must not be null");
  if (n < 1 || n > p->n_blocks) return bad("n must be in [1, n_blocks]");
  if (table_groups(*p) + std::min(n, kMoves) * page_items(*p, kMoveDeep) > kMostGroups)
    return bad("the blocks or the table are too large for one call");
  moves->resize(n);
  std::vector<int32_t> d(dst, dst + n);
  for (int i = 0; i < n; ++i) {
    if (src[i] < 0 || src[i] >= p->n_blocks || dst[i] < 0 || dst[i] >= p->n_blocks) return bad("block out of range");
    (*moves)[i] = {src[i], dst[i]};
  }
  std::sort(moves->begin(), moves->end());
  std::sort(d.begin(), d.end());
  for (int i = 1; i < n; ++i) {
    if ((*moves)[i].first == (*moves)[i - 1].first) return bad("src listed twice");
    if (d[i] == d[i - 1]) return bad("dst listed twice");
  }
  for (int i = 0; i < n; ++i)
    if (std::binary_search(d.begin(), d.end(), (*moves)[i].first)) return bad("a dst is also a src");
  return SPR_OK;
}

// Columns that one attention work-group takes: up to 32, whose four waves share
// out the blocks, or 64 or 128 (no more than `most`), whose waves share out the
// columns.  More columns read the cache less often; fewer make more work-groups
// of shorter steps, which counts as long as a CU gets no more than two of 32 or
// one of 128.  On 256 CUs, 32 heads, bf16, in us with 32 / 64 / 128 columns:
//   1 x 512 rows at position 0    11 / 22 / 27     16 x 64 rows at position 500   34 / 27 / 26
//   1 x 256 rows at 2000          28 / 33 / 40      1 x 1024 rows at 500          41 / 37 / 50
//   1 x 512 rows at 8000         109 / 113 / 113    1 x 2048 rows at 2000        175 / 164 / 121
// (over 264 shapes of 0 to 8000 positions 0.6% behind the best of the three on
// average, with the widest that fit 22%; fp32, which has no 128, 0.7% and 16%.)
inline int cache_cols_per_group(const CacheInfo& t, int G, int Hkv, int n_cu, int most) {
  const int64_t cols = static_cast<int64_t>(t.max_rows) * G, all = static_cast<int64_t>(t.rows) * G * Hkv;
  if (cols <= 16) return 16;
  if (cols <= 32 || all <= int64_t{64} * n_cu) return 32;
  return cols <= 64 || all <= int64_t{128} * n_cu ? 64 : most;
}

// Work items of one attention launch: per request its column groups, each in
// KV splits of bps blocks (a group whose rows end early has fewer; the items
// behind them find nothing to do).
struct CacheSplit {
  int bps = 1, groups = 0;
  bool split = false;  // some request has several splits
  int order[kCacheReqs], ncg[kCacheReqs], cg0[kCacheReqs];
  int item0[kCacheReqs + 1];
};

constexpr int kCacheSplits = 64;

// Splits hold `least` blocks (a step of every wave that walks blocks) until
// the launch has more than `slots` resident work-groups take at once; they
// grow further while the partials exceed `floats` or a request has more than
// kCacheSplits.  No splits where the column groups alone are as many, unless one
// request is far longer than a slot's share (32 requests of 32 heads, 80 to 1450
// positions: 21.5 us, with splits 22.5; one of 20000 among them would alone take
// that many steps), nor where there are more of them than `counters`.
inline CacheSplit cache_split(const CacheInfo& t, int G, int Hkv, int hd, int cw, int least, int slots, size_t floats,
                              int counters) {
  CacheSplit s;
  const auto blocks_of = [&](int i) { return (static_cast<int64_t>(t.len[i]) + t.n_rows[i] + 15) / 16; };
  for (int i = 0; i < t.n; ++i) s.order[i] = i;
  std::stable_sort(s.order, s.order + t.n, [&](int i, int j) { return blocks_of(i) > blocks_of(j); });
  int64_t blocks = 0, cg = 0;
  for (int r = 0; r < t.n; ++r) {
    const int i = s.order[r];
    s.ncg[r] = static_cast<int>((static_cast<int64_t>(t.n_rows[i]) * G + cw - 1) / cw);
    s.cg0[r] = static_cast<int>(cg);
    cg += s.ncg[r];
    blocks += s.ncg[r] * blocks_of(i);
  }
  s.groups = static_cast<int>(cg);
  const int64_t per = static_cast<int64_t>(Hkv) * cw * (hd + 4);
  const int64_t share = std::max<int64_t>(1, (blocks * Hkv + slots - 1) / slots), longest = blocks_of(s.order[0]);
  const bool whole = cg * Hkv > counters || (cg * Hkv >= slots && longest <= 4 * share);
  int64_t bps = whole ? longest : share;
  // Rounding every request up to whole splits can leave more work-groups than
  // stay resident; splits up to twice as long that fit them into one round are
  // taken, but not longer ones.
  const auto items_at = [&](int64_t w) {
    int64_t n = 0;
    for (int r = 0; r < t.n; ++r) n += (blocks_of(s.order[r]) + w - 1) / w * s.ncg[r];
    return n;
  };
  for (int k = 0; k <= 8 && !whole; ++k) {
    const int64_t w = (bps + bps * k / 8 + least - 1) / least * least;
    if (items_at(w) * Hkv <= slots) {
      bps = w;
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
    s.split = most > 1;
    if (!s.split || (most <= kCacheSplits && items * per <= static_cast<int64_t>(floats))) break;
  }
  s.bps = static_cast<int>(bps);
  return s;
}

}  // namespace sprk
