// C ABI of the 4-bit cache's operators: argument checks and the launches of
// all but attention (cache_attn.hip).
#include <cstring>
#include <string>

#include "cache_launch.h"
#include "cache_pages_kernels.h"
#include "cache_rows_kernels.h"
#include "op_handle.h"
#include "tree_rule.h"

using namespace sprk;

struct spr_cache_ops : OpHandle {};

namespace {

using spr::set_error;

// A tensor of rows: `what` names it in the message.
bool rows_ok(const void* p, int64_t stride, int64_t width, int size) {
  return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride >= width && stride <= (int64_t{1} << 40) &&
         stride * size % 16 == 0;
}

bool overlap(const void* a, int64_t as, const void* b, int64_t bs, int64_t width, int size, int rows) {
  const char *pa = static_cast<const char*>(a), *pb = static_cast<const char*>(b);
  if (pa + ((rows - 1) * as + width) * size <= pb || pb + ((rows - 1) * bs + width) * size <= pa) return false;
  return rows_overlap(reinterpret_cast<uintptr_t>(a), as * size, reinterpret_cast<uintptr_t>(b), bs * size, width * size,
                      rows);
}

int size_of(int dtype) { return dtype == SPR_F32 ? 4 : 2; }

// Heads of a work-group: as many as leave the chip `groups` of them, in whole
// rounds of its threads.
int heads_per_group(int tiles, int heads, int at_once, int groups) {
  int per = at_once;
  while (per < heads && static_cast<int64_t>(tiles) * ((heads + 2 * per - 1) / (2 * per)) >= groups) per *= 2;
  return per;
}

// What append and read have in common.
spr_status rows_call(spr_cache_ops* o, const char* what, const spr_kv4_view* kv, int layer, const spr_cache_batch* batch,
                     const spr_rotary* rotary, int dtype, const void* k, int64_t ks, const void* v, int64_t vs, bool append) {
  spr_status s = check_handle(o);
  if (s != SPR_OK) return s;
  std::string err;
  const std::string w = what;
  if ((s = check_kv4_view(kv, layer, what, &err)) != SPR_OK) return set_error(s, err);
  CacheInfo t;
  if ((s = parse_cache(batch, kv->n_slots, kv->max_blocks, what, &t, &err)) != SPR_OK) return set_error(s, err);
  if (dtype != SPR_F32 && dtype != SPR_BF16) return set_error(SPR_ERR_INVALID_ARG, w + ": unknown dtype");
  const int64_t width = static_cast<int64_t>(kv->n_kv_heads) * kv->head_dim;
  const int size = size_of(dtype);
  if (!rows_ok(k, ks, width, size) || !rows_ok(v, vs, width, size))
    return set_error(SPR_ERR_INVALID_ARG,
                     w + ": k and v must be 16-byte aligned, with strides >= n_kv_heads * head_dim and a multiple of 16 bytes");
  if (!append && overlap(k, ks, v, vs, width, size, t.rows)) return set_error(SPR_ERR_INVALID_ARG, w + ": k and v must not overlap");
  if (rotary != nullptr && (s = check_rotary(rotary, kv->head_dim, what, &err)) != SPR_OK) return set_error(s, err);
  DeviceGuard dev(o->dev);
  if (dev.e != hipSuccess) return hip_failed(o, what, dev.e);
  CacheRowsArgs a{};
  a.bt = kv->block_table;
  a.pool = static_cast<uint8_t*>(kv->data) +
           static_cast<size_t>(layer) * kv->n_blocks * kv->n_kv_heads * 17 * kv->head_dim;
  a.err = o->err_dev;
  a.k = k;
  a.v = v;
  a.ks = ks;
  a.vs = vs;
  a.n = t.n;
  a.Hkv = kv->n_kv_heads;
  a.mb = kv->max_blocks;
  a.nb = kv->n_blocks;
  if (rotary != nullptr) {
    a.turned = 1;
    a.r = rotary_args(*rotary);
  }
  const bool single = t.max_rows == 1;
  int tiles = 0;
  for (int i = 0; i < t.n; ++i) {
    a.slot[i] = t.slot[i];
    a.len[i] = t.len[i];
    a.rows[i] = t.n_rows[i];
    a.row0[i] = t.row0[i];
    a.tile0[i] = tiles;
    tiles += single ? 1 : (t.len[i] + t.n_rows[i] - 1) / 16 - t.len[i] / 16 + 1;
  }
  a.tile0[t.n] = tiles;
  const int at_once = (single ? 16 : 1) * (128 / kv->head_dim);
  // Appending, a work-group's sines serve all its heads (5600 rows of 8 heads: 14.5
  // us with 2 work-groups a CU, with 8 of them 18); reading has no such table.
  a.per = heads_per_group(tiles, a.Hkv, at_once, (append ? 2 : 8) * o->n_cu);
  const dim3 grid(tiles, (a.Hkv + a.per - 1) / a.per);
  const auto launch = [&](auto n, auto hd, auto rg) {
    constexpr int N = decltype(n)::value, HD = decltype(hd)::value, RG = decltype(rg)::value;
    static_assert(kRowHeads<RG, HD> == (RG == 1 ? 16 : 1) * (128 / HD), "at_once");
    if (append) k_cache_append<N, HD, RG><<<grid, 256, 0, o->st>>>(a);
    else k_cache_read<N, HD, RG><<<grid, 256, 0, o->st>>>(a);
  };
  const auto run = [&](auto n, auto hd) {
    if (single) launch(n, hd, std::integral_constant<int, 1>{});
    else launch(n, hd, std::integral_constant<int, kRowsOfBlock>{});
  };
  using std::integral_constant;
  if (kv->head_dim == 128) {
    if (dtype == SPR_F32) run(integral_constant<int, 4>{}, integral_constant<int, 128>{});
    else run(integral_constant<int, 8>{}, integral_constant<int, 128>{});
  } else {
    if (dtype == SPR_F32) run(integral_constant<int, 4>{}, integral_constant<int, 64>{});
    else run(integral_constant<int, 8>{}, integral_constant<int, 64>{});
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SPR_OK : hip_failed(o, what, e);
}

// What a launch has to know of the pools; deep: 16-byte pieces of a thread.
PageCopy page_copy(const spr_pages& p, int deep) {
  PageCopy c{};
  c.pool[0] = static_cast<char*>(p.k);
  c.pool[1] = static_cast<char*>(p.v);
  c.pools = p.v != nullptr ? 2 : 1;
  c.layers = p.n_layers;
  c.pieces = static_cast<int>(p.block_bytes / 16);
  c.chunks = (c.pieces + 256 * deep - 1) / (256 * deep);
  c.chunk = (c.pieces + c.chunks - 1) / c.chunks;
  c.block_bytes = p.block_bytes;
  c.layer_bytes = p.block_bytes * p.n_blocks;
  return c;
}

}  // namespace

extern "C" {

spr_status spr_rotary_init(int32_t dims, int32_t pairs, double base, double factor, double original, double low,
                           double high, double amplitude, spr_rotary* out) {
  return guarded([&]() -> spr_status {
    std::string err;
    const spr_status s = make_rotary(dims, pairs, base, factor, original, low, high, amplitude, out, &err);
    return s == SPR_OK ? SPR_OK : set_error(s, err);
  });
}

size_t spr_cache_ops_workspace_bytes(void) { return kOpWorkspaceBytes; }

spr_status spr_cache_ops_init(void* dev_ws, size_t ws_bytes, void* hip_stream, spr_cache_ops** out) {
  return init_handle("cache_ops_init", dev_ws, ws_bytes, hip_stream, out);
}

spr_status spr_cache_ops_set_stream(spr_cache_ops* o, void* hip_stream) {
  if (o == nullptr) return bad_arg("cache_ops_set_stream: handle is null");
  o->st = static_cast<hipStream_t>(hip_stream);
  return SPR_OK;
}

spr_status spr_cache_ops_release(spr_cache_ops* o) {
  if (o == nullptr) return bad_arg("cache_ops_release: handle is null");
  delete o;
  return SPR_OK;
}

spr_status spr_cache_rotary(spr_cache_ops* o, const spr_rotary* rotary, int32_t rows, int32_t n_heads, int32_t head_dim,
                            int32_t dtype, const int32_t* positions, const void* x, int64_t x_stride, void* out,
                            int64_t out_stride) {
  return guarded([&]() -> spr_status {
    spr_status s = check_handle(o);
    if (s != SPR_OK) return s;
    std::string err;
    if (rows < 1 || rows > kCacheMaxRows) return bad_arg("cache_rotary: rows must be in [1, SPR_MAX_CACHE_ROWS]");
    if (rotary == nullptr || positions == nullptr) return bad_arg("cache_rotary: rotary and positions must not be null");
    if (n_heads < 1 || n_heads > 8192) return bad_arg("cache_rotary: n_heads must be in [1, 8192]");
    if (head_dim != 64 && head_dim != 128) return bad_arg("cache_rotary: head_dim must be 64 or 128");
    if (dtype != SPR_F32 && dtype != SPR_BF16) return bad_arg("cache_rotary: unknown dtype");
    if ((s = check_rotary(rotary, head_dim, "cache_rotary", &err)) != SPR_OK) return set_error(s, err);
    const int64_t width = static_cast<int64_t>(n_heads) * head_dim;
    const int size = size_of(dtype);
    if (!rows_ok(x, x_stride, width, size) || !rows_ok(out, out_stride, width, size))
      return bad_arg("cache_rotary: x and out must be 16-byte aligned, with strides >= n_heads * head_dim and a multiple of 16 bytes");
    if (!(x == out && (x_stride == out_stride || rows == 1)) && overlap(x, x_stride, out, out_stride, width, size, rows))
      return bad_arg("cache_rotary: out must be x itself or not overlap it");
    DeviceGuard dev(o->dev);
    if (dev.e != hipSuccess) return hip_failed(o, "cache_rotary", dev.e);
    RotaryCall a{};
    a.r = rotary_args(*rotary);
    a.positions = positions;
    a.x = x;
    a.out = out;
    a.xs = x_stride;
    a.os = out_stride;
    a.heads = n_heads;
    const int at_once = 256 / (head_dim * size / 16);
    a.per = heads_per_group(rows, n_heads, at_once, 8 * o->n_cu);
    const dim3 grid(rows, (n_heads + a.per - 1) / a.per);
    if (head_dim == 128) {
      if (dtype == SPR_F32) k_rotary<4, 128><<<grid, 256, 0, o->st>>>(a);
      else k_rotary<8, 128><<<grid, 256, 0, o->st>>>(a);
    } else {
      if (dtype == SPR_F32) k_rotary<4, 64><<<grid, 256, 0, o->st>>>(a);
      else k_rotary<8, 64><<<grid, 256, 0, o->st>>>(a);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SPR_OK : hip_failed(o, "cache_rotary", e);
  });
}

spr_status spr_cache_append(spr_cache_ops* o, const spr_kv4_view* kv, int32_t layer, const spr_cache_batch* batch,
                            const spr_rotary* rotary, int32_t dtype, const void* k, int64_t k_stride, const void* v,
                            int64_t v_stride) {
  return guarded([&] { return rows_call(o, "cache_append", kv, layer, batch, rotary, dtype, k, k_stride, v, v_stride, true); });
}

spr_status spr_cache_read(spr_cache_ops* o, const spr_kv4_view* kv, int32_t layer, const spr_cache_batch* batch,
                          int32_t dtype, void* k, int64_t k_stride, void* v, int64_t v_stride) {
  return guarded([&] { return rows_call(o, "cache_read", kv, layer, batch, nullptr, dtype, k, k_stride, v, v_stride, false); });
}

spr_status spr_cache_attention(spr_cache_ops* o, const spr_kv4_view* kv, int32_t layer, const spr_cache_batch* batch,
                               int32_t n_heads, int32_t dtype, const void* q, int64_t q_stride, void* out,
                               int64_t out_stride) {
  return guarded([&]() -> spr_status {
    spr_status s = check_handle(o);
    if (s != SPR_OK) return s;
    std::string err;
    if ((s = check_kv4_view(kv, layer, "cache_attention", &err)) != SPR_OK) return set_error(s, err);
    CacheInfo t;
    if ((s = parse_cache(batch, kv->n_slots, kv->max_blocks, "cache_attention", &t, &err)) != SPR_OK) return set_error(s, err);
    if (n_heads < 1 || n_heads % kv->n_kv_heads != 0 || n_heads / kv->n_kv_heads > 16)
      return bad_arg("cache_attention: n_heads must be a multiple of n_kv_heads, at most 16 times it");
    if (dtype != SPR_F32 && dtype != SPR_BF16) return bad_arg("cache_attention: unknown dtype");
    const int64_t width = static_cast<int64_t>(n_heads) * kv->head_dim;
    const int size = size_of(dtype);
    if (!rows_ok(q, q_stride, width, size) || !rows_ok(out, out_stride, width, size))
      return bad_arg("cache_attention: q and out must be 16-byte aligned, with strides >= n_heads * head_dim and a multiple of 16 bytes");
    if (overlap(q, q_stride, out, out_stride, width, size, t.rows)) return bad_arg("cache_attention: out must not overlap q");
    DeviceGuard dev(o->dev);
    if (dev.e != hipSuccess) return hip_failed(o, "cache_attention", dev.e);
    CacheAttnCall c{};
    c.st = o->st;
    c.batch = &t;
    c.kv = *kv;
    c.layer = layer;
    c.H = n_heads;
    c.bf16 = dtype == SPR_BF16;
    c.q = q;
    c.qs = q_stride;
    c.out = out;
    c.os = out_stride;
    c.part = o->part();
    c.part_floats = kOpPartBytes / sizeof(float);
    c.cnt = o->counters();
    c.n_cnt = kOpCounters;
    c.err = o->err_dev;
    c.n_cu = o->n_cu;
    const hipError_t e = launch_cache_attention(c);
    return e == hipSuccess ? SPR_OK : hip_failed(o, "cache_attention", e);
  });
}

spr_status spr_cache_fork(spr_cache_ops* o, const spr_pages* pages, int32_t n, const int32_t* source,
                          const int32_t* target, const int32_t* lens, const int32_t* fresh) {
  return guarded([&]() -> spr_status {
    spr_status s = check_handle(o);
    if (s != SPR_OK) return s;
    std::string err;
    if ((s = check_pages(pages, "cache_fork", &err)) != SPR_OK) return set_error(s, err);
    ForkPlan f;
    if ((s = plan_fork(pages, n, source, target, lens, fresh, &f, &err)) != SPR_OK) return set_error(s, err);
    DeviceGuard dev(o->dev);
    if (dev.e != hipSuccess) return hip_failed(o, "cache_fork", dev.e);
    ForkArgs a{};
    a.c = page_copy(*pages, kForkDeep);
    a.bt = pages->block_table;
    a.err = o->err_dev;
    a.mb = pages->max_blocks;
    a.nb = pages->n_blocks;
    a.n = f.n;
    a.groups = f.groups;
    std::memcpy(a.source, f.source, sizeof(int) * f.n);
    std::memcpy(a.target, f.target, sizeof(int) * f.n);
    std::memcpy(a.len, f.len, sizeof(int) * f.n);
    std::fill(std::copy(f.fresh, f.fresh + f.n, a.fresh), a.fresh + kCacheReqs, -1);
    for (int g = 0; g <= f.groups; ++g) a.first[g] = static_cast<uint8_t>(f.first[g]);
    for (int g = 0; g < f.groups; ++g)
      a.part[g] = static_cast<int64_t>(f.source[f.first[g]]) * a.mb + f.len[f.first[g]] / spr::kKvBlock;
    k_cache_fork<<<static_cast<unsigned>(f.n + f.groups * page_items(*pages, kForkDeep)), 256, 0, o->st>>>(a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SPR_OK : hip_failed(o, "cache_fork", e);
  });
}

spr_status spr_cache_move(spr_cache_ops* o, const spr_pages* pages, int32_t n, const int32_t* src, const int32_t* dst) {
  return guarded([&]() -> spr_status {
    spr_status s = check_handle(o);
    if (s != SPR_OK) return s;
    std::string err;
    if ((s = check_pages(pages, "cache_move", &err)) != SPR_OK) return set_error(s, err);
    std::vector<std::pair<int32_t, int32_t>> moves;
    if ((s = plan_move(pages, n, src, dst, &moves, &err)) != SPR_OK) return set_error(s, err);
    MoveArgs a{};
    a.c = page_copy(*pages, kMoveDeep);
    a.bt = pages->block_table;
    a.entries = static_cast<int64_t>(pages->n_slots) * pages->max_blocks;
    const int64_t items = page_items(*pages, kMoveDeep), groups = table_groups(*pages);
    a.table_groups = static_cast<int>(groups);
    DeviceGuard dev(o->dev);
    if (dev.e != hipSuccess) return hip_failed(o, "cache_move", dev.e);
    for (int i = 0; i < n; i += kMoves) {
      a.n = std::min(n - i, kMoves);
      for (int k = 0; k < a.n; ++k) {
        a.src[k] = moves[i + k].first;
        a.dst[k] = moves[i + k].second;
      }
      k_cache_move<<<static_cast<unsigned>(groups + a.n * items), 256, 0, o->st>>>(a);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return hip_failed(o, "cache_move", e);
    }
    return SPR_OK;
  });
}

}  // extern "C"
