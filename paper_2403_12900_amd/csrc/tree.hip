// C ABI of the drafted-tree operators: the operator handle, argument checks
// and the launches of verification and compaction (attention: tree_attn.hip).
#include <cmath>
#include <exception>
#include <new>
#include <string>

#include "tree_keep_kernels.h"
#include "tree_launch.h"
#include "tree_verify_kernels.h"

using namespace sprk;

// Operator workspace: attention partials (or verification's sums), and
// attention's counters: one per column group and KV head.
constexpr size_t kTreePartBytes = size_t{32} << 20;
constexpr int kTreeCounters = kTreeRows * 512;

struct spr_tree_ops {
  char* ws = nullptr;
  hipStream_t st = nullptr;
  int dev = 0, n_cu = 1;
  spr_status sticky = SPR_OK;
  std::string sticky_msg;
  int* err_host = nullptr;  // device check flag in mapped pinned host memory
  int* err_dev = nullptr;
  ~spr_tree_ops() {
    if (err_host != nullptr) (void)hipHostFree(err_host);
  }
};

namespace sprk {
namespace {

// Requests of a tree step: table row and first token row.
struct TreeRowArgs {
  int n;
  int slot[kTreeReqs], row0[kTreeReqs + 1];
};
TreeRowArgs row_args(const TreeInfo& t) {
  TreeRowArgs a{};
  a.n = t.n;
  for (int i = 0; i < t.n; ++i) {
    a.slot[i] = t.slot[i];
    a.row0[i] = t.row0[i];
  }
  a.row0[t.n] = t.rows;
  return a;
}

// One work-group of a thread per request.
__global__ __launch_bounds__(64) void k_tree_tokens(TreeRowArgs a, const int32_t* tok, const int32_t* tokens,
                                                    int32_t* out) {
  const int i = threadIdx.x;
  if (i >= a.n) return;
  out[a.row0[i]] = tok[a.slot[i]];
  for (int r = a.row0[i] + 1; r < a.row0[i + 1]; ++r) out[r] = tokens[r];
}

__global__ __launch_bounds__(64) void k_tree_last(TreeRowArgs a, const int32_t* emitted, const int32_t* count,
                                                  int32_t* tok) {
  const int i = threadIdx.x;
  if (i >= a.n || count[i] < 1) return;
  tok[a.slot[i]] = emitted[a.row0[i] + count[i] - 1];
}

}  // namespace

int tree_max_vocab() { return kVMaxVocab; }

hipError_t launch_tree_tokens(hipStream_t st, const TreeInfo& t, const int32_t* tok, const int32_t* tokens,
                              int32_t* out) {
  k_tree_tokens<<<1, 64, 0, st>>>(row_args(t), tok, tokens, out);
  return hipGetLastError();
}

hipError_t launch_tree_last(hipStream_t st, const TreeInfo& t, const int32_t* emitted, const int32_t* count,
                            int32_t* tok) {
  k_tree_last<<<1, 64, 0, st>>>(row_args(t), emitted, count, tok);
  return hipGetLastError();
}

size_t tree_verify_bytes(int rows, int V) {
  const size_t S = static_cast<size_t>(V + kVChunk - 1) / kVChunk;
  return rows * S * 16 + rows * S * 8;
}

hipError_t launch_tree_verify(const TreeVerifyCall& c) {
  const TreeInfo& t = *c.tree;
  TreeVerifyArgs a{};
  a.logits = c.logits;
  a.draft = c.draft;
  a.ls = c.ls;
  a.ds = c.ds;
  a.tok = c.tokens;
  a.accept = c.accept;
  a.sample = c.sample;
  a.emitted = c.emitted;
  a.path = c.path;
  a.count = c.count;
  a.err = c.err;
  a.V = c.V;
  a.S = (c.V + kVChunk - 1) / kVChunk;
  a.n = t.n;
  a.rows = t.rows;
  a.stat = static_cast<uint64_t*>(c.scratch);
  a.rest = reinterpret_cast<double*>(a.stat + static_cast<size_t>(t.rows) * a.S * 2);
  const int size = c.bf16 ? 2 : 4;
  const auto aligned = [&](const void* p, int64_t stride) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride * size % 16 == 0;
  };
  a.vec_l = aligned(c.logits, c.ls);
  a.vec_d = c.draft != nullptr && aligned(c.draft, c.ds);
  int arrays = 0, last = 0;
  bool drafted[kTreeReqs];  // children are tested against q
  for (int i = 0; i < t.n; ++i) {
    a.temp[i] = c.temperature != nullptr ? c.temperature[i] : 1.f;
    a.row0[i] = static_cast<uint8_t>(t.row0[i]);
    a.nodes[i] = static_cast<uint8_t>(t.nodes[i]);
    drafted[i] = c.draft != nullptr && a.temp[i] > 0.f;
    if (drafted[i]) last = std::max(last, t.children[i]);
    for (int r = t.row0[i]; r < t.row0[i + 1]; ++r) {
      a.req[r] = static_cast<uint8_t>(i);
      a.kids[r] = t.kids[r];
      a.rank[r] = t.rank[r];
      a.parent[r] = t.parent[r];
      a.parent_row[r] = static_cast<uint8_t>(t.parent[r] < 0 ? kTreeRows : t.row0[i] + t.parent[r]);
      a.rest0[r] = static_cast<uint8_t>(arrays);
      arrays += t.kids[r];
    }
  }
  hipError_t e;
  const dim3 grid(a.S, t.rows);
  if (c.bf16) k_tree_stats<uint16_t><<<grid, kSumThreads, 0, c.st>>>(a);
  else k_tree_stats<float><<<grid, kSumThreads, 0, c.st>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  for (a.k = 1; a.k <= last; ++a.k) {
    int n = 0;
    for (int i = 0; i < t.n; ++i)
      for (int r = t.row0[i]; r < t.row0[i + 1]; ++r)
        if (drafted[i] && t.kids[r] >= a.k) a.list[n++] = static_cast<uint8_t>(r);
    if (c.bf16) k_tree_rest<uint16_t><<<dim3(a.S, n), kSumThreads, 0, c.st>>>(a);
    else k_tree_rest<float><<<dim3(a.S, n), kSumThreads, 0, c.st>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (c.bf16) k_tree_walk<uint16_t><<<t.n, kDrawThreads, 0, c.st>>>(a);
  else k_tree_walk<float><<<t.n, kDrawThreads, 0, c.st>>>(a);
  return hipGetLastError();
}

hipError_t launch_tree_keep(hipStream_t st, const TreeInfo& t, const spr_kv_view& kv, const int32_t* path,
                            const int32_t* count, int* err) {
  TreeKeepArgs a{};
  const bool bf = kv.kv_dtype == SPR_BF16;
  a.k = static_cast<char*>(kv.k);
  a.v = static_cast<char*>(kv.v);
  a.bt = kv.block_table;
  a.path = path;
  a.count = count;
  a.err = err;
  a.layer_elems = static_cast<size_t>(kv.n_blocks) * kv.n_kv_heads * 16 * kv.head_dim;
  a.Hkv = kv.n_kv_heads;
  a.hd = kv.head_dim;
  a.mb = kv.max_blocks;
  a.nb = kv.n_blocks;
  for (int i = 0; i < t.n; ++i) {
    a.slot[i] = t.slot[i];
    a.len[i] = t.len[i];
    a.row0[i] = static_cast<uint8_t>(t.row0[i]);
    a.nodes[i] = static_cast<uint8_t>(t.nodes[i]);
  }
  const int columns = a.Hkv * (a.hd + a.hd / (bf ? 8 : 4));
  const dim3 grid((columns + 255) / 256, kv.n_layers, t.n);
  if (bf) k_tree_keep<BF16><<<grid, 256, 0, st>>>(a);
  else k_tree_keep<F32><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace sprk

namespace {

using spr::set_error;

// Makes the handle's device current for the call.
struct DeviceGuard {
  int before = -1;
  hipError_t e;
  explicit DeviceGuard(int dev) {
    e = hipGetDevice(&before);
    if (e == hipSuccess && before != dev) e = hipSetDevice(dev);
    else before = -1;
  }
  ~DeviceGuard() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

spr_status hip_failed(spr_tree_ops* o, const char* what, hipError_t e) {
  const std::string msg = std::string(what) + ": " + hipGetErrorString(e);
  if (o != nullptr) {
    o->sticky = SPR_ERR_HIP;
    o->sticky_msg = "an earlier HIP error left the handle unusable; release it (" + msg + ")";
  }
  return set_error(SPR_ERR_HIP, msg);
}

spr_status check_ops(spr_tree_ops* o) {
  if (o == nullptr) return set_error(SPR_ERR_INVALID_ARG, "operator handle is null");
  if (o->sticky == SPR_OK) {
    const int bits = *reinterpret_cast<volatile int*>(o->err_host);
    if (bits != 0) {
      o->sticky = SPR_ERR_DEVICE_CHECK;
      o->sticky_msg = "a device check failed on an earlier call:";
      if (bits & kErrTokenRange) o->sticky_msg += " a drafted token outside [0, vocab);";
      if (bits & kErrLogits) o->sticky_msg += " a logits row with a NaN or no finite maximum;";
      if (bits & kErrBlockId) o->sticky_msg += " a block id outside the pool;";
      if (bits & kErrPath) o->sticky_msg += " a malformed path of tree nodes;";
      o->sticky_msg += " release the handle";
    }
  }
  return o->sticky == SPR_OK ? SPR_OK : set_error(o->sticky, o->sticky_msg);
}

// No exception crosses the ABI (a failed host allocation is the only source).
template <class F>
spr_status guarded(F f) {
  try {
    spr::clear_error();
    return f();
  } catch (const std::exception&) {
    return SPR_ERR_HIP;
  }
}

spr_status bad_arg(const char* msg) { return set_error(SPR_ERR_INVALID_ARG, msg); }

}  // namespace

extern "C" {

size_t spr_tree_ops_workspace_bytes(void) { return kTreePartBytes + kTreeCounters * sizeof(int32_t); }

spr_status spr_tree_ops_init(void* dev_ws, size_t ws_bytes, void* hip_stream, spr_tree_ops** out) {
  return guarded([&]() -> spr_status {
    if (out == nullptr) return bad_arg("tree_ops_init: out must not be null");
    *out = nullptr;
    if (dev_ws == nullptr || (reinterpret_cast<uintptr_t>(dev_ws) & 255) != 0)
      return set_error(SPR_ERR_WORKSPACE, "tree_ops_init: workspace must be a non-null, 256-byte aligned device pointer");
    if (ws_bytes < spr_tree_ops_workspace_bytes())
      return set_error(SPR_ERR_WORKSPACE, "tree_ops_init: workspace has " + std::to_string(ws_bytes) + " bytes, " +
                                              std::to_string(spr_tree_ops_workspace_bytes()) + " needed");
    spr_tree_ops* o = new (std::nothrow) spr_tree_ops();
    if (o == nullptr) return SPR_ERR_HIP;
    o->ws = static_cast<char*>(dev_ws);
    o->st = static_cast<hipStream_t>(hip_stream);
    hipError_t e = hipGetDevice(&o->dev);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&o->n_cu, hipDeviceAttributeMultiprocessorCount, o->dev);
    if (e == hipSuccess) e = hipHostMalloc(reinterpret_cast<void**>(&o->err_host), sizeof(int), hipHostMallocMapped);
    if (e == hipSuccess) {
      *o->err_host = 0;
      e = hipHostGetDevicePointer(reinterpret_cast<void**>(&o->err_dev), o->err_host, 0);
    }
    if (e == hipSuccess) e = hipMemsetAsync(o->ws + kTreePartBytes, 0, kTreeCounters * sizeof(int32_t), o->st);
    if (e == hipSuccess) e = hipStreamSynchronize(o->st);
    if (e != hipSuccess) {
      delete o;
      return hip_failed(nullptr, "tree_ops_init", e);
    }
    *out = o;
    return SPR_OK;
  });
}

spr_status spr_tree_ops_set_stream(spr_tree_ops* o, void* hip_stream) {
  if (o == nullptr) return bad_arg("tree_ops_set_stream: handle is null");
  o->st = static_cast<hipStream_t>(hip_stream);
  return SPR_OK;
}

spr_status spr_tree_ops_release(spr_tree_ops* o) {
  if (o == nullptr) return bad_arg("tree_ops_release: handle is null");
  delete o;
  return SPR_OK;
}

spr_status spr_tree_attention(spr_tree_ops* o, const spr_kv_view* kv, int32_t layer, const spr_tree_batch* batch,
                              int32_t n_heads, int32_t io_dtype, const void* q, int64_t q_stride, void* out,
                              int64_t out_stride) {
  return guarded([&]() -> spr_status {
    spr_status s = check_ops(o);
    if (s != SPR_OK) return s;
    std::string err;
    if ((s = check_view(kv, layer, "tree_attention", &err)) != SPR_OK) return set_error(s, err);
    TreeInfo t;
    if ((s = parse_tree(batch, true, kv->n_slots, kv->max_blocks, "tree_attention", &t, &err)) != SPR_OK)
      return set_error(s, err);
    if (n_heads < 1 || n_heads % kv->n_kv_heads != 0 || n_heads / kv->n_kv_heads > 16)
      return bad_arg("tree_attention: n_heads must be a multiple of n_kv_heads, at most 16 times it");
    if (io_dtype != SPR_F32 && io_dtype != SPR_BF16) return bad_arg("tree_attention: unknown io_dtype");
    if (q == nullptr || out == nullptr || ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) != 0)
      return bad_arg("tree_attention: q and out must be non-null and 16-byte aligned");
    const int size = io_dtype == SPR_F32 ? 4 : 2;
    const int64_t width = static_cast<int64_t>(n_heads) * kv->head_dim, most = int64_t{1} << 40;
    if (q_stride < width || out_stride < width || q_stride > most || out_stride > most || q_stride * size % 16 != 0 ||
        out_stride * size % 16 != 0)
      return bad_arg("tree_attention: row strides must be >= n_heads * head_dim and a multiple of 16 bytes");
    if (rows_overlap(reinterpret_cast<uintptr_t>(q), q_stride * size, reinterpret_cast<uintptr_t>(out), out_stride * size,
                     width * size, t.rows))
      return bad_arg("tree_attention: out must not overlap q");
    DeviceGuard dev(o->dev);
    if (dev.e != hipSuccess) return hip_failed(o, "tree_attention", dev.e);
    TreeAttnCall c{};
    c.st = o->st;
    c.tree = &t;
    c.kv = *kv;
    c.layer = layer;
    c.H = n_heads;
    c.io = io_dtype == SPR_F32 ? kTreeF32 : kTreeBF16;
    c.q = q;
    c.qs = q_stride;
    c.out = out;
    c.os = out_stride;
    c.sc = TreeScratch{reinterpret_cast<float*>(o->ws), kTreePartBytes / sizeof(float),
                       reinterpret_cast<int32_t*>(o->ws + kTreePartBytes), kTreeCounters};
    c.err = o->err_dev;
    c.n_cu = o->n_cu;
    const hipError_t e = launch_tree_attention(c);
    return e == hipSuccess ? SPR_OK : hip_failed(o, "tree_attention", e);
  });
}

spr_status spr_tree_verify(spr_tree_ops* o, const spr_tree_batch* batch, int32_t vocab, int32_t dtype,
                           const int32_t* tokens, const void* logits, int64_t logits_stride, const void* draft_probs,
                           int64_t draft_stride, const float* temperature, const float* accept, const float* sample,
                           int32_t* emitted, int32_t* path, int32_t* count) {
  return guarded([&]() -> spr_status {
    spr_status s = check_ops(o);
    if (s != SPR_OK) return s;
    std::string err;
    TreeInfo t;
    if ((s = parse_tree(batch, false, 0, 0, "tree_verify", &t, &err)) != SPR_OK) return set_error(s, err);
    if (vocab < 1 || vocab > kVMaxVocab) return bad_arg("tree_verify: vocab must be in [1, 1048576]");
    if (dtype != SPR_F32 && dtype != SPR_BF16) return bad_arg("tree_verify: unknown dtype");
    if (tokens == nullptr || logits == nullptr || emitted == nullptr || path == nullptr || count == nullptr)
      return bad_arg("tree_verify: tokens, logits, emitted, path and count must not be null");
    const int size = dtype == SPR_F32 ? 4 : 2;
    const int64_t most = int64_t{1} << 40;
    if (logits_stride < vocab || logits_stride > most ||
        (draft_probs != nullptr && (draft_stride < vocab || draft_stride > most)))
      return bad_arg("tree_verify: row strides must be >= vocab");
    if (((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(draft_probs)) & (size - 1)) != 0)
      return bad_arg("tree_verify: logits and draft_probs must be aligned to their elements");
    if ((s = check_temperatures(t.n, temperature, accept, sample, "tree_verify", &err)) != SPR_OK)
      return set_error(s, err);
    DeviceGuard dev(o->dev);
    if (dev.e != hipSuccess) return hip_failed(o, "tree_verify", dev.e);
    TreeVerifyCall c{};
    c.st = o->st;
    c.tree = &t;
    c.V = vocab;
    c.bf16 = dtype == SPR_BF16;
    c.tokens = tokens;
    c.logits = logits;
    c.ls = logits_stride;
    c.draft = draft_probs;
    c.ds = draft_stride;
    c.temperature = temperature;
    c.accept = accept;
    c.sample = sample;
    c.emitted = emitted;
    c.path = path;
    c.count = count;
    c.scratch = o->ws;
    c.err = o->err_dev;
    const hipError_t e = launch_tree_verify(c);
    return e == hipSuccess ? SPR_OK : hip_failed(o, "tree_verify", e);
  });
}

spr_status spr_tree_keep(spr_tree_ops* o, const spr_kv_view* kv, const spr_tree_batch* batch, const int32_t* path,
                         const int32_t* count) {
  return guarded([&]() -> spr_status {
    spr_status s = check_ops(o);
    if (s != SPR_OK) return s;
    std::string err;
    if ((s = check_view(kv, 0, "tree_keep", &err)) != SPR_OK) return set_error(s, err);
    if (kv->n_layers > 65535) return bad_arg("tree_keep: more than 65535 layers");
    TreeInfo t;
    if ((s = parse_tree(batch, true, kv->n_slots, kv->max_blocks, "tree_keep", &t, &err)) != SPR_OK)
      return set_error(s, err);
    if (path == nullptr || count == nullptr) return bad_arg("tree_keep: path and count must not be null");
    DeviceGuard dev(o->dev);
    if (dev.e != hipSuccess) return hip_failed(o, "tree_keep", dev.e);
    const hipError_t e = launch_tree_keep(o->st, t, *kv, path, count, o->err_dev);
    return e == hipSuccess ? SPR_OK : hip_failed(o, "tree_keep", e);
  });
}

}  // extern "C"
