// Launches of the drafted-tree operators (tree.hip, tree_attn.hip), for the C
// ABI's operator handle and for a model's tree step.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "device_common.h"
#include "tree_rule.h"

namespace sprk {

enum TreeIo { kTreeF32 = 0, kTreeBF16 = 1, kTreeActBF16 = 2, kTreeActF32 = 3 };

// Scratch of one launch: partials and counters (zero between launches).
struct TreeScratch {
  float* part;
  size_t part_floats;
  int32_t* cnt;
  int n_cnt;
};

struct TreeAttnCall {
  hipStream_t st;
  const TreeInfo* tree;
  spr_kv_view kv;
  int layer, H, io;
  const void* q;
  int64_t qs;
  void* out;
  int64_t os;
  ActRec rec;
  TreeScratch sc;
  int* err;
  int n_cu;
};
hipError_t launch_tree_attention(const TreeAttnCall& c);

struct TreeVerifyCall {
  hipStream_t st;
  const TreeInfo* tree;
  int V, bf16;
  const int32_t* tokens;
  const void* logits;
  int64_t ls;
  const void* draft;
  int64_t ds;
  const float* temperature;  // host [n] or null
  const float *accept, *sample;
  int32_t *emitted, *path, *count;
  void* scratch;             // tree_verify_bytes, 8-byte aligned
  int* err;
};
size_t tree_verify_bytes(int rows, int V);
hipError_t launch_tree_verify(const TreeVerifyCall& c);

int tree_max_vocab();

// out[row] = the row's input token: tok[slot] for a root, else tokens[row].
hipError_t launch_tree_tokens(hipStream_t st, const TreeInfo& t, const int32_t* tok, const int32_t* tokens,
                              int32_t* out);
// tok[slot] = each request's last emitted token.
hipError_t launch_tree_last(hipStream_t st, const TreeInfo& t, const int32_t* emitted, const int32_t* count,
                            int32_t* tok);

hipError_t launch_tree_keep(hipStream_t st, const TreeInfo& t, const spr_kv_view& kv, const int32_t* path,
                            const int32_t* count, int* err);

}  // namespace sprk

namespace spr {
// The calling thread's last error message (spr_last_error).
spr_status set_error(spr_status s, const std::string& msg);
void clear_error();
}  // namespace spr
