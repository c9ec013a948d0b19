// Launches of the 4-bit cache's operators (cache.hip, cache_attn.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "cache_rule.h"

namespace sprk {

struct CacheAttnCall {
  hipStream_t st;
  const CacheInfo* batch;
  spr_kv4_view kv;
  int layer, H;
  bool bf16;
  const void* q;
  int64_t qs;
  void* out;
  int64_t os;
  float* part;
  size_t part_floats;
  int32_t* cnt;
  int n_cnt;
  int* err;
  int n_cu;
};
hipError_t launch_cache_attention(const CacheAttnCall& c);

}  // namespace sprk
