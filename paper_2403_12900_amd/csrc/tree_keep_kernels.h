// Compaction of the cache onto the accepted path: node path[k] of a request
// moves from position len + path[k] to len + k, for every layer.
//
// A path's nodes ascend, so path[k] >= k, and a move never writes a position
// that a later one reads (its target k is below every later source).  Each
// thread owns one column of the cache -- a 16-byte piece of a key, or one
// dimension of a value, which the value tiles hold position by position -- and
// takes it along the whole path in ascending order, so moves need no order
// between threads.
#pragma once

#include "tree_attn_kernels.h"

namespace sprk {

struct TreeKeepArgs {
  char* k;
  char* v;
  const int32_t* bt;
  const int32_t* path;
  const int32_t* count;
  int* err;
  size_t layer_bytes;
  int Hkv, hd, mb, nb;
  int slot[kTreeReqs], len[kTreeReqs];
  uint8_t row0[kTreeReqs], nodes[kTreeReqs];
};

constexpr int kKeepBatch = 8;  // moves in flight per thread

// Grid (column groups of 256, layers, requests).
template <class KP>
__global__ __launch_bounds__(256) void k_tree_keep(TreeKeepArgs a) {
  using E = typename KP::elem;
  const int i = blockIdx.z, layer = blockIdx.y, row0 = a.row0[i], nn = a.nodes[i], len = a.len[i];
  const int lane = threadIdx.x & 63;
  const int count = a.count[i];
  if (count < 1) return;
  // The path, one node per lane, checked as a whole; block of each node.
  __shared__ int node_s[kTreeNodes], src_s[kTreeNodes], dst_s[kTreeNodes];
  const int steps = min(count, nn);
  const int node = lane < steps ? a.path[row0 + lane] : 0;
  const int before = __shfl_up(node, 1);
  bool bad = count > nn;
  bad |= lane < steps && (node < lane || node >= nn || (lane > 0 && node <= before));
  int from = 0, to = 0;
  if (lane < steps && !bad) {
    const int32_t* btrow = a.bt + static_cast<size_t>(a.slot[i]) * a.mb;
    from = btrow[(len + node) >> 4];
    to = btrow[(len + lane) >> 4];
    bad |= static_cast<unsigned>(from) >= static_cast<unsigned>(a.nb) || static_cast<unsigned>(to) >= static_cast<unsigned>(a.nb);
  }
  if (__ballot(bad) != 0) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && layer == 0) raise_check(a.err, kErrPath);
    return;
  }
  const uint64_t moved = __ballot(lane < steps && node != lane);
  if (moved == 0) return;
  if (threadIdx.x < 64) {
    node_s[lane] = node;
    src_s[lane] = from;
    dst_s[lane] = to;
  }
  __syncthreads();
  const int first = __ffsll(static_cast<unsigned long long>(moved)) - 1;  // from there on every node moves
  const int pieces = a.hd / KP::per16;
  const int item = blockIdx.x * 256 + threadIdx.x;
  const size_t tile = static_cast<size_t>(16) * a.hd;
  if (item < a.Hkv * a.hd) {
    E* v = reinterpret_cast<E*>(a.v + layer * a.layer_bytes);
    const int kvh = item / a.hd, dd = item - kvh * a.hd;
    for (int s0 = first; s0 < steps; s0 += kKeepBatch) {
      E x[kKeepBatch];
#pragma unroll
      for (int b = 0; b < kKeepBatch; ++b) {
        const int s = min(s0 + b, steps - 1);
        x[b] = v[(static_cast<size_t>(src_s[s]) * a.Hkv + kvh) * tile + vtile_offset<KP>((len + node_s[s]) & 15, dd)];
      }
#pragma unroll
      for (int b = 0; b < kKeepBatch; ++b) {
        const int s = s0 + b;
        if (s < steps) v[(static_cast<size_t>(dst_s[s]) * a.Hkv + kvh) * tile + vtile_offset<KP>((len + s) & 15, dd)] = x[b];
      }
    }
  } else if (item < a.Hkv * (a.hd + pieces)) {
    E* k = reinterpret_cast<E*>(a.k + layer * a.layer_bytes);
    const int at = item - a.Hkv * a.hd, kvh = at / pieces, dd = (at - kvh * pieces) * KP::per16;
    for (int s0 = first; s0 < steps; s0 += kKeepBatch) {
      uint4 x[kKeepBatch];
#pragma unroll
      for (int b = 0; b < kKeepBatch; ++b) {
        const int s = min(s0 + b, steps - 1);
        x[b] = *reinterpret_cast<const uint4*>(
            k + (static_cast<size_t>(src_s[s]) * a.Hkv + kvh) * tile + ktile_offset<KP>((len + node_s[s]) & 15, dd));
      }
#pragma unroll
      for (int b = 0; b < kKeepBatch; ++b) {
        const int s = s0 + b;
        if (s < steps)
          *reinterpret_cast<uint4*>(k + (static_cast<size_t>(dst_s[s]) * a.Hkv + kvh) * tile +
                                    ktile_offset<KP>((len + s) & 15, dd)) = x[b];
      }
    }
  }
}

}  // namespace sprk
