// Compaction of the cache onto the accepted path: node path[k] of a request
// moves from position len + path[k] to len + k, for every layer.
//
// A path's nodes ascend, so path[k] >= k, and a move never writes a position
// that a later one reads (its target k is below every later source).  Each
// thread owns one column of the cache -- a 16-byte piece of a key, or one
// dimension of a value, which the value tiles hold position by position -- and
// takes it along the whole path in ascending order, so moves need no order
// between threads.
//
// Bound by lines of memory that it touches in part: a position is 16 bytes of
// every 256 of the keys and 2 (bf16) or 4 bytes of every 8 or 16 of the values,
// as the attention kernels read them.  40 heads, 40 layers, 16 requests: 22 us
// for 20 MB of moved bytes (the counters show twice as much written and more
// read: about 66 MB, which alone would take 12); 8 heads in fp32, 80 layers, 16
// requests: 18 us.  The number of work-groups does not matter from 1000 of them
// (several layers each) to 14720 (one).  One request, 32 layers: 4.2 us.
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
  size_t layer_elems;
  int Hkv, hd, mb, nb;
  int slot[kTreeReqs], len[kTreeReqs];
  uint8_t row0[kTreeReqs], nodes[kTreeReqs];
};

constexpr int kKeepBatch = 8;  // moves in flight per thread

// Piece of 16 bytes of a key, or one element of a value.
template <class KP, bool kKey>
struct KeepItem {
  using type = typename KP::elem;
  static __device__ __forceinline__ int offset(int t, int dd) { return vtile_offset<KP>(t, dd); }
};
template <class KP>
struct KeepItem<KP, true> {
  using type = u32x4_t;
  static __device__ __forceinline__ int offset(int t, int dd) { return ktile_offset<KP>(t, dd); }
};

// Moves of one column (head kvh, dimension dd) of a layer, in path order,
// kKeepBatch at a time: all of a batch's loads come before its stores, and no
// store of a batch or an earlier one writes a later source.
template <class KP, bool kKey>
__device__ __forceinline__ void keep_column(typename KP::elem* layer, int Hkv, int hd, int kvh, int dd, int len, int first,
                                            int steps, const int* node, const int* from, const int* to) {
  using Item = KeepItem<KP, kKey>;
  using T = typename Item::type;
  const size_t tile = static_cast<size_t>(16) * hd;
  const auto at = [&](int block, int pos) {
    return reinterpret_cast<T*>(layer + (static_cast<size_t>(block) * Hkv + kvh) * tile + Item::offset(pos & 15, dd));
  };
  for (int s = first; s < steps; s += kKeepBatch) {
    T x[kKeepBatch];
#pragma unroll
    for (int b = 0; b < kKeepBatch; ++b)
      if (s + b < steps) x[b] = *at(from[s + b], len + node[s + b]);
#pragma unroll
    for (int b = 0; b < kKeepBatch; ++b)
      if (s + b < steps) *at(to[s + b], len + s + b) = x[b];
  }
}

// Grid (column groups of 256, layers, requests).
template <class KP>
__global__ __launch_bounds__(256) void k_tree_keep(TreeKeepArgs a) {
  using E = typename KP::elem;
  const int i = blockIdx.z, row0 = a.row0[i], nn = a.nodes[i], len = a.len[i];
  const int lane = threadIdx.x & 63;
  // The path, one node per lane, checked as a whole; blocks of every node.
  __shared__ int node_s[kTreeNodes], src_s[kTreeNodes], dst_s[kTreeNodes];
  const int32_t* btrow = a.bt + static_cast<size_t>(a.slot[i]) * a.mb;
  const int node = lane < nn ? a.path[row0 + lane] : 0;
  const int to = lane < nn ? btrow[(len + lane) >> 4] : 0;  // block of node `lane`, and of path position `lane`
  const int count = a.count[i];
  if (count < 1) return;
  const int steps = min(count, nn);
  const int before = __shfl_up(node, 1);
  bool bad = count > nn;
  bad |= lane < steps && (node < lane || node >= nn || (lane > 0 && node <= before));
  const uint64_t moved = __ballot(lane < steps && node != lane);
  const int from = __shfl(to, node & 63);
  bool lost = lane < steps && node != lane &&
              (static_cast<unsigned>(from) >= static_cast<unsigned>(a.nb) || static_cast<unsigned>(to) >= static_cast<unsigned>(a.nb));
  const uint64_t bads = __ballot(bad), losts = __ballot(lost);
  if ((bads | losts) != 0) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) raise_check(a.err, bads != 0 ? kErrPath : kErrBlockId);
    return;
  }
  if (moved == 0) return;
  if (threadIdx.x < 64) {
    node_s[lane] = node;
    src_s[lane] = from;
    dst_s[lane] = to;
  }
  __syncthreads();
  const int first = __ffsll(static_cast<unsigned long long>(moved)) - 1;  // from there on every node moves
  const size_t layer = blockIdx.y * a.layer_elems;
  const int pieces = a.hd / KP::per16;
  const int item = blockIdx.x * 256 + threadIdx.x;
  if (item < a.Hkv * a.hd) {
    const int kvh = item / a.hd;
    keep_column<KP, false>(reinterpret_cast<E*>(a.v) + layer, a.Hkv, a.hd, kvh, item - kvh * a.hd, len, first, steps,
                           node_s, src_s, dst_s);
  } else if (item < a.Hkv * (a.hd + pieces)) {
    const int at = item - a.Hkv * a.hd, kvh = at / pieces;
    keep_column<KP, true>(reinterpret_cast<E*>(a.k) + layer, a.Hkv, a.hd, kvh, (at - kvh * pieces) * KP::per16, len, first,
                          steps, node_s, src_s, dst_s);
  }
}

}  // namespace sprk
