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
  size_t layer_elems;
  int Hkv, hd, mb, nb, n_layers, layers;  // layers: per work-group
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

// Moves of one column (head kvh, dimension dd) for layers [l0, l1), in order
// of (layer, path step), kKeepBatch at a time: all of a batch's loads come
// before its stores, and no store of a batch or an earlier one writes a later
// source.
template <class KP, bool kKey>
__device__ __forceinline__ void keep_column(typename KP::elem* pool, size_t layer_elems, int Hkv, int hd, int kvh, int dd,
                                            int len, int l0, int l1, int first, int steps, const int* node,
                                            const int* from, const int* to) {
  using Item = KeepItem<KP, kKey>;
  using T = typename Item::type;
  const size_t tile = static_cast<size_t>(16) * hd;
  const int per = steps - first, total = (l1 - l0) * per;
  const auto at = [&](int layer, int block, int pos) {
    return reinterpret_cast<T*>(pool + layer * layer_elems + (static_cast<size_t>(block) * Hkv + kvh) * tile +
                                Item::offset(pos & 15, dd));
  };
  int layer = l0, s = first;
  for (int n0 = 0; n0 < total; n0 += kKeepBatch) {
    T x[kKeepBatch];
    int lb = layer, sb = s;
#pragma unroll
    for (int b = 0; b < kKeepBatch; ++b) {
      if (n0 + b < total) {
        x[b] = *at(lb, from[sb], len + node[sb]);
        if (++sb == steps) {
          sb = first;
          ++lb;
        }
      }
    }
#pragma unroll
    for (int b = 0; b < kKeepBatch; ++b) {
      if (n0 + b < total) {
        *at(layer, to[s], len + s) = x[b];
        if (++s == steps) {
          s = first;
          ++layer;
        }
      }
    }
  }
}

// Grid (column groups of 256, layer groups, requests): a work-group takes its
// columns through `layers` layers, so that it finds the path and its blocks
// once for all of them.
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
  const int l0 = blockIdx.y * a.layers, l1 = min(l0 + a.layers, a.n_layers);
  const int pieces = a.hd / KP::per16;
  const int item = blockIdx.x * 256 + threadIdx.x;
  if (item < a.Hkv * a.hd) {
    const int kvh = item / a.hd;
    keep_column<KP, false>(reinterpret_cast<E*>(a.v), a.layer_elems, a.Hkv, a.hd, kvh, item - kvh * a.hd, len, l0, l1,
                           first, steps, node_s, src_s, dst_s);
  } else if (item < a.Hkv * (a.hd + pieces)) {
    const int at = item - a.Hkv * a.hd, kvh = at / pieces;
    keep_column<KP, true>(reinterpret_cast<E*>(a.k), a.layer_elems, a.Hkv, a.hd, kvh, (at - kvh * pieces) * KP::per16,
                          len, l0, l1, first, steps, node_s, src_s, dst_s);
  }
}

}  // namespace sprk
