// Forking and moving the blocks of a paged cache: copies of whole blocks in
// every layer, and the block table's entries.
#pragma once

#include <hip/hip_runtime.h>

#include "cache_rule.h"
#include "device_common.h"
#include "op_handle.h"

namespace sprk {

typedef unsigned int page_piece_t __attribute__((ext_vector_type(4)));

// How a block's bytes are shared out: chunks of `chunk` 16-byte pieces, for
// every layer of every pool.
struct PageCopy {
  char* pool[2];
  int pools, layers, chunks, chunk, pieces;  // pieces of a block
  int64_t block_bytes, layer_bytes;
};

// Work item w of a block: its chunk in some layer of some pool.
struct PageItem {
  char* base;  // of block 0 of the layer
  int first, end;
};
__device__ __forceinline__ PageItem page_item(const PageCopy& c, int w) {
  const int chunk = w % c.chunks, l = w / c.chunks;
  PageItem it;
  it.base = (l < c.layers ? c.pool[0] : c.pool[1]) + (l < c.layers ? l : l - c.layers) * c.layer_bytes;
  it.first = chunk * c.chunk;
  it.end = min(it.first + c.chunk, c.pieces);
  return it;
}

struct ForkArgs {
  PageCopy c;
  int32_t* bt;
  int* err;
  int mb, nb, n, groups;
  int source[kCacheReqs], target[kCacheReqs], len[kCacheReqs];
  int fresh[kCacheReqs];           // -1 from first[groups] on
  int64_t part[kCacheReqs];        // table entry of each group's block
  uint8_t first[kCacheReqs + 1];
};
static_assert(sizeof(ForkArgs) <= 3584, "kernel arguments");
static_assert(kCacheReqs <= 255 && kCacheReqs % 8 == 0, "first's type, and fresh in eights");

// What keeps the forks f0 .. f1 - 1 from taking a copy of block id (0: nothing): id
// outside the pool, or a fresh block of the call that another of its forks copies
// from, be it id or one of their own.  The same for all threads of a work-group.
__device__ __forceinline__ int fork_fault(const ForkArgs& a, int f0, int f1, int id) {
  const int tid = threadIdx.x;
  bool fresh = false;
  for (int i = tid; i < a.first[a.groups]; i += 256) fresh |= a.fresh[i] == id;
  for (int i = tid; i < a.groups * (f1 - f0); i += 256) {  // (block that is copied, fresh block of these)
    const int f = i / a.groups;
    fresh |= a.fresh[f0 + f] == a.bt[a.part[i - f * a.groups]];
  }
  if (__syncthreads_or(fresh)) return kErrFresh;
  return static_cast<unsigned>(id) >= static_cast<unsigned>(a.nb) ? kErrBlockId : 0;
}

// Work-groups: n for the table rows, then the chunks of each group of forks
// that copy one block: it is read once and written to all of their blocks.
// Bound by the writes: 60 forks of 3 blocks, 40 layers of 40 heads in bf16 (524
// MB): 98 us, 5.6 TB/s of the 6.9 that a fill of 4 GiB reaches.  Stores that stay
// in the cache: 112 us with chunks of 16 KB, 107 without them; chunks of 8 KB 103,
// of 4 KB 98.  Looking the forks over takes less than 1 us of these, beside the
// block's read.
__global__ __launch_bounds__(256) void k_cache_fork(ForkArgs a) {
  const int tid = threadIdx.x;
  if (static_cast<int>(blockIdx.x) < a.n) {
    const int i = blockIdx.x, full = a.len[i] / 16;
    const int32_t* from = a.bt + static_cast<size_t>(a.source[i]) * a.mb;
    int32_t* to = a.bt + static_cast<size_t>(a.target[i]) * a.mb;
    const int copies = a.first[a.groups];
    constexpr int kDeep = 8;  // entries of a thread in flight
    for (int e0 = tid; e0 < full; e0 += 256 * kDeep) {
      int id[kDeep], fault = 0;
      uint32_t fresh = 0;
#pragma unroll
      for (int k = 0; k < kDeep; ++k) id[k] = from[min(e0 + 256 * k, full - 1)];
      for (int f = 0; f < copies; f += 8)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int k = 0; k < kDeep; ++k) fresh |= id[k] == a.fresh[f + j] ? 1u << k : 0u;
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        if (e0 + 256 * k >= full) break;
        const bool lost = static_cast<unsigned>(id[k]) >= static_cast<unsigned>(a.nb);
        if (lost || fresh >> k & 1) fault = lost ? kErrBlockId : kErrFresh;
        else to[e0 + 256 * k] = id[k];
      }
      if (fault) raise_check(a.err, fault);
    }
    if (i >= copies) return;
    const int group = __syncthreads_count(tid < a.groups && a.first[tid] <= i) - 1;
    if (fork_fault(a, a.first[group], a.first[group + 1], from[full]) == 0 && tid == 0) to[full] = a.fresh[i];
    return;
  }
  const int items = a.c.pools * a.c.layers * a.c.chunks;
  const int w = blockIdx.x - a.n, group = w / items;
  const int f0 = a.first[group], f1 = a.first[group + 1];
  const int id = a.bt[a.part[group]];
  const PageItem it = page_item(a.c, w - group * items);
  const int x = it.first + tid;
  // Read while the forks are looked over (block 0 where there is no such block).
  const int at = static_cast<unsigned>(id) < static_cast<unsigned>(a.nb) ? id : 0;
  const page_piece_t v = reinterpret_cast<const page_piece_t*>(it.base + at * a.c.block_bytes)[min(x, it.end - 1)];
  if (const int fault = fork_fault(a, f0, f1, id)) {
    if (tid == 0) raise_check(a.err, fault);
    return;
  }
  if (x >= it.end) return;
  for (int f = f0; f < f1; ++f)
    __builtin_nontemporal_store(v, reinterpret_cast<page_piece_t*>(it.base + a.fresh[f] * a.c.block_bytes) + x);
}

struct MoveArgs {
  PageCopy c;
  int32_t* bt;
  int n, table_groups;
  int64_t entries;
  int src[kMoves], dst[kMoves];  // src ascending
};
static_assert(sizeof(MoveArgs) <= 3584, "kernel arguments");

// Work-groups: table_groups for the table's entries (each looked up among the
// moved blocks), then the chunks of each moved block.  Bound by memory, at the
// rate of a plain copy: 175 blocks, 32 layers of 32 heads (780 MB read and
// written): 159 us, 4.9 TB/s (a 4 GiB copy: 4.8).
__global__ __launch_bounds__(256) void k_cache_move(MoveArgs a) {
  const int tid = threadIdx.x;
  if (static_cast<int>(blockIdx.x) < a.table_groups) {
    __shared__ int src[kMoves], dst[kMoves];
    for (int i = tid; i < a.n; i += 256) {
      src[i] = a.src[i];
      dst[i] = a.dst[i];
    }
    __syncthreads();
    const int64_t e1 = min(static_cast<int64_t>(blockIdx.x + 1) * kTableEntries, a.entries);
    for (int64_t e = static_cast<int64_t>(blockIdx.x) * kTableEntries + tid; e < e1; e += 256) {
      const int id = a.bt[e];
      int lo = 0, hi = a.n;  // the first src >= id lies in [lo, hi]
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (src[mid] < id) lo = mid + 1;
        else hi = mid;
      }
      if (lo < a.n && src[lo] == id) a.bt[e] = dst[lo];
    }
    return;
  }
  const int items = a.c.pools * a.c.layers * a.c.chunks;
  const int w = blockIdx.x - a.table_groups, m = w / items;
  const PageItem it = page_item(a.c, w - m * items);
  const page_piece_t* src = reinterpret_cast<const page_piece_t*>(it.base + a.src[m] * a.c.block_bytes);
  page_piece_t* dst = reinterpret_cast<page_piece_t*>(it.base + a.dst[m] * a.c.block_bytes);
  page_piece_t v[kMoveDeep];
#pragma unroll
  for (int k = 0; k < kMoveDeep; ++k) v[k] = src[min(it.first + tid + 256 * k, it.end - 1)];
#pragma unroll
  for (int k = 0; k < kMoveDeep; ++k) {
    const int x = it.first + tid + 256 * k;
    if (x < it.end) dst[x] = v[k];
  }
}

}  // namespace sprk
