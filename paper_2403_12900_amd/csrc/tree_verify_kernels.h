// Verification of drafted tokens against the target's distribution, from given
// random numbers.
//
// At a node with target distribution p = softmax(logits / T), the children are
// tried in order, each against what the rejections before it left:
//   r_0 = p,   r_k = max(r_{k-1} - q, 0) / sum.
// With N_k the sum before normalisation (N_0 = 1) this has the closed form
//   r_k = max(p - c_k q, 0) / N_k,  c_0 = 0,  c_{k+1} = c_k + N_k,
//   N_k = sum_v max(p(v) - c_k q(v), 0),
// (the nested maxima collapse: q >= 0), so every N_k is one pass over p and q
// and no distribution is ever written.  A point mass at the child instead
// removes its token: r_k is p without the rejected tokens, N_k the sum of the
// others.  It is added up (the sum without any child's token, then those of the
// children yet to be tried) and never a difference: k rejections may leave
// 2^-24k, which 1 less their sum does not hold from the second one on.
//
// A chosen token is a whole number that an error in a sum can flip, so
// exponentials, sums and cumulative sums are fp64.
//
// Each vocabulary row is cut into chunks of kVChunk entries, one work-group
// each, so that few rows still fill the chip:
//   k_tree_stats  per (row, chunk): maximum, its lowest index, sum of exp, and
//                 without draft_probs the sum without the children's tokens
//   k_tree_rest   per (row with >= k children, chunk): its part of N_k (one
//                 launch per k; none without draft_probs)
//   k_tree_walk   per request: every child's test at once (it depends on its
//                 parent's row alone), then the path by bit masks, then the
//                 draw: the chunk sums locate the chunk, which alone is read
//                 again.
// No work-group waits on another, nothing is counted, and all sums run in a
// fixed order.  Bound by latency while the rows are few -- 5 rows of 32000: 14.5
// us, sums 5.5 (4.4 without the children's own) and walk 9.2 (8 of its loads and
// barriers follow one another) -- and by vector instructions where they are many:
// 128 rows of 131072 with draft probabilities, up to 4 children a node, 65 us: sums
// 23 (16.4 M entries of 42 instructions, 21 of them the exponential's fp64
// operations, the rest maximum, index, NaN test and conversion; the 33 MB alone
// would take 5), four N_k passes of 9, walk 12.  16 x 8 nodes of 32000: 28 us.  A
// node of many children costs a pass for each: 63 below the root, 64 rows of
// 32000, 335 us (of 131072: 414); without draft probabilities 45 (52).  (The walk
// as the end of the last sums' launch, in the work-group that finishes a request's
// last chunk, cost what the launch saves and held greedy requests' walks between
// two launches.)
#pragma once

#include "tree_attn_kernels.h"
#include "tree_exp.h"

namespace sprk {

constexpr int kVChunk = 4096;
constexpr int kVMaxChunks = 256;
constexpr int kVMaxVocab = kVChunk * kVMaxChunks;
// Entries of a chunk per thread: 16 where the sums are taken (256 threads: 4000
// work-groups of twice the waves took 26 us, as long as it takes to start
// them), 8 in the walk's draw, which one work-group makes alone.
constexpr int kSumOwn = 16, kDrawOwn = 8;
constexpr int kSumThreads = kVChunk / kSumOwn, kDrawThreads = kVChunk / kDrawOwn;

struct TreeVerifyArgs {
  const void* logits;
  const void* draft;       // or null
  int64_t ls, ds;          // row strides (elements)
  const int32_t* tok;
  const float* accept;
  const float* sample;
  int32_t *emitted, *path, *count;
  int* err;
  uint64_t* stat;          // [rows][S][2]: (maximum, its index), sum of exp((x - maximum) / T)
  double* rest;            // with draft: [rest0[row] + k - 1][S], parts of N_k; without:
                           // [row][S], the chunk's sum without the children's tokens
  int V, S, n, k, rows;    // k: the pass of k_tree_rest
  int vec_l, vec_d;        // rows of logits / draft_probs are 16-byte aligned
  float temp[kTreeReqs];
  uint8_t row0[kTreeReqs], nodes[kTreeReqs];
  uint8_t list[kTreeRows];     // rows of this launch
  uint8_t req[kTreeRows], kids[kTreeRows], rank[kTreeRows], rest0[kTreeRows];
  uint8_t parent_row[kTreeRows];  // kTreeRows for a root
  int8_t parent[kTreeRows];
};
static_assert(sizeof(TreeVerifyArgs) <= 2048, "kernel arguments");

// OWN consecutive entries of one vocabulary chunk per thread: entry thread *
// OWN + e, as floats; those past V read as `fill`.
template <int OWN>
__device__ __forceinline__ int chunk_index(int chunk) {
  return chunk * kVChunk + static_cast<int>(threadIdx.x) * OWN;
}
__device__ __forceinline__ float vocab_value(float x) { return x; }
__device__ __forceinline__ float vocab_value(uint16_t x) { return bf16_bits_to_f32(x); }
template <int OWN, class T>
__device__ __forceinline__ void load_chunk(const T* row, int V, int chunk, int vec, float fill, float* x) {
  constexpr int EV = 16 / static_cast<int>(sizeof(T));
  static_assert(OWN % EV == 0, "whole 16-byte loads");
  const int i0 = chunk_index<OWN>(chunk);
  if (vec && i0 + OWN <= V) {
#pragma unroll
    for (int j = 0; j < OWN / EV; ++j) {
      const uint4 u = *reinterpret_cast<const uint4*>(row + i0 + j * EV);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < EV; ++e) {
        if constexpr (sizeof(T) == 4) x[j * EV + e] = __uint_as_float(w[e]);
        else x[j * EV + e] = __uint_as_float(e % 2 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < OWN; ++e) x[e] = i0 + e < V ? vocab_value(row[i0 + e]) : fill;
  }
}

constexpr int kSumWaves = kSumThreads / 64, kDrawWaves = kDrawThreads / 64;
struct TreeWalkSmem {
  double d[kDrawWaves];
  int hit[kDrawWaves], tail[kDrawWaves];
  // Per node: its row's sum; with draft per array of parts: N_k, without per
  // node: its row's sum without the children's tokens.
  double z[kTreeNodes], total[kTreeNodes];
  double px[kTreeNodes];                        // per node as a child: p(its token)
  float m[kTreeNodes];                          // per node: its row's maximum (NaN: a bad row)
  int best[kTreeNodes], tok[kTreeNodes], order[kTreeNodes];
  int8_t parent[kTreeNodes];
  double w[kVMaxChunks];
};

// Wave scans and reductions on DPP moves (row shifts by 1, 2, 4, 8, then the
// row broadcasts): no trip through LDS.  Lanes that a move has no source for
// take `old`.
template <int kCtrl, int kRowMask>
__device__ __forceinline__ int dpp_move(int v, int old) {
  return __builtin_amdgcn_update_dpp(old, v, kCtrl, kRowMask, 0xF, false);
}
template <int kCtrl, int kRowMask>
__device__ __forceinline__ double dpp_add(double v) {
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(v));
  const uint32_t lo = static_cast<uint32_t>(dpp_move<kCtrl, kRowMask>(static_cast<int>(u), 0));
  const uint32_t hi = static_cast<uint32_t>(dpp_move<kCtrl, kRowMask>(static_cast<int>(u >> 32), 0));
  return v + __longlong_as_double(static_cast<long long>(static_cast<uint64_t>(hi) << 32 | lo));
}
// Inclusive sum over the lanes up to this one.
__device__ __forceinline__ double wave_scan(double v) {
  v = dpp_add<0x111, 0xF>(v);
  v = dpp_add<0x112, 0xF>(v);
  v = dpp_add<0x114, 0xF>(v);
  v = dpp_add<0x118, 0xF>(v);
  v = dpp_add<0x142, 0xA>(v);
  v = dpp_add<0x143, 0xC>(v);
  return v;
}
__device__ __forceinline__ double lane_value(double v, int lane) {
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(v));
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(u), lane));
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(u >> 32), lane));
  return __longlong_as_double(static_cast<long long>(static_cast<uint64_t>(hi) << 32 | lo));
}
__device__ __forceinline__ double wave_sum(double v) { return lane_value(wave_scan(v), 63); }
template <int kCtrl, int kRowMask>
__device__ __forceinline__ float dpp_max(float v) {
  return fmaxf(v, __int_as_float(dpp_move<kCtrl, kRowMask>(__float_as_int(v), static_cast<int>(0xFF800000u))));
}
__device__ __forceinline__ float wave_maximum(float v) {
  v = dpp_max<0x111, 0xF>(v);
  v = dpp_max<0x112, 0xF>(v);
  v = dpp_max<0x114, 0xF>(v);
  v = dpp_max<0x118, 0xF>(v);
  v = dpp_max<0x142, 0xA>(v);
  v = dpp_max<0x143, 0xC>(v);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
// Maximum of the wave and the index that its first lane with it holds.
__device__ __forceinline__ void wave_best(float& m, int& index) {
  const float w = wave_maximum(m);
  const uint64_t who = __ballot(m == w);
  index = who == 0 ? 0x7fffffff : __builtin_amdgcn_readlane(index, __ffsll(static_cast<unsigned long long>(who)) - 1);
  m = w;
}

// Sum over the work-group, in a fixed order; every thread gets it.
__device__ __forceinline__ double group_sum(double v, double* part) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < kSumWaves; ++w) s += part[w];
  return s;
}

__device__ __forceinline__ double as_double(uint64_t u) { return __longlong_as_double(static_cast<long long>(u)); }

// A draft probability as it counts: entries that are negative or NaN are 0.
__device__ __forceinline__ double draft_value(float q) { return q > 0.f ? static_cast<double>(q) : 0.0; }

// Maximum (NaN: a row with a NaN or no finite maximum), its lowest index and
// sum of a row from its chunks; every wave works them out by itself.
struct RowStat {
  float m;
  double z, rest;
  int best;
};
struct ChunkStat {
  uint64_t top, z;  // (maximum, its index); sum
  double rest;      // sum without the children's tokens
};
template <bool kRest>
__device__ __forceinline__ ChunkStat load_stat(const TreeVerifyArgs& a, int row, int c, bool with_rest = kRest) {
  ChunkStat s{0xFF800000u, 0, 0.0};  // no entries: maximum -inf
  if (c < a.S) {
    const size_t at = static_cast<size_t>(row) * a.S + c;
    s.top = a.stat[at * 2];
    s.z = a.stat[at * 2 + 1];
    if (kRest && with_rest) s.rest = a.rest[at];
  }
  return s;
}
// s: this lane's chunk of the first 64, loaded before.
template <bool kRest>
__device__ __forceinline__ RowStat row_stat(const TreeVerifyArgs& a, int row, ChunkStat s, double inv_t, bool want_z,
                                            bool with_rest = kRest) {
  const int lane = threadIdx.x & 63;
  RowStat r{-INFINITY, 0.0, 0.0, 0x7fffffff};
  bool bad = false;
#pragma unroll 1
  for (int c0 = 0;;) {
    const float m = __uint_as_float(static_cast<uint32_t>(s.top));
    int best = static_cast<int>(s.top >> 32);
    bad |= m != m;
    // The maximum so far, and the sum scaled to it.
    float wm = m == m ? m : -INFINITY;
    const float mine = wm;
    wave_best(wm, best);
    const float up = fmaxf(r.m, wm);
    if (wm > r.m) r.best = best;
    if (want_z && up > -INFINITY) {
      const double scale = mine > -INFINITY ? exp_neg((static_cast<double>(mine) - up) * inv_t) : 0.0;
      const double before = r.m > -INFINITY ? exp_neg((static_cast<double>(r.m) - up) * inv_t) : 0.0;
      r.z = r.z * before + wave_sum(as_double(s.z) * scale);
      if (kRest && with_rest) r.rest = r.rest * before + wave_sum(s.rest * scale);
    }
    r.m = up;
    c0 += 64;
    if (c0 >= a.S) break;
    s = load_stat<kRest>(a, row, c0 + lane, with_rest);
  }
  if (__ballot(bad) != 0 || !(fabsf(r.m) <= 3.402823466e38f)) r.m = __uint_as_float(0x7FC00000u);
  return r;
}

// T: storage of logits and draft_probs (float, or uint16_t for bf16).  Grid
// (chunks, rows); 8 waves per SIMD, which the fp64 exponentials need to overlap.
template <class T>
__global__ __launch_bounds__(kSumThreads, 8) void k_tree_stats(TreeVerifyArgs a) {
  __shared__ double part[kSumWaves], part2[kSumWaves];
  __shared__ float top_s[kSumWaves];
  __shared__ int best_s[kSumWaves];
  const int chunk = blockIdx.x, row = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float temp = a.temp[a.req[row]];
  float x[kSumOwn];
  load_chunk<kSumOwn>(static_cast<const T*>(a.logits) + row * a.ls, a.V, chunk, a.vec_l, -INFINITY, x);
  // Without draft_probs: the call's tokens, two per lane, and whether their
  // parent is this row (all asked for at once, with the logits).
  int tok[2] = {-1, -1};
  bool child[2] = {false, false};
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (a.draft == nullptr && 64 * h < a.rows) {
      const int r = min(64 * h + lane, a.rows - 1);
      tok[h] = a.tok[r];
      child[h] = 64 * h + lane < a.rows && a.parent_row[r] == row;
    }
  // Maximum with the lowest index that has it; a NaN anywhere makes it NaN.
  float m = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int e = 0; e < kSumOwn; ++e) {
    nan |= x[e] != x[e];
    m = fmaxf(m, x[e]);
  }
  int best = 0;
#pragma unroll
  for (int e = kSumOwn - 1; e >= 0; --e) best = x[e] == m ? e : best;
  best += chunk_index<kSumOwn>(chunk);
  wave_best(m, best);
  if (lane == 0) {
    top_s[wave] = m;
    best_s[wave] = best;
  }
  uint64_t children[2];  // with a token in this chunk
#pragma unroll
  for (int h = 0; h < 2; ++h)
    children[h] = __ballot(child[h] && tok[h] >= chunk * kVChunk && tok[h] < min(a.V, (chunk + 1) * kVChunk));
  nan = __syncthreads_or(nan);
  m = -INFINITY;
  best = 0x7fffffff;
#pragma unroll
  for (int w = 0; w < kSumWaves; ++w) better_of(m, best, top_s[w], best_s[w]);
  double s = 0.0, rest = 0.0;
  if (temp > 0.f) {
    const double inv_t = 1.0 / static_cast<double>(temp);
    double taken = 0.0;
    if (m > -INFINITY && m < INFINITY && !nan) {
      // The children's entries leave the others' sum, each once, and have one of their own.
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll 1
        for (uint64_t left = children[h]; left != 0; left &= left - 1) {
          const int at = __builtin_amdgcn_readlane(tok[h], __ffsll(static_cast<unsigned long long>(left)) - 1) -
                         chunk_index<kSumOwn>(chunk);
          float v = -INFINITY;
#pragma unroll
          for (int e = 0; e < kSumOwn; ++e) {
            v = at == e ? x[e] : v;
            x[e] = at == e ? -INFINITY : x[e];
          }
          if (__ballot(v > -INFINITY) != 0) taken += exp_neg((static_cast<double>(v) - m) * inv_t);
        }
      }
#pragma unroll
      for (int e = 0; e < kSumOwn; ++e) s += exp_neg((static_cast<double>(x[e]) - m) * inv_t);
    }
    rest = s = group_sum(s, part);
    if ((children[0] | children[1]) != 0) s += group_sum(taken, part2);
  }
  if (threadIdx.x == 0) {
    const size_t at = static_cast<size_t>(row) * a.S + chunk;
    const float mm = nan ? __uint_as_float(0x7FC00000u) : m;
    a.stat[at * 2] = __float_as_uint(mm) | static_cast<uint64_t>(static_cast<uint32_t>(best)) << 32;
    a.stat[at * 2 + 1] = static_cast<uint64_t>(__double_as_longlong(s));
    if (a.draft == nullptr) a.rest[at] = rest;
  }
}

// Grid (chunks, rows of a.list).
template <class T>
__global__ __launch_bounds__(kSumThreads) void k_tree_rest(TreeVerifyArgs a) {
  __shared__ double part[kSumWaves];
  const int chunk = blockIdx.x, row = a.list[blockIdx.y], lane = threadIdx.x & 63;
  const double inv_t = 1.0 / static_cast<double>(a.temp[a.req[row]]);
  float x[kSumOwn], q[kSumOwn];
  load_chunk<kSumOwn>(static_cast<const T*>(a.logits) + row * a.ls, a.V, chunk, a.vec_l, -INFINITY, x);
  load_chunk<kSumOwn>(static_cast<const T*>(a.draft) + row * a.ds, a.V, chunk, a.vec_d, 0.f, q);
  const ChunkStat first = load_stat<false>(a, row, lane);
  // c_k = 1 + N_1 + ... + N_{k-1}: all parts that the earlier passes left.
  double* rest = a.rest + static_cast<size_t>(a.rest0[row]) * a.S;
  double c = 0.0;
  for (int t = lane; t < (a.k - 1) * a.S; t += 64) c += rest[t];
  const RowStat st = row_stat<false>(a, row, first, inv_t, true);
  c = 1.0 + wave_sum(c);
  double s = 0.0;
  if (st.m == st.m) {
    const double inv_z = 1.0 / st.z;
#pragma unroll
    for (int e = 0; e < kSumOwn; ++e)
      s += fmax(exp_neg((static_cast<double>(x[e]) - st.m) * inv_t) * inv_z - c * draft_value(q[e]), 0.0);
  }
  s = group_sum(s, part);
  if (threadIdx.x == 0) rest[static_cast<size_t>(a.k - 1) * a.S + chunk] = s;
}

// Grid (requests).  The code is written for its size as much as for its work:
// it runs in a few work-groups, whose instruction fetches nothing hides
// (unrolled over 16 entries per thread, one draw from 32000 took 45 us).
template <class T>
__global__ __launch_bounds__(kDrawThreads) void k_tree_walk(TreeVerifyArgs a) {
  __shared__ TreeWalkSmem shared;
  TreeWalkSmem* const sm = &shared;
  const int i = blockIdx.x;
  const int row0 = a.row0[i], nn = a.nodes[i], tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float temp = a.temp[i];
  const bool greedy = !(temp > 0.f), drafted = a.draft != nullptr && !greedy, pointed = !greedy && !drafted;
  const double inv_t = greedy ? 1.0 : 1.0 / static_cast<double>(temp);
  const T* logits = static_cast<const T*>(a.logits);
  const T* draft = static_cast<const T*>(a.draft);
  const int base0 = a.rest0[row0];

  // Lane = node, in every wave: token, uniform, and its entries of the
  // parent's rows, loaded while the totals below are.
  const int j = min(lane, nn - 1);
  const int par = lane < nn ? a.parent[row0 + j] : -1;
  const bool child = par >= 0;
  const int t = child ? a.tok[row0 + j] : -1;
  const bool ranged = child && t >= 0 && t < a.V;
  float xt = 0.f, qt = 0.f, u = 0.f;
  if (ranged && !greedy) {
    u = a.accept[row0 + j];
    xt = vocab_value(logits[(row0 + par) * a.ls + t]);
    if (drafted) qt = vocab_value(draft[(row0 + par) * a.ds + t]);
  }
  if (wave == 0 && lane < nn) {
    sm->tok[lane] = t;
    sm->parent[lane] = static_cast<int8_t>(par);
    if (child && !ranged) raise_check(a.err, kErrTokenRange);
  }
  // Totals: rows by waves, then the arrays of parts (one per child) likewise,
  // kAhead of them asked for at once.
  constexpr int kAhead = 4;
#pragma unroll 1
  for (int r0 = wave; r0 < nn; r0 += kAhead * kDrawWaves) {
    ChunkStat s[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int r = row0 + min(r0 + k * kDrawWaves, nn - 1);
      s[k] = load_stat<true>(a, r, lane, pointed && a.kids[r] > 0);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int r = r0 + k * kDrawWaves;
      if (r >= nn) break;
      const RowStat st = row_stat<true>(a, row0 + r, s[k], inv_t, !greedy, pointed && a.kids[row0 + r] > 0);
      if (lane == 0) {
        sm->m[r] = st.m;
        sm->z[r] = st.z;
        if (pointed) sm->total[r] = st.rest;
        sm->best[r] = st.best;
      }
    }
  }
  if (drafted) {
#pragma unroll 1
    for (int r0 = wave; r0 < nn - 1; r0 += kAhead * kDrawWaves) {
      double s[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const double* parts = a.rest + (static_cast<size_t>(base0) + min(r0 + k * kDrawWaves, nn - 2)) * a.S;
        s[k] = lane < a.S ? parts[lane] : 0.0;
        for (int c = lane + 64; c < a.S; c += 64) s[k] += parts[c];
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const double sum = wave_sum(s[k]);
        if (lane == 0 && r0 + k * kDrawWaves < nn - 1) sm->total[r0 + k * kDrawWaves] = sum;
      }
    }
  }
  __syncthreads();
  const float pm = child ? sm->m[par] : 0.f;
  double px = 0.0;
  if (ranged && !greedy && pm == pm) px = exp_neg((static_cast<double>(xt) - pm) * inv_t) / sm->z[par];
  if (wave == 0 && lane < nn) sm->px[lane] = px;
  __syncthreads();
  bool ok = false;
  if (ranged && greedy) {
    ok = t == sm->best[par];
  } else if (ranged && drafted) {
    // c_k and N_k of its rank at the parent.
    double c = 0.0, n = 1.0;
    const int r0 = a.rest0[row0 + par] - base0, rank = a.rank[row0 + j];
#pragma unroll 1
    for (int k = 0; k < rank; ++k) {
      c += n;
      n = sm->total[r0 + k];
    }
    const double qx = draft_value(qt);
    ok = static_cast<double>(u) * qx * n < fmax(px - c * qx, 0.0);
  } else if (pointed) {
    // What the earlier siblings left: the tokens of none of the children, then
    // those of this child and the later ones, each once (at the first child
    // that has it).
    bool again = false;
#pragma unroll 1
    for (int s = 1; s < nn - 1; ++s) again |= s < j && sm->parent[s] == par && sm->tok[s] == t;
    const uint64_t firsts = __ballot(ranged && !again);
    double left = 1.0;
    if (ranged && a.rank[row0 + j] > 0) {
      left = sm->total[par] / sm->z[par];
#pragma unroll 1
      for (int s = j; s < nn; ++s) left += sm->parent[s] == par && (firsts >> s & 1) ? sm->px[s] : 0.0;
    }
    ok = ranged && !again && static_cast<double>(u) * left < px;
  }
  // The path: from the root, the first accepted child each time.
  const float mine = sm->m[j];
  const uint64_t oks = __ballot(ok && lane < nn), bads = __ballot(lane < nn && mine != mine);
  int node = 0, steps = 0;
  bool failed = false;
  for (;;) {
    if (bads >> node & 1) {
      failed = true;
      break;
    }
    if (tid == 0) sm->order[steps] = node;
    ++steps;
    const uint64_t next = __ballot(lane < nn && par == node) & oks;
    if (next == 0) break;
    node = __ffsll(static_cast<unsigned long long>(next)) - 1;
  }
  __syncthreads();
  if (failed) {
    if (tid == 0) {
      raise_check(a.err, kErrLogits);
      a.count[i] = 0;
    }
    if (tid < nn) a.emitted[row0 + tid] = a.path[row0 + tid] = -1;
    return;
  }

  int drawn = sm->best[node];
  if (!greedy) {
    const int row = row0 + node, kids = a.kids[row];
    const float m = sm->m[node];
    const double inv_z = 1.0 / sm->z[node];
    // What the draw takes: p (times its row's sum) without the rejected
    // tokens, or max(p - c q, 0) after all the children.
    double c = 0.0, left = 1.0;
    const int r0 = a.rest0[row] - base0;
    if (drafted) {
#pragma unroll 1
      for (int k = 0; k < kids; ++k) {
        c += left;
        left = sm->total[r0 + k];
      }
    }
    bool rested = drafted && kids > 0 && left > 0.0;
    bool skip = pointed && kids > 0;
    // Chunk sums of the weights.
    const auto chunk_sums = [&](bool parts, bool without) {
      __syncthreads();
      if (tid < a.S) {
        double w;
        if (parts) {
          w = a.rest[(static_cast<size_t>(base0) + r0 + kids - 1) * a.S + tid];
        } else {
          const ChunkStat s = load_stat<true>(a, row, tid, without);
          const float mc = __uint_as_float(static_cast<uint32_t>(s.top));
          w = mc > -INFINITY ? (without ? s.rest : as_double(s.z)) * exp_neg((static_cast<double>(mc) - m) * inv_t) : 0.0;
        }
        sm->w[tid] = w;
      }
      __syncthreads();
    };
    double all, target, base;
    int chunk;
    // The first chunk whose cumulative sum exceeds the target, by every wave.
    const auto pick = [&]() {
      double v[4], own = 0.0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int at = 4 * lane + k;
        v[k] = at < a.S ? sm->w[at] : 0.0;
        own += v[k];
      }
      const double scan = wave_scan(own);
      all = lane_value(scan, 63);
      target = static_cast<double>(a.sample[i]) * all;
      double at = scan - own, start = 0.0;
      int hit = -1, some = -1;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (v[k] > 0.0) {
          some = 4 * lane + k;
          if (hit < 0 && at + v[k] > target) {
            hit = 4 * lane + k;
            start = at;
          }
        }
        at += v[k];
      }
      const uint64_t hits = __ballot(hit >= 0), somes = __ballot(some >= 0);
      if (hits != 0) {
        const int from = __ffsll(static_cast<unsigned long long>(hits)) - 1;
        chunk = __builtin_amdgcn_readlane(hit, from);
        base = lane_value(start, from);
      } else {  // nothing exceeds it: the last entry of positive weight
        chunk = somes != 0 ? __builtin_amdgcn_readlane(some, 63 - __clzll(static_cast<long long>(somes))) : 0;
        base = 0.0;
        target = INFINITY;
      }
    };
    chunk_sums(rested, skip);
    pick();
    // A chunk whose sum is above 0 by rounding alone (c q took all of its weights,
    // or they are below what exp_neg holds) has no entry to draw: its sum is
    // cleared, and the draw made again.
#pragma unroll 1
    for (;;) {
      if ((skip || rested) && !(all > 0.0)) {  // nothing left: draw from p
        skip = rested = false;
        chunk_sums(false, false);
        pick();
      }
      // The chunk's lowest entry whose cumulative weight exceeds the target (else
      // its last of positive weight), each thread over its kDrawOwn.
      float x[kDrawOwn], q[kDrawOwn];
      load_chunk<kDrawOwn>(logits + row * a.ls, a.V, chunk, a.vec_l, -INFINITY, x);
      if (rested) load_chunk<kDrawOwn>(draft + row * a.ds, a.V, chunk, a.vec_d, 0.f, q);
      const int i0 = chunk_index<kDrawOwn>(chunk);
      if (skip) {  // without the children's tokens
#pragma unroll 1
        for (int s = 1; s < nn; ++s) {
          const int gone = sm->parent[s] == node ? sm->tok[s] - i0 : -1;
#pragma unroll
          for (int e = 0; e < kDrawOwn; ++e) x[e] = gone == e ? -INFINITY : x[e];
        }
      }
      double w[kDrawOwn], own = 0.0;
#pragma unroll
      for (int e = 0; e < kDrawOwn; ++e) {
        w[e] = exp_neg((static_cast<double>(x[e]) - m) * inv_t);
        if (rested) w[e] = fmax(w[e] * inv_z - c * draft_value(q[e]), 0.0);
        own += w[e];
      }
      const double scan = wave_scan(own);
      if (lane == 63) sm->d[wave] = scan;
      __syncthreads();
      double at = base + (scan - own);
#pragma unroll
      for (int v = 0; v < kDrawWaves - 1; ++v) at += v < wave ? sm->d[v] : 0.0;
      int hit = 0x7fffffff, tail = -1;
#pragma unroll
      for (int e = 0; e < kDrawOwn; ++e) {
        at += w[e];
        if (w[e] > 0.0) {
          tail = i0 + e;
          if (at > target) hit = min(hit, tail);
        }
      }
      const uint64_t hits = __ballot(hit != 0x7fffffff), tails = __ballot(tail >= 0);
      if (lane == 0) {
        sm->hit[wave] = sm->tail[wave] = -1;
        if (hits != 0) sm->hit[wave] = __builtin_amdgcn_readlane(hit, __ffsll(static_cast<unsigned long long>(hits)) - 1);
        if (tails != 0) sm->tail[wave] = __builtin_amdgcn_readlane(tail, 63 - __clzll(static_cast<long long>(tails)));
      }
      __syncthreads();
      int got = -1;
#pragma unroll
      for (int v = 0; v < kDrawWaves; ++v) got = max(got, sm->tail[v]);
#pragma unroll
      for (int v = kDrawWaves - 1; v >= 0; --v) got = sm->hit[v] >= 0 ? sm->hit[v] : got;
      if (got >= 0) {
        drawn = got;
        break;
      }
      if (!(all > 0.0)) break;
      if (tid == 0) sm->w[chunk] = 0.0;
      __syncthreads();
      pick();
    }
  }
  // Accepted tokens and the drawn one, then -1.
  if (tid < nn) {
    const bool on = tid < steps;
    a.path[row0 + tid] = on ? sm->order[tid] : -1;
    a.emitted[row0 + tid] = tid + 1 < steps ? sm->tok[sm->order[min(tid + 1, nn - 1)]] : tid + 1 == steps ? drawn : -1;
  }
  if (tid == 0) a.count[i] = steps;
}

}  // namespace sprk
