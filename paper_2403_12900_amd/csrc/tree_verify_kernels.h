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
// removes its token: r_k is p without the rejected tokens, N_k = 1 - their sum.
//
// A chosen token is a whole number that an error in a sum can flip, so
// exponentials, sums and cumulative sums are fp64.
//
// Each vocabulary row is cut into chunks of kVChunk entries, one work-group
// each, so that few rows still fill the chip:
//   k_tree_verify<.., kStats>  per (row, chunk): maximum, its lowest index, sum of exp
//   k_tree_verify<.., kRest>   per (row with >= k children, chunk): its part of N_k
//                              (one launch per k; none without draft_probs)
// The work-group that finishes a request's last chunk walks its tree: every
// child's test at once (it depends on its parent's row alone), then the path
// by bit masks, then the draw: the chunk sums locate the chunk, which alone is
// read again.  No work-group waits on another, and all sums run in a fixed
// order.
#pragma once

#include "tree_attn_kernels.h"

namespace sprk {

constexpr int kVChunk = 4096;
constexpr int kVMaxChunks = 256;
constexpr int kVMaxVocab = kVChunk * kVMaxChunks;

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
  double* rest;            // [rest0[row] + k - 1][S]: parts of N_k
  int32_t* cnt;            // [n] finished work-groups; zero between launches
  int V, S, n, k;          // k: the pass (0: statistics)
  int vec_l, vec_d;        // rows of logits / draft_probs are 16-byte aligned
  float temp[kTreeReqs];
  uint16_t expect[kTreeReqs];  // work-groups of the request in this launch, if it ends with it (0: it does not)
  uint8_t row0[kTreeReqs], nodes[kTreeReqs];
  uint8_t list[kTreeRows];     // rows of this launch
  uint8_t req[kTreeRows], kids[kTreeRows], rank[kTreeRows], rest0[kTreeRows];
  int8_t parent[kTreeRows];
};
static_assert(sizeof(TreeVerifyArgs) <= 2048, "kernel arguments");

// Entries of one vocabulary chunk in registers: entry (j * 256 + thread) * EV
// + e of the chunk, EV entries per 16 bytes.
template <class T>
struct VChunkRegs {
  static constexpr int EV = 16 / static_cast<int>(sizeof(T)), NJ = kVChunk / (256 * EV);
  static __device__ __forceinline__ int index(int chunk, int j, int e) {
    return chunk * kVChunk + (j * 256 + static_cast<int>(threadIdx.x)) * EV + e;
  }
  static __device__ __forceinline__ float value(T x) {
    if constexpr (sizeof(T) == 4) return x;
    else return bf16_bits_to_f32(x);
  }
  // Entries past V read as `fill`.
  static __device__ __forceinline__ void load(const T* row, int V, int chunk, int vec, float fill, float (*x)[EV]) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int i0 = index(chunk, j, 0);
      if (vec && i0 + EV <= V) {
        union {
          uint4 u;
          T t[EV];
        } v;
        v.u = *reinterpret_cast<const uint4*>(row + i0);
#pragma unroll
        for (int e = 0; e < EV; ++e) x[j][e] = value(v.t[e]);
      } else {
#pragma unroll
        for (int e = 0; e < EV; ++e) x[j][e] = i0 + e < V ? value(row[i0 + e]) : fill;
      }
    }
  }
};

struct TreeVerifySmem {
  double d[4];
  float f[4];
  int i[4];
  int last, hit, tail;
  double z[kTreeNodes], m[kTreeNodes], fc[kTreeNodes], fn[kTreeNodes];  // per node: sum, maximum, state past its children
  double cc[kTreeNodes], cn[kTreeNodes], px[kTreeNodes];                // per node as a child: c_k, N_k, p(token)
  int best[kTreeNodes], bad[kTreeNodes], tok[kTreeNodes], order[kTreeNodes];
  double w[kVMaxChunks];
};

// Sums and maxima over the work-group, in a fixed order; every thread gets the result.
__device__ __forceinline__ double wave_sum(double v) {
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ double group_sum(double v, TreeVerifySmem* sm) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm->d[threadIdx.x >> 6] = v;
  __syncthreads();
  return ((sm->d[0] + sm->d[1]) + sm->d[2]) + sm->d[3];
}
__device__ __forceinline__ float group_max(float v, TreeVerifySmem* sm) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm->f[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(sm->f[0], sm->f[1]), fmaxf(sm->f[2], sm->f[3]));
}
__device__ __forceinline__ int group_min(int v, TreeVerifySmem* sm) {
  for (int o = 32; o >= 1; o >>= 1) v = min(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm->i[threadIdx.x >> 6] = v;
  __syncthreads();
  return min(min(sm->i[0], sm->i[1]), min(sm->i[2], sm->i[3]));
}

__device__ __forceinline__ void put64(uint64_t* p, uint64_t v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t get64(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ double get_double(const double* p) {
  return __longlong_as_double(static_cast<long long>(get64(reinterpret_cast<const uint64_t*>(p))));
}

// A draft probability as it counts: entries that are negative or NaN are 0.
__device__ __forceinline__ double draft_value(float q) { return q > 0.f ? static_cast<double>(q) : 0.0; }

// Maximum and sum of a row from its chunks (all threads of the work-group; S <= 256).
struct RowStat {
  float m;   // NaN: the row holds a NaN or has no finite maximum
  double z;
};
__device__ __forceinline__ RowStat row_stat(const TreeVerifyArgs& a, int row, double inv_t, TreeVerifySmem* sm) {
  float m = -INFINITY;
  double z = 0.0;
  bool bad = false;
  if (static_cast<int>(threadIdx.x) < a.S) {
    const uint64_t* st = a.stat + (static_cast<size_t>(row) * a.S + threadIdx.x) * 2;
    m = __uint_as_float(static_cast<uint32_t>(get64(st)));
    z = __longlong_as_double(static_cast<long long>(get64(st + 1)));
    bad = m != m;
  }
  bad = __syncthreads_or(bad);
  RowStat r;
  r.m = group_max(bad ? -INFINITY : m, sm);
  if (bad || !(fabsf(r.m) <= 3.402823466e38f)) r.m = __uint_as_float(0x7FC00000u);
  r.z = group_sum(m > -INFINITY ? z * exp((static_cast<double>(m) - r.m) * inv_t) : 0.0, sm);
  return r;
}

enum { kStats = 0, kRest = 1 };

template <class T>
__device__ __forceinline__ void tree_walk(const TreeVerifyArgs& a, int i, TreeVerifySmem* sm);

// T: storage of logits and draft_probs (float, or uint16_t for bf16).
template <class T, int kPhase>
__global__ __launch_bounds__(256) void k_tree_verify(TreeVerifyArgs a) {
  using Regs = VChunkRegs<T>;
  constexpr int EV = Regs::EV, NJ = Regs::NJ;
  __shared__ TreeVerifySmem sm;
  const int chunk = blockIdx.x, row = a.list[blockIdx.y], i = a.req[row];
  const float temp = a.temp[i];
  const double inv_t = temp > 0.f ? 1.0 / static_cast<double>(temp) : 1.0;
  float x[NJ][EV];
  Regs::load(static_cast<const T*>(a.logits) + row * a.ls, a.V, chunk, a.vec_l, -INFINITY, x);
  if constexpr (kPhase == kStats) {
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < EV; ++e) {
        nan |= x[j][e] != x[j][e];
        m = fmaxf(m, x[j][e]);
      }
    nan = __syncthreads_or(nan);
    m = group_max(m, &sm);
    int best = 0x7fffffff;
#pragma unroll
    for (int j = NJ - 1; j >= 0; --j)
#pragma unroll
      for (int e = EV - 1; e >= 0; --e)
        if (x[j][e] == m) best = min(best, Regs::index(chunk, j, e));
    best = group_min(best, &sm);
    double s = 0.0;
    if (temp > 0.f && m > -INFINITY && m < INFINITY) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < EV; ++e) s += exp((static_cast<double>(x[j][e]) - m) * inv_t);
    }
    s = group_sum(s, &sm);
    if (threadIdx.x == 0) {
      uint64_t* st = a.stat + (static_cast<size_t>(row) * a.S + chunk) * 2;
      const float mm = nan ? __uint_as_float(0x7FC00000u) : m;
      put64(st, __float_as_uint(mm) | static_cast<uint64_t>(static_cast<uint32_t>(best)) << 32);
      put64(st + 1, static_cast<uint64_t>(__double_as_longlong(s)));
    }
  } else {
    float q[NJ][EV];
    Regs::load(static_cast<const T*>(a.draft) + row * a.ds, a.V, chunk, a.vec_d, 0.f, q);
    const RowStat st = row_stat(a, row, inv_t, &sm);
    // c_k = 1 + N_1 + ... + N_{k-1}: all parts that the earlier passes left.
    const double* rest = a.rest + static_cast<size_t>(a.rest0[row]) * a.S;
    double c = 0.0;
    for (int t = threadIdx.x; t < (a.k - 1) * a.S; t += 256) c += get_double(rest + t);
    c = 1.0 + group_sum(c, &sm);
    double s = 0.0;
    if (st.m == st.m) {
      const double inv_z = 1.0 / st.z;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < EV; ++e)
          s += fmax(exp((static_cast<double>(x[j][e]) - st.m) * inv_t) * inv_z - c * draft_value(q[j][e]), 0.0);
    }
    s = group_sum(s, &sm);
    if (threadIdx.x == 0)
      put64(reinterpret_cast<uint64_t*>(a.rest + (static_cast<size_t>(a.rest0[row]) + a.k - 1) * a.S + chunk),
            static_cast<uint64_t>(__double_as_longlong(s)));
  }
  if (a.expect[i] == 0) return;
  // The work-group that completes the request walks its tree.
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this work-group's sums are stored
  if (threadIdx.x == 0)
    sm.last = __hip_atomic_fetch_add(a.cnt + i, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.expect[i] - 1;
  __syncthreads();
  if (!sm.last) return;
  if (threadIdx.x == 0) __hip_atomic_store(a.cnt + i, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  tree_walk<T>(a, i, &sm);
}

// Draw from one chunk: the lowest entry whose cumulative weight, from `base`
// on, exceeds `target`; else its last entry of positive weight.  w: this
// thread's weights in the chunk's register order.
template <class T>
__device__ __forceinline__ int draw_in_chunk(int chunk, const double (*w)[VChunkRegs<T>::EV], double base,
                                             double target, TreeVerifySmem* sm) {
  using Regs = VChunkRegs<T>;
  constexpr int EV = Regs::EV, NJ = Regs::NJ;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) {
    sm->hit = 0x7fffffff;
    sm->tail = -1;
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    double own = 0.0;
#pragma unroll
    for (int e = 0; e < EV; ++e) own += w[j][e];
    double scan = own;
    for (int o = 1; o < 64; o <<= 1) {
      const double up = __shfl_up(scan, o);
      if (lane >= o) scan += up;
    }
    __syncthreads();
    if (lane == 63) sm->d[wave] = scan;
    __syncthreads();
    double at = base + (scan - own);
    for (int v = 0; v < wave; ++v) at += sm->d[v];
#pragma unroll
    for (int e = 0; e < EV; ++e) {
      at += w[j][e];
      if (w[j][e] > 0.0) {
        if (at > target) atomicMin(&sm->hit, Regs::index(chunk, j, e));
        atomicMax(&sm->tail, Regs::index(chunk, j, e));
      }
    }
    base += ((sm->d[0] + sm->d[1]) + sm->d[2]) + sm->d[3];
  }
  __syncthreads();
  return sm->hit != 0x7fffffff ? sm->hit : sm->tail;
}

template <class T>
__device__ __forceinline__ void tree_walk(const TreeVerifyArgs& a, int i, TreeVerifySmem* sm) {
  using Regs = VChunkRegs<T>;
  constexpr int EV = Regs::EV, NJ = Regs::NJ;
  const int row0 = a.row0[i], nn = a.nodes[i], tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float temp = a.temp[i];
  const bool greedy = !(temp > 0.f), drafted = a.draft != nullptr && !greedy;
  const double inv_t = greedy ? 1.0 : 1.0 / static_cast<double>(temp);
  const T* logits = static_cast<const T*>(a.logits);
  const T* draft = static_cast<const T*>(a.draft);

  // Totals of every node's row, 16 lanes per node.
  for (int j0 = 0; j0 < nn; j0 += 16) {
    const int j = j0 + tid / 16, row = row0 + min(j, nn - 1);
    float m = -INFINITY;
    int best = 0x7fffffff;
    bool bad = false;
    for (int c = tid % 16; c < a.S; c += 16) {
      const uint64_t u = get64(a.stat + (static_cast<size_t>(row) * a.S + c) * 2);
      const float mc = __uint_as_float(static_cast<uint32_t>(u));
      bad |= mc != mc;
      better_of(m, best, mc, static_cast<int>(u >> 32));
    }
    for (int o = 8; o >= 1; o >>= 1) {
      better_of(m, best, __shfl_xor(m, o), __shfl_xor(best, o));
      bad |= __shfl_xor(static_cast<int>(bad), o) != 0;
    }
    bad |= !(fabsf(m) <= 3.402823466e38f);
    double z = 0.0;
    for (int c = tid % 16; c < a.S && !bad; c += 16) {
      const uint64_t* st = a.stat + (static_cast<size_t>(row) * a.S + c) * 2;
      const float mc = __uint_as_float(static_cast<uint32_t>(get64(st)));
      const double zc = __longlong_as_double(static_cast<long long>(get64(st + 1)));
      if (mc > -INFINITY) z += zc * exp((static_cast<double>(mc) - m) * inv_t);
    }
    for (int o = 8; o >= 1; o >>= 1) z += __shfl_xor(z, o);
    // c_k and N_k at the node, k = 0 .. children, to the child of rank k.
    double cc = 0.0, cn = 1.0;
    const int kids = a.kids[row];
    for (int k = 0;; ++k) {
      if (tid % 16 == 0 && j < nn) {
        if (k == kids) {
          sm->fc[j] = cc;
          sm->fn[j] = cn;
        } else {
          for (int t = j + 1; t < nn; ++t) {
            if (a.parent[row0 + t] == j && a.rank[row0 + t] == k) {
              sm->cc[t] = cc;
              sm->cn[t] = cn;
            }
          }
        }
      }
      if (k == kids || !drafted) break;
      cc += cn;
      cn = 0.0;
      const double* rest = a.rest + (static_cast<size_t>(a.rest0[row]) + k) * a.S;
      for (int c = tid % 16; c < a.S; c += 16) cn += get_double(rest + c);
      for (int o = 8; o >= 1; o >>= 1) cn += __shfl_xor(cn, o);
    }
    if (tid % 16 == 0 && j < nn) {
      sm->m[j] = m;
      sm->z[j] = z;
      sm->best[j] = best;
      sm->bad[j] = bad;
    }
  }
  if (tid < nn) {
    const int t = tid > 0 ? a.tok[row0 + tid] : -1;
    sm->tok[tid] = t;
    if (tid > 0 && (t < 0 || t >= a.V)) raise_check(a.err, kErrTokenRange);
  }
  __syncthreads();
  const int j = min(lane, nn - 1);  // every wave: lane = node
  const int par = lane < nn ? a.parent[row0 + j] : -1;
  const int t = sm->tok[j];
  const bool child = par >= 0, ranged = child && t >= 0 && t < a.V;
  double px = 0.0;
  if (!greedy && ranged && !sm->bad[par])
    px = exp((static_cast<double>(Regs::value(logits[(row0 + par) * a.ls + t])) - sm->m[par]) * inv_t) / sm->z[par];
  if (wave == 0 && lane < nn) sm->px[lane] = px;
  __syncthreads();
  bool ok = false, again = false;
  if (ranged && greedy) {
    ok = t == sm->best[par];
  } else if (ranged) {
    const double u = a.accept[row0 + j];
    if (drafted) {
      const double qx = draft_value(Regs::value(draft[(row0 + par) * a.ds + t]));
      ok = u * qx * sm->cn[j] < fmax(px - sm->cc[j] * qx, 0.0);
    } else {
      // Earlier siblings' tokens are gone, each token once.
      double left = 1.0;
      for (int s = 1; s < j; ++s) {
        if (a.parent[row0 + s] != par) continue;
        if (sm->tok[s] == t) again = true;
        bool first = true;
        for (int r = 1; r < s; ++r) first &= a.parent[row0 + r] != par || sm->tok[r] != sm->tok[s];
        if (first) left -= sm->px[s];
      }
      ok = !again && u * left < px;
    }
  }
  // The path: from the root, the first accepted child each time.
  const uint64_t oks = __ballot(ok && lane < nn), bads = __ballot(lane < nn && sm->bad[j] != 0);
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
    const float m = static_cast<float>(sm->m[node]);
    const T* lrow = logits + row * a.ls;
    // Chunk sums of the weights: of p (times the row's sum), or what the
    // rejections left of it.
    const bool rested = drafted && kids > 0 && sm->fn[node] > 0.0;
    float x[NJ][EV], q[NJ][EV];
    double w[NJ][EV];
    const auto weights = [&](int chunk, bool skip) {
      Regs::load(lrow, a.V, chunk, a.vec_l, -INFINITY, x);
      if (rested) Regs::load(draft + row * a.ds, a.V, chunk, a.vec_d, 0.f, q);
      const double inv_z = 1.0 / sm->z[node], c = sm->fc[node];
      double sum = 0.0;
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
        for (int e = 0; e < EV; ++e) {
          double v = exp((static_cast<double>(x[jj][e]) - m) * inv_t);
          if (rested) v = fmax(v * inv_z - c * draft_value(q[jj][e]), 0.0);
          w[jj][e] = v;
        }
      if (skip) {  // without the children's tokens
        for (int s = 1; s < nn; ++s) {
          if (a.parent[row0 + s] != node) continue;
          const int gone = sm->tok[s];
#pragma unroll
          for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
            for (int e = 0; e < EV; ++e)
              if (Regs::index(chunk, jj, e) == gone) w[jj][e] = 0.0;
        }
      }
#pragma unroll
      for (int jj = 0; jj < NJ; ++jj)
#pragma unroll
        for (int e = 0; e < EV; ++e) sum += w[jj][e];
      return sum;
    };
    const auto chunk_sums = [&](bool use_rest) {
      __syncthreads();
      if (tid < a.S) {
        if (use_rest) {
          sm->w[tid] = get_double(a.rest + (static_cast<size_t>(a.rest0[row]) + kids - 1) * a.S + tid);
        } else {
          const uint64_t* st = a.stat + (static_cast<size_t>(row) * a.S + tid) * 2;
          const float mc = __uint_as_float(static_cast<uint32_t>(get64(st)));
          const double zc = __longlong_as_double(static_cast<long long>(get64(st + 1)));
          sm->w[tid] = mc > -INFINITY ? zc * exp((static_cast<double>(mc) - m) * inv_t) : 0.0;
        }
      }
      __syncthreads();
    };
    bool skip = !drafted && kids > 0;
    chunk_sums(rested);
    if (skip) {
      // Chunks that hold a rejected token are summed again without it.
      for (int s = 1; s < nn; ++s) {
        if (a.parent[row0 + s] != node || sm->tok[s] < 0 || sm->tok[s] >= a.V) continue;
        const int chunk = sm->tok[s] / kVChunk;
        bool done = false;
        for (int r = 1; r < s; ++r)
          done |= a.parent[row0 + r] == node && sm->tok[r] >= 0 && sm->tok[r] < a.V && sm->tok[r] / kVChunk == chunk;
        if (done) continue;
        const double sum = group_sum(weights(chunk, true), sm);
        if (tid == 0) sm->w[chunk] = sum;
      }
      __syncthreads();
    }
    double all = 0.0;
    for (int c = 0; c < a.S; ++c) all += sm->w[c];
    if (skip && !(all > 0.0)) {  // nothing left: draw from p
      skip = false;
      chunk_sums(false);
      all = 0.0;
      for (int c = 0; c < a.S; ++c) all += sm->w[c];
    }
    double target = static_cast<double>(a.sample[i]) * all;
    double base = 0.0;
    int chunk = -1, some = 0;
    for (int c = 0; c < a.S; ++c) {
      if (sm->w[c] > 0.0) some = c;
      if (base + sm->w[c] > target) {
        chunk = c;
        break;
      }
      base += sm->w[c];
    }
    if (chunk < 0) {  // nothing exceeds it: the last entry of positive weight
      chunk = some;
      target = INFINITY;
    }
    weights(chunk, skip);
    drawn = draw_in_chunk<T>(chunk, w, base, target, sm);
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
