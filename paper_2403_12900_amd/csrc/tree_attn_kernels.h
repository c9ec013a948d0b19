// Attention of drafted trees over the paged KV cache: row r = (request, node)
// and head h,
//   out[r][h] = softmax(q[r][h] . K^T / sqrt(hd)) V
// over the request's cached positions 0 .. len - 1 and the positions len + a
// of the node itself and its ancestors (bits of a 64-bit mask).
//
// The rows of one request share its keys and values, and so do the G query
// heads of a KV head: the columns of one (request, KV head) are (node, head of
// the group).  Reading the cache once is the floor while the columns are few;
// past about nine 16-column tiles (bf16 cache, fp32 queries) the products are.
//
// On MFMA, per block of 16 positions and tile of 16 columns:
//   S[t][c]   = K_tile(16 x hd) . Q^T(hd x 16)
//   O^T[e][c] += V^T_tile(16 dims x positions) . P(positions x 16)
// P is the S accumulator re-used in place as the B operand.  Two bf16 blocks
// make one 16x16x32 product: the K index of a lane's eight values may be
// assigned freely as long as both operands agree, so the first four are block
// 0's positions 4 g .. 4 g + 3 and the rest block 1's.
// fp32 queries meet a bf16 cache in three bf16 parts (all 24 bits), and the
// probabilities enter their product in three parts too, so that an fp32
// output is an fp32 result (two parts of the probabilities alone put 1e-6 of
// error on it); a bf16 output takes bf16 probabilities (their rounding, 2^-8
// relative and independent per position, is at most that of the output).
//
// The running maximum of a column is raised only when a step exceeds it by
// kRaise (in log2 units): until then probabilities of at most 2^kRaise stay
// exact enough in fp32, and steps need neither the exchange between lanes nor
// the rescaling of O.
//
// Two kernels.  Both cut a request's blocks into KV splits, one work-group
// each, merged by the split that arrives last:
//   k_tree_attn         up to 32 columns: the four waves of a work-group take
//                       runs of blocks, K and V go straight into registers.
//   k_tree_attn_shared  more: the four waves take 16 NT columns each and share
//                       every block through LDS, so the cache is read once per
//                       64 NT columns and a wave's work per byte stays high.
#pragma once

#include "gemm_kernels.h"
#include "tree_rule.h"

namespace sprk {

struct TreeAttnArgs {
  const void* q;
  void* out;
  int64_t qs, os;      // row strides of q and out (elements)
  const void* kc;      // this layer's K blocks
  const void* vc;      // this layer's V blocks
  const int32_t* bt;
  float* part;         // [item][Hkv][columns of an item][hd + 4]: m, l, -, -, o[hd]
  int32_t* cnt;        // [column group][Hkv] arrived splits; zero between launches
  int* err;
  int n, H, Hkv, G, mb, nb, bps;  // bps: blocks per split
  uint32_t part_bytes;
  float qscale;        // log2(e) / sqrt(hd)
  ActRec rec;          // layout of out, where it is an activation record
  int slot[kTreeReqs], len[kTreeReqs];
  int item0[kTreeReqs + 1];      // first work item of each request
  uint8_t nodes[kTreeReqs], ncg[kTreeReqs];
  uint8_t row0[kTreeReqs], cg0[kTreeReqs];  // first row, first column group
  uint64_t anc[kTreeRows];
};
static_assert(sizeof(TreeAttnArgs) <= 3584, "kernel arguments");

// Formats of q and out.  load: per16 values of a row as floats (kRaw: as the
// 16-byte bf16 fragment piece itself).
struct TreeIoF32 {
  using elem = float;
  static constexpr bool kRaw = false;
  static __device__ __forceinline__ void store4(const TreeAttnArgs& a, int row, int n0, f32x4_t v) {
    *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + row * a.os + n0) = v;
  }
};
struct TreeIoBF16 {
  using elem = uint16_t;
  static constexpr bool kRaw = true;
  static __device__ __forceinline__ void store4(const TreeAttnArgs& a, int row, int n0, f32x4_t v) {
    uint2 o;
    o.x = f32_to_bf16_bits(v[0]) | static_cast<uint32_t>(f32_to_bf16_bits(v[1])) << 16;
    o.y = f32_to_bf16_bits(v[2]) | static_cast<uint32_t>(f32_to_bf16_bits(v[3])) << 16;
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + row * a.os + n0) = o;
  }
};
// Inside a model pass: fp32 queries, and the output as the next projection's
// activation record.
template <class AP>
struct TreeIoAct {
  using elem = float;
  static constexpr bool kRaw = false;
  static __device__ __forceinline__ void store4(const TreeAttnArgs& a, int row, int n0, f32x4_t v) {
    store_act4<AP>(static_cast<typename AP::elem*>(a.out), a.rec, row, n0, v[0], v[1], v[2], v[3]);
  }
};

// The storage rounding of v as one 16-byte piece, taken from v.
template <class KP>
__device__ __forceinline__ uint4 next_part(float* v) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (KP::per16 == 4) {
      w[j] = __float_as_uint(v[j]);
    } else {
      const uint32_t lo = f32_to_bf16_bits(v[2 * j]), hi = f32_to_bf16_bits(v[2 * j + 1]);
      w[j] = lo | hi << 16;
      v[2 * j] -= bf16_bits_to_f32(lo);
      v[2 * j + 1] -= bf16_bits_to_f32(hi);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Zeroes the infinite and NaN values of a 16-byte piece; returns whether it
// had one.
template <class KP>
__device__ __forceinline__ bool clean_piece(uint4& u) {
  bool odd = false;
  const auto clean = [&](uint32_t x) {
    if constexpr (KP::per16 == 4) {
      const bool o = (x & 0x7F800000u) == 0x7F800000u;
      odd |= o;
      return o ? 0u : x;
    } else {
      const bool lo = (x & 0x7F80u) == 0x7F80u, hi = (x & 0x7F800000u) == 0x7F800000u;
      odd |= lo || hi;
      return x & ((lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u));
    }
  };
  u.x = clean(u.x);
  u.y = clean(u.y);
  u.z = clean(u.z);
  u.w = clean(u.w);
  return odd;
}

// Zeroes the positions of a 16-byte V piece (4 g .. 4 g + 3 of its block) whose
// bit of keep is clear.
template <class KP>
__device__ __forceinline__ void keep_piece(uint4& u, uint32_t keep) {
  if constexpr (KP::per16 == 4) {
    u.x = keep & 1 ? u.x : 0u;
    u.y = keep & 2 ? u.y : 0u;
    u.z = keep & 4 ? u.z : 0u;
    u.w = keep & 8 ? u.w : 0u;
  } else {
    const uint32_t m01 = (keep & 1 ? 0xFFFFu : 0u) | (keep & 2 ? 0xFFFF0000u : 0u);
    const uint32_t m23 = (keep & 4 ? 0xFFFFu : 0u) | (keep & 8 ? 0xFFFF0000u : 0u);
    u.x &= m01;
    u.y &= m23;
    u.z &= m01;
    u.w &= m23;
  }
}

// Bits: which of the four positions from `pos` on lie before `end`.
__device__ __forceinline__ uint32_t live_bits(int pos, int end) {
  const int room = end - pos;
  return room >= 4 ? 15u : room <= 0 ? 0u : (1u << room) - 1;
}

// Bits of the four positions from `pos` on that a column sees: cached ones
// (before len), then the nodes that its ancestor set holds.  Shifts only, no
// branches.
__device__ __forceinline__ uint32_t seen_bits(int pos, int len, uint64_t anc) {
  const int base = pos - len, cached = min(max(-base, 0), 4);
  const uint32_t nodes = static_cast<uint32_t>(anc >> min(max(base, 0), 63)) << cached;
  return (((1u << cached) - 1) | nodes) & 15u;
}

// Infinite and NaN values were zeroed in the products (0 times one must not
// reach the columns that do not see it): adds p times each of them to the
// columns that do.  One step's blocks tile[] of one KV head, p and sees as the
// step's scores are held; values are read again, element by element.
template <class KP, int HD, int BP>
__device__ __forceinline__ void add_odd_values(f32x4_t* O, const float (*p)[4], const uint32_t* sees, const void* vc,
                                               const size_t* tile, const uint32_t* live, int lane) {
  const int h = lane & 15, g = lane >> 4;
#pragma unroll 1
  for (int t = 0; t < 16 * BP; ++t) {
    const int b = t >> 4, gt = t >> 2 & 3, r = t & 3;
    float pt = 0.f;
    uint32_t st = 0, lt = 0;
    size_t at = tile[0];
#pragma unroll
    for (int k = 0; k < BP; ++k)
      if (k == b) {
        pt = r == 0 ? p[k][0] : r == 1 ? p[k][1] : r == 2 ? p[k][2] : p[k][3];
        st = sees[k];
        lt = live[k];
        at = tile[k];
      }
    pt = __shfl(pt, h + 16 * gt);
    st = __shfl(static_cast<int>(st), h + 16 * gt) >> r & 1;
    lt = __shfl(static_cast<int>(lt), 16 * gt) >> r & 1;
    if (!lt) continue;
    const typename KP::elem* v = static_cast<const typename KP::elem*>(vc) + at * 16 * HD;
#pragma unroll
    for (int e = 0; e < HD / 16; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = KP::to_f32(v[vtile_offset<KP>(t & 15, 16 * e + 4 * g + i)]);
        O[e][i] += st && !(fabsf(x) <= 3.402823466e38f) ? pt * x : 0.f;
      }
  }
}

// K and V of one step: kBlocks blocks of one KV head, in registers.
template <class KP, int HD>
struct TreeStep;

template <int HD>
struct TreeStep<BF16, HD> {
  static constexpr int kBlocks = 2, NF = HD / 32, NV = HD / 32;
  uint4 k[2][NF], v[2][NV];

  __device__ __forceinline__ void load(const void* kc, const void* vc, const size_t* tile, int lane) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint4* kt = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(kc) + tile[b] * 16 * HD) + lane;
      const uint4* vt = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(vc) + tile[b] * 16 * HD) + lane;
#pragma unroll
      for (int f = 0; f < NF; ++f) k[b][f] = kt[f * 64];
#pragma unroll
      for (int f = 0; f < NV; ++f) v[b][f] = vt[f * 64];
    }
  }
  // Zeroes the values of this lane's positions 4 g + i of block b whose bit i
  // of keep[b] is clear.
  __device__ __forceinline__ void keep_v(const uint32_t* keep) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int f = 0; f < NV; ++f) keep_piece<BF16>(v[b][f], keep[b]);
  }
  // Zeroes infinite and NaN values; returns whether this lane had one.
  __device__ __forceinline__ bool clean_v() {
    bool odd = false;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int f = 0; f < NV; ++f) odd |= clean_piece<BF16>(v[b][f]);
    return odd;
  }
  template <int PP>
  __device__ __forceinline__ void pv(f32x4_t* O, const float (*p)[4]) const {
    uint4 b[PP];
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = p[i / 4][i % 4];
#pragma unroll
    for (int q = 0; q < PP; ++q) {
      b[q] = next_part<BF16>(r);
    }
#pragma unroll
    for (int f = 0; f < NV; ++f) {
      const uint4 a0 = make_uint4(v[0][f].x, v[0][f].y, v[1][f].x, v[1][f].y);
      const uint4 a1 = make_uint4(v[0][f].z, v[0][f].w, v[1][f].z, v[1][f].w);
#pragma unroll
      for (int q = 0; q < PP; ++q) {
        O[2 * f] = BF16::mma(O[2 * f], a0, b[q]);
        O[2 * f + 1] = BF16::mma(O[2 * f + 1], a1, b[q]);
      }
    }
  }
};

template <int HD>
struct TreeStep<F32, HD> {
  static constexpr int kBlocks = 1, NF = HD / 16, NV = HD / 16;
  uint4 k[1][NF], v[1][NV];

  __device__ __forceinline__ void load(const void* kc, const void* vc, const size_t* tile, int lane) {
    const uint4* kt = reinterpret_cast<const uint4*>(static_cast<const float*>(kc) + tile[0] * 16 * HD) + lane;
    const uint4* vt = reinterpret_cast<const uint4*>(static_cast<const float*>(vc) + tile[0] * 16 * HD) + lane;
#pragma unroll
    for (int f = 0; f < NF; ++f) k[0][f] = kt[f * 64];
#pragma unroll
    for (int f = 0; f < NV; ++f) v[0][f] = vt[f * 64];
  }
  __device__ __forceinline__ void keep_v(const uint32_t* keep) {
#pragma unroll
    for (int f = 0; f < NV; ++f) keep_piece<F32>(v[0][f], keep[0]);
  }
  __device__ __forceinline__ bool clean_v() {
    bool odd = false;
#pragma unroll
    for (int f = 0; f < NV; ++f) odd |= clean_piece<F32>(v[0][f]);
    return odd;
  }
  template <int PP>
  __device__ __forceinline__ void pv(f32x4_t* O, const float (*p)[4]) const {
#pragma unroll
    for (int f = 0; f < NV; ++f) {
      O[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[0][f].x), p[0][0], O[f], 0, 0, 0);
      O[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[0][f].y), p[0][1], O[f], 0, 0, 0);
      O[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[0][f].z), p[0][2], O[f], 0, 0, 0);
      O[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[0][f].w), p[0][3], O[f], 0, 0, 0);
    }
  }
};

// Parts of q and of the probabilities by cache and io format.
template <class KP, class IO>
struct TreeParts {
  static constexpr int q = KP::per16 == 4 || IO::kRaw ? 1 : 3;
  static constexpr int p = KP::per16 == 4 || IO::kRaw ? 1 : 3;
};

template <class KP, class IO, int HD, int NT>
struct TreeSmem {
  static constexpr int NF = HD / KP::kblk;
  union {
    uint4 q[NT][NF][TreeParts<KP, IO>::q][64];
    f32x4_t so[4][HD / 16][64];
  };
  float2 sml[4][NT][16];
  int last;
};

constexpr float kTreeFloor = -1e38f;  // running maximum before the first score
constexpr float kRaise = 8.f;

// Column c of a request (c < its nodes * G): token row and query head.
struct TreeColumn {
  int row, hq;
};
__device__ __forceinline__ TreeColumn tree_column(const TreeAttnArgs& a, int row0, int kvh, int c) {
  const int node = c / a.G;
  return TreeColumn{row0 + node, kvh * a.G + c - node * a.G};
}

// This lane's piece (K-block c, group g) of one column's query, in fp32, or
// (kRaw with a bf16 cache) as the fragment piece itself.
template <class KP, class IO, int HD>
__device__ __forceinline__ void load_query(const TreeAttnArgs& a, const TreeColumn& col, int c, int g, uint4* out) {
  const typename IO::elem* src =
      static_cast<const typename IO::elem*>(a.q) + col.row * a.qs + col.hq * HD + c * KP::kblk + g * KP::per16;
  constexpr int QP = TreeParts<KP, IO>::q;
  if constexpr (IO::kRaw && KP::per16 == 8) {
    out[0] = *reinterpret_cast<const uint4*>(src);
  } else {
    float v[KP::per16];
    if constexpr (IO::kRaw) {
      const uint2 u = *reinterpret_cast<const uint2*>(src);
      v[0] = __uint_as_float(u.x << 16);
      v[1] = __uint_as_float(u.x & 0xFFFF0000u);
      v[2] = __uint_as_float(u.y << 16);
      v[3] = __uint_as_float(u.y & 0xFFFF0000u);
    } else {
#pragma unroll
      for (int j = 0; j < KP::per16; j += 4) {
        const float4 x = *reinterpret_cast<const float4*>(src + j);
        v[j] = x.x;
        v[j + 1] = x.y;
        v[j + 2] = x.z;
        v[j + 3] = x.w;
      }
    }
#pragma unroll
    for (int q = 0; q < QP; ++q) out[q] = next_part<KP>(v);
  }
}

// Online softmax of one column tile's scores of one step: raises the running
// maximum where needed, turns S into probabilities and adds them to l.
template <int BP, int NE>
__device__ __forceinline__ void softmax_step(const f32x4_t* S, float qscale, float& m, float& l, f32x4_t* O, float (*p)[4]) {
  float mx = fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3]));
#pragma unroll
  for (int b = 1; b < BP; ++b) mx = fmaxf(mx, fmaxf(fmaxf(S[b][0], S[b][1]), fmaxf(S[b][2], S[b][3])));
  mx *= qscale;
  if (__ballot(mx > m + kRaise) != 0) {
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float up = fmaxf(m, mx);
    const float alpha = __builtin_amdgcn_exp2f(m - up);
    l *= alpha;
    m = up;
#pragma unroll
    for (int e = 0; e < NE; ++e) O[e] *= alpha;
  }
#pragma unroll
  for (int b = 0; b < BP; ++b) {
#pragma unroll
    for (int r = 0; r < 4; ++r) p[b][r] = __builtin_amdgcn_exp2f(fmaf(S[b][r], qscale, -m));
    l += (p[b][0] + p[b][1]) + (p[b][2] + p[b][3]);
  }
}

// What a work item is: its request, blocks and columns.
struct TreeItem {
  int rank, cg, nsplit, ncg;
  int len, total, nblk, row0, cols;
  int first, count;          // blocks of the split
  const int32_t* btrow;
};
__device__ __forceinline__ TreeItem tree_item(const TreeAttnArgs& a, int f) {
  const int lane = threadIdx.x & 63;
  TreeItem t;
  // Request: the number of requests whose items all precede f.
  t.rank = __builtin_amdgcn_readfirstlane(
      __popcll(__ballot(lane < a.n - 1 && a.item0[min(lane + 1, kTreeReqs)] <= f)));
  t.ncg = a.ncg[t.rank];
  const int w = f - a.item0[t.rank], s = w / t.ncg;
  t.cg = w - s * t.ncg;  // column groups of one split run side by side and share its blocks
  t.nsplit = (a.item0[t.rank + 1] - a.item0[t.rank]) / t.ncg;
  t.len = a.len[t.rank];
  t.total = t.len + a.nodes[t.rank];
  t.nblk = (t.total + 15) >> 4;
  t.row0 = a.row0[t.rank];
  t.cols = a.nodes[t.rank] * a.G;
  t.first = a.bps * s;
  t.count = min(t.nblk - t.first, a.bps);
  t.btrow = a.bt + static_cast<size_t>(a.slot[t.rank]) * a.mb;
  return t;
}

// Block id of block i (< end) of the table row; one outside the pool is
// reported and reads block 0.
__device__ __forceinline__ int block_id(const TreeAttnArgs& a, const int32_t* btrow, int i, int end) {
  int id = i < end ? btrow[i] : 0;
  if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.nb)) {
    raise_check(a.err, kErrBlockId);
    id = 0;
  }
  return id;
}

// Counts a split in and, in the one that arrives last, merges all partials of
// its column group (CW columns): no work-group waits on another.  The
// caller's partials are stored (agent-coherent).
template <class IO, int HD, int CW>
__device__ __forceinline__ void merge_splits(const TreeAttnArgs& a, const TreeItem& t, int kvh, const CoherentBuffer& pb,
                                             int* last) {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's partial stores are complete
  __syncthreads();
  int32_t* cnt = a.cnt + (a.cg0[t.rank] + t.cg) * a.Hkv + kvh;
  if (threadIdx.x == 0)
    *last = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == t.nsplit - 1;
  __syncthreads();
  if (!*last) return;
  if (threadIdx.x == 0) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const uint32_t base = (static_cast<uint32_t>(a.item0[t.rank] + t.cg) * a.Hkv + kvh) * CW * (HD + 4) * 4;
  const uint32_t stride = static_cast<uint32_t>(t.ncg) * a.Hkv * CW * (HD + 4) * 4;
  constexpr int kChunk = 8;  // partials read per round
  const int c0 = CW * t.cg, mine = min(t.cols - c0, CW);
  for (int idx = threadIdx.x; idx < mine * (HD / 4); idx += 256) {
    const int c = idx / (HD / 4), d0 = idx % (HD / 4) * 4;
    const uint32_t at = base + c * (HD + 4) * 4;
    float M = kTreeFloor, L = 0.f;
    f32x4_t R = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int t0 = 0; t0 < t.nsplit; t0 += kChunk) {
      f32x4_t ml[kChunk], o[kChunk];
#pragma unroll
      for (int k = 0; k < kChunk; ++k) {
        const uint32_t b = at + min(t0 + k, t.nsplit - 1) * stride;
        ml[k] = pb.load4(b);
        o[k] = pb.load4(b + 16 + d0 * 4);
      }
      float up = M;
#pragma unroll
      for (int k = 0; k < kChunk; ++k) up = t0 + k < t.nsplit ? fmaxf(up, ml[k][0]) : up;
      const float sc = __builtin_amdgcn_exp2f(M - up);
      L *= sc;
      R *= sc;
#pragma unroll
      for (int k = 0; k < kChunk; ++k) {
        if (t0 + k < t.nsplit) {
          const float wt = __builtin_amdgcn_exp2f(ml[k][0] - up);
          L += wt * ml[k][1];
          R += wt * o[k];
        }
      }
      M = up;
    }
    const TreeColumn col = tree_column(a, t.row0, kvh, c0 + c);
    IO::store4(a, col.row, col.hq * HD + d0, R * (1.f / L));
  }
}

template <class KP, class IO, int HD, int NT>
__global__ __launch_bounds__(256) void k_tree_attn(TreeAttnArgs a) {
  using Step = TreeStep<KP, HD>;
  using Parts = TreeParts<KP, IO>;
  constexpr int BP = Step::kBlocks, NF = Step::NF, NE = HD / 16, EPW = NE / 4, CW = 16 * NT;
  __shared__ TreeSmem<KP, IO, HD, NT> sm;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane & 15, g = lane >> 4;
  const int f = blockIdx.y, kvh = blockIdx.x;
  const TreeItem t = tree_item(a, f);
  // Runs of the four waves: equal shares of the split, in whole steps.
  const int run = (t.count + 4 * BP - 1) / (4 * BP) * BP;
  const int lo = t.first + min(t.count, wave * run), hi = t.first + min(t.count, (wave + 1) * run);
  int ids = block_id(a, t.btrow, lo + lane, hi);  // of the next 64 blocks of the run

  // Q fragments into LDS (every wave reads them all); columns past the
  // request's read its last one's row.
#pragma unroll
  for (int n = 0; n < (NT * NF + 3) / 4; ++n) {
    const int k = wave + 4 * n, jt = k / NF, c = k % NF;
    if (k >= NT * NF) break;
    uint4 x[Parts::q];
    load_query<KP, IO, HD>(a, tree_column(a, t.row0, kvh, min(16 * jt + h, t.cols - 1)), c, g, x);
#pragma unroll
    for (int q = 0; q < Parts::q; ++q) sm.q[jt][c][q][lane] = x[q];
  }
  uint64_t anc[NT];
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) anc[jt] = a.anc[tree_column(a, t.row0, kvh, min(16 * jt + h, t.cols - 1)).row];
  __syncthreads();

  f32x4_t O[NT][NE];
  float m[NT], l[NT];
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    m[jt] = kTreeFloor;
    l[jt] = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) O[jt][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  for (int i = lo; i < hi; i += BP) {
    const int k = i - lo;
    if ((k & 63) == 0 && k != 0) ids = block_id(a, t.btrow, i + lane, hi);
    Step B;
    size_t tile[BP];
#pragma unroll
    for (int b = 0; b < BP; ++b)  // a missing second block re-reads the first, masked
      tile[b] = static_cast<size_t>(__builtin_amdgcn_readlane(ids, (i + b < hi ? k + b : k) & 63)) * a.Hkv + kvh;
    B.load(a.kc, a.vc, tile, lane);
    // A step that reaches past the cached positions or the run is masked.
    const bool tail = 16 * (i + BP) > t.len || i + BP > hi;
    uint32_t live[BP];  // bits: this lane's positions of the block that hold a cached position or a node
    bool odd = false;
    if (tail) {
#pragma unroll
      for (int b = 0; b < BP; ++b) live[b] = i + b < hi ? live_bits(16 * (i + b) + 4 * g, t.total) : 0u;
      B.keep_v(live);
      odd = __ballot(B.clean_v()) != 0;
    }
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
      f32x4_t S[BP];
#pragma unroll
      for (int b = 0; b < BP; ++b) S[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NF; ++c)
#pragma unroll
        for (int q = 0; q < Parts::q; ++q) {
          const uint4 x = sm.q[jt][c][q][lane];
#pragma unroll
          for (int b = 0; b < BP; ++b) S[b] = KP::mma(S[b], B.k[b][c], x);
        }
      uint32_t sees[BP];
      if (tail) {
#pragma unroll
        for (int b = 0; b < BP; ++b) {
          sees[b] = live[b] & seen_bits(16 * (i + b) + 4 * g, t.len, anc[jt]);
#pragma unroll
          for (int r = 0; r < 4; ++r) S[b][r] = sees[b] >> r & 1 ? S[b][r] : -INFINITY;
        }
      }
      float p[BP][4];
      softmax_step<BP, NE>(S, a.qscale, m[jt], l[jt], O[jt], p);
      B.template pv<Parts::p>(O[jt], p);
      if (odd) add_odd_values<KP, HD, BP>(O[jt], p, sees, a.vc, tile, live, lane);
    }
  }

  // Merge of the four waves, column tile by column tile; wave w combines and
  // stores output operands [w EPW, (w + 1) EPW).
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    l[jt] += __shfl_xor(l[jt], 16);
    l[jt] += __shfl_xor(l[jt], 32);
    if (g == 0) sm.sml[wave][jt][h] = make_float2(m[jt], l[jt]);
  }
  const CoherentBuffer pb(a.part, a.part_bytes);
  const uint32_t item = (static_cast<uint32_t>(f) * a.Hkv + kvh) * CW * (HD + 4) * 4;
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    __syncthreads();  // Q (and the previous tile's outputs) have been read
#pragma unroll
    for (int e = 0; e < NE; ++e) sm.so[wave][e][lane] = O[jt][e];
    __syncthreads();
    float M = kTreeFloor, L = 0.f, cw[4];
    float2 ml[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      ml[v] = sm.sml[v][jt][h];
      M = fmaxf(M, ml[v].x);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      cw[v] = __builtin_amdgcn_exp2f(ml[v].x - M);
      L += cw[v] * ml[v].y;
    }
    const int c = 16 * jt + h;
    const TreeColumn col = tree_column(a, t.row0, kvh, c);
#pragma unroll
    for (int k = 0; k < EPW; ++k) {
      f32x4_t R = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const f32x4_t o = sm.so[v][wave * EPW + k][lane];
#pragma unroll
        for (int r = 0; r < 4; ++r) R[r] += cw[v] * o[r];
      }
      if (c >= t.cols) continue;
      const int d0 = 16 * (wave * EPW + k) + 4 * g;
      if (t.nsplit == 1) {
        IO::store4(a, col.row, col.hq * HD + d0, R * (1.f / L));
      } else {
        pb.store4(item + (c * (HD + 4) + 4 + d0) * 4, R);
        if (wave == 0 && k == 0 && g == 0) pb.store4(item + c * (HD + 4) * 4, f32x4_t{M, L, 0.f, 0.f});
      }
    }
  }
  if (t.nsplit > 1) merge_splits<IO, HD, CW>(a, t, kvh, pb, &sm.last);
}

// ---------------------------------------------------------------------------

// K and V blocks of one step in LDS, [K block 0][K block 1]..[V block 0].., each
// in its tile's order, two steps deep.
template <class KP, int HD>
struct TreeStage {
  static constexpr int BP = KP::per16 == 8 ? 2 : 1;
  static constexpr int kTile = 16 * HD * static_cast<int>(sizeof(typename KP::elem)) / 16;  // 16-byte pieces of a tile
  static constexpr int kPieces = 2 * BP * kTile;                                             // of a step
  static constexpr int kPer = kPieces / 256;                                                 // per thread
};

// Work-group: a request's column group of 64 NT columns (16 NT per wave) over
// the blocks of one split.  The blocks of step s + 1 are on their way into
// registers while step s is computed from LDS, and go to the other LDS buffer
// after it: one barrier per step.
template <class KP, class IO, int HD, int NT>
__global__ __launch_bounds__(256) void k_tree_attn_shared(TreeAttnArgs a) {
  using Stage = TreeStage<KP, HD>;
  using Parts = TreeParts<KP, IO>;
  constexpr int BP = Stage::BP, NF = HD / KP::kblk, NV = Stage::kTile / 64, NE = HD / 16, CW = 64 * NT;
  __shared__ uint4 buf[2][Stage::kPieces];
  __shared__ int odd_s[2], last;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane & 15, g = lane >> 4;
  const int f = blockIdx.y, kvh = blockIdx.x;
  const TreeItem t = tree_item(a, f);
  const int end = t.first + t.count, c0 = CW * t.cg + 16 * NT * wave;
  const bool busy = c0 < t.cols;  // this wave has columns

  uint4 Q[NT][NF][Parts::q];
  uint64_t anc[NT];
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    const TreeColumn col = tree_column(a, t.row0, kvh, min(c0 + 16 * jt + h, t.cols - 1));
    anc[jt] = a.anc[col.row];
#pragma unroll
    for (int c = 0; c < NF; ++c) load_query<KP, IO, HD>(a, col, c, g, Q[jt][c]);
  }
  f32x4_t O[NT][NE];
  float m[NT], l[NT];
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    m[jt] = kTreeFloor;
    l[jt] = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) O[jt][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  int ids = 0;
  uint4 next[Stage::kPer];
  // Pieces of the step from block i on: this thread's 16 bytes of each 4 KiB.
  const auto fetch = [&](int i) {
    const int k = i - t.first;
    if ((k & 63) == 0) ids = block_id(a, t.btrow, i + lane, end);
#pragma unroll
    for (int r = 0; r < Stage::kPer; ++r) {
      const int piece = r * 256 + tid;
      // The tile is the same for all lanes of a wave.
      const int which = __builtin_amdgcn_readfirstlane(piece / Stage::kTile), b = which % BP;
      const size_t tile = static_cast<size_t>(__builtin_amdgcn_readlane(ids, (i + b < end ? k + b : k) & 63)) * a.Hkv + kvh;
      const char* base = static_cast<const char*>(which < BP ? a.kc : a.vc) + tile * Stage::kTile * 16;
      next[r] = reinterpret_cast<const uint4*>(base)[piece % Stage::kTile];
    }
  };
  // Into LDS; V pieces of a masked step without stale positions and without
  // infinite or NaN values.
  const auto put = [&](int i, int to) {
    bool odd = false;
    const bool tail = 16 * (i + BP) > t.len || i + BP > end;
#pragma unroll
    for (int r = 0; r < Stage::kPer; ++r) {
      const int piece = r * 256 + tid;
      const int which = __builtin_amdgcn_readfirstlane(piece / Stage::kTile), b = which % BP;
      if (tail && which >= BP) {
        // Piece n of a V tile: positions 4 g .. 4 g + 3 with g = n / 16 % 4.
        const int gp = piece % Stage::kTile / 16 % 4;
        keep_piece<KP>(next[r], i + b < end ? live_bits(16 * (i + b) + 4 * gp, t.total) : 0u);
        odd |= clean_piece<KP>(next[r]);
      }
      buf[to][piece] = next[r];
    }
    if (tail && __ballot(odd) != 0 && lane == 0) odd_s[to] = 1;
  };

  if (tid < 2) odd_s[tid] = 0;
  __syncthreads();
  fetch(t.first);
  put(t.first, 0);
  for (int i = t.first; i < end; i += BP) {
    const int at = (i - t.first) / BP & 1;
    __syncthreads();  // step i is in buf[at]; the other buffer has been read
    if (i + BP < end) fetch(i + BP);
    if (busy) {
      const bool tail = 16 * (i + BP) > t.len || i + BP > end;
      const uint4* kb = buf[at] + lane;
      const uint4* vb = buf[at] + BP * Stage::kTile + lane;
      f32x4_t S[NT][BP];
#pragma unroll
      for (int jt = 0; jt < NT; ++jt)
#pragma unroll
        for (int b = 0; b < BP; ++b) S[jt][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NF; ++c)
#pragma unroll
        for (int b = 0; b < BP; ++b) {
          const uint4 x = kb[b * Stage::kTile + c * 64];
#pragma unroll
          for (int jt = 0; jt < NT; ++jt)
#pragma unroll
            for (int q = 0; q < Parts::q; ++q) S[jt][b] = KP::mma(S[jt][b], x, Q[jt][c][q]);
        }
      uint32_t live[BP], sees[NT][BP];
      if (tail) {
#pragma unroll
        for (int b = 0; b < BP; ++b) {
          const int pos = 16 * (i + b) + 4 * g;
          live[b] = i + b < end ? live_bits(pos, t.total) : 0u;
#pragma unroll
          for (int jt = 0; jt < NT; ++jt) {
            sees[jt][b] = live[b] & seen_bits(pos, t.len, anc[jt]);
#pragma unroll
            for (int r = 0; r < 4; ++r) S[jt][b][r] = sees[jt][b] >> r & 1 ? S[jt][b][r] : -INFINITY;
          }
        }
      }
      float p[NT][BP][4];
#pragma unroll
      for (int jt = 0; jt < NT; ++jt) softmax_step<BP, NE>(S[jt], a.qscale, m[jt], l[jt], O[jt], p[jt]);
      if constexpr (KP::per16 == 8) {
        uint4 pp[NT][Parts::p];
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) {
          float v[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) v[r] = p[jt][r / 4][r % 4];
#pragma unroll
          for (int q = 0; q < Parts::p; ++q) pp[jt][q] = next_part<BF16>(v);
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
          const uint4 v0 = vb[c * 64], v1 = vb[Stage::kTile + c * 64];
          const uint4 a0 = make_uint4(v0.x, v0.y, v1.x, v1.y), a1 = make_uint4(v0.z, v0.w, v1.z, v1.w);
#pragma unroll
          for (int jt = 0; jt < NT; ++jt)
#pragma unroll
            for (int q = 0; q < Parts::p; ++q) {
              O[jt][2 * c] = BF16::mma(O[jt][2 * c], a0, pp[jt][q]);
              O[jt][2 * c + 1] = BF16::mma(O[jt][2 * c + 1], a1, pp[jt][q]);
            }
        }
      } else {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
          const uint4 x = vb[c * 64];
#pragma unroll
          for (int jt = 0; jt < NT; ++jt) {
            const float* pj = p[jt][0];
            O[jt][c] = F32::mma(O[jt][c], x, make_uint4(__float_as_uint(pj[0]), __float_as_uint(pj[1]),
                                                         __float_as_uint(pj[2]), __float_as_uint(pj[3])));
          }
        }
      }
      if (tail && odd_s[at]) {
        size_t tile[BP];
#pragma unroll
        for (int b = 0; b < BP; ++b)
          tile[b] = static_cast<size_t>(block_id(a, t.btrow, min(i + b, end - 1), end)) * a.Hkv + kvh;
#pragma unroll
        for (int jt = 0; jt < NT; ++jt)
          add_odd_values<KP, HD, BP>(O[jt], p[jt], sees[jt], a.vc, tile, live, lane);
      }
    }
    if (i + BP < end) put(i + BP, at ^ 1);
  }

  const CoherentBuffer pb(a.part, a.part_bytes);
  const uint32_t item = (static_cast<uint32_t>(f) * a.Hkv + kvh) * CW * (HD + 4) * 4;
  if (busy) {
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
      float L = l[jt];
      L += __shfl_xor(L, 16);
      L += __shfl_xor(L, 32);
      const int c = 16 * (NT * wave + jt) + h;  // within the group
      if (CW * t.cg + c >= t.cols) continue;
      const TreeColumn col = tree_column(a, t.row0, kvh, CW * t.cg + c);
      const float inv = 1.f / L;
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const int d0 = 16 * e + 4 * g;
        if (t.nsplit == 1) IO::store4(a, col.row, col.hq * HD + d0, O[jt][e] * inv);
        else pb.store4(item + (c * (HD + 4) + 4 + d0) * 4, O[jt][e]);
      }
      if (t.nsplit > 1 && g == 0) pb.store4(item + c * (HD + 4) * 4, f32x4_t{m[jt], L, 0.f, 0.f});
    }
  }
  if (t.nsplit > 1) merge_splits<IO, HD, CW>(a, t, kvh, pb, &last);
}

}  // namespace sprk
