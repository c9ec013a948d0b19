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
// error on it).  A bf16 output takes them in two parts: 2^-16 of a probability
// is left out, so its error is the output's one rounding (2 x 24000 positions:
// 0.00166 of the outputs' norm; with one part 0.0023).
//
// The running maximum of a column is raised only when a step exceeds it by
// kRaise (in log2 units): until then probabilities of at most 2^kRaise stay
// exact enough in fp32, and steps need neither the exchange between lanes nor
// the rescaling of O (512 columns over 2 x 24000 positions: 180 us, raised at
// every larger score 196).
//
// Two kernels.  Both cut a request's blocks into KV splits, one work-group
// each, and write a partial result where a request has several:
//   k_tree_attn         up to 32 columns: the four waves of a work-group take
//                       runs of blocks, K and V go straight into registers.
//                       Bound by the cache's bytes: 32 requests of 32 heads,
//                       4 nodes, about 470 positions (bf16 cache of 253 MB):
//                       45 us, 5.6 TB/s.  One request of 600 positions and 9
//                       nodes: 9.6 us, nearly all of it latency (arguments,
//                       block ids, blocks, merge, one after the other).
//   k_tree_attn_shared  more: the four waves take 16 NT columns each and share
//                       every block through LDS, so the cache is read once per
//                       64 NT columns and a wave's work per byte stays high
//                       (64 columns on the other kernel's plan: 110 us where
//                       this took 78 at first; 512 columns: 504 and 227).
//                       Bound by the matrix
//                       unit in fp32 (64 columns, 16 x 5632 positions: 236 us,
//                       100 of 154 TFLOP/s), by products, exponentials and LDS
//                       reads in turn in bf16 (512 columns, 2 x 24000 positions:
//                       175 us, 575 TFLOP/s of the formula's products, half as
//                       many again for the probabilities' second part; with one
//                       part 147 us), and at short contexts by its ends:
//                       several trips to memory until the first step runs, 8 to
//                       9 us of merge at its end.
// The partials are merged by the split that arrives last where that is little,
// else by k_tree_merge.  (With 64 columns and more in that one work-group, and
// one-part probabilities: 512 columns over 2 x 6000 positions 65 us, with
// k_tree_merge 51; with two parts now 57.)
#pragma once

#include <type_traits>

#include "gemm_kernels.h"
#include "lds_pipe.h"
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
  int apart;           // splits are merged by k_tree_merge
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

// Two values rounded to bf16 (nearest even), the first in the low half: one
// conversion instruction.
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{lo, hi}), bf16x2_t));
}

// Formats of q and out (kRaw: bf16, which a bf16 cache's operand takes as it is).
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
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + row * a.os + n0) =
        make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
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
      w[j] = bf16_pair(v[2 * j], v[2 * j + 1]);
      v[2 * j] -= __uint_as_float(w[j] << 16);
      v[2 * j + 1] -= __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A V word without its infinite and NaN values; odd is raised where it had one.
template <class KP>
__device__ __forceinline__ uint32_t clean_word(uint32_t x, uint32_t& odd) {
  if constexpr (KP::per16 == 4) {
    const bool o = (x & 0x7F800000u) == 0x7F800000u;
    odd |= o ? 1u : 0u;
    return o ? 0u : x;
  } else {
    const uint32_t keep = ((x & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((x & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
    odd |= ~keep;
    return x & keep;
  }
}
template <class KP>
__device__ __forceinline__ u32x4_t clean_piece(u32x4_t u, uint32_t& odd) {
  return u32x4_t{clean_word<KP>(u.x, odd), clean_word<KP>(u.y, odd), clean_word<KP>(u.z, odd), clean_word<KP>(u.w, odd)};
}

// A 16-byte V piece (positions 4 g .. 4 g + 3 of its block) without the
// positions whose bit of keep is clear.
template <class KP>
__device__ __forceinline__ u32x4_t keep_piece(u32x4_t u, uint32_t keep) {
  if constexpr (KP::per16 == 4) {
    return u32x4_t{keep & 1 ? u.x : 0u, keep & 2 ? u.y : 0u, keep & 4 ? u.z : 0u, keep & 8 ? u.w : 0u};
  } else {
    const uint32_t m01 = (keep & 1 ? 0xFFFFu : 0u) | (keep & 2 ? 0xFFFF0000u : 0u);
    const uint32_t m23 = (keep & 4 ? 0xFFFFu : 0u) | (keep & 8 ? 0xFFFF0000u : 0u);
    return u32x4_t{u.x & m01, u.y & m23, u.z & m01, u.w & m23};
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
// columns that do.  One step's blocks (tile0, tile1) of one KV head, p and sees as the
// step's scores are held; values are read again, element by element.
template <class KP, int HD, int BP>
__device__ __forceinline__ void add_odd_values(f32x4_t* O, const float (*p)[4], const uint32_t* sees, const void* vc,
                                               size_t tile0, size_t tile1, const uint32_t* live, int lane) {
  const int h = lane & 15, g = lane >> 4;
#pragma unroll 1
  for (int t = 0; t < 16 * BP; ++t) {
    const int b = t >> 4, gt = t >> 2 & 3, r = t & 3;
    float pt = 0.f;
    uint32_t st = 0, lt = 0;
    const size_t at = b == 0 ? tile0 : tile1;
#pragma unroll
    for (int k = 0; k < BP; ++k)
      if (k == b) {
        pt = r == 0 ? p[k][0] : r == 1 ? p[k][1] : r == 2 ? p[k][2] : p[k][3];
        st = sees[k];
        lt = live[k];
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
  u32x4_t k0[NF], k1[NF], v0[NV], v1[NV];

  static __device__ __forceinline__ const u32x4_t* tile_at(const void* pool, size_t tile, int lane) {
    return reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(pool) + tile * 16 * HD) + lane;
  }
  __device__ __forceinline__ void load_k(const void* kc, size_t t0, size_t t1, int lane) {
    const u32x4_t *p0 = tile_at(kc, t0, lane), *p1 = tile_at(kc, t1, lane);
#pragma unroll
    for (int f = 0; f < NF; ++f) k0[f] = __builtin_nontemporal_load(p0 + f * 64);
#pragma unroll
    for (int f = 0; f < NF; ++f) k1[f] = __builtin_nontemporal_load(p1 + f * 64);
  }
  __device__ __forceinline__ void load_v(const void* vc, size_t t0, size_t t1, int lane) {
    const u32x4_t *p0 = tile_at(vc, t0, lane), *p1 = tile_at(vc, t1, lane);
#pragma unroll
    for (int f = 0; f < NV; ++f) v0[f] = __builtin_nontemporal_load(p0 + f * 64);
#pragma unroll
    for (int f = 0; f < NV; ++f) v1[f] = __builtin_nontemporal_load(p1 + f * 64);
  }
  // S[b] += K block b . x for K-block c.
  __device__ __forceinline__ void qk(f32x4_t* S, int c, const uint4& x) const {
    S[0] = BF16::mma(S[0], __builtin_bit_cast(uint4, k0[c]), x);
    S[1] = BF16::mma(S[1], __builtin_bit_cast(uint4, k1[c]), x);
  }
  // Zeroes the values of this lane's positions 4 g + i of block b whose bit i
  // of keep[b] is clear, and infinite and NaN ones; returns whether this lane
  // had one of the latter.
  __device__ __forceinline__ bool mask_v(const uint32_t* keep) {
    uint32_t odd = 0;
#pragma unroll
    for (int f = 0; f < NV; ++f) {
      v0[f] = clean_piece<BF16>(keep_piece<BF16>(v0[f], keep[0]), odd);
      v1[f] = clean_piece<BF16>(keep_piece<BF16>(v1[f], keep[1]), odd);
    }
    return odd != 0;
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
      const uint4 a0 = make_uint4(v0[f].x, v0[f].y, v1[f].x, v1[f].y);
      const uint4 a1 = make_uint4(v0[f].z, v0[f].w, v1[f].z, v1[f].w);
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
  u32x4_t k[NF], v[NV];

  static __device__ __forceinline__ const u32x4_t* tile_at(const void* pool, size_t tile, int lane) {
    return reinterpret_cast<const u32x4_t*>(static_cast<const float*>(pool) + tile * 16 * HD) + lane;
  }
  __device__ __forceinline__ void load_k(const void* kc, size_t t0, size_t, int lane) {
    const u32x4_t* p0 = tile_at(kc, t0, lane);
#pragma unroll
    for (int f = 0; f < NF; ++f) k[f] = __builtin_nontemporal_load(p0 + f * 64);
  }
  __device__ __forceinline__ void load_v(const void* vc, size_t t0, size_t, int lane) {
    const u32x4_t* p0 = tile_at(vc, t0, lane);
#pragma unroll
    for (int f = 0; f < NV; ++f) v[f] = __builtin_nontemporal_load(p0 + f * 64);
  }
  __device__ __forceinline__ void qk(f32x4_t* S, int c, const uint4& x) const {
    S[0] = F32::mma(S[0], __builtin_bit_cast(uint4, k[c]), x);
  }
  __device__ __forceinline__ bool mask_v(const uint32_t* keep) {
    uint32_t odd = 0;
#pragma unroll
    for (int f = 0; f < NV; ++f) v[f] = clean_piece<F32>(keep_piece<F32>(v[f], keep[0]), odd);
    return odd != 0;
  }
  template <int PP>
  __device__ __forceinline__ void pv(f32x4_t* O, const float (*p)[4]) const {
#pragma unroll
    for (int f = 0; f < NV; ++f) {
      O[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[f].x), p[0][0], O[f], 0, 0, 0);
      O[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[f].y), p[0][1], O[f], 0, 0, 0);
      O[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[f].z), p[0][2], O[f], 0, 0, 0);
      O[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[f].w), p[0][3], O[f], 0, 0, 0);
    }
  }
};

// Parts of q and of the probabilities by cache and io format.
template <class KP, class IO>
struct TreeParts {
  static constexpr int q = KP::per16 == 4 || IO::kRaw ? 1 : 3;
  static constexpr int p = KP::per16 == 4 ? 1 : IO::kRaw ? 2 : 3;
};

template <class KP, class IO, int HD, int NT>
struct TreeSmem {
  static constexpr int NF = HD / KP::kblk;
  union {
    uint4 q[NT][NF][TreeParts<KP, IO>::q][64];
    f32x4_t so[4][HD / 16][64];
    float weights[kTreeSplits * 16 * NT];
  };
  float2 sml[4][NT][16];
  int last;
};

// Running maximum before the first score: below every finite one (a score times
// log2(e) / 8 stays above -6.2e37), and finite, so that a masked score less it is
// -infinity and not NaN.
constexpr float kTreeFloor = -1e38f;
constexpr float kRaise = 8.f;

// Column c of a request (c < its nodes * G): token row and query head.
struct TreeColumn {
  int row, hq;
};
__device__ __forceinline__ TreeColumn tree_column(const TreeAttnArgs& a, int row0, int kvh, int c) {
  const int node = c / a.G;
  return TreeColumn{row0 + node, kvh * a.G + c - node * a.G};
}

// This lane's piece (K-block c, group g) of one column's query: as it is stored,
// and in the operand's parts.
struct QueryPiece {
  uint4 x, y;
};
template <class KP, class IO, int HD>
__device__ __forceinline__ QueryPiece load_query(const TreeAttnArgs& a, const TreeColumn& col, int c, int g) {
  const typename IO::elem* src =
      static_cast<const typename IO::elem*>(a.q) + col.row * a.qs + col.hq * HD + c * KP::kblk + g * KP::per16;
  QueryPiece p{};
  if constexpr (IO::kRaw && KP::per16 == 4) {
    const uint2 u = *reinterpret_cast<const uint2*>(src);
    p.x.x = u.x;
    p.x.y = u.y;
  } else {
    p.x = *reinterpret_cast<const uint4*>(src);
    if constexpr (!IO::kRaw && KP::per16 == 8) p.y = *reinterpret_cast<const uint4*>(src + 4);
  }
  return p;
}
template <class KP, class IO>
__device__ __forceinline__ void query_parts(const QueryPiece& p, uint4* out) {
  if constexpr (IO::kRaw == (KP::per16 == 8)) {  // stored as the operand takes it
    out[0] = p.x;
  } else if constexpr (IO::kRaw) {
    out[0] = make_uint4(p.x.x << 16, p.x.x & 0xFFFF0000u, p.x.y << 16, p.x.y & 0xFFFF0000u);
  } else {
    const uint32_t w[8] = {p.x.x, p.x.y, p.x.z, p.x.w, p.y.x, p.y.y, p.y.z, p.y.w};
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
#pragma unroll
    for (int q = 0; q < TreeParts<KP, IO>::q; ++q) out[q] = next_part<KP>(v);
  }
}

// Online softmax of one column tile's scores of one step: turns S into
// probabilities, adds them to l, and raises the running maximum first where a
// score exceeds it by more than kRaise.  (The test runs on the exponents, which
// are needed anyway.)
template <int BP, int NE>
__device__ __forceinline__ void softmax_step(const f32x4_t* S, float qscale, float& m, float& l, f32x4_t* O, float (*p)[4]) {
  const auto highest = [](const float (*x)[4]) {
    float v = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3]));
#pragma unroll
    for (int b = 1; b < BP; ++b) v = fmaxf(fmaxf(v, fmaxf(x[b][0], x[b][1])), fmaxf(x[b][2], x[b][3]));
    return v;
  };
#pragma unroll
  for (int b = 0; b < BP; ++b)
#pragma unroll
    for (int r = 0; r < 4; ++r) p[b][r] = fmaf(S[b][r], qscale, -m);
  if (__ballot(highest(p) > kRaise) != 0) {
#pragma unroll
    for (int b = 0; b < BP; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) p[b][r] = S[b][r] * qscale;
    float mx = highest(p);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float up = fmaxf(m, mx);
    const float alpha = __builtin_amdgcn_exp2f(m - up);
    l *= alpha;
    m = up;
#pragma unroll
    for (int e = 0; e < NE; ++e) O[e] *= alpha;
#pragma unroll
    for (int b = 0; b < BP; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) p[b][r] = fmaf(S[b][r], qscale, -m);
  }
#pragma unroll
  for (int b = 0; b < BP; ++b) {
#pragma unroll
    for (int r = 0; r < 4; ++r) p[b][r] = __builtin_amdgcn_exp2f(p[b][r]);
    l += (p[b][0] + p[b][1]) + (p[b][2] + p[b][3]);
  }
}

// What a work item is: its request, blocks and columns.
struct TreeItem {
  int cg, cg0, nsplit, ncg, item0;
  int len, total, nblk, row0, cols;
  int first, count;          // blocks of the split
  const int32_t* btrow;
};
__device__ __forceinline__ TreeItem tree_item(const TreeAttnArgs& a, int f) {
  const int lane = threadIdx.x & 63;
  TreeItem t;
  // Lane = request, all of it at once: one trip to memory.
  const int r = min(lane, a.n - 1);
  const int item0 = a.item0[r], item1 = a.item0[r + 1], slot = a.slot[r], len = a.len[r];
  const int nodes = a.nodes[r], ncg = a.ncg[r], row0 = a.row0[r], cg0 = a.cg0[r];
  // Request: the number of requests whose items all precede f.
  const int rank = __popcll(__ballot(lane < a.n && item1 <= f));
  const auto mine = [&](int v) { return __builtin_amdgcn_readlane(v, rank); };
  t.ncg = mine(ncg);
  t.cg0 = mine(cg0);
  t.item0 = mine(item0);
  const int w = f - t.item0, s = w / t.ncg;
  t.cg = w - s * t.ncg;  // column groups of one split run side by side and share its blocks
  t.nsplit = (mine(item1) - t.item0) / t.ncg;
  t.len = mine(len);
  const int n = mine(nodes);
  t.total = t.len + n;
  t.nblk = (t.total + 15) >> 4;
  t.row0 = mine(row0);
  t.cols = n * a.G;
  t.first = a.bps * s;
  t.count = min(t.nblk - t.first, a.bps);
  t.btrow = a.bt + static_cast<size_t>(mine(slot)) * a.mb;
  return t;
}

// A block id from the table; one outside the pool is reported and reads block 0.
__device__ __forceinline__ int in_pool(const TreeAttnArgs& a, int id) {
  if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.nb)) {
    raise_check(a.err, kErrBlockId);
    id = 0;
  }
  return id;
}
// Id of block i (< end) of the table row.
__device__ __forceinline__ int block_id(const TreeAttnArgs& a, const int32_t* btrow, int i, int end) {
  return in_pool(a, i < end ? btrow[i] : 0);
}

// Counts a split in and, in the one that arrives last, merges all partials of
// its column group (CW columns): no work-group waits on another.  The
// caller's partials are stored (agent-coherent).  weights: LDS for kTreeSplits
// * CW floats that no wave reads or writes any more.
template <class IO, int HD, int CW>
__device__ __forceinline__ void merge_splits(const TreeAttnArgs& a, const TreeItem& t, int kvh, const CoherentBuffer& pb,
                                             int* last, float* weights) {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's partial stores are complete
  __syncthreads();
  int32_t* cnt = a.cnt + (t.cg0 + t.cg) * a.Hkv + kvh;
  if (threadIdx.x == 0)
    *last = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == t.nsplit - 1;
  __syncthreads();
  if (!*last) return;
  if (threadIdx.x == 0) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const uint32_t base = (static_cast<uint32_t>(t.item0 + t.cg) * a.Hkv + kvh) * CW * (HD + 4) * 4;
  const uint32_t stride = static_cast<uint32_t>(t.ncg) * a.Hkv * CW * (HD + 4) * 4;
  const int c0 = CW * t.cg, mine = min(t.cols - c0, CW);
  // Weight of each (split, column), exp2(m - M) / L, in LDS: lanes of one
  // column side by side, kLanes each.
  constexpr int kLanes = 256 / CW >= 4 ? 256 / CW : 4;
  for (int c = threadIdx.x / kLanes; c < CW; c += 256 / kLanes) {
    const uint32_t at = base + min(c, mine - 1) * (HD + 4) * 4;
    float M = kTreeFloor, L = 0.f;
    for (int s = threadIdx.x % kLanes; s < t.nsplit; s += kLanes) {
      const f32x4_t ml = pb.load4(at + s * stride);
      const float up = fmaxf(M, ml[0]);
      L = L * __builtin_amdgcn_exp2f(M - up) + ml[1] * __builtin_amdgcn_exp2f(ml[0] - up);
      M = up;
      weights[s * CW + c] = ml[0];
    }
#pragma unroll
    for (int o = kLanes / 2; o >= 1; o >>= 1) {
      const float m2 = __shfl_xor(M, o), l2 = __shfl_xor(L, o), up = fmaxf(M, m2);
      L = L * __builtin_amdgcn_exp2f(M - up) + l2 * __builtin_amdgcn_exp2f(m2 - up);
      M = up;
    }
    const float inv = 1.f / L;
    for (int s = threadIdx.x % kLanes; s < t.nsplit; s += kLanes)
      weights[s * CW + c] = __builtin_amdgcn_exp2f(weights[s * CW + c] - M) * inv;
  }
  __syncthreads();
  // Outputs, 16 bytes each: kItems per thread and kSplits partials of each in flight.
  constexpr int kItems = CW * HD / 4 / 256 >= 4 ? 4 : CW * HD / 4 / 256, kChunk = 4;
  for (int x0 = threadIdx.x; x0 < mine * (HD / 4); x0 += 256 * kItems) {
    f32x4_t R[kItems];
    uint32_t at[kItems];
    int c[kItems];
#pragma unroll
    for (int n = 0; n < kItems; ++n) {
      const int idx = min(x0 + 256 * n, mine * (HD / 4) - 1);
      c[n] = idx / (HD / 4);
      at[n] = base + (c[n] * (HD + 4) + 4 + idx % (HD / 4) * 4) * 4;
      R[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    for (int s0 = 0; s0 < t.nsplit; s0 += kChunk) {
      f32x4_t o[kItems][kChunk];
#pragma unroll
      for (int k = 0; k < kChunk; ++k)
#pragma unroll
        for (int n = 0; n < kItems; ++n) o[n][k] = pb.load4(at[n] + min(s0 + k, t.nsplit - 1) * stride);
#pragma unroll
      for (int k = 0; k < kChunk; ++k)
        if (s0 + k < t.nsplit) {
#pragma unroll
          for (int n = 0; n < kItems; ++n) R[n] += weights[(s0 + k) * CW + c[n]] * o[n][k];
        }
    }
#pragma unroll
    for (int n = 0; n < kItems; ++n) {
      const int idx = x0 + 256 * n;
      if (idx >= mine * (HD / 4)) break;
      const TreeColumn col = tree_column(a, t.row0, kvh, c0 + c[n]);
      IO::store4(a, col.row, col.hq * HD + idx % (HD / 4) * 4, R[n]);
    }
  }
}

template <class KP, class IO, int HD, int NT>
__global__ __launch_bounds__(256, NT == 1 ? 3 : 2) void k_tree_attn(TreeAttnArgs a) {
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
    query_parts<KP, IO>(load_query<KP, IO, HD>(a, tree_column(a, t.row0, kvh, min(16 * jt + h, t.cols - 1)), c, g), x);
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

  // The step's K registers take the next step's keys as soon as its scores are
  // there, the V registers the next values after its products: a wave always
  // has loads in flight, in the registers of one step.
  Step B;
  size_t t0 = 0, t1 = 0;  // tiles of the blocks that are being loaded
  const auto block_tile = [&](int i) {
    return static_cast<size_t>(__builtin_amdgcn_readlane(ids, (i - lo) & 63)) * a.Hkv + kvh;
  };
  const auto next_tiles = [&](int i) {
    if (((i - lo) & 63) == 0 && i != lo) ids = block_id(a, t.btrow, i + lane, hi);
    t0 = block_tile(i);
    if constexpr (BP == 2) t1 = block_tile(i + 1 < hi ? i + 1 : i);  // a missing second block re-reads the first, masked
  };
  if (lo < hi) {
    next_tiles(lo);
    B.load_k(a.kc, t0, t1, lane);
    B.load_v(a.vc, t0, t1, lane);
  }
  for (int i = lo; i < hi; i += BP) {
    const bool more = i + BP < hi;
    f32x4_t S[NT][BP];
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
#pragma unroll
      for (int b = 0; b < BP; ++b) S[jt][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NF; ++c)
#pragma unroll
        for (int q = 0; q < Parts::q; ++q) {
          B.qk(S[jt], c, sm.q[jt][c][q][lane]);
        }
    }
    const size_t now0 = t0, now1 = t1;
    if (more) {
      next_tiles(i + BP);
      B.load_k(a.kc, t0, t1, lane);
    }
    // A step that reaches past the cached positions or the run is masked.
    const bool tail = 16 * (i + BP) > t.len || i + BP > hi;
    uint32_t live[BP], sees[NT][BP];  // bits of this lane's positions: cached or a node; seen by the column
    bool odd = false;
    if (tail) {
#pragma unroll
      for (int b = 0; b < BP; ++b) {
        const int pos = 16 * (i + b) + 4 * g;
        live[b] = i + b < hi ? live_bits(pos, t.total) : 0u;
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) {
          sees[jt][b] = live[b] & seen_bits(pos, t.len, anc[jt]);
#pragma unroll
          for (int r = 0; r < 4; ++r) S[jt][b][r] = sees[jt][b] >> r & 1 ? S[jt][b][r] : -INFINITY;
        }
      }
      odd = __ballot(B.mask_v(live)) != 0;
    }
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
      float p[BP][4];
      softmax_step<BP, NE>(S[jt], a.qscale, m[jt], l[jt], O[jt], p);
      B.template pv<Parts::p>(O[jt], p);
      if (odd) add_odd_values<KP, HD, BP>(O[jt], p, sees[jt], a.vc, now0, now1, live, lane);
    }
    if (more) B.load_v(a.vc, t0, t1, lane);
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
  if (t.nsplit > 1 && !a.apart) merge_splits<IO, HD, CW>(a, t, kvh, pb, &sm.last, sm.weights);
}

// ---------------------------------------------------------------------------

// One step's blocks in LDS, two steps deep: the K tiles in their own order
// (fragment by fragment), then the V operands.  For bf16 an operand's lane
// holds its 8 bytes of block 0 and of block 1 side by side, as the 16x16x32
// product takes them.
template <class KP, int HD>
struct TreeStage {
  static constexpr int BP = KP::per16 == 8 ? 2 : 1;
  static constexpr int kTile = 16 * HD * static_cast<int>(sizeof(typename KP::elem)) / 16;  // 16-byte pieces of a tile
  static constexpr int kPieces = 2 * BP * kTile;                                             // of a step
  static constexpr int kPer = kPieces / 256;                                                 // per thread
  static_assert(kPer >= 2 && (kTile % 256 == 0 || kTile == 128), "pieces of a wave lie in one tile");
};

// Work-group: a request's column group of 64 NT columns (16 NT per wave) over
// the blocks of one split.  While a step is computed from LDS, the next one's
// blocks lie in registers or arrive there, and the one's after it are asked
// for; after the step the next one goes to the other LDS buffer: one barrier
// per step.  Steps that reach past the cached positions or the split (the last
// few) run masked, the others without a test.
//
// Work-groups of a CU: three with fp32 operands (16 x 5632 positions, 64 columns:
// 236 us, with two 241; 128 columns, 8 x 6000: 222 and 230; but 16 x 704: 46 and
// 44), two with bf16 ones (16 x 5632: 85 us, with three 89; 16 x 704: 21.6 and
// 26; with 128 columns three leave too few registers, 8 x 6000: 66 and 137).
template <class KP>
constexpr int kSharedPerCu = KP::per16 == 4 ? 3 : 2;
template <class KP, class IO, int HD, int NT>
__global__ __launch_bounds__(256, kSharedPerCu<KP>) void k_tree_attn_shared(TreeAttnArgs a) {
  using Stage = TreeStage<KP, HD>;
  using Parts = TreeParts<KP, IO>;
  constexpr int BP = Stage::BP, NF = HD / KP::kblk, NE = HD / 16, CW = 64 * NT;
  __shared__ uint4 lds[2 * Stage::kPieces];  // two steps
  __shared__ int odd_s[2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane & 15, g = lane >> 4;
  const int f = blockIdx.y, kvh = blockIdx.x;
  const TreeItem t = tree_item(a, f);
  const int end = t.first + t.count, c0 = CW * t.cg + 16 * NT * wave;
  const bool busy = c0 < t.cols;  // this wave has columns

  // Block ids are asked for one step before the blocks they name; past the
  // split's end they are its last one's, so that every fetch reads the cache (a
  // missing second block re-reads the first, masked).
  int ids[BP];
  const auto ask = [&](int i) {
#pragma unroll
    for (int b = 0; b < BP; ++b) ids[b] = t.btrow[min(i + b, end - 1)];
  };
  ask(t.first);

  uint4 Q[NT][NF][Parts::q];
  uint64_t anc[NT];
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    const TreeColumn col = tree_column(a, t.row0, kvh, min(c0 + 16 * jt + h, t.cols - 1));
    anc[jt] = a.anc[col.row];
#pragma unroll
    for (int c = 0; c < NF; ++c) query_parts<KP, IO>(load_query<KP, IO, HD>(a, col, c, g), Q[jt][c]);
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

  // Piece r of this thread: piece r * 256 + tid of the step, in tile r * 256 /
  // kTile (of 128 pieces: plus the wave's half); K tiles first.
  const int half = Stage::kTile == 128 ? wave >> 1 : 0;
  const int in_tile = tid % Stage::kTile;
  constexpr int kRounds = Stage::kTile >= 256 ? Stage::kTile / 256 : 1;  // rounds of 256 pieces per tile
  const auto round_tile = [&](int r) { return Stage::kTile == 128 ? 2 * r + half : r / kRounds; };
  const auto round_piece = [&](int r) { return in_tile + (r % kRounds) * 256; };

  u32x4_t next[2][Stage::kPer];  // of even and odd steps
  // The blocks whose ids were asked for, then the ids of the step at `then`.
  const auto fetch = [&](int then, auto parity) {
    uint64_t at[BP];
#pragma unroll
    for (int b = 0; b < BP; ++b)
      at[b] = (static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(in_pool(a, ids[b]))) * a.Hkv + kvh) * (Stage::kTile * 16);
    ask(then);
#pragma unroll
    for (int r = 0; r < Stage::kPer; ++r) {
      const int which = round_tile(r);
      const char* pool = static_cast<const char*>(r * 256 / Stage::kTile < BP ? a.kc : a.vc);
      const char* base = pool + (BP == 2 && which % 2 == 1 ? at[BP - 1] : at[0]);
      next[decltype(parity)::value][r] = reinterpret_cast<const u32x4_t*>(base)[round_piece(r)];
    }
  };
  // Into LDS.  tail: V pieces without stale positions and without infinite or
  // NaN values.
  const auto put = [&](int i, auto parity, auto tail) {
    constexpr int to = decltype(parity)::value;
    uint32_t odd = 0;
#pragma unroll
    for (int r = 0; r < Stage::kPer; ++r) {
      const int which = round_tile(r), n = round_piece(r);
      u32x4_t x = next[to][r];
      if (r * 256 / Stage::kTile < BP) {
        lds[to * Stage::kPieces + which * Stage::kTile + n] = __builtin_bit_cast(uint4, x);
        continue;
      }
      const int b = which - BP;
      if constexpr (decltype(tail)::value) {
        // Piece n of a V tile: positions 4 g .. 4 g + 3 with g = n / 16 % 4.
        const uint32_t live = i + b < end ? live_bits(16 * (i + b) + 4 * (n / 16 % 4), t.total) : 0u;
        x = clean_piece<KP>(keep_piece<KP>(x, live), odd);
      }
      uint4* v = lds + to * Stage::kPieces + BP * Stage::kTile;
      if constexpr (BP == 1) {
        v[n] = __builtin_bit_cast(uint4, x);
      } else {
        // Load n / 64 holds operands 2 (n / 64) and 2 (n / 64) + 1.
        uint2* op = reinterpret_cast<uint2*>(v + (n / 64) * 128 + n % 64) + b;
        op[0] = make_uint2(x.x, x.y);
        op[128] = make_uint2(x.z, x.w);
      }
    }
    if constexpr (decltype(tail)::value)
      if (__ballot(odd != 0) != 0 && lane == 0) odd_s[to] = 1;
  };
  const auto is_tail = [&](int i) { return 16 * (i + BP) > t.len || i + BP > end; };
  const auto compute = [&](int i, auto parity, auto tail) {
    constexpr int at = decltype(parity)::value;
    const uint4* kb = lds + at * Stage::kPieces + lane;
    const uint4* vb = kb + BP * Stage::kTile;
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
        for (int q = 0; q < Parts::q; ++q)
#pragma unroll
          for (int jt = 0; jt < NT; ++jt) S[jt][b] = KP::mma(S[jt][b], x, Q[jt][c][q]);
      }
    uint32_t live[BP], sees[NT][BP];
    if constexpr (decltype(tail)::value) {
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
    if constexpr (BP == 2) {
      uint4 pp[NT][Parts::p];
#pragma unroll
      for (int jt = 0; jt < NT; ++jt) {
        float v[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = p[jt][r / 4][r % 4];
#pragma unroll
        for (int q = 0; q < Parts::p; ++q) pp[jt][q] = next_part<BF16>(v);
      }
      // Four operands at a time, so that the parts of one accumulator do not
      // follow each other (2 x 24000 positions, 512 columns: 180 us, so 175).
#pragma unroll
      for (int e0 = 0; e0 < NE; e0 += 4) {
        uint4 x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = vb[(e0 + e) * 64];
#pragma unroll
        for (int q = 0; q < Parts::p; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int jt = 0; jt < NT; ++jt) O[jt][e0 + e] = BF16::mma(O[jt][e0 + e], x[e], pp[jt][q]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const uint4 x = vb[e * 64];
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) {
          const float* pj = p[jt][0];
          O[jt][e] = F32::mma(O[jt][e], x, make_uint4(__float_as_uint(pj[0]), __float_as_uint(pj[1]),
                                                       __float_as_uint(pj[2]), __float_as_uint(pj[3])));
        }
      }
    }
    if constexpr (decltype(tail)::value) {
      if (odd_s[at]) {
        const size_t tile0 = static_cast<size_t>(block_id(a, t.btrow, i, end)) * a.Hkv + kvh;
        const size_t tile1 = static_cast<size_t>(block_id(a, t.btrow, min(i + 1, end - 1), end)) * a.Hkv + kvh;
#pragma unroll
        for (int jt = 0; jt < NT; ++jt)
          add_odd_values<KP, HD, BP>(O[jt], p[jt], sees[jt], a.vc, tile0, tile1, live, lane);
      }
    }
  };
  constexpr std::false_type kPlain{};
  constexpr std::true_type kTail{};

  constexpr std::integral_constant<int, 0> kEven{};
  constexpr std::integral_constant<int, 1> kOdd{};
  // One step: fetch the one after the next, compute, put the next.  Whole steps
  // do so without a condition: behind a fetch that may not have been made the
  // put would wait for all loads, the newest included.
  const auto step = [&](int i, auto parity, auto other, auto tail) {
    constexpr bool whole = !decltype(tail)::value;
    __syncthreads();  // this step is in its buffer; the other buffer has been read
    if (whole || i + 2 * BP < end) fetch(i + 3 * BP, parity);
    if (busy) compute(i, parity, tail);
    if (whole || i + BP < end) put(i + BP, other, tail);
  };

  if (tid < 2) odd_s[tid] = 0;
  __syncthreads();
  int i = t.first;
  fetch(i + BP, kEven);
  fetch(i + 2 * BP, kOdd);
  if (is_tail(i)) put(i, kEven, kTail);
  else put(i, kEven, kPlain);
  for (; i + 3 * BP < end && !is_tail(i + 2 * BP); i += 2 * BP) {  // two steps and the one after them are whole
    step(i, kEven, kOdd, kPlain);
    step(i + BP, kOdd, kEven, kPlain);
  }
  for (; i < end; i += 2 * BP) {
    step(i, kEven, kOdd, kTail);
    if (i + BP < end) step(i + BP, kOdd, kEven, kTail);
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
}

// ---------------------------------------------------------------------------

// Merge of the splits in a launch of its own, whose work-groups share out all
// outputs: 16 columns of one (column group of CW, KV head) each, a thread kMine
// pieces of 16 bytes with the first kChunk splits' loads in flight while it
// finds the weights.  22 to 32 MB of partials (480 to 744 work-groups of 64 or
// 128 columns): 8 to 9 us, half of it the launch and two trips to memory.
constexpr int kMergeColumns = 16;
template <class IO, int HD, int CW>
__global__ __launch_bounds__(256) void k_tree_merge(TreeAttnArgs a) {
  constexpr int kPer = HD / 4, kMine = kMergeColumns * kPer / 256, kChunk = 8;
  __shared__ float weights[kTreeSplits * kMergeColumns];
  const int kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  // Request: the last one whose first column group is not behind this one.
  const int rank = __builtin_amdgcn_readfirstlane(
      __popcll(__ballot(lane < a.n && a.cg0[min(lane, a.n - 1)] <= static_cast<int>(blockIdx.y))) - 1);
  const int ncg = a.ncg[rank], cg = blockIdx.y - a.cg0[rank], cols = a.nodes[rank] * a.G;
  const int nsplit = (a.item0[rank + 1] - a.item0[rank]) / ncg;
  const int c0 = blockIdx.z * kMergeColumns;  // within the group
  if (nsplit == 1 || CW * cg + c0 >= cols) return;
  const int mine = min(cols - CW * cg - c0, kMergeColumns);
  constexpr size_t kColumn = HD + 4;
  const float* part = a.part + ((static_cast<size_t>(a.item0[rank] + cg) * a.Hkv + kvh) * CW + c0) * kColumn;
  const size_t stride = static_cast<size_t>(ncg) * a.Hkv * CW * kColumn;
  // A lane per (column, split): maximum and sum; sixteen lanes share a column.
  const float* ml = part + min(tid / 16, mine - 1) * kColumn;
  float sm[2], sl[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int s = tid % 16 + 16 * k;
    const float2 x = *reinterpret_cast<const float2*>(ml + min(s, nsplit - 1) * stride);
    sm[k] = s < nsplit ? x.x : kTreeFloor;
    sl[k] = s < nsplit ? x.y : 0.f;
  }
  const float* at[kMine];
  f32x4_t R[kMine], o[kMine][kChunk];
#pragma unroll
  for (int n = 0; n < kMine; ++n) {
    const int idx = tid + 256 * n;
    at[n] = part + min(idx / kPer, mine - 1) * kColumn + 4 + idx % kPer * 4;
    R[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const auto load = [&](int s0) {
#pragma unroll
    for (int k = 0; k < kChunk; ++k)
#pragma unroll
      for (int n = 0; n < kMine; ++n) o[n][k] = *reinterpret_cast<const f32x4_t*>(at[n] + min(s0 + k, nsplit - 1) * stride);
  };
  load(0);
  float M = fmaxf(sm[0], sm[1]);
#pragma unroll
  for (int x = 8; x >= 1; x >>= 1) M = fmaxf(M, __shfl_xor(M, x));
  float w[2], L = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    w[k] = __builtin_amdgcn_exp2f(sm[k] - M);
    L += sl[k] * w[k];
  }
#pragma unroll
  for (int x = 8; x >= 1; x >>= 1) L += __shfl_xor(L, x);
  const float inv = 1.f / L;
#pragma unroll
  for (int k = 0; k < 2; ++k) weights[(tid % 16 + 16 * k) * kMergeColumns + tid / 16] = w[k] * inv;
  __syncthreads();
  for (int s0 = 0;;) {
#pragma unroll
    for (int k = 0; k < kChunk; ++k)
      if (s0 + k < nsplit) {
#pragma unroll
        for (int n = 0; n < kMine; ++n) R[n] += weights[(s0 + k) * kMergeColumns + (tid + 256 * n) / kPer] * o[n][k];
      }
    s0 += kChunk;
    if (s0 >= nsplit) break;
    load(s0);
  }
#pragma unroll
  for (int n = 0; n < kMine; ++n) {
    const int idx = tid + 256 * n, c = idx / kPer;
    if (c >= mine) break;
    const TreeColumn col = tree_column(a, a.row0[rank], kvh, CW * cg + c0 + c);
    IO::store4(a, col.row, col.hq * HD + idx % kPer * 4, R[n]);
  }
}

}  // namespace sprk
