// Attention of drafted trees over the paged KV cache: row r = (request, node)
// and head h,
//   out[r][h] = softmax(q[r][h] . K^T / sqrt(hd)) V
// over the request's cached positions 0 .. len - 1 and the positions len + a
// of the node itself and its ancestors (bits of a 64-bit mask).
//
// The rows of one request share its keys and values, and so do the G query
// heads of a KV head: the kernel's columns are (node, head of the group), and
// a cache block that a wave loads serves 16 NT of them.  Reading the cache
// once is the floor while the columns are few; past about nine 16-column
// tiles the products are.
//
// Work item = (request, column group of 16 NT columns, KV split), times the KV
// head.  A work-group's four waves each take a run of 16-position blocks of
// the split, two (bf16) or one (fp32) per step, on MFMA:
//   S[t][c]   = K_tile(16 x hd) . Q^T(hd x 16)
//   O^T[e][c] += V^T_tile(16 dims x positions) . P(positions x 16)
// P is the S accumulator re-used in place as the B operand.  Two bf16 blocks
// make one 16x16x32 product: the K index of a lane's eight values may be
// assigned freely as long as both operands agree, so the first four are block
// 0's positions 4 g .. 4 g + 3 and the rest block 1's.
// fp32 queries meet a bf16 cache in three bf16 parts (all 24 bits), and the
// probabilities enter their product in three parts too, so that an fp32
// output is an fp32 result (two parts of the probabilities alone put 1e-6 of
// error on it); a bf16 output takes bf16 probabilities (their rounding, 2^-9
// relative and independent per position, is at most that of the output).
// Q sits in LDS (every wave of the group reads the same fragments), which
// leaves the registers to K, V and the accumulators.
//
// The running maximum of a column is raised only when a step exceeds it by
// kRaise (in log2 units): until then probabilities of at most 2^kRaise stay
// exact enough in fp32, and steps need neither the exchange between lanes nor
// the rescaling of O.
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
  float* part;         // [item][Hkv][16 NT][hd + 4]: m, l, -, -, o[hd]
  int32_t* cnt;        // [column group][Hkv] arrived splits; zero between launches
  int* err;
  int n, H, Hkv, G, mb, nb, bpw;
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
    for (int b = 0; b < 2; ++b) {
      const uint32_t m01 = (keep[b] & 1 ? 0xFFFFu : 0u) | (keep[b] & 2 ? 0xFFFF0000u : 0u);
      const uint32_t m23 = (keep[b] & 4 ? 0xFFFFu : 0u) | (keep[b] & 8 ? 0xFFFF0000u : 0u);
#pragma unroll
      for (int f = 0; f < NV; ++f) {
        v[b][f].x &= m01;
        v[b][f].y &= m23;
        v[b][f].z &= m01;
        v[b][f].w &= m23;
      }
    }
  }
  // Whether a value of this lane is infinite or NaN.
  __device__ __forceinline__ bool odd_v() const {
    const auto odd = [](uint32_t x) { return (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u; };
    bool o = false;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int f = 0; f < NV; ++f) o |= odd(v[b][f].x) || odd(v[b][f].y) || odd(v[b][f].z) || odd(v[b][f].w);
    return o;
  }
  template <int PP>
  __device__ __forceinline__ void pv(f32x4_t* O, const float (*p)[4]) const {
    uint4 b[PP];
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = p[i / 4][i % 4];
#pragma unroll
    for (int q = 0; q < PP; ++q) {
      uint16_t e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = f32_to_bf16_bits(r[i]);
        r[i] -= bf16_bits_to_f32(e[i]);
      }
      b[q] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
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
    for (int f = 0; f < NV; ++f) {
      v[0][f].x = keep[0] & 1 ? v[0][f].x : 0u;
      v[0][f].y = keep[0] & 2 ? v[0][f].y : 0u;
      v[0][f].z = keep[0] & 4 ? v[0][f].z : 0u;
      v[0][f].w = keep[0] & 8 ? v[0][f].w : 0u;
    }
  }
  __device__ __forceinline__ bool odd_v() const {
    const auto odd = [](uint32_t x) { return (x & 0x7F800000u) == 0x7F800000u; };
    bool o = false;
#pragma unroll
    for (int f = 0; f < NV; ++f) o |= odd(v[0][f].x) || odd(v[0][f].y) || odd(v[0][f].z) || odd(v[0][f].w);
    return o;
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

template <class KP, class IO, int HD, int NT>
__global__ __launch_bounds__(256) void k_tree_attn(TreeAttnArgs a) {
  using Step = TreeStep<KP, HD>;
  using Parts = TreeParts<KP, IO>;
  constexpr int BP = Step::kBlocks, NF = Step::NF, NE = HD / 16, EPW = NE / 4;
  __shared__ TreeSmem<KP, IO, HD, NT> sm;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane & 15, g = lane >> 4;
  const int f = blockIdx.y, kvh = blockIdx.x;
  // Request of this item: the number of requests whose items all precede it.
  const int rank = __builtin_amdgcn_readfirstlane(
      __popcll(__ballot(lane < a.n - 1 && a.item0[min(lane + 1, kTreeReqs)] <= f)));
  const int ncg = a.ncg[rank];
  const int w = f - a.item0[rank];
  const int s = w / ncg, cg = w - s * ncg;  // column groups of one split run side by side and share its blocks
  const int nsplit = (a.item0[rank + 1] - a.item0[rank]) / ncg;
  const int len = a.len[rank], nn = a.nodes[rank], row0 = a.row0[rank];
  const int cols = nn * a.G, c0 = 16 * NT * cg;
  const int total = len + nn, nblk = (total + 15) >> 4;
  const int first = 4 * a.bpw * s, count = min(nblk - first, 4 * a.bpw);
  const int lo = first + min(count, wave * a.bpw), hi = first + min(count, (wave + 1) * a.bpw);
  const int32_t* btrow = a.bt + static_cast<size_t>(a.slot[rank]) * a.mb;
  // Block ids of the next 64 blocks of the run; one outside the pool reads block 0.
  const auto block_ids = [&](int i) {
    int id = i + lane < hi ? btrow[i + lane] : 0;
    if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.nb)) {
      raise_check(a.err, kErrBlockId);
      id = 0;
    }
    return id;
  };
  int ids = block_ids(lo);

  // Q fragments into LDS; columns past the request's read its last one's row.
  for (int t = wave; t < NT * NF; t += 4) {
    const int jt = t / NF, c = t % NF;
    const int col = min(c0 + 16 * jt + h, cols - 1);
    const int node = col / a.G, hq = kvh * a.G + col - node * a.G;
    const typename IO::elem* src =
        static_cast<const typename IO::elem*>(a.q) + (row0 + node) * a.qs + hq * HD + c * KP::kblk + g * KP::per16;
    if constexpr (IO::kRaw && KP::per16 == 8) {
      sm.q[jt][c][0][lane] = *reinterpret_cast<const uint4*>(src);
    } else {
      float v[KP::per16];
      if constexpr (IO::kRaw) {
        const uint2 u = *reinterpret_cast<const uint2*>(src);
        v[0] = bf16_bits_to_f32(u.x & 0xFFFF);
        v[1] = __uint_as_float(u.x & 0xFFFF0000u);
        v[2] = bf16_bits_to_f32(u.y & 0xFFFF);
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
      for (int q = 0; q < Parts::q; ++q) {
        union {
          uint4 u;
          typename KP::elem e[KP::per16];
        } o;
#pragma unroll
        for (int j = 0; j < KP::per16; ++j) {
          o.e[j] = KP::from_f32(v[j]);
          v[j] -= KP::to_f32(o.e[j]);
        }
        sm.q[jt][c][q][lane] = o.u;
      }
    }
  }
  uint64_t anc[NT];
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) anc[jt] = a.anc[row0 + min(c0 + 16 * jt + h, cols - 1) / a.G];
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
    if ((k & 63) == 0 && k != 0) ids = block_ids(i);
    Step B;
    size_t tile[BP];
#pragma unroll
    for (int b = 0; b < BP; ++b)  // a missing second block re-reads the first, masked
      tile[b] = static_cast<size_t>(__builtin_amdgcn_readlane(ids, (i + b < hi ? k + b : k) & 63)) * a.Hkv + kvh;
    B.load(a.kc, a.vc, tile, lane);
    // A step that reaches past the cached positions or the run is masked.
    const bool tail = 16 * (i + BP) > len || i + BP > hi;
    uint32_t live[BP];  // bits: this lane's positions of the block that hold a cached position or a node
    bool odd = false;
    if (tail) {
#pragma unroll
      for (int b = 0; b < BP; ++b) {
        const int room = i + b < hi ? total - (16 * (i + b) + 4 * g) : 0;
        live[b] = room >= 4 ? 15u : room <= 0 ? 0u : (1u << room) - 1;
      }
      B.keep_v(live);
      odd = __ballot(B.odd_v()) != 0;
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
          // Bits of this lane's four positions: cached ones, then the nodes that
          // the column's ancestor set holds.  Shifts only, no branches.
          const int base = 16 * (i + b) + 4 * g - len;
          const int cached = min(max(-base, 0), 4);
          const uint32_t nodes = static_cast<uint32_t>(anc[jt] >> min(max(base, 0), 63)) << cached;
          sees[b] = live[b] & (((1u << cached) - 1) | nodes);
#pragma unroll
          for (int r = 0; r < 4; ++r) S[b][r] = sees[b] >> r & 1 ? S[b][r] : -INFINITY;
        }
      }
      float mx = fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3]));
#pragma unroll
      for (int b = 1; b < BP; ++b) mx = fmaxf(mx, fmaxf(fmaxf(S[b][0], S[b][1]), fmaxf(S[b][2], S[b][3])));
      mx *= a.qscale;
      if (__ballot(mx > m[jt] + kRaise) != 0) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float up = fmaxf(m[jt], mx);
        const float alpha = __builtin_amdgcn_exp2f(m[jt] - up);
        l[jt] *= alpha;
        m[jt] = up;
#pragma unroll
        for (int e = 0; e < NE; ++e) O[jt][e] *= alpha;
      }
      float p[BP][4];
#pragma unroll
      for (int b = 0; b < BP; ++b) {
#pragma unroll
        for (int r = 0; r < 4; ++r) p[b][r] = __builtin_amdgcn_exp2f(fmaf(S[b][r], a.qscale, -m[jt]));
        l[jt] += (p[b][0] + p[b][1]) + (p[b][2] + p[b][3]);
      }
      if (!odd) {
        B.template pv<Parts::p>(O[jt], p);
      } else {
        // A node's value (or a cached one) is infinite or NaN: 0 times it must
        // not reach the columns that do not see it.  One position at a time
        // into a sum of its own, added where it is seen.
        for (int t = 0; t < 16 * BP; ++t) {
          uint32_t one[BP];
          float pt[BP][4];
#pragma unroll
          for (int b = 0; b < BP; ++b) {
            one[b] = t / 16 == b && t % 16 / 4 == g ? 1u << (t & 3) : 0u;
#pragma unroll
            for (int r = 0; r < 4; ++r) pt[b][r] = one[b] >> r & 1 ? p[b][r] : 0.f;
          }
          Step V = B;
          V.keep_v(one);
          f32x4_t T[NE];
#pragma unroll
          for (int e = 0; e < NE; ++e) T[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          V.template pv<Parts::p>(T, pt);
          uint32_t seen = 0;
#pragma unroll
          for (int b = 0; b < BP; ++b) seen |= sees[b] & one[b];
          // The bit sits in the lanes of one g: every lane of the column asks.
          const uint64_t who = __ballot(seen != 0);
          const bool mine = (who >> h | who >> (h + 16) | who >> (h + 32) | who >> (h + 48)) & 1;
#pragma unroll
          for (int e = 0; e < NE; ++e)
#pragma unroll
            for (int r = 0; r < 4; ++r) O[jt][e][r] += mine ? T[e][r] : 0.f;
        }
      }
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
  const uint32_t item = (static_cast<uint32_t>(f) * a.Hkv + kvh) * (16 * NT) * (HD + 4) * 4;
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
    const int col = c0 + 16 * jt + h;
    const int node = col / a.G, hq = kvh * a.G + col - node * a.G;
#pragma unroll
    for (int k = 0; k < EPW; ++k) {
      f32x4_t R = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const f32x4_t o = sm.so[v][wave * EPW + k][lane];
#pragma unroll
        for (int r = 0; r < 4; ++r) R[r] += cw[v] * o[r];
      }
      if (col >= cols) continue;
      const int d0 = 16 * (wave * EPW + k) + 4 * g;
      if (nsplit == 1) {
        const float inv = 1.f / L;
        IO::store4(a, row0 + node, hq * HD + d0, R * inv);
      } else {
        pb.store4(item + ((16 * jt + h) * (HD + 4) + 4 + d0) * 4, R);
        if (wave == 0 && k == 0 && g == 0)
          pb.store4(item + (16 * jt + h) * (HD + 4) * 4, f32x4_t{M, L, 0.f, 0.f});
      }
    }
  }
  if (nsplit == 1) return;
  // Publish, count in, and let the split that arrives last merge them all: no
  // work-group waits on another.
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's partial stores are complete
  __syncthreads();
  int32_t* cnt = a.cnt + (a.cg0[rank] + cg) * a.Hkv + kvh;
  if (threadIdx.x == 0)
    sm.last = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == nsplit - 1;
  __syncthreads();
  if (!sm.last) return;
  if (threadIdx.x == 0) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const uint32_t base = (static_cast<uint32_t>(a.item0[rank] + cg) * a.Hkv + kvh) * (16 * NT) * (HD + 4) * 4;
  const uint32_t stride = static_cast<uint32_t>(ncg) * a.Hkv * (16 * NT) * (HD + 4) * 4;
  constexpr int kChunk = 8;  // partials read per round
  const int mine = min(cols - c0, 16 * NT);
  for (int idx = threadIdx.x; idx < mine * (HD / 4); idx += 256) {
    const int c = idx / (HD / 4), d0 = idx % (HD / 4) * 4;
    const uint32_t at = base + c * (HD + 4) * 4;
    float M = kTreeFloor, L = 0.f;
    f32x4_t R = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int t0 = 0; t0 < nsplit; t0 += kChunk) {
      f32x4_t ml[kChunk], o[kChunk];
#pragma unroll
      for (int t = 0; t < kChunk; ++t) {
        const uint32_t b = at + min(t0 + t, nsplit - 1) * stride;
        ml[t] = pb.load4(b);
        o[t] = pb.load4(b + 16 + d0 * 4);
      }
      float up = M;
#pragma unroll
      for (int t = 0; t < kChunk; ++t) up = t0 + t < nsplit ? fmaxf(up, ml[t][0]) : up;
      const float sc = __builtin_amdgcn_exp2f(M - up);
      L *= sc;
      R *= sc;
#pragma unroll
      for (int t = 0; t < kChunk; ++t) {
        if (t0 + t < nsplit) {
          const float wt = __builtin_amdgcn_exp2f(ml[t][0] - up);
          L += wt * ml[t][1];
          R += wt * o[t];
        }
      }
      M = up;
    }
    const int col = c0 + c, node = col / a.G, hq = kvh * a.G + col - node * a.G;
    IO::store4(a, row0 + node, hq * HD + d0, R * (1.f / L));
  }
}

}  // namespace sprk
