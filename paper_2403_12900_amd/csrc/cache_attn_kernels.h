// Attention over the 4-bit cache: row j of a request and head h,
//   out[r][h] = softmax(q[r][h] . K^T / sqrt(hd)) V
// over the request's positions 0 .. len + j.
//
// The columns of one (request, KV head) are (row, head of the group): c = j * G
// + head.  On MFMA, per block of 16 positions and tile of 16 columns:
//   S[t][c]   = K_tile(16 x hd) . Q^T(hd x 16)
//   O^T[e][c] += V^T_tile(16 dims x positions) . P(positions x 16)
// with P the S accumulator re-used in place as the B operand; two blocks make
// one 16x16x32 product.  One pass, with a running maximum m and sum l.
//
// Codes times their scales are exact in bf16, and so are the products of fp32
// queries in three bf16 parts.  Probabilities and values meet in fp16, whose 11
// bits of a probability bf16 would take two parts for, where fp16 holds the
// values exactly (any code at scales 2^-18 .. 2^13); else in bf16, the
// probabilities in two parts (bf16 outputs, 16 bits) or three (fp32, 24).
#pragma once

#include <type_traits>

#include "cache_bits.h"
#include "cache_format.h"
#include "cache_rule.h"
#include "tree_attn_kernels.h"

namespace sprk {

struct CacheAttnArgs {
  const void* q;
  void* out;
  int64_t qs, os;       // row strides of q and out (elements)
  const uint8_t* pool;  // this layer
  const int32_t* bt;
  float* part;          // [item][Hkv][columns of an item][hd + 4]: m, l, -, -, o[hd]
  int32_t* cnt;         // [column group][Hkv] arrived splits; zero between launches
  int* err;
  int n, H, Hkv, G, mb, nb, bps;  // bps: blocks per split
  uint32_t part_bytes;
  float qscale;         // log2(e) / sqrt(hd)
  int slot[kCacheReqs], len[kCacheReqs], rows[kCacheReqs], row0[kCacheReqs], cg0[kCacheReqs];
  int item0[kCacheReqs + 1];  // first work item of each request
};
static_assert(sizeof(CacheAttnArgs) <= 3584, "kernel arguments");

// What a work item is: its request, column group and blocks.
struct CacheItem {
  int cg, cg0, nsplit, ncg, item0;
  int item;                   // of its partial result
  int len, nblk, row0, cols;  // nblk: blocks that the column group's rows see
  int first, count;           // blocks of the split (count < 1: nothing to do)
  const int32_t* btrow;
};
template <int CW>
__device__ __forceinline__ CacheItem cache_item(const CacheAttnArgs& a, int f) {
  const int lane = threadIdx.x & 63;
  CacheItem t;
  int slot;
  // Lane = request, 64 at a time and all of them at once: one trip to memory.
  for (int k = 0;; k += 64) {
    const int r = min(k + lane, a.n - 1);
    const int item0 = a.item0[r], item1 = a.item0[r + 1], cg0 = a.cg0[r], len = a.len[r], row0 = a.row0[r];
    const int rows = a.rows[r], slots = a.slot[r];
    // Request: the number of requests whose items all precede f.
    const int before = __popcll(__ballot(k + lane < a.n && item1 <= f));
    if (before == 64 && k + 64 < a.n) continue;
    const auto mine = [&](int v) { return __builtin_amdgcn_readlane(v, before); };
    t.item0 = mine(item0);
    t.cg0 = mine(cg0);
    t.len = mine(len);
    t.row0 = mine(row0);
    t.cols = mine(rows) * a.G;
    slot = mine(slots);
    break;
  }
  t.ncg = (t.cols + CW - 1) / CW;
  // Column groups of one split run side by side and share its blocks.  Later rows
  // see more: the groups go down from the last one, and the second half of them
  // up from the first, so that two of a CU are together as long everywhere.
  const int w = f - t.item0, s = w / t.ncg, j = w - s * t.ncg, down = t.ncg - t.ncg / 2;
  t.cg = j < down ? t.ncg - 1 - j : j - down;
  t.item = t.item0 + s * t.ncg + t.cg;
  const int last = (min(t.cols, (t.cg + 1) * CW) - 1) / a.G;  // row
  t.nblk = (t.len + last + 16) >> 4;
  t.nsplit = (t.nblk + a.bps - 1) / a.bps;
  t.first = a.bps * s;
  t.count = min(t.nblk - t.first, a.bps);
  t.btrow = a.bt + static_cast<size_t>(slot) * a.mb;
  return t;
}
__device__ __forceinline__ int pool_id(const CacheAttnArgs& a, int id) {
  if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.nb)) {
    raise_check(a.err, kErrBlockId);
    id = 0;
  }
  return id;
}

// Values of a word (4 positions of dimensions e, in low nibbles, and e + 16)
// as two operand halves of bf16: positions 0 .. 3 of each dimension.
__device__ __forceinline__ void value_halves(uint32_t w, uint32_t scales, uint2& lo, uint2& hi) {
  const uint32_t x0 = codes_to_bf16<0>(w, scale_of<0>(scales)), x1 = codes_to_bf16<1>(w, scale_of<1>(scales));
  const uint32_t x2 = codes_to_bf16<2>(w, scale_of<2>(scales)), x3 = codes_to_bf16<3>(w, scale_of<3>(scales));
  lo = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x05040100u), __builtin_amdgcn_perm(x3, x2, 0x05040100u));
  hi = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x07060302u), __builtin_amdgcn_perm(x3, x2, 0x07060302u));
}

// K and V of one step of a wave: two blocks of one KV head, in registers.
template <int HD>
struct CacheStep {
  using F = Mx4<HD>;
  static constexpr int P = F::P;  // words of a lane and block, keys or values
  uint32_t k[2][P], v[2][P], ks[2], vs[2][P];

  template <int N>
  static __device__ __forceinline__ void words(const uint8_t* p, uint32_t* w) {
    if constexpr (N == 4) {
      const u32x4_t x = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
      w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    } else {
      const uint64_t x = __builtin_nontemporal_load(reinterpret_cast<const uint64_t*>(p));
      w[0] = static_cast<uint32_t>(x), w[1] = static_cast<uint32_t>(x >> 32);
    }
  }
  // Lane r + 16 g: keys of position r, dimensions HD / 4 g on.
  static __device__ __forceinline__ int key_at(int r, int g) { return F::key_code(r, HD / 4 * g); }
  __device__ __forceinline__ void load_keys(const uint8_t* pool, const size_t* tile, int lane) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint8_t* t = pool + tile[b] * F::kTile;
      words<P>(t + key_at(r, g), k[b]);
      ks[b] = t[F::key_scale(r, HD / 4 * g / 32)];
    }
  }
  __device__ __forceinline__ void load_values(const uint8_t* pool, const size_t* tile, int lane) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint8_t* t = pool + tile[b] * F::kTile;
      words<P>(t + F::value_word(g, r, 0), v[b]);
      words<P>(t + F::value_scales(g, 0), vs[b]);
    }
  }
  __device__ __forceinline__ void load(const uint8_t* pool, const size_t* tile, int lane) {
    load_keys(pool, tile, lane);
    load_values(pool, tile, lane);
  }
  // Part c of block b's keys as an operand.
  __device__ __forceinline__ uint4 key(int b, int c) const {
    const float s = scale_of<0>(ks[b]);
    return make_uint4(codes_to_bf16<0>(k[b][c], s), codes_to_bf16<1>(k[b][c], s), codes_to_bf16<2>(k[b][c], s),
                      codes_to_bf16<3>(k[b][c], s));
  }
  // Zeroes the values at positions whose bit of live is clear, and NaN ones;
  // odd[b][p]: which were NaN.
  __device__ __forceinline__ bool mask_values(const uint32_t* live, uint32_t (*odd)[P]) {
    bool any = false;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int p = 0; p < P; ++p) {
        odd[b][p] = nan_bits(vs[b][p]) & live[b];
        const uint32_t keep = byte_mask(live[b] & ~nan_bits(vs[b][p]));
        any |= odd[b][p] != 0;
        v[b][p] &= keep;
        vs[b][p] = (vs[b][p] & keep) | (0x7F7F7F7Fu & ~keep);
      }
    return any;
  }
  template <int PP>
  __device__ __forceinline__ void pv(f32x4_t* O, const uint4* x) const {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      uint2 lo[2], hi[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) value_halves(v[b][p], vs[b][p], lo[b], hi[b]);
#pragma unroll
      for (int q = 0; q < PP; ++q) {
        O[2 * p] = BF16::mma(O[2 * p], make_uint4(lo[0].x, lo[0].y, lo[1].x, lo[1].y), x[q]);
        O[2 * p + 1] = BF16::mma(O[2 * p + 1], make_uint4(hi[0].x, hi[0].y, hi[1].x, hi[1].y), x[q]);
      }
    }
  }
};

// NaN values were zeroed in the products (0 times one must not reach the
// columns that do not see it): NaN into the 32 dimensions of those that do.
// odd, sees: by position of this lane's quarter.
template <int P>
__device__ __forceinline__ void add_nan_values(f32x4_t* O, const uint32_t (*odd)[P], const uint32_t* sees) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    int x = ((odd[0][p] & sees[0]) | (odd[1][p] & sees[1])) != 0;
    x |= __shfl_xor(x, 16);
    x |= __shfl_xor(x, 32);
    if (x) {
      O[2 * p] += __builtin_nanf("");
      O[2 * p + 1] += __builtin_nanf("");
    }
  }
}

template <class IO>
struct CacheParts {
  static constexpr int q = IO::kRaw ? 1 : 3;
  static constexpr int p = IO::kRaw ? 2 : 3;
};

// Positions 0 .. 3 of dimensions e (low nibbles) and e + 16 of a word, in fp16.
__device__ __forceinline__ void value_halves_f16(uint32_t w, uint32_t scales, uint2& lo, uint2& hi) {
  const uint32_t x0 = codes_to_f16<0>(w, scale_of<0>(scales)), x1 = codes_to_f16<1>(w, scale_of<1>(scales));
  const uint32_t x2 = codes_to_f16<2>(w, scale_of<2>(scales)), x3 = codes_to_f16<3>(w, scale_of<3>(scales));
  lo = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x05040100u), __builtin_amdgcn_perm(x3, x2, 0x05040100u));
  hi = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x07060302u), __builtin_amdgcn_perm(x3, x2, 0x07060302u));
}

// The eight probabilities of a step, rounded to fp16, as one operand part; taken
// from v.
__device__ __forceinline__ uint4 next_part_f16(float* v) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f16x2_t x = __builtin_convertvector((f32x2_t{v[2 * j], v[2 * j + 1]}), f16x2_t);
    w[j] = __builtin_bit_cast(uint32_t, x);
    v[2 * j] -= static_cast<float>(x.x);
    v[2 * j + 1] -= static_cast<float>(x.y);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ f32x4_t mma_f16(f32x4_t acc, uint4 a, uint4 b) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), acc, 0, 0, 0);
}

constexpr uint4 kHalfOnes{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u};  // eight fp16 ones

// Parts of a probability in fp16, and how far it is lifted: a row's largest one so
// far lies in [2^lift, 2^limit], below fp16's largest number, so that fp16's last
// step, 2^-24, is 2^-31 (bf16 outputs) or 2^-35 (fp32) of it: one part's 2^-11 holds
// down to 2^-21 of the largest, two parts' 2^-22 down to 2^-14.  More lift raises the
// maximum more often (4 x 1024 first rows of 32 heads, lift 7 / 10 / 11 / 12: fp32
// 115 / 116 / 116 / 119 us; bf16 74 with 7, 81 with 12).
template <class IO>
struct HalfParts {
  static constexpr int p = IO::kRaw ? 1 : 2;
  static constexpr float lift = IO::kRaw ? 7.f : 11.f, limit = IO::kRaw ? 15.f : 15.9f;
};

// Online softmax of a wave's column tiles as softmax_step, without the sum:
// scores S to probabilities p, lifted as above.
template <class IO, int NT, int NE>
__device__ __forceinline__ void lifted_softmax(const f32x4_t (*S)[2], float qscale, float* m, f32x4_t* l, f32x4_t (*O)[NE],
                                             float (*p)[8]) {
  const auto highest = [](const float* x) {
    return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  };
  bool over = false;
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
#pragma unroll
    for (int r = 0; r < 8; ++r) p[jt][r] = fmaf(S[jt][r / 4][r % 4], qscale, -m[jt]);
    over |= highest(p[jt]) > HalfParts<IO>::limit;
  }
  if (__ballot(over) != 0) {
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
#pragma unroll
      for (int r = 0; r < 8; ++r) p[jt][r] = S[jt][r / 4][r % 4] * qscale;
      float mx = highest(p[jt]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float up = fmaxf(m[jt], mx - HalfParts<IO>::lift);
      const float alpha = __builtin_amdgcn_exp2f(m[jt] - up);
      m[jt] = up;
      l[jt] *= alpha;
#pragma unroll
      for (int e = 0; e < NE; ++e) O[jt][e] *= alpha;
#pragma unroll
      for (int r = 0; r < 8; ++r) p[jt][r] = fmaf(S[jt][r / 4][r % 4], qscale, -up);
    }
  }
#pragma unroll
  for (int jt = 0; jt < NT; ++jt)
#pragma unroll
    for (int r = 0; r < 8; ++r) p[jt][r] = __builtin_amdgcn_exp2f(p[jt][r]);
}

template <class IO, int HD, int NT>
struct CacheSmem {
  union {
    uint4 q[NT][HD / 32][CacheParts<IO>::q][64];
    f32x4_t so[4][HD / 16][64];
    float weights[kCacheSplits * 16 * NT];
  };
  float2 sml[4][NT][16];
  int last;
};

// This lane's piece of one column's query as an operand: dimensions HD / 4 g +
// 8 c on (the keys' order), in its parts.
template <class IO, int HD>
__device__ __forceinline__ void query_operand(const CacheAttnArgs& a, const TreeColumn& col, int c, int g, uint4* out) {
  const typename IO::elem* src =
      static_cast<const typename IO::elem*>(a.q) + col.row * a.qs + col.hq * HD + HD / 4 * g + 8 * c;
  const uint4 x = *reinterpret_cast<const uint4*>(src);
  if constexpr (IO::kRaw) {
    out[0] = x;
  } else {
    // The first part is cut, not rounded (which would take the largest numbers to
    // infinity): 16 bits are left, of which the second takes 8 and the third the rest.
    const uint4 y = *reinterpret_cast<const uint4*>(src + 4);
    const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    uint32_t first[4];
    float v[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) first[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x07060302u);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]) - __uint_as_float(w[j] & 0xFFFF0000u);
    out[0] = make_uint4(first[0], first[1], first[2], first[3]);
#pragma unroll
    for (int q = 1; q < CacheParts<IO>::q; ++q) out[q] = next_part<BF16>(v);
  }
}

// Scores of a step whose keys lie in registers, before their scale.  q(jt, c,
// part): a piece of the queries.
template <class IO, int HD, int NT, class Queries>
__device__ __forceinline__ void key_products(const CacheStep<HD>& B, const Queries& q, f32x4_t (*S)[2]) {
#pragma unroll
  for (int jt = 0; jt < NT; ++jt)
#pragma unroll
    for (int b = 0; b < 2; ++b) S[jt][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < HD / 32; ++c)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint4 x = B.key(b, c);
#pragma unroll
      for (int jt = 0; jt < NT; ++jt)
#pragma unroll
        for (int k = 0; k < CacheParts<IO>::q; ++k) S[jt][b] = BF16::mma(S[jt][b], x, q(jt, c, k));
    }
}

// One step of a wave whose keys and values lie in registers: 16 NT columns, the
// blocks at i and i + 1 (< hi).  all, some: positions that every column of the group sees, and that one of them
// does; seen: that this lane's columns do.
template <class IO, int HD, int NT, class Queries>
__device__ __forceinline__ void cache_step(const CacheAttnArgs& a, CacheStep<HD>& B, int i, int hi, int all, int some,
                                           const int* seen, const Queries& q, float* m, float* l,
                                           f32x4_t (*O)[HD / 16], int lane) {
  using Parts = CacheParts<IO>;
  constexpr int P = HD / 32, NE = HD / 16;
  const int g = lane >> 4;
  f32x4_t S[NT][2];
  key_products<IO, HD, NT>(B, q, S);
  // A step that reaches past what all columns see, or past hi, is masked.
  const bool tail = 16 * (i + 2) > all || i + 2 > hi;
  uint32_t sees[NT][2], odd[2][P];
  bool any = false;
  if (tail) {
    uint32_t live[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int pos = 16 * (i + b) + 4 * g;
      live[b] = i + b < hi ? live_bits(pos, some) : 0u;
#pragma unroll
      for (int jt = 0; jt < NT; ++jt) {
        sees[jt][b] = live[b] & live_bits(pos, seen[jt]);
#pragma unroll
        for (int r = 0; r < 4; ++r) S[jt][b][r] = sees[jt][b] >> r & 1 ? S[jt][b][r] : -INFINITY;
      }
    }
    any = __ballot(B.mask_values(live, odd)) != 0;
  }
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    float p[2][4];
    softmax_step<2, NE>(S[jt], a.qscale, m[jt], l[jt], O[jt], p);
    float v[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) v[r] = p[r / 4][r % 4];
    uint4 x[Parts::p];
#pragma unroll
    for (int k = 0; k < Parts::p; ++k) x[k] = next_part<BF16>(v);
    B.template pv<Parts::p>(O[jt], x);
    if (any) add_nan_values<P>(O[jt], odd, sees[jt]);
  }
}

// Up to 32 columns: the four waves of a work-group take runs of the split's
// blocks, K and V go straight into registers, and the waves' results are merged
// through LDS, the splits' by the one that arrives last.  A wave that meets a
// value that fp16 does not hold exactly, or a NaN that not all columns see,
// starts its run over with cache_step.
//
// Bound by memory in long caches: 8 requests of about 24000 positions, 64 heads on
// 8, bf16 (228 MB): 46.5 us, 4.9 TB/s with launch, prologue and merge (the same
// loads alone: 45); by the trips to memory of a run's few steps in short ones: 32
// requests of about 400 positions, 32 heads, fp32 (67 MB): 21.3 us, the loads alone
// 17.5.  Two steps on their way in registers: three measured 22.8 / 47.2 (short /
// long), four work-groups on a CU with fewer registers 23.3 / 50.3, loads that stay
// in the cache 20.5 / 52, work-groups of two waves 32 (short).
template <class IO, int HD, int NT>
__global__ __launch_bounds__(256, NT == 1 ? 3 : 2) void k_cache_attn(CacheAttnArgs a) {
  using Step = CacheStep<HD>;
  using Parts = CacheParts<IO>;
  constexpr int NF = HD / 32, NE = HD / 16, EPW = NE / 4, CW = 16 * NT, P = Step::P;
  __shared__ CacheSmem<IO, HD, NT> sm;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane & 15, g = lane >> 4;
  const int f = blockIdx.x / a.Hkv, kvh = blockIdx.x - f * a.Hkv;
  const CacheItem t = cache_item<CW>(a, f);
  if (t.count < 1) return;
  // Runs of the four waves: equal shares of the split, in whole steps.
  const int run = (t.count + 7) / 8 * 2;
  const int lo = t.first + min(t.count, wave * run), hi = t.first + min(t.count, (wave + 1) * run);
  const auto ask = [&](int i) { return pool_id(a, i < hi ? t.btrow[i] : 0); };
  int ids = ask(lo + lane);  // of the next 64 blocks of the run

  const auto tile_of = [&](int i) {
    return static_cast<size_t>(__builtin_amdgcn_readlane(ids, (i - lo) & 63)) * a.Hkv + kvh;
  };
  // The blocks of the step at i; a missing second one re-reads the first, masked.
  size_t tile[2] = {};
  const auto find = [&](int i) {
    if (((i - lo) & 63) == 0 && i != lo) ids = ask(i + lane);
    tile[0] = tile_of(i);
    tile[1] = tile_of(i + 1 < hi ? i + 1 : i);
  };
  // A step's key registers take the next but one's keys as soon as its scores are
  // there, the value registers the values after its outputs.
  Step X, Y;
  if (lo < hi) {
    find(lo);
    X.load(a.pool, tile, lane);
  }
  if (lo + 2 < hi) {
    find(lo + 2);
    Y.load(a.pool, tile, lane);
  }

  const int c0 = CW * t.cg;
#pragma unroll
  for (int n = 0; n < (NT * NF + 3) / 4; ++n) {
    const int k = wave + 4 * n, jt = k / NF, c = k % NF;
    if (k >= NT * NF) break;
    uint4 x[Parts::q];
    query_operand<IO, HD>(a, tree_column(a, t.row0, kvh, min(c0 + 16 * jt + h, t.cols - 1)), c, g, x);
#pragma unroll
    for (int q = 0; q < Parts::q; ++q) sm.q[jt][c][q][lane] = x[q];
  }
  int seen[NT];  // positions that this lane's columns see
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) seen[jt] = t.len + 1 + min(c0 + 16 * jt + h, t.cols - 1) / a.G;
  const int all = t.len + 1 + c0 / a.G;       // positions that every column sees
  const int some = t.len + 1 + (min(t.cols, c0 + CW) - 1) / a.G;
  __syncthreads();

  f32x4_t O[NT][NE], l[NT];  // l: the sum, in every register
  float m[NT];
  const auto reset = [&] {
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
      m[jt] = kTreeFloor;
      l[jt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < NE; ++e) O[jt][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  };
  const auto queries = [&](int jt, int c, int k) { return sm.q[jt][c][k][lane]; };
  bool beyond = false;  // (uniform)
  const auto compute = [&](Step& B, int i, bool more, auto tail) {
    f32x4_t S[NT][2];
    key_products<IO, HD, NT>(B, queries, S);
    if (more) {
      find(i + 4);
      B.load_keys(a.pool, tile, lane);
    }
    if constexpr (decltype(tail)::value) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int pos = 16 * (i + b) + 4 * g;
        const uint32_t keep = byte_mask(i + b < hi ? live_bits(pos, some) : 0u);
#pragma unroll
        for (int p = 0; p < P; ++p) {
          B.v[b][p] &= keep;
          B.vs[b][p] = (B.vs[b][p] & keep) | (0x7F7F7F7Fu & ~keep);
        }
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) {
          const uint32_t sees = i + b < hi ? live_bits(pos, seen[jt]) : 0u;
#pragma unroll
          for (int r = 0; r < 4; ++r) S[jt][b][r] = sees >> r & 1 ? S[jt][b][r] : -INFINITY;
        }
      }
    }
    uint32_t out = 0;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int p = 0; p < P; ++p) out |= odd_scales(B.vs[b][p]);
    if (__ballot(out != 0) != 0) {
      asm volatile("");  // (keeps what follows behind the branch)
      bool x = false;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int p = 0; p < P; ++p) x |= beyond_f16(B.v[b][p], B.vs[b][p]);
      beyond |= __ballot(x) != 0;
    }
    float p[NT][8];
    lifted_softmax<IO, NT, NE>(S, a.qscale, m, l, O, p);
    uint4 pp[NT][HalfParts<IO>::p];
#pragma unroll
    for (int jt = 0; jt < NT; ++jt)
#pragma unroll
      for (int q = 0; q < HalfParts<IO>::p; ++q) {
        pp[jt][q] = next_part_f16(p[jt]);
        l[jt] = mma_f16(l[jt], kHalfOnes, pp[jt][q]);
      }
#pragma unroll
    for (int w = 0; w < P; ++w) {
      uint2 lo2[2], hi2[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) value_halves_f16(B.v[b][w], B.vs[b][w], lo2[b], hi2[b]);
      const uint4 x0 = make_uint4(lo2[0].x, lo2[0].y, lo2[1].x, lo2[1].y), x1 = make_uint4(hi2[0].x, hi2[0].y, hi2[1].x, hi2[1].y);
#pragma unroll
      for (int q = 0; q < HalfParts<IO>::p; ++q)
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) {
          O[jt][2 * w] = mma_f16(O[jt][2 * w], x0, pp[jt][q]);
          O[jt][2 * w + 1] = mma_f16(O[jt][2 * w + 1], x1, pp[jt][q]);
        }
    }
    if (more) B.load_values(a.pool, tile, lane);
  };
  reset();
  // Whole steps without a mask, then the rest with one.
  const int whole = lo + max(0, min(hi, all / 16) - lo) / 2 * 2;
  int i = lo;
  for (; i + 2 < whole; i += 4) {
    compute(X, i, i + 4 < hi, std::false_type{});
    compute(Y, i + 2, i + 6 < hi, std::false_type{});
  }
  for (; i < hi; i += 4) {
    compute(X, i, i + 4 < hi, std::true_type{});
    if (i + 2 < hi) compute(Y, i + 2, i + 6 < hi, std::true_type{});
  }
  if (beyond) {
    reset();
    float sum[NT] = {};
    ids = ask(lo + lane);
    for (i = lo; i < hi; i += 2) {
      find(i);
      X.load(a.pool, tile, lane);
      cache_step<IO, HD, NT>(a, X, i, hi, all, some, seen, queries, m, sum, O, lane);
    }
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
      sum[jt] += __shfl_xor(sum[jt], 16);
      l[jt][0] = sum[jt] + __shfl_xor(sum[jt], 32);
    }
  }

  // Merge of the four waves, column tile by column tile; wave w combines and
  // stores output operands [w EPW, (w + 1) EPW).
#pragma unroll
  for (int jt = 0; jt < NT; ++jt)
    if (g == 0) sm.sml[wave][jt][h] = make_float2(m[jt], l[jt][0]);
  const CoherentBuffer pb(a.part, a.part_bytes);
  const uint32_t item = (static_cast<uint32_t>(t.item) * a.Hkv + kvh) * CW * (HD + 4) * 4;
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
    const TreeColumn col = tree_column(a, t.row0, kvh, c0 + c);
#pragma unroll
    for (int k = 0; k < EPW; ++k) {
      f32x4_t R = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const f32x4_t o = sm.so[v][wave * EPW + k][lane];
#pragma unroll
        for (int r = 0; r < 4; ++r) R[r] += cw[v] * o[r];
      }
      if (c0 + c >= t.cols) continue;
      const int d0 = 16 * (wave * EPW + k) + 4 * g;
      if (t.nsplit == 1) {
        IO::store4(a, col.row, col.hq * HD + d0, R * (1.f / L));
      } else {
        pb.store4(item + (c * (HD + 4) + 4 + d0) * 4, R);
        if (wave == 0 && k == 0 && g == 0) pb.store4(item + c * (HD + 4) * 4, f32x4_t{M, L, 0.f, 0.f});
      }
    }
  }
  if (t.nsplit > 1) merge_splits<IO, HD, CW>(a, t, kvh, pb, &sm.last, sm.weights);
}

// ---------------------------------------------------------------------------

// More than 32 columns.  Work-group: a request's column group of 64 NT columns
// (16 NT per wave) over the blocks of one split.  The waves share every block
// through LDS: the thread that fetched a word of codes expands it, keys to bf16
// and values to fp16, and puts it there as a piece of an operand.
//
// Probabilities enter their product in fp16: to 2^-11 of themselves for bf16
// outputs (whose own rounding is 2^-8; two parts: 313 us where one takes 235, and
// outputs 0.00166 of their norm from 64 bits instead of 0.00167), to 2^-22 in two
// parts for fp32 ones; small ones to 2^-32 and 2^-36 of the row's largest (half of
// fp16's last step, see HalfParts).  The sums in fp32 round by more: a step's 32
// positions move them by 2^-24.  Their sum is one more product, with ones.  Where
// a step meets a value that fp16 does not hold exactly, or a NaN that not all
// columns see, the work-group starts over, its waves reading the blocks themselves
// as the other kernel's do (all of them doing so: 621 us for the 232 below).
//
// Bound by the vector unit's issue (softmax and expansion) beside the products:
// 2048 rows of 32 heads behind 6150 positions, bf16, 230 us, 1050 TFLOP/s of the
// 1359 that a library product of 16384^3 reaches.  Expanded keys in each wave
// instead of once 241; a barrier per step instead of every other, and scores in
// the outputs' own step, 274; 32x32 products no faster; 256 columns 276.
template <class IO, int HD, int NT>
__global__ __launch_bounds__(256, 2) void k_cache_attn_wide(CacheAttnArgs a) {
  using F = Mx4<HD>;
  using Parts = CacheParts<IO>;
  constexpr int NF = HD / 32, NE = HD / 16, P = F::P, CW = 64 * NT;
  constexpr int kKeys = 4 * HD;                             // words of a step's key codes; as many of its values
  constexpr int W = kKeys / 256;                            // words of a thread, keys or values
  // Operands of a step's keys: piece c of block b at [(2 c + b) * 64 + lane], the
  // second half of the pieces moved by 64 bytes (a thread writes pieces of either).
  struct Keys {
    uint4 op[NF * 2 * 64 + 4];
    static __device__ __forceinline__ int at(int c, int b) { return (2 * c + b) * 64 + c / 2 * 4; }
  };
  __shared__ uint4 vals[4][NE * 64];  // of a step: operands: a lane's 8 bytes of block 0, of block 1
  __shared__ __attribute__((aligned(16))) Keys keys[4];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane & 15, g = lane >> 4;
  const int f = blockIdx.x / a.Hkv, kvh = blockIdx.x - f * a.Hkv;
  const CacheItem t = cache_item<CW>(a, f);
  if (t.count < 1) return;
  const int end = t.first + t.count, c0 = CW * t.cg + 16 * NT * wave;
  const bool busy = c0 < t.cols;  // this wave has columns
  const int all = t.len + 1 + CW * t.cg / a.G;  // positions that every column of the group sees
  const int some = t.len + 1 + (min(t.cols, CW * (t.cg + 1)) - 1) / a.G;

  // Steps are numbered from the split's start; past its end their blocks are its
  // last one (a missing second block re-reads the first, masked).  A wave fetches
  // from one block of a step.  Ids are held 64 at a time, a lane each, and asked
  // for as many ahead.
  const int steps = (t.count + 1) / 2;
  const auto ask = [&](int i) { return pool_id(a, t.btrow[min(t.first + i + lane, end - 1)]); };
  int ids = ask(0), ids_next = ask(64);

  uint4 Q[NT][NF][Parts::q];
  int seen[NT];  // positions that this lane's columns see
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    const int c = min(c0 + 16 * jt + h, t.cols - 1);
    const TreeColumn col = tree_column(a, t.row0, kvh, c);
    seen[jt] = t.len + 1 + c / a.G;
#pragma unroll
    for (int k = 0; k < NF; ++k) query_operand<IO, HD>(a, col, k, g, Q[jt][k]);
  }

  // This thread's share of a step: W words of block fb's key codes, and W value
  // words (groups vp on) of its lane vl, whose positions are 4 (vl / 16) on.
  const int fb = wave >> 1, ft = tid & 127;
  const int at = ft * W, vl = at / P, vp = at % P;
  const auto words = [](const uint8_t* p, uint32_t* w) {
    if constexpr (W == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[0] = x.x, w[1] = x.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
  };
  // This wave's tile of a step; called for each step in order.
  const auto tile_of = [&](int step) {
    const int i = min(2 * step + fb, t.count - 1);
    if ((step & 31) == 0 && step > 0) {
      ids = ids_next;
      ids_next = ask(2 * step + 64);
    }
    return a.pool + (static_cast<size_t>(__builtin_amdgcn_readlane(ids, i & 63)) * a.Hkv + kvh) * F::kTile;
  };
  struct {
    uint32_t k[W], ks, v[W], vs[W];
  } next[2] = {};  // two steps on their way into LDS
  const auto fetch_keys = [&](int n, const uint8_t* tile) {
    words(tile + at * 4, next[n].k);
    next[n].ks = tile[F::kKs + at / 4];
  };
  const auto fetch_values = [&](int n, const uint8_t* tile) {
    words(tile + F::kV + at * 4, next[n].v);
    words(tile + F::value_scales(vl / 16, vp), next[n].vs);
  };
  // Whether a step reaches past what all columns see, or past the split.
  const auto is_tail = [&](int step) { return 16 * (t.first + 2 * step + 2) > all || t.first + 2 * step + 2 > end; };
  const auto put_keys = [&](int n, Keys& to) {
    const float s = scale_of<0>(next[n].ks);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const uint32_t x = next[n].k[w];
      const int d0 = at / 64 * 32 + at % 4 * 8 + 8 * w, kg = d0 / (HD / 4), c = d0 % (HD / 4) / 8;
      to.op[Keys::at(c, fb) + at / 4 % 16 + 16 * kg] =
          make_uint4(codes_to_bf16<0>(x, s), codes_to_bf16<1>(x, s), codes_to_bf16<2>(x, s), codes_to_bf16<3>(x, s));
    }
  };
  uint32_t beyond = 0;  // not 0: this thread met a value that fp16 does not hold, or a NaN
  const auto put_values = [&](int n, int step, uint4* to, auto tail) {
    uint32_t v[W], x[W], out = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      v[w] = next[n].v[w], x[w] = next[n].vs[w];
      if constexpr (decltype(tail)::value) {
        const int b = t.first + 2 * step + fb;
        const uint32_t keep = byte_mask(b < end ? live_bits(16 * b + 4 * (vl / 16), some) : 0u);
        v[w] &= keep;
        x[w] = (x[w] & keep) | (0x7F7F7F7Fu & ~keep);
      }
      out |= odd_scales(x[w]);
    }
    if (__ballot(out != 0) != 0) {
      asm volatile("");  // (keeps what follows behind the branch: 247 us where checking every word took 255)
#pragma unroll
      for (int w = 0; w < W; ++w) beyond |= beyond_f16(v[w], x[w]) ? 1u : 0u;
    }
#pragma unroll
    for (int w = 0; w < W; ++w) {
      uint2 lo, hi;
      value_halves_f16(v[w], x[w], lo, hi);
      uint2* op = reinterpret_cast<uint2*>(to + 2 * (vp + w) * 64 + vl) + fb;
      op[0] = lo;
      op[128] = hi;
    }
  };

  f32x4_t O[NT][NE], l[NT];  // l: the sum, in every register
  float m[NT];
  const auto reset = [&] {
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
      m[jt] = kTreeFloor;
      l[jt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < NE; ++e) O[jt][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  };
  struct Scores {
    f32x4_t x[NT][2];
  };
  const auto scores = [&](int step, const Keys& from, Scores& S, auto tail) {
#pragma unroll
    for (int jt = 0; jt < NT; ++jt)
#pragma unroll
      for (int b = 0; b < 2; ++b) S.x[jt][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NF; ++c)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint4 x = from.op[Keys::at(c, b) + lane];
#pragma unroll
        for (int q = 0; q < Parts::q; ++q)
#pragma unroll
          for (int jt = 0; jt < NT; ++jt) S.x[jt][b] = BF16::mma(S.x[jt][b], x, Q[jt][c][q]);
      }
    if constexpr (decltype(tail)::value) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int block = t.first + 2 * step + b, pos = 16 * block + 4 * g;
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) {
          const uint32_t sees = block < end ? live_bits(pos, seen[jt]) : 0u;
#pragma unroll
          for (int r = 0; r < 4; ++r) S.x[jt][b][r] = sees >> r & 1 ? S.x[jt][b][r] : -INFINITY;
        }
      }
    }
  };
  const auto outputs = [&](const Scores& S, const uint4* from) {
    float p[NT][8];
    lifted_softmax<IO, NT, NE>(S.x, a.qscale, m, l, O, p);
    uint4 pp[NT][HalfParts<IO>::p];
#pragma unroll
    for (int jt = 0; jt < NT; ++jt)
#pragma unroll
      for (int q = 0; q < HalfParts<IO>::p; ++q) {
        pp[jt][q] = next_part_f16(p[jt]);
        l[jt] = mma_f16(l[jt], kHalfOnes, pp[jt][q]);
      }
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      const uint4 x = from[e * 64 + lane];
#pragma unroll
      for (int q = 0; q < HalfParts<IO>::p; ++q)
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) O[jt][e] = mma_f16(O[jt][e], x, pp[jt][q]);
    }
    // Schedule: three operands ahead of the exponentials, the others between the
    // products, so that none is waited for (236 us without).
    __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
    __builtin_amdgcn_sched_group_barrier(0x402, NT * 12, 0);
    const auto group = [](auto) {
      __builtin_amdgcn_sched_group_barrier(0x8, NT * HalfParts<IO>::p, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    };
    static_for<NE>(group);
  };

  // Pair q of steps, 2q and 2q + 1.  While it is computed the next pair's values
  // and the keys of the two steps from 2q + 3 on go to LDS, and what follows them
  // is fetched; scores run a step ahead of the outputs, so that their products run
  // while scores become probabilities.  One barrier per pair.
  const auto walk = [&](auto busy_wave) {
    constexpr bool kBusy = decltype(busy_wave)::value;
    constexpr std::integral_constant<int, 0> kEven{};
    constexpr std::integral_constant<int, 1> kOdd{};
    Scores S[2];
    const uint8_t* first;  // tile of the first step whose values are fetched next
    int asked = 1;         // step whose keys are
    const auto fetch = [&] {
      const uint8_t *t0 = tile_of(asked), *t1 = tile_of(asked + 1);
      fetch_keys(0, t0);
      fetch_keys(1, t1);
      fetch_values(0, first);
      fetch_values(1, t0);
      first = t1;
      asked += 2;
    };
    const auto put = [&](int q, auto parity, auto tail) {
      constexpr int to = 2 * decltype(parity)::value;
      put_keys(0, keys[to + 1]);
      put_keys(1, keys[(to + 2) & 3]);
      put_values(0, 2 * q, vals[to], tail);
      put_values(1, 2 * q + 1, vals[to + 1], tail);
    };
    const auto pair = [&](int q, auto parity, auto other, auto tail) {
      constexpr int from = 2 * decltype(parity)::value;
      __syncthreads();
      put(q + 1, other, tail);
      fetch();
      if constexpr (kBusy) {
        scores(2 * q + 1, keys[from + 1], S[1], tail);
        outputs(S[0], vals[from]);
        scores(2 * q + 2, keys[(from + 2) & 3], S[0], tail);
        outputs(S[1], vals[from + 1]);
      }
    };
    first = tile_of(0);
    fetch_keys(0, first);
    put_keys(0, keys[0]);
    fetch();
    put(0, kEven, std::true_type{});
    fetch();
    __syncthreads();
    if constexpr (kBusy) scores(0, keys[0], S[0], std::true_type{});
    const int pairs = (steps + 1) / 2;
    int q = 0;
    for (; q + 1 < pairs && !is_tail(2 * q + 5); q += 2) {
      pair(q, kEven, kOdd, std::false_type{});
      pair(q + 1, kOdd, kEven, std::false_type{});
    }
    for (; q < pairs; q += 2) {
      pair(q, kEven, kOdd, std::true_type{});
      if (q + 1 < pairs) pair(q + 1, kOdd, kEven, std::true_type{});
    }
  };
  // Two walks, not a condition in one: where some steps leave the accumulators as
  // they are, the compiler copies them all after each step's products.
  reset();
  if (busy) walk(std::true_type{});
  else walk(std::false_type{});
  if (__syncthreads_or(static_cast<int>(beyond))) {
    reset();
    float sum[NT] = {};
    const auto queries = [&](int jt, int c, int k) { return Q[jt][c][k]; };
    for (int i = t.first; i < end && busy; i += 2) {
      const size_t tile[2] = {static_cast<size_t>(pool_id(a, t.btrow[i])) * a.Hkv + kvh,
                              static_cast<size_t>(pool_id(a, t.btrow[min(i + 1, end - 1)])) * a.Hkv + kvh};
      CacheStep<HD> B;
      B.load(a.pool, tile, lane);
      cache_step<IO, HD, NT>(a, B, i, end, all, some, seen, queries, m, sum, O, lane);
    }
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
      sum[jt] += __shfl_xor(sum[jt], 16);
      l[jt][0] = sum[jt] + __shfl_xor(sum[jt], 32);
    }
  }

  const CoherentBuffer pb(a.part, a.part_bytes);
  const uint32_t item = (static_cast<uint32_t>(t.item) * a.Hkv + kvh) * CW * (HD + 4) * 4;
  if (!busy) return;
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    const int c = 16 * (NT * wave + jt) + h;  // within the group
    if (CW * t.cg + c >= t.cols) continue;
    const TreeColumn col = tree_column(a, t.row0, kvh, CW * t.cg + c);
    const float inv = 1.f / l[jt][0];
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      const int d0 = 16 * e + 4 * g;
      if (t.nsplit == 1) IO::store4(a, col.row, col.hq * HD + d0, O[jt][e] * inv);
      else pb.store4(item + (c * (HD + 4) + 4 + d0) * 4, O[jt][e]);
    }
    if (t.nsplit > 1 && g == 0) pb.store4(item + c * (HD + 4) * 4, f32x4_t{m[jt], l[jt][0], 0.f, 0.f});
  }
}

// Merge of the wide kernel's splits in a launch of its own, whose work-groups
// share out all outputs: 16 columns of one (column group of CW, KV head) each.
// (One last arrival would have 64 or 128 columns of up to 64 splits to itself.)
constexpr int kMergeWide = 16;
template <class IO, int HD, int CW>
__global__ __launch_bounds__(256) void k_cache_merge(CacheAttnArgs a) {
  constexpr int kPer = HD / 4, kMine = kMergeWide * kPer / 256, kChunk = 8, kLane = kCacheSplits / 16;
  __shared__ float weights[kCacheSplits * kMergeWide];
  const int tid = threadIdx.x, lane = tid & 63;
  constexpr int kParts = CW / kMergeWide;
  const int part16 = blockIdx.x % kParts, gk = blockIdx.x / kParts;
  const int group = gk / a.Hkv, kvh = gk - group * a.Hkv;
  int before = 0;  // requests whose first column group is not behind this one
  for (int k = 0; k < a.n; k += 64)
    before += __popcll(__ballot(k + lane < a.n && a.cg0[min(k + lane, a.n - 1)] <= group));
  const int r = __builtin_amdgcn_readfirstlane(before) - 1;
  const int cols = a.rows[r] * a.G, ncg = (cols + CW - 1) / CW, cg = group - a.cg0[r];
  const int nblk = (a.len[r] + (min(cols, (cg + 1) * CW) - 1) / a.G + 16) >> 4;
  const int nsplit = (nblk + a.bps - 1) / a.bps;
  const int c0 = part16 * kMergeWide;  // within the group
  if (nsplit == 1 || CW * cg + c0 >= cols) return;
  const int mine = min(cols - CW * cg - c0, kMergeWide);
  constexpr size_t kColumn = HD + 4;
  const float* part = a.part + ((static_cast<size_t>(a.item0[r] + cg) * a.Hkv + kvh) * CW + c0) * kColumn;
  const size_t stride = static_cast<size_t>(ncg) * a.Hkv * CW * kColumn;
  // A lane per (column, split): maximum and sum; sixteen lanes share a column.
  const float* ml = part + min(tid / 16, mine - 1) * kColumn;
  float sm[kLane], sl[kLane], M = kTreeFloor;
#pragma unroll
  for (int k = 0; k < kLane; ++k) {
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
#pragma unroll
  for (int k = 0; k < kLane; ++k) M = fmaxf(M, sm[k]);
#pragma unroll
  for (int x = 8; x >= 1; x >>= 1) M = fmaxf(M, __shfl_xor(M, x));
  float w[kLane], L = 0.f;
#pragma unroll
  for (int k = 0; k < kLane; ++k) {
    w[k] = __builtin_amdgcn_exp2f(sm[k] - M);
    L += sl[k] * w[k];
  }
#pragma unroll
  for (int x = 8; x >= 1; x >>= 1) L += __shfl_xor(L, x);
  const float inv = 1.f / L;
#pragma unroll
  for (int k = 0; k < kLane; ++k) weights[(tid % 16 + 16 * k) * kMergeWide + tid / 16] = w[k] * inv;
  __syncthreads();
  for (int s0 = 0;;) {
#pragma unroll
    for (int k = 0; k < kChunk; ++k)
      if (s0 + k < nsplit) {
#pragma unroll
        for (int n = 0; n < kMine; ++n) R[n] += weights[(s0 + k) * kMergeWide + (tid + 256 * n) / kPer] * o[n][k];
      }
    s0 += kChunk;
    if (s0 >= nsplit) break;
    load(s0);
  }
#pragma unroll
  for (int n = 0; n < kMine; ++n) {
    const int idx = tid + 256 * n, c = idx / kPer;
    if (c >= mine) break;
    const TreeColumn col = tree_column(a, a.row0[r], kvh, CW * cg + c0 + c);
    IO::store4(a, col.row, col.hq * HD + idx % kPer * 4, R[n]);
  }
}

}  // namespace sprk
