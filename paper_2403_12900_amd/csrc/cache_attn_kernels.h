// Attention over the 4-bit cache: row j of a request and head h,
//   out[r][h] = softmax(q[r][h] . K^T / sqrt(hd)) V
// over the request's positions 0 .. len + j.
//
// The columns of one (request, KV head) are (row, head of the group): c = j * G
// + head.  On MFMA, per block of 16 positions and tile of 16 columns:
//   S[t][c]   = K_tile(16 x hd) . Q^T(hd x 16)
//   O^T[e][c] += V^T_tile(16 dims x positions) . P(positions x 16)
// with P the S accumulator re-used in place as the B operand; two blocks make
// one 16x16x32 product.
//
// Codes times their scales are exact in bf16, and so are the products of
// fp32 queries in three bf16 parts; the probabilities enter their product in
// three parts for fp32 outputs (24 bits) and in two for bf16 ones (16 bits).
#pragma once

#include <type_traits>

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
  int len, nblk, row0, cols;  // nblk: blocks that the column group's rows see
  int first, count;           // blocks of the split (count < 1: nothing to do)
  const int32_t* btrow;
};
template <int CW>
__device__ __forceinline__ CacheItem cache_item(const CacheAttnArgs& a, int f) {
  const int lane = threadIdx.x & 63;
  int rank = 0;
  for (int k = 0; k < a.n; k += 64)
    rank += __popcll(__ballot(k + lane < a.n && a.item0[min(k + lane, a.n - 1) + 1] <= f));
  const int r = __builtin_amdgcn_readfirstlane(rank);
  CacheItem t;
  t.item0 = a.item0[r];
  t.cg0 = a.cg0[r];
  t.len = a.len[r];
  t.row0 = a.row0[r];
  t.cols = a.rows[r] * a.G;
  t.ncg = (t.cols + CW - 1) / CW;
  const int w = f - t.item0, s = w / t.ncg;
  t.cg = w - s * t.ncg;  // column groups of one split run side by side and share its blocks
  const int last = (min(t.cols, (t.cg + 1) * CW) - 1) / a.G;  // row
  t.nblk = (t.len + last + 16) >> 4;
  t.nsplit = (t.nblk + a.bps - 1) / a.bps;
  t.first = a.bps * s;
  t.count = min(t.nblk - t.first, a.bps);
  t.btrow = a.bt + static_cast<size_t>(a.slot[r]) * a.mb;
  return t;
}
__device__ __forceinline__ int pool_id(const CacheAttnArgs& a, int id) {
  if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.nb)) {
    raise_check(a.err, kErrBlockId);
    id = 0;
  }
  return id;
}

// Bytes whose bit of b (4 of them) is set, as a mask.
__device__ __forceinline__ uint32_t byte_mask(uint32_t b) { return ((b * 0x00204081u) & 0x01010101u) * 255u; }

// Which of a word's scale bytes are 255 (NaN): the top bit of each.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & w & 0x80808080u; }
__device__ __forceinline__ uint32_t nan_bits(uint32_t w) {
  const uint32_t x = nan_bytes(w) >> 7;
  return (x | x >> 7 | x >> 14 | x >> 21) & 15u;
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
  __device__ __forceinline__ void load(const uint8_t* pool, const size_t* tile, int lane) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint8_t* t = pool + tile[b] * F::kTile;
      words<P>(t + key_at(r, g), k[b]);
      ks[b] = t[F::key_scale(r, HD / 4 * g / 32)];
      words<P>(t + F::value_word(g, r, 0), v[b]);
      words<P>(t + F::value_scales(g, 0), vs[b]);
    }
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
  QueryPiece p{};
  p.x = *reinterpret_cast<const uint4*>(src);
  if constexpr (!IO::kRaw) p.y = *reinterpret_cast<const uint4*>(src + 4);
  query_parts<BF16, IO>(p, out);
}

// Up to 32 columns: the four waves of a work-group take runs of the split's
// blocks, K and V go straight into registers, and the waves' results are merged
// through LDS, the splits' by the one that arrives last.
template <class IO, int HD, int NT>
__global__ __launch_bounds__(256, 2) void k_cache_attn(CacheAttnArgs a) {
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
  int end[NT];  // positions that this lane's columns see
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) end[jt] = t.len + 1 + min(c0 + 16 * jt + h, t.cols - 1) / a.G;
  const int all = t.len + 1 + c0 / a.G;       // positions that every column sees
  const int some = t.len + 1 + (min(t.cols, c0 + CW) - 1) / a.G;
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

  const auto tile_of = [&](int i) {
    return static_cast<size_t>(__builtin_amdgcn_readlane(ids, (i - lo) & 63)) * a.Hkv + kvh;
  };
  // The blocks of the step at i; a missing second one re-reads the first, masked.
  const auto fetch = [&](Step& B, int i) {
    if (((i - lo) & 63) == 0 && i != lo) ids = ask(i + lane);
    const size_t tile[2] = {tile_of(i), tile_of(i + 1 < hi ? i + 1 : i)};
    B.load(a.pool, tile, lane);
  };
  const auto compute = [&](Step& B, int i) {
    f32x4_t S[NT][2];
#pragma unroll
    for (int jt = 0; jt < NT; ++jt)
#pragma unroll
      for (int b = 0; b < 2; ++b) S[jt][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NF; ++c)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint4 x = B.key(b, c);
#pragma unroll
        for (int jt = 0; jt < NT; ++jt)
#pragma unroll
          for (int q = 0; q < Parts::q; ++q) S[jt][b] = BF16::mma(S[jt][b], x, sm.q[jt][c][q][lane]);
      }
    // A step that reaches past what all columns see, or past the run, is masked.
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
          sees[jt][b] = live[b] & live_bits(pos, end[jt]);
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
      for (int q = 0; q < Parts::p; ++q) x[q] = next_part<BF16>(v);
      B.template pv<Parts::p>(O[jt], x);
      if (any) add_nan_values<P>(O[jt], odd, sees[jt]);
    }
  };
  Step A, B;
  if (lo < hi) fetch(A, lo);
  for (int i = lo; i < hi; i += 4) {
    if (i + 2 < hi) fetch(B, i + 2);
    compute(A, i);
    if (i + 2 >= hi) break;
    if (i + 4 < hi) fetch(A, i + 4);
    compute(B, i + 2);
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

}  // namespace sprk
