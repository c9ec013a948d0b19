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

// ---------------------------------------------------------------------------

// Positions 0 .. 3 of dimensions e (low nibbles) and e + 16 of a word, in fp16.
__device__ __forceinline__ void value_halves_f16(uint32_t w, uint32_t scales, uint2& lo, uint2& hi) {
  const uint32_t x0 = codes_to_f16<0>(w, scale_of<0>(scales)), x1 = codes_to_f16<1>(w, scale_of<1>(scales));
  const uint32_t x2 = codes_to_f16<2>(w, scale_of<2>(scales)), x3 = codes_to_f16<3>(w, scale_of<3>(scales));
  lo = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x05040100u), __builtin_amdgcn_perm(x3, x2, 0x05040100u));
  hi = make_uint2(__builtin_amdgcn_perm(x1, x0, 0x07060302u), __builtin_amdgcn_perm(x3, x2, 0x07060302u));
}

// Whether a word's values are not all exact in fp16: a scale outside 2^-18 ..
// 2^13 (bytes 109 .. 140: a byte out of that range leaves a top bit, and the
// lowest such byte has no borrow from below) with codes that are not zero, or a
// NaN.
__device__ __forceinline__ bool beyond_f16(uint32_t w, uint32_t scales) {
  return ((scales - 0x6D6D6D6Du) & 0xE0E0E0E0u) != 0 && ((w & 0x77777777u) != 0 || nan_bytes(scales) != 0);
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

// More than 32 columns.  Work-group: a request's column group of 64 NT columns
// (16 NT per wave) over the blocks of one split.  Its waves share every block
// through LDS: keys as codes, which each wave expands to bf16 in registers,
// values expanded to fp16 by the thread that fetched them.  While a step is
// computed from LDS, the next one's codes lie in registers or arrive there, and
// the one's after it are asked for; after the step the next one goes to the
// other LDS buffer: one barrier per step.
//
// Probabilities enter their product in fp16: 2^-12 of themselves for bf16
// outputs (whose own rounding is 2^-8), 2^-23 in two parts for fp32 ones.  Held
// 2^7 above the running maximum's place they keep those bits down to 2^-21 of
// the largest.  A step with a value that fp16 does not hold exactly, or a NaN
// that not all columns see, takes its values from memory once more, as the
// other kernel does.
template <class IO>
struct WideParts {
  static constexpr int p = IO::kRaw ? 1 : 2;
};
constexpr int kWideLift = 7;

template <class IO, int HD, int NT>
__global__ __launch_bounds__(256, 2) void k_cache_attn_wide(CacheAttnArgs a) {
  using F = Mx4<HD>;
  using Parts = CacheParts<IO>;
  constexpr int NF = HD / 32, NE = HD / 16, P = F::P, CW = 64 * NT;
  constexpr int W = HD / 64;                       // words of a thread, keys or values
  constexpr int kKeys = 2 * 8 * HD / 4;            // words of a step's key codes
  constexpr int kScales = HD / 4;                  // and key scales
  __shared__ uint4 vals[2][NE * 64];               // operands: lane's 8 bytes of block 0, of block 1
  __shared__ __attribute__((aligned(16))) uint32_t keys[2][kKeys + kScales];
  __shared__ int slow_s[2];
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

  // Block ids are asked for one step before the blocks they name; past the
  // split's end they are its last one's (a missing second block re-reads the
  // first, masked).
  int ids[2];
  const auto ask = [&](int i) {
#pragma unroll
    for (int b = 0; b < 2; ++b) ids[b] = t.btrow[min(i + b, end - 1)];
  };
  ask(t.first);

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
  f32x4_t O[NT][NE];
  float m[NT], l[NT];
#pragma unroll
  for (int jt = 0; jt < NT; ++jt) {
    m[jt] = kTreeFloor;
    l[jt] = 0.f;
#pragma unroll
    for (int e = 0; e < NE; ++e) O[jt][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // This thread's share of a step: W words of block tid / 128's key codes, and W
  // value words (groups vp on) of its lane vl, whose positions are 4 (vl / 16) on.
  const int fb = tid >> 7, at = (tid & 127) * W;
  const int vl = at / P, vp = at % P;
  struct Next {
    uint32_t k[W], v[W], vs[W], ks;
  } next[2];  // of even and odd steps
  const auto words = [](const uint8_t* p, uint32_t* w) {
    if constexpr (W == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[0] = x.x, w[1] = x.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
  };
  const auto fetch = [&](int then, auto parity) {
    Next& x = next[decltype(parity)::value];
    const uint8_t* tile[2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
      tile[b] = a.pool + (static_cast<size_t>(__builtin_amdgcn_readfirstlane(pool_id(a, ids[b]))) * a.Hkv + kvh) * F::kTile;
    ask(then);
    const uint8_t* mine = fb ? tile[1] : tile[0];
    words(mine + at * 4, x.k);
    words(mine + F::kV + at * 4, x.v);
    words(mine + F::value_scales(vl / 16, vp), x.vs);
    // Key scales of both blocks: HD / 8 words each, by the first threads.
    if (tid < kScales)
      x.ks = *reinterpret_cast<const uint32_t*>((tid < kScales / 2 ? tile[0] : tile[1]) + F::kKs + tid % (kScales / 2) * 4);
  };
  const auto put = [&](int i, auto parity, auto tail) {
    constexpr int to = decltype(parity)::value;
    Next& x = next[to];
    uint32_t* k = keys[to] + fb * (kKeys / 2) + at;
#pragma unroll
    for (int w = 0; w < W; ++w) k[w] = x.k[w];
    if (tid < kScales) keys[to][kKeys + tid] = x.ks;
    uint32_t live = 15;
    if constexpr (decltype(tail)::value) live = i + fb < end ? live_bits(16 * (i + fb) + 4 * (vl / 16), some) : 0u;
    bool beyond = false;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      uint32_t v = x.v[w], s = x.vs[w];
      if constexpr (decltype(tail)::value) {
        const uint32_t keep = byte_mask(live);
        v &= keep;
        s = (s & keep) | (0x7F7F7F7Fu & ~keep);
      }
      beyond |= beyond_f16(v, s);
      uint2 lo, hi;
      value_halves_f16(v, s, lo, hi);
      uint2* op = reinterpret_cast<uint2*>(vals[to] + 2 * (vp + w) * 64 + vl) + fb;
      op[0] = lo;
      op[128] = hi;
    }
    if (__ballot(beyond) != 0 && lane == 0) slow_s[to] = i + 1;
  };
  const auto is_tail = [&](int i) { return 16 * (i + 2) > all || i + 2 > end; };
  const auto compute = [&](int i, auto parity, auto tail) {
    constexpr int from = decltype(parity)::value;
    f32x4_t S[NT][2];
#pragma unroll
    for (int jt = 0; jt < NT; ++jt)
#pragma unroll
      for (int b = 0; b < 2; ++b) S[jt][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint8_t* kb = reinterpret_cast<const uint8_t*>(keys[from]) + b * (kKeys * 2);
      uint32_t kw[P];
      if constexpr (P == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(kb + F::key_code(h, HD / 4 * g));
        kw[0] = x.x, kw[1] = x.y, kw[2] = x.z, kw[3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(kb + F::key_code(h, HD / 4 * g));
        kw[0] = x.x, kw[1] = x.y;
      }
      const uint8_t* sb = reinterpret_cast<const uint8_t*>(keys[from] + kKeys) + b * (HD / 2);
      const float ks = scale_of<0>(sb[HD / 4 * g / 32 * 16 + h]);
#pragma unroll
      for (int c = 0; c < NF; ++c) {
        const uint4 x = make_uint4(codes_to_bf16<0>(kw[c], ks), codes_to_bf16<1>(kw[c], ks), codes_to_bf16<2>(kw[c], ks),
                                   codes_to_bf16<3>(kw[c], ks));
#pragma unroll
        for (int q = 0; q < Parts::q; ++q)
#pragma unroll
          for (int jt = 0; jt < NT; ++jt) S[jt][b] = BF16::mma(S[jt][b], x, Q[jt][c][q]);
      }
    }
    uint32_t live[2], sees[NT][2];
    if constexpr (decltype(tail)::value) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int pos = 16 * (i + b) + 4 * g;
        live[b] = i + b < end ? live_bits(pos, some) : 0u;
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) {
          sees[jt][b] = live[b] & live_bits(pos, seen[jt]);
#pragma unroll
          for (int r = 0; r < 4; ++r) S[jt][b][r] = sees[jt][b] >> r & 1 ? S[jt][b][r] : -INFINITY;
        }
      }
    }
    float p[NT][2][4];
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) softmax_step<2, NE, kWideLift>(S[jt], a.qscale, m[jt], l[jt], O[jt], p[jt]);
    if (slow_s[from] == i + 1) {
      CacheStep<HD> B;
      const size_t tile[2] = {static_cast<size_t>(pool_id(a, t.btrow[i])) * a.Hkv + kvh,
                              static_cast<size_t>(pool_id(a, t.btrow[min(i + 1, end - 1)])) * a.Hkv + kvh};
      B.load(a.pool, tile, lane);
      uint32_t odd[2][P];
      bool any = false;
      if constexpr (decltype(tail)::value) any = __ballot(B.mask_values(live, odd)) != 0;
#pragma unroll
      for (int jt = 0; jt < NT; ++jt) {
        float v[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = p[jt][r / 4][r % 4];
        uint4 x[Parts::p];
#pragma unroll
        for (int q = 0; q < Parts::p; ++q) x[q] = next_part<BF16>(v);
        B.template pv<Parts::p>(O[jt], x);
        if constexpr (decltype(tail)::value)
          if (any) add_nan_values<P>(O[jt], odd, sees[jt]);
      }
      return;
    }
    uint4 pp[NT][WideParts<IO>::p];
#pragma unroll
    for (int jt = 0; jt < NT; ++jt) {
      float v[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] = p[jt][r / 4][r % 4];
#pragma unroll
      for (int q = 0; q < WideParts<IO>::p; ++q) pp[jt][q] = next_part_f16(v);
    }
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      const uint4 x = vals[from][e * 64 + lane];
#pragma unroll
      for (int q = 0; q < WideParts<IO>::p; ++q)
#pragma unroll
        for (int jt = 0; jt < NT; ++jt) O[jt][e] = mma_f16(O[jt][e], x, pp[jt][q]);
    }
  };
  constexpr std::false_type kPlain{};
  constexpr std::true_type kTail{};
  constexpr std::integral_constant<int, 0> kEven{};
  constexpr std::integral_constant<int, 1> kOdd{};
  // One step: fetch the one after the next, compute, put the next.  Whole steps
  // do so without a condition.
  const auto step = [&](int i, auto parity, auto other, auto tail) {
    constexpr bool whole = !decltype(tail)::value;
    __syncthreads();  // this step is in its buffer; the other buffer has been read
    if (whole || i + 4 < end) fetch(i + 6, parity);
    if (busy) compute(i, parity, tail);
    if (whole || i + 2 < end) put(i + 2, other, tail);
  };
  if (tid < 2) slow_s[tid] = 0;
  __syncthreads();
  int i = t.first;
  fetch(i + 2, kEven);
  fetch(i + 4, kOdd);
  if (is_tail(i)) put(i, kEven, kTail);
  else put(i, kEven, kPlain);
  for (; i + 6 < end && !is_tail(i + 4); i += 4) {  // two steps and the one after them are whole
    step(i, kEven, kOdd, kPlain);
    step(i + 2, kOdd, kEven, kPlain);
  }
  for (; i < end; i += 4) {
    step(i, kEven, kOdd, kTail);
    if (i + 2 < end) step(i + 2, kOdd, kEven, kTail);
  }

  const CoherentBuffer pb(a.part, a.part_bytes);
  const uint32_t item = (static_cast<uint32_t>(f) * a.Hkv + kvh) * CW * (HD + 4) * 4;
  if (!busy) return;
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

// Merge of the wide kernel's splits in a launch of its own, whose work-groups
// share out all outputs: 16 columns of one (column group of CW, KV head) each.
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
