// Rotary positions, and rows of keys and values into and out of the 4-bit cache.
#pragma once

#include "cache_format.h"
#include "cache_rule.h"

namespace sprk {

struct RotaryArgs {
  int dims, pairs;
  double amplitude;
  double turns[64];
};
inline RotaryArgs rotary_args(const spr_rotary& r) {
  RotaryArgs a{};
  a.dims = r.dims;
  a.pairs = r.pairs;
  a.amplitude = r.amplitude;
  for (int k = 0; k < r.dims / 2; ++k) a.turns[k] = r.turns[k];
  return a;
}

// (cos, sin) of pair k at a position, times the amplitude.  The angle is held
// in turns: its whole ones drop out exactly, so positions far out lose nothing
// but the product's rounding (2^-53 of the angle).
__device__ __forceinline__ double2 rotary_turn(const RotaryArgs& a, int position, int k) {
  double t = position * a.turns[k];
  t -= rint(t);
  double s, c;
  sincospi(2 * t, &s, &c);
  return make_double2(a.amplitude * c, a.amplitude * s);
}

// 16 bytes of a row as fp32 (N = 4: fp32, 8: bf16) and back.
template <int N>
struct RowPiece;
template <>
struct RowPiece<4> {
  using elem = float;
  static __device__ __forceinline__ void load(const void* p, float* x) {
    const float4 v = *static_cast<const float4*>(p);
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  }
  static __device__ __forceinline__ void store(void* p, const float* x) {
    *static_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  }
  static __device__ __forceinline__ float one(const void* p) { return *static_cast<const float*>(p); }
};
template <>
struct RowPiece<8> {
  using elem = uint16_t;
  static __device__ __forceinline__ void load(const void* p, float* x) {
    const uint4 v = *static_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void store(void* p, const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = f32_to_bf16_bits(x[2 * j]) | static_cast<uint32_t>(f32_to_bf16_bits(x[2 * j + 1])) << 16;
    *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float one(const void* p) { return bf16_bits_to_f32(*static_cast<const uint16_t*>(p)); }
};

// Partners of the N elements from dimension d0 of a head (in the half layout;
// of no use where a dimension is not turned).
template <int N>
__device__ __forceinline__ void load_partners(const typename RowPiece<N>::elem* head, int d0, int dims, float* y) {
  const int half = dims / 2;
  if (half % N == 0) {  // whole pieces
    if (d0 < dims) RowPiece<N>::load(head + (d0 < half ? d0 + half : d0 - half), y);
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int d = d0 + j;
    y[j] = d < dims ? RowPiece<N>::one(head + (d < half ? d + half : d - half)) : 0.f;
  }
}

// Element j of the N from d0 on, turned; cs: this position's table of (cos, sin).
template <int N>
__device__ __forceinline__ double turn_element(const float* x, const float* y, int j, int d0, int dims, int pairs,
                                               const double2* cs) {
  const int d = d0 + j;
  if (d >= dims) return x[j];
  const int half = dims / 2;
  const int k = pairs ? d >> 1 : d < half ? d : d - half;
  const bool first = pairs ? (j & 1) == 0 : d < half;
  const float beside = x[j ^ 1], across = y[j];
  const float other = pairs ? beside : across;
  const double2 t = cs[k];
  return first ? fma(static_cast<double>(x[j]), t.x, -(static_cast<double>(other) * t.y))
               : fma(static_cast<double>(x[j]), t.x, static_cast<double>(other) * t.y);
}

// ---------------------------------------------------------------------------

struct RotaryCall {
  RotaryArgs r;
  const int32_t* positions;
  const void* x;
  void* out;
  int64_t xs, os;
  int heads, per;  // heads of a work-group
};

// Grid (rows, head groups): the row's table of sines first, then its heads, a
// 16-byte piece per thread.  A head's threads lie in one wave, whose loads all
// come before its stores: x may be turned in place.
template <int N, int HD>
__global__ __launch_bounds__(256) void k_rotary(RotaryCall a) {
  using Piece = RowPiece<N>;
  using E = typename Piece::elem;
  constexpr int kPieces = HD / N;
  __shared__ double2 cs[HD / 2];
  const int row = blockIdx.x, tid = threadIdx.x;
  const int h0 = blockIdx.y * a.per, h1 = min(h0 + a.per, a.heads);
  if (tid < a.r.dims / 2) cs[tid] = rotary_turn(a.r, a.positions[row], tid);
  __syncthreads();
  const E* x = static_cast<const E*>(a.x) + row * a.xs;
  E* out = static_cast<E*>(a.out) + row * a.os;
  const int d0 = tid % kPieces * N;
  for (int h = h0 + tid / kPieces; h < h1; h += 256 / kPieces) {
    float v[N], y[N] = {}, r[N];
    Piece::load(x + h * HD + d0, v);
    if (!a.r.pairs) load_partners<N>(x + h * HD, d0, a.r.dims, y);
#pragma unroll
    for (int j = 0; j < N; ++j) r[j] = static_cast<float>(turn_element<N>(v, y, j, d0, a.r.dims, a.r.pairs, cs));
    Piece::store(out + h * HD + d0, r);
  }
}

// ---------------------------------------------------------------------------

// The blocks that a batch's rows lie in: tile0[i] counts those of the requests
// before i.
struct CacheRowsArgs {
  const int32_t* bt;
  uint8_t* pool;  // this layer
  int* err;
  const void *k, *v;  // (read: written)
  int64_t ks, vs;
  int n, Hkv, mb, nb, per;  // per: KV heads of a work-group
  int turned;
  RotaryArgs r;
  int slot[kCacheReqs], len[kCacheReqs], row0[kCacheReqs + 1];
  int tile0[kCacheReqs + 1];
};
static_assert(sizeof(CacheRowsArgs) <= 3584, "kernel arguments");

struct CacheTile {
  int first, end;  // positions 16 b + [first, end) of block b
  int base;        // row of position 16 b (before the request's first row where first > 0)
  int pos;         // 16 b
  int id;
};
__device__ __forceinline__ CacheTile cache_tile(const CacheRowsArgs& a, int f) {
  const int lane = threadIdx.x & 63;
  int rank = 0;
  for (int k = 0; k < a.n; k += 64)
    rank += __popcll(__ballot(k + lane < a.n && a.tile0[min(k + lane, a.n - 1) + 1] <= f));
  const int i = __builtin_amdgcn_readfirstlane(rank);
  const int len = a.len[i], total = len + a.row0[i + 1] - a.row0[i];
  const int b = len / 16 + f - a.tile0[i];
  CacheTile t;
  t.pos = 16 * b;
  t.first = max(len - t.pos, 0);
  t.end = min(total - t.pos, 16);
  t.base = a.row0[i] + t.pos - len;
  t.id = a.bt[static_cast<size_t>(a.slot[i]) * a.mb + b];
  return t;
}

// Lane of a wave: KV head `head` of the wave's 128 / HD, positions 4 g .. 4 g +
// 3 of the tile and eight dimensions from 8 m on.
template <int HD>
struct RowLane {
  int head, g, m;
  __device__ __forceinline__ RowLane() {
    const int lane = threadIdx.x & 63;
    m = lane % (HD / 8);
    g = lane / (HD / 8) & 3;
    head = lane / (HD / 2);
  }
};

template <int N>
__device__ __forceinline__ void load8(const typename RowPiece<N>::elem* p, float* x) {
#pragma unroll
  for (int j = 0; j < 8; j += N) RowPiece<N>::load(p + j, x + j);
}

// Largest magnitude (bits) of the group of 32 dimensions that four lanes hold;
// above infinity's where one is NaN.
__device__ __forceinline__ uint32_t group_top(const float* x) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
  return max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
}

// Eight values as a scale byte and codes (0 in a NaN group).
__device__ __forceinline__ uint32_t quantise(const float* x, uint32_t& byte) {
  byte = scale_byte(group_top(x));
  return byte == 255 ? 0u : to_codes(x, __uint_as_float(byte << 23));
}

// Append: a work-group takes a tile's rows of `per` KV heads, a wave 128 / HD
// of them at a time.  Keys: a lane's eight codes are a word of the tile.
// Values: it trades half its codes with the lane 16 dimensions on, and has four
// bytes of each of its four positions, stored as four words where the call
// writes all four positions, else byte by byte.
template <int N, int HD>
__global__ __launch_bounds__(256) void k_cache_append(CacheRowsArgs a) {
  using F = Mx4<HD>;
  using E = typename RowPiece<N>::elem;
  constexpr int kHeads = 4 * (128 / HD);  // at a time
  __shared__ double2 cs[16][HD / 2];
  const CacheTile t = cache_tile(a, blockIdx.x);
  if (static_cast<unsigned>(t.id) >= static_cast<unsigned>(a.nb)) {
    if (threadIdx.x == 0) raise_check(a.err, kErrBlockId);
    return;
  }
  if (a.turned) {
    const int half = a.r.dims / 2, n = (t.end - t.first) * half;
    for (int x = threadIdx.x; x < n; x += 256) {
      const int p = x / half, k = x - p * half;
      cs[t.first + p][k] = rotary_turn(a.r, t.pos + t.first + p, k);
    }
    __syncthreads();
  }
  const RowLane<HD> l;
  const int wave = threadIdx.x >> 6;
  const int h1 = min(static_cast<int>(blockIdx.y + 1) * a.per, a.Hkv);
  for (int h0 = blockIdx.y * a.per; h0 < h1; h0 += kHeads) {
    const int head = h0 + wave * (128 / HD) + l.head;
    const bool mine = head < h1;  // the lanes of a head agree
    uint8_t* tile = a.pool + (static_cast<size_t>(t.id) * a.Hkv + min(head, h1 - 1)) * F::kTile;
    const int p = l.m / 4, q = l.m % 4;
    const auto live = [&](int r) { return mine && 4 * l.g + r >= t.first && 4 * l.g + r < t.end; };
    const auto row_of = [&](int r) { return static_cast<int64_t>(t.base + min(max(4 * l.g + r, t.first), t.end - 1)); };
    const int at = min(head, h1 - 1) * HD;
    float x[4][8], y[4][8] = {}, v[4][8];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const E* k = static_cast<const E*>(a.k) + row_of(r) * a.ks + at;
      load8<N>(k + 8 * l.m, x[r]);
      if (a.turned && !a.r.pairs) {
#pragma unroll
        for (int j = 0; j < 8; j += N) load_partners<N>(k, 8 * l.m + j, a.r.dims, y[r] + j);
      }
      load8<N>(static_cast<const E*>(a.v) + row_of(r) * a.vs + at + 8 * l.m, v[r]);
    }
    uint32_t words[4] = {0, 0, 0, 0}, scales = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int pos = 4 * l.g + r;
      if (a.turned) {
        float z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          z[j] = odd_f32(turn_element<8>(x[r], y[r], j, 8 * l.m, a.r.dims, a.r.pairs, cs[min(max(pos, t.first), t.end - 1)]));
#pragma unroll
        for (int j = 0; j < 8; ++j) x[r][j] = z[j];
      }
      uint32_t byte;
      const uint32_t kw = quantise(x[r], byte);
      if (live(r)) {
        *reinterpret_cast<uint32_t*>(tile + F::key_code(pos, 8 * l.m)) = kw;
        if (q == 0) tile[F::key_scale(pos, p)] = static_cast<uint8_t>(byte);
      }
      const uint32_t vw = quantise(v[r], byte);
      const uint32_t ow = __shfl_xor(static_cast<int>(vw), 2);
      // Dimensions 32 p + e and 32 p + 16 + e, four e of this lane's eight.
      const uint32_t lo = q < 2 ? vw : ow >> 16, hi = q < 2 ? ow : vw >> 16;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        words[e] |= ((lo >> 4 * e & 15u) | (hi >> 4 * e & 15u) << 4) << 8 * r;
      scales |= byte << 8 * r;
    }
    const int e0 = q < 2 ? 8 * q : 8 * (q - 2) + 4;
    if (live(0) && live(3)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(tile + F::value_word(l.g, e0 + e, p)) = words[e];
      if (q == 0) *reinterpret_cast<uint32_t*>(tile + F::value_scales(l.g, p)) = scales;
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (!live(r)) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) tile[F::value_word(l.g, e0 + e, p) + r] = static_cast<uint8_t>(words[e] >> 8 * r);
        if (q == 0) tile[F::value_scales(l.g, p) + r] = static_cast<uint8_t>(scales >> 8 * r);
      }
    }
  }
}

// Read: the same lanes the other way.
template <int N, int HD>
__global__ __launch_bounds__(256) void k_cache_read(CacheRowsArgs a) {
  using F = Mx4<HD>;
  using E = typename RowPiece<N>::elem;
  constexpr int kHeads = 4 * (128 / HD);
  CacheTile t = cache_tile(a, blockIdx.x);
  if (static_cast<unsigned>(t.id) >= static_cast<unsigned>(a.nb)) {
    if (threadIdx.x == 0) raise_check(a.err, kErrBlockId);
    t.id = 0;
  }
  const RowLane<HD> l;
  const int wave = threadIdx.x >> 6;
  const int h1 = min(static_cast<int>(blockIdx.y + 1) * a.per, a.Hkv);
  for (int h0 = blockIdx.y * a.per; h0 < h1; h0 += kHeads) {
    const int head = h0 + wave * (128 / HD) + l.head;
    if (head >= h1) continue;
    const uint8_t* tile = a.pool + (static_cast<size_t>(t.id) * a.Hkv + head) * F::kTile;
    const int p = l.m / 4, q = l.m % 4;
    uint32_t kw[4], kb[4], vw[8];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      kw[r] = *reinterpret_cast<const uint32_t*>(tile + F::key_code(4 * l.g + r, 8 * l.m));
      kb[r] = tile[F::key_scale(4 * l.g + r, p)];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) vw[e] = *reinterpret_cast<const uint32_t*>(tile + F::value_word(l.g, 8 * (q % 2) + e, p));
    const uint32_t vb = *reinterpret_cast<const uint32_t*>(tile + F::value_scales(l.g, p));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int pos = 4 * l.g + r;
      if (pos < t.first || pos >= t.end) continue;
      const int64_t row = t.base + pos;
      float x[8];
      const float ks = __uint_as_float(kb[r] << 23);
      const auto pair = [&](int j, f32x2_t v) { x[j] = v.x, x[j + 1] = v.y; };
      pair(0, codes_to_f32<0>(kw[r], ks));
      pair(2, codes_to_f32<1>(kw[r], ks));
      pair(4, codes_to_f32<2>(kw[r], ks));
      pair(6, codes_to_f32<3>(kw[r], ks));
      E* dk = static_cast<E*>(const_cast<void*>(a.k)) + row * a.ks + head * HD + 8 * l.m;
#pragma unroll
      for (int j = 0; j < 8; j += N) RowPiece<N>::store(dk + j, x + j);
      const float vs = __uint_as_float((vb >> 8 * r & 255u) << 23);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const f32x2_t v = codes_to_f32<0>(vw[e] >> 8 * r, vs);
        x[e] = q < 2 ? v.x : v.y;
      }
      E* dv = static_cast<E*>(const_cast<void*>(a.v)) + row * a.vs + head * HD + 8 * l.m;
#pragma unroll
      for (int j = 0; j < 8; j += N) RowPiece<N>::store(dv + j, x + j);
    }
  }
}

}  // namespace sprk
