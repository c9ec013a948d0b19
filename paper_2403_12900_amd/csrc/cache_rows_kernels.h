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
// come before its stores: x may be turned in place.  Bound by memory: 4096 rows of
// 64 heads in fp32 (268 MB) 53 us, 5.1 TB/s, what a copy reaches; 32 rows of 32
// heads take 3.8 us, the arguments, the position and the row one after the other.
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
    // (To bf16 in one rounding: the compiler takes this conversion and the store's as
    // one, through a rounding to odd.)
#pragma unroll
    for (int j = 0; j < N; ++j) r[j] = static_cast<float>(turn_element<N>(v, y, j, d0, a.r.dims, a.r.pairs, cs));
    Piece::store(out + h * HD + d0, r);
  }
}

// ---------------------------------------------------------------------------

// Rows of keys and values.  A thread takes eight dimensions of a row and KV
// head.  A work-group's 256 threads are either the 16 positions of one block for
// a head (HD = 64: two) at a time, or, where every request has a single row, that
// row for 16 (32) heads.  tile0[i] counts the blocks, or rows, of the requests
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
  int slot[kCacheReqs], len[kCacheReqs], row0[kCacheReqs];
  int tile0[kCacheReqs + 1];
  int rows[kCacheReqs];
};
static_assert(sizeof(CacheRowsArgs) <= 3584, "kernel arguments");

// Positions of a block that a work-group takes (1: a single row's).
constexpr int kRowsOfBlock = 16;
template <int RG, int HD>
constexpr int kRowHeads = 256 / (RG * (HD / 8));  // heads at a time

struct CacheTile {
  int pos, first, end;  // positions pos + [first, end) of the block at pos
  int base;             // row of position pos (before the request's first row where first > 0)
  int id;
};
template <int RG>
__device__ __forceinline__ CacheTile cache_tile(const CacheRowsArgs& a, int f) {
  const int lane = threadIdx.x & 63;
  // Lane = request, 64 at a time and all of them at once: one trip to memory.
  for (int k = 0;; k += 64) {
    const int r = min(k + lane, a.n - 1);
    const int tile0 = a.tile0[r], tile1 = a.tile0[r + 1], lens = a.len[r], row0 = a.row0[r], rows = a.rows[r];
    const int slot = a.slot[r];
    // Request: the number of requests whose tiles all precede f.
    const int before = __popcll(__ballot(k + lane < a.n && tile1 <= f));
    if (before == 64 && k + 64 < a.n) continue;
    const auto mine = [&](int v) { return __builtin_amdgcn_readlane(v, before); };
    const int len = mine(lens), total = len + mine(rows), w = f - mine(tile0);
    CacheTile t;
    if constexpr (RG == 1) {
      t.pos = (len + w) & ~15;
      t.first = (len + w) & 15;
      t.end = t.first + 1;
    } else {
      t.pos = 16 * (len / 16 + w);
      t.first = max(len - t.pos, 0);
      t.end = min(total - t.pos, 16);
    }
    t.base = mine(row0) + t.pos - len;
    t.id = a.bt[static_cast<size_t>(mine(slot)) * a.mb + t.pos / 16];
    return t;
  }
}

// A thread's place: position t of the block, head `head` of those at a time,
// eight dimensions from 8 m on (group p of 32, quarter q of it).
template <int RG, int HD>
struct RowThread {
  int t, head, m, p, q;
  bool live;
  __device__ __forceinline__ RowThread(const CacheTile& tile) {
    const int tid = threadIdx.x;
    m = tid % (HD / 8);
    p = m / 4;
    q = m % 4;
    if constexpr (RG == 1) {
      t = tile.first;
      head = tid / (HD / 8);
      live = true;
    } else {
      t = tid / (HD / 8) % 16;
      head = tid / (2 * HD);
      live = t >= tile.first && t < tile.end;
    }
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

// Eight turned values of a lane in fp32.  What decides a code or a scale is on
// which side of a border a value lies, and borders have three significant bits:
// rounding to nearest can only mislead where it ends on such a number, and there
// the values are rounded to odd instead.
// turned: how many of the eight are (the rest are exact).
template <class Turn>
__device__ __forceinline__ void turn_lane(float* x, int turned, const Turn& turn) {
  double z[8];
  bool near = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    z[j] = turn(j);
    x[j] = static_cast<float>(z[j]);
    const uint32_t u = __float_as_uint(x[j]);
    near |= (j < turned) & (((u & 0xFFFFFu) == 0) | ((u & 0x7F800000u) == 0x7F800000u));
  }
  if (__ballot(near) != 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = odd_f32(z[j]);
  }
}

// Append.  Keys: a thread's eight codes are a word of the tile.  Values: it
// trades half its codes with the thread 16 dimensions on, and stores four bytes.
// (A lane's position is the same for all heads, and so are its sines.)  8 prompts
// of about 700 rows, 8 KV heads, fp32 (46 MB read, 6 written): 15 us, 3.5 TB/s,
// the sines in 64 bits and single bytes of values in turn with the loads; a
// work-group for every two heads took 18.  A single row of 32 requests 5.6 us.
template <int N, int HD, int RG>
__global__ __launch_bounds__(256) void k_cache_append(CacheRowsArgs a) {
  using F = Mx4<HD>;
  using E = typename RowPiece<N>::elem;
  constexpr int kHeads = kRowHeads<RG, HD>;
  __shared__ double2 cs[RG][HD / 2];
  const CacheTile t = cache_tile<RG>(a, blockIdx.x);
  const RowThread<RG, HD> l(t);
  const int h1 = min(static_cast<int>(blockIdx.y + 1) * a.per, a.Hkv);
  const int64_t row = t.base + (l.live ? l.t : t.first);
  const E* k = static_cast<const E*>(a.k) + row * a.ks;
  const E* v = static_cast<const E*>(a.v) + row * a.vs;
  float x[8], y[8] = {}, w[8];
  const auto load = [&](int h0) {
    const int at = min(h0 + l.head, h1 - 1) * HD;
    load8<N>(k + at + 8 * l.m, x);
    if (a.turned && !a.r.pairs) {
#pragma unroll
      for (int j = 0; j < 8; j += N) load_partners<N>(k + at, 8 * l.m + j, a.r.dims, y + j);
    }
    load8<N>(v + at + 8 * l.m, w);
  };
  int h0 = blockIdx.y * a.per;
  load(h0);
  if (a.turned) {
    const int half = a.r.dims / 2, n = (t.end - t.first) * half;
    for (int i = threadIdx.x; i < n; i += 256) {
      const int at = i / half, d = i - at * half;
      cs[RG == 1 ? 0 : t.first + at][d] = rotary_turn(a.r, t.pos + t.first + at, d);
    }
    __syncthreads();
  }
  if (static_cast<unsigned>(t.id) >= static_cast<unsigned>(a.nb)) {
    if (threadIdx.x == 0) raise_check(a.err, kErrBlockId);
    return;
  }
  const double2* table = cs[RG == 1 ? 0 : l.live ? l.t : t.first];
  for (;;) {
    const int head = h0 + l.head;
    uint8_t* tile = a.pool + (static_cast<size_t>(t.id) * a.Hkv + min(head, h1 - 1)) * F::kTile;
    if (a.turned) {
      float z[8];
      turn_lane(z, a.r.dims - 8 * l.m, [&](int j) { return turn_element<8>(x, y, j, 8 * l.m, a.r.dims, a.r.pairs, table); });
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = z[j];
    }
    uint32_t kb, vb;
    const uint32_t kw = quantise(x, kb), vw = quantise(w, vb);
    const uint32_t ow = __shfl_xor(static_cast<int>(vw), 2);
    // Dimensions 32 p + e and 32 p + 16 + e, four e of this thread's eight.
    const uint32_t lo = l.q < 2 ? vw : ow >> 16, hi = l.q < 2 ? ow : vw >> 16;
    const int e0 = l.q < 2 ? 8 * l.q : 8 * (l.q - 2) + 4;
    if (l.live && head < h1) {
      *reinterpret_cast<uint32_t*>(tile + F::key_code(l.t, 8 * l.m)) = kw;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        tile[F::value_word(l.t / 4, e0 + e, l.p) + l.t % 4] = static_cast<uint8_t>((lo >> 4 * e & 15u) | (hi >> 4 * e & 15u) << 4);
      if (l.q == 0) {
        tile[F::key_scale(l.t, l.p)] = static_cast<uint8_t>(kb);
        tile[F::value_scales(l.t / 4, l.p) + l.t % 4] = static_cast<uint8_t>(vb);
      }
    }
    h0 += kHeads;
    if (h0 >= h1) break;
    load(h0);
  }
}

// Read: the same threads the other way; the prompts above 14 us.
template <int N, int HD, int RG>
__global__ __launch_bounds__(256) void k_cache_read(CacheRowsArgs a) {
  using F = Mx4<HD>;
  using E = typename RowPiece<N>::elem;
  CacheTile t = cache_tile<RG>(a, blockIdx.x);
  if (static_cast<unsigned>(t.id) >= static_cast<unsigned>(a.nb)) {
    if (threadIdx.x == 0) raise_check(a.err, kErrBlockId);
    t.id = 0;
  }
  const RowThread<RG, HD> l(t);
  if (!l.live) return;
  const int h1 = min(static_cast<int>(blockIdx.y + 1) * a.per, a.Hkv);
  const int64_t row = t.base + l.t;
  E* k = static_cast<E*>(const_cast<void*>(a.k)) + row * a.ks + 8 * l.m;
  E* v = static_cast<E*>(const_cast<void*>(a.v)) + row * a.vs + 8 * l.m;
  for (int head = blockIdx.y * a.per + l.head; head < h1; head += kRowHeads<RG, HD>) {
    const uint8_t* tile = a.pool + (static_cast<size_t>(t.id) * a.Hkv + head) * F::kTile;
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(tile + F::key_code(l.t, 8 * l.m));
    const float ks = __uint_as_float(static_cast<uint32_t>(tile[F::key_scale(l.t, l.p)]) << 23);
    const float vs = __uint_as_float(static_cast<uint32_t>(tile[F::value_scales(l.t / 4, l.p) + l.t % 4]) << 23);
    // Four value bytes, and the four of the thread 16 dimensions on.
    const int e0 = l.q < 2 ? 8 * l.q : 8 * (l.q - 2) + 4;
    uint32_t own = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) own |= static_cast<uint32_t>(tile[F::value_word(l.t / 4, e0 + e, l.p) + l.t % 4]) << 8 * e;
    const uint32_t other = __shfl_xor(static_cast<int>(own), 2);
    const uint32_t v0 = l.q < 2 ? own : other, v1 = l.q < 2 ? other : own;
    float x[8];
    const auto pair = [&](int j, f32x2_t z) { x[j] = z.x, x[j + 1] = z.y; };
    pair(0, codes_to_f32<0>(kw, ks));
    pair(2, codes_to_f32<1>(kw, ks));
    pair(4, codes_to_f32<2>(kw, ks));
    pair(6, codes_to_f32<3>(kw, ks));
#pragma unroll
    for (int j = 0; j < 8; j += N) RowPiece<N>::store(k + head * HD + j, x + j);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const f32x2_t z = codes_to_f32<0>((e < 4 ? v0 : v1) >> 8 * (e % 4), vs);
      x[e] = l.q < 2 ? z.x : z.y;
    }
#pragma unroll
    for (int j = 0; j < 8; j += N) RowPiece<N>::store(v + head * HD + j, x + j);
  }
}

}  // namespace sprk
