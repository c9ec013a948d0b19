// Instantiations of the 4-bit cache's attention kernels and their launch.
#include <cmath>

#include "cache_attn_kernels.h"
#include "cache_launch.h"

namespace sprk {
namespace {

// CW columns per work-group: up to 32 on k_cache_attn, 64 and more on
// k_cache_attn_wide.
template <class IO, int HD, int CW>
constexpr auto kernel() {
  if constexpr (CW <= 32) return &k_cache_attn<IO, HD, CW / 16>;
  else return &k_cache_attn_wide<IO, HD, CW / 64>;
}

// Work-groups of the kernel that a CU holds at once.
template <class IO, int HD, int CW>
int groups_per_cu() {
  static const int n = [] {
    int o = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&o, reinterpret_cast<const void*>(kernel<IO, HD, CW>()), 256, 0) !=
            hipSuccess || o < 1)
      o = 1;
    return o;
  }();
  return n;
}

template <class IO, int HD, int CW>
hipError_t launch(const CacheAttnCall& c) {
  const CacheInfo& t = *c.batch;
  CacheAttnArgs a{};
  a.q = c.q;
  a.out = c.out;
  a.qs = c.qs;
  a.os = c.os;
  a.pool = static_cast<const uint8_t*>(c.kv.data) + static_cast<size_t>(c.layer) * c.kv.n_blocks * c.kv.n_kv_heads * Mx4<HD>::kTile;
  a.bt = c.kv.block_table;
  a.part = c.part;
  a.cnt = c.cnt;
  a.err = c.err;
  a.n = t.n;
  a.H = c.H;
  a.Hkv = c.kv.n_kv_heads;
  a.G = a.H / a.Hkv;
  a.mb = c.kv.max_blocks;
  a.nb = c.kv.n_blocks;
  a.qscale = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(HD)));
  const size_t floats = std::min(c.part_floats, size_t{1} << 28);
  a.part_bytes = static_cast<uint32_t>(floats * 4);
  const CacheSplit sp = cache_split(t, a.G, a.Hkv, HD, CW, CW <= 32 ? 8 : 2, groups_per_cu<IO, HD, CW>() * c.n_cu, floats, c.n_cnt);
  a.bps = sp.bps;
  for (int r = 0; r < t.n; ++r) {
    const int i = sp.order[r];
    a.slot[r] = t.slot[i];
    a.len[r] = t.len[i];
    a.rows[r] = t.n_rows[i];
    a.row0[r] = t.row0[i];
    a.cg0[r] = sp.cg0[r];
    a.item0[r] = sp.item0[r];
  }
  a.item0[t.n] = sp.item0[t.n];
  kernel<IO, HD, CW>()<<<static_cast<unsigned>(sp.item0[t.n]) * a.Hkv, 256, 0, c.st>>>(a);
  hipError_t e = hipGetLastError();
  if constexpr (CW > 32)
    if (e == hipSuccess && sp.split) {
      k_cache_merge<IO, HD, CW><<<static_cast<unsigned>(sp.groups) * a.Hkv * (CW / kMergeWide), 256, 0, c.st>>>(a);
      e = hipGetLastError();
    }
  return e;
}

template <class IO, int HD>
hipError_t by_columns(const CacheAttnCall& c) {
  constexpr int most = IO::kRaw ? 128 : 64;  // three-part queries leave too few registers for more
  switch (cache_cols_per_group(*c.batch, c.H / c.kv.n_kv_heads, c.kv.n_kv_heads, c.n_cu, most)) {
    case 16: return launch<IO, HD, 16>(c);
    case 32: return launch<IO, HD, 32>(c);
    case 64: return launch<IO, HD, 64>(c);
    case 128:
      if constexpr (most == 128) return launch<IO, HD, 128>(c);
      break;
  }
  return hipErrorInvalidValue;  // not reached: no more than `most`
}

template <class IO>
hipError_t by_shape(const CacheAttnCall& c) {
  return c.kv.head_dim == 128 ? by_columns<IO, 128>(c) : by_columns<IO, 64>(c);
}

}  // namespace

hipError_t launch_cache_attention(const CacheAttnCall& c) {
  return c.bf16 ? by_shape<TreeIoBF16>(c) : by_shape<TreeIoF32>(c);
}

}  // namespace sprk
