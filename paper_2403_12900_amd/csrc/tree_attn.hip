// Instantiations of the drafted-tree attention kernel and its launch.
#include <cmath>

#include "tree_attn_kernels.h"
#include "tree_launch.h"

namespace sprk {
namespace {

// CW columns per work-group: up to 32 on k_tree_attn, 64 and more on
// k_tree_attn_shared.
template <class KP, class IO, int HD, int CW>
constexpr auto kernel() {
  if constexpr (CW <= 32) return &k_tree_attn<KP, IO, HD, CW / 16>;
  else return &k_tree_attn_shared<KP, IO, HD, CW / 64>;
}

// Floats of partial outputs that the last split's work-group merges by itself:
// more cost more there than a second launch does (192 columns times splits of
// 128 dimensions: 12.5 us against 13.0 with the launch, 1 request of 352: 14.2
// against 13.3, of 1024: 20.2 against 16.3).
constexpr int kMergeInside = 192 * 128;

// Work-groups of the kernel that a CU holds, or is to hold, at once.
template <class KP, class IO, int HD, int CW>
int groups_per_cu() {
  static const int n = [] {
    int o = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&o, reinterpret_cast<const void*>(kernel<KP, IO, HD, CW>()), 256,
                                                     0) != hipSuccess || o < 1)
      o = 1;
    return CW > 32 ? std::min(o, kSharedPerCu<KP>) : o;
  }();
  return n;
}

template <class KP, class IO, int HD, int CW>
hipError_t launch(const TreeAttnCall& c) {
  const TreeInfo& t = *c.tree;
  TreeAttnArgs a{};
  if (static_cast<int64_t>(t.rows) * c.kv.n_kv_heads > c.sc.n_cnt) return hipErrorInvalidValue;  // a column group has a row at least
  const size_t layer = static_cast<size_t>(c.kv.n_blocks) * c.kv.n_kv_heads * 16 * HD * c.layer;
  a.q = c.q;
  a.out = c.out;
  a.qs = c.qs;
  a.os = c.os;
  a.kc = static_cast<const typename KP::elem*>(c.kv.k) + layer;
  a.vc = static_cast<const typename KP::elem*>(c.kv.v) + layer;
  a.bt = c.kv.block_table;
  a.part = c.sc.part;
  a.cnt = c.sc.cnt;
  a.err = c.err;
  a.n = t.n;
  a.H = c.H;
  a.Hkv = c.kv.n_kv_heads;
  a.G = a.H / a.Hkv;
  a.mb = c.kv.max_blocks;
  a.nb = c.kv.n_blocks;
  a.qscale = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(HD)));
  a.rec = c.rec;
  const size_t floats = std::min(c.sc.part_floats, size_t{1} << 28);
  a.part_bytes = static_cast<uint32_t>(floats * 4);
  constexpr int step = KP::per16 == 8 ? 2 : 1;
  const int slots = groups_per_cu<KP, IO, HD, CW>() * c.n_cu;
  const TreeSplit sp = tree_split(t, a.G, a.Hkv, HD, CW, CW <= 32 ? 4 * step : step, slots, floats);
  a.bps = sp.bps;
  for (int r = 0; r < t.n; ++r) {
    const int i = sp.order[r];
    a.slot[r] = t.slot[i];
    a.len[r] = t.len[i];
    a.nodes[r] = static_cast<uint8_t>(t.nodes[i]);
    a.row0[r] = static_cast<uint8_t>(t.row0[i]);
    a.ncg[r] = sp.ncg[r];
    a.cg0[r] = sp.cg0[r];
    a.item0[r] = sp.item0[r];
  }
  a.item0[t.n] = sp.item0[t.n];
  for (int r = 0; r < t.rows; ++r) a.anc[r] = t.anc[r];
  // Where the last work-group of a column group would have much to read, the
  // merge is a launch of its own over all outputs; else it stays in the kernel.
  const int groups = sp.cg0[t.n - 1] + sp.ncg[t.n - 1];
  int most = 0;  // columns times splits of one merge
  for (int r = 0; r < t.n; ++r)
    most = std::max(most, std::min(CW, t.nodes[sp.order[r]] * a.G) * ((sp.item0[r + 1] - sp.item0[r]) / sp.ncg[r]));
  a.apart = sp.item0[t.n] > groups && (CW > 32 || most * HD > kMergeInside);
  kernel<KP, IO, HD, CW>()<<<dim3(a.Hkv, sp.item0[t.n]), 256, 0, c.st>>>(a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.apart) {
    k_tree_merge<IO, HD, CW><<<dim3(a.Hkv, groups, CW / kMergeColumns), 256, 0, c.st>>>(a);
    e = hipGetLastError();
  }
  return e;
}

// Columns per work-group: two-byte operands 128 (8 x 128 columns of 128
// dimensions, 6000 positions: 66 us, of 64 columns 70; 2 x 512 columns, 24000
// positions: 180 and 197; but at 700 positions 24 and 21), the others 64 (fp32,
// 8 x 128 columns, 6000 positions: 222 us against 366 with 128, at 700 positions
// 41 against 67; three-part queries leave no registers for more).
template <class KP, class IO, int HD>
hipError_t by_columns(const TreeAttnCall& c) {
  constexpr int most = KP::per16 == 8 && TreeParts<KP, IO>::q == 1 ? 128 : 64;
  switch (tree_cols_per_group(*c.tree, c.H / c.kv.n_kv_heads, most)) {
    case 16: return launch<KP, IO, HD, 16>(c);
    case 32: return launch<KP, IO, HD, 32>(c);
    case 64: return launch<KP, IO, HD, 64>(c);
    case 128:
      if constexpr (most == 128) return launch<KP, IO, HD, 128>(c);
      break;
  }
  return hipErrorInvalidValue;  // not reached: no more than `most`
}

template <class KP, class IO>
hipError_t by_shape(const TreeAttnCall& c) {
  return c.kv.head_dim == 128 ? by_columns<KP, IO, 128>(c) : by_columns<KP, IO, 64>(c);
}

}  // namespace

hipError_t launch_tree_attention(const TreeAttnCall& c) {
  const bool bf = c.kv.kv_dtype == SPR_BF16;
  switch (c.io) {
    case kTreeF32: return bf ? by_shape<BF16, TreeIoF32>(c) : by_shape<F32, TreeIoF32>(c);
    case kTreeBF16: return bf ? by_shape<BF16, TreeIoBF16>(c) : by_shape<F32, TreeIoBF16>(c);
    case kTreeActBF16: return bf ? by_shape<BF16, TreeIoAct<BF16>>(c) : by_shape<F32, TreeIoAct<BF16>>(c);
    default: return by_shape<F32, TreeIoAct<F32>>(c);
  }
}

}  // namespace sprk
