"""Infinite and NaN values of drafted nodes: rows that see them get them element by element, the others nothing
(needs an MI355X).  Bounds of the finite outputs: test_gpu_tree_bounds.py."""
import numpy as np
import pytest
import torch

from . import tree_ref as ref
from .test_gpu_tree_bounds import batch_of, bound, reference

pytestmark = pytest.mark.gpu

PARENTS = [-1, 0, 0, 1, 2, 4, 3, 0]
POISONED, SEEING = 2, [2, 4, 5]


@pytest.mark.parametrize("kv", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hkv,hd", [(2, 2, 64), (4, 1, 128), (8, 1, 64), (8, 1, 128), (16, 1, 64), (16, 1, 128)])
def test_poisoned_values_reach_the_rows_that_see_them(H, Hkv, hd, io, kv):
    """8 to 128 columns (every work-group width), in one split and in the last of several; values alone, so that every
    probability is finite and only the values' own path can bring them in."""
    from paper_2403_12900_amd.tree import TreeOps
    ops = TreeOps()
    rng = np.random.default_rng(H + hd)
    dims = np.arange(hd)
    for L in (0, 13, 32, 200, 1500):
        cache = ref.Cache(rng, 1, Hkv, hd, [L + len(PARENTS)], kv, fill=float("nan"))
        at = L + POISONED
        row = cache.v[0, cache.table[0, at // 16], :, at % 16]
        row[:, dims % 5 == 1] = float("inf")
        row[:, dims % 7 == 2] = float("nan")
        row[:, dims % 11 == 3] = float("-inf")
        cache.v[0, cache.table[0, at // 16], :, at % 16] = row
        q = torch.from_numpy(rng.standard_normal((len(PARENTS), H, hd), dtype=np.float32)).to(io)
        got = ops.attention(cache.device(), 0, batch_of([0], [L], [PARENTS]), q.cuda()).double().cpu().numpy()
        with np.errstate(all="ignore"):
            want, mass, err = reference(cache, 0, [0], [L], [PARENTS], q)
            over = np.abs(got - want) > bound(want, mass, err, io, kv)
        odd = ~np.isfinite(want)
        assert odd[SEEING].any(-1).all() and not odd[[r for r in range(len(PARENTS)) if r not in SEEING]].any()
        for what, f in (("NaN", np.isnan), ("+inf", np.isposinf), ("-inf", np.isneginf)):
            assert np.array_equal(f(got), f(want)), (L, what, int((f(got) != f(want)).sum()))
        assert not over[~odd].any(), (L, int(over[~odd].sum()))
    ops.close()
