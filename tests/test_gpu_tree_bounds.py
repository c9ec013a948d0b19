"""Attention of drafted trees against a bound of its own for every output (needs an MI355X; the bound's own test does not).

The bound, for inputs of unit variance (eps = 2^-24, an fp32 rounding), from the 64-bit reference's p, v and out:
  * what fp32 scores, exponentials, sums and merges may add, as derived in test_gpu_tree_ops.py, with sum p |v| of the
    output in the place of max |v| (a change of the weights by a factor 1 + d moves a mean by at most d sum p |v|, and its
    normalisation by as much again):  F = 2 (2 * 4 eps |q| |k| + (26 + 8 sqrt(T)) eps) sum p |v|;
  * probabilities in two bf16 parts: each part's rounding is at most 2^-8 of what it rounds, so 2^-16 of the probability
    is left: 2^-16 sum p |v|;
  * a bf16 output is rounded once more, by at most 2^-8 of its value.
"""
import numpy as np
import pytest
import torch

from . import tree_ref as ref
from ._harness import say

EPS = 2.0 ** -24


def reference(cache, layer, slots, lens, trees, q, drop=None):
    """(out, sum p |v|, bound of fp32 errors), [rows, H, hd] in 64 bits.  drop: positions (of request 0) whose part of the
    sums is left out of out's numerator and denominator, as a lost split would."""
    q = q.double().numpy()
    H, hd = q.shape[1:]
    G = H // cache.k.shape[2]
    out, mass, err = np.empty(q.shape), np.empty(q.shape), np.empty(q.shape)
    r = 0
    for i, (s, n, par) in enumerate(zip(slots, lens, trees)):
        k, v = (cache.rows(x, layer, s, range(n + len(par))) for x in (cache.k, cache.v))
        for j in range(len(par)):
            pos = list(range(n)) + sorted(n + a for a in ref.ancestors(par, j))
            kk, vv = np.repeat(k[pos], G, 1), np.repeat(v[pos], G, 1)
            z = np.einsum("hd,thd->ht", q[r], kk) / np.sqrt(hd)
            p = np.exp(z - z.max(1, keepdims=True))
            if drop is not None and i == 0:
                p[:, [t for t, x in enumerate(pos) if x in drop]] = 0
            p /= p.sum(1, keepdims=True)
            out[r], mass[r] = np.einsum("ht,thd->hd", p, vv), np.einsum("ht,thd->hd", p, np.abs(vv))
            norms = np.linalg.norm(q[r], axis=1) * np.linalg.norm(kk, axis=2).max(0)
            err[r] = 2 * (8 * EPS * norms + (26 + 8 * np.sqrt(len(pos))) * EPS)[:, None] * mass[r]
            r += 1
    return out, mass, err


def bound(want, mass, err, io, kv):
    b = err + (2.0 ** -16 * mass if kv == torch.bfloat16 else 0.0)
    return b if io == torch.float32 else b * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)


def batch_of(slots, lens, trees):
    from paper_2403_12900_amd.tree import TreeBatch
    return TreeBatch(slots, lens, [len(t) for t in trees], [p for t in trees for p in t])


def make(rng, H, Hkv, hd, kv, io, lens, trees):
    cache = ref.Cache(rng, 1, Hkv, hd, [a + len(t) for a, t in zip(lens, trees)], kv, spare=1)
    q = torch.from_numpy(rng.standard_normal((sum(len(t) for t in trees), H, hd), dtype=np.float32)).to(io)
    return cache, q


# (heads, KV heads, head dimension, nodes, context): 16, 32, 64 and 128 columns per work-group; one split, several that the
# last one merges, several that a launch of their own merges.
CASES = [(4, 4, 64, 3, 40), (8, 2, 128, 8, 90), (8, 1, 64, 8, 50), (16, 1, 128, 9, 70), (8, 1, 128, 4, 700), (8, 1, 128, 4, 3000),
         (8, 1, 64, 4, 6000), (3, 3, 64, 16, 4100), (4, 2, 128, 3, 7001), (16, 2, 128, 6, 2500), (16, 2, 64, 33, 1700)]


@pytest.mark.gpu
@pytest.mark.parametrize("kv", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hkv,hd,nodes,L", CASES)
def test_every_output_within_its_bound(H, Hkv, hd, nodes, L, kv, io):
    """Split and merged requests beside one of a single split and an almost empty one."""
    from paper_2403_12900_amd.tree import TreeOps
    rng = np.random.default_rng(L + nodes)
    lens = [L, 9, 0]
    trees = [ref.random_tree(rng, nodes, "random"), [-1], ref.random_tree(rng, 2, "chain")]
    cache, q = make(rng, H, Hkv, hd, kv, io, lens, trees)
    say(f"tree attention bounds: H {H}/{Hkv} hd {hd} cache {kv} io {io} nodes {nodes} context {L}")
    ops = TreeOps()
    got = ops.attention(cache.device(), 0, batch_of([0, 1, 2], lens, trees), q.cuda()).double().cpu().numpy()
    ops.close()
    want, mass, err = reference(cache, 0, [0, 1, 2], lens, trees, q)
    share = np.abs(got - want) / bound(want, mass, err, io, kv)
    worst, over = float(share.max()), int((share > 1).sum())
    assert worst <= 1, f"{over} of {share.size} outputs, worst {worst:.1f} times the bound"


@pytest.mark.parametrize("kv", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hkv,hd,nodes,L", [c for c in CASES if c[4] >= 700])
def test_the_bound_rejects_a_lost_split(H, Hkv, hd, nodes, L, kv):
    """bf16 outputs: the reference without four blocks of the cache (the shortest split there is) is outside."""
    rng = np.random.default_rng(L)
    lens, trees = [L], [ref.random_tree(rng, min(nodes, 4), "random")]
    cache, q = make(rng, H, Hkv, hd, kv, torch.bfloat16, lens, trees)
    want, mass, err = reference(cache, 0, [0], lens, trees, q)
    b = bound(want, mass, err, torch.bfloat16, kv)
    for first in (0, L // 64 // 2 * 64):
        lost = reference(cache, 0, [0], lens, trees, q, drop=set(range(first, first + 64)))[0]
        assert (np.abs(lost - want) > b).mean() > 0.25
