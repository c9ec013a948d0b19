"""Verification without draft probabilities where rejections leave next to nothing (needs an MI355X).

A rejected child may have held all but 2^-24 of what was there (accept < 1), so after k of them 2^-24k is left: far below
what a sum of the whole row resolves, and still the distribution that the next test and the draw go by.
"""
import numpy as np
import pytest
import torch

from . import tree_ref as ref

pytestmark = pytest.mark.gpu

TOP = np.float32(1 - 2.0 ** -24)  # the largest uniform
STEP = 16.2                       # e^-16.2 = 2^-23.4: the next token's weight in units of the last one's
# TOP rejects a token of weight 1 beside 2^-23.4 (its share is 1 - 2^-23.4 < TOP) with a margin of 3e-8, and accepts a token
# that has all of what is left, so no rounding of 64-bit sums decides a test here.


def check(trees, tokens, logits, accept, sample):
    from paper_2403_12900_amd.tree import TreeBatch, TreeOps
    ops = TreeOps()
    b = TreeBatch(None, None, [len(t) for t in trees], [p for t in trees for p in t])
    cu = lambda x: torch.as_tensor(x).cuda()  # noqa: E731
    got = ops.verify(b, cu(tokens), cu(logits), cu(accept), cu(sample))
    got = [x.cpu().numpy() for x in got]
    ops.close()
    want = ref.verify(trees, tokens, logits.astype(np.float64), accept, sample)
    for g, w, name in zip(got, want, ("emitted", "path", "count")):
        assert np.array_equal(g, w), (name, g.tolist(), w.tolist())
    return got


@pytest.mark.parametrize("V,at", [(40, [3, 9, 17, 21, 30, 33, 38]), (10000, [5, 4200, 9000, 77, 8191, 4096, 300])])
@pytest.mark.parametrize("rejections", [1, 2, 3, 4, 5])
def test_siblings_that_take_all_but_a_rest_each(V, at, rejections):
    """The heaviest tokens rejected one after the other; then a child of probability 0, then the one token left."""
    z = np.full((1, V), -np.inf, np.float32)
    for k in range(rejections + 1):
        z[0, at[k]] = -STEP * k
    tokens = np.array([0] + at[:rejections] + [at[6], at[rejections]], np.int32)
    trees = [[-1] + [0] * (len(tokens) - 1)]
    accept = np.full(len(tokens), TOP, np.float32)
    logits = z.repeat(len(tokens), 0)
    got = check(trees, tokens, logits, accept, np.array([0.5], np.float32))
    assert got[0][0] == at[rejections] and got[1][1] == len(tokens) - 1
    # Without the last child the draw takes it.
    got = check([trees[0][:-1]], tokens[:-1], logits[:-1], accept[:-1], np.array([0.5], np.float32))
    assert got[2][0] == 1 and got[0][0] == at[rejections]


@pytest.mark.parametrize("V", [60, 5000, 20000])
@pytest.mark.parametrize("rejections", [1, 2, 3, 4])
def test_the_draw_from_a_small_rest(V, rejections):
    """Fifty tokens share what the rejections leave: every sample's token, and the same with a child listed twice."""
    rng = np.random.default_rng(V + rejections)
    ids = rng.permutation(V)[:rejections + 50]
    z = np.full((1, V), -np.inf, np.float32)
    z[0, ids[:rejections]] = -STEP * np.arange(rejections)
    # Together 2^-23.4 of the last rejected token's weight.
    z[0, ids[rejections:]] = -STEP * rejections - np.log(50) + rng.uniform(-0.1, 0.1, 50)
    child = [int(x) for x in ids[:rejections]]
    for tokens in ([0] + child, [0] + child + child):
        tokens = np.array(tokens, np.int32)
        n = len(tokens)
        samples = (np.arange(8, dtype=np.float32) + 0.37) / 8
        B = min(8, 128 // n)
        got = check([[-1] + [0] * (n - 1)] * B, np.tile(tokens, B), z.repeat(B * n, 0), np.full(B * n, TOP, np.float32), samples[:B])
        assert (got[2] == 1).all() and not set(got[0][::n].tolist()) & set(child)
