"""The drafted-tree operators against plain 64-bit implementations (needs an MI355X).

Tolerances of attention, derived for inputs of unit variance (eps = 2^-24, an fp32 rounding):
  * a score is a sum of hd products of fp32-exact operands whose partial sums stay below |q| |k|; its hd roundings of
    random sign add up to less than 4 sqrt(hd) eps |q| |k|, which the scale 1 / sqrt(hd) takes to ds = 4 eps |q| |k|;
  * a change of at most ds in every score changes the weighted mean of v by at most 2 ds max|v|;
  * exp2 (1 ulp, and its argument's rounding: |s log2 e| <= 2^5 here, 2^5 eps ln 2 < 24 eps), the sums over T positions
    (4 sqrt(T) eps, on numerator and denominator) and the merges add (26 + 8 sqrt(T)) eps max|v|;
  * bf16 outputs: probabilities rounded to bf16 (half a step, 2^-8 relative) move the mean by at most 2^-8 max|v|, and
    the output's own rounding adds 2^-8 of it.
Whole numbers (verification) and copies (compaction) are exact.
"""
import numpy as np
import pytest
import torch

from . import tree_ref as ref
from ._harness import say

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def ops():
    from paper_2403_12900_amd.tree import TreeOps
    o = TreeOps()
    yield o
    o.close()


def fresh_ops():
    from paper_2403_12900_amd.tree import TreeOps
    return TreeOps()


def batch_of(slots, lens, trees):
    from paper_2403_12900_amd.tree import TreeBatch
    return TreeBatch(slots, lens, [len(t) for t in trees], [p for t in trees for p in t])


def attention_tolerance(cache, q, T, io):
    kn = float(cache.k.double().nan_to_num(0, 0, 0).norm(dim=-1).max())
    qn = float(q.double().norm(dim=-1).max())
    vm = float(cache.v.double().nan_to_num(0, 0, 0).abs().max())
    tol = (2 * 4 * EPS * qn * kn + (26 + 8 * np.sqrt(T)) * EPS) * vm
    return tol if io == torch.float32 else tol + 2.0 ** -8 * 2 * vm


def check_attention(ops, rng, H, Hkv, hd, kv, io, lens, trees, fill=float("nan"), layers=1, layer=0, tag="", spare=1):
    n = len(lens)
    slots = [int(s) for s in rng.permutation(n)]
    positions = [0] * n
    for i, s in enumerate(slots):
        positions[s] = lens[i] + len(trees[i])
    cache = ref.Cache(rng, layers, Hkv, hd, positions, kv, fill=fill, spare=spare)
    R = sum(len(t) for t in trees)
    q = torch.from_numpy(rng.standard_normal((R, H, hd), dtype=np.float32)).to(io)
    say(f"tree attention {tag}: H {H}/{Hkv} hd {hd} cache {kv} io {io} lens {lens} nodes {[len(t) for t in trees]}")
    out = ops.attention(cache.device(), layer, batch_of(slots, lens, trees), q.cuda())
    torch.cuda.synchronize()
    want = ref.attention(cache, layer, slots, lens, trees, q)
    got = out.double().cpu().numpy()
    tol = attention_tolerance(cache, q, max(lens) + 64, io)
    assert np.isfinite(got).all()
    d = np.abs(got - want).max()
    assert d <= tol, f"max error {d:.3e} > {tol:.3e}"
    return d, tol


SHAPES = [(4, 4, 64), (8, 2, 128), (65, 5, 64), (3, 3, 128), (16, 1, 128), (15, 5, 64)]


@pytest.mark.parametrize("kv", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hkv,hd", SHAPES)
def test_attention_shapes_and_types(ops, H, Hkv, hd, kv, io):
    rng = np.random.default_rng(H * 100 + hd)
    lens = [0, 1, 15, 16, 17, 130, 47]
    trees = [ref.random_tree(rng, n, kind) for n, kind in
             [(1, "chain"), (2, "chain"), (5, "random"), (16, "star"), (17, "levels"), (33, "random"), (7, "chain")]]
    check_attention(ops, rng, H, Hkv, hd, kv, io, lens, trees)


@pytest.mark.parametrize("kv", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lens,nodes", [([0], [1]), ([1], [1]), ([31], [1]), ([32], [64]), ([0], [64]), ([63, 64, 65], [16, 17, 33]),
                                        ([200] * 64, [2] * 64), ([5000], [3]), ([20000, 3], [9, 1])])
def test_attention_lengths_and_splits(ops, kv, lens, nodes):
    """One position to many KV splits; single tokens; the largest batches; a two-layer cache's second layer."""
    rng = np.random.default_rng(7)
    trees = [ref.random_tree(rng, n, "random") for n in nodes]
    check_attention(ops, rng, 4, 2, 64, kv, torch.float32, lens, trees, layers=2, layer=1)


@pytest.mark.parametrize("kv", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hkv,hd,nodes", [(16, 2, 128, 64), (16, 2, 64, 64), (32, 2, 128, 5), (4, 4, 128, 33), (8, 8, 64, 20)])
def test_attention_of_wide_trees_over_long_contexts(ops, H, Hkv, hd, nodes, kv, io):
    """Several column groups and KV splits at once, whole steps of either parity, beside a short request."""
    rng = np.random.default_rng(hd + nodes)
    for lens in ([1700, 5], [1683, 40]):
        trees = [ref.random_tree(rng, nodes, "random"), ref.random_tree(rng, 3, "chain")]
        check_attention(ops, rng, H, Hkv, hd, kv, io, lens, trees, tag="wide")


@pytest.mark.parametrize("kv", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hkv,hd,nodes,L", [(8, 1, 128, 4, 700), (8, 1, 128, 4, 3000), (8, 1, 64, 4, 6000), (3, 3, 64, 16, 4100),
                                              (4, 2, 128, 3, 7001)])
def test_attention_merged_in_the_kernel_and_apart(ops, H, Hkv, hd, nodes, L, kv, io):
    """Few columns and many splits, beside a request of one split and an almost empty one; twice, bit for bit."""
    rng = np.random.default_rng(L)
    trees = [ref.random_tree(rng, nodes, "random"), [-1], ref.random_tree(rng, 2, "chain")]
    check_attention(ops, rng, H, Hkv, hd, kv, io, [L, 9, 0], trees, tag="merge")
    cache = ref.Cache(rng, 1, Hkv, hd, [L + nodes], kv)
    view, b = cache.device(), batch_of([0], [L], trees[:1])
    q = torch.from_numpy(rng.standard_normal((nodes, H, hd), dtype=np.float32)).to(io).cuda()
    first = ops.attention(view, 0, b, q)
    assert all(torch.equal(ops.attention(view, 0, b, q), first) for _ in range(3))


@pytest.mark.parametrize("kv", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_ignores_what_a_row_does_not_see(ops, kv, hd):
    """NaN and infinities in other branches' keys and values reach only the rows that see them."""
    rng = np.random.default_rng(8)
    par = [-1, 0, 0, 1, 2, 4, 3, 0]
    for where, bad in ((("v",), float("nan")), (("k",), float("inf")), (("k", "v"), float("-inf")), (("v",), float("inf"))):
        for length in (0, 13, 32, 300):
            cache = ref.Cache(rng, 1, 2, hd, [length + 8], kv, fill=float("nan"))
            p = length + 2  # node 2: seen by itself and its descendants 4 and 5
            for name in where:
                getattr(cache, name)[0, cache.table[0, p // 16], :, p % 16] = bad
            q = torch.from_numpy(rng.standard_normal((8, 4, hd), dtype=np.float32))
            out = ops.attention(cache.device(), 0, batch_of([0], [length], [par]), q.cuda()).double().cpu().numpy()
            want = ref.attention(cache, 0, [0], [length], [par], q)
            blind = [0, 1, 3, 6, 7]
            assert np.isfinite(want[blind]).all()
            tol = attention_tolerance(cache, q, length + 8, torch.float32)
            d = np.abs(out[blind] - want[blind]).max()
            assert d <= tol, (where, bad, length, d, tol)
            assert not np.isfinite(out[[2, 4, 5]]).all(), (where, bad, length)


def test_wide_trees_ignore_what_a_row_does_not_see(ops):
    """The same for column groups that share their blocks: many heads per KV head, poison in one branch."""
    rng = np.random.default_rng(18)
    par = [-1, 0, 0, 1, 2, 4, 3, 0]
    for kv in (torch.float32, torch.bfloat16):
        for hd in (64, 128):
            for length in (0, 30, 200):
                cache = ref.Cache(rng, 1, 1, hd, [length + 8], kv, fill=float("inf"))
                p = length + 2
                cache.v[0, cache.table[0, p // 16], :, p % 16, ::3] = float("nan")
                cache.k[0, cache.table[0, p // 16], :, p % 16] = float("inf")
                q = torch.from_numpy(rng.standard_normal((8, 16, hd), dtype=np.float32))
                out = ops.attention(cache.device(), 0, batch_of([0], [length], [par]), q.cuda()).double().cpu().numpy()
                want = ref.attention(cache, 0, [0], [length], [par], q)
                blind = [0, 1, 3, 6, 7]
                assert np.isfinite(want[blind]).all()
                assert np.abs(out[blind] - want[blind]).max() <= attention_tolerance(cache, q, length + 8, torch.float32), (kv, hd, length)
                assert not np.isfinite(out[[2, 4, 5]]).all()


def test_attention_of_strided_rows_leaves_the_rest(ops):
    rng = np.random.default_rng(9)
    H, Hkv, hd, lens = 8, 2, 64, [40, 3]
    trees = [ref.random_tree(rng, 6, "random"), ref.random_tree(rng, 4, "chain")]
    cache = ref.Cache(rng, 1, Hkv, hd, [46, 7], torch.bfloat16, fill=float("nan"))
    packed = torch.from_numpy(rng.standard_normal((14, H + 2 * Hkv, hd), dtype=np.float32)).cuda()
    wide = torch.full((14, H + 4, hd), 7.0, device="cuda")
    view = cache.device()
    b = batch_of([0, 1], lens, trees)
    plain = ops.attention(view, 0, b, packed[:10, :H].contiguous())
    out = ops.attention(view, 0, b, packed[:10, :H], out=wide[:10, 2:2 + H])
    torch.cuda.synchronize()
    assert torch.equal(out, plain)
    assert (wide[10:] == 7).all() and (wide[:, :2] == 7).all() and (wide[:, 2 + H:] == 7).all()


def test_attention_repeats_bit_for_bit(ops):
    rng = np.random.default_rng(10)
    cache = ref.Cache(rng, 1, 4, 128, [3000, 77], torch.bfloat16)
    trees = [ref.random_tree(rng, 20, "random"), ref.random_tree(rng, 5, "chain")]
    view, b = cache.device(), batch_of([0, 1], [2980, 72], trees)
    q = torch.from_numpy(rng.standard_normal((25, 8, 128), dtype=np.float32)).cuda()
    first = ops.attention(view, 0, b, q)
    for _ in range(5):
        assert torch.equal(ops.attention(view, 0, b, q), first)


def test_bad_block_ids_are_read_as_block_0_and_reported():
    rng = np.random.default_rng(11)
    for bad in (-1, 1 << 30, 9):
        o = fresh_ops()
        cache = ref.Cache(rng, 1, 2, 64, [70], torch.float32, extra_blocks=1)
        good = cache.table.copy()
        cache.table[0, 2] = 0
        view = cache.device()
        q = torch.from_numpy(rng.standard_normal((3, 4, 64), dtype=np.float32)).cuda()
        b = batch_of([0], [64], [[-1, 0, 1]])
        want = o.attention(view, 0, b, q)
        view.block_table[0, 2] = bad
        got = o.attention(view, 0, b, q)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        with pytest.raises(Exception, match="block id"):
            o.attention(view, 0, b, q)
        o.close()
        assert good.shape == cache.table.shape


# ------------------------------------------------------------------------------------------------------- verification


def make_verify(rng, V, trees, dtype, draft, spread=2.0, agree=0.7):
    R = sum(len(t) for t in trees)
    logits = torch.from_numpy(rng.standard_normal((R, V)).astype(np.float32) * spread)
    hot = rng.integers(0, V, size=(R, 4))
    logits.scatter_(1, torch.from_numpy(hot), torch.from_numpy(rng.uniform(4, 12, size=(R, 4)).astype(np.float32)))
    logits = logits.to(dtype)
    q = torch.softmax(logits.float() + agree * torch.from_numpy(rng.standard_normal((R, V)).astype(np.float32)), 1).to(dtype)
    tokens = np.zeros(R, np.int32)
    r0 = 0
    for t in trees:
        for j in range(1, len(t)):
            p = q[r0 + t[j]].double().numpy()
            tokens[r0 + j] = rng.choice(V, p=p / p.sum())
        r0 += len(t)
    return logits, (q if draft else None), tokens, rng.random(R, dtype=np.float32), rng.random(len(trees), dtype=np.float32)


def run_verify(ops, trees, tokens, logits, accept, sample, q=None, temperature=None):
    cu = lambda x: None if x is None else torch.as_tensor(x).cuda()  # noqa: E731
    e, p, c = ops.verify(batch_of(None, None, trees), cu(tokens), cu(logits), cu(accept), cu(sample), draft_probs=cu(q),
                         temperature=temperature)
    torch.cuda.synchronize()
    return e.cpu().numpy(), p.cpu().numpy(), c.cpu().numpy()


def same(got, want):
    for g, w, name in zip(got, want, ("emitted", "path", "count")):
        assert np.array_equal(g, w), (name, np.flatnonzero(g != w)[:8], g[g != w][:8], w[g != w][:8])


@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 3, 500, 4095, 4096, 4097, 12289, 32000, 131072])
def test_verify_vocabularies(ops, V, dtype, draft):
    rng = np.random.default_rng(V + draft)
    trees = [ref.random_tree(rng, n, k) for n, k in [(1, "chain"), (5, "chain"), (9, "star"), (14, "levels"), (12, "random"), (3, "star")]]
    temps = [1.0, 0.7, 1.3, 0.0, 0.9, 0.0]
    say(f"tree verify V {V} {dtype} draft {draft}")
    for _ in range(3):
        logits, q, tokens, ua, us = make_verify(rng, V, trees, dtype, draft)
        got = run_verify(ops, trees, tokens, logits, ua, us, q, temps)
        same(got, ref.verify(trees, tokens, logits.double().numpy(), ua, us, None if q is None else q.double().numpy(), temps))


@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("n,kind,B", [(64, "star", 2), (64, "chain", 2), (64, "random", 2), (2, "chain", 64), (1, "chain", 64), (8, "levels", 16)])
def test_verify_trees(ops, n, kind, B, draft):
    rng = np.random.default_rng(n + B + draft)
    trees = [ref.random_tree(rng, n, kind) for _ in range(B)]
    say(f"tree verify {B} x {n} {kind} draft {draft}")
    for agree in (0.0, 0.5, 3.0):
        logits, q, tokens, ua, us = make_verify(rng, 300, trees, torch.float32, draft, agree=agree)
        got = run_verify(ops, trees, tokens, logits, ua, us, q)
        same(got, ref.verify(trees, tokens, logits.double().numpy(), ua, us, None if q is None else q.double().numpy()))


def test_verify_uniforms_at_their_ends(ops):
    """0 accepts whatever has any probability; values that round to 1 (and past it) draw the last token of positive weight."""
    rng = np.random.default_rng(20)
    trees = [ref.random_tree(rng, 6, "levels") for _ in range(4)]
    logits, q, tokens, ua, us = make_verify(rng, 700, trees, torch.float32, True)
    logits[:, 650:] = float("-inf")
    for a, s in ((0.0, 0.0), (np.float32(1 - EPS), np.float32(1 - EPS)), (1.0, 1.0), (0.0, 1.0)):
        for d in (None, q):
            ua[:], us[:] = a, s
            got = run_verify(ops, trees, tokens, logits, ua, us, d)
            same(got, ref.verify(trees, tokens, logits.double().numpy(), ua, us, None if d is None else d.double().numpy()))
            assert s != 1.0 or d is not None or (got[0][np.cumsum([0, 6, 6, 6]) + got[2] - 1] == 649).sum() >= 1


def test_verify_ties_and_repeated_tokens(ops):
    """Equal maxima: the lowest index.  The same drafted token twice below one node: the second is never accepted after the
    first was not."""
    V, trees = 9000, [[-1, 0, 0, 0, 1], [-1, 0, 0]]
    logits = np.zeros((8, V), np.float32)
    logits[:, [4500, 8191, 8192]] = 3.0
    tokens = np.array([0, 8191, 4500, 4500, 4500, 0, 77, 77], np.int32)
    ua, us = np.full(8, 0.9, np.float32), np.array([0.5, 0.3], np.float32)
    same(run_verify(ops, trees, tokens, logits, ua, us, None, 0.0), ref.verify(trees, tokens, logits, ua, us, None, [0, 0]))
    same(run_verify(ops, trees, tokens, logits, ua, us), ref.verify(trees, tokens, logits, ua, us))
    two = np.full((8, V), -np.inf, np.float32)
    two[:, 4500], two[:, 77] = 0.0, 0.0  # half of the mass on each: rejecting 77 leaves 4500 alone
    ua[:] = 0.6
    got = run_verify(ops, trees, tokens, two, ua, us)
    same(got, ref.verify(trees, tokens, two, ua, us))
    assert got[0][5] == 4500 and got[2][1] == 1


def test_verify_never_draws_a_rejected_token(ops):
    """Whole chunks of the vocabulary whose weight the rejected tokens took, where rounding (49 * (1 / 49) < 1) leaves a
    trace of it, at both ends of the draw."""
    V = 12000
    for others in (48, 97, 102):
        for home in (10, 5000, 11999):
            z = torch.full((3, V), -float("inf"))
            z[:, home] = 0.0
            at = [t for t in range(1000, 1000 + 50 * others, 50) if t // 4096 != home // 4096][:others]
            at += [t for t in range(9000, 11900) if t // 4096 != home // 4096][:others - len(at)]
            at += list(range(2000, 4000))[:others - len(at)]
            z[:, at] = 0.0
            tokens = torch.tensor([0, home, home], dtype=torch.int32)
            ua = torch.tensor([0.0, 0.99, 0.99])
            for us in (0.0, 0.5, 1 - 2.0**-24):
                # Equal weights: the k-th entry's cumulative weight is (k + 1) / others up to rounding, so a target that
                # is exactly k / others may fall to entry k - 1 as well.
                x = us * others
                right = [sorted(at)[k] for k in {int(np.floor(x)), int(np.ceil(x)) - 1} if k >= 0]
                # a child that is the chunk's only weight, once and twice; and the same as a draft that puts all on it
                e, p, c = run_verify(ops, [[-1, 0, 0]], tokens, z, ua, torch.tensor([us]))
                assert c[0] == 1 and e[0] in right, (others, home, us)
                q = torch.zeros(3, V)
                q[:, home] = 1.0
                e, p, c = run_verify(ops, [[-1, 0, 0]], tokens, z, ua, torch.tensor([us]), q)
                assert c[0] == 1 and e[0] in right, (others, home, us)


def test_verify_strides_and_alignment(ops):
    rng = np.random.default_rng(21)
    trees = [ref.random_tree(rng, 7, "levels"), ref.random_tree(rng, 4, "chain")]
    for dtype in (torch.float32, torch.bfloat16):
        logits, q, tokens, ua, us = make_verify(rng, 5001, trees, dtype, True)
        want = ref.verify(trees, tokens, logits.double().numpy(), ua, us, q.double().numpy())
        for pad, off in ((7, 0), (7, 3), (8, 8), (0, 0)):
            def wide(x):
                w = torch.full((11, 5001 + pad + off), float("nan"), dtype=dtype, device="cuda")
                w[:, off:off + 5001] = x.cuda()
                return w[:, off:off + 5001]
            e = ops.verify(batch_of(None, None, trees), torch.as_tensor(tokens).cuda(), wide(logits), torch.as_tensor(ua).cuda(),
                           torch.as_tensor(us).cuda(), draft_probs=wide(q))
            same([x.cpu().numpy() for x in e], want)


def test_verify_odd_draft_probabilities(ops):
    """Negative and NaN entries count as 0; rows that do not sum to 1, rows of zeros, and rows that leave nothing."""
    rng = np.random.default_rng(22)
    trees = [ref.random_tree(rng, 9, "star") for _ in range(6)]
    logits, q, tokens, ua, us = make_verify(rng, 1200, trees, torch.float32, True)
    q = q.numpy().copy()
    q[0:9, ::3] = -1.0
    q[9:18, 1::2] = np.nan
    q[18:27] = 0.0
    q[27:36] *= 40.0
    q[36:45] = 1.0
    q[45:54] = np.inf
    clean = np.where(np.isnan(q), 0, q)
    ua[36:54] = 0.5
    with np.errstate(all="ignore"):
        want = ref.verify(trees, tokens, logits.double().numpy(), ua, us, clean)
    same(run_verify(ops, trees, tokens, logits, ua, us, q), want)


def test_verify_bad_rows_and_tokens_are_reported():
    rng = np.random.default_rng(23)
    trees = [[-1, 0], [-1, 0], [-1, 0, 1]]
    for kind in ("nan", "inf", "empty", "token"):
        o = fresh_ops()
        logits, _, tokens, ua, us = make_verify(rng, 5000, trees, torch.float32, False)
        if kind == "nan":
            logits[2, 4990] = float("nan")
        elif kind == "inf":
            logits[2, 17] = float("inf")
        elif kind == "empty":
            logits[2] = float("-inf")
        else:
            tokens[[3, 5]] = [-4, 1 << 30]
        got = run_verify(o, trees, tokens, logits, ua, us)
        same(got, ref.verify(trees, tokens, logits.double().numpy(), ua, us))
        if kind != "token":
            assert got[2][1] == 0 and (got[0][2:4] == -1).all() and (got[1][2:4] == -1).all()
        with pytest.raises(Exception, match="device check"):
            run_verify(o, trees, tokens, logits, ua, us)
        o.close()


def test_verify_emits_the_targets_distribution(ops):
    """First emitted token over many independent draws, with draft probabilities far from the target's: its frequencies are
    p's.  64 requests a call; per token, 5 standard deviations of a binomial count."""
    rng = np.random.default_rng(24)
    V, calls = 12, 150
    p = rng.dirichlet(np.full(V, 0.5))
    q = rng.dirichlet(np.full(V, 0.5))
    trees = [[-1, 0]] * 64
    logits = np.log(p).astype(np.float32)[None].repeat(128, 0)
    p = np.exp(logits[0].astype(np.float64))
    p /= p.sum()
    seen = np.zeros(V)
    for _ in range(calls):
        tokens = rng.choice(V, size=128, p=q).astype(np.int32)
        e, _, _ = run_verify(ops, trees, tokens, logits, rng.random(128, dtype=np.float32), rng.random(64, dtype=np.float32),
                             q.astype(np.float32)[None].repeat(128, 0))
        seen += np.bincount(e[::2], minlength=V)
    n = calls * 64
    assert np.all(np.abs(seen - n * p) <= 5 * np.sqrt(n * p * (1 - p)) + 1), (seen / n, p)


# --------------------------------------------------------------------------------------------------------- compaction


@pytest.mark.parametrize("kv", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("Hkv,hd,layers", [(1, 64, 1), (5, 64, 3), (8, 128, 2), (3, 128, 2)])
def test_keep_moves_paths(ops, kv, Hkv, hd, layers):
    """Random ascending paths (overlapping moves among them), whole trees, single nodes, and requests that keep nothing."""
    rng = np.random.default_rng(30)
    nodes = [9, 64, 1, 12, 17, 5]
    lens = [0, 37, 15, 16, 100, 3]
    trees = [ref.random_tree(rng, n, "random") for n in nodes]
    slots = [5, 0, 3, 1, 4, 2]
    positions = [0] * 6
    for i, s in enumerate(slots):
        positions[s] = lens[i] + nodes[i]
    for trial in range(4):
        cache = ref.Cache(rng, layers, Hkv, hd, positions, kv)
        path = np.full(sum(nodes), -1, np.int32)
        count = np.zeros(6, np.int32)
        r0 = 0
        for i, n in enumerate(nodes):
            c = [n, min(n, 20), 1, max(1, n // 2), min(n, 3), 0][(i + trial) % 6]
            path[r0:r0 + c] = np.concatenate([[0], 1 + np.sort(rng.permutation(n - 1)[:c - 1])]) if c else []
            count[i] = c if c else rng.integers(-3, 1)
            r0 += n
        view = cache.device()
        ops.keep(view, batch_of(slots, lens, trees), torch.as_tensor(path).cuda(), torch.as_tensor(count).cuda())
        torch.cuda.synchronize()
        ref.keep(cache, slots, lens, trees, path, count)
        assert torch.equal(view.k.cpu(), ref.to_tiles(cache.k, False)), trial
        assert torch.equal(view.v.cpu(), ref.to_tiles(cache.v, True)), trial


def test_keep_with_a_bad_block_id_moves_nothing():
    rng = np.random.default_rng(32)
    for pos, bad in ((40, -1), (16, 99)):  # a source's block, a target's
        o = fresh_ops()
        cache = ref.Cache(rng, 2, 2, 64, [46, 30], torch.float32)
        view = cache.device()
        view.block_table[0, pos // 16] = bad
        b = batch_of([0, 1], [28, 9], [[-1] + [0] * 15, [-1, 0, 0]])
        p = torch.tensor([0, 13] + [-1] * 14 + [0, 2, -1], dtype=torch.int32).cuda()
        o.keep(view, b, p, torch.tensor([2, 2], dtype=torch.int32).cuda())
        torch.cuda.synchronize()
        ref.keep(cache, [1], [9], [[-1, 0, 0]], [0, 2], [2])  # the other request's
        assert torch.equal(view.k.cpu(), ref.to_tiles(cache.k, False)) and torch.equal(view.v.cpu(), ref.to_tiles(cache.v, True))
        with pytest.raises(Exception, match="block id"):
            o.keep(view, b, p, torch.tensor([2, 2], dtype=torch.int32).cuda())
        o.close()


def test_keep_refuses_malformed_paths():
    rng = np.random.default_rng(31)
    for path, count in (([0, 3, 2, -1], 3), ([0, 0, 1, -1], 3), ([0, 1, 4, -1], 3), ([0, 1, 2, 3], 5), ([0, -1, 2, 3], 3),
                        ([0, 1, 1 << 30, 3], 3), ([-1, 1, 2, 3], 3)):
        o = fresh_ops()
        cache = ref.Cache(rng, 2, 2, 64, [30, 30], torch.bfloat16)
        view = cache.device()
        k, v = view.k.clone(), view.v.clone()
        b = batch_of([0, 1], [20, 21], [[-1, 0, 0, 0], [-1, 0, 0, 0]])
        p, c = torch.tensor(path + [0, 2, -1, -1], dtype=torch.int32).cuda(), torch.tensor([count, 2], dtype=torch.int32).cuda()
        o.keep(view, b, p, c)
        torch.cuda.synchronize()
        ref.keep(cache, [1], [21], [[-1, 0, 0, 0]], [0, 2], [2])  # the other request's path is fine
        assert torch.equal(view.k.cpu(), ref.to_tiles(cache.k, False)) and torch.equal(view.v.cpu(), ref.to_tiles(cache.v, True))
        assert not torch.equal(view.k, k) or not torch.equal(view.v, v)
        with pytest.raises(Exception, match="path"):
            o.keep(view, b, p, c)
        o.close()


# ------------------------------------------------------------------------------------------- streams, graphs, the set


def setup_set(rng):
    H, Hkv, hd, V = 8, 2, 64, 900
    lens, trees = [50, 7, 333], [ref.random_tree(rng, n, "levels") for n in (9, 4, 13)]
    slots = [1, 2, 0]
    positions = [346, 59, 11]
    cache = ref.Cache(rng, 2, Hkv, hd, positions, torch.bfloat16, fill=float("nan"))
    R = 26
    q = torch.from_numpy(rng.standard_normal((R, H, hd), dtype=np.float32))
    logits, d, tokens, ua, us = make_verify(rng, V, trees, torch.float32, True)
    return cache, slots, lens, trees, q, logits, d, tokens, ua, us


def test_the_operators_together(ops):
    """Attention in each layer, verification, compaction: as one step uses them."""
    rng = np.random.default_rng(40)
    cache, slots, lens, trees, q, logits, d, tokens, ua, us = setup_set(rng)
    view, b = cache.device(), batch_of(slots, lens, trees)
    cu = lambda x: torch.as_tensor(x).cuda()  # noqa: E731
    outs = [ops.attention(view, layer, b, q.cuda()) for layer in range(2)]
    e, p, c = ops.verify(b, cu(tokens), cu(logits), cu(ua), cu(us), draft_probs=cu(d))
    ops.keep(view, b, p, c)
    torch.cuda.synchronize()
    for layer in range(2):
        want = ref.attention(cache, layer, slots, lens, trees, q)
        assert np.abs(outs[layer].double().cpu().numpy() - want).max() <= attention_tolerance(cache, q, 400, torch.float32)
    want = ref.verify(trees, tokens, logits.double().numpy(), ua, us, d.double().numpy())
    same([x.cpu().numpy() for x in (e, p, c)], want)
    ref.keep(cache, slots, lens, trees, want[1], want[2])
    # Bitwise, the NaN of the never-written positions too.
    ints = lambda x: x.view(torch.int16)  # noqa: E731
    assert torch.equal(ints(view.k.cpu()), ints(ref.to_tiles(cache.k, False)))
    assert torch.equal(ints(view.v.cpu()), ints(ref.to_tiles(cache.v, True)))


def test_another_stream(ops):
    """Inputs made on a side stream, the call on it, and a call back on the default stream."""
    rng = np.random.default_rng(41)
    cache, slots, lens, trees, q, *_ = setup_set(rng)
    view, b, qd = cache.device(), batch_of(slots, lens, trees), q.cuda()
    want = ops.attention(view, 0, b, qd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        big = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            big = big @ big * 1e-2
        got = ops.attention(view, 0, b, qd * 1.0)
    again = ops.attention(view, 0, b, qd)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(again, want)


def test_two_handles_on_two_streams():
    """Concurrent calls of a handle each; split rows, so that shared counters or partials would show."""
    rng = np.random.default_rng(45)
    handles, jobs = [fresh_ops(), fresh_ops()], []
    for o in handles:
        cache = ref.Cache(rng, 1, 2, 128, [5000, 900], torch.bfloat16)
        b = batch_of([0, 1], [4990, 880], [ref.random_tree(rng, 9, "levels"), ref.random_tree(rng, 12, "random")])
        q = torch.from_numpy(rng.standard_normal((21, 8, 128), dtype=np.float32)).cuda()
        z = torch.randn(21, 20000, device="cuda")
        tok = torch.randint(0, 20000, (21,), dtype=torch.int32, device="cuda")
        view, f = cache.device(), torch.rand(21, device="cuda")
        want = (o.attention(view, 0, b, q), *o.verify(b, tok, z, f, f[:2]))
        jobs.append((o, view, b, q, z, tok, f, want))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(20):
        for s, (o, view, b, q, z, tok, f, _) in zip(streams, jobs):
            with torch.cuda.stream(s):
                got.append((o.attention(view, 0, b, q), *o.verify(b, tok, z, f, f[:2])))
    torch.cuda.synchronize()
    for k, outs in enumerate(got):
        assert all(torch.equal(x, y) for x, y in zip(outs, jobs[k % 2][-1])), k
    for o in handles:
        o.close()


def test_captured_without_a_call_before():
    """A handle's first call of a kernel may be the captured one."""
    rng = np.random.default_rng(43)
    o = fresh_ops()
    cache = ref.Cache(rng, 1, 1, 128, [90], torch.bfloat16)
    view, b = cache.device(), batch_of([0], [80], [[-1, 0, 0, 1, 1]])
    q = torch.from_numpy(rng.standard_normal((5, 5, 128), dtype=np.float32)).to(torch.bfloat16).cuda()
    logits = torch.randn(5, 77, device="cuda").to(torch.bfloat16)
    tokens = torch.zeros(5, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = o.attention(view, 0, b, q)
        e, p, c = o.verify(b, tokens, logits, temperature=0.0)
        o.keep(view, b, p, c)
    k0 = view.k.clone()
    for _ in range(3):
        view.k.copy_(k0)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = ref.attention(cache, 0, [0], [80], [[-1, 0, 0, 1, 1]], q.cpu())
        assert np.abs(out.double().cpu().numpy() - want).max() <= attention_tolerance(cache, q.cpu(), 90, torch.bfloat16)
        same([x.cpu().numpy() for x in (e, p, c)], ref.verify([[-1, 0, 0, 1, 1]], np.zeros(5, np.int32), logits.double().cpu().numpy(),
                                                              None, None, None, [0]))
    o.close()


def test_refusals_leave_the_handle_usable(ops):
    from paper_2403_12900_amd.binding import SPR_ERR_INVALID_ARG, SproutError
    rng = np.random.default_rng(44)
    cache = ref.Cache(rng, 2, 2, 64, [40, 40], torch.bfloat16)
    view, b = cache.device(), batch_of([0, 1], [20, 30], [[-1, 0, 0], [-1]])
    q = torch.randn(4, 4, 64, device="cuda")
    f = torch.rand(4, device="cuda")
    tok = torch.zeros(4, dtype=torch.int32, device="cuda")
    z = torch.randn(4, 50, device="cuda")
    n2 = torch.zeros(2, dtype=torch.int32, device="cuda")
    calls = [lambda: ops.attention(view, 2, b, q), lambda: ops.attention(view, -1, b, q),
             lambda: ops.attention(view, 0, batch_of([0, 2], [20, 30], [[-1, 0, 0], [-1]]), q),
             lambda: ops.attention(view, 0, batch_of([0, 1], [20, 48], [[-1, 0, 0], [-1]]), q),
             lambda: ops.attention(view, 0, b, q[:3]), lambda: ops.attention(view, 0, b, q.half()), lambda: ops.attention(view, 0, b, q.cpu()),
             lambda: ops.attention(view, 0, b, torch.randn(4, 3, 64, device="cuda")),
             lambda: ops.attention(view, 0, b, torch.randn(4, 34, 64, device="cuda")),
             lambda: ops.attention(view, 0, b, torch.randn(4, 4, 128, device="cuda")[..., ::2]),
             lambda: ops.attention(view, 0, b, torch.randn(4, 4, 65, device="cuda")[..., 1:]),
             lambda: ops.attention(view, 0, b, q, out=q[:, :2]),
             lambda: ops.verify(b, tok[:3], z, f, f[:2]), lambda: ops.verify(b, tok.long(), z, f, f[:2]),
             lambda: ops.verify(b, tok, z, None, None), lambda: ops.verify(b, tok, z, f, None), lambda: ops.verify(b, tok, z, f, f),
             lambda: ops.verify(b, tok, z.half(), f, f[:2]), lambda: ops.verify(b, tok, z.t().contiguous().t(), f, f[:2]),
             lambda: ops.verify(b, tok, z, f, f[:2], draft_probs=z[:, :40]), lambda: ops.verify(b, tok, z, f, f[:2], draft_probs=z.bfloat16()),
             lambda: ops.verify(b, tok, z, f, f[:2], temperature=-1.0), lambda: ops.verify(b, tok, z, f, f[:2], temperature=[1.0]),
             lambda: ops.verify(b, tok, z[:, :0], f, f[:2]),
             lambda: ops.keep(view, b, tok[:3], n2), lambda: ops.keep(view, b, tok, n2.long()), lambda: ops.keep(view, b, tok.cpu(), n2)]
    for k, call in enumerate(calls):
        with pytest.raises(SproutError) as e:
            call()
        assert e.value.status == SPR_ERR_INVALID_ARG, k
    ops.attention(view, 1, b, q)
    ops.verify(b, tok, z, temperature=0.0)
    torch.cuda.synchronize()


def test_captured_and_replayed():
    """Graphs of the set, replayed with new inputs in place and eager calls between the replays; two graphs of one handle."""
    rng = np.random.default_rng(42)
    o = fresh_ops()
    cache, slots, lens, trees, q, logits, d, tokens, ua, us = setup_set(rng)
    view, b = cache.device(), batch_of(slots, lens, trees)
    k0, v0 = view.k.clone(), view.v.clone()
    cu = lambda x: torch.as_tensor(x).cuda()  # noqa: E731
    sq, sl, sd, st, sa, ss = q.cuda(), cu(logits), cu(d), cu(tokens), cu(ua), cu(us)

    def step():
        a = [o.attention(view, layer, b, sq) for layer in range(2)]
        e, p, c = o.verify(b, st, sl, sa, ss, draft_probs=sd)
        o.keep(view, b, p, c)
        return a, e, p, c

    step()  # warm
    view.k.copy_(k0), view.v.copy_(v0)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held = step()
        graphs.append((g, held))
    torch.cuda.synchronize()
    for round_ in range(4):
        sq.copy_(torch.from_numpy(rng.standard_normal(tuple(q.shape), dtype=np.float32)))
        sa.copy_(torch.from_numpy(rng.random(len(ua), dtype=np.float32)))
        for g, held in graphs:
            view.k.copy_(k0), view.v.copy_(v0)
            want = step()
            torch.cuda.synchronize()
            wk, wv = view.k.clone(), view.v.clone()
            view.k.copy_(k0), view.v.copy_(v0)
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip([*held[0], *held[1:]], [*want[0], *want[1:]]):
                assert torch.equal(x, y), round_
            assert torch.equal(view.k.view(torch.int16), wk.view(torch.int16))
            assert torch.equal(view.v.view(torch.int16), wv.view(torch.int16))
    o.close()
