"""Host side of the drafted-tree operators (no GPU): what a call's arguments must satisfy, the relations derived from a
batch, the launch split, the slot bookkeeping of a tree step, and the plain implementations that the GPU tests compare with.
"""
import ctypes

import numpy as np
import pytest
import torch

from paper_2403_12900_amd import binding
from paper_2403_12900_amd.binding import SprKvView, SprTreeBatch, SproutError
from paper_2403_12900_amd.tree import KVView, TreeBatch

from . import tree_ref as ref
from .test_abi_host import HOST_LIB, Host

I32 = ctypes.POINTER(ctypes.c_int32)


def host():
    L = ctypes.CDLL(HOST_LIB)
    L.sprh_last_error.restype = ctypes.c_char_p
    L.sprh_tree_split.argtypes = [ctypes.c_void_p] + [ctypes.c_int] * 5 + [ctypes.c_size_t, I32]
    return L


def a32(x):
    return np.ascontiguousarray(np.asarray(x, dtype=np.int32))


def p32(x):
    return x.ctypes.data_as(I32)


def raw_batch(n, slots, lens, nodes, parents):
    keep = [None if x is None else a32(x) for x in (slots, lens, nodes, parents)]
    b = SprTreeBatch(n, *(None if x is None else p32(x) for x in keep))
    b._keep = keep
    return b


def parse(b, with_cache=1, n_slots=8, max_blocks=100):
    L = host()
    depth, rank, kids, levels, children = (np.zeros(128, np.int32) for _ in range(5))
    anc = np.zeros(128, np.uint64)
    st = L.sprh_tree_parse(ctypes.byref(b) if b is not None else None, with_cache, n_slots, max_blocks, p32(depth), p32(rank),
                           p32(kids), anc.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64)), p32(levels), p32(children))
    return st, L.sprh_last_error().decode(), depth, rank, kids, anc, levels, children


def test_relations_of_a_batch():
    rng = np.random.default_rng(1)
    trees = [ref.random_tree(rng, n, k) for n, k in ((1, "chain"), (64, "random"), (20, "levels"), (7, "star"), (30, "chain"))]
    b = raw_batch(5, [3, 0, 7, 1, 2], [0, 5, 16, 1000, 1500], [len(t) for t in trees], sum(trees, []))
    st, _, depth, rank, kids, anc, levels, children = parse(b)
    assert st == 0
    r = 0
    for i, t in enumerate(trees):
        for j, p in enumerate(t):
            chain = ref.ancestors(t, j)
            assert depth[r + j] == len(chain) - 1
            assert int(anc[r + j]) == sum(1 << c for c in chain)
            assert rank[r + j] == sum(1 for q in t[1:j] if q == p) if j else rank[r] == 0
            assert kids[r + j] == sum(1 for q in t[1:] if q == j)
        assert levels[i] == max(len(ref.ancestors(t, j)) for j in range(len(t)))
        assert children[i] == max(kids[r:r + len(t)])
        r += len(t)


@pytest.mark.parametrize("n,slots,lens,nodes,parents,what", [
    (0, [0], [0], [1], [-1], "n must be"),
    (65, [0] * 65, [0] * 65, [1] * 65, [-1] * 65, "n must be"),
    (1, None, [0], [1], [-1], "null"),
    (1, [0], None, [1], [-1], "null"),
    (1, [0], [0], None, [-1], "null"),
    (1, [0], [0], [1], None, "null"),
    (1, [0], [0], [0], [-1], "n_nodes"),
    (1, [0], [0], [-3], [-1], "n_nodes"),
    (1, [0], [0], [65], [-1] + list(range(64)), "n_nodes"),
    (3, [0, 1, 2], [0] * 3, [64, 64, 1], ([-1] + list(range(63))) * 2 + [-1], "SPR_MAX_TREE_ROWS"),
    (1, [8], [0], [1], [-1], "slot id"),
    (1, [-1], [0], [1], [-1], "slot id"),
    (2, [4, 4], [0, 0], [1, 1], [-1, -1], "twice"),
    (1, [0], [-1], [1], [-1], "lens"),
    (1, [0], [2 ** 31 - 1], [1], [-1], "lens"),
    (1, [0], [1600], [1], [-1], "block-table row"),
    (1, [0], [1599], [2], [-1, 0], "block-table row"),
    (1, [0], [0], [1], [0], "parents"),
    (1, [0], [0], [2], [-1, -1], "parents"),
    (1, [0], [0], [3], [-1, 0, 2], "parents"),
    (1, [0], [0], [3], [-1, 2, 0], "parents"),
    (2, [0, 1], [0, 0], [2, 2], [-1, 0, 0, 0], "parents"),
])
def test_batches_that_are_refused(n, slots, lens, nodes, parents, what):
    st, msg, *_ = parse(raw_batch(n, slots, lens, nodes, parents))
    assert st == binding.SPR_ERR_INVALID_ARG and what in msg, msg


def test_batch_limits_that_are_taken():
    assert parse(None)[0] == binding.SPR_ERR_INVALID_ARG
    assert parse(raw_batch(1, [0], [1598], [2], [-1, 0]))[0] == 0
    assert parse(raw_batch(2, [0, 1], [0, 0], [64, 64], ([-1] + [0] * 63) * 2))[0] == 0
    assert parse(raw_batch(2, None, None, [2, 1], [-1, 0, -1]), with_cache=0)[0] == 0
    assert parse(raw_batch(1, [0], [1 << 30], [64], [-1] + [0] * 63), max_blocks=1 << 27)[0] == 0


def view(**kw):
    d = dict(k=4096, v=8192, kv_dtype=1, n_layers=2, n_blocks=3, n_kv_heads=4, head_dim=64, block_table=16, n_slots=2, max_blocks=5)
    d.update(kw)
    return SprKvView(**d)


@pytest.mark.parametrize("kw,layer", [({"k": None}, 0), ({"v": None}, 0), ({"block_table": None}, 0), ({"k": 4104}, 0), ({"v": 8196}, 0),
                                      ({"block_table": 18}, 0), ({"kv_dtype": 2}, 0), ({"kv_dtype": -1}, 0), ({"head_dim": 96}, 0),
                                      ({"n_kv_heads": 0}, 0), ({"n_kv_heads": 513}, 0), ({"n_layers": 0}, 0), ({"n_blocks": 0}, 0),
                                      ({"n_slots": 0}, 0), ({"max_blocks": -1}, 0), ({}, 2), ({}, -1)])
def test_views_that_are_refused(kw, layer):
    assert host().sprh_tree_view(ctypes.byref(view()), 1) == 0
    assert host().sprh_tree_view(ctypes.byref(view(**kw)), layer) == binding.SPR_ERR_INVALID_ARG
    assert host().sprh_tree_view(None, 0) == binding.SPR_ERR_INVALID_ARG


def test_temperatures():
    L = host()
    f = lambda *x: (ctypes.c_float * len(x))(*x)  # noqa: E731
    u = ctypes.c_void_p(64)
    assert L.sprh_tree_temperatures(2, f(0.0, 1.5), u, u) == 0
    assert L.sprh_tree_temperatures(2, f(0.0, 0.0), None, None) == 0
    assert L.sprh_tree_temperatures(2, None, u, u) == 0
    for bad in (-0.5, float("nan"), float("inf")):
        assert L.sprh_tree_temperatures(2, f(1.0, bad), u, u) == binding.SPR_ERR_INVALID_ARG
    for acc, smp in ((None, u), (u, None)):
        assert L.sprh_tree_temperatures(2, f(0.0, 1.0), acc, smp) == binding.SPR_ERR_INVALID_ARG
        assert L.sprh_tree_temperatures(2, None, acc, smp) == binding.SPR_ERR_INVALID_ARG


def test_launch_split_covers_every_block_within_its_room():
    L, rng = host(), np.random.default_rng(2)
    for _ in range(400):
        n = int(rng.integers(1, 65))
        nodes = [int(rng.integers(1, max(2, min(65, 128 // n + 1)))) for _ in range(n)]
        lens = [int(2 ** rng.uniform(0, rng.choice([8, 14, 20, 30]))) for _ in range(n)]
        G, Hkv, hd, step = int(rng.choice([1, 8, 13, 16])), int(rng.choice([1, 8, 40, 512])), int(rng.choice([64, 128])), int(rng.choice([1, 2, 4, 8]))
        floats = int(rng.choice([1 << 18, 1 << 23, 1 << 28]))
        out = np.zeros(140, np.int32)
        b = raw_batch(n, range(n), lens, nodes, sum(([-1] + [0] * (k - 1) for k in nodes), []))
        assert L.sprh_tree_split(ctypes.byref(b), G, Hkv, hd, step, int(rng.choice([256, 1024])), floats, p32(out)) == 0
        cw, bps = int(out[0]), int(out[1])
        assert cw in (16, 32, 64, 128, 256) and bps >= 1 and bps % step == 0
        split = False
        order = out[3 + n:3 + 2 * n].tolist()
        assert sorted(order) == list(range(n))
        size = [-(-(lens[i] + nodes[i]) // 16) for i in order]
        assert size == sorted(size, reverse=True)
        for r, i in enumerate(order):
            ncg = -(-nodes[i] * G // cw)
            ns = -(-(-(-(lens[i] + nodes[i]) // 16)) // bps)
            assert out[2 + r + 1] - out[2 + r] == ncg * ns
            assert ns <= 32
            split |= ns > 1
        assert out[2] == 0 and out[2 + n] <= 65535
        if split:
            assert int(out[2 + n]) * Hkv * cw * (hd + 4) <= floats


def test_tree_step_bookkeeping():
    h = Host(max_slots=4, max_ctx=64, kv_blocks=8)
    L = host()

    def step(slots, lens, nodes, levels, count):
        x = [a32(v) for v in (slots, lens, nodes, levels, count)]
        r = np.full(len(slots), -1, np.int32)
        L.sprh_tree_step.argtypes = [ctypes.c_void_p, ctypes.c_int] + [I32] * 6
        return L.sprh_tree_step(h.h, len(slots), *[p32(v) for v in x], p32(r)), r, L.sprh_last_error().decode()

    assert h.prefill([1, 3], [20, 5], [13, 4])[0] == 0   # slot 1: 2 blocks, 12 tokens to go; slot 3: 1 block, 3 to go
    st, r, _ = step([1, 3], [20, 5], [12, 6], [12, 3], [5, 3])
    assert st == 0 and r.tolist() == [0, 1]
    assert h.slot(1) == (25, 6, 13, 1) and h.slot(3) == (8, 4, 4, 2)
    for args, want in ((([1], [24], [1], [1], [1]), binding.SPR_ERR_STATE),           # wrong length
                       (([3], [8], [1], [1], [1]), binding.SPR_ERR_STATE),            # finished
                       (([0], [0], [1], [1], [1]), binding.SPR_ERR_STATE),            # free
                       (([1], [25], [8], [3], [1]), binding.SPR_ERR_KV_FULL),         # 33 positions in 2 blocks
                       (([1], [25], [7], [8], [1]), binding.SPR_ERR_INVALID_ARG),     # 7 tokens to go
                       (([1, 1], [25, 25], [1, 1], [1, 1], [1, 1]), binding.SPR_ERR_INVALID_ARG),
                       (([4], [0], [1], [1], [1]), binding.SPR_ERR_INVALID_ARG)):
        assert step(*args)[0] == want, args
        assert h.slot(1) == (25, 6, 13, 1)
    assert step([1], [25], [7], [7], [7])[0] == 0
    assert h.slot(1) == (32, 13, 13, 2)
    assert h.L.sprh_rewind(h.h, 1, 22, 3) == 0 and h.slot(1) == (22, 3, 13, 1)
    assert h.decode([1], [22])[0] == 0


def test_calls_without_a_handle_are_refused():
    L = binding.load_library()
    b = TreeBatch([0], [0], [1], [-1])
    calls = (lambda: L.spr_tree_attention(None, None, 0, b.ref, 1, 0, None, 0, None, 0),
             lambda: L.spr_tree_verify(None, b.ref, 1, 0, None, None, 1, None, 0, None, None, None, None, None, None),
             lambda: L.spr_tree_keep(None, None, b.ref, None, None),
             lambda: L.spr_tree_ops_release(None), lambda: L.spr_tree_ops_set_stream(None, None),
             lambda: L.spr_model_kv_view(None, None),
             lambda: L.spr_tree_step(None, b.ref, None, None, None, None, None, None, None, None, None, None))
    for c in calls:
        assert c() == binding.SPR_ERR_INVALID_ARG
        assert L.spr_last_error()
    h = ctypes.c_void_p()
    assert L.spr_tree_ops_init(None, 1 << 30, None, ctypes.byref(h)) == binding.SPR_ERR_WORKSPACE
    assert L.spr_tree_ops_init(4096 + 8, 1 << 30, None, ctypes.byref(h)) == binding.SPR_ERR_WORKSPACE
    assert L.spr_tree_ops_init(4096, 100, None, ctypes.byref(h)) == binding.SPR_ERR_WORKSPACE and b"needed" in L.spr_last_error()
    assert L.spr_tree_ops_init(4096, 1 << 30, None, None) == binding.SPR_ERR_INVALID_ARG and not h.value


def test_python_side_refusals():
    k, table = torch.zeros(2, 3, 4, 1024), torch.zeros(2, 3, dtype=torch.int32)
    v = KVView(k, k.clone(), table)
    assert (v.head_dim, v.n_kv_heads) == (64, 4)
    for bad in ((k, k.double(), table), (k.half(), k.half(), table), (k, k[:1], table), (k, k, table.long()), (k, k, table[0]),
                (k[..., ::2], k[..., ::2], table), (k[0], k[0], table), (torch.zeros(2, 3, 4, 1000), torch.zeros(2, 3, 4, 1000), table),
                (k, k, table.t())):
        with pytest.raises(SproutError):
            KVView(*bad)
    for bad in (([0, 1], [0], [1, 1], [-1, -1]), ([0], [0], [2], [-1]), ([0], [0], [-1], [-1]), ([0], [0, 1], [1], [-1])):
        with pytest.raises(SproutError):
            TreeBatch(*bad)
    b = TreeBatch(None, None, [2, 1], [-1, 0, -1])
    parents = np.array([-1, 0, -1], dtype=np.int32)
    b2 = TreeBatch(None, None, [2, 1], parents)
    parents[:] = 99  # the batch keeps what it was given
    assert [b2._c.parents[i] for i in range(3)] == [-1, 0, -1]
    t = b.temperatures(0.5)
    assert [t[0], t[1]] == [0.5, 0.5] and b.temperatures(None) is None
    with pytest.raises(SproutError):
        b.temperatures([1.0, 2.0, 3.0])


# ------------------------------------------------------------- the plain implementations


def test_tiles_hold_every_element_once():
    for size, hd in ((4, 64), (4, 128), (2, 64), (2, 128)):
        for values in (False, True):
            off = ref.tile_offsets(size, hd, values)
            assert sorted(off.reshape(-1)) == list(range(16 * hd))
    x = torch.randn(2, 3, 16, 64).to(torch.bfloat16)
    assert torch.equal(ref.from_tiles(ref.to_tiles(x, True), True), x)


def test_nested_residuals_have_the_closed_form():
    """r_k = max(r_{k-1} - q, 0) / sum equals max(p - c_k q, 0) / N_k with c_{k+1} = c_k + N_k."""
    rng = np.random.default_rng(3)
    for _ in range(50):
        V = int(rng.integers(2, 40))
        p, q = rng.dirichlet(np.full(V, 0.7)), rng.dirichlet(np.full(V, 0.7))
        r, c, n = p, 0.0, 1.0
        for _ in range(6):
            nxt = np.maximum(r - q, 0)
            if nxt.sum() < 1e-9:
                break
            r = nxt / nxt.sum()
            c, n = c + n, None
            n = np.maximum(p - c * q, 0).sum()
            assert np.abs(np.maximum(p - c * q, 0) / n - r).max() < 1e-9


@pytest.mark.parametrize("children", [1, 2, 3])
def test_verification_preserves_the_targets_distribution(children):
    """Exactly, for the plain implementation's rule: children drawn from q, each accepted with probability min(1, r/q)."""
    rng = np.random.default_rng(4)
    V = 5
    p, q = rng.dirichlet(np.full(V, 0.6)), rng.dirichlet(np.full(V, 0.6))

    def emit(r, left):
        """Distribution of the emitted token given residual r and `left` children to try."""
        if left == 0:
            return r
        out = np.zeros(V)
        rest = np.maximum(r - q, 0)
        tail = emit(rest / rest.sum(), left - 1) if rest.sum() > 0 else np.zeros(V)
        for x in range(V):
            a = min(1.0, r[x] / q[x])
            out[x] += q[x] * a
            out += q[x] * (1 - a) * tail
        return out

    assert np.abs(emit(p, children) - p).max() < 1e-12
    # The implementation takes the same branch on either side of the acceptance border.
    trees = [[-1] + [0] * children]
    for x in range(V):
        a = min(1.0, p[x] / q[x])
        tokens = np.array([0] + [x] * children)
        logits = np.log(p)[None].repeat(1 + children, 0)
        for u in (a - 1e-6, a + 1e-6):
            if not 0 <= u < 1:
                continue
            e, _, c = ref.verify(trees, tokens, logits, np.full(1 + children, u), np.array([0.5]), q[None].repeat(1 + children, 0))
            assert (u < a) == (c[0] == 2 and e[0] == x) or children > 1


def test_a_planted_mistake_shows():
    """The comparisons notice a wrong ancestor, a wrong residual and a wrong move in the plain implementations."""
    rng = np.random.default_rng(5)
    cache = ref.Cache(rng, 1, 2, 64, [30], torch.float32)
    q = torch.randn(4, 4, 64)
    right = ref.attention(cache, 0, [0], [20], [[-1, 0, 0, 1]], q)
    wrong = ref.attention(cache, 0, [0], [20], [[-1, 0, 0, 2]], q)
    assert np.abs(right[:3] - wrong[:3]).max() == 0 and np.abs(right[3] - wrong[3]).max() > 1e-3
    before = cache.k.clone()
    ref.keep(cache, [0], [20], [[-1, 0, 0, 1]], [0, 2], [2])
    assert torch.equal(cache.k[0, cache.table[0, 1], :, 5], before[0, cache.table[0, 1], :, 6])
    assert int((cache.k != before).any(-1).sum()) == 2
