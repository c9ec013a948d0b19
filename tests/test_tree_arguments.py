"""Arguments of the drafted-tree operators that must not be taken for others (no GPU unless marked)."""
import numpy as np
import pytest
import torch

from paper_2403_12900_amd import binding
from paper_2403_12900_amd.binding import SproutError
from paper_2403_12900_amd.tree import TreeBatch


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("bad", [np.array([2 ** 32 + 1], dtype=np.int64), np.array([2 ** 32], dtype=np.uint64), [2 ** 40],
                                 np.array([-2 ** 31 - 1]), [1.5], np.array([float("nan")]), [float("inf")], ["1"], [None], [1 + 0j],
                                 [[1], [1, 2]]])
def test_numbers_that_are_no_int32_are_refused(which, bad):
    args = [[0], [5], [1], [-1]]
    args[which] = bad
    with pytest.raises(SproutError) as e:
        TreeBatch(*args)
    assert e.value.status == binding.SPR_ERR_INVALID_ARG


@pytest.mark.parametrize("kind", [list, tuple, lambda x: np.array(x, dtype=np.int64), lambda x: np.array(x, dtype=np.uint8), lambda x: np.array(x, dtype=np.float64),
                                  lambda x: torch.tensor(x), lambda x: np.array(x, dtype=object), lambda x: [[v] for v in x],
                                  lambda x: [torch.tensor(v) for v in x], lambda x: [float(v) for v in x], lambda x: [np.int64(v) for v in x]])
def test_whole_numbers_of_any_type_are_taken(kind):
    b = TreeBatch(kind([3, 1]), kind([70, 200]), kind([2, 1]), np.array([-1, 0, -1], dtype=np.int64))
    assert [b._c.slots[i] for i in (0, 1)] == [3, 1] and [b._c.lens[i] for i in (0, 1)] == [70, 200]
    assert [b._c.n_nodes[i] for i in (0, 1)] == [2, 1] and [b._c.parents[i] for i in range(3)] == [-1, 0, -1]


class FakeLibrary:
    """Counts the calls that reach the library."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


def host_ops():
    """TreeOps whose tensors are the host's (device index -1) and whose library only counts."""
    from paper_2403_12900_amd.tree import TreeOps
    o = TreeOps.__new__(TreeOps)
    o.lib, o.h, o.index, o.device, o._enter = FakeLibrary(), None, -1, torch.device("cpu"), lambda: None
    return o


def test_attention_refuses_tensors_that_want_gradients():
    """It has no backward pass: an output without one would stop the gradient in silence."""
    from paper_2403_12900_amd.tree import KVView
    k, v, table = torch.zeros(1, 2, 2, 1024), torch.zeros(1, 2, 2, 1024), torch.zeros(1, 2, dtype=torch.int32)
    b, q = TreeBatch([0], [4], [2], [-1, 0]), torch.zeros(2, 4, 64)
    o = host_ops()
    o.attention(KVView(k, v, table), 0, b, q)
    assert o.lib.calls == 1
    grad = lambda t: t.clone().requires_grad_()  # noqa: E731
    calls = [lambda: o.attention(KVView(k, v, table), 0, b, grad(q)), lambda: o.attention(KVView(grad(k), v, table), 0, b, q),
             lambda: o.attention(KVView(k, grad(v), table), 0, b, q), lambda: o.attention(KVView(k, v, table), 0, b, grad(q) * 2)]
    for call in calls:
        with pytest.raises(SproutError, match="gradient") as e:
            call()
        assert e.value.status == binding.SPR_ERR_INVALID_ARG and o.lib.calls == 1
    with torch.no_grad():
        for call in calls:
            call()
    o.attention(KVView(k, v, table), 0, b, grad(q).detach())
    assert o.lib.calls == 2 + len(calls)


def test_attention_refuses_tangents_and_outputs_that_want_gradients():
    from torch.autograd import forward_ad

    from paper_2403_12900_amd.tree import KVView
    k, table = torch.zeros(1, 2, 2, 1024), torch.zeros(1, 2, dtype=torch.int32)
    b, q, o = TreeBatch([0], [4], [2], [-1, 0]), torch.zeros(2, 4, 64), host_ops()
    with pytest.raises(SproutError, match="gradient"):
        o.attention(KVView(k, k, table), 0, b, q, out=q.clone().requires_grad_())
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t.clone(), torch.ones_like(t))  # noqa: E731
        for call in (lambda: o.attention(KVView(k, k, table), 0, b, dual(q)), lambda: o.attention(KVView(dual(k), k, table), 0, b, q),
                     lambda: o.attention(KVView(k, dual(k), table), 0, b, q), lambda: o.attention(KVView(k, k, table), 0, b, q, out=dual(q))):
            with pytest.raises(SproutError, match="tangent"):
                call()
        assert o.lib.calls == 0
        o.attention(KVView(k, k, table), 0, b, dual(q).detach())
    assert o.lib.calls == 1


def test_rows_that_overlap():
    """The rule that attention's q and out go by, against the sets of bytes themselves."""
    import ctypes
    from .test_abi_host import HOST_LIB
    L = ctypes.CDLL(HOST_LIB)
    L.sprh_rows_overlap.argtypes = [ctypes.c_uint64, ctypes.c_int64] * 2 + [ctypes.c_int64, ctypes.c_int]
    rng = np.random.default_rng(6)
    seen = [0, 0]
    for _ in range(4000):
        rows, width = int(rng.integers(1, 9)), int(rng.integers(1, 20))
        a, b = (int(x) for x in 1000 + rng.integers(0, 300, 2))
        sa, sb = (width + int(rng.choice([0, 1, width, 3 * width, 40])) for _ in range(2))
        if rng.random() < 0.5:
            sb = sa  # columns of one tensor
        cells = lambda at, s: {at + r * s + k for r in range(rows) for k in range(width)}  # noqa: E731
        want = bool(cells(a, sa) & cells(b, sb))
        assert bool(L.sprh_rows_overlap(a, sa, b, sb, width, rows)) == want, (a, sa, b, sb, width, rows)
        seen[want] += 1
    assert min(seen) > 500
    top = 1 << 40
    assert L.sprh_rows_overlap(1 << 47, 4 * top, (1 << 47) + 127 * 4 * top + 8, 4 * top, 16, 128)
    assert not L.sprh_rows_overlap(1 << 47, 4 * top, (1 << 47) + 127 * 4 * top + 16, 4 * top, 16, 128)


@pytest.mark.gpu
def test_attention_refuses_an_output_over_its_queries():
    from paper_2403_12900_amd.tree import KVView, TreeOps
    o = TreeOps()
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(1, 6, 2, 1024, device="cuda", generator=g) for _ in range(2))
    view = KVView(k, v, torch.arange(6, dtype=torch.int32, device="cuda").view(1, 6))
    b = TreeBatch([0], [80], [5], [-1, 0, 0, 1, 1])
    packed = torch.randn(7, 12, 64, device="cuda", generator=g)
    want = o.attention(view, 0, b, packed[:5, :4].contiguous())
    for q, out in ((packed[:5, :4], packed[:5, :4]), (packed[:5, :4], packed[:5, 3:7]), (packed[:5, :4], packed[1:6, 2:6]),
                   (packed[2:7, 4:8], packed[:5, 5:9])):
        before = packed.clone()
        with pytest.raises(SproutError, match="overlap") as e:
            o.attention(view, 0, b, q, out=out)
        assert e.value.status == binding.SPR_ERR_INVALID_ARG and torch.equal(packed, before)
    # Side by side in one tensor they do not.
    got = o.attention(view, 0, b, packed[:5, :4], out=packed[:5, 4:8])
    assert torch.equal(got, want) and torch.equal(packed[:5, 4:8], want)
    o.close()
