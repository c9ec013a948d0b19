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
                                  lambda x: torch.tensor(x), lambda x: [np.int64(v) for v in x]])
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
