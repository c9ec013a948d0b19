"""The verification kernels' fp64 exponential, compiled for the host (no GPU).

Bound: the polynomial's rest is 2.4e-16 of the result, the roundings of r (two, of 2^-55 each), of the last products
(2^-53 of at most 1.42, then |r| <= 0.35 times as much each) and their ratio to the smallest e^r = 0.707 add up to 3e-16:
below 2^-50 = 8.9e-16.
"""
import ctypes

import numpy as np

from .test_abi_host import HOST_LIB

F64 = ctypes.POINTER(ctypes.c_double)


def exp_neg(x):
    x = np.ascontiguousarray(x, dtype=np.float64)
    y = np.empty_like(x)
    L = ctypes.CDLL(HOST_LIB)
    L.sprh_exp_neg(x.ctypes.data_as(F64), y.ctypes.data_as(F64), ctypes.c_int(len(x)))
    return y


def test_error_is_below_its_bound():
    rng = np.random.default_rng(1)
    n = np.arange(1021)
    x = np.concatenate([-rng.uniform(0, 708, 200000), -rng.uniform(0, 40, 200000), -rng.uniform(0, 0.35, 100000),
                        -(2.0 ** -rng.uniform(0, 60, 10000)),
                        np.ravel([-(n + 0.5 + d) * np.log(2) for d in (-1e-3, -1e-9, 0, 1e-9, 1e-3)])])
    x = x[x >= -708]
    want = np.exp(x.astype(np.longdouble))  # 64 bits of mantissa
    worst = float((np.abs(exp_neg(x).astype(np.longdouble) - want) / want).max())
    assert worst < 2.0 ** -50, worst


def test_ends():
    assert exp_neg([0.0, -0.0]).tolist() == [1.0, 1.0]
    assert exp_neg([-709.0, -1e4, -1e300, -np.inf]).tolist() == [0.0] * 4
    assert exp_neg([-708.0])[0] > 0
