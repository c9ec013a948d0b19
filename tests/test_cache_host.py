"""Host side of the 4-bit cache's operators (no GPU): what a call's arguments must satisfy, the plans that launches are made
from, and the plain implementations that the GPU tests compare with.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2403_12900_amd import binding
from paper_2403_12900_amd.binding import SprCacheBatch, SprKv4View, SprPages, SprRotary, SproutError
from paper_2403_12900_amd.cache import CacheBatch, CacheOps, KV4View, Rotary
from paper_2403_12900_amd.tree import KVView

from . import cache_ref as ref
from .test_abi_host import HOST_LIB

I32 = ctypes.POINTER(ctypes.c_int32)
F64 = ctypes.c_double


def host():
    L = ctypes.CDLL(HOST_LIB)
    L.sprh_last_error.restype = ctypes.c_char_p
    L.sprh_cache_split.argtypes = [ctypes.c_void_p] + [ctypes.c_int] * 7 + [ctypes.c_size_t, ctypes.c_int, I32]
    L.sprh_rotary.argtypes = [ctypes.c_int] * 2 + [F64] * 6 + [ctypes.c_void_p, ctypes.c_int]
    return L


def a32(x):
    return np.ascontiguousarray(np.asarray(x, dtype=np.int32))


def p32(x):
    return None if x is None else x.ctypes.data_as(I32)


def raw_batch(n, slots, lens, rows):
    keep = [None if x is None else a32(x) for x in (slots, lens, rows)]
    b = SprCacheBatch(n, *(p32(x) for x in keep))
    b._keep = keep
    return b


def refused(L, status, what):
    assert status == binding.SPR_ERR_INVALID_ARG and what in L.sprh_last_error().decode()


# ------------------------------------------------------------------------------------------------ the plain forms


def test_quantisation_of_the_oracle():
    """Against the definition, number by number: no other value of the grid is nearer, ties go to the even code, no smaller
    scale holds the group."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 64)) * np.exp(rng.normal(0, 8, (200, 2))).repeat(32, 1)
    x[0] = 0
    x[1, :32], x[1, 32] = -0.0, 7 * 2.0 ** 3
    x[2, 0], x[2, 40] = np.nextafter(7.0, 8), 7.0
    x[3] = np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.9], 8)  # ties, at scale 1
    x[4, 3], x[4, 35] = np.inf, np.nan
    x[5], x[6] = 2.0 ** -140, 3.3e38
    codes, scales = ref.quantise(x)
    back = ref.values(codes, scales)
    for r in range(len(x)):
        for p in range(2):
            g, s = x[r, 32 * p:32 * p + 32], int(scales[r, p])
            if not np.isfinite(g).all():
                assert s == 255 and np.isnan(back[r, 32 * p:32 * p + 32]).all()
                continue
            top, e = np.abs(g).max(), s - 127
            assert -120 <= e <= 125 and (top <= 7 * 2.0 ** e or e == 125) and (e == -120 or top > 7 * 2.0 ** (e - 1))
            for j, v in enumerate(g):
                a, c = abs(v) / 2.0 ** e, int(codes[r, 32 * p + j])
                near = [k for k in range(8) if abs(ref.GRID[k] - a) == np.abs(ref.GRID - a).min()]
                assert (c & 7) in near and (len(near) == 1 or c % 2 == 0) and (c >> 3) == np.signbit(v)
                assert back[r, 32 * p + j] == math.copysign(ref.GRID[c & 7], v) * 2.0 ** e
    assert codes[3, :8].tolist() == [0, 2, 2, 4, 4, 6, 6, 7]


@pytest.mark.parametrize("hd", [64, 128])
def test_tiles_of_the_oracle(hd):
    """Every byte of a tile has one owner, and what is put comes back."""
    rng = np.random.default_rng(hd)
    ko, vo, kso, vso, khi, vhi = ref.offsets(hd)
    for at, high, lo in ((ko, khi, 0), (vo, vhi, 8 * hd)):
        assert sorted((2 * at + high).reshape(-1)) == list(range(2 * lo, 2 * lo + 16 * hd))
    assert sorted(set(kso.reshape(-1)) | set(vso.reshape(-1))) == list(range(16 * hd, 17 * hd))
    tile = rng.integers(0, 256, 17 * hd, dtype=np.uint8)
    x = rng.standard_normal((2, 16, hd))
    for t in rng.permutation(16):
        ref.put(tile, t, *ref.quantise(x[0, t]), *ref.quantise(x[1, t]))
    for got, want in zip(ref.get(tile), x):
        assert np.array_equal(got, ref.values(*ref.quantise(want)))


# ------------------------------------------------------------------------------------------------ what is refused


@pytest.mark.parametrize("n,slots,lens,rows,what", [
    (0, [0], [0], [1], "n must be"),
    (129, list(range(129)), [0] * 129, [1] * 129, "n must be"),
    (1, None, [0], [1], "null"),
    (1, [0], None, [1], "null"),
    (1, [0], [0], None, "null"),
    (1, [200], [0], [1], "slot id"),
    (1, [-1], [0], [1], "slot id"),
    (2, [4, 4], [0, 0], [1, 1], "twice"),
    (20, list(range(19)) + [3], [0] * 20, [1] * 20, "twice"),
    (1, [0], [-1], [1], "lens"),
    (1, [0], [2 ** 30 + 1], [1], "lens"),
    (1, [0], [2 ** 31 - 1], [1], "lens"),
    (1, [0], [0], [0], "rows must"),
    (1, [0], [0], [-4], "rows must"),
    (1, [0], [0], [2 ** 20 + 1], "SPR_MAX_CACHE_ROWS"),
    (3, [0, 1, 2], [0] * 3, [2 ** 19, 2 ** 19, 1], "SPR_MAX_CACHE_ROWS"),
    (1, [0], [1600], [1], "block-table row"),
    (1, [0], [1599], [2], "block-table row"),
    (1, [0], [0], [1601], "block-table row"),
])
def test_batches_that_are_refused(n, slots, lens, rows, what):
    L = host()
    b = raw_batch(n, slots, lens, rows)
    wide = 1 << 20 if what == "SPR_MAX_CACHE_ROWS" else 100
    refused(L, L.sprh_cache_parse(ctypes.byref(b), 200, wide, p32(np.zeros(130, np.int32))), what)
    refused(L, L.sprh_cache_parse(None, 200, 100, p32(np.zeros(130, np.int32))), "null")


def test_batches_that_are_taken():
    L = host()
    row0 = np.zeros(130, np.int32)
    b = raw_batch(128, np.arange(128)[::-1], [0] * 64 + [1584] * 64, [1600] * 64 + [16] * 64)
    assert L.sprh_cache_parse(ctypes.byref(b), 128, 100, p32(row0)) == 0
    assert row0[:129].tolist() == np.cumsum([0] + [1600] * 64 + [16] * 64).tolist()
    b = raw_batch(1, [0], [2 ** 30], [2 ** 20])
    assert L.sprh_cache_parse(ctypes.byref(b), 1, 2 ** 27, p32(row0)) == 0


def kv4(**k):
    d = dict(data=4096, n_layers=2, n_blocks=9, n_kv_heads=4, head_dim=64, block_table=4096, n_slots=3, max_blocks=5)
    d.update(k)
    return SprKv4View(*d.values())


@pytest.mark.parametrize("change,layer,what", [
    (dict(data=None), 0, "null"), (dict(block_table=None), 0, "null"), (dict(data=4104), 0, "16-byte"),
    (dict(block_table=4098), 0, "4-byte"), (dict(head_dim=96), 0, "head_dim"), (dict(head_dim=0), 0, "head_dim"),
    (dict(n_kv_heads=0), 0, "n_kv_heads"), (dict(n_kv_heads=513), 0, "n_kv_heads"), (dict(n_layers=0), 0, "n_layers"),
    (dict(n_blocks=-1), 0, "n_blocks"), (dict(n_slots=0), 0, "n_slots"), (dict(max_blocks=0), 0, "max_blocks"),
    (dict(), 2, "layer must"), (dict(), -1, "layer must")])
def test_views_that_are_refused(change, layer, what):
    L = host()
    assert L.sprh_kv4_view(ctypes.byref(kv4()), 1) == 0
    refused(L, L.sprh_kv4_view(ctypes.byref(kv4(**change)), layer), what)


@pytest.mark.parametrize("args,head_dim,what", [
    ((1, 0, 1e4, 1, 0, 0, 0, 1), 64, "dims"), ((0, 0, 1e4, 1, 0, 0, 0, 1), 64, "dims"), ((130, 0, 1e4, 1, 0, 0, 0, 1), 128, "dims"),
    ((66, 0, 1e4, 1, 0, 0, 0, 1), 64, "dims"), ((64, 2, 1e4, 1, 0, 0, 0, 1), 64, "pairs"), ((64, 0, 0.0, 1, 0, 0, 0, 1), 64, "base"),
    ((64, 0, math.inf, 1, 0, 0, 0, 1), 64, "base"), ((64, 0, math.nan, 1, 0, 0, 0, 1), 64, "base"),
    ((64, 0, 5e-324, 1, 0, 0, 0, 1), 64, "frequency"), ((64, 0, 1e4, 0.5, 0, 0, 0, 1), 64, "factor"),
    ((64, 0, 1e4, math.nan, 8192, 1, 32, 1), 64, "factor"), ((64, 0, 1e4, 2, 0, 1, 32, 1), 64, "original"),
    ((64, 0, 1e4, 2, 8192, 4, 4, 1), 64, "high above low"), ((64, 0, 1e4, 2, 8192, 1, math.inf, 1), 64, "finite"),
    ((64, 0, 1e4, 1, 0, 0, 0, math.nan), 64, "amplitude")])
def test_rotaries_that_are_refused(args, head_dim, what):
    L = host()
    r = SprRotary()
    refused(L, L.sprh_rotary(*args, ctypes.byref(r), head_dim), what)  # (5e-324 = 2^-1074, to the power of -62 / 64: 2^1040)


@pytest.mark.parametrize("field,value,what", [("dims", 3, "dims"), ("dims", 128, "dims"), ("pairs", 7, "pairs"),
                                              ("amplitude", math.inf, "amplitude"), ("turns", math.nan, "frequencies")])
def test_rotaries_that_were_filled_in_badly(field, value, what):
    L = host()
    r = SprRotary()
    assert L.sprh_rotary(32, 0, 1e4, 1, 0, 0, 0, 1, ctypes.byref(r), 64) == 0
    if field == "turns":
        r.turns[7] = value
    else:
        setattr(r, field, value)
    refused(L, L.sprh_rotary_check(ctypes.byref(r), 64), what)


def test_frequencies():
    L = host()
    r = SprRotary()
    for dims, base, factor, original, low, high in ((128, 1e4, 1, 0, 0, 0), (46, 5e5, 8, 8192, 1, 32), (2, 1e4, 4, 100, 1, 2)):
        assert L.sprh_rotary(dims, 1, base, factor, original, low, high, 1.25, ctypes.byref(r), 128) == 0
        assert (r.dims, r.pairs, r.amplitude) == (dims, 1, 1.25)
        for k in range(64):
            w = base ** (-2 * k / dims) if k < dims // 2 else 0.0
            if factor > 1 and w:
                keep = min(1, max(0, (original * w / (2 * math.pi) - low) / (high - low)))
                w = w * (keep + (1 - keep) / factor)
            assert abs(r.turns[k] * 2 * math.pi - w) <= 8 * 2.0 ** -52 * w  # pow, four products, two sums


def pages(**k):
    d = dict(k=4096, v=None, block_bytes=1088, n_layers=2, n_blocks=40, block_table=4096, n_slots=8, max_blocks=5)
    d.update(k)
    return SprPages(*d.values())


@pytest.mark.parametrize("change,what", [
    (dict(k=None), "null"), (dict(block_table=None), "null"), (dict(k=4097), "16-byte"), (dict(v=4104), "16-byte"),
    (dict(block_table=4097), "4-byte"), (dict(block_bytes=0), "block_bytes"), (dict(block_bytes=1096), "block_bytes"),
    (dict(block_bytes=2 ** 31), "block_bytes"), (dict(n_layers=0), "n_layers"), (dict(n_blocks=0), "n_blocks"),
    (dict(n_slots=0), "n_slots"), (dict(max_blocks=0), "max_blocks")])
def test_pages_that_are_refused(change, what):
    L = host()
    a, out = a32([0]), np.zeros(99, np.int32)
    p = pages(**change)
    refused(L, L.sprh_fork(ctypes.byref(p), 1, p32(a), p32(a32([1])), p32(a32([5])), p32(a), p32(out)), what)
    refused(L, L.sprh_move(ctypes.byref(p), 1, p32(a), p32(a32([1])), p32(out)), what)
    refused(L, L.sprh_move(None, 1, p32(a), p32(a32([1])), p32(out)), "null")


@pytest.mark.parametrize("n,source,target,lens,fresh,what", [
    (0, [0], [1], [5], [9], "n must"), (129, [0] * 129, [1] * 129, [5] * 129, [9] * 129, "n must"),
    (1, None, [1], [5], [9], "null"), (1, [0], None, [5], [9], "null"), (1, [0], [1], None, [9], "null"),
    (1, [0], [1], [5], None, "null"), (1, [8], [1], [5], [9], "slot id"), (1, [-1], [1], [5], [9], "slot id"),
    (1, [0], [8], [5], [9], "slot id"), (1, [0], [1], [-1], [9], "lens"), (1, [0], [1], [81], [9], "lens"),
    (1, [0], [1], [5], [40], "fresh"), (1, [0], [1], [5], [-1], "fresh"), (2, [0, 0], [1, 1], [5, 5], [9, 8], "target"),
    (2, [0, 0], [1, 2], [5, 5], [9, 9], "fresh"), (1, [1], [1], [5], [9], "also a source"),
    (2, [0, 1], [1, 2], [5, 5], [9, 8], "also a source")])
def test_forks_that_are_refused(n, source, target, lens, fresh, what):
    L = host()
    a = [None if x is None else a32(x) for x in (source, target, lens, fresh)]
    p = pages()
    refused(L, L.sprh_fork(ctypes.byref(p), n, *(p32(x) for x in a), p32(np.zeros(999, np.int32))), what)


def test_forks_of_one_block_are_grouped():
    rng = np.random.default_rng(4)
    L = host()
    for _ in range(300):
        n, slots = int(rng.integers(1, 129)), 300
        targets = rng.permutation(slots - 6)[:n]
        a = [a32(slots - 6 + rng.integers(0, 6, n)), a32(targets), a32(rng.choice([0, 5, 15, 16, 17, 31, 32, 80], n)), a32(rng.permutation(400)[:n])]
        p = pages(n_slots=slots, n_blocks=400)
        out = np.zeros(1 + 4 * n + 130, np.int32)
        assert L.sprh_fork(ctypes.byref(p), n, *(p32(x) for x in a), p32(out)) == 0
        groups, body = out[0], out[1:1 + 4 * n].reshape(4, n)
        first = out[1 + 4 * n:2 + 4 * n + groups]
        want = {(int(s), int(t), int(x), int(f) if x % 16 else -1) for s, t, x, f in zip(*a)}
        assert {tuple(int(v) for v in c) for c in body.T} == want
        assert first[0] == 0 and first[groups] == sum(1 for x in a[2] if x % 16) and (np.diff(first) > 0).all()
        keys = []
        for i in range(groups):
            ks = {(int(s), int(x) // 16) for s, x in zip(body[0, first[i]:first[i + 1]], body[2, first[i]:first[i + 1]])}
            assert len(ks) == 1
            keys += ks
        assert len(set(keys)) == groups


@pytest.mark.parametrize("both", [False, True])
def test_work_groups_of_a_launch_are_limited(both):
    """The largest calls that the header allows, and the next ones: a fork's pieces of 4 KiB, a move's of 16 and its table."""
    L, most = host(), 2 ** 24 - 1
    out, v = np.zeros(2000, np.int32), 8192 if both else None
    fork = lambda p, n, lens: L.sprh_fork(ctypes.byref(p), n, p32(a32([0] * n)), p32(a32(range(1, n + 1))), p32(a32(lens)), p32(a32(range(n))), p32(out))  # noqa: E731
    move = lambda p, n: L.sprh_move(ctypes.byref(p), n, p32(a32(range(n))), p32(a32(range(n, 2 * n))), p32(out))  # noqa: E731
    pools = 2 if both else 1
    for size, pieces in ((4096, 1), (4112, 2), (1088, 1), (2 ** 30, 2 ** 18)):
        layers = (most - 1) // (pools * pieces)  # beside the one table row
        assert fork(pages(v=v, block_bytes=size, n_layers=layers), 1, [5]) == 0
        assert fork(pages(v=v, block_bytes=size, n_layers=layers + 1), 1, [16]) == 0  # nothing to copy
        refused(L, fork(pages(v=v, block_bytes=size, n_layers=layers + 1), 1, [5]), "too large")
    layers = (most - 3) // (2 * pools)
    assert fork(pages(v=v, block_bytes=4096, n_layers=layers), 3, [5, 6, 17]) == 0  # three forks of two blocks
    refused(L, fork(pages(v=v, block_bytes=4096, n_layers=layers + 1), 3, [5, 6, 17]), "too large")
    for size, pieces in ((16384, 1), (16400, 2), (1088, 1), (2 ** 30, 2 ** 16)):
        layers = (most - 1) // (pools * pieces)  # beside the table of 40 entries
        assert move(pages(v=v, block_bytes=size, n_layers=layers), 1) == 0
        refused(L, move(pages(v=v, block_bytes=size, n_layers=layers + 1), 1), "too large")
    layers = (most - 1) // (384 * pools)
    assert move(pages(v=v, block_bytes=1024, n_layers=layers, n_blocks=2000), 900) == 0
    refused(L, move(pages(v=v, block_bytes=1024, n_layers=layers + 1, n_blocks=2000), 900), "too large")
    assert move(pages(v=v, n_slots=1024, max_blocks=most - 2 * pools), 1) == 0
    refused(L, move(pages(v=v, n_slots=1024, max_blocks=most - 2 * pools + 1), 1), "too large")


@pytest.mark.parametrize("n,src,dst,what", [
    (0, [0], [1], "n must"), (41, list(range(41)), [0] * 41, "n must"), (1, None, [1], "null"), (1, [0], None, "null"),
    (1, [40], [1], "out of range"), (1, [-1], [1], "out of range"), (1, [0], [40], "out of range"), (1, [0], [-7], "out of range"),
    (2, [3, 3], [1, 2], "src listed"), (2, [3, 4], [1, 1], "dst listed"), (1, [3], [3], "also a src"), (2, [3, 4], [4, 5], "also a src")])
def test_moves_that_are_refused(n, src, dst, what):
    L = host()
    a = [None if x is None else a32(x) for x in (src, dst)]
    p = pages()
    refused(L, L.sprh_move(ctypes.byref(p), n, *(p32(x) for x in a), p32(np.zeros(999, np.int32))), what)


def test_moves_are_sorted():
    L = host()
    out = np.zeros(6, np.int32)
    p = pages()
    assert L.sprh_move(ctypes.byref(p), 3, p32(a32([30, 7, 12])), p32(a32([1, 2, 0])), p32(out)) == 0
    assert out.tolist() == [7, 12, 30, 2, 0, 1]


def test_work_items_of_an_attention_launch():
    """Items cover every column group's blocks, stay inside the workspace, and one item is one split where nothing is split."""
    rng = np.random.default_rng(5)
    L = host()
    for trial in range(400):
        n = int(rng.integers(1, 129))
        lens = np.minimum(np.exp(rng.uniform(0, 13 if trial % 9 == 0 else 8, n)), 2 ** 20).astype(np.int32) - 1
        rows = np.ones(n, np.int32) if trial % 3 else np.exp(rng.uniform(0, 8, n)).astype(np.int32)
        G, Hkv, hd = int(rng.integers(1, 17)), int(rng.choice([1, 4, 8, 40, 512])), int(rng.choice([64, 128]))
        n_cu, least, slots, floats, counters = 256, int(rng.choice([2, 8])), int(rng.choice([256, 768, 1024])), 1 << 23, 65536
        b = raw_batch(n, np.arange(n), lens, rows)
        out = np.zeros(5 + 4 * n, np.int32)
        assert L.sprh_cache_split(ctypes.byref(b), G, Hkv, hd, n_cu, 128, least, slots, floats, counters, p32(out)) == 0
        cw, bps, groups, split = (int(x) for x in out[:4])
        item0, order, ncg, cg0 = out[4:5 + n], out[5 + n:5 + 2 * n], out[5 + 2 * n:5 + 3 * n], out[5 + 3 * n:]
        cols, every = int(rows.max()) * G, int(rows.sum()) * G * Hkv
        assert cw == (16 if cols <= 16 else 32 if cols <= 32 or every <= 64 * n_cu else 64 if cols <= 64 or every <= 128 * n_cu else 128)
        assert sorted(order) == list(range(n)) and bps % least == 0 and item0[0] == 0
        blocks = (lens.astype(np.int64) + rows + 15) // 16
        assert (np.diff(blocks[order]) <= 0).all()
        assert ncg.tolist() == [-(-int(rows[i]) * G // cw) for i in order] and groups == ncg.sum()
        assert cg0.tolist() == (np.cumsum(ncg) - ncg).tolist()
        ns = -(-blocks[order] // bps)
        assert np.diff(item0).tolist() == (ns * ncg).tolist() and split == int(ns.max() > 1)
        if split:
            assert ns.max() <= 64 and int(item0[-1]) * Hkv * cw * (hd + 4) <= floats and groups * Hkv <= counters


def test_masks_of_code_and_scale_bytes():
    """Position by position.  Values are not exact in fp16 where a position's scale is out of 2^-18 .. 2^13 and one of its two
    codes is not zero, or where it is NaN: a position of zeros (scale 2^-120) beside others is."""
    rng = np.random.default_rng(11)
    L, n = host(), 200000
    scales = rng.choice([0, 7, 108, 109, 110, 127, 140, 141, 252, 255], (n, 4), p=[.05, .2, .05, .1, .1, .1, .1, .1, .1, .1]).astype(np.uint8)
    scales[:n // 4] = rng.integers(0, 256, (n // 4, 4))
    scales[-n // 4:][rng.random((n // 4, 4)) < 0.8] = 120
    words = rng.choice([0x00, 0x80, 0x08, 0x88, 0x01, 0x10, 0x7F, 0xF7, 0x40], (n, 4)).astype(np.uint8)
    words[scales == 7] &= 0x88
    bits = rng.integers(0, 16, n).astype(np.uint32)
    out = np.zeros((n, 4), np.uint32)
    u = lambda a: ctypes.c_void_p(np.ascontiguousarray(a).ctypes.data)  # noqa: E731
    w, s = (np.ascontiguousarray(x).view("<u4").reshape(-1) for x in (words, scales))
    L.sprh_cache_bits(u(w), u(s), u(bits), u(out), n)
    assert np.array_equal(out[:, 0], ((bits[:, None] >> np.arange(4) & 1) * 255 << 8 * np.arange(4)).sum(1))
    assert np.array_equal(out[:, 1], ((scales == 255) << np.arange(4)).sum(1))
    odd = (scales < 109) | (scales > 140)
    assert np.array_equal(out[:, 2] != 0, odd.any(1))
    assert np.array_equal(out[:, 3] != 0, (odd & (words & 0x77 != 0) | (scales == 255)).any(1))
    zero = (scales == 7).any(1) & ~(odd & (scales != 7)).any(1)
    assert zero.sum() > 1000 and not out[zero, 3].any()


# ------------------------------------------------------------------------------------------------ the Python surface


class FakeLibrary:
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


def host_ops():
    """CacheOps whose tensors are the host's (device index -1) and whose library only counts."""
    o = CacheOps.__new__(CacheOps)
    o.lib, o.h, o.index, o.device, o._enter = FakeLibrary(), None, -1, torch.device("cpu"), lambda: None
    return o


def cpu_view(Hkv=2, hd=64):
    return KV4View(torch.zeros(1, 4, Hkv, 17 * hd, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32))


@pytest.mark.parametrize("which", range(3))
@pytest.mark.parametrize("bad", [[2 ** 40], [1.5], [float("nan")], ["1"], [None]])
def test_numbers_that_are_no_int32_are_refused(which, bad):
    args = [[0], [5], [1]]
    args[which] = bad
    with pytest.raises(SproutError, match="cache batch"):
        CacheBatch(*args)
    for call, n in ((host_ops().fork, 4), (host_ops().move, 2)):
        with pytest.raises(SproutError, match="32 bits"):
            call(cpu_view(), *([0], bad, [0], [0])[:n])


def test_batches_of_unequal_lengths_are_refused():
    for args in (([0, 1], [5], [1]), ([0], [5, 6], [1]), ([0], [5], [1, 1])):
        with pytest.raises(SproutError, match="one length"):
            CacheBatch(*args)
    o = host_ops()
    with pytest.raises(SproutError, match="one length"):
        o.fork(cpu_view(), [0, 0], [1], [5], [2])
    with pytest.raises(SproutError, match="one length"):
        o.move(cpu_view(), [0], [1, 2])
    assert o.lib.calls == 0


def test_a_batch_keeps_its_own_copy():
    lens = np.array([5], dtype=np.int32)
    b = CacheBatch([0], lens, [3])
    lens[0] = 99
    assert b._c.lens[0] == 5 and b.rows == 3


@pytest.mark.parametrize("make", [
    lambda: KV4View(torch.zeros(1, 4, 2, 17 * 64), torch.zeros(2, 2, dtype=torch.int32)),
    lambda: KV4View(torch.zeros(4, 2, 17 * 64, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32)),
    lambda: KV4View(torch.zeros(1, 4, 2, 16 * 64, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.int32)),
    lambda: KV4View(torch.zeros(1, 4, 2, 17 * 64, dtype=torch.uint8), torch.zeros(2, 2)),
    lambda: KV4View(torch.zeros(1, 4, 2, 17 * 64, dtype=torch.uint8), torch.zeros(2, dtype=torch.int32)),
    lambda: KV4View(torch.zeros(1, 4, 17 * 64, 2, dtype=torch.uint8).transpose(2, 3), torch.zeros(2, 2, dtype=torch.int32)),
    lambda: KV4View(torch.zeros(1, 4, 2, 17 * 64, dtype=torch.uint8), torch.zeros(2, 4, dtype=torch.int32)[:, ::2])])
def test_malformed_views_are_refused(make):
    with pytest.raises(SproutError, match="kv4 view"):
        make()


def test_tensors_that_do_not_fit_are_refused():
    o, b, v = host_ops(), CacheBatch([0], [5], [3]), cpu_view()
    r = Rotary(64)
    t = torch.zeros(3, 4, 64)
    k = torch.zeros(3, 2, 64)
    pos = torch.zeros(3, dtype=torch.int32)
    o.attention(v, 0, b, t), o.append(v, 0, b, k, k), o.rotary(r, t, pos), o.read(v, 0, b)
    assert o.lib.calls == 4
    grad = lambda x: x.clone().requires_grad_()  # noqa: E731
    wide = torch.zeros(3, 64, 4).transpose(1, 2)
    for call, what in [
            (lambda: o.attention(v, 0, b, t[:2]), "q must"), (lambda: o.attention(v, 0, b, t.double()), "q must"),
            (lambda: o.attention(v, 0, b, torch.zeros(3, 4, 128)), "q must"), (lambda: o.attention(v, 0, b, wide), "contiguous rows"),
            (lambda: o.attention(v, 0, b, t, out=t.bfloat16()), "out must"), (lambda: o.attention(v, 0, b, t, out=t[:, :2]), "out must"),
            (lambda: o.attention(v, 0, b, grad(t)), "gradient"), (lambda: o.append(v, 0, b, k[:2], k), "k and v"),
            (lambda: o.append(v, 0, b, k, k.bfloat16()), "k and v"), (lambda: o.append(v, 0, b, k.half(), k.half()), "k and v"),
            (lambda: o.append(v, 0, b, torch.zeros(3, 64, 2).transpose(1, 2), k), "contiguous rows"),
            (lambda: o.append(v, 0, b, k, grad(k)), "gradient"), (lambda: o.read(v, 0, b, torch.float16), "dtype"),
            (lambda: o.rotary(r, t[0], pos), "x must"), (lambda: o.rotary(r, t, pos.long()), "positions"),
            (lambda: o.rotary(r, t, pos[:2]), "positions"), (lambda: o.rotary(r, grad(t), pos), "gradient"),
            (lambda: o.rotary(r, t, torch.zeros(6, dtype=torch.int32)[::2]), "positions")]:
        with pytest.raises(SproutError, match=what):
            call()
    o.index = 0  # a handle on another device than the tensors'
    for call in (lambda: o.attention(v, 0, b, t), lambda: o.append(v, 0, b, k, k), lambda: o.read(v, 0, b),
                 lambda: o.fork(v, [0], [1], [5], [2]), lambda: o.move(v, [0], [1]), lambda: o.rotary(r, t, pos)):
        with pytest.raises(SproutError, match="must be"):
            call()
    assert o.lib.calls == 4


def test_tensors_that_autograd_follows_are_refused():
    """None of the operators has a derivative: tangents of its inputs, and gradients of what it writes to, would be lost in
    silence."""
    import torch.autograd.forward_ad as fw
    o, b, v, r = host_ops(), CacheBatch([0], [5], [3]), cpu_view(), Rotary(64)
    q, k, pos = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32)
    pool, table = torch.zeros(1, 4, 2, 1024), torch.zeros(2, 2, dtype=torch.int32)
    lists = ([0], [1], [5], [2])
    over = [(lambda x: o.attention(v, 0, b, x), q), (lambda x: o.attention(v, 0, b, q, out=x), q), (lambda x: o.rotary(r, x, pos), q),
            (lambda x: o.rotary(r, q, pos, out=x), q), (lambda x: o.append(v, 0, b, x, k), k), (lambda x: o.append(v, 0, b, k, x), k),
            (lambda x: o.fork(KVView(x, pool, table), *lists), pool), (lambda x: o.fork(KVView(pool, x, table), *lists), pool),
            (lambda x: o.move(KVView(x, pool, table), [0], [1]), pool), (lambda x: o.move(KVView(pool, x, table), [0], [1]), pool)]
    for i, (call, x) in enumerate(over):
        calls = o.lib.calls
        leaf = x.clone().requires_grad_()
        with pytest.raises(SproutError, match="gradient") as e:
            call(leaf)
        assert e.value.status == binding.SPR_ERR_INVALID_ARG
        with pytest.raises(SproutError, match="gradient"):
            call(leaf * 2)
        with fw.dual_level():
            dual = fw.make_dual(x.clone(), torch.ones_like(x))
            for t in (dual, dual * 2):
                with pytest.raises(SproutError, match="tangent"):
                    call(t)
            assert o.lib.calls == calls
            call(dual.detach()), call(x)
        with torch.no_grad():
            call(leaf)
        assert o.lib.calls == calls + 3
    with pytest.raises(Exception):
        torch.func.jvp(lambda x: o.rotary(r, x, pos), (q,), (torch.ones_like(q),))


def test_any_paged_cache_can_be_forked_and_moved():
    o = host_ops()
    table = torch.zeros(2, 2, dtype=torch.int32)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.zeros(3, 4, 2, 16 * 64, dtype=dtype)
        p = o._pages("x", KVView(x, x.clone(), table))._obj
        assert (p.block_bytes, p.n_layers, p.n_blocks, p.n_slots, p.max_blocks) == (2 * 1024 * x.element_size(), 3, 4, 2, 2) and p.v
    p = o._pages("x", cpu_view(Hkv=3, hd=128))._obj
    assert (p.block_bytes, p.v) == (3 * 17 * 128, None)


def test_a_rotary_that_is_refused():
    for args in (dict(dims=63), dict(dims=64, layout="whole"), dict(dims=64, factor=0.5), dict(dims=64, factor=2.0)):
        with pytest.raises(SproutError) as e:
            Rotary(**args)
        assert e.value.status == binding.SPR_ERR_INVALID_ARG


def test_null_handles_are_refused():
    lib = binding.load_library()
    for name, n in (("spr_cache_ops_set_stream", 1), ("spr_cache_ops_release", 0)):
        assert getattr(lib, name)(None, *[None] * n) == binding.SPR_ERR_INVALID_ARG
    assert lib.spr_cache_read(None, None, 0, None, 0, None, 0, None, 0) == binding.SPR_ERR_INVALID_ARG
    assert lib.spr_cache_move(None, None, 0, None, None) == binding.SPR_ERR_INVALID_ARG
    h = ctypes.c_void_p()
    assert lib.spr_cache_ops_init(None, 0, None, ctypes.byref(h)) == binding.SPR_ERR_WORKSPACE
    assert lib.spr_cache_ops_init(4096, 64, None, ctypes.byref(h)) == binding.SPR_ERR_WORKSPACE
    assert b"cache_ops_init" in lib.spr_last_error()
