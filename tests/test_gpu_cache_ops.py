"""The 4-bit cache's operators against plain 64-bit implementations (needs an MI355X).

What is stored is exact: codes and scales are compared byte by byte with the oracle's.  A turned key is first computed in 64
bits on either side; the sides differ by a few 2^-53 of it, and no input here lies so near a border of two codes.

Tolerances of the rest, derived (eps = 2^-24, half a step of fp32; half a step of bf16 is 2^-8):
  * rotary: angles, sines and products are held in 64 bits (the angle's product rounds at 2^-53 of it, 2^-32 of a radian at
    2^21 radians), so that an output is off by its one rounding, half a step of the output, and by 2^-30 of the pair's length;
  * attention, for inputs of unit variance:
    - stored values and their products with queries are exact in the kernel's parts; a score is a sum whose roundings
      of random sign add up to less than 4 sqrt(hd) eps |q| |k|, which the scale 1 / sqrt(hd) takes to ds = 4 eps |q| |k|;
      a change of at most ds in every score changes the weighted mean of v by at most 2 ds max|v|;
    - exp2 (1 ulp, and its argument's rounding: |s log2 e| <= 2^5 here, 2^5 eps ln 2 < 24 eps), the sums over T positions
      (4 sqrt(T) eps, on numerator and denominator) and the merges add (26 + 8 sqrt(T)) eps max|v|;
    - fp32 outputs: probabilities enter their product, and their sum, to 2^-22 of themselves, which moves the mean by at most
      2^-22 of the mean distance of v from it, no more than max|v|;
    - bf16 outputs: they enter it to 2^-11 of themselves (2 * 2^-12 below), and the output's own rounding is 2^-8 of it;
    - small probabilities are off by 2^-36 (fp32) or 2^-32 (bf16) of the largest: all T of them below the sums' 8 sqrt(T) eps.
"""
import ctypes

import numpy as np
import pytest
import torch

from paper_2403_12900_amd import binding
from paper_2403_12900_amd.binding import SproutError
from paper_2403_12900_amd.cache import CacheBatch, CacheOps, KV4View, Rotary
from paper_2403_12900_amd.tree import KVView

from . import cache_ref as ref
from ._harness import say

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    o = CacheOps()
    yield o
    o.close()


def rounded(x, dtype):
    """x as the device gets it, and its value in 64 bits."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(dtype)
    return t.cuda(), t.double().numpy()


def columns(t, before=1, behind=2):
    """The same values as columns of a wider tensor, other values around them."""
    wide = torch.full((t.shape[0], t.shape[1] + before + behind, t.shape[2]), 7.0, dtype=t.dtype, device=t.device)
    wide[:, before:before + t.shape[1]] = t
    return wide[:, before:before + t.shape[1]]


# ------------------------------------------------------------------------------------------------ rotary


def check_rotary(ops, rng, H, hd, dims, layout, io, positions, scaling=None, strided=False, in_place=False):
    scaling = scaling or {}
    say(f"rotary: H {H} hd {hd} dims {dims} {layout} {io} rows {len(positions)} {scaling} strided {strided} in place {in_place}")
    x, want = rounded(rng.standard_normal((len(positions), H, hd)), io)
    exact = ref.turn(want, positions, dims, layout, **scaling)
    if strided:
        x = columns(x)
    pos = torch.from_numpy(np.asarray(positions, dtype=np.int32)).cuda()
    before = x.clone()
    out = ops.rotary(Rotary(dims, layout=layout, **scaling), x, pos, out=x if in_place else None)
    torch.cuda.synchronize()
    assert (out.data_ptr() == x.data_ptr()) == in_place and (in_place or torch.equal(x, before))
    got = out.double().cpu().numpy()
    half = EPS if io == F32 else 2.0 ** -8
    pair = np.abs(want).max() * 1.5 * abs(scaling.get("amplitude", 1.0))
    assert (np.abs(got - exact) <= half * np.abs(exact) + 2.0 ** -30 * pair).all(), np.abs(got - exact).max()
    assert np.array_equal(got[..., dims:], want[..., dims:])


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("hd,dims", [(64, 64), (128, 128), (64, 2), (128, 2), (64, 46), (128, 126), (128, 32), (64, 24), (128, 90)])
def test_rotary_layouts_and_parts(ops, hd, dims, layout, io):
    rng = np.random.default_rng(hd + dims)
    for H, positions in ((1, [0]), (3, [0, 1, 17, 4095]), (33, rng.integers(0, 10000, 5))):
        check_rotary(ops, rng, H, hd, dims, layout, io, positions)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rotary_far_positions_and_long_contexts(ops, layout):
    rng = np.random.default_rng(9)
    positions = np.concatenate([rng.integers(0, 2 ** 21, 40), [2 ** 21, 0, 1], -rng.integers(1, 5000, 5)])
    for scaling in (None, dict(base=500000.0, factor=8.0, original=8192, low=1.0, high=4.0, amplitude=1.2),
                    dict(base=10000.0, factor=32.0, original=64, low=1.0, high=32.0, amplitude=-0.5)):
        for hd, dims in ((128, 128), (64, 40)):
            check_rotary(ops, rng, 5, hd, dims, layout, F32, positions, scaling)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rotary_positions_of_31_bits(ops, layout):
    """The angle is off by its stored frequency's and its product's roundings, (8 * 2^-52 + 2^-53) of it, which turns a pair
    by as much; then the output rounds once."""
    rng = np.random.default_rng(13)
    positions = np.concatenate([[2 ** 31 - 1, -2 ** 31, 10 ** 9, 2 ** 30], rng.integers(2 ** 21, 2 ** 31, 20)])
    for hd, dims, scaling in ((128, 128, {}), (64, 40, dict(base=500000.0, factor=8.0, original=8192, low=1.0, high=4.0))):
        x, want = rounded(rng.standard_normal((len(positions), 3, hd)), F32)
        exact = ref.turn(want, positions, dims, layout, **scaling)
        got = ops.rotary(Rotary(dims, layout=layout, **scaling), x, torch.from_numpy(positions.astype(np.int32)).cuda())
        angle = np.abs(positions)[:, None, None] * 17 * 2.0 ** -53  # (the quickest frequency is 1)
        assert (np.abs(got.double().cpu().numpy() - exact) <= EPS * np.abs(exact) + angle * 1.5 * np.abs(want).max()).all()


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("hd,dims", [(64, 64), (128, 90), (128, 128), (64, 6)])
def test_rotary_strides_and_in_place(ops, hd, dims, io):
    rng = np.random.default_rng(3)
    for layout in ("half", "pairs"):
        for strided, in_place in ((True, False), (False, True), (True, True)):
            check_rotary(ops, rng, 21, hd, dims, layout, io, rng.integers(0, 5000, 37), strided=strided, in_place=in_place)


def nearest_bf16(z):
    """z in 64 bits (normal bf16 numbers), rounded once to bf16, and whether it is not too near a border of two to tell."""
    u = np.ascontiguousarray(z).view(np.int64)
    step, low = 1 << 45, u & ((1 << 45) - 1)
    up = (u + (step // 2 - 1) + (u >> 45 & 1)) & ~np.int64(step - 1)
    return up.view(np.float64), np.abs(low - step // 2) > 1 << 16  # (2^-36 of z)


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("hd,dims", [(64, 64), (128, 128), (64, 46)])
def test_rotary_rounds_bf16_once(ops, hd, dims, layout):
    """Results that lie 2^-40 of themselves beside the middle of two bf16 numbers (fp32 would put them onto it), and so many
    others that some dozen of them do by chance."""
    rng = np.random.default_rng(hd + dims)
    x, want = rounded(rng.choice([-1, 1], (5, 3, hd)) * 2.0 ** rng.integers(-60, 60, (5, 3, hd)), BF16)
    at0 = torch.zeros(5, dtype=torch.int32, device="cuda")
    for odd in (1, 3):  # 1 + odd / 256: a tie, which goes down, and up
        for beside in (-1, 0, 1):
            got = ops.rotary(Rotary(dims, layout=layout, amplitude=1 + odd / 256 + beside * 2.0 ** -40), x, at0).double().cpu().numpy()
            to = 1 + (odd + (beside if beside else 1 if odd == 3 else -1)) / 256
            assert np.array_equal(got[..., :dims], to * want[..., :dims]), (odd, beside)
    rows = 2000
    x, want = rounded(rng.standard_normal((rows, 8, hd)), BF16)
    positions = rng.integers(0, 5000, rows)
    got = ops.rotary(Rotary(dims, layout=layout), x, torch.from_numpy(positions.astype(np.int32)).cuda()).double().cpu().numpy()
    to, sure = nearest_bf16(ref.turn(want, positions, dims, layout))
    sure[..., dims:] = True
    assert sure.mean() > 0.999 and np.array_equal(got[sure], to[sure]), (got != to)[sure].sum()


def test_rotary_of_many_rows_and_heads(ops):
    rng = np.random.default_rng(4)
    check_rotary(ops, rng, 64, 64, 64, "half", BF16, np.arange(700) + 5)
    check_rotary(ops, rng, 300, 128, 128, "pairs", F32, [3, 70000])


def test_rotary_refusals(ops):
    x, pos, r = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), Rotary(64)
    wide = torch.zeros(5, 8, 64, device="cuda")
    for call, what in ((lambda: ops.rotary(Rotary(128), x, pos), "dims"),
                       (lambda: ops.rotary(r, torch.zeros(4, 2, 96, device="cuda"), pos), "head_dim"),
                       (lambda: ops.rotary(r, torch.zeros(0, 2, 64, device="cuda"), pos[:0]), "rows"),
                       (lambda: ops.rotary(r, wide[:4, :2], pos, out=wide[:4, 1:3]), "overlap"),
                       (lambda: ops.rotary(r, wide[:4, :2], pos, out=wide[1:, :2]), "overlap"),
                       (lambda: ops.rotary(r, torch.zeros(4 * 131, device="cuda")[:524].view(4, 131)[:, 1:129].view(4, 2, 64), pos), "aligned")):
        with pytest.raises(SproutError, match=what) as e:
            call()
        assert e.value.status == binding.SPR_ERR_INVALID_ARG
    ops.rotary(r, wide[:4, :2], pos, out=wide[:4, 2:4])


# ------------------------------------------------------------------------------------------------ append and read


def check_append(ops, rng, Hkv, hd, io, lens, rows, rotary=None, strided=False, k=None, v=None, layers=2, layer=1):
    """The whole cache, byte by byte, after an append; then what is read back."""
    n, R = len(lens), sum(rows)
    slots = [int(s) for s in rng.permutation(n)]
    positions = [0] * n
    for i, s in enumerate(slots):
        positions[s] = lens[i] + rows[i]
    cache = ref.Cache(rng, layers, Hkv, hd, positions, spare=1)
    say(f"append: Hkv {Hkv} hd {hd} {io} lens {lens} rows {rows} rotary {rotary} strided {strided}")
    gain = np.exp(0.7 * rng.standard_normal((Hkv, hd)))
    k, kx = rounded(gain * rng.standard_normal((R, Hkv, hd)) if k is None else k, io)
    v, vx = rounded(rng.standard_normal((R, Hkv, hd)) if v is None else v, io)
    if strided:
        k, v = columns(k), columns(v, 3, 1)
    view, batch = cache.device(), CacheBatch(slots, lens, rows)
    ops.append(view, layer, batch, k, v, rotary=Rotary(**rotary) if rotary else None)
    gk, gv = ops.read(view, layer, batch, dtype=io)
    fk, fv = ops.read(view, layer, batch)
    torch.cuda.synchronize()
    pos = np.concatenate([length + np.arange(m) for length, m in zip(lens, rows)])
    if rotary:
        kx = ref.turn(kx, pos, **rotary)
    r0 = 0
    for s, length, m in zip(slots, lens, rows):
        cache.append(layer, s, length, kx[r0:r0 + m], vx[r0:r0 + m])
        r0 += m
    got = view.data.cpu().numpy()
    assert np.array_equal(got, cache.data), f"{(got != cache.data).sum()} bytes differ"
    for got, want in ((gk, kx), (gv, vx), (fk, kx), (fv, vx)):
        np.testing.assert_array_equal(got.double().cpu().numpy(), ref.values(*ref.quantise(want)))


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("Hkv,hd", [(1, 64), (1, 128), (4, 64), (5, 64), (8, 128), (3, 128), (11, 64)])
def test_append_and_read(ops, Hkv, hd, io):
    rng = np.random.default_rng(Hkv * 1000 + hd)
    check_append(ops, rng, Hkv, hd, io, [0, 3, 15, 16, 31, 5, 0], [1, 1, 1, 1, 2, 11, 16])
    check_append(ops, rng, Hkv, hd, io, [7, 0], [50, 33], strided=True)


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("hd,dims", [(64, 64), (128, 128), (64, 2), (128, 126), (128, 32), (64, 46)])
def test_append_turns_keys(ops, hd, dims, layout, io):
    rng = np.random.default_rng(hd * 7 + dims)
    check_append(ops, rng, 4, hd, io, [0, 30, 4000, 9], [1, 5, 20, 40], rotary=dict(dims=dims, layout=layout))
    check_append(ops, rng, 2, hd, io, [100], [3], strided=True,
                 rotary=dict(dims=dims, layout=layout, base=5e5, factor=8.0, original=512, low=1.0, high=32.0, amplitude=1.1))


def test_append_many_requests_and_long_prompts(ops):
    rng = np.random.default_rng(8)
    check_append(ops, rng, 2, 64, BF16, [int(x) for x in rng.integers(0, 60, 128)], [1] * 128, rotary=dict(dims=64), layers=1, layer=0)
    check_append(ops, rng, 40, 64, F32, [5], [300], layers=1, layer=0)
    check_append(ops, rng, 8, 128, BF16, [0, 17, 300], [200, 1, 90], rotary=dict(dims=128, layout="pairs"), layers=1, layer=0)


@pytest.mark.parametrize("io", [F32, BF16])
def test_append_ties_extremes_and_odd_values(ops, io):
    """Ties at every scale, borders of scales, zeros of both signs, the largest and smallest numbers, infinities and NaN."""
    rng = np.random.default_rng(2)
    x = np.zeros((40, 2, 64))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5])
    for r in range(24):  # the 7 pins the scale; the border itself, and just above it
        x[r] = rng.choice(ties, (2, 64)) * rng.choice([-1, 1], (2, 64)) * 2.0 ** (5 * r - 60)
        x[r, :, ::32] = 7 * 2.0 ** (5 * r - 60) * (1 + (2.0 ** -7 if r % 2 else 0))
    x[24], x[25], x[26] = -0.0, 0.0, 1e-44
    x[27], x[28], x[29] = 3.3e38, 2.0 ** -122, 2.0 ** -121 * rng.choice(ties, (2, 64))
    x[30, 0, 5], x[31, 1, 40], x[32, 0, 63] = np.inf, -np.inf, np.nan
    x[33] = np.nan
    x[34:] = rng.standard_normal((6, 2, 64)) * np.exp(rng.normal(0, 30, (6, 2, 64)))
    check_append(ops, rng, 2, 64, io, [3], [40], k=x, v=x[::-1])


def test_append_of_odd_values_that_are_turned(ops):
    """An infinity or NaN spoils its pair and so both their groups; huge ones stay finite."""
    rng = np.random.default_rng(6)
    x = rng.standard_normal((6, 1, 64))
    x[1, 0, 3], x[2, 0, 40] = np.inf, np.nan
    x[3] *= 2.9e38 / np.abs(x[3]).max()
    with np.errstate(invalid="ignore"):
        check_append(ops, rng, 1, 64, F32, [77], [6], k=x, rotary=dict(dims=64))


def test_append_and_read_refusals(ops):
    rng = np.random.default_rng(1)
    view = ref.Cache(rng, 1, 2, 64, [40]).device()
    b = CacheBatch([0], [5], [3])
    k = torch.zeros(3, 2, 64, device="cuda")
    odd = torch.zeros(3 * 131, device="cuda").view(3, 131)[:, 1:129].view(3, 2, 64)
    before = view.data.clone()
    for call, what in ((lambda: ops.append(view, 1, b, k, k), "layer"), (lambda: ops.append(view, 0, b, k, odd), "aligned"),
                       (lambda: ops.append(view, 0, CacheBatch([0], [46], [3]), k, k), "block-table row"),
                       (lambda: ops.append(view, 0, CacheBatch([1], [5], [3]), k, k), "slot"),
                       (lambda: ops.append(view, 0, b, k, k, rotary=Rotary(128)), "dims"),
                       (lambda: ops.read(view, -1, b), "layer"), (lambda: ops.read(view, 0, CacheBatch([0], [0], [49])), "block-table row"),
                       (lambda: ops.attention(view, 0, b, torch.zeros(3, 3, 64, device="cuda")), "n_heads"),
                       (lambda: ops.attention(view, 0, b, torch.zeros(3, 34, 64, device="cuda")), "n_heads"),
                       (lambda: ops.attention(view, 0, b, k, out=k), "overlap"), (lambda: ops.attention(view, 2, b, k), "layer"),
                       (lambda: ops.attention(view, 0, b, odd), "aligned")):
        with pytest.raises(SproutError, match=what) as e:
            call()
        assert e.value.status == binding.SPR_ERR_INVALID_ARG
    with pytest.raises(SproutError, match="overlap"):
        binding._check(ops.lib.spr_cache_read(ops.h, view.ref, 0, b.ref, 0, k.data_ptr(), 128, k.data_ptr() + 256, 128))
    assert torch.equal(view.data, before)


def test_a_block_outside_the_pool_is_not_written():
    rng = np.random.default_rng(12)
    for bad in (-1, 4, 2 ** 31 - 1):
        for call in ("append", "read", "attention"):
            o = CacheOps()
            cache = ref.Cache(rng, 1, 2, 64, [20, 20], extra_blocks=0)
            cache.table[0, 1] = bad
            view, b = cache.device(), CacheBatch([0, 1], [14, 14], [4, 4])
            k, kx = rounded(rng.standard_normal((8, 2, 64)), F32)
            if call == "append":
                o.append(view, 0, b, k, k)
            elif call == "read":
                o.read(view, 0, b)
            else:
                o.attention(view, 0, b, k)
            torch.cuda.synchronize()
            if call == "append":  # all other rows are
                cache.table[0, 1] = cache.table[0, 0]
                want = cache.data.copy()
                cache.append(0, 0, 14, kx[:2], kx[:2])
                cache.append(0, 1, 14, kx[4:], kx[4:])
                assert np.array_equal(view.data.cpu().numpy(), cache.data) and not np.array_equal(want, cache.data)
            with pytest.raises(SproutError, match="block id") as e:
                o.read(view, 0, CacheBatch([1], [0], [1]))
            assert e.value.status == binding.SPR_ERR_DEVICE_CHECK
            o.close()


# ------------------------------------------------------------------------------------------------ attention


def tolerance(cache, layer, slots, lens, rows, q, io, want):
    kn = vm = 0.0
    for s, length, n in zip(slots, lens, rows):
        k, v = cache.rows(layer, s, length + n)
        kn = max(kn, np.sqrt((np.nan_to_num(k) ** 2).sum(-1)).max())
        vm = max(vm, np.abs(np.nan_to_num(v)).max())
    qn, T = np.sqrt((np.nan_to_num(q) ** 2).sum(-1)).max(), max(a + b for a, b in zip(lens, rows))
    tol = (2 * 4 * EPS * qn * kn + (26 + 8 * np.sqrt(T)) * EPS) * vm
    if io == F32:
        return tol + 2.0 ** -22 * vm
    return tol + 2 * 2.0 ** -12 * vm + 2.0 ** -8 * np.abs(want)


def filled(rng, layers, layer, Hkv, hd, slots, lens, rows, spare=1, extra_blocks=2):
    """A cache of random bytes (scale bytes of all kinds among them) that holds the requests' positions in one layer."""
    positions = [0] * len(slots)
    for i, s in enumerate(slots):
        positions[s] = lens[i] + rows[i]
    cache = ref.Cache(rng, layers, Hkv, hd, positions, spare=spare, extra_blocks=extra_blocks)
    for s, p in enumerate(positions):
        blocks = cache.table[s, :(p + 15) // 16]
        x = rng.standard_normal((2, len(blocks), Hkv, 16, hd))
        (kc, ks), (vc, vs) = ref.quantise(x[0]), ref.quantise(x[1])
        ko, vo, kso, vso, khi, vhi = ref.offsets(hd)
        for j, b in enumerate(blocks):
            n = min(16, p - 16 * j)
            for h in range(Hkv):
                tile = cache.data[layer, b, h]
                for at, high, c in ((ko, khi, kc), (vo, vhi, vc)):
                    byte = np.zeros(17 * hd, np.int64)
                    np.add.at(byte, at[:n], c[j, h, :n].astype(np.int64) << np.where(high[:n], 4, 0))
                    tile[np.unique(at[:n])] = byte[np.unique(at[:n])]
                tile[kso[:n]] = np.repeat(ks[j, h, :n], 32, -1)
                tile[vso[:n]] = np.repeat(vs[j, h, :n], 32, -1)
    return cache


def check_attention(ops, rng, H, Hkv, hd, io, lens, rows, layers=1, layer=0, strided=False, tag="", slots=None):
    slots = [int(s) for s in rng.permutation(len(lens))] if slots is None else slots
    cache = filled(rng, layers, layer, Hkv, hd, slots, lens, rows)
    q, qx = rounded(rng.standard_normal((sum(rows), H, hd)), io)
    say(f"attention {tag}: H {H}/{Hkv} hd {hd} {io} lens {lens[:9]} rows {rows[:9]} strided {strided}")
    if strided:
        q = columns(q)
    out = ops.attention(cache.device(), layer, CacheBatch(slots, lens, rows), q)
    torch.cuda.synchronize()
    want = ref.attention(cache, layer, slots, lens, rows, qx)
    got = out.double().cpu().numpy()
    tol = tolerance(cache, layer, slots, lens, rows, qx, io, want)
    assert np.isfinite(got).all()
    worst = (np.abs(got - want) / tol).max()
    assert worst <= 1, f"{worst} of the tolerance, max error {np.abs(got - want).max():.3e}"


SHAPES = [(4, 4, 64), (8, 2, 128), (65, 5, 64), (3, 3, 128), (16, 1, 128), (16, 1, 64)]


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("H,Hkv,hd", SHAPES)
def test_attention_shapes_and_types(ops, H, Hkv, hd, io):
    rng = np.random.default_rng(H * 100 + hd)
    check_attention(ops, rng, H, Hkv, hd, io, [0, 1, 15, 16, 17, 130, 47], [1] * 7)
    check_attention(ops, rng, H, Hkv, hd, io, [0, 3, 14, 40], [2, 1, 5, 3], strided=True)
    check_attention(ops, rng, H, Hkv, hd, io, [0, 37, 90], [33, 1, 20])


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("lens,rows", [([0], [1]), ([0], [2]), ([15], [1]), ([15], [2]), ([16], [1]), ([31], [16]), ([32], [33]),
                                       ([0], [200]), ([63, 64, 65], [16, 17, 33]), ([0, 500], [130, 1]), ([40] * 128, [1] * 128),
                                       ([3000], [1]), ([9000, 3], [2, 1]), ([2000, 0], [70, 260])])
def test_attention_lengths_and_splits(ops, io, lens, rows):
    """One position to many KV splits; single tokens, chunks of all sizes; the largest batch; a two-layer cache's second layer."""
    rng = np.random.default_rng(7)
    check_attention(ops, rng, 4, 2, 64, io, lens, rows, layers=2, layer=1)


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("H,Hkv,hd,rows", [(16, 2, 128, 64), (16, 2, 64, 70), (32, 2, 128, 5), (4, 4, 128, 33), (8, 8, 64, 20), (2, 2, 128, 150)])
def test_attention_of_chunks_over_long_contexts(ops, H, Hkv, hd, rows, io):
    """Several column groups and KV splits at once, whole steps of either parity, beside a short request."""
    rng = np.random.default_rng(hd + rows)
    for lens in ([1700, 5], [1683, 40]):
        check_attention(ops, rng, H, Hkv, hd, io, lens, [rows, 3], tag="chunks")


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("lens,rows", [([20, 12000] + [33] * 30, [1] * 32), ([0, 6000, 9, 40], [300, 1, 1, 70]),
                                       ([1030] + list(range(60)), [1] + [2] * 60)])
def test_attention_of_mixed_batches(ops, lens, rows, io):
    """One request far longer than the rest; prompts beside single tokens."""
    rng = np.random.default_rng(len(lens))
    check_attention(ops, rng, 8, 4, 128, io, lens, rows, tag="mixed")


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("H,Hkv,hd", [(512, 32, 128), (512, 32, 64), (1000, 200, 64), (260, 260, 128)])
@pytest.mark.parametrize("lens,rows", [([0], [35]), ([37, 0, 90], [33, 1, 70]), ([15, 3], [200, 2]), ([129], [97])])
def test_attention_of_many_rows_and_heads(ops, H, Hkv, hd, lens, rows, io):
    """Enough of them that work-groups take 64 and 128 columns."""
    rng = np.random.default_rng(H + hd + rows[0])
    check_attention(ops, rng, H, Hkv, hd, io, lens, rows, strided=rows[0] == 97, tag="many")


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("H,Hkv,hd,rows", [(512, 32, 128, 34), (512, 32, 64, 34), (512, 32, 128, 100), (512, 32, 64, 100), (600, 40, 64, 85)])
def test_attention_of_many_rows_and_heads_over_long_contexts(ops, H, Hkv, hd, rows, io):
    """Those with KV splits, of either parity of whole steps."""
    rng = np.random.default_rng(hd + rows)
    for length in (700, 683):
        check_attention(ops, rng, H, Hkv, hd, io, [length], [rows], tag="many, long")


# Heads and KV heads of the tests below: few, whose rows' columns work-groups share 16 or 32 at a time, and so many that from
# 33 rows on they take 64 and from 65 on, in bf16, 128.
HEADS = pytest.mark.parametrize("H,Hkv", [(4, 2), (512, 32)])


@pytest.mark.parametrize("io", [F32, BF16])
@HEADS
def test_attention_scores_of_all_sizes(ops, H, Hkv, io):
    """A few positions take nearly all weight, early or late ones: maxima that rise and fall; and values of many scales."""
    rng = np.random.default_rng(21)
    n = 2000 if Hkv == 2 else 200
    for rows, at in ((1, (5, n - 100)), (40, (0, n // 3)), (130, (n // 2, n - 10))):
        lens, slots = [n], [0]
        cache = filled(rng, 1, 0, Hkv, 128, slots, lens, [rows])
        q, qx = rounded(0.2 * rng.standard_normal((rows, H, 128)), io)
        k = 0.2 * rng.standard_normal((n + rows, Hkv, 128))
        v = rng.standard_normal((n + rows, Hkv, 128)) * 2.0 ** rng.integers(-18, 15, (n + rows, 1, 1))
        for p in at:
            k[p] = qx[0, ::H // Hkv] * 60
        cache.append(0, 0, 0, k, v)
        want = ref.attention(cache, 0, slots, lens, [rows], qx)
        got = ops.attention(cache.device(), 0, CacheBatch(slots, lens, [rows]), q).double().cpu().numpy()
        tol = tolerance(cache, 0, slots, lens, [rows], qx, io, want)
        assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()


@HEADS
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [1, 40, 100])
def test_attention_of_fp32_small_probabilities(ops, H, Hkv, hd, rows):
    """Every 16th position takes nearly all weight and has the value 0 but in one dimension of each group, the others have p =
    2^-20 of its weight and the value 1: an output is about 15 p, to what p is held to.

    A score is one exact product (dimension 0) or 0.  p is off by 2^-36 of the largest from its parts (2^-22 of itself is less),
    by 20 * 2^-24 ln 2 < 2^-20 of itself from the factor of the scores (a difference of 20 between two), by 2^-20 from the
    exponent's argument (below 16 in magnitude: half a step is 2^-21) and 2^-23 from exp2; the two sums, one addition for each 16
    positions at most, by (T / 16 + 8) eps each, merges and the output's own rounding among them."""
    rng = np.random.default_rng(hd + rows)
    length = 500
    T = length + rows
    q = rng.standard_normal((rows, H, hd))
    q[..., 0] = rng.uniform(19.5, 20.5, (rows, H)) * np.log(2) * np.sqrt(hd)
    q, qx = rounded(q, F32)
    k, v = np.zeros((T, Hkv, hd)), np.ones((T, Hkv, hd))
    k[::16, :, 0], v[::16] = 1, np.arange(hd) % 32 == 0
    cache = ref.Cache(rng, 1, Hkv, hd, [T])
    cache.append(0, 0, 0, k, v)
    want = ref.attention(cache, 0, [0], [length], [rows], qx)
    got = ops.attention(cache.device(), 0, CacheBatch([0], [length], [rows]), q).double().cpu().numpy()
    p = np.exp(-qx[..., :1] / np.sqrt(hd))
    tol = 2.0 ** -36 / p + 2.0 ** -22 + 2 * 2.0 ** -20 + 2.0 ** -23 + 2 * (T / 16 + 8) * EPS
    worst = (np.abs(got - want) / (tol * want))[..., np.arange(hd) % 32 > 0].max()
    assert worst <= 1, f"{worst} of the tolerance"


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("hd", [64, 128])
@HEADS
def test_attention_of_values_that_are_zero(ops, H, Hkv, hd, io):
    """Positions, and groups of some, whose values are zeros (of the lowest scale), whole blocks of them too."""
    rng = np.random.default_rng(hd)
    n = 300 if Hkv == 2 else 60
    for rows in (1, 50, 100):
        cache = filled(rng, 1, 0, Hkv, hd, [0], [n], [rows])
        q, qx = rounded(rng.standard_normal((rows, H, hd)), io)
        k, v = (rng.standard_normal((n + rows, Hkv, hd)) for _ in range(2))
        v[rng.random(n + rows) < 0.3] = 0
        v[16:48], v[::3, :, 32:64] = 0, -0.0
        cache.append(0, 0, 0, k, v)
        want = ref.attention(cache, 0, [0], [n], [rows], qx)
        got = ops.attention(cache.device(), 0, CacheBatch([0], [n], [rows]), q).double().cpu().numpy()
        tol = tolerance(cache, 0, [0], [n], [rows], qx, io, want)
        assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 90])
@HEADS
def test_attention_of_values_far_from_one(ops, H, Hkv, io, scale):
    """Values of any scale give outputs of it, to the same relative tolerance."""
    rng = np.random.default_rng(30)
    n = 300 if Hkv == 2 else 60
    for rows in (1, 50, 100):
        cache = filled(rng, 1, 0, Hkv, 128, [0], [n], [rows])
        q, qx = rounded(rng.standard_normal((rows, H, 128)), io)
        v = rng.standard_normal((n + rows, Hkv, 128))
        k = rng.standard_normal((n + rows, Hkv, 128))
        cache.append(0, 0, 0, k, v)
        want = ref.attention(cache, 0, [0], [n], [rows], qx)
        tol = tolerance(cache, 0, [0], [n], [rows], qx, io, want)
        cache.append(0, 0, 0, k, v * scale)
        got = ops.attention(cache.device(), 0, CacheBatch([0], [n], [rows]), q).double().cpu().numpy() / scale
        assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("hd,rows", [(64, 3), (128, 3), (64, 40), (128, 40), (128, 130)])
@HEADS
def test_attention_of_one_large_value(ops, H, Hkv, hd, rows, io):
    """One group of one position, of the first blocks or of others, far above the rest: whoever reads it first."""
    rng = np.random.default_rng(hd + rows)
    q, qx = rounded(rng.standard_normal((rows, H, hd)), io)
    n = 200 if Hkv == 2 else 70
    k, v = (rng.standard_normal((n + rows, Hkv, hd)) for _ in range(2))
    cache = filled(rng, 1, 0, Hkv, hd, [0], [n], [rows])
    for pos in (0, 6, 9, 15, 17, 20, 27, 30, 33, 61, n // 2, n - 1) if Hkv == 2 else (0, 9, 20, 27, n - 1):
        big = v.copy()
        big[pos, Hkv - 1, 32:64] *= 2.0 ** 40
        cache.append(0, 0, 0, k, big)
        want = ref.attention(cache, 0, [0], [n], [rows], qx)
        got = ops.attention(cache.device(), 0, CacheBatch([0], [n], [rows]), q).double().cpu().numpy()
        tol = np.broadcast_to(tolerance(cache, 0, [0], [n], [rows], qx, io, want), want.shape)
        assert (np.abs(got - want) <= tol).all(), (pos, (np.abs(got - want) / tol).max())


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("hd,rows", [(64, 5), (128, 5), (64, 50), (128, 50), (128, 200)])
@HEADS
def test_attention_nan_reaches_the_rows_that_see_it(ops, H, Hkv, hd, rows, io):
    """A NaN group of a value reaches its 32 dimensions of the rows that see its position, one of a key reaches those rows
    whole, and no other row changes."""
    rng = np.random.default_rng(hd + rows)
    length, G = 37, H // Hkv
    q, qx = rounded(rng.standard_normal((rows, H, hd)), io)
    for pos, key in ((length + rows // 2, False), (length + rows // 2, True), (length - 2, False), (length + rows - 1, True),
                     (length + 1, False)):
        cache = filled(rng, 1, 0, Hkv, hd, [0], [length], [rows])
        want = ref.attention(cache, 0, [0], [length], [rows], qx)
        tol = np.broadcast_to(tolerance(cache, 0, [0], [length], [rows], qx, io, want), want.shape)
        _, _, kso, vso, _, _ = ref.offsets(hd)
        cache.data[0, cache.table[0, pos // 16], 1, (kso if key else vso)[pos % 16, 32]] = 255  # KV head 1, second group
        got = ops.attention(cache.device(), 0, CacheBatch([0], [length], [rows]), q).double().cpu().numpy()
        hit = np.zeros(want.shape, bool)
        first = max(0, pos - length)
        hit[first:, G:2 * G, slice(None) if key else slice(32, 64)] = True
        assert np.isnan(got[hit]).all(), (pos, key)
        assert (np.abs(got - want)[~hit] <= tol[~hit]).all(), (pos, key)


@pytest.mark.parametrize("io", [F32, BF16])
@HEADS
def test_attention_queries_that_are_no_numbers(ops, H, Hkv, io):
    """They spoil their own row and head."""
    rng = np.random.default_rng(2)
    for rows in (3, 60, 110):
        cache = filled(rng, 1, 0, Hkv, 128, [0], [40], [rows])
        q, qx = rounded(rng.standard_normal((rows, H, 128)), io)
        want = ref.attention(cache, 0, [0], [40], [rows], qx)
        tol = np.broadcast_to(tolerance(cache, 0, [0], [40], [rows], qx, io, want), want.shape)
        q[1, 2, 77], q[rows - 1, 0, 3] = float("nan"), float("inf")
        got = ops.attention(cache.device(), 0, CacheBatch([0], [40], [rows]), q).double().cpu().numpy()
        bad = np.zeros(want.shape, bool)
        bad[1, 2] = bad[rows - 1, 0] = True
        assert np.isnan(got[bad]).all() and (np.abs(got - want)[~bad] <= tol[~bad]).all()


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("lens,rows", [([20, 0], [1, 3]), ([3000], [2]), ([30], [40]), ([700], [100])])
@HEADS
def test_attention_into_columns_of_a_wider_tensor(ops, H, Hkv, lens, rows, io):
    """The same bits as into a tensor of its own, and nothing beside them, in rows before and behind either."""
    rng = np.random.default_rng(sum(lens))
    cache = filled(rng, 1, 0, Hkv, 64, list(range(len(lens))), lens, rows)
    q, _ = rounded(rng.standard_normal((sum(rows), H, 64)), io)
    view, batch, R = cache.device(), CacheBatch(list(range(len(lens))), lens, rows), sum(rows)
    want = ops.attention(view, 0, batch, q)
    wide = torch.full((R + 4, H + 3, 64), 7.0, dtype=io, device="cuda")
    out = wide[2:2 + R, 1:1 + H]
    assert ops.attention(view, 0, batch, q, out=out) is out and torch.equal(out, want)
    out.fill_(7.0)
    assert (wide == 7.0).all()


@pytest.mark.parametrize("hd", [64, 128])
@HEADS
def test_attention_of_the_largest_queries(ops, H, Hkv, hd):
    """Finite fp32 queries beyond bf16's largest number, whose scores are ordinary: their keys have the lowest scale.

    A score's roundings are below (hd + 4) eps of the sum of its products' magnitudes."""
    rng = np.random.default_rng(hd)
    top = float(np.finfo(np.float32).max)
    n = 300 if Hkv == 2 else 60
    for rows in (1, 50, 100):
        T = n + rows
        q = rng.standard_normal((rows, H, hd))
        q[..., 0] = rng.choice([-1, 1], (rows, H)) * top * rng.choice([1, 1 - 2.0 ** -23, 0.999, 0.9], (rows, H))
        k, v = (rng.standard_normal((T, Hkv, hd)) for _ in range(2))
        k[..., :32] = 0
        k[..., 0] = rng.integers(-2, 3, (T, Hkv)) * 2.0 ** -121
        q, qx = rounded(q, F32)
        cache = ref.Cache(rng, 1, Hkv, hd, [T])
        cache.append(0, 0, 0, k, v)
        want = ref.attention(cache, 0, [0], [n], [rows], qx)
        got = ops.attention(cache.device(), 0, CacheBatch([0], [n], [rows]), q).double().cpu().numpy()
        kx, vx = cache.rows(0, 0, T)
        size = (np.abs(qx).max((0, 1)) * np.abs(kx).max((0, 1))).sum() / np.sqrt(hd)
        tol = (2 * (hd + 4) * EPS * size + (2 * size + 26 + 8 * np.sqrt(T)) * EPS + 2.0 ** -22) * np.abs(vx).max()
        assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max() / tol


@pytest.mark.parametrize("rows", [1, 70, 2100])
def test_attention_far_into_a_large_pool(ops, rows):
    """Blocks behind byte 2^32 of the pool and of the layer."""
    rng = np.random.default_rng(5)
    small = filled(rng, 1, 0, 8, 128, [0], [200], [rows])
    q, qx = rounded(rng.standard_normal((rows, 8, 128)), BF16)
    want = ref.attention(small, 0, [0], [200], [rows], qx)
    n = small.data.shape[1]
    blocks = 2 ** 32 // (8 * 17 * 128) + 100
    data = torch.zeros(2, blocks, 8, 17 * 128, dtype=torch.uint8, device="cuda")
    data[1, blocks - n:] = torch.from_numpy(small.data[0]).cuda()
    view = KV4View(data, torch.from_numpy(small.table + blocks - n).cuda())
    got = ops.attention(view, 1, CacheBatch([0], [200], [rows]), q).double().cpu().numpy()
    assert (np.abs(got - want) <= tolerance(small, 0, [0], [200], [rows], qx, BF16, want)).all()
    x, xx = rounded(rng.standard_normal((1, 8, 128)), F32)
    b = CacheBatch([0], [199], [1])
    ops.append(view, 1, b, x, x)
    assert np.array_equal(ops.read(view, 1, b)[1].double().cpu().numpy(), ref.values(*ref.quantise(xx)))
    last = blocks - 1
    ops.move(view, [last - 5], [3])
    assert torch.equal(data[:, 3], data[:, last - 5])


# ------------------------------------------------------------------------------------------------ pages


def any_cache(rng, kind, layers, blocks, Hkv, hd, slots, mb):
    table = torch.from_numpy(rng.integers(0, blocks, (slots, mb)).astype(np.int32)).cuda()
    if kind == "mx4":
        return KV4View(torch.from_numpy(rng.integers(0, 256, (layers, blocks, Hkv, 17 * hd), dtype=np.uint8)).cuda(), table)
    k, v = (torch.from_numpy(rng.standard_normal((layers, blocks, Hkv, 16 * hd))).to(kind).cuda() for _ in range(2))
    return KVView(k, v, table)


def pools(view):
    return [view.data] if isinstance(view, KV4View) else [view.k, view.v]


@pytest.mark.parametrize("kind", ["mx4", F32, BF16])
@pytest.mark.parametrize("layers,Hkv,hd", [(1, 1, 64), (3, 5, 64), (2, 8, 128), (2, 40, 128)])
def test_fork(ops, kind, layers, Hkv, hd):
    rng = np.random.default_rng(Hkv + hd)
    for trial in range(6):
        slots, mb, blocks, n = 12, 6, 90, int(rng.integers(1, 9))
        view = any_cache(rng, kind, layers, blocks, Hkv, hd, slots, mb)
        ids = rng.permutation(blocks)
        at = rng.permutation(slots)
        target, sources = at[:n], at[9:]
        source = rng.choice(sources[:1 + trial % 3], n)
        table = view.block_table.cpu().numpy()
        table[sources] = ids[20:20 + 3 * mb].reshape(3, mb)
        view.block_table.copy_(torch.from_numpy(table))
        lens = rng.choice([0, 1, 15, 16, 17, 33, 80, 95, 96], n)
        fresh = np.where(lens % 16 == 0, -5, ids[:n])
        before = [p.clone() for p in pools(view)]
        say(f"fork: {kind} layers {layers} Hkv {Hkv} hd {hd} source {source} lens {lens}")
        ops.fork(view, source, target, lens, fresh)
        torch.cuda.synchronize()
        for s, t, x, f in zip(source, target, lens, fresh):
            table[t, :x // 16] = table[s, :x // 16]
            if x % 16:
                for p in before:
                    p[:, int(f)] = p[:, int(table[s, x // 16])]
                table[t, x // 16] = f
        assert np.array_equal(view.block_table.cpu().numpy(), table)
        assert all(torch.equal(a, b) for a, b in zip(pools(view), before))


def test_fork_of_the_largest_batch(ops):
    rng = np.random.default_rng(3)
    view = any_cache(rng, "mx4", 2, 400, 4, 64, 140, 4)
    table = view.block_table.cpu().numpy()
    table[:3] = np.arange(12).reshape(3, 4)
    view.block_table.copy_(torch.from_numpy(table))
    before = view.data.clone()
    source, fresh = np.arange(128) % 3, 20 + rng.permutation(128)
    ops.fork(view, source, 5 + np.arange(128), [39] * 128, fresh)
    for i in range(128):
        table[5 + i, :2] = table[source[i], :2]
        table[5 + i, 2] = fresh[i]
        before[:, int(fresh[i])] = before[:, int(table[source[i], 2])]
    assert np.array_equal(view.block_table.cpu().numpy(), table) and torch.equal(view.data, before)


@pytest.mark.parametrize("what", ["outside", "negative", "fresh"])
def test_fork_of_a_source_that_is_not_there(what):
    """Nothing is copied, and the handle's next call says so."""
    o = CacheOps()
    rng = np.random.default_rng(3)
    view = any_cache(rng, BF16, 2, 20, 2, 64, 3, 2)
    view.block_table[0] = torch.tensor([1, {"outside": 20, "negative": -3, "fresh": 7}[what]], dtype=torch.int32)
    before = [p.clone() for p in pools(view)]
    o.fork(view, [0, 0], [1, 2], [20, 5], [7, 8])
    torch.cuda.synchronize()
    for p, b in zip(pools(view), before):
        b[:, 8] = b[:, 1]
        assert torch.equal(p, b)
    with pytest.raises(SproutError, match="fresh block" if what == "fresh" else "block id") as e:
        o.move(view, [1], [2])
    assert e.value.status == binding.SPR_ERR_DEVICE_CHECK
    o.close()


def check_faulty_fork(source_rows, target, source, lens, fresh, want_rows, copied, match):
    """A fork over sources with these table rows, its targets' rows afterwards, the blocks that were copied, the next call."""
    o = CacheOps()
    view = any_cache(np.random.default_rng(3), BF16, 2, 30, 2, 64, 6, 3)
    for s, row in source_rows.items():
        view.block_table[s] = torch.tensor(row, dtype=torch.int32)
    for t in target:
        view.block_table[t] = 29  # (what was there)
    table, before = view.block_table.clone(), [p.clone() for p in pools(view)]
    o.fork(view, source, target, lens, fresh)
    torch.cuda.synchronize()
    for t, row in want_rows.items():
        table[t] = torch.tensor(row, dtype=torch.int32)
    assert torch.equal(view.block_table, table)
    for p, b in zip(pools(view), before):
        for src, dst in copied:
            b[:, dst] = b[:, src]
        assert torch.equal(p, b)
    with pytest.raises(SproutError, match=match) as e:
        o.move(view, [1], [2])
    assert e.value.status == binding.SPR_ERR_DEVICE_CHECK
    o.close()


@pytest.mark.parametrize("bad", [-1, 30, 2 ** 31 - 1])
@pytest.mark.parametrize("partly", [False, True])
def test_fork_of_a_source_whose_entry_is_outside_the_pool(bad, partly):
    """A full block's, and a partly filled one's: the target's row takes all entries but that one."""
    if partly:
        check_faulty_fork({0: [4, 5, bad]}, [3, 4], [0, 0], [37, 20], [7, 8], {3: [4, 5, 29], 4: [4, 8, 29]}, [(5, 8)], "block id")
    else:
        check_faulty_fork({0: [4, bad, 6]}, [3, 4], [0, 0], [37, 48], [7, -1], {3: [4, 29, 7], 4: [4, 29, 6]}, [(6, 7)], "block id")


def test_fork_of_a_full_block_that_is_fresh():
    check_faulty_fork({0: [4, 5, 6], 1: [8, 9, 10]}, [3, 4], [0, 1], [32, 20], [-1, 5], {3: [4, 29, 29], 4: [8, 5, 29]}, [(9, 5)], "fresh block")


def test_fork_onto_a_block_that_another_fork_copies_from():
    """Neither fork is carried out, whose source would change under the other, nor the first's second target; the third is."""
    check_faulty_fork({0: [4, 5, 6], 1: [8, 9, 10]}, [3, 4, 5, 2], [0, 1, 1, 0], [20, 35, 33, 7], [7, 5, 11, 12],
                      {3: [4, 29, 29], 4: [8, 9, 29], 5: [8, 9, 29], 2: [12, 29, 29]}, [(4, 12)], "fresh block")


@pytest.mark.parametrize("kind", ["mx4", F32, BF16])
@pytest.mark.parametrize("layers,Hkv,hd,blocks,n,slots,mb", [(1, 1, 64, 2, 1, 1, 1), (3, 5, 64, 60, 20, 7, 9), (2, 8, 128, 40, 13, 300, 21),
                                                          (1, 1, 64, 1500, 750, 40, 60)])
def test_move(ops, kind, layers, Hkv, hd, blocks, n, slots, mb):
    """One pair to more than a launch takes; tables of one entry to many, with blocks that several entries share."""
    rng = np.random.default_rng(n)
    view = any_cache(rng, kind, layers, blocks, Hkv, hd, slots, mb)
    ids = rng.permutation(blocks)
    src, dst = ids[:n], ids[n:2 * n]
    table, before = view.block_table.cpu().numpy(), [p.clone() for p in pools(view)]
    say(f"move: {kind} layers {layers} Hkv {Hkv} hd {hd} blocks {blocks} moved {n}")
    ops.move(view, src, dst)
    torch.cuda.synchronize()
    now = np.arange(blocks)
    now[src] = dst
    for p, b in zip(pools(view), before):
        b[:, torch.from_numpy(dst).cuda()] = b[:, torch.from_numpy(src).cuda()]
        assert torch.equal(p, b)
    assert np.array_equal(view.block_table.cpu().numpy(), now[table])


def test_pages_refusals(ops):
    rng = np.random.default_rng(3)
    view = any_cache(rng, "mx4", 1, 20, 2, 64, 3, 2)
    before = (view.data.clone(), view.block_table.clone())
    for call, what in ((lambda: ops.fork(view, [0], [0], [5], [3]), "also a source"), (lambda: ops.fork(view, [0], [1], [33], [3]), "lens"),
                       (lambda: ops.fork(view, [], [], [], []), "n must"), (lambda: ops.move(view, [], []), "n must"),
                       (lambda: ops.move(view, [3], [20]), "out of range"), (lambda: ops.move(view, [3, 4], [4, 5]), "also a src")):
        with pytest.raises(SproutError, match=what) as e:
            call()
        assert e.value.status == binding.SPR_ERR_INVALID_ARG
    # Pools of a size that a launch has too many work-groups for (refused before anything is touched).
    huge = binding.SprPages(view.data.data_ptr(), None, 1 << 30, 1000, 20, view.block_table.data_ptr(), 3, 2)
    one = [np.array([x], dtype=np.int32) for x in (0, 1, 20, 3)]
    at = [x.ctypes.data for x in one]
    for status in (ops.lib.spr_cache_fork(ops.h, ctypes.byref(huge), 1, *at),
                   ops.lib.spr_cache_move(ops.h, ctypes.byref(huge), 1, at[0], at[1])):
        assert status == binding.SPR_ERR_INVALID_ARG
    huge = binding.SprPages(view.data.data_ptr(), None, 1 << 10, 1, 20, view.block_table.data_ptr(), 1 << 20, 1 << 20)
    assert ops.lib.spr_cache_move(ops.h, ctypes.byref(huge), 1, at[0], at[1]) == binding.SPR_ERR_INVALID_ARG
    assert torch.equal(view.data, before[0]) and torch.equal(view.block_table, before[1])


def test_a_models_own_cache_is_not_forked_or_moved(ops):
    from paper_2403_12900_amd.binding import DecodeModel
    from paper_2403_12900_amd.configs import ModelConfig
    dm = DecodeModel(ModelConfig(n_layers=1, d_model=64, n_heads=1, n_kv_heads=1, head_dim=64, d_ff=64, vocab=300), 5,
                     max_slots=2, max_ctx=40)
    view = dm.kv_view()
    parts = [t.view(torch.uint8) for t in (view.k, view.v, view.block_table)]  # (a fresh cache may hold NaN)
    before = [t.clone() for t in parts]
    for call in (lambda: ops.fork(view, [0], [1], [16], [-1]), lambda: ops.move(view, [0], [1])):
        with pytest.raises(SproutError, match="model's own") as e:
            call()
        assert e.value.status == binding.SPR_ERR_INVALID_ARG
    assert all(torch.equal(t, b) for t, b in zip(parts, before))
    dm.close()


# ------------------------------------------------------------------------------------------------ together


class Serving:
    """Requests of a small model's one layer over a 4-bit cache on the device, with the plain forms beside it."""

    def __init__(self, rng, io, H=4, Hkv=2, hd=64, blocks=80, slots=8, mb=8):
        self.rng, self.io, self.H, self.Hkv, self.hd = rng, io, H, Hkv, hd
        self.cache = ref.Cache(rng, 1, Hkv, hd, [0] * slots, extra_blocks=blocks)
        self.cache.mb = mb
        self.cache.table = np.zeros((slots, mb), np.int32)
        self.free = self.cache.free
        self.view = self.cache.device()
        self.turn = dict(dims=48, layout="pairs", base=5e5, factor=4.0, original=64, low=1.0, high=32.0, amplitude=1.1)
        self.rotary = Rotary(**self.turn)
        self.length = [0] * slots

    def sync(self):
        self.view.block_table.copy_(torch.from_numpy(self.cache.table))

    def step(self, ops, slots, rows):
        """A projection's rows through rotary, append and attention; the same beside it; returns both outputs."""
        lens = [self.length[s] for s in slots]
        for s, n in zip(slots, rows):
            for b in range((self.length[s] + 15) // 16, (self.length[s] + n + 15) // 16):
                self.cache.table[s, b] = self.free.pop()
        self.sync()
        x, xx = rounded(self.rng.standard_normal((sum(rows), self.H + 2 * self.Hkv, self.hd)), self.io)
        pos = np.concatenate([length + np.arange(n) for length, n in zip(lens, rows)])
        H, e = self.H, self.H + self.Hkv
        batch = CacheBatch(slots, lens, rows)
        p = torch.from_numpy(pos.astype(np.int32)).cuda()
        ops.append(self.view, 0, batch, x[:, H:e], x[:, e:], rotary=self.rotary)
        q = ops.rotary(self.rotary, x[:, :H], p)
        out = ops.attention(self.view, 0, batch, q)
        r0 = 0
        for s, length, n in zip(slots, lens, rows):
            self.cache.append(0, s, length, ref.turn(xx[r0:r0 + n, H:e], pos[r0:r0 + n], **self.turn), xx[r0:r0 + n, e:])
            self.length[s] += n
            r0 += n
        qx = q.double().cpu().numpy()
        want = ref.attention(self.cache, 0, slots, lens, rows, qx)
        tol = tolerance(self.cache, 0, slots, lens, rows, qx, self.io, want)
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
        return out


@pytest.mark.parametrize("io", [F32, BF16])
def test_a_serving_loop(ops, io):
    """Prompts, decode steps, a prompt's continuations by forking, requests that leave, compaction; the cache byte by byte."""
    rng = np.random.default_rng(40)
    s = Serving(rng, io)
    s.step(ops, [0, 3], [37, 16])                 # two prompts
    s.step(ops, [3, 0], [1, 1])
    fresh = [s.free.pop() for _ in range(2)]      # 38 positions: two full blocks and six positions; and 32 of them alone
    ops.fork(s.view, [0, 0, 0], [1, 2, 5], [38, 38, 32], fresh + [-1])
    for t, f in ((1, fresh[0]), (2, fresh[1])):
        s.cache.table[t, :2] = s.cache.table[0, :2]
        s.cache.table[t, 2] = f
        s.cache.data[:, f] = s.cache.data[:, s.cache.table[0, 2]]
        s.length[t] = 38
    s.cache.table[5, :2] = s.cache.table[0, :2]
    s.length[5] = 32
    assert np.array_equal(s.view.block_table.cpu().numpy(), s.cache.table)
    for _ in range(12):                           # each goes its own way
        s.step(ops, [0, 1, 2, 5, 3], [1] * 5)
    s.step(ops, [1], [40])                        # a second turn's prompt
    s.length[2] = 0                               # request 2 has left; its blocks but the shared ones are free
    used = sorted({int(b) for t in (0, 1, 3, 5) for b in s.cache.table[t, :(s.length[t] + 15) // 16]})
    holes = [b for b in range(len(used)) if b not in used]
    src = [b for b in used if b >= len(used)]
    ops.move(s.view, src, holes)
    now = np.arange(s.cache.data.shape[1])
    now[src] = holes
    s.cache.data[:, holes] = s.cache.data[:, src]
    s.cache.table = now[s.cache.table].astype(np.int32)
    s.free[:] = [b for b in range(s.cache.data.shape[1]) if b >= len(used)]
    assert np.array_equal(s.view.block_table.cpu().numpy(), s.cache.table)
    for rows in (1, 3):
        s.step(ops, [5, 0, 1, 3], [rows] * 4)
    assert np.array_equal(s.view.data.cpu().numpy(), s.cache.data)


def test_a_captured_step_replays(ops):
    """A graph of append, rotary, attention and read with eager work between its replays, on the same handle."""
    rng = np.random.default_rng(41)
    io, H, Hkv, hd = BF16, 8, 2, 128
    for lens, rows in (([700, 20], [1, 1]), ([300, 64], [40, 9]), ([300, 1], [2100, 3])):
        cache = filled(rng, 1, 0, Hkv, hd, [0, 1], lens, rows)
        view, batch, r = cache.device(), CacheBatch([0, 1], lens, rows), Rotary(128)
        x = torch.zeros(sum(rows), H + 2 * Hkv, hd, dtype=io, device="cuda")
        pos = torch.from_numpy(np.concatenate([a + np.arange(n) for a, n in zip(lens, rows)]).astype(np.int32)).cuda()

        def step():
            ops.append(view, 0, batch, x[:, H:H + Hkv], x[:, H + Hkv:], rotary=r)
            return ops.attention(view, 0, batch, ops.rotary(r, x[:, :H], pos)), ops.read(view, 0, batch, dtype=io)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got, (gk, gv) = step()
        for trial in range(4):
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape))).to(io))
            want, (wk, wv) = step()
            want, wk, wv = want.clone(), wk.clone(), wv.clone()
            view.data[..., -1] ^= 0  # eager work of the program's own
            x2 = x.clone()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(gk, wk) and torch.equal(gv, wv) and torch.equal(x, x2)


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("lens,rows", [([700, 20], [1, 1]), ([300, 64], [40, 9]), ([300, 1], [2100, 3])])
def test_a_captured_step_writes_its_rows(ops, lens, rows, io):
    """Replays over positions that an eager append has just filled with other values; the same step, eager, on a cache of its
    own that never held them: outputs, what is read back, and the caches whole."""
    rng = np.random.default_rng(47)
    H, Hkv, hd = 8, 2, 128
    cache = filled(rng, 1, 0, Hkv, hd, [0, 1], lens, rows)
    view, beside, batch, r = cache.device(), cache.device(), CacheBatch([0, 1], lens, rows), Rotary(128)
    x = torch.zeros(sum(rows), H + 2 * Hkv, hd, dtype=io, device="cuda")
    pos = torch.from_numpy(np.concatenate([a + np.arange(n) for a, n in zip(lens, rows)]).astype(np.int32)).cuda()

    def step(v):
        ops.append(v, 0, batch, x[:, H:H + Hkv], x[:, H + Hkv:], rotary=r)
        return (ops.attention(v, 0, batch, ops.rotary(r, x[:, :H], pos)), *ops.read(v, 0, batch, dtype=io))

    step(view)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(view)
    for trial in range(3):
        x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape))).to(io))
        other = torch.from_numpy(rng.standard_normal((sum(rows), Hkv, hd))).to(io).cuda()
        ops.append(view, 0, batch, other, other)
        for g in got:
            g.fill_(trial)
        want = step(beside)
        torch.cuda.synchronize()
        assert not torch.equal(view.data, beside.data)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want)) and torch.equal(view.data, beside.data)


def test_captured_pages_replay(ops):
    """A captured fork and move keep the numbers they were given."""
    rng = np.random.default_rng(42)
    view = any_cache(rng, "mx4", 2, 30, 2, 64, 4, 3)
    ops.fork(view, [0], [1], [20], [9])
    view.block_table[0] = torch.tensor([4, 5, 6], dtype=torch.int32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    fresh = np.array([7, 8], dtype=np.int32)
    with torch.cuda.graph(graph):
        ops.fork(view, [0, 0], [1, 2], [20, 37], fresh)
        ops.move(view, [5], [2])
    fresh[:] = 0
    for trial in range(3):
        view.block_table[0] = torch.tensor([4, 5, 6], dtype=torch.int32)
        view.data.copy_(torch.from_numpy(rng.integers(0, 256, tuple(view.data.shape), dtype=np.uint8)))
        want = view.data.clone()
        want[:, 7], want[:, 8], want[:, 2] = want[:, 5], want[:, 6], want[:, 5]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(view.data, want)
        assert view.block_table[:3].tolist()[0] == [4, 2, 6] and view.block_table[1, :2].tolist() == [4, 7]
        assert view.block_table[2].tolist() == [4, 2, 8]


def test_graphs_of_one_handle_take_turns(ops):
    """Two captured calls that share the handle's partial results and counters, one after the other, and eager ones between."""
    rng = np.random.default_rng(46)
    calls = []
    for lens, rows, io in (([5000, 30], [1, 2], F32), ([2100, 9], [90, 1], BF16), ([700, 20], [2100, 5], BF16)):
        cache = filled(rng, 1, 0, 2, 128, [0, 1], lens, rows)
        view, batch = cache.device(), CacheBatch([0, 1], lens, rows)
        q = torch.from_numpy(rng.standard_normal((sum(rows), 8, 128))).to(io).cuda()
        want = ops.attention(view, 0, batch, q).clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = ops.attention(view, 0, batch, q)
        calls.append((graph, out, want, (view, 0, batch, q)))
    for trial in range(4):
        for graph, out, want, _ in calls:
            out.zero_()
            graph.replay()
        eager = [ops.attention(*args) for _, _, _, args in calls[::-1]]
        torch.cuda.synchronize()
        for (_, out, want, _), e in zip(calls, eager[::-1]):
            assert torch.equal(out, want) and torch.equal(e, want)


def test_streams_take_turns_and_handles_run_beside_each_other():
    """Calls of one handle on two streams in turn; two handles on two streams at once: the results of calls alone."""
    rng = np.random.default_rng(43)
    a, b = CacheOps(), CacheOps()
    lens, rows = [3000, 100, 7], [1, 2, 1]
    cache = filled(rng, 1, 0, 2, 128, [0, 1, 2], lens, rows)
    view, batch = cache.device(), CacheBatch([0, 1, 2], lens, rows)
    q = [torch.from_numpy(rng.standard_normal((4, 16, 128))).float().cuda() for _ in range(6)]
    want = [a.attention(view, 0, batch, x) for x in q]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for i, x in enumerate(q):
        with torch.cuda.stream((s1, s2)[i % 2]):
            got.append(a.attention(view, 0, batch, x))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    got = []
    for i, x in enumerate(q):
        with torch.cuda.stream((s1, s2)[i % 2]):
            got.append((a, b)[i % 2].attention(view, 0, batch, x))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    a.close(), b.close()


def test_results_do_not_change_from_call_to_call(ops):
    """Splits are merged in a fixed order, whichever arrives last."""
    rng = np.random.default_rng(44)
    for lens, rows, io in (([9000, 300], [1, 1], F32), ([4000], [70], BF16), ([4000], [2100], BF16), ([4000], [2100], F32)):
        cache = filled(rng, 1, 0, 2, 64, list(range(len(lens))), lens, rows)
        view, batch = cache.device(), CacheBatch(list(range(len(lens))), lens, rows)
        q = torch.from_numpy(rng.standard_normal((sum(rows), 8, 64))).to(io).cuda()
        want = ops.attention(view, 0, batch, q)
        for _ in range(5):
            assert torch.equal(ops.attention(view, 0, batch, q), want)
