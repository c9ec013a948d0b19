"""Plain 64-bit implementations of the 4-bit cache's operators, for their tests (numpy on the CPU, nothing of the library).

A cache is held by position here, as the values it stands for; to_bytes puts them into the tiles that include/sprout.h
documents, byte by byte of its formulas.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantise(x: np.ndarray):
    """x [..., 32 n] in 64 bits: codes 0 .. 15 like x, and scale bytes [..., n]."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(g).max(-1)
    nan = ~np.isfinite(g).all(-1)
    s = np.full(top.shape, -120)
    for e in range(-119, 126):  # the smallest s with top <= 7 * 2^s, as far as 125
        s = np.where(top > 7.0 * 2.0 ** (e - 1), e, s)
    a = np.where(nan[..., None], 0.0, np.abs(g)) / 2.0 ** s[..., None].astype(np.float64)
    d = np.abs(a[..., None] - GRID)
    code = d.argmin(-1)  # the first of two as near; the next one where that is odd
    tie = (code < 7) & (np.take_along_axis(d, np.minimum(code + 1, 7)[..., None], -1)[..., 0] == d.min(-1))
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    code = np.where(nan[..., None], 0, code + 8 * np.signbit(g))
    return code.reshape(x.shape).astype(np.uint8), np.where(nan, 255, s + 127).astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    c = codes.reshape(*codes.shape[:-1], -1, 32)
    v = np.where(c >= 8, -1.0, 1.0) * GRID[c & 7]
    s = scales.astype(np.float64)
    return (v * np.where(scales == 255, np.nan, 2.0 ** (s - 127))[..., None]).reshape(codes.shape)


def offsets(hd: int):
    """Of a tile's element (t, d): key byte, value byte, key scale, value scale; and whether its nibble is the high one."""
    t, d = np.meshgrid(np.arange(16), np.arange(hd), indexing="ij")
    P = hd // 32
    key = (d // 32 * 16 + t) * 16 + d % 32 // 2
    value = 8 * hd + ((t // 4 * 16 + d % 16) * P + d // 32) * 4 + t % 4
    return (key, value, 16 * hd + d // 32 * 16 + t, 16 * hd + hd // 2 + (t // 4 * P + d // 32) * 4 + t % 4, d % 2 == 1, d % 32 >= 16)


def put(tile: np.ndarray, t: int, kc, ks, vc, vs):
    """Writes position t of one tile [17 * hd]: codes [hd] and scales [hd / 32] of its key and value."""
    hd = len(kc)
    ko, vo, kso, vso, khi, vhi = (o[t] for o in offsets(hd))
    for at, code, high in ((ko, kc, khi), (vo, vc, vhi)):
        byte = np.zeros(17 * hd, np.int64)
        np.add.at(byte, at, code.astype(np.int64) << np.where(high, 4, 0))
        tile[np.unique(at)] = byte[np.unique(at)]
    tile[kso] = np.repeat(ks, 32)
    tile[vso] = np.repeat(vs, 32)


def get(tiles: np.ndarray):
    """Values of tiles [..., 17 * hd]: keys and values [..., 16, hd]."""
    hd = tiles.shape[-1] // 17
    ko, vo, kso, vso, khi, vhi = offsets(hd)
    out = []
    for at, so, high in ((ko, kso, khi), (vo, vso, vhi)):
        code = tiles[..., at] >> np.where(high, 4, 0) & 15
        out.append(values(code, tiles[..., so][..., ::32]))
    return out


def turn(x: np.ndarray, positions, dims, layout="half", base=10000.0, factor=1.0, original=0.0, low=1.0, high=32.0, amplitude=1.0):
    """x [rows, heads, hd] in 64 bits at its positions; the angle's whole turns taken off in long double."""
    k = np.arange(dims // 2)
    w = np.longdouble(base) ** (-2.0 * k.astype(np.longdouble) / dims)
    pi = np.longdouble("3.14159265358979323846264338327950288")
    if factor > 1:
        keep = np.clip((original * w / (2 * pi) - low) / (np.longdouble(high) - low), 0, 1)
        w = w * (keep + (1 - keep) / factor)
    a = np.asarray(positions).astype(np.longdouble)[:, None] * w
    a = a - 2 * pi * np.rint(a / (2 * pi))
    z = (np.cos(a) + 1j * np.sin(a)).astype(np.complex128)[:, None, :] * amplitude
    out = x.astype(np.float64).copy()
    i, j = (k, k + dims // 2) if layout == "half" else (2 * k, 2 * k + 1)
    y = (out[..., i] + 1j * out[..., j]) * z
    out[..., i], out[..., j] = y.real, y.imag
    return out


class Cache:
    """A cache of slots with room for `positions` each: its bytes [layers, blocks, Hkv, 17 * hd] and block table."""

    def __init__(self, rng, layers, Hkv, hd, positions, extra_blocks=2, spare=0, fill="random"):
        n = len(positions)
        need = [(p + 15) // 16 for p in positions]
        self.hd, self.Hkv, self.mb = hd, Hkv, max(max(need), 1) + spare
        nb = sum(need) + extra_blocks
        ids = rng.permutation(nb)
        self.table = np.zeros((n, self.mb), dtype=np.int32)
        at = 0
        for s in range(n):
            self.table[s, :need[s]] = ids[at:at + need[s]]
            at += need[s]
        self.free = [int(b) for b in ids[at:]]
        shape = (layers, nb, Hkv, 17 * hd)
        self.data = rng.integers(0, 256, shape, dtype=np.uint8) if fill == "random" else np.full(shape, fill, np.uint8)

    def append(self, layer, slot, first, k, v):
        """k, v [rows, Hkv, hd] in 64 bits."""
        kc, ks = quantise(k)
        vc, vs = quantise(v)
        for r in range(len(k)):
            block = self.table[slot, (first + r) // 16]
            for h in range(self.Hkv):
                put(self.data[layer, block, h], (first + r) % 16, kc[r, h], ks[r, h], vc[r, h], vs[r, h])

    def rows(self, layer, slot, n):
        """Keys and values [n, Hkv, hd] of the first n positions."""
        k, v = get(self.data[layer, self.table[slot, :(n + 15) // 16]])  # [blocks, Hkv, 16, hd]
        return [x.transpose(0, 2, 1, 3).reshape(-1, self.Hkv, self.hd)[:n] for x in (k, v)]

    def device(self):
        import torch
        from paper_2403_12900_amd.cache import KV4View
        return KV4View(torch.from_numpy(self.data).cuda(), torch.from_numpy(self.table).cuda())


def attention(cache: Cache, layer, slots, lens, rows, q: np.ndarray) -> np.ndarray:
    """q [rows, H, hd] in 64 bits."""
    H, hd = q.shape[1:]
    G = H // cache.Hkv
    out, r0 = np.empty(q.shape), 0
    for slot, length, n in zip(slots, lens, rows):
        k, v = cache.rows(layer, slot, length + n)
        for h in range(H):
            kh, vh = k[:, h // G], v[:, h // G]
            if np.isfinite(kh).all() and np.isfinite(vh).all():  # all rows at once: nothing masked is infinite or NaN
                s = np.where(np.arange(length + n) <= length + np.arange(n)[:, None], q[r0:r0 + n, h] @ kh.T / np.sqrt(hd), -np.inf)
                p = np.exp(s - s.max(-1, keepdims=True))
                out[r0:r0 + n, h] = (p @ vh) / p.sum(-1, keepdims=True)
                continue
            for j in range(n):
                see = length + j + 1
                s = kh[:see] @ q[r0 + j, h] / np.sqrt(hd)
                p = np.exp(s - s.max())
                out[r0 + j, h] = (p @ vh[:see]) / p.sum()
        r0 += n
    return out
