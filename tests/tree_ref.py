"""Plain 64-bit implementations of the drafted-tree operators, for their tests (numpy on the CPU, nothing of the library).

The cache is held by position here; to_tiles / from_tiles convert to and from the tile order that include/sprout.h
documents, element by element of its formula.
"""
from __future__ import annotations

import numpy as np
import torch


def tile_offsets(elem_size: int, hd: int, values: bool) -> np.ndarray:
    """[16, hd]: offset of element (position, dimension) inside a tile."""
    P = 16 // elem_size
    t, d = np.meshgrid(np.arange(16), np.arange(hd), indexing="ij")
    if not values:
        return ((d // (4 * P)) * 64 + (d % (4 * P)) // P * 16 + t) * P + d % P
    if elem_size == 4:
        return (((d // 16) * 4 + t // 4) * 16 + d % 16) * 4 + t % 4
    return ((((d // 32) * 4 + t // 4) * 16 + d % 16) * 2 + (d // 16) % 2) * 4 + t % 4


def to_tiles(x: torch.Tensor, values: bool) -> torch.Tensor:
    """[..., 16, hd] -> [..., 16 * hd]."""
    off = torch.from_numpy(tile_offsets(x.element_size(), x.shape[-1], values).reshape(-1)).to(x.device)
    out = torch.empty(*x.shape[:-2], 16 * x.shape[-1], dtype=x.dtype, device=x.device)
    out[..., off] = x.reshape(*x.shape[:-2], -1)
    return out


def from_tiles(x: torch.Tensor, values: bool) -> torch.Tensor:
    hd = x.shape[-1] // 16
    off = torch.from_numpy(tile_offsets(x.element_size(), hd, values).reshape(-1)).to(x.device)
    return x[..., off].reshape(*x.shape[:-1], 16, hd)


class Cache:
    """A paged cache of n slots: k, v [layers, blocks, Hkv, 16, hd] by position (CPU) and the block table."""

    def __init__(self, rng, layers, Hkv, hd, positions, dtype, extra_blocks=2, spare=0, fill=None):
        n = len(positions)
        need = [(p + 15) // 16 for p in positions]
        self.mb = max(need) + spare
        nb = sum(need) + extra_blocks
        ids = rng.permutation(nb)
        self.table = np.zeros((n, self.mb), dtype=np.int32)
        at = 0
        for s in range(n):
            self.table[s, :need[s]] = ids[at:at + need[s]]
            at += need[s]
        shape = (layers, nb, Hkv, 16, hd)
        self.k = torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(dtype)
        self.v = torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(dtype)
        if fill is not None:  # everything but the slots' positions
            keep = torch.zeros(nb, 16, dtype=torch.bool)
            for s, p in enumerate(positions):
                for t in range(p):
                    keep[self.table[s, t // 16], t % 16] = True
            for x in (self.k, self.v):
                x.masked_fill_(~keep[None, :, None, :, None], fill)
        self.hd = hd

    def rows(self, x, layer, slot, pos):
        """[len(pos), Hkv, hd] in 64 bits."""
        pos = np.asarray(pos, dtype=np.int64)
        return x[layer, self.table[slot, pos // 16], :, pos % 16].double().numpy()

    def device(self):
        from paper_2403_12900_amd.tree import KVView
        return KVView(to_tiles(self.k, False).cuda().contiguous(), to_tiles(self.v, True).cuda().contiguous(),
                      torch.from_numpy(self.table).cuda())


def ancestors(parents, j):
    out = []
    while j >= 0:
        out.append(j)
        j = parents[j]
    return out


def attention(cache: Cache, layer, slots, lens, trees, q: torch.Tensor) -> np.ndarray:
    """trees: parents per request; q [rows, H, hd].  [rows, H, hd] in 64 bits."""
    q = q.double().numpy()
    H, hd = q.shape[1:]
    Hkv = cache.k.shape[2]
    out = np.empty(q.shape)
    r = 0
    with np.errstate(all="ignore"):
        for s, n, par in zip(slots, lens, trees):
            for j in range(len(par)):
                pos = list(range(n)) + sorted(n + a for a in ancestors(par, j))
                k, v = cache.rows(cache.k, layer, s, pos), cache.rows(cache.v, layer, s, pos)
                z = np.einsum("hd,thd->ht", q[r], np.repeat(k, H // Hkv, 1)) / np.sqrt(hd)
                p = np.exp(z - z.max(1, keepdims=True))
                out[r] = np.einsum("ht,thd->hd", p / p.sum(1, keepdims=True), np.repeat(v, H // Hkv, 1))
                r += 1
    return out


def verify(trees, tokens, logits, accept, sample, draft=None, temperature=None):
    """(emitted, path, count) of the definition, one request after the other; arrays in 64 bits on the host."""
    R = sum(len(p) for p in trees)
    emitted, path = np.full(R, -1, np.int32), np.full(R, -1, np.int32)
    count = np.zeros(len(trees), np.int32)
    r0 = 0
    for i, par in enumerate(trees):
        T = 1.0 if temperature is None else temperature[i]
        node, steps, ok = 0, [], True
        while True:
            z = logits[r0 + node].astype(np.float64)
            if np.isnan(z).any() or not np.isfinite(z.max()):
                ok = False
                break
            steps.append(node)
            if T == 0:
                r = np.zeros_like(z)
                r[np.argmax(z)] = 1.0
            else:
                with np.errstate(over="ignore"):
                    r = np.exp((z - z.max()) / np.float64(np.float32(T)))
                r /= r.sum()
            p, taken = r, None
            for j in range(node + 1, len(par)):
                if par[j] != node:
                    continue
                x = tokens[r0 + j]
                if x < 0 or x >= len(z):
                    if T > 0 and draft is not None:  # rejected like any other child
                        q = np.where(draft[r0 + node] > 0, draft[r0 + node], 0).astype(np.float64)
                        r = np.maximum(r - q, 0)
                        r = r / r.sum() if r.sum() > 0 else np.zeros_like(r)
                    continue
                if T == 0:
                    if r[x] == 1.0:
                        taken = j
                        break
                    continue
                if draft is not None:
                    q = np.where(draft[r0 + node] > 0, draft[r0 + node], 0).astype(np.float64)
                    rest = np.maximum(r - q, 0)
                else:
                    q = np.zeros_like(r)
                    q[x] = 1.0
                    rest = r.copy()
                    rest[x] = 0.0
                if np.float64(accept[r0 + j]) * q[x] < r[x]:
                    taken = j
                    break
                r = rest / rest.sum() if rest.sum() > 0 else np.zeros_like(r)
            if taken is None:
                break
            node = taken
        if ok:
            if T == 0:
                drawn = int(np.argmax(r))
            else:
                if not r.sum() > 0:
                    r = p
                c = np.cumsum(r)
                hit = np.flatnonzero(c > np.float64(sample[i]) * c[-1])
                drawn = int(hit[0]) if len(hit) else int(np.flatnonzero(r > 0)[-1])
            path[r0:r0 + len(steps)] = steps
            emitted[r0:r0 + len(steps)] = [tokens[r0 + j] for j in steps[1:]] + [drawn]
            count[i] = len(steps)
        r0 += len(par)
    return emitted, path, count


def keep(cache: Cache, slots, lens, trees, path, count):
    """In place on the CPU cache."""
    r0 = 0
    for i, (s, n, par) in enumerate(zip(slots, lens, trees)):
        for c in range(count[i]):
            a, b = n + path[r0 + c], n + c
            for x in (cache.k, cache.v):
                x[:, cache.table[s, b // 16], :, b % 16] = x[:, cache.table[s, a // 16], :, a % 16].clone()
        r0 += len(par)


def random_tree(rng, n, kind):
    if kind == "chain":
        return [-1] + list(range(n - 1))
    if kind == "star":
        return [-1] + [0] * (n - 1)
    if kind == "levels":
        return [-1] + [(j - 1) // 3 for j in range(1, n)]
    return [-1] + [int(rng.integers(0, j)) for j in range(1, n)]
