"""The operators of a paged KV cache held in 4 bits as timed cases: rotary positions, appending keys and values to the cache,
attention over it, and forking and compacting its pages.

The cache stores blocks of 32 consecutive dimensions of one position as 4-bit floating point (sign, two exponent bits, one
mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) times a power of two of their own, the smallest that leaves no element off by
more than half a step: 2^s with max|x| <= 7 * 2^s, s in -120 .. 125.  Rounding is to nearest, ties to the even mantissa.

  * "rotary": the first dims of every head are turned by position * frequency, in pairs (d, d + dims / 2) or (2d, 2d + 1);
    frequency k is base^(-2k / dims), for long contexts lowered where it turns seldom over the original length.
  * "append": keys are turned at their cache positions, keys and values are rounded to 4 bits and written to the request's
    blocks; what is stored is read back as values.
  * "attention": row j of a request with len cached positions before the call's rows attends to positions 0 .. len + j.
  * "fork": a request's table row gets another's full blocks and a copy of its last, partly filled one, in every layer.
  * "compact": blocks move to lower places of the pool in every layer, and every table entry that names them follows.

Sizes are those of the package's configurations (heads, layers, batches, context lengths as quantiles of the serving
recipe's lognormal distribution) or generic ones (contexts of tens of thousands of positions, prompts in chunks).
"""
from __future__ import annotations

import math
import statistics

import numpy as np
import torch

own = False

SIGMA = 0.6  # of the serving recipe's lengths

# (query heads, KV heads, head dimension, layers) of the package's models, and one uneven grouped shape.
HEADS = {"tiny": (4, 4, 64, 2), "7b": (32, 32, 128, 32), "13b": (40, 40, 128, 40), "70b": (64, 8, 128, 80), "gqa13": (65, 5, 64, 6)}


def listed():
    return [
        # One decode step's queries of the 7B shape's serving batch: launches and latency.
        {"name": "rotary_7b_b32", "op": "rotary", "heads": 32, "head_dim": 128, "dims": 128, "layout": "half", "factor": 1.0, "io": "bf16", "rows": 32, "far": 1000},
        # A prompt chunk of the 70B shape, positions far past the original length, part of the head, interleaved pairs.
        {"name": "rotary_prompt", "op": "rotary", "heads": 64, "head_dim": 128, "dims": 96, "layout": "pairs", "factor": 16.0, "io": "f32", "rows": 4096, "far": 120000},
        # One decode step's keys and values of the 7B shape's serving batch.
        {"name": "append_7b_b32", "op": "append", "heads": "7b", "layout": "half", "dims": 128, "factor": 1.0, "io": "bf16", "requests": 32, "rows": 1, "median": 400},
        # Prompt chunks of eight requests, grouped heads, fp32, part of the head, long contexts.
        {"name": "append_prompt", "op": "append", "heads": "70b", "layout": "pairs", "dims": 64, "factor": 8.0, "io": "f32", "requests": 8, "rows": 700, "median": 3000},
        # The smallest model, a handful of positions: launches and latency.
        {"name": "attn_tiny_b4", "op": "attention", "heads": "tiny", "io": "f32", "requests": 4, "rows": 1, "median": 24},
        # The serving batch of the 7B shape, one token each.
        {"name": "attn_7b_b32", "op": "attention", "heads": "7b", "io": "f32", "requests": 32, "rows": 1, "median": 400},
        # Eight long conversations, grouped heads, one token each: the cache's bytes.
        {"name": "attn_long_b8", "op": "attention", "heads": "70b", "io": "bf16", "requests": 8, "rows": 1, "median": 24000},
        # A long prompt's chunk of 2048 tokens over what is cached already, 7B shape: the products.
        {"name": "attn_prompt", "op": "attention", "heads": "7b", "io": "bf16", "requests": 1, "rows": 2048, "median": 6150},
        # Eight continuations of one prompt, 7B shape, all layers.
        {"name": "fork_7b_x8", "op": "fork", "heads": "7b", "kv": "mx4", "sources": 1, "forks": 8, "median": 200},
        # Three directives' prompts shared by sixty requests, 13B shape with its bf16 cache.
        {"name": "fork_13b_x60", "op": "fork", "heads": "13b", "kv": "bf16", "sources": 3, "forks": 60, "median": 200},
        # The smallest model with its fp32 cache: launches and latency.
        {"name": "compact_tiny", "op": "compact", "heads": "tiny", "kv": "f32", "blocks": 40, "live": 20, "slots": 6},
        # A pool of the 7B shape two thirds full after requests have come and gone, all layers.
        {"name": "compact_7b", "op": "compact", "heads": "7b", "kv": "mx4", "blocks": 768, "live": 500, "slots": 32},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any of the operators: 1 to 64 requests, 1 to 2048 rows each, contexts of 1 to 24000 positions, all head shapes."""
    op = rng.choice(["rotary", "append", "attention", "attention", "attention", "fork", "compact"])
    if op == "rotary":
        hd = rng.choice([64, 128])
        heads = _log_int(rng, 1, 64)
        return {"op": op, "heads": heads, "head_dim": hd, "dims": rng.choice([hd, hd, hd // 2, 2 * rng.randint(1, hd // 2)]), "layout": rng.choice(["half", "pairs"]),
                "factor": rng.choice([1.0, 4.0, 32.0]), "io": rng.choice(["f32", "bf16"]), "rows": _log_int(rng, 1, 4096), "far": _log_int(rng, 100, 1000000)}
    heads = rng.choice(sorted(HEADS))
    H, Hkv, hd, layers = HEADS[heads]
    if op == "append":
        requests = _log_int(rng, 1, 64)
        return {"op": op, "heads": heads, "layout": rng.choice(["half", "pairs"]), "dims": rng.choice([0, hd, hd, hd // 2, 2 * rng.randint(1, hd // 2)]), "factor": rng.choice([1.0, 1.0, 8.0]),
                "io": rng.choice(["f32", "bf16"]), "requests": requests, "rows": _log_int(rng, 1, max(1, 45000 // (requests * Hkv))), "median": _log_int(rng, 1, 8000)}
    if op == "attention":
        requests = _log_int(rng, 1, 64)
        rows = rng.choice([1, 1, _log_int(rng, 2, 40), _log_int(rng, 40, max(41, 2048 // requests))])
        # At most the cache bytes and the products of the largest listed cases.
        top = min(24000, 24000 * 8 * 8 * 128 // (requests * Hkv * hd), 32 * 2048 * 2000 // (H * rows * requests))
        return {"op": op, "heads": heads, "io": rng.choice(["f32", "bf16", "bf16"]), "requests": requests, "rows": rows, "median": _log_int(rng, 1, max(2, top))}
    kv = rng.choice(["mx4", "mx4", "bf16", "f32"])
    wide = {"mx4": 1.0625, "bf16": 4, "f32": 8}[kv] * 16 * hd * Hkv * layers  # bytes of a block
    if op == "fork":
        forks = _log_int(rng, 1, max(1, min(60, int(7.5e8 / wide))))
        return {"op": op, "heads": heads, "kv": kv, "sources": rng.randint(1, min(4, forks)), "forks": forks, "median": _log_int(rng, 4, 300)}
    blocks = _log_int(rng, 8, max(9, min(1000, int(1.6e9 / wide))))
    return {"op": op, "heads": heads, "kv": kv, "blocks": blocks, "live": max(1, int(blocks * rng.uniform(0.2, 0.9))), "slots": rng.randint(1, 40)}


# ---------------------------------------------------------------------------------------------------------------- shapes


def _quantiles(n, median):
    """n lengths: quantiles of the recipe's lognormal distribution around the median."""
    z = statistics.NormalDist()
    return [max(1, round(median * math.exp(SIGMA * z.inv_cdf((i + 0.5) / n)))) for i in range(n)]


def _requests(case):
    """Cached positions and rows of each request; every third of several has a row or two fewer."""
    n = case["requests"]
    rows = [max(1, case["rows"] - (i % 3 if n > 2 else 0)) for i in range(n)]
    lens = _quantiles(n, case["median"])
    if n > 4:
        lens[1] = 0  # a request's first rows
    return lens, rows


def _size(name):
    return {"f32": 4, "bf16": 2}[name]


def _block_bytes(case):
    """Of one block in one layer, keys and values."""
    _, Hkv, hd, _ = HEADS[case["heads"]]
    return Hkv * hd * (17 if case["kv"] == "mx4" else 32 * _size(case["kv"]))


def work(case):
    op = case["op"]
    if op == "rotary":
        n = case["rows"] * case["heads"]
        return {"bytes": 2 * n * case["head_dim"] * _size(case["io"]) + 4 * case["rows"], "flops": 3 * n * case["dims"]}
    H, Hkv, hd, layers = HEADS[case["heads"]]
    if op in ("append", "attention"):
        lens, rows = _requests(case)
        R, io = sum(rows), _size(case["io"])
        if op == "append":  # keys and values in, stored, read, out
            return {"bytes": 2 * R * Hkv * hd * (2 * io + 2 * 17 / 32), "flops": R * Hkv * (3 * case["dims"] + 4 * hd)}
        seen = sum(n * length + n * (n + 1) // 2 for length, n in zip(lens, rows))
        cached = sum(length + n for length, n in zip(lens, rows))
        return {"bytes": cached * Hkv * hd * 17 / 16 + 2 * R * H * hd * io, "flops": 4 * H * hd * seen}
    if op == "fork":
        lens = _quantiles(case["sources"], case["median"])
        parts = [lens[i % len(lens)] % 16 != 0 for i in range(case["forks"])]
        read = sum(length % 16 != 0 for length in lens)
        rows = sum(lens[i % len(lens)] // 16 + 1 for i in range(case["forks"]))
        return {"bytes": (read + sum(parts)) * layers * _block_bytes(case) + 8 * rows, "flops": 0}
    moved = case["live"] - case["live"] * case["live"] // case["blocks"]  # see _inputs: live blocks lie evenly
    return {"bytes": 2 * moved * layers * _block_bytes(case) + 8 * case["blocks"], "flops": 0}


# ---------------------------------------------------------------------------------------------------------------- inputs


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _place(hd, device):
    """[16, 17 * hd / 16]: where the bytes of position t lie in a tile.  A position's bytes are those of its key (byte j:
    dims 2j, 2j + 1), of its value (byte 16p + e: dims 32p + e, 32p + 16 + e), its key's scales and its value's."""
    P = hd // 32
    t = torch.arange(16, device=device)[:, None]
    j = torch.arange(hd // 2, device=device)[None, :]
    g = torch.arange(P, device=device)[None, :]
    k = (j // 16 * 16 + t) * 16 + j % 16
    v = 8 * hd + ((t // 4 * 16 + j % 16) * P + j // 16) * 4 + t % 4
    return torch.cat([k, v, 16 * hd + g * 16 + t, 16 * hd + hd // 2 + (t // 4 * P + g) * 4 + t % 4], 1)


def _codes(x):
    """x [..., 32 n] in 4 bits: codes 0 .. 15 like x, and the scales' exponents [..., n]."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)  # top = m 2^e, 0.5 <= m < 1
    s = torch.where(top > 0, e - 3 + (m > 0.875), -120).clamp(-120, 125)
    y = torch.ldexp(x, -s[..., None])
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp_max(6)
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code += 8 * torch.signbit(x).to(torch.uint8)
    return code.flatten(-2), s


def _records(k, v):
    """The bytes of each (position, head): k, v [..., hd] -> uint8 [..., 17 * hd / 16]."""
    ck, sk = _codes(k)
    cv, sv = _codes(v)
    ck, cv = ck.unflatten(-1, (-1, 2)), cv.unflatten(-1, (-1, 2, 16))
    byte = lambda s: (s + 127).to(torch.uint8)  # noqa: E731
    return torch.cat([ck[..., 0] + 16 * ck[..., 1], (cv[..., 0, :] + 16 * cv[..., 1, :]).flatten(-2), byte(sk), byte(sv)], -1)


def _values(rec, hd):
    """Keys and values in 32 bits that records stand for."""
    P = hd // 32
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=rec.device)
    rec = rec.int()
    k, v = rec[..., :hd // 2], rec[..., hd // 2:hd].unflatten(-1, (P, 16))
    k = table[torch.stack([k & 15, k >> 4], -1).flatten(-2)].unflatten(-1, (P, 32))
    v = table[torch.stack([v & 15, v >> 4], -2).flatten(-2)]
    k = torch.ldexp(k, rec[..., hd:hd + P, None] - 127)
    v = torch.ldexp(v, rec[..., hd + P:, None] - 127)
    return k.flatten(-2), v.flatten(-2)


def _inputs(case, seed):
    """What the seed makes: tensors on the GPU and the host's arrays."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = np.random.default_rng(seed)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    op = case["op"]
    s = {"case": case, "op": op}
    if op == "rotary":
        R, H, hd = case["rows"], case["heads"], case["head_dim"]
        first = int(host.integers(0, case["far"]))
        # A prompt's rows, or tokens of requests at places of their own.
        pos = first + np.arange(R) if R > 200 else host.integers(0, case["far"], R)
        s["positions"] = torch.from_numpy(pos.astype(np.int32)).cuda()
        # Query rows as a projection of queries, keys and values leaves them.
        s["x"] = randn(R, H + 2, hd).to(_dtype(case["io"]))[:, :H]
        return s
    H, Hkv, hd, layers = HEADS[case["heads"]]
    if op in ("append", "attention"):
        lens, rows = _requests(case)
        B, R = len(lens), sum(rows)
        s["lens"], s["rows"] = np.array(lens, dtype=np.int32), np.array(rows, dtype=np.int32)
        s["slots"] = host.permutation(B).astype(np.int32)
        blocks = [(length + n + 15) // 16 for length, n in zip(lens, rows)]
        NB = sum(blocks)
        ids = host.permutation(NB)  # a pool that requests have come and gone in
        table = np.zeros((B, max(blocks)), dtype=np.int32)
        at = 0
        for i, n in enumerate(blocks):
            table[s["slots"][i], :n] = ids[at:at + n]
            at += n
        s["table"] = torch.from_numpy(table).cuda()
        # Keys have a few large dimensions, as trained models' do.
        gain = torch.exp(0.5 * randn(Hkv, hd))
        if op == "append":
            s["pool"] = torch.randint(0, 120, (1, NB, Hkv, 17 * hd), generator=g, device="cuda", dtype=torch.uint8)
            x = randn(R, 2 * Hkv, hd)
            x[:, :Hkv] *= gain
            x = x.to(_dtype(case["io"]))
            s["k"], s["v"] = x[:, :Hkv], x[:, Hkv:]
            return s
        s["pool"] = torch.empty(1, NB, Hkv, 17 * hd, dtype=torch.uint8, device="cuda")
        place = _place(hd, "cuda").flatten()
        for b in range(0, NB, 2048):
            n = min(2048, NB - b)
            s["pool"][0, b:b + n][..., place] = _records(randn(n, Hkv, 16, hd) * gain[:, None], randn(n, Hkv, 16, hd)).flatten(-2)
        s["q"] = (1.2 * randn(R, H + 2 * Hkv, hd)).to(_dtype(case["io"]))[:, :H]
        return s
    # Pages: blocks of keys and values as bytes of a 4-bit cache or as two tensors.
    if op == "fork":
        lens = _quantiles(case["sources"], case["median"])
        blocks = [(length + 15) // 16 for length in lens]
        S, F = case["sources"], case["forks"]
        NB = sum(blocks) + F + 5
        ids = host.permutation(NB).astype(np.int32)
        slots = host.permutation(S + F).astype(np.int32)
        table = host.integers(0, NB, (S + F, max(blocks) + 4)).astype(np.int32)
        at = 0
        for i, n in enumerate(blocks):
            table[slots[i], :n] = ids[at:at + n]
            at += n
        s["source"], s["target"] = slots[np.arange(F) % S], slots[S:]
        s["lens"] = np.array([lens[i % S] for i in range(F)], dtype=np.int32)
        s["fresh"] = ids[at:at + F]
    else:
        NB, live, slots = case["blocks"], case["live"], case["slots"]
        used = np.arange(live) * NB // live  # every NB / live-th block, as far as whole numbers go
        holes = np.setdiff1d(np.arange(live), used)
        s["src"] = host.permutation(used[used >= live]).astype(np.int32)
        s["dst"] = holes[:len(s["src"])].astype(np.int32)
        table = used[host.integers(0, live, (slots, 2 * live // slots + 3))].astype(np.int32)  # a few blocks are shared
    s["table"] = torch.from_numpy(table).cuda()
    if case["kv"] == "mx4":
        s["pool"] = torch.randint(0, 256, (layers, NB, Hkv, 17 * hd), generator=g, device="cuda", dtype=torch.uint8)
    else:
        s["k"], s["v"] = (torch.empty(layers, NB, Hkv, 16 * hd, dtype=_dtype(case["kv"]), device="cuda").normal_(generator=g) for _ in range(2))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("append", "attention"):
        # The plan of the plain forms: the request and the place in it of every row.
        lens, rows = s["lens"].astype(np.int64), s["rows"].astype(np.int64)
        B, start = len(rows), np.concatenate([[0], np.cumsum(rows)])
        cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        req = np.repeat(np.arange(B), rows)
        local = np.arange(start[-1]) - start[:-1][req]
        s["req"], s["local"], s["position"] = cuda(req), cuda(local), cuda(lens[req] + local)
        s["rows_of"] = cuda(start[:-1][:, None] + np.minimum(np.arange(rows.max())[None, :], rows[:, None] - 1))  # [B, N], padded
        s["lens_dev"], s["slots_dev"] = cuda(lens), cuda(s["slots"].astype(np.int64))
        s["place"] = _place(HEADS[case["heads"]][2], "cuda")
    if own:
        from paper_2403_12900_amd.cache import CacheBatch, CacheOps, KV4View, Rotary
        from paper_2403_12900_amd.tree import KVView
        s["ops"] = CacheOps()
        if op == "rotary" or op == "append" and case["dims"]:
            s["rotary"] = Rotary(case["dims"], layout=case["layout"], **_scaling(case))
        if op in ("append", "attention"):
            s["batch"] = CacheBatch(s["slots"], s["lens"], s["rows"])
        if op != "rotary":
            s["view"] = KV4View(s["pool"], s["table"]) if "pool" in s else KVView(s["k"], s["v"], s["table"])
    return s


def _scaling(case):
    """Contexts `factor` times the 8192 positions that a model was made for: frequencies that turn less than once over
    those are divided by the factor, ones that turn more than 32 times are kept."""
    if case["factor"] == 1.0:
        return {"base": 10000.0}
    return {"base": 500000.0, "factor": case["factor"], "original": 8192, "low": 1.0, "high": 32.0, "amplitude": 0.1 * math.log(case["factor"]) + 1}


# ------------------------------------------------------------------------------------------------------------ the passes


def run(s):
    op, case = s["op"], s["case"]
    if op == "rotary":
        return s["ops"].rotary(s["rotary"], s["x"], s["positions"]) if own else _turn(s["x"], s["positions"], case).to(s["x"].dtype)
    if op == "append":
        if own:
            s["ops"].append(s["view"], 0, s["batch"], s["k"], s["v"], rotary=s.get("rotary"))
            return s["ops"].read(s["view"], 0, s["batch"], dtype=s["k"].dtype)
        return _append(s)
    if op == "attention":
        return s["ops"].attention(s["view"], 0, s["batch"], s["q"]) if own else _attention(s)
    if op == "fork":
        if own:
            s["ops"].fork(s["view"], s["source"], s["target"], s["lens"], s["fresh"])
        else:
            _fork(s)
    elif own:
        s["ops"].move(s["view"], s["src"], s["dst"])
    else:
        _compact(s)
    return (s["table"], s["pool"]) if "pool" in s else (s["table"], s["k"], s["v"])


def _turn(x, positions, case):
    """x [rows, heads, hd] turned at its positions, in 64 bits (angles of far positions, values next to a rounding border)."""
    n, sc = case["dims"], _scaling(case)
    w = sc["base"] ** (-torch.arange(0, n, 2, device=x.device, dtype=torch.float64) / n)
    if "factor" in sc:
        keep = ((sc["original"] * w / (2 * math.pi) - sc["low"]) / (sc["high"] - sc["low"])).clamp(0, 1)
        w = w * (keep + (1 - keep) / sc["factor"])
    angle = positions.double()[:, None, None] * w
    amp = sc.get("amplitude", 1.0)
    c, si = amp * torch.cos(angle), amp * torch.sin(angle)
    x = x.double()
    if case["layout"] == "half":
        a, b = x[..., :n // 2], x[..., n // 2:n]
        return torch.cat([a * c - b * si, b * c + a * si, x[..., n:]], -1)
    a, b = x[..., 0:n:2], x[..., 1:n:2]
    return torch.cat([torch.stack([a * c - b * si, b * c + a * si], -1).flatten(-2), x[..., n:]], -1)


def _append(s):
    case = s["case"]
    hd = HEADS[case["heads"]][2]
    k = _turn(s["k"], s["position"], case) if case["dims"] else s["k"].double()
    rec = _records(k, s["v"].double())  # [rows, KV heads, bytes]
    block = s["table"][s["slots_dev"][s["req"]], s["position"] // 16].long()
    at = (block[:, None, None], torch.arange(rec.shape[1], device=block.device)[None, :, None], s["place"][s["position"] % 16][:, None, :])
    s["pool"][0][at] = rec
    k, v = _values(s["pool"][0][at], hd)
    return k.to(s["k"].dtype), v.to(s["v"].dtype)


def _attention(s):
    H, Hkv, hd, _ = HEADS[s["case"]["heads"]]
    G = H // Hkv
    idx = s["table"][s["slots_dev"]].long()  # [B, blocks]
    B, nb = idx.shape
    N = s["rows_of"].shape[1]
    rec = s["pool"][0][idx].transpose(1, 2)[..., s["place"]].flatten(2, 3)  # [B, KV heads, positions, bytes]
    k, v = _values(rec, hd)
    del rec
    # What lies behind the request's last position does not count, whatever it is.
    t = torch.arange(nb * 16, device=idx.device)
    last = s["lens_dev"] + torch.from_numpy(s["rows"]).to(idx.device)
    v = torch.where((t < last[:, None])[:, None, :, None], v, 0)
    q = s["q"].float()[s["rows_of"]].view(B, N, Hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * N, hd)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(hd)
    sees = t <= (s["lens_dev"][:, None] + torch.arange(N, device=idx.device))[:, :, None]  # [B, N, positions]
    scores.view(B, Hkv, G, N, -1).masked_fill_(~sees[:, None, None], -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    out = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    out = out.view(B, Hkv, G, N, hd).permute(0, 3, 1, 2, 4).reshape(B, N, H, hd)
    return out[s["req"], s["local"]].to(s["q"].dtype)


def _pools(s):
    return (s["pool"],) if "pool" in s else (s["k"], s["v"])


def _fork(s):
    dev = s["table"].device
    to = lambda a: torch.from_numpy(a).to(dev).long()  # noqa: E731
    source, target, lens, fresh = to(s["source"]), to(s["target"]), to(s["lens"]), to(s["fresh"])
    full = lens // 16
    entry = torch.arange(s["table"].shape[1], device=dev)
    rows = torch.where(entry < full[:, None], s["table"][source], s["table"][target])
    old = torch.where(lens % 16 > 0, s["table"][source, full].long(), fresh)  # nothing to copy: onto itself
    part = (entry == full[:, None]) & (lens % 16 > 0)[:, None]
    s["table"][target] = torch.where(part, fresh[:, None].int(), rows)
    _copy(_pools(s)[0], old, fresh)
    if "pool" not in s:
        _copy(s["v"], old, fresh)


def _copy(pool, src, dst):
    pool[:, dst] = pool[:, src]


def _compact(s):
    dev = s["table"].device
    src, dst = torch.from_numpy(s["src"]).to(dev).long(), torch.from_numpy(s["dst"]).to(dev).long()
    _copy(_pools(s)[0], src, dst)
    if "pool" not in s:
        _copy(s["v"], src, dst)
    now = torch.arange(s["case"]["blocks"], device=dev, dtype=torch.int32)
    now[src] = dst.int()
    s["table"].copy_(now[s["table"].long()])


# ---------------------------------------------------------------------------------------------------- results in 64 bits


GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def exact(case, seed):
    s = _inputs(case, seed)
    return {"rotary": _exact_rotary, "append": _exact_append, "attention": _exact_attention, "fork": _exact_fork, "compact": _exact_compact}[case["op"]](case, s)


def _exact_turn(x, positions, case):
    """Pair by pair as a complex number."""
    n, out = case["dims"], x.double().clone()
    sc = _scaling(case)
    pos = positions.double()
    for k in range(n // 2):
        w = math.exp(-2 * k / n * math.log(sc["base"]))
        if "factor" in sc:
            turns = sc["original"] * w / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - sc["low"]) / (sc["high"] - sc["low"])))
            w = keep * w + (1 - keep) * w / sc["factor"]
        i, j = (k, k + n // 2) if case["layout"] == "half" else (2 * k, 2 * k + 1)
        z = torch.complex(out[..., i], out[..., j]) * torch.polar(torch.full_like(pos, sc.get("amplitude", 1.0)), pos * w)[:, None]
        out[..., i], out[..., j] = z.real, z.imag
    return out


def _exact_rotary(case, s):
    return _exact_turn(s["x"], s["positions"], case)


def _exact_stored(x):
    """The value nearest to each element among the block's, the even one of two as near."""
    out = torch.empty_like(x)
    for at in range(0, x.shape[-1], 32):
        b = x[..., at:at + 32]
        top = b.abs().amax(-1, keepdim=True)
        scale = torch.full_like(top, 2.0 ** -120)
        for e in range(-119, 126):
            scale = torch.where(top > 7 * 2.0 ** (e - 1), 2.0 ** e, scale)
        a = b.abs() / scale
        best = torch.zeros_like(a)
        for i in range(1, 8):
            mid = (GRID[i - 1] + GRID[i]) / 2
            best = torch.where((a > mid) | ((a == mid) if i % 2 == 0 else False), GRID[i], best)
        out[..., at:at + 32] = torch.copysign(best, b) * scale
    return out


def _exact_append(case, s):
    pos = torch.from_numpy(np.concatenate([length + np.arange(n) for length, n in zip(s["lens"], s["rows"])])).cuda()
    k = _exact_turn(s["k"], pos, case) if case["dims"] else s["k"].double()
    return _exact_stored(k), _exact_stored(s["v"].double())


def _rows_of_cache(pool, blocks, n, hd, values):
    """Keys (or values) of the first n positions of the blocks, [KV heads, n, hd] in 64 bits, element by element."""
    pos = torch.arange(n, device=pool.device)[:, None]
    d = torch.arange(hd, device=pool.device)[None, :]
    t, P = pos % 16, hd // 32
    if values:
        code, high = 8 * hd + (t // 4 * 16 + d % 16) * 4 * P + d // 32 * 4 + t % 4, (d // 16 % 2).expand(n, hd)
        scale = 16 * hd + hd // 2 + t // 4 * 4 * P + d // 32 * 4 + t % 4
    else:
        code, high = d // 32 * 256 + t * 16 + d % 32 // 2, (d % 2).expand(n, hd)
        scale = 16 * hd + d // 32 * 16 + t
    tiles = pool[0][blocks[pos[:, 0] // 16].long()].transpose(0, 1)  # [KV heads, positions, bytes]
    byte = lambda at: torch.gather(tiles, 2, at.expand(tiles.shape[0], n, hd)).int()  # noqa: E731
    c = byte(code) >> 4 * high & 15
    mag = torch.tensor(GRID, dtype=torch.float64, device=pool.device)[c & 7]
    return torch.where(c > 7, -mag, mag) * torch.exp2((byte(scale) - 127).double())


def _exact_attention(case, s):
    H, Hkv, hd, _ = HEADS[case["heads"]]
    out, r0 = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0
    for i, (length, n) in enumerate(zip(s["lens"].tolist(), s["rows"].tolist())):
        blocks = s["table"][int(s["slots"][i])]
        k, v = (_rows_of_cache(s["pool"], blocks, length + n, hd, x) for x in (False, True))
        hidden = torch.arange(length + n, device="cuda")[None, :] > length + torch.arange(n, device="cuda")[:, None]
        for h in range(H):
            z = s["q"][r0:r0 + n, h].double() @ k[h // (H // Hkv)].T.contiguous() / math.sqrt(hd)
            out[r0:r0 + n, h] = torch.softmax(z.masked_fill(hidden, -math.inf), 1) @ v[h // (H // Hkv)]
        r0 += n
    return out


def _exact_fork(case, s):
    table = s["table"].cpu().numpy()
    for a, b, length, new in zip(s["source"].tolist(), s["target"].tolist(), s["lens"].tolist(), s["fresh"].tolist()):
        table[b, :length // 16] = table[a, :length // 16]
        if length % 16:
            table[b, length // 16] = new
            for pool in _pools(s):
                pool[:, new] = pool[:, int(table[a, length // 16])].clone()
    return (torch.from_numpy(table).cuda(), *_pools(s))


def _exact_compact(case, s):
    table = s["table"].cpu().numpy()
    new = table.copy()
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        new[table == a] = b
        for pool in _pools(s):
            pool[:, b] = pool[:, a].clone()
    return (torch.from_numpy(new).cuda(), *_pools(s))
