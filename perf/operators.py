"""The operators of speculative decoding as timed cases: attention of a tree of drafted tokens over the paged KV cache,
verification of the drafted tokens against the target's probabilities, and the compaction of the cache onto the accepted
path.

A drafted tree of one request holds the last committed token as node 0 and drafted tokens as nodes 1 .. n - 1, each after
its parent.  Node j's keys and values sit at cache position len + j.

  * "attention": every node attends to the len cached positions, to its ancestors and to itself.
  * "verify": from the root down, the children of a node are tried in their order: child x is accepted where
    u q(x) < r(x), r the target's distribution at the node after the rejections so far and q the distribution that the
    children were drawn from (without one: a point mass at x); past the last child the next token is drawn from r by
    inversion of its cumulative sum.  Temperature 0 accepts the argmax and emits it.
  * "keep": the accepted nodes' keys and values move to positions len .. len + count - 1 of every layer.

Sizes are those of the package's configurations (heads, vocabularies, batches, context lengths as quantiles of the serving
recipe's lognormal distribution) or generic ones (a vocabulary of 131072, contexts of tens of thousands of positions).
"""
from __future__ import annotations

import math
import statistics

import numpy as np
import torch

own = False

SIGMA = 0.6     # of the serving recipe's lengths
MAX_ROWS = 128  # token rows of one pass

# (query heads, KV heads, head dimension) of the package's models, and one uneven grouped shape.
HEADS = {"tiny": (4, 4, 64), "7b": (32, 32, 128), "13b": (40, 40, 128), "70b": (64, 8, 128), "gqa13": (65, 5, 64)}


def listed():
    return [
        # The smallest model, fp32 cache, a handful of positions: launches and latency.
        {"name": "attn_tiny_b4", "op": "attention", "heads": "tiny", "kv": "f32", "io": "f32", "rows": 4, "nodes": 3, "width": 1, "median": 24},
        # One interactive request of the 7B shape with a tree of 8 drafted tokens.
        {"name": "attn_7b_b1", "op": "attention", "heads": "7b", "kv": "bf16", "io": "f32", "rows": 1, "nodes": 9, "width": 2, "median": 600},
        # The serving batch of the 7B shape, short chains: as many token rows as one pass takes.
        {"name": "attn_7b_b32", "op": "attention", "heads": "7b", "kv": "bf16", "io": "f32", "rows": 32, "nodes": 4, "width": 1, "median": 400},
        # The 70B shape (grouped heads, fp32 cache) at its configuration's batch.
        {"name": "attn_70b_b16", "op": "attention", "heads": "70b", "kv": "f32", "io": "f32", "rows": 16, "nodes": 8, "width": 2, "median": 700},
        # Two long conversations with wide trees, grouped heads, bf16 throughout.
        {"name": "attn_long_b2", "op": "attention", "heads": "70b", "kv": "bf16", "io": "bf16", "rows": 2, "nodes": 64, "width": 4, "median": 24000},
        # One interactive request: a chain of four drafted tokens without draft probabilities (n-gram drafts).
        {"name": "verify_b1", "op": "verify", "vocab": 32000, "rows": 1, "nodes": 5, "width": 1, "draft": False, "dtype": "f32", "temperature": 1.0, "greedy_every": 0},
        # The serving batch, every request greedy.
        {"name": "verify_b32_greedy", "op": "verify", "vocab": 32000, "rows": 32, "nodes": 4, "width": 1, "draft": False, "dtype": "f32", "temperature": 1.0, "greedy_every": 1},
        # Trees drafted by a smaller model, with its probabilities; a few requests greedy.
        {"name": "verify_b16_draft", "op": "verify", "vocab": 32000, "rows": 16, "nodes": 8, "width": 2, "draft": True, "dtype": "f32", "temperature": 0.8, "greedy_every": 5},
        # A large vocabulary, bf16 logits and draft probabilities, wide trees.
        {"name": "verify_v131072", "op": "verify", "vocab": 131072, "rows": 4, "nodes": 32, "width": 4, "draft": True, "dtype": "bf16", "temperature": 1.2, "greedy_every": 0},
        # One request of the 7B shape, all 32 layers.
        {"name": "keep_7b_b1", "op": "keep", "heads": "7b", "layers": 32, "kv": "bf16", "rows": 1, "chains": 2, "length": 4},
        # Many requests of the 13B shape, all 40 layers.
        {"name": "keep_13b_b16", "op": "keep", "heads": "13b", "layers": 40, "kv": "bf16", "rows": 16, "chains": 2, "length": 2},
        # The 70B shape's 80 layers with its fp32 cache.
        {"name": "keep_70b_b16", "op": "keep", "heads": "70b", "layers": 80, "kv": "f32", "rows": 16, "chains": 2, "length": 3},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any of the three operators: batches of 1 to 32 requests, trees of 1 to 64 nodes, contexts of 8 to 24000 positions,
    vocabularies of 500 to 131072."""
    op = rng.choice(["attention", "attention", "verify", "verify", "keep"])
    if op == "attention":
        heads = rng.choice(sorted(HEADS))
        nodes = _log_int(rng, 1, 64)
        rows = _log_int(rng, 1, min(32, MAX_ROWS // nodes))
        H, Hkv, hd = HEADS[heads]
        # At most the cache bytes and the products of the largest listed case.
        top = min(24000, 300000000 // (rows * Hkv * hd * 8), 2 * 64 * 64 * 24000 * 128 // (rows * nodes * H * hd))
        return {"op": op, "heads": heads, "kv": rng.choice(["f32", "bf16"]) if heads != "7b" else "bf16", "io": rng.choice(["f32", "f32", "bf16"]),
                "rows": rows, "nodes": nodes, "width": rng.choice([1, 2, 3, 5]), "median": _log_int(rng, 8, max(16, top // 2))}
    if op == "verify":
        nodes = _log_int(rng, 1, 40)
        return {"op": op, "vocab": _log_int(rng, 500, 131072), "rows": _log_int(rng, 1, min(32, MAX_ROWS // nodes)), "nodes": nodes,
                "width": rng.choice([1, 1, 2, 3, 7]), "draft": rng.random() < 0.5, "dtype": rng.choice(["f32", "f32", "bf16"]),
                "temperature": round(rng.uniform(0.3, 1.5), 2), "greedy_every": rng.choice([0, 0, 1, 3])}
    heads = rng.choice(["tiny", "7b", "13b", "70b"])
    length = rng.randint(1, 3)
    return {"op": op, "heads": heads, "layers": _log_int(rng, 2, 40), "kv": rng.choice(["f32", "bf16"]) if heads in ("tiny", "70b") else "bf16",
            "rows": _log_int(rng, 1, 10), "chains": rng.randint(2, 4), "length": length}


# ---------------------------------------------------------------------------------------------------------------- shapes


def _lens(case):
    """Context lengths: quantiles of the recipe's lognormal distribution around the case's median."""
    if case["op"] != "attention":
        return [20 + 3 * i for i in range(case["rows"])]  # the cached positions are not touched
    n = case["rows"]
    z = statistics.NormalDist()
    return [max(1, min(4 * case["median"], round(case["median"] * math.exp(SIGMA * z.inv_cdf((i + 0.5) / n))))) for i in range(n)]


def _trees(case):
    """Nodes per request and their parents (local node numbers, -1 for the root)."""
    if case["op"] == "keep":  # equally long chains side by side below the root: several drafted continuations
        m = case["length"]
        one = [-1] + [0 if k % m == 0 else k for k in range(case["chains"] * m)]
        return [len(one)] * case["rows"], [one] * case["rows"]
    # Trees of `width` children per node, filled level by level; every third request has a node or two fewer.
    nodes = [max(1, case["nodes"] - (i % 3 if case["rows"] > 2 else 0)) for i in range(case["rows"])]
    return nodes, [[-1] + [(j - 1) // case["width"] for j in range(1, n)] for n in nodes]


def _kept(case):
    """Accepted nodes behind the root per request ("keep"): every fifth request accepts none."""
    return [0 if i % 5 == 4 else 1 + i % case["length"] for i in range(case["rows"])]


def work(case):
    nodes, parents = _trees(case)
    R = sum(nodes)
    if case["op"] == "verify":
        # Every logits row once, the draft distribution of the node where a request's walk ends, tokens and uniforms.
        size = 4 if case["dtype"] == "f32" else 2
        rows = R + (case["rows"] if case["draft"] else 0)
        return {"bytes": rows * case["vocab"] * size + R * 16 + case["rows"] * 8, "flops": 4 * R * case["vocab"]}
    H, Hkv, hd = HEADS[case["heads"]]
    size = 4 if case["kv"] == "f32" else 2
    if case["op"] == "keep":
        # Chain 0 is in place already (see _inputs: every fourth request): nothing moves there.
        moved = sum(a for i, a in enumerate(_kept(case)) if i % 4 != 3)
        return {"bytes": moved * case["layers"] * Hkv * hd * size * 2 * 2 + R * 4 + case["rows"] * 4, "flops": 0}
    io = 4 if case["io"] == "f32" else 2
    lens = _lens(case)
    flops = 0
    for n, length, par in zip(nodes, lens, parents):
        depth = [0] * n
        for j in range(1, n):
            depth[j] = depth[par[j]] + 1
        flops += 4 * H * hd * sum(length + d + 1 for d in depth)
    return {"bytes": sum(length + n for n, length in zip(nodes, lens)) * Hkv * hd * size * 2 + 2 * R * H * hd * io, "flops": flops}


# ---------------------------------------------------------------------------------------------------------------- inputs


def _k_view(k, hd):
    """The K pool [layers, blocks, KV heads, 16 * hd] with its tile order split up: [..., dim / P, 4, position, dim], P =
    16 fp32 or 32 bf16 dimensions (a 16-byte piece holds consecutive dimensions of one position)."""
    per = 16 // k.element_size()
    return k.view(*k.shape[:3], hd // (4 * per), 4, 16, per)


def _v_view(v, hd):
    """The V pool likewise: [..., dim / 16, position / 4, dim % 16, position % 4] for fp32; for bf16 the pieces of two
    16-dimension groups are adjacent: [..., dim / 32, position / 4, dim % 16, (dim / 16) % 2, position % 4]."""
    if v.element_size() == 4:
        return v.view(*v.shape[:3], hd // 16, 4, 16, 4)
    return v.view(*v.shape[:3], hd // 32, 4, 16, 2, 4)


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _inputs(case, seed):
    """What the seed makes: tensors on the GPU and the host's lists."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    hostrng = np.random.default_rng(seed)
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    B = case["rows"]
    lens = _lens(case)
    nodes, parents = _trees(case)
    start = [0]
    for n in nodes:
        start.append(start[-1] + n)
    R = start[-1]
    s = {"case": case, "lens": lens, "nodes": nodes, "start": start, "parents": [p for par in parents for p in par]}
    s["slots"] = [int(x) for x in hostrng.permutation(B)]
    if case["op"] == "verify":
        V = case["vocab"]
        # A model's logits: a broad bulk and a few likely tokens.
        logits = randn(R, V)
        logits += 14 * torch.relu(rand(R, V) - (1 - 20 / V)) * V / 20
        logits = logits.to(_dtype(case["dtype"]))
        par = torch.tensor([start[i] + max(p, 0) for i in range(B) for p in parents[i]], device="cuda")
        # The draft model agrees roughly; a node's children are independent draws from its distribution.
        q = torch.softmax(logits.float() + 0.7 * randn(R, V), 1).to(logits.dtype)
        noise = -torch.log(-torch.log(rand(R, V).clamp(1e-20, 1 - 1e-7)))
        s["tokens"] = torch.argmax(torch.log(q[par].float().clamp_min(1e-30)) + noise, 1).to(torch.int32)
        s["logits"] = logits
        s["draft"] = q if case["draft"] else None
        every = case["greedy_every"]
        s["temperature"] = [0.0 if every and i % every == 0 else case["temperature"] for i in range(B)]
        s["accept"], s["sample"] = rand(R), rand(B)
        return s
    H, Hkv, hd = HEADS[case["heads"]]
    L = case.get("layers", 1)
    blocks = [(length + n + 15) // 16 for length, n in zip(lens, nodes)]
    NB = sum(blocks)
    ids = hostrng.permutation(NB)  # a pool that requests have come and gone in
    table = np.zeros((B, max(blocks)), dtype=np.int32)
    at = 0
    for i, n in enumerate(blocks):
        table[s["slots"][i], :n] = ids[at:at + n]
        at += n
    s["table"] = torch.from_numpy(table).cuda()
    s["k"] = randn(L, NB, Hkv, 16 * hd).to(_dtype(case["kv"]))
    s["v"] = randn(L, NB, Hkv, 16 * hd).to(_dtype(case["kv"]))
    if case["op"] == "attention":
        s["q"] = (1.5 * randn(R, H, hd)).to(_dtype(case["io"]))
        return s
    # "keep": every fourth request accepted its first chain, which is in place; the others one of the later chains, whose
    # nodes all lie behind the kept positions (so a pass leaves its sources as they were).
    path = np.full(R, -1, dtype=np.int32)
    kept = _kept(case)
    for i in range(B):
        first = 1 + (0 if i % 4 == 3 else int(hostrng.integers(1, case["chains"]))) * case["length"]
        path[start[i]] = 0
        path[start[i] + 1:start[i] + 1 + kept[i]] = first + np.arange(kept[i])
    s["path"] = torch.from_numpy(path).cuda()
    s["count"] = torch.tensor([a + 1 for a in kept], dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    B, nodes, start, R = case["rows"], s["nodes"], s["start"], s["start"][-1]
    N = max(nodes)
    # The plan of the plain forms: relations between the token rows of the batch.
    anc = np.zeros((R, R), dtype=bool)      # [row, row']: row' is the row's node or one of its ancestors
    earlier = np.zeros((R, R), dtype=bool)  # row' is an earlier child of the same parent
    rank = np.zeros(R, dtype=np.int64)      # earlier children of the same parent
    for i in range(B):
        for j in range(nodes[i]):
            r, p = start[i] + j, s["parents"][start[i] + j]
            if p >= 0:
                anc[r] = anc[start[i] + p]
                for j2 in range(1, j):
                    if s["parents"][start[i] + j2] == p:
                        earlier[r, start[i] + j2] = True
            anc[r, r] = True
            rank[r] = earlier[r].sum()
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    req = np.repeat(np.arange(B), nodes)
    s["anc"], s["earlier"], s["rank"] = cuda(anc), cuda(earlier), cuda(rank)
    s["req"], s["first"] = cuda(req), cuda(np.array(start[:-1]))
    s["local"] = cuda(np.arange(R) - np.array(start[:-1])[req])
    s["parent_row"] = cuda(np.array([start[i] + max(p, 0) for i, p in zip(req, s["parents"])]))
    s["is_root"] = s["local"] == 0
    s["children"] = int(rank.max()) + 1 if R > B else 0
    s["lens_dev"], s["nodes_dev"] = cuda(np.array(s["lens"])), cuda(np.array(nodes))
    s["slots_dev"] = cuda(np.array(s["slots"]))
    s["rows_of"] = cuda(np.array([[start[i] + min(j, nodes[i] - 1) for j in range(N)] for i in range(B)]))  # [B, N], padded
    if own:
        from paper_2403_12900_amd.tree import KVView, TreeBatch, TreeOps
        s["ops"] = TreeOps()
        s["batch"] = TreeBatch(s["slots"], s["lens"], nodes, s["parents"])
        if case["op"] != "verify":
            s["view"] = KVView(s["k"], s["v"], s["table"])
    return s


# ------------------------------------------------------------------------------------------------------------ the passes


def run(s):
    op = s["case"]["op"]
    if op == "attention":
        if own:
            return s["ops"].attention(s["view"], 0, s["batch"], s["q"])
        return _attention(s)
    if op == "verify":
        if own:
            return s["ops"].verify(s["batch"], s["tokens"], s["logits"], s["accept"], s["sample"], draft_probs=s["draft"],
                                   temperature=s["temperature"])
        return _verify(s)
    if own:
        s["ops"].keep(s["view"], s["batch"], s["path"], s["count"])
        return s["k"], s["v"]
    return _keep(s)


def _attention(s):
    H, Hkv, hd = HEADS[s["case"]["heads"]]
    G = H // Hkv
    idx = s["table"][s["slots_dev"]].long()  # [B, blocks]
    B, nb = idx.shape
    N = s["rows_of"].shape[1]
    # [B, blocks, KV heads, ...tile] -> [B, KV heads, positions, dims], in 32 bits
    k = _k_view(s["k"][0][idx].view(1, B * nb, Hkv, 16 * hd), hd)[0].float()
    k = k.view(B, nb, *k.shape[1:]).permute(0, 2, 1, 5, 3, 4, 6).reshape(B, Hkv, nb * 16, hd)
    v = _v_view(s["v"][0][idx].view(1, B * nb, Hkv, 16 * hd), hd)[0].float()
    v = v.view(B, nb, *v.shape[1:])
    v = v.permute(0, 2, 1, 4, 6, 3, 5) if v.dim() == 7 else v.permute(0, 2, 1, 4, 7, 3, 6, 5)
    v = v.reshape(B, Hkv, nb * 16, hd)
    q = s["q"].float()[s["rows_of"]].view(B, N, Hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * N, hd)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(hd)
    # Position t: cached (t < len), or the drafted node t - len where that is the row's node or an ancestor.
    t = torch.arange(nb * 16, device=idx.device)
    node = t[None, :] - s["lens_dev"][:, None]  # [B, positions]
    inside = (node >= 0) & (node < s["nodes_dev"][:, None])
    col = s["first"][:, None] + node.clamp(0, N - 1).minimum(s["nodes_dev"][:, None] - 1)
    sees = (node < 0)[:, None, :] | (inside[:, None, :] & s["anc"][s["rows_of"][:, :, None], col[:, None, :]])  # [B, N, positions]
    scores.view(B, Hkv, G, N, -1).masked_fill_(~sees[:, None, None], -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    out = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    out = out.view(B, Hkv, G, N, hd).permute(0, 3, 1, 2, 4).reshape(B, N, H, hd)
    return out[s["req"], s["local"]].to(s["q"].dtype)


def _verify(s):
    logits, tok, par = s["logits"].double(), s["tokens"].long(), s["parent_row"]
    R, V = logits.shape
    temp = torch.tensor(s["temperature"], dtype=torch.float64, device=logits.device)
    greedy = temp == 0
    x = logits / torch.where(greedy, 1.0, temp)[s["req"]][:, None]
    p = torch.exp(x - x.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    best = torch.where(logits == logits.amax(1, keepdim=True), torch.arange(V, device=logits.device), V).amin(1)
    u = s["accept"].double()
    px = p[par, tok]
    c, left = torch.zeros(R, dtype=torch.float64, device=logits.device), torch.ones(R, dtype=torch.float64, device=logits.device)
    if s["draft"] is not None:
        # After k rejections at a node r = max(p - c q, 0) / left, c the sum of the earlier `left`.
        q = s["draft"].double()
        qx = q[par, tok]
        ok = torch.zeros(R, dtype=torch.bool, device=logits.device)
        kids = torch.zeros(R, dtype=torch.int64, device=logits.device).index_add_(0, par, (~s["is_root"]).long())
        for k in range(s["children"]):
            ok |= (s["rank"] == k) & (u * qx * left[par] < (px - c[par] * qx).clamp_min(0))
            more = kids > k
            c = torch.where(more, c + left, c)
            left = torch.where(more, (p - c[:, None] * q).clamp_min(0).sum(1), left)
    else:
        # A point mass at each child: a rejected token leaves r, and so does every later child of the same token.
        again = (s["earlier"] & (tok[:, None] == tok[None, :])).any(1)
        left_x = 1 - (s["earlier"] * torch.where(again, 0.0, px)[None, :]).sum(1)
        ok = ~again & (u * left_x < px)
    ok = torch.where(greedy[s["req"]], tok == best[par], ok) & ~s["is_root"]
    ok &= ~(s["earlier"] & ok[None, :]).any(1)                       # the first accepted child of its parent
    reached = ~(s["anc"] & ~(ok | s["is_root"])[None, :]).any(1)     # and so are all its ancestors
    count = torch.zeros_like(s["first"]).index_add_(0, s["req"], reached.long())
    place = torch.cumsum(reached.long(), 0)
    place = place - place[s["first"]][s["req"]]                      # its place on the path (0: the root)
    last = s["first"].scatter_reduce(0, s["req"], torch.where(reached, torch.arange(R, device=tok.device), -1), "amax")
    # The next token at the path's last node.
    w = p[last]
    if s["draft"] is not None:
        rest = (p[last] - c[last][:, None] * q[last]).clamp_min(0)
    else:
        child = (par[None, :] == last[:, None]) & ~s["is_root"][None, :]  # [B, R]
        gone = torch.zeros_like(w).index_put_((torch.arange(len(w), device=tok.device)[:, None], tok[None, :].expand(len(w), R)),
                                              child.double(), accumulate=True)
        rest = torch.where(gone > 0, 0.0, w)
    w = torch.where(rest.sum(1, keepdim=True) > 0, rest, w)
    cdf = torch.cumsum(w, 1)
    above = cdf > s["sample"].double()[:, None] * cdf[:, -1:]
    ids = torch.arange(V, device=tok.device)
    drawn = torch.where(above.any(1), torch.where(above, ids, V).amin(1), torch.where(w > 0, ids, -1).amax(1))
    drawn = torch.where(greedy, best[last], drawn)
    # Row-sized outputs, a request's entries from its first row on, -1 behind them; a last entry takes what falls outside.
    path = torch.full((R + 1,), -1, dtype=torch.int32, device=tok.device)
    emitted = path.clone()
    path[torch.where(reached, s["first"][s["req"]] + place, R)] = s["local"].int()
    emitted[torch.where(reached & ~s["is_root"], s["first"][s["req"]] + place - 1, R)] = s["tokens"]
    emitted[s["first"] + count - 1] = drawn.int()
    return emitted[:R], path[:R], count.int()


def _keep(s):
    hd = HEADS[s["case"]["heads"]][2]
    # Entries past a request's count copy the root onto itself.
    valid = s["local"] < s["count"].long()[s["req"]]
    base = s["lens_dev"][s["req"]]
    src = base + torch.where(valid, s["path"].long(), 0)
    dst = base + torch.where(valid, s["local"], 0)
    row = s["slots_dev"][s["req"]]
    block = lambda t: s["table"][row, t // 16].long()  # noqa: E731
    k, v = _k_view(s["k"], hd), _v_view(s["v"], hd)
    k[:, block(dst), :, :, :, dst % 16] = k[:, block(src), :, :, :, src % 16]
    if v.dim() == 7:
        v[:, block(dst), :, :, dst % 16 // 4, :, dst % 4] = v[:, block(src), :, :, src % 16 // 4, :, src % 4]
    else:
        v[:, block(dst), :, :, dst % 16 // 4, :, :, dst % 4] = v[:, block(src), :, :, src % 16 // 4, :, :, src % 4]
    return s["k"], s["v"]


# ---------------------------------------------------------------------------------------------------- results in 64 bits


def exact(case, seed):
    s = _inputs(case, seed)
    return {"attention": _exact_attention, "verify": _exact_verify, "keep": _exact_keep}[case["op"]](case, s)


def _rows_of_cache(pool, table_row, positions, hd, values):
    """Keys (or values) of the given positions of one request, [positions, KV heads, hd] in 64 bits, element by element of
    the tile order."""
    per = 16 // pool.element_size()
    pos = torch.tensor(positions, device=pool.device)
    dims = torch.arange(hd, device=pool.device)
    t = (pos % 16)[:, None]
    if not values:
        off = ((dims // (4 * per)) * 64 + (dims % (4 * per)) // per * 16)[None, :] * per + t * per + (dims % per)[None, :]
    elif per == 8:
        off = (((dims // 32 * 4)[None, :] + t // 4) * 16 + (dims % 16)[None, :]) * 8 + (dims // 16 % 2 * 4)[None, :] + t % 4
    else:
        off = (((dims // 16 * 4)[None, :] + t // 4) * 16 + (dims % 16)[None, :]) * 4 + t % 4
    tiles = pool[table_row[pos // 16].long()]  # [positions, KV heads, 16 hd]
    return torch.gather(tiles, 2, off[:, None, :].expand(-1, tiles.shape[1], -1)).double()


def _exact_attention(case, s):
    H, Hkv, hd = HEADS[case["heads"]]
    out = torch.empty(s["start"][-1], H, hd, dtype=torch.float64, device="cuda")
    for i in range(case["rows"]):
        n, length, r0 = s["nodes"][i], s["lens"][i], s["start"][i]
        row = s["table"][s["slots"][i]]
        k = _rows_of_cache(s["k"][0], row, range(length + n), hd, False)
        v = _rows_of_cache(s["v"][0], row, range(length + n), hd, True)
        sees = torch.zeros(n, length + n, dtype=torch.bool)
        sees[:, :length] = True
        for j in range(n):
            a = j
            while a >= 0:
                sees[j, length + a] = True
                a = s["parents"][r0 + a]
        sees = sees.cuda()
        for h in range(H):
            q = s["q"][r0:r0 + n, h].double()
            z = q @ k[:, h // (H // Hkv)].T.contiguous() / math.sqrt(hd)
            z[~sees] = -math.inf
            out[r0:r0 + n, h] = torch.softmax(z, 1) @ v[:, h // (H // Hkv)]
    return out


def _exact_verify(case, s):
    tok, u, us = s["tokens"].cpu().numpy(), s["accept"].double().cpu().numpy(), s["sample"].double().cpu().numpy()
    R = s["start"][-1]
    emitted, path = np.full(R, -1, dtype=np.int32), np.full(R, -1, dtype=np.int32)
    count = np.zeros(case["rows"], dtype=np.int32)
    for i in range(case["rows"]):
        r0, temp = s["start"][i], s["temperature"][i]
        node, steps = 0, []
        while True:
            steps.append(node)
            z = s["logits"][r0 + node].double().cpu().numpy()
            q = s["draft"][r0 + node].double().cpu().numpy() if s["draft"] is not None else None
            if temp == 0:
                r = np.zeros_like(z)
                r[np.argmax(z)] = 1
            else:
                r = np.exp((z - z.max()) / temp)
                r /= r.sum()
            target, taken = r, None
            for j in range(node + 1, s["nodes"][i]):
                if s["parents"][r0 + j] != node:
                    continue
                x = tok[r0 + j]
                if temp == 0:
                    if r[x] == 1:
                        taken = j
                        break
                    continue
                draft = np.zeros_like(r) if q is None else q
                if q is None:
                    draft[x] = 1
                if u[r0 + j] * draft[x] < r[x]:
                    taken = j
                    break
                rest = np.maximum(r - draft, 0) if q is not None else np.where(draft > 0, 0.0, r)
                r = rest / rest.sum() if rest.sum() > 0 else np.zeros_like(r)
            if taken is None:
                break
            node = taken
        if r.sum() <= 0:
            r = target
        cdf = np.cumsum(r)
        hit = np.flatnonzero(cdf > us[i] * cdf[-1]) if temp else np.flatnonzero(r)
        emitted[r0:r0 + len(steps) - 1] = tok[[r0 + j for j in steps[1:]]]
        emitted[r0 + len(steps) - 1] = hit[0] if len(hit) else np.flatnonzero(r)[-1]
        path[r0:r0 + len(steps)] = steps
        count[i] = len(steps)
    return emitted, path, count


def _exact_keep(case, s):
    hd = HEADS[case["heads"]][2]
    path, count, table = s["path"].cpu().numpy(), s["count"].cpu().numpy(), s["table"].cpu().numpy()
    for pool, view in ((s["k"], _k_view(s["k"], hd)), (s["v"], _v_view(s["v"], hd))):
        at = (lambda b, t: view[:, b, :, :, :, t]) if pool is s["k"] else (lambda b, t: view.select(-1, t % 4).select(1, b)[:, :, :, t // 4])
        for i in range(case["rows"]):
            row, length = table[s["slots"][i]], s["lens"][i]
            for to in range(1, int(count[i])):
                a, b = length + int(path[s["start"][i] + to]), length + to
                at(int(row[b // 16]), b % 16).copy_(at(int(row[a // 16]), a % 16).clone())
    return s["k"], s["v"]
