"""spr_tree_step over contexts whose attention is split over the cache and merged (needs an MI355X where marked).

The attention of a model pass writes activation records, a form of its own of every kernel; here each merges splits, inside
the kernel and in a launch of its own.  Gates on logits as in the decode parity tests: max abs 1e-4 / relative 1e-5 (fp32
models), 5e-2 / 1e-2 (bf16).  That they would notice a lost split is tested on the CPU.
"""
import ctypes

import numpy as np
import pytest
import torch

from oracle import llama_ref as R
from paper_2403_12900_amd.configs import ModelConfig

from . import tree_ref as ref
from ._harness import oracle_shape, say
from .test_gpu_tree_step import near, start, tree_batch
from .test_tree_host import host, p32, raw_batch

WIDE = dict(d_model=256, n_heads=8, n_kv_heads=1, head_dim=128, d_ff=400, vocab=1501)
MODELS = {
    "bf16_gqa": ModelConfig(n_layers=3, d_model=160, n_heads=4, n_kv_heads=2, head_dim=64, d_ff=344, vocab=777),
    "bf16_wide": ModelConfig(n_layers=2, **WIDE),
    "bf16_wide_fp32kv": ModelConfig(n_layers=2, kv_bf16=False, **WIDE),
    "fp32": ModelConfig(n_layers=2, d_model=128, n_heads=8, n_kv_heads=1, head_dim=64, d_ff=176, vocab=1000, bf16=False),
}
# model, nodes and context of the long request; columns per work-group, least splits, merged by a launch of its own.
CASES = [("bf16_gqa", 5, 700, 16, 5, False), ("bf16_wide", 2, 1800, 16, 13, True), ("bf16_wide", 4, 500, 32, 3, False),
         ("bf16_wide", 4, 1100, 32, 9, True), ("bf16_wide", 9, 700, 64, 2, True), ("bf16_wide_fp32kv", 2, 400, 16, 6, False),
         ("bf16_wide_fp32kv", 4, 1100, 32, 9, True), ("bf16_wide_fp32kv", 9, 700, 64, 2, True), ("fp32", 2, 1100, 16, 9, False),
         ("fp32", 4, 1100, 32, 13, True), ("fp32", 9, 700, 64, 2, True)]
SHORT = 30  # the other request's context


@pytest.mark.parametrize("name,nodes,L,columns,splits,apart", CASES)
def test_the_cases_split_as_they_are_meant_to(name, nodes, L, columns, splits, apart):
    m = MODELS[name]
    trees = [[-1] + [0] * (nodes - 1), [-1, 0]]
    b = raw_batch(2, [0, 1], [L, SHORT], [nodes, 2], trees[0] + trees[1])
    out, step = np.zeros(140, np.int32), 2 if m.kv_is_bf16 else 1
    st = host().sprh_tree_split(ctypes.byref(b), m.n_heads // m.n_kv_heads, m.n_kv_heads, m.head_dim, step if columns > 32 else 4 * step,
                                512, 2048 * m.n_heads * (m.head_dim + 4), p32(out))
    cols = nodes * m.n_heads // m.n_kv_heads
    cw = min(int(out[0]), 64)  # fp32 queries: at most 64 columns
    groups = -(-cols // cw)
    got = -(-(-(-(L + nodes) // 16)) // int(out[1]))
    assert st == 0 and cw == columns and got >= splits and (cw > 32 or groups == 1)
    assert (cw > 32 or min(cols, cw) * got * m.head_dim > 192 * 128) == apart


def drafted(name, nodes, L):
    m = MODELS[name]
    rng = np.random.default_rng(L + nodes)
    trees = [ref.random_tree(rng, nodes, "random"), [-1, 0]]
    return m, trees, rng.integers(0, m.vocab, size=nodes + 2).astype(np.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("name,nodes,L,columns,splits,apart", CASES)
def test_long_contexts_against_the_oracle(name, nodes, L, columns, splits, apart):
    m, trees, tokens = drafted(name, nodes, L)
    dm, _, prompts, tok = start(m, [L, SHORT], [24, 24])
    first = tok.cpu().numpy()
    say(f"tree step {name}: {nodes} nodes at {L}")
    count, emitted, z, _ = dm.tree_step(tree_batch([0, 1], [L, SHORT], trees), torch.as_tensor(tokens).cuda(), tok, temperature=0.0)
    z = z.cpu().numpy()
    dm.close()
    w = R.Weights(oracle_shape(m), 5)
    r0 = 0
    for s, t in enumerate(trees):
        for j in sorted({0, len(t) - 1, len(t) // 2}):
            path = sorted(ref.ancestors(t, j))
            seq = [first[s]] + [tokens[r0 + a] for a in path[1:]]
            want = R.teacher_forced_logits(w, prompts[s], list(seq) + [0], steps=[len(seq)])[0]
            near(z[r0 + j], want, m, f"{name} request {s} node {j}")
        r0 += len(t)
    want = ref.verify(trees, tokens, z, None, None, None, [0, 0])
    assert np.array_equal(emitted.cpu().numpy(), want[0]) and np.array_equal(count, want[2])


@pytest.mark.parametrize("name,L,lost", [("bf16_gqa", 700, 128), ("bf16_wide", 1800, 128), ("bf16_wide_fp32kv", 1100, 64), ("fp32", 1100, 64)])
def test_the_gates_reject_a_lost_split(name, L, lost, monkeypatch):
    """The oracle without one split's positions in its last row's attention, in every layer, is outside the gates."""
    m = MODELS[name]
    w = R.Weights(oracle_shape(m), 5)
    tokens = np.random.default_rng(L).integers(0, m.vocab, size=L)
    right = R.forward_causal(w, tokens, [L - 1])[0]
    plain = R.causal_attention

    def without(q, k, v):
        o = plain(q, k, v).reshape(len(q), -1)
        keep = np.r_[0:lost, 2 * lost:len(k)]
        G = q.shape[1] // k.shape[1]
        for h in range(q.shape[1]):
            s = k[keep, h // G] @ q[-1, h] / np.sqrt(q.shape[2])
            p = np.exp(s - s.max())
            o[-1, h * q.shape[2]:(h + 1) * q.shape[2]] = p / p.sum() @ v[keep, h // G]
        return o

    monkeypatch.setattr(R, "causal_attention", without)
    wrong = R.forward_causal(w, tokens, [L - 1])[0]
    with pytest.raises(AssertionError):
        near(wrong, right, m, name)
    assert np.linalg.norm(wrong - right) > 2 * (1e-2 if m.bf16 else 1e-5) * np.linalg.norm(right)
