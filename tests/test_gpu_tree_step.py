"""spr_tree_step: drafted trees through the whole model (needs an MI355X).

Gates on logits as in the decode parity tests: max abs 1e-4 / relative 1e-5 (fp32 models), 5e-2 / 1e-2 (bf16), against the
oracle run on each node's own token sequence.  Tokens, paths and counts are whole numbers and have to equal the plain
verification of the returned logits.
"""
import numpy as np
import pytest
import torch

from oracle import llama_ref as R
from paper_2403_12900_amd.configs import ModelConfig

from . import tree_ref as ref
from ._harness import oracle_shape, say

pytestmark = pytest.mark.gpu

MODELS = {
    "fp32": ModelConfig(n_layers=2, d_model=128, n_heads=4, n_kv_heads=4, head_dim=64, d_ff=176, vocab=1000, bf16=False),
    "bf16_gqa": ModelConfig(n_layers=3, d_model=160, n_heads=8, n_kv_heads=2, head_dim=64, d_ff=344, vocab=777),
    "bf16_hd128_fp32kv": ModelConfig(n_layers=2, d_model=256, n_heads=8, n_kv_heads=1, head_dim=128, d_ff=400, vocab=1501,
                                     kv_bf16=False),
    # A vocabulary whose verification sums outgrow the partials' region of so small a model, and uneven heads.
    "large_vocab": ModelConfig(n_layers=1, d_model=64, n_heads=1, n_kv_heads=1, head_dim=64, d_ff=64, vocab=700001),
}
TOL = {False: (1e-4, 1e-5), True: (5e-2, 1e-2)}


def start(m, lens, stops, seed=11, slack=0):
    from paper_2403_12900_amd.binding import DecodeModel
    rng = np.random.default_rng(seed)
    prompts = [rng.integers(0, m.vocab, size=n).astype(np.int32) for n in lens]
    dm = DecodeModel(m, 5, max_slots=len(lens), max_ctx=max(a + b for a, b in zip(lens, stops)) + slack)
    tok = dm.new_token_buffer()
    dm.prefill(list(range(len(lens))), prompts, stops, tok)
    torch.cuda.synchronize()
    return dm, rng, prompts, tok


def tree_batch(slots, lens, trees):
    from paper_2403_12900_amd.tree import TreeBatch
    return TreeBatch(slots, lens, [len(t) for t in trees], [p for t in trees for p in t])


def near(z, want, m, tag):
    tol = TOL[m.bf16]
    d, rel = np.abs(z - want).max(), np.linalg.norm(z - want) / np.linalg.norm(want)
    assert d <= tol[0] and rel <= tol[1], f"{tag}: max abs {d:.2e}, relative {rel:.2e}"


@pytest.mark.parametrize("name", sorted(MODELS))
def test_every_nodes_logits_against_the_oracle(name):
    m = MODELS[name]
    lens = [21, 6, 40, 15]
    dm, rng, prompts, tok = start(m, lens, [20] * 4)
    first = tok.cpu().numpy()
    trees = [ref.random_tree(rng, n, k) for n, k in ((9, "random"), (1, "chain"), (12, "levels"), (5, "chain"))]
    slots = [2, 0, 3, 1]
    R_ = sum(len(t) for t in trees)
    tokens = rng.integers(0, m.vocab, size=R_).astype(np.int32)
    say(f"tree step {name}")
    count, emitted, z, _ = dm.tree_step(tree_batch(slots, [lens[s] for s in slots], trees), torch.as_tensor(tokens).cuda(), tok,
                                        temperature=0.0)
    z = z.cpu().numpy()
    w = R.Weights(oracle_shape(m), 5)
    r0 = 0
    for s, t in zip(slots, trees):
        for j in sorted({0, len(t) - 1, len(t) // 2}):
            path = sorted(ref.ancestors(t, j))
            seq = [first[s]] + [tokens[r0 + a] for a in path[1:]]
            want = R.teacher_forced_logits(w, prompts[s], list(seq) + [0])[len(seq)]
            near(z[r0 + j], want, m, f"{name} slot {s} node {j}")
        r0 += len(t)
    want = ref.verify(trees, tokens, z, None, None, None, [0] * 4)
    assert np.array_equal(emitted.cpu().numpy(), want[0]) and np.array_equal(count, want[2])
    dm.close()


@pytest.mark.parametrize("name", ["fp32", "bf16_gqa", "bf16_hd128_fp32kv"])
def test_greedy_tree_steps_follow_greedy_decode(name):
    """Trees that hold the greedy continuation in one branch (at any node order) and noise elsewhere: every step emits a
    whole level more than its depth of accepted tokens, the sequence is greedy decode's, and the cache that compaction left
    gives the logits that decode's gives."""
    m = MODELS[name]
    lens, stop = [19, 33, 4], 40
    dm, rng, prompts, tok = start(m, lens, [stop] * 3)
    slots = [0, 1, 2]
    seqs = [[int(t)] for t in tok.cpu().numpy()]
    cur = list(lens)
    plain_z = []
    for _ in range(stop - 1):
        z, _ = dm.decode_step(slots, cur, tok, want_logits=True)
        plain_z.append(z.cpu().numpy())
        cur = [c + 1 for c in cur]
        for s, t in enumerate(tok.cpu().numpy()):
            seqs[s].append(int(t))
    for s in slots:
        dm.rewind(s, lens[s], 1)
    tok.copy_(torch.tensor([q[0] for q in seqs], dtype=torch.int32))
    done = [1, 1, 1]
    while max(done) <= stop - 14:  # room for a tree of 13 nodes
        # A chain of 4 right tokens whose last one is wrong now and then, hidden among wrong siblings.
        trees, tokens, want = [], [], []
        for s in slots:
            right = seqs[s][done[s]:done[s] + 4]
            ok = int(rng.integers(0, 5))
            par, tk, at = [-1], [0], 0
            for d, x in enumerate(right):
                noise = [int((x + 1 + k) % m.vocab) for k in range(int(rng.integers(0, 3)))]
                for y in noise:
                    par.append(at)
                    tk.append(y)
                par.append(at)
                tk.append(x if d < ok else int((x + 5) % m.vocab))
                at = len(par) - 1
            trees.append(par)
            tokens += tk
            want.append(min(ok, 4) + 1)
        live = [dm.slot_info(s)[0] for s in slots]
        count, emitted, z, _ = dm.tree_step(tree_batch(slots, live, trees), torch.tensor(tokens, dtype=torch.int32).cuda(), tok,
                                            temperature=[0.0] * 3)
        e, z = emitted.cpu().numpy(), z.cpu().numpy()
        assert count.tolist() == want
        r0 = 0
        for s, t in enumerate(trees):
            got = e[r0:r0 + count[s]].tolist()
            assert got == seqs[s][done[s]:done[s] + count[s]], (name, s, done[s])
            near(z[r0], plain_z[done[s] - 1][s], m, f"{name} slot {s} token {done[s]}")
            done[s] += int(count[s])
            assert dm.slot_info(s)[:2] == (lens[s] + done[s] - 1, done[s])
            r0 += len(t)
        assert tok.cpu().numpy().tolist() == [seqs[s][done[s] - 1] for s in slots]
        # A plain decode step in between.
        zz, _ = dm.decode_step(slots, [dm.slot_info(s)[0] for s in slots], tok, want_logits=True)
        zz = zz.cpu().numpy()
        for s in slots:
            near(zz[s], plain_z[done[s] - 1][s], m, f"{name} slot {s} decode {done[s]}")
            done[s] += 1
        assert tok.cpu().numpy().tolist() == [seqs[s][done[s] - 1] for s in slots]
    dm.close()


@pytest.mark.parametrize("name", ["fp32", "bf16_gqa", "large_vocab"])
@pytest.mark.parametrize("draft", [False, True])
def test_sampled_tree_steps_equal_the_plain_verification(name, draft):
    m = MODELS[name]
    lens = [12, 30]
    dm, rng, _, tok = start(m, lens, [24, 24])
    for _ in range(3):
        live = [dm.slot_info(s)[0] for s in (0, 1)]
        left = [dm.slot_info(s)[2] - dm.slot_info(s)[1] for s in (0, 1)]
        trees = [ref.random_tree(rng, 6, "levels"), ref.random_tree(rng, 5, "star")]
        assert min(left) >= 4
        tokens = rng.integers(0, m.vocab, size=11).astype(np.int32)
        ua, us = rng.random(11, dtype=np.float32), rng.random(2, dtype=np.float32)
        q = torch.softmax(torch.from_numpy(rng.standard_normal((11, m.vocab), dtype=np.float32)), 1) if draft else None
        ua[::2] = 1e-6  # some acceptances
        cu = lambda x: None if x is None else torch.as_tensor(x).cuda()  # noqa: E731
        temps = [0.9, 1.4]
        count, emitted, z, retired = dm.tree_step(tree_batch([0, 1], live, trees), cu(tokens), tok, temperature=temps, accept=cu(ua),
                                                  sample=cu(us), draft_probs=cu(q))
        want = ref.verify(trees, tokens, z.double().cpu().numpy(), ua, us, None if q is None else q.double().numpy(), temps)
        assert np.array_equal(emitted.cpu().numpy(), want[0]) and np.array_equal(count, want[2])
        assert [dm.slot_info(s)[0] for s in (0, 1)] == [a + int(c) for a, c in zip(live, count)]
        assert retired.tolist() == [0, 0]
    dm.close()


def test_one_node_trees_are_decode_steps():
    m = MODELS["bf16_gqa"]
    lens = list(range(3, 67))
    dm, _, _, tok = start(m, lens, [5] * 64)
    t0 = tok.clone()
    slots = list(range(64))
    z, _ = dm.decode_step(slots, lens, tok, want_logits=True)
    t1 = tok.cpu().numpy()
    for s in slots:
        dm.rewind(s, lens[s], 1)
    tok.copy_(t0)
    count, emitted, zt, _ = dm.tree_step(tree_batch(slots, lens, [[-1]] * 64), torch.zeros(64, dtype=torch.int32).cuda(), tok, temperature=0.0)
    assert count.tolist() == [1] * 64
    near(zt.cpu().numpy(), z.cpu().numpy(), m, "one-node trees")
    assert np.array_equal(tok.cpu().numpy(), t1) and np.array_equal(emitted.cpu().numpy(), t1)
    dm.close()


def test_retirement_and_refusals():
    from paper_2403_12900_amd.binding import SPR_ERR_DEVICE_CHECK, SPR_ERR_INVALID_ARG, SPR_ERR_KV_FULL, SPR_ERR_STATE, SproutError
    m = MODELS["fp32"]
    dm, rng, _, tok = start(m, [20, 9], [5, 8])
    z = torch.zeros(16, dtype=torch.int32).cuda()

    def step(slots, lens, trees, **kw):
        n = sum(len(t) for t in trees)
        return dm.tree_step(tree_batch(slots, lens, trees), z[:n], tok, **{"temperature": 0.0, **kw})

    chain = lambda n: [-1] + list(range(n - 1))  # noqa: E731
    for args, st in ((([0], [19], [chain(2)]), SPR_ERR_STATE), (([0], [20], [chain(5)]), SPR_ERR_INVALID_ARG),
                     (([0], [20], [[-1] + [0] * 12]), SPR_ERR_KV_FULL), (([2], [20], [chain(1)]), SPR_ERR_INVALID_ARG),
                     (([0, 0], [20, 20], [chain(1), chain(1)]), SPR_ERR_INVALID_ARG)):
        with pytest.raises(SproutError) as e:
            step(*args)
        assert e.value.status == st, args
    for kw in ({"temperature": -1.0}, {"temperature": float("nan")}, {"temperature": 1.0},
               {"accept": torch.zeros(3).cuda()}, {"draft_probs": torch.zeros(2, 3).cuda()}):
        with pytest.raises(SproutError) as e:
            step([0], [20], [chain(2)], **kw)
        assert e.value.status == SPR_ERR_INVALID_ARG
    assert dm.slot_info(0) == (20, 1, 5) and dm.slot_info(1) == (9, 1, 8)
    # The whole rest of slot 0's generation in one step: the greedy tokens as drafts.
    first, seq = tok.clone(), []
    for k in range(4):
        dm.decode_step([0], [20 + k], tok)
        seq.append(int(tok[0].item()))
    dm.rewind(0, 20, 1)
    tok.copy_(first)
    drafts = torch.tensor([0] + seq[:3], dtype=torch.int32).cuda()
    count, emitted, _, retired = dm.tree_step(tree_batch([0], [20], [chain(4)]), drafts, tok, temperature=0.0)
    assert count.tolist() == [4] and emitted.cpu().numpy().tolist() == seq and retired.tolist() == [1]
    with pytest.raises(SproutError) as e:
        step([0], [24], [chain(1)])
    assert e.value.status == SPR_ERR_STATE
    dm.rewind(0, 21, 2)  # drops three of them again
    assert dm.slot_info(0) == (21, 2, 5)
    # A drafted token outside the vocabulary fails the call and leaves the model to be released.
    bad = torch.tensor([0, m.vocab, 3], dtype=torch.int32).cuda()
    with pytest.raises(SproutError) as e:
        dm.tree_step(tree_batch([1], [9], [[-1, 0, 0]]), bad, tok, temperature=0.0)
    assert e.value.status == SPR_ERR_DEVICE_CHECK
    with pytest.raises(SproutError):
        dm.decode_step([1], [9], tok)
    dm.close()


def test_operators_on_a_models_cache():
    """kv_view: the operators read the model's own cache, and reading it back gives keys and values by position."""
    from paper_2403_12900_amd.tree import TreeOps
    m = MODELS["bf16_gqa"]
    lens = [37, 20]
    dm, rng, prompts, tok = start(m, lens, [6, 6])
    v = dm.kv_view()
    k, val = ref.from_tiles(v.k.cpu(), False), ref.from_tiles(v.v.cpu(), True)

    class Read:
        pass
    cache = Read()
    cache.k, cache.v, cache.table = k, val, v.block_table.cpu().numpy()
    cache.rows = lambda x, layer, slot, pos: x[layer, cache.table[slot, np.asarray(pos) // 16], :, np.asarray(pos) % 16].double().numpy()
    q = torch.from_numpy(rng.standard_normal((2, 8, 64), dtype=np.float32))
    ops = TreeOps()
    # One-node trees at the last cached position: attention over the whole prompt.
    out = ops.attention(v, 2, tree_batch([0, 1], [36, 19], [[-1], [-1]]), q.cuda()).double().cpu().numpy()
    want = ref.attention(cache, 2, [0, 1], [36, 19], [[-1], [-1]], q)
    held = [(cache.rows(k, 2, s, range(n)), cache.rows(val, 2, s, range(n))) for s, n in enumerate(lens)]
    kn = max(np.linalg.norm(a, axis=-1).max() for a, _ in held)
    vm, qn = max(np.abs(b).max() for _, b in held), float(q.double().norm(dim=-1).max())
    # As derived in test_gpu_tree_ops.py, T = 37.
    assert np.abs(out - want).max() <= (8 * 2.0 ** -24 * qn * kn + (26 + 8 * 6.1) * 2.0 ** -24) * vm
    ops.close()
    dm.close()
