"""Verification of trees whose candidates come back on later levels, as a draft's do: a
token that was rejected at one node is a token like any other below its siblings."""
import itertools

import numpy as np
import pytest
import torch

import paged_ref as R
import synth
from gpu_helpers import make_session
from paper_2402_15758_amd import binding as B
from test_gpu_accept import run, tree
from test_gpu_sampled import parents_of, uniform

pytestmark = pytest.mark.gpu


def came_back(tokens, parents, new, path):
    """Whether a walk emits a token that it rejected at an earlier node."""
    gone = set()
    for d, node in enumerate(path):
        if new[d] in gone:
            return True
        for c in (c for c, p in enumerate(parents) if p == node):
            if d + 1 < len(path) and c == path[d + 1]:
                break
            gone.add(int(tokens[c]))
    return False


def repeated(batch, parents, vocab, dtype, seed, temperature, few=6):
    """Every node's children are tokens of the same `few`, which hold nine tenths of the
    mass of every row in uneven shares."""
    g = torch.Generator().manual_seed(seed)
    N = len(parents)
    live = torch.randperm(vocab, generator=g)[:few]
    p = torch.log_softmax(torch.randn(batch, N, vocab, generator=g), -1) + np.log(0.1)
    p[:, :, live] = torch.log_softmax(1.5 * torch.randn(batch, N, few, generator=g), -1) + np.log(0.9)
    tokens = torch.zeros(batch, N, dtype=torch.int64)
    for u in range(N):
        kids = [c for c in range(N) if parents[c] == u]
        for b in range(batch):
            tokens[b, kids] = live[torch.randperm(few, generator=g)[:len(kids)]]
    u = torch.rand(batch, N, generator=g, dtype=torch.float64)
    return (temperature * p + 2.0).to(R.TYPES[dtype]).view(batch * N, vocab), tokens, u


# the last two: over 10000 parts of 1024 tokens of bf16 rows, by a table from a temperature
# of 1/4 on
@pytest.mark.parametrize("nodes,arity,vocab,batch,dtype,temperature", [
    (13, 3, 50, 300, "f32", 1.0), (13, 3, 50, 300, "bf16", 1.0), (40, 3, 1500, 60, "f32", 0.7),
    (64, 5, 1500, 60, "bf16", 1.3), (13, 3, 2049, 400, "bf16", 0.2), (13, 3, 2049, 400, "bf16", 0.25)])
def test_tokens_on_several_levels(nodes, arity, vocab, batch, dtype, temperature):
    parents = tree(nodes, arity)
    logits, tokens, u = repeated(batch, parents, vocab, dtype, nodes + vocab, temperature)
    got = run(logits, None, tokens, parents, u, temperature, vocab)
    back = 0
    for b in range(batch):
        new, path, margin = R.accept(logits.view(batch, nodes, vocab)[b], None, tokens[b].tolist(), parents,
                                     u[b].tolist(), temperature)
        assert margin > vocab * 2.0 ** -50  # 64 bits decide
        assert got[b] == (new, path), (b, got[b], new, path)
        back += came_back(tokens[b].tolist(), parents, new, path)
    assert back >= batch // 50


def test_pairs_at_the_targets_rate():
    """Of 20000 walks, the frequencies of pairs of tokens are the products of the target's
    probabilities (5 standard deviations), in trees whose two levels hold the same tokens."""
    n, V, live = 20000, 9, [1, 4, 6]
    parents = [-1, 0, 0, 0] + [1] * 3 + [2] * 3 + [3] * 3
    N = len(parents)
    g = torch.Generator().manual_seed(5)
    first = 1.2 * torch.randn(V, generator=g)
    after = 1.5 * torch.randn(V, V, generator=g)  # after token t
    after[4, 1] += 3.0
    after[6, 1] += 2.0
    tokens = torch.tensor([0] + live + [1, 6, 4] + [1, 4, 6] + [4, 1, 6])
    rows = torch.stack([first] + [after[int(t)] for t in tokens[1:]])
    u = torch.rand(n, N, generator=g, dtype=torch.float64)
    out = run(rows.repeat(n, 1), None, tokens.repeat(n, 1), parents, u, 1.0, V)
    p1, p2 = torch.softmax(first.double(), 0), torch.softmax(after.double(), -1)
    singles = torch.bincount(torch.tensor([o[0][0] for o in out]), minlength=V).double() / n
    assert bool(((singles - p1).abs() <= 5 * torch.sqrt(p1 * (1 - p1) / n)).all())
    for a, b in itertools.product(live, range(V)):
        f = sum(o[0][:2] == [a, b] for o in out) / n
        p = float(p1[a] * p2[a, b])
        assert abs(f - p) <= 5 * (p * (1 - p) / n) ** 0.5, (a, b, f, p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_engine_steps_over_trees_of_repeated_tokens(dtype):
    """Session.set_sampling over injected trees whose nodes all have the same few tokens as
    children, by a model that likes those: every step is the rule on its own logits."""
    import dataclasses
    cfg = dataclasses.replace(synth.TINY if dtype == "f32" else synth.small_config(), vocab=64)
    w = synth.make_weights(cfg, device="cuda", std=0.06)
    live, g = [3, 17, 18, 40, 41, 63], torch.Generator().manual_seed(7)
    head = torch.zeros(w["lm_head"].shape)
    head[:, live] = 0.16 * torch.randn(cfg.d_model, len(live), generator=g)  # logits of 2.5 or so
    w["lm_head"] = head.to(w["lm_head"].dtype).cuda()
    ranks = [(r,) for r in range(4)] + [(r, s) for r in range(4) for s in range(4)]
    parents, batch, seed, T = parents_of(ranks), 3, 21, 0.6
    N = len(parents)
    ps = [synth.make_prompt(n, cfg.vocab, 5 + n) for n in (30, 7, 64)]
    sess = make_session(cfg, w, ranks, max_batch=batch, max_len=512)
    sess.set_sampling(T, seed)
    last, n = sess.prefill(ps).tolist(), [len(p) for p in ps]
    back = 0
    for _ in range(60):
        inject = np.zeros((batch, N), dtype=np.int32)
        for b in range(batch):
            for u in range(N):
                kids = [c for c in range(N) if parents[c] == u]
                inject[b, kids] = [live[i] for i in torch.randperm(len(live), generator=g)[:len(kids)].tolist()]
        sess.set_tree_tokens(inject[:, 1:])
        toks, cnt, path = sess.step()
        logits = torch.from_numpy(sess.debug(B.DBG_VERIFY_LOGITS)).view(batch, N, -1)
        for b in range(batch):
            L, inject[b, 0] = int(cnt[b]), last[b]
            u = [uniform(seed, b, n[b], i) for i in range(N)]
            new, nodes, _ = R.accept(logits[b], None, inject[b].tolist(), parents, u, T)
            assert toks[b, :L].tolist() == new and path[b, :L].tolist() == nodes
            back += came_back(inject[b].tolist(), parents, new, nodes)
            last[b], n[b] = new[-1], n[b] + L
    sess.close()
    assert back >= 3
