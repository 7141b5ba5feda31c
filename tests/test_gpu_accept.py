"""Verification of drafted tokens on the GPU against float64 (paged_ref): every token
and node equal, over trees, chains, types, vocabularies and rows without a
distribution."""
import math

import numpy as np
import pytest
import torch

import paged_ref as R
from paper_2402_15758_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": B.CHIMERA_BF16, "f32": B.CHIMERA_F32}


def tree(nodes, arity):
    return [-1] + [(i - 1) // arity for i in range(1, nodes)]


def depths(parents):
    d = []
    for p in parents:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def run(logits, draft, tokens, parents, u, temperature, vocab, ld=None, want_path=True):
    """Operator results as lists of (new tokens, path) a sequence."""
    Bn, N = tokens.shape
    K1 = max(depths(parents)) + 1
    dtype = "bf16" if logits.dtype == torch.bfloat16 else "f32"
    dl, dd = logits.cuda(), None if draft is None else draft.cuda()
    dtok, du = tokens.int().cuda(), u.double().cuda()
    new = torch.full((Bn, K1), 99, dtype=torch.int32, device="cuda")
    cnt = torch.full((Bn,), 99, dtype=torch.int32, device="cuda")
    path = torch.full((Bn, K1), 99, dtype=torch.int32, device="cuda")
    nb = B.chimera_accept_bytes(Bn, N, vocab, draft is not None)
    ws = torch.full((nb + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    par = np.array(parents, dtype=np.int32)
    B.chimera_accept(DT[dtype], dl.data_ptr(), dl.stride(0), None if dd is None else dd.data_ptr(),
                     0 if dd is None else dd.stride(0), vocab, dtok.data_ptr(), par, N, Bn, temperature, du.data_ptr(),
                     new.data_ptr(), cnt.data_ptr(), path.data_ptr() if want_path else None, ws.data_ptr(), nb,
                     torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (ws[nb:] == 0xFF).all()
    out = []
    for b in range(Bn):
        n = int(cnt[b])
        out.append((new[b, :n].tolist(), path[b, :n].tolist()))
        assert (new[b, n:] == -1).all() and (not want_path or (path[b, n:] == -1).all())
    return out


def inputs(batch, parents, vocab, drawn, dtype, seed, rate=0.6, temperature=1.0):
    g = torch.Generator().manual_seed(seed)
    N = len(parents)
    p = torch.log_softmax(2.0 * torch.randn(batch, N, vocab, generator=g), -1)
    tokens = torch.randint(0, vocab, (batch, N), generator=g)
    draft = None
    if drawn:
        q = torch.log_softmax(2.0 * torch.randn(batch, N, vocab, generator=g), -1)
        p = torch.logaddexp(q + math.log(rate), p + math.log1p(-rate))
        for c in range(1, N):
            tokens[:, c] = torch.multinomial(q[:, c - 1].exp(), 1, generator=g)[:, 0]
        draft = (temperature * q).to(R.TYPES[dtype]).view(batch * N, vocab)
    else:
        for u in range(N):
            kids = [c for c in range(N) if parents[c] == u]
            for b in range(batch):
                ids = torch.randperm(vocab, generator=g)[:len(kids)]
                tokens[b, kids[:len(ids)]] = ids
                if len(ids):
                    p[b, u, ids] = math.log(rate / len(ids))
    logits = (temperature * p + 3.0).to(R.TYPES[dtype]).view(batch * N, vocab)
    u = torch.rand(batch, N, generator=g, dtype=torch.float64)
    return logits, draft, tokens, u


def check(logits, draft, tokens, parents, u, temperature, vocab, **kw):
    got = run(logits, draft, tokens, parents, u, temperature, vocab, **kw)
    Bn, N = tokens.shape
    seen = []
    for b in range(Bn):
        lo = logits.view(Bn, N, -1)[b, :, :vocab]
        dr = None if draft is None else draft.view(Bn, N, -1)[b, :, :vocab]
        new, path, margin = R.accept(lo, dr, tokens[b].tolist(), parents, u[b].tolist(), temperature)
        # a border nearer than 64-bit sums of the vocabulary resolve would decide nothing
        assert margin > vocab * 2.0 ** -50 or got[b][0] == new
        assert got[b][0] == new and (not kw.get("want_path", True) or got[b][1] == path), (b, got[b], new, path)
        seen.append(len(new))
    return seen


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("nodes,arity,vocab,batch", [(1, 1, 1, 3), (1, 1, 1000, 9), (2, 1, 2, 40), (5, 1, 4096, 20),
                                                     (6, 1, 4097, 12), (9, 1, 33000, 6), (64, 1, 130, 12)])
def test_chains(dtype, drawn, nodes, arity, vocab, batch):
    parents = tree(nodes, arity)
    for seed, rate, T in ((1, 0.6, 1.0), (2, 0.95, 0.7), (3, 0.2, 1.4)):
        check(*inputs(batch, parents, vocab, drawn, dtype, seed + vocab, rate, T)[:3], parents,
              inputs(batch, parents, vocab, drawn, dtype, seed + vocab, rate, T)[3], T, vocab)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,arity,vocab,batch", [(3, 2, 7, 40), (8, 3, 1000, 25), (32, 4, 5000, 8), (64, 4, 32000, 3),
                                                     (64, 63, 300, 30), (37, 2, 4096, 8)])
def test_trees(dtype, nodes, arity, vocab, batch):
    parents = tree(nodes, arity)
    lengths = []
    for seed, rate in ((1, 0.5), (2, 0.9), (3, 0.99)):
        logits, _, tokens, u = inputs(batch, parents, vocab, False, dtype, seed, rate)
        lengths += check(logits, None, tokens, parents, u, 1.0, vocab)
    assert min(lengths) == 1 and max(lengths) > 1


def test_strided_rows_and_no_path():
    parents = tree(8, 3)
    logits, _, tokens, u = inputs(5, parents, 997, False, "bf16", 5)
    wide = torch.full((40, 1003), 9.0, dtype=torch.bfloat16)  # past the vocabulary: larger than all
    wide[:, :997] = logits
    check(wide, None, tokens, parents, u, 1.0, 997, want_path=False)


def test_the_same_token_twice():
    """A token already rejected has no mass left for a sibling of its id."""
    parents = [-1, 0, 0, 0]
    V = 50
    logits = torch.randn(4 * 30, V, generator=torch.Generator().manual_seed(1))
    tokens = torch.tensor([[0, 7, 7, 9]] * 30)
    logits.view(30, 4, V)[:, 0, 7] += 4.0
    u = torch.rand(30, 4, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
    u[:, 1] = 0.999  # 7 is rejected
    out = run(logits, None, tokens, parents, u, 1.0, V)
    for b, (new, path) in enumerate(out):
        assert path[:2] != [0, 2]
        ref, rpath, _ = R.accept(logits.view(30, 4, V)[b], None, tokens[b].tolist(), parents, u[b].tolist(), 1.0)
        assert (new, path) == (ref, rpath)


def test_padding_and_empty_places():
    parents = tree(6, 1)
    for drawn in (False, True):
        logits, draft, tokens, u = inputs(6, parents, 500, drawn, "f32", 7, 0.99)
        tokens[0, 3] = -1      # ends after node 2
        tokens[1, 1] = 500     # none
        tokens[2, 0] = -1      # an empty place
        logits.view(6, 6, 500)[2] = math.nan
        got = run(logits, draft, tokens, parents, u, 1.0, 500)
        assert got[2] == ([], []) and len(got[1][0]) == 1 and len(got[0][0]) <= 3
        check(logits, draft, tokens, parents, u, 1.0, 500)
    parents = tree(8, 3)
    logits, _, tokens, u = inputs(6, parents, 500, False, "f32", 8, 0.99)
    tokens[:, 2] = -1
    check(logits, None, tokens, parents, u, 1.0, 500)


def test_rows_without_a_distribution():
    parents = tree(3, 1)
    for drawn in (False, True):
        for bad in (math.nan, math.inf, None):
            logits, draft, tokens, u = inputs(4, parents, 9000, drawn, "f32", 9, 0.999)
            u[:, 1:] = 0.0  # tests pass
            x = logits.view(4, 3, -1)
            if bad is None:
                x[0, 0], x[1, 1], x[2, 2] = -math.inf, -math.inf, -math.inf
            else:
                x[0, 0, 8999], x[1, 1, 17], x[2, 2, 4096] = bad, bad, bad
            got = run(logits, draft, tokens, parents, u, 1.0, 9000)
            assert [len(g[0]) for g in got] == [1, 2, 3, 3]
            assert [g[0][-1] == -1 for g in got] == [True, True, True, False]
            check(logits, draft, tokens, parents, u, 1.0, 9000)
    logits, draft, tokens, u = inputs(4, parents, 9000, True, "f32", 9, 0.999)
    draft.view(4, 3, -1)[1, 0, 5] = math.nan
    got = run(logits, draft, tokens, parents, u, 1.0, 9000)
    assert got[1] == ([-1], [0]) and got[0][0][-1] >= 0


def test_masked_vocabulary_is_never_drawn():
    """-inf logits, whole parts of a row among them; the last and the first entries."""
    V = 3 * 4096 + 5
    logits = torch.full((64, V), -math.inf)
    live = [0, 4096, 2 * 4096 - 1, V - 1]
    logits[:, live] = torch.randn(64, 4, generator=torch.Generator().manual_seed(3))
    u = torch.linspace(0, 1 - 2.0 ** -53, 64, dtype=torch.float64).view(64, 1)
    tokens = torch.zeros(64, 1, dtype=torch.int64)
    check(logits, None, tokens, [-1], u, 1.0, V)
    got = run(logits, None, tokens, [-1], u, 1.0, V)
    assert {g[0][0] for g in got} == set(live) and got[0][0] == [0] and got[-1][0] == [V - 1]


def test_extreme_temperatures_and_levels():
    parents = tree(4, 3)
    for T in (1e-3, 1e-30, 100.0, 1e30):
        for level in (0.0, 3e4, -3e4):
            logits, _, tokens, u = inputs(10, parents, 300, False, "f32", 11)
            logits = logits + level
            check(logits, None, tokens, parents, u, T, 300)


def test_everything_rejected_takes_the_rest():
    """Candidates that hold all but 2^-40 of the mass, all rejected."""
    parents = tree(4, 3)
    logits = torch.full((4 * 8, 5000), -40.0)
    tokens = torch.tensor([[0, 10, 20, 30]] * 8)
    logits[:, [10, 20, 30]] = 0.0
    u = torch.full((8, 4), 1 - 2.0 ** -53, dtype=torch.float64)
    u[:, 0] = torch.linspace(0, 0.999, 8)
    check(logits, None, tokens, parents, u, 1.0, 5000)


def test_accepted_at_the_targets_rate():
    """20000 one-step draws: each token's frequency is the target's, whatever was
    drafted (5 standard deviations)."""
    V, n = 8, 20000
    g = torch.Generator().manual_seed(12)
    z = torch.randn(V, generator=g)
    p = torch.softmax(z.double(), 0)
    for drawn in (False, True):
        parents = [-1, 0] if drawn else [-1, 0, 0]
        N = len(parents)
        logits = z.expand(n * N, V).contiguous()
        draft, tokens = None, torch.tensor([[0, 3, 5][:N]] * n)
        if drawn:
            zq = torch.randn(V, generator=g)
            draft = zq.expand(n * N, V).contiguous()
            tokens[:, 1] = torch.multinomial(torch.softmax(zq, 0), n, replacement=True, generator=g)
        u = torch.rand(n, N, generator=g, dtype=torch.float64)
        first = torch.tensor([o[0][0] for o in run(logits, draft, tokens, parents, u, 1.0, V)])
        freq = torch.bincount(first, minlength=V).double() / n
        assert bool(((freq - p).abs() <= 5 * torch.sqrt(p * (1 - p) / n)).all())


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("temperature", [0.2499, 0.25, 1.0, 7.0])
@pytest.mark.parametrize("vocab,pad", [(2048, 0), (2049, 0), (2050, 6)])
def test_many_bf16_rows(drawn, temperature, vocab, pad):
    """Enough parts for the sums by a table (from 1/4 on): the walks of the rule, and those
    of few rows at once."""
    parents = tree(9, 1) if drawn else tree(64, 4)
    batch = 420 if drawn else 85
    logits, draft, tokens, u = inputs(batch, parents, vocab, drawn, "bf16", 31, 0.8, temperature)
    logits = torch.nn.functional.pad(logits, (0, pad), value=90.0)
    draft = torch.nn.functional.pad(draft, (0, pad), value=90.0) if drawn else None
    check(logits, draft, tokens, parents, u, temperature, vocab)
    all_of = run(logits, draft, tokens, parents, u, temperature, vocab)
    N = len(parents)
    few = run(logits[:5 * N], None if draft is None else draft[:5 * N], tokens[:5], parents, u[:5], temperature, vocab)
    assert all_of[:5] == few


@pytest.mark.parametrize("drawn", [False, True])
def test_many_bf16_rows_outside_the_table(drawn):
    """Zeros, tiny and large logits, masked ones and rows without a distribution among
    rows of a table: parts of either kind in one row, too."""
    vocab, N = 4096, 9
    parents = tree(N, 1)
    logits, draft, tokens, u = inputs(320, parents, vocab, drawn, "bf16", 32, 0.9)
    for x in (logits, draft) if drawn else (logits,):
        x = x.view(320, N, vocab)
        x[0:20, :, 100] = 0.0
        x[20:40, :, :1024] = 0.0
        x[40:60, :, 1024:2048] = 2.0 ** -30
        x[60:80] += 127.0
        x[80:100] -= 140.0
        x[100:120] *= 2000.0
        x[120:140, :, 1000:] = -math.inf
        x[140:160, :, 5:4090] = -math.inf
        x[160:180, :, ::2] = -math.inf
        x[180:190, 1:] = -math.inf
        x[190:200, 2, 77] = math.nan
        x[200:210, 1, 4095] = math.inf
        x[210:230] = 3.0
        x[230:250] = -0.0
        x[250:260] = 2.0 ** 7
        x[260:270] = -(2.0 ** 7 - 0.5)
        x[270:280] = 2.0 ** -25
    g = torch.Generator().manual_seed(33)
    for temperature in (1.0, 0.25):
        if drawn:  # from what the draft's rows became
            q = torch.softmax(draft.double() / temperature, -1)
            rows = [r for r in range(320 * N) if r % N < N - 1 and not bool(q[r].isnan().any())]
            tokens.view(-1)[[r + 1 for r in rows]] = torch.multinomial(q[rows], 1, generator=g)[:, 0]
        check(logits, draft, tokens, parents, u, temperature, vocab)
