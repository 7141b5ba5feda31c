"""Verification over vocabularies of more than 64 parts of 1024 tokens, and what is drawn
where nothing is left of a row's mass."""
import math

import pytest
import torch

import paged_ref as R
from test_gpu_accept import inputs, run, tree

pytestmark = pytest.mark.gpu
LAST = 1 - 2.0 ** -53


def agree(logits, draft, tokens, parents, u, temperature, vocab):
    """Results by the rule; the walks' lengths."""
    Bn, N = tokens.shape
    got, lengths = run(logits, draft, tokens, parents, u, temperature, vocab), []
    for b in range(Bn):
        dr = None if draft is None else draft.view(Bn, N, vocab)[b]
        new, path, margin = R.accept(logits.view(Bn, N, vocab)[b], dr, tokens[b].tolist(), parents, u[b].tolist(),
                                     temperature)
        assert margin > vocab * 2.0 ** -50  # 64 bits decide
        assert got[b] == (new, path), (b, got[b], new, path)
        lengths.append(len(new))
    return lengths


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("vocab", [65536, 65537, 70001, 128256, 200000])
def test_long_rows(dtype, drawn, vocab):
    """Row maxima, candidates and draws in front and back; rows whose first 64 parts and
    more are masked, and others whose last are."""
    parents = tree(4, 1) if drawn else tree(7, 3)
    N, batch = len(parents), 12
    for rate in (0.3, 0.9):
        logits, draft, tokens, u = inputs(batch, parents, vocab, drawn, dtype, vocab + int(10 * rate), rate)
        for x in (logits, draft) if drawn else (logits,):
            x = x.view(batch, N, vocab)
            x[1, :, vocab - 3] = 9.0     # the largest, in the last part
            x[2, :, 65535] = 9.0
            x[3, :, :65000] = -math.inf  # candidates there have no mass
            x[4, :, 70:] = -math.inf
            x[5, :, : vocab - 500] -= 40.0
        if not drawn:
            # candidates of the last part, with and without much of the mass
            kids = [c for c in range(N) if parents[c] == 0]
            for b in (6, 7, 8):
                for i, c in enumerate(kids):
                    tokens[b, c] = vocab - 2 - 7 * i
                    logits.view(batch, N, vocab)[b, 0, vocab - 2 - 7 * i] = 4.0 if b == 6 else 12.0 + i
        else:
            g = torch.Generator().manual_seed(vocab)
            q = torch.softmax(draft.double(), -1)
            keep = [r for r in range(batch * N) if r % N < N - 1]
            tokens.view(-1)[[r + 1 for r in keep]] = torch.multinomial(q[keep], 1, generator=g)[:, 0]
        u[8, 1:] = 0.999
        u[9, 0], u[10, 0], u[6, 0] = 1e-9, 1 - 1e-9, 1 - 1e-6
        lengths = agree(logits, draft, tokens, parents, u, 1.0, vocab)
        assert len(set(lengths)) > 1


@pytest.mark.parametrize("at", [3, 65535, 65536, 69000])
def test_rejected_tokens_with_most_of_the_mass(at):
    """Nearly all of a long row's mass in rejected candidates of one part: what is left
    decides, and the part's own sum does not."""
    V, parents = 70001, tree(4, 3)
    logits = torch.full((8 * 4, V), -16.0)
    kids = [at, at + 5, at + 20]
    logits[:, kids] = 0.0
    logits[:, 64 * 1024 + 700:] -= 3.0
    tokens = torch.tensor([[0] + kids] * 8)
    u = torch.full((8, 4), LAST, dtype=torch.float64)
    u[:, 0] = torch.linspace(0.001, 0.999, 8)
    for dtype in ("f32", "bf16"):
        assert agree(logits.to(R.TYPES[dtype]), None, tokens, parents, u, 1.0, V) == [1] * 8


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [300, 70001])
def test_nothing_left_takes_the_row(dtype, vocab):
    """Candidates are the only tokens with mass.  Where rounding rejects all of them, the
    next token comes from the row as if none had been."""
    batch, parents = 400, tree(5, 4)
    g = torch.Generator().manual_seed(vocab)
    logits = torch.full((batch, 5, vocab), -math.inf)
    ids = torch.stack([torch.randperm(vocab, generator=g)[:4] for _ in range(batch)])
    tokens = torch.cat((torch.zeros(batch, 1, dtype=torch.int64), ids), 1)
    z = (2.0 * torch.randn(batch, 4, generator=g)).to(R.TYPES[dtype]).float()
    for c in range(5):
        logits[:, c].scatter_(1, ids, z)
    logits = logits.to(R.TYPES[dtype]).view(batch * 5, vocab)
    u = torch.full((batch, 5), LAST, dtype=torch.float64)
    u[:, 0] = torch.rand(batch, generator=g, dtype=torch.float64)
    got = run(logits, None, tokens, parents, u, 1.0, vocab)
    order = ids.argsort(1)
    p = torch.softmax(z.double().gather(1, order), 1).cumsum(1)
    empty = 0
    for b, (new, path) in enumerate(got):
        if len(path) == 1:  # all rejected
            want = int(ids[b, order[b, int((p[b] <= u[b, 0] * p[b, -1]).sum())]])
            assert float((p[b] - u[b, 0]).abs().min()) > 2.0 ** -40 and new == [want]
            empty += 1
        else:
            assert new[0] in ids[b].tolist() and new[1] in ids[b].tolist()
    assert empty > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_residual_left_takes_the_row(dtype):
    """A draft that is the target but for a row's level: a rejection can only be rounding's,
    and a token with mass comes out."""
    batch, parents, vocab = 400, [-1, 0], 300
    g = torch.Generator().manual_seed(3)
    z = torch.full((batch, 2, vocab), -math.inf)
    ids = torch.stack([torch.randperm(vocab, generator=g)[:3] for _ in range(batch)])
    top = torch.randint(-8, 9, (batch, 3), generator=g).float()
    for c in range(2):
        z[:, c].scatter_(1, ids, top)
    logits, draft = z.to(R.TYPES[dtype]).view(-1, vocab), (z + 16.0).to(R.TYPES[dtype]).view(-1, vocab)
    tokens = torch.stack((torch.zeros(batch, dtype=torch.int64), ids[:, 0]), 1)
    u = torch.full((batch, 2), LAST, dtype=torch.float64)
    u[:, 0] = torch.rand(batch, generator=g, dtype=torch.float64)
    for b, (new, path) in enumerate(run(logits, draft, tokens, parents, u, 1.0, vocab)):
        assert all(t in ids[b].tolist() for t in new)


@pytest.mark.parametrize("low,high,first", [(-57.0, 130.0, 1024 + 77), (-50.0, 130.0, 0), (127.0, 190.0, 0),
                                            (100.0, 300.0, 1024 + 77)])
def test_weights_at_the_end_of_the_range(low, high, first):
    """1024 equal logits, then a part of far larger ones: the draw at 0 goes to the first
    token whose weight is above 0 in 64 bits, also where a part's weights have a sum and are
    no numbers themselves, in calls large enough for the table of exponentials and in small
    ones."""
    V = 2048
    row = torch.full((V,), -math.inf)
    row[:1024], row[1024 + 77], row[1024 + 300] = low, high, high - 2.0
    row = row.bfloat16()
    want = [R.accept(row[None], None, [0], [-1], [x], 0.25)[0] for x in (0.0, 0.5, LAST)]
    assert want == [[first], [1024 + 77], [1024 + 300]]
    for batch in (3, 5200):
        u = torch.tensor([0.0, 0.5, LAST], dtype=torch.float64).repeat(-(-batch // 3))[:batch, None]
        got = run(row.expand(batch, V).contiguous(), None, torch.zeros(batch, 1, dtype=torch.int64), [-1], u, 0.25, V)
        assert all(o == (want[i % 3], [0]) for i, o in enumerate(got)), got[:3]
