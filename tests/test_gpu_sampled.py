"""Sampled decoding in the engine: every step is the rule of chimera_accept on the step's
own logits and the documented random numbers, in every launch mode; and the operators
over the plain paged cache used one after another, as a decoding layer would."""
import math

import numpy as np
import pytest
import torch

import paged_ref as R
import synth
from gpu_helpers import make_session
from paper_2402_15758_amd import Session
from paper_2402_15758_amd import binding as B

pytestmark = pytest.mark.gpu
M64 = (1 << 64) - 1
SMALL = synth.small_config()


def mix(x):
    z = (x + 0x9E3779B97F4A7C15) & M64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    return z ^ (z >> 31)


def uniform(seed, b, n, i):
    return (mix(mix(mix(mix(seed) ^ b) ^ n) ^ i) >> 11) * 2.0 ** -53


# three levels of up to six children, out of order of ranks
WIDE = [(r,) for r in (3, 0, 1, 2, 5, 4)] + [(0, 1), (0, 0), (3, 0), (3, 2), (1, 0), (2, 0)] + [(0, 1, 0), (0, 0, 2),
                                                                                              (0, 0, 0), (3, 0, 1)]
TREES = {"T8": synth.TREES["T8"], "wide": WIDE, "none": ()}


def parents_of(tree):
    """Parents of synth's rank tuples, breadth first, the root's -1."""
    nodes = [()] + [tuple(t) for t in tree]
    return [-1] + [nodes.index(t[:-1]) for t in nodes[1:]]


def run_steps(sess, prompts, steps, seed, temperature, parents, check=True):
    first = sess.prefill(prompts)
    n = [len(p) for p in prompts]
    N = len(parents)
    out, lens = [[int(t)] for t in first], []
    for _ in range(steps):
        toks, cnt, path = sess.step()
        if check:
            logits = torch.from_numpy(sess.debug(B.DBG_VERIFY_LOGITS)).view(len(prompts), N, -1)
            tree = sess.debug(B.DBG_TREE_TOKENS)
        for b in range(len(prompts)):
            L = int(cnt[b])
            if check:
                assert int(tree[b, 0]) == out[b][-1]
                u = [uniform(seed, b, n[b], i) for i in range(N)]
                new, nodes, _ = R.accept(logits[b], None, tree[b].tolist(), parents, u, temperature)
                assert toks[b, :L].tolist() == new and path[b, :L].tolist() == nodes
            out[b] += toks[b, :L].tolist()
            n[b] += L
            lens.append(L)
    return out, lens


@pytest.mark.parametrize("tree_name", sorted(TREES))
def test_every_step_is_the_rule(tree_name):
    cfg = synth.TINY
    tree = TREES[tree_name]
    w = synth.make_weights(cfg, device="cuda", std=0.06)
    ps = [synth.make_prompt(n, cfg.vocab, 5 + n) for n in (30, 7, 64)]
    parents = parents_of(tree)
    sess = make_session(cfg, w, tree, max_batch=3, max_len=256)
    for seed, T in ((11, 1.0), (12, 0.25)):
        sess.set_sampling(T, seed)
        out, lens = run_steps(sess, ps, 8, seed, T, parents)
        assert all(len(o) == 1 + sum(lens[b::3]) for b, o in enumerate(out))
    # the same seed gives the same stream, replayed, eager and pipelined
    sess.set_sampling(0.25, 12)
    sess.set_graph(False)
    assert run_steps(sess, ps, 8, 12, 0.25, parents, check=False)[0] == out
    sess.set_graph(True)
    first = sess.prefill(ps)
    toks, cnt, _ = sess.steps(8)
    again = [[int(first[b])] + [int(t) for s in range(8) for t in toks[s, b, :cnt[s, b]]] for b in range(3)]
    assert again == out
    # and greedy decoding afterwards is what it was
    sess.set_decoding(False)
    greedy = sess.generate(ps, 10)[0]
    sess.close()
    fresh = make_session(cfg, w, tree, max_batch=3, max_len=256)
    assert fresh.generate(ps, 10)[0] == greedy
    fresh.close()


def test_first_tokens_follow_the_target():
    """One-step frequencies over 4000 seeds against the target's probabilities, from the
    prompt's last logits: 5 standard deviations; and the branch draft and bf16 weights run."""
    cfg = synth.TINY
    w = synth.make_weights(cfg, device="cuda", std=0.06)
    p = synth.make_prompt(20, cfg.vocab, 3)
    sess = make_session(cfg, w, (), max_len=64)
    counts, n = np.zeros(cfg.vocab), 4000
    sess.prefill([p])
    logits = torch.from_numpy(sess.debug(B.DBG_VERIFY_LOGITS))[0]
    q = R.softmax(logits, 0.5).numpy()
    for seed in range(n):
        sess.set_sampling(0.5, seed)
        t = int(sess.prefill([p])[0])
        counts[t] += 1
        if seed < 20:
            run = np.cumsum(q)
            assert t == int((run <= run[-1] * uniform(seed, 0, 20, 64)).sum())
    f = counts / n
    assert (np.abs(f - q) <= 5 * np.sqrt(q * (1 - q) / n) + 1.0 / n).all()
    sess.close()


def test_drafting_modes_and_formats():
    tree = synth.TREES["T32"]
    w = synth.make_weights(SMALL, device="cuda", std=0.06)
    ps = [synth.make_prompt(n, SMALL.vocab, n) for n in (40, 18)]
    for branch, kw in ((False, {}), (True, {}), (False, dict(weight_format="fp4", kv_format="fp4"))):
        sess = Session(SMALL, w, tree, max_batch=2, max_len=256, **kw)
        sess.set_drafting(branch)
        sess.trigram_cache(1 << 10)
        sess.set_sampling(0.7, 3)
        run_steps(sess, ps, 5, 3, 0.7, parents_of(tree))
        sess.close()


def test_refusals():
    cfg = synth.TINY
    w = synth.make_weights(cfg, device="cuda")
    sess = make_session(cfg, w, (), max_len=64)
    for t in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(B.ChimeraError):
            sess.set_sampling(t)
    with pytest.raises(B.ChimeraError):
        B.chimera_set_decoding(sess.ctx, 3)
    sess.close()


# ---- the operators one after another -------------------------------------------------
class Layer:
    """A decoding layer's operators over one paged cache: rows in, attention, a
    projection to logits, verification.  Everything a step changes lies on the device."""

    def __init__(self, dtype, Hq, H, hd, page, batch, chain, vocab, seed, window=0, sinks=0):
        g = torch.Generator().manual_seed(seed)
        self.dt = {"bf16": B.CHIMERA_BF16, "f32": B.CHIMERA_F32}[dtype]
        t = R.TYPES[dtype]
        self.shape = (Hq, H, hd, page, batch, chain, vocab)
        self.window, self.sinks = window, sinks
        per = 20
        self.table = torch.randperm(batch * per, generator=g).view(batch, per).int().cuda()
        self.pool = torch.full((batch * per, 2, H, page, hd), math.nan, dtype=t, device="cuda")
        self.cache = B.chimera_paged(self.pool.data_ptr(), self.pool.numel() * self.pool.element_size(),
                                     self.table.data_ptr(), batch, per, batch * per, page, H, hd, self.dt)
        self.rope = B.chimera_rope(hd, 0, per * page, 10000.0, 0, 1.0, 0, 0.0, 0.0, 1.0)
        nb = B.chimera_rope_bytes(self.rope)
        self.rt = torch.empty(nb, dtype=torch.uint8, device="cuda")
        B.chimera_rope_table(self.rope, self.rt.data_ptr(), nb, torch.cuda.current_stream().cuda_stream)
        self.gain = (1 + 0.2 * torch.randn(2, hd, generator=g)).cuda()
        self.head = (0.3 * torch.randn(Hq * hd, vocab, generator=g)).cuda()
        rows = batch * chain
        self.qkv = torch.zeros(rows, (Hq + 2 * H) * hd, dtype=t, device="cuda")
        self.n = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.seq = torch.arange(batch).repeat_interleave(chain).int().cuda()
        self.step = torch.arange(chain).repeat(batch).int().cuda()
        self.row0 = (torch.arange(batch + 1) * chain).int().cuda()
        self.tokens = torch.zeros(batch, chain, dtype=torch.int32, device="cuda")
        self.u = torch.zeros(batch, chain, dtype=torch.float64, device="cuda")
        self.q = torch.empty(rows, Hq * hd, dtype=t, device="cuda")
        self.out = torch.empty_like(self.q)
        self.logits = torch.empty(rows, vocab, device="cuda")
        self.pos = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.new = torch.zeros(batch, chain, dtype=torch.int32, device="cuda")
        self.count = torch.zeros(batch, dtype=torch.int32, device="cuda")
        wa = B.chimera_paged_attn_bytes(self.cache, Hq, rows)
        wb = B.chimera_accept_bytes(batch, chain, vocab, False)
        self.wa, self.wb = (torch.empty(k + 256, dtype=torch.uint8, device="cuda") for k in (wa, wb))
        self.sizes = (wa, wb)

    def enqueue(self):
        Hq, H, hd, page, batch, chain, vocab = self.shape
        st = torch.cuda.current_stream().cuda_stream
        torch.add(self.n.repeat_interleave(chain), self.step, out=self.pos)
        es, p = self.qkv.element_size(), self.qkv.data_ptr()
        B.chimera_paged_append(self.cache, self.dt, p, p + Hq * hd * es, p + (Hq + H) * hd * es, self.qkv.shape[1], Hq,
                               self.seq.data_ptr(), self.pos.data_ptr(), batch * chain, self.rope, self.rt.data_ptr(),
                               self.gain[0].data_ptr(), self.gain[1].data_ptr(), 1e-5, self.q.data_ptr(), Hq * hd, st)
        B.chimera_paged_attn(self.cache, self.q.data_ptr(), Hq * hd, Hq, self.row0.data_ptr(), self.n.data_ptr(),
                             batch * chain, self.window, self.sinks, hd ** -0.5, self.out.data_ptr(), Hq * hd,
                             self.wa.data_ptr(), self.sizes[0], st)
        torch.matmul(self.out.float(), self.head, out=self.logits)
        B.chimera_accept(B.CHIMERA_F32, self.logits.data_ptr(), vocab, None, 0, vocab, self.tokens.data_ptr(), None,
                         chain, batch, 0.9, self.u.data_ptr(), self.new.data_ptr(), self.count.data_ptr(), None,
                         self.wb.data_ptr(), self.sizes[1], st)
        self.n += self.count

    def feed(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=g, device="cuda"))
        self.tokens.copy_(torch.randint(0, self.shape[6], self.tokens.shape, generator=g, device="cuda"))
        self.u.copy_(0.2 * torch.rand(self.u.shape, generator=g, device="cuda", dtype=torch.float64))

    def check(self, held, n):
        """This step against float64; held: K and V rows so far, [batch] lists of rows."""
        Hq, H, hd, page, batch, chain, vocab = self.shape
        x = self.qkv.cpu().double().view(batch * chain, -1, hd)
        th = R.theta(hd, 10000.0)
        gain = self.gain.cpu()
        pos = (n.repeat_interleave(chain) + self.step.cpu())
        q = R.turn(R.norm(x[:, :Hq], gain[0], 1e-5), pos, th, "half")[0]
        k = R.turn(R.norm(x[:, Hq:Hq + H], gain[1], 1e-5), pos, th, "half")[0]
        got_q = self.q.cpu().double().view(batch * chain, Hq, hd)
        assert float((got_q - q).abs().max()) <= (0.05 if self.dt == B.CHIMERA_BF16 else 1e-4)
        lens, rows = n.tolist(), [chain] * batch
        pool = self.pool.cpu()
        out, mag, big = R.attention(got_q.to(R.TYPES["bf16" if self.dt == B.CHIMERA_BF16 else "f32"]), pool,
                                    self.table.cpu(), lens, rows, R.f32(hd ** -0.5), self.window, self.sinks)
        bound = R.attention_bound("bf16" if self.dt == B.CHIMERA_BF16 else "f32", out, mag, big, 400, hd)
        got = self.out.cpu().double().view(batch * chain, Hq, hd)
        assert bool(((got - out).abs() <= bound).all())
        logits = self.logits.cpu()
        for b in range(batch):
            new, _, _ = R.accept(logits[b * chain:(b + 1) * chain], None, self.tokens[b].tolist(),
                                 [i - 1 for i in range(chain)], self.u[b].tolist(), 0.9)
            assert self.new[b, :int(self.count[b])].tolist() == new


@pytest.mark.parametrize("dtype,window", [("bf16", 0), ("f32", 0), ("bf16", 40)])
def test_a_layer_step_by_step(dtype, window):
    layer = Layer(dtype, 6, 2, 64, 16, 3, 5, 500, 1, window, 3)
    for i in range(12):
        layer.feed(i)
        n = layer.n.cpu().clone()
        layer.enqueue()
        layer.check(None, n)
    assert int(layer.n.min()) >= 12


def test_two_captured_layers_replayed_with_eager_work_between():
    """Two graphs of a step, each with its own workspaces, replayed in turn on two streams
    with eager steps between: every replay gives the eager bits."""
    def fresh():
        return [Layer("bf16", 4, 2, 128, 16, 4, 4, 3000, s) for s in (1, 2)]

    want, layers = [], fresh()
    for i in range(6):
        for k, l in enumerate(layers):
            l.feed(10 * i + k)
            l.enqueue()
            torch.cuda.synchronize()
            want.append((l.out.clone(), l.new.clone(), l.count.clone(), l.n.clone()))
    layers, other = fresh(), Layer("f32", 4, 2, 64, 8, 2, 60, 100, 3)
    streams, graphs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for l, s in zip(layers, streams):
        with torch.cuda.stream(s):  # once outside: libraries set themselves up
            l.enqueue()
        torch.cuda.synchronize()
        l.n.zero_()
        l.pool.fill_(math.nan)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            l.enqueue()
        graphs.append(g)
        torch.cuda.synchronize()
        l.n.zero_()
    for i in range(6):
        for k, l in enumerate(layers):
            l.feed(10 * i + k)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):  # both at once
            with torch.cuda.stream(s):
                g.replay()
        other.feed(i)
        other.n.zero_()
        other.enqueue()
        torch.cuda.synchronize()
        for k, l in enumerate(layers):
            for got, ref in zip((l.out, l.new, l.count, l.n), want[2 * i + k]):
                assert torch.equal(got, ref), (i, k)
