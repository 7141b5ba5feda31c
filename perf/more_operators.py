"""Operators of sampled speculative decoding over a paged cache: what is timed
and compared, case by case.

Three operators, through the C ABI's names:

* ``append``: rows of a fused projection into a paged K/V cache, queries and keys
  normalised head by head and rotated on the way (chimera_paged_append).
* ``attn``: attention of a chunk of new tokens a sequence (one token, a prompt's
  chunk, a ragged mixture) over that cache, causal, with grouped heads and
  optionally a sliding window behind a few first tokens that stay visible
  (chimera_paged_attn).
* ``accept``: drafted tokens verified against the target's probabilities from
  given random numbers, and the next token (chimera_accept).

The cache: [page][K | V][head][slot][head_dim]; position p of sequence b lies in
slot p % page_size of page table[b][p // page_size].

Rotation: theta_i = base^(-2i / rot); "linear" divides it by the factor; "ramp"
multiplies it by w + (1 - w) / factor with w = clamp((t - low) / (high - low), 0, 1),
t = original * theta_i / (2 pi).  Pairs are (i, i + rot / 2) ("half") or
(2i, 2i + 1) ("pairs"); dimensions from rot on pass.

Verification: with candidates that were chosen (no draft logits) a node's children
are tested in order, child c accepted where u[c] (1 - mass of the rejected
siblings) < p(token of c); where all are rejected the next token comes from p
without them.  With a chain whose tokens were drawn from the draft, child c is
accepted where u[c] q < p at its token, else the next token comes from
max(p - q, 0).  A leaf's next token comes from p.  The next token is the first at
which the running sum of weights passes u[0] times their total.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ROPES = {
    # plain, over the whole head; part of a head in neighbouring pairs; both scaled forms
    "half": {"rot": 1.0, "layout": "half", "scaling": "none", "base": 10000.0},
    "pairs": {"rot": 0.5, "layout": "pairs", "scaling": "none", "base": 10000.0},
    "linear": {"rot": 1.0, "layout": "half", "scaling": "linear", "base": 10000.0, "factor": 4.0},
    "ramp": {"rot": 1.0, "layout": "half", "scaling": "ramp", "base": 500000.0, "factor": 8.0, "original": 8192,
             "low": 1.0, "high": 4.0, "gain": 1.05},
    "quarter": {"rot": 0.25, "layout": "half", "scaling": "none", "base": 10000.0},
}
EPS = 1e-5
MAX_POSITIONS = 33024


def _append(name, dtype, held, batch, rows, heads, kv_heads, hd, page, first, rope, norm):
    return {"name": name, "op": "append", "dtype": dtype, "held": held, "batch": batch, "rows": rows, "heads": heads,
            "kv_heads": kv_heads, "hd": hd, "page": page, "first": first, "rope": rope, "norm": norm}


def _attn(name, dtype, batch, lo, hi, rows_lo, rows, heads, kv_heads, hd, page, window=0, sinks=0):
    return {"name": name, "op": "attn", "dtype": dtype, "batch": batch, "lo": lo, "hi": hi, "rows_lo": rows_lo,
            "rows": rows, "heads": heads, "kv_heads": kv_heads, "hd": hd, "page": page, "window": window,
            "sinks": sinks}


def _accept(name, dtype, batch, nodes, arity, vocab, drawn, rate, temperature):
    return {"name": name, "op": "accept", "dtype": dtype, "batch": batch, "nodes": nodes, "arity": arity,
            "vocab": vocab, "drawn": drawn, "rate": rate, "temperature": temperature}


def listed():
    return [
        # one token of a 7B layer: launches and latency
        _append("append_bf16_m1", "bf16", "bf16", 1, 1, 32, 32, 128, 16, 512, "half", False),
        # eight sequences' eight new tokens, grouped heads, norms, half of a head rotated in pairs
        _append("append_bf16_b8_norm", "bf16", "bf16", 8, 8, 32, 8, 128, 16, 1000, "pairs", True),
        # a prompt's 2044 tokens, from a product's 32-bit output into a 16-bit cache, far positions
        _append("append_f32_bf16_prefill", "f32", "bf16", 4, 511, 32, 8, 128, 16, 16000, "ramp", True),
        # the smallest model's 8 tokens after a 32-token prompt: latency
        _attn("attn_f32_r8", "f32", 1, 32, 32, 8, 8, 4, 4, 64, 16),
        # greedy decoding of eight long ragged sequences: one token each
        _attn("attn_bf16_b8_single", "bf16", 8, 1024, 4096, 1, 1, 32, 32, 128, 16),
        # one token over a long context with grouped heads
        _attn("attn_bf16_long", "bf16", 1, 32768, 32768, 1, 1, 32, 8, 128, 64),
        # the second 2048-token chunk of a 4096-token prompt at 7B width
        _attn("attn_bf16_chunk", "bf16", 1, 2048, 2048, 2048, 2048, 32, 32, 128, 16),
        # a served mixture: single tokens beside chunks, windowed with four first tokens kept
        _attn("attn_bf16_mixed_window", "bf16", 8, 500, 16000, 1, 300, 32, 8, 128, 16, 1024, 4),
        # a 300-token prompt of a 32-bit model
        _attn("attn_f32_prompt", "f32", 1, 0, 0, 300, 300, 16, 16, 64, 8),
        # a 64-node tree of chosen candidates
        _accept("accept_f32_t64", "f32", 1, 64, 4, 32000, False, 0.7, 1.0),
        # eight chains of four drawn tokens
        _accept("accept_f32_b8_drawn", "f32", 8, 5, 1, 32000, True, 0.8, 0.8),
        # a large batch over a large vocabulary in 16 bits
        _accept("accept_bf16_b64_drawn", "bf16", 64, 6, 1, 128256, True, 0.7, 1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "attn", "attn", "attn", "accept", "accept"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "append":
        batch = rng.choice([1, 1, 2, 3, 8])
        kv_heads = rng.choice([1, 4, 8, 32])
        heads = kv_heads * (rng.choice([1, 2, 4, 7]) if kv_heads <= 8 else 1)
        hd = rng.choice([64, 128])
        most = 2044 * (32 + 16) * 128 // ((heads + 2 * kv_heads) * hd * batch)
        c = _append("", dtype, rng.choice(["bf16", dtype]), batch, _log(rng, 1, min(2044 // batch, most)), heads,
                    kv_heads, hd, rng.choice([1, 8, 16, 64, 256]), rng.choice([0, 1, 37, 1000, 30000]),
                    rng.choice(sorted(ROPES)), rng.choice([False, True]))
    elif op == "attn":
        while True:
            batch = rng.choice([1, 1, 2, 3, 8])
            kv_heads = rng.choice([1, 4, 8, 32])
            heads = kv_heads * (rng.choice([1, 1, 2, 4, 7]) if kv_heads <= 8 else 1)
            rows = rng.choice([1, 1, _log(rng, 1, 64), _log(rng, 1, 2048)])
            hi = _log(rng, 1, 32768 // max(1, batch * kv_heads // 8))
            lo = max(0, int(hi * rng.uniform(0.0, 1.0)))
            window = rng.choice([0, 0, _log(rng, 1, 4096)])
            c = _attn("", dtype, batch, lo, hi, rng.choice([1, rows]), rows, heads, kv_heads, rng.choice([64, 128]),
                      rng.choice([1, 8, 16, 16, 64, 256]), window, rng.choice([0, 1, 4, 30]) if window else 0)
            if batch * rows * heads <= 2048 * 32 and work(c)["flops"] * (12 if dtype == "f32" else 1) <= 1.03e11:
                break
    else:
        drawn = rng.choice([False, True])
        arity = 1 if drawn else rng.choice([1, 2, 4])
        nodes = rng.choice([1, 2, 3, 6, 9]) if arity == 1 else rng.choice([3, 8, 32, 37, 64])
        vocab = rng.choice([1000, _log(rng, 100, 128256), 32000, 128256])
        batch = max(1, min(_log(rng, 1, 64), 64 * 6 * 128256 // (nodes * vocab)))
        c = _accept("", rng.choice(["bf16", "f32"]), batch, nodes, arity, vocab, drawn, rng.uniform(0.3, 0.95),
                    rng.choice([0.6, 0.8, 1.0, 1.3]))
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _pages(g, batch, positions, page):
    """A shuffled page table that covers `positions` a sequence and the pages
    in all; one page is nobody's."""
    per = -(-positions // page)
    order = torch.randperm(batch * per + 1, generator=g, device="cuda")[: batch * per]
    return order.view(batch, per).to(torch.int32), batch * per + 1


def _append_inputs(c, seed):
    g, t = _gen(seed), TYPES[c["dtype"]]
    B, R, H, Hk, hd = c["batch"], c["rows"], c["heads"], c["kv_heads"], c["hd"]
    # the table names the pages of the whole context, the pool holds those the rows touch
    lead, per = c["first"] // c["page"], -(-(c["first"] + R) // c["page"])
    part, n_pages = _pages(g, B, (per - lead) * c["page"], c["page"])
    table = torch.zeros(B, per, dtype=torch.int32, device="cuda")
    table[:, lead:] = part
    width = (H + 2 * Hk) * hd
    qkv = (_randn(g, B * R, width) * torch.exp(0.7 * _randn(g, width))).to(t)
    seq = torch.arange(B, device="cuda").repeat_interleave(R).to(torch.int32)
    pos = (c["first"] + torch.arange(R, device="cuda")).repeat(B).to(torch.int32)
    gains = 1.0 + 0.2 * _randn(g, 2, hd)
    return qkv, seq, pos, table, n_pages, gains


def _spread(lo, hi, n, i):
    return int(lo + (hi - lo) * ((5 * i + 3) % n) / (n - 1)) if n > 1 else hi


def _lens(c):
    return [_spread(c["lo"], c["hi"], c["batch"], i) for i in range(c["batch"])]


def _rows(c):
    """New tokens a sequence: in a mixture one place in four holds a chunk."""
    n = c["batch"]
    if c["rows_lo"] == c["rows"] or n == 1:
        return [c["rows"]] * n
    return [c["rows"] if i % 4 == 1 else c["rows_lo"] for i in range(n)]


def _attn_inputs(c, seed):
    g, t = _gen(seed), TYPES[c["dtype"]]
    B, Hk, hd, page = c["batch"], c["kv_heads"], c["hd"], c["page"]
    lens, rows = _lens(c), _rows(c)
    table, n_pages = _pages(g, B, max(n + r for n, r in zip(lens, rows)), page)
    q = _randn(g, sum(rows), c["heads"] * hd).to(t)
    wide = torch.exp(0.4 * _randn(g, hd))  # keys with a few wide dimensions
    pool = torch.empty(n_pages, 2, Hk, page, hd, dtype=t, device="cuda")
    step = max(1, (1 << 26) // (2 * Hk * page * hd))
    for i in range(0, n_pages, step):
        kv = _randn(g, *pool[i:i + step].shape)
        kv[:, 0] *= wide
        pool[i:i + step] = kv.to(t)
    for b in range(B):  # slots past a sequence's tokens: nobody has written them
        p = torch.arange(lens[b] + rows[b], table.shape[1] * page, device="cuda")
        pool[table[b][p // page].long(), :, :, p % page] = math.nan
    return q, pool, table, n_pages, lens, rows


def _parents(c):
    """Breadth-first tree of the given arity; arity 1 is a chain."""
    return [-1] + [(i - 1) // c["arity"] for i in range(1, c["nodes"])]


def _depth(c):
    d = [0] * c["nodes"]
    for i, p in enumerate(_parents(c)):
        d[i] = d[p] + 1 if p >= 0 else 0
    return max(d)


def _peaked(g, rows, vocab):
    """Log-probabilities like a language model's: a few likely tokens, a long tail."""
    z = 1.5 * _randn(g, rows, vocab)
    top = torch.randint(0, vocab, (rows, 12), generator=g, device="cuda")
    z.scatter_(1, top, 8.0 + 2.0 * _randn(g, rows, 12))
    return torch.log_softmax(z, -1)


def _accept_inputs(c, seed):
    g, t = _gen(seed), TYPES[c["dtype"]]
    B, N, V, T, a = c["batch"], c["nodes"], c["vocab"], c["temperature"], c["rate"]
    parents = _parents(c)
    tokens = torch.zeros(B, N, dtype=torch.int64, device="cuda")
    p = _peaked(g, B * N, V)
    draft = None
    if c["drawn"]:
        # p = a q + (1 - a) another: a draw from q is accepted with a little over a
        q = _peaked(g, B * N, V)
        p = torch.logaddexp(q + math.log(a), p + math.log1p(-a))
        for u in range(1, N):
            e = -torch.log(-torch.log(torch.rand(B, V, generator=g, device="cuda").clamp(1e-30, 1 - 1e-7)))
            tokens[:, u] = (q.view(B, N, V)[:, u - 1] + e).argmax(-1)
        draft = (T * q + _randn(g, B * N, 1)).to(t)
    else:
        # a node's candidates: distinct tokens that hold the mass a, the first ones more
        p = p.view(B, N, V)
        for u in range(N):
            kids = [i for i in range(N) if parents[i] == u]
            if kids:
                ids = torch.topk(torch.rand(B, V, generator=g, device="cuda"), len(kids), -1).indices
                tokens[:, kids] = ids
                share = torch.tensor([0.5 ** i for i in range(len(kids))], device="cuda")
                p[:, u].scatter_(1, ids, -math.inf)
                rest = torch.log1p(torch.tensor(-a, device="cuda")) - torch.logsumexp(p[:, u], -1, keepdim=True)
                p[:, u] += rest
                p[:, u].scatter_(1, ids, torch.log(a * share / share.sum()).expand(B, -1))
        p = p.view(B * N, V)
    # logits: a row's level is free
    logits = (T * p + _randn(g, B * N, 1)).to(t)
    u = torch.rand(B, N, generator=g, device="cuda", dtype=torch.float64)
    return logits, draft, tokens.to(torch.int32), u


# ---- the rotation's table --------------------------------------------------------
def _rot(c):
    r = ROPES[c["rope"]]
    return int(r["rot"] * c["hd"])


def _theta(c):
    r, rot = ROPES[c["rope"]], _rot(c)
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    th = float(r["base"]) ** (-2.0 * i / rot)
    if r["scaling"] == "linear":
        th = th / r["factor"]
    elif r["scaling"] == "ramp":
        t = r["original"] * th / (2 * math.pi)
        w = ((t - r["low"]) / (r["high"] - r["low"])).clamp(0, 1)
        th = th * (w + (1 - w) / r["factor"])
    return th, r.get("gain", 1.0)


def _table(c):
    th, gain = _theta(c)
    ang = torch.arange(MAX_POSITIONS, dtype=torch.float64, device="cuda")[:, None] * th
    return (torch.cos(ang) * gain).float(), (torch.sin(ang) * gain).float()


# ---- what is measured ------------------------------------------------------------
def prepare(case, seed):
    c = dict(case)
    st = {"case": c}
    if own:
        import numpy as np
        from paper_2402_15758_amd import binding as B
        st["B"] = B
        dts = {"bf16": B.CHIMERA_BF16, "f32": B.CHIMERA_F32}
        st["dt"] = dts[c["dtype"]]
    if c["op"] == "append":
        qkv, seq, pos, table, n_pages, gains = _append_inputs(c, seed)
        H, page, hd = c["kv_heads"], c["page"], c["hd"]
        pool = torch.zeros(n_pages, 2, H, page, hd, dtype=TYPES[c["held"]], device="cuda")
        st.update(qkv=qkv, seq=seq, pos=pos, table=table, pool=pool, gains=gains)
        if own:
            r = ROPES[c["rope"]]
            st["rope"] = B.chimera_rope(
                _rot(c), B.CHIMERA_ROPE_PAIRS if r["layout"] == "pairs" else B.CHIMERA_ROPE_HALF, MAX_POSITIONS,
                r["base"], {"none": B.CHIMERA_ROPE_NONE, "linear": B.CHIMERA_ROPE_LINEAR,
                            "ramp": B.CHIMERA_ROPE_RAMP}[r["scaling"]],
                r.get("factor", 1.0), r.get("original", 0), r.get("low", 0.0), r.get("high", 0.0), r.get("gain", 1.0))
            nb = B.chimera_rope_bytes(st["rope"])
            st["rt"] = torch.empty(nb, dtype=torch.uint8, device="cuda")
            B.chimera_rope_table(st["rope"], st["rt"].data_ptr(), nb, torch.cuda.current_stream().cuda_stream)
            st["kv"] = B.chimera_paged(pool.data_ptr(), pool.numel() * pool.element_size(), table.data_ptr(),
                                       table.shape[0], table.shape[1], n_pages, page, H, hd, dts[c["held"]])
            torch.cuda.synchronize()
        else:
            st["cos"], st["sin"] = _table(c)
        return st
    if c["op"] == "attn":
        q, pool, table, n_pages, lens, rows = _attn_inputs(c, seed)
        st.update(q=q, pool=pool, table=table, lens=lens, rows=rows,
                  n=torch.tensor(lens, dtype=torch.int32, device="cuda"))
        if own:
            st["kv"] = B.chimera_paged(pool.data_ptr(), pool.numel() * pool.element_size(), table.data_ptr(),
                                       table.shape[0], table.shape[1], n_pages, c["page"], c["kv_heads"], c["hd"],
                                       st["dt"])
            starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
            # single tokens need no starts
            st["row0"] = None if max(rows) == 1 else torch.from_numpy(starts).cuda()
            wb = B.chimera_paged_attn_bytes(st["kv"], c["heads"], sum(rows))
            st["ws"], st["wsb"] = torch.empty(wb + 256, dtype=torch.uint8, device="cuda"), wb
        return st
    logits, draft, tokens, u = _accept_inputs(c, seed)
    st.update(logits=logits, draft=draft, tokens=tokens, u=u, parents=_parents(c), depth=_depth(c))
    if own:
        st["parent"] = np.array(st["parents"], dtype=np.int32)
        wb = B.chimera_accept_bytes(c["batch"], c["nodes"], c["vocab"], c["drawn"])
        st["ws"], st["wsb"] = torch.empty(wb + 256, dtype=torch.uint8, device="cuda"), wb
    return st


def run(st):
    c = st["case"]
    return {"append": _run_append, "attn": _run_attn, "accept": _run_accept}[c["op"]](st, c)


def _run_append(st, c):
    H, Hk, hd, page = c["heads"], c["kv_heads"], c["hd"], c["page"]
    qkv, pool = st["qkv"], st["pool"]
    rows, width = qkv.shape
    if own:
        B, es = st["B"], qkv.element_size()
        q_out = torch.empty(rows, H * hd, dtype=pool.dtype, device="cuda")
        gq, gk = (st["gains"][0].data_ptr(), st["gains"][1].data_ptr()) if c["norm"] else (None, None)
        p = qkv.data_ptr()
        B.chimera_paged_append(st["kv"], st["dt"], p, p + H * hd * es, p + (H + Hk) * hd * es, width, H,
                               st["seq"].data_ptr(), st["pos"].data_ptr(), rows, st["rope"], st["rt"].data_ptr(), gq,
                               gk, EPS, q_out.data_ptr(), H * hd, torch.cuda.current_stream().cuda_stream)
        return q_out, pool
    x = qkv.float().view(rows, H + 2 * Hk, hd)
    qk, v = x[:, :H + Hk], x[:, H + Hk:]
    if c["norm"]:
        gain = torch.cat((st["gains"][0].expand(H, hd), st["gains"][1].expand(Hk, hd)))
        qk = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + EPS) * gain
    rot, pos = _rot(c), st["pos"].long()
    cos, sin = st["cos"][pos][:, None], st["sin"][pos][:, None]
    out = qk.clone()
    if ROPES[c["rope"]]["layout"] == "half":
        a, b = qk[..., :rot // 2], qk[..., rot // 2:rot]
        out[..., :rot // 2], out[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = qk[..., 0:rot:2], qk[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
    pg, slot = st["table"][st["seq"].long(), pos // page].long(), pos % page
    pool[pg, 0, :, slot] = out[:, H:].to(pool.dtype)
    pool[pg, 1, :, slot] = v.to(pool.dtype)
    return out[:, :H].to(pool.dtype).reshape(rows, H * hd), pool


def _run_attn(st, c):
    Hq, Hk, page, hd, W = c["heads"], c["kv_heads"], c["page"], c["hd"], c["window"]
    q = st["q"]
    if own:
        out = torch.empty_like(q)
        row0 = st["row0"]
        st["B"].chimera_paged_attn(st["kv"], q.data_ptr(), Hq * hd, Hq, None if row0 is None else row0.data_ptr(),
                                   st["n"].data_ptr(), q.shape[0], W, c["sinks"], hd ** -0.5, out.data_ptr(), Hq * hd,
                                   st["ws"].data_ptr(), st["wsb"], torch.cuda.current_stream().cuda_stream)
        return out
    outs, r0 = [], 0
    for b, (n, R) in enumerate(zip(st["lens"], st["rows"])):
        at = torch.arange(n, n + R, device="cuda")
        keys = torch.arange(n + R, device="cuda")
        if W:
            keys = keys[(keys > n - W) | (keys < c["sinks"])]
        pg, slot = st["table"][b][keys // page].long(), keys % page
        kv = st["pool"][pg, :, :, slot].float()  # [keys][2][Hk][hd]
        x = q[r0:r0 + R].float().view(R, Hk, Hq // Hk, hd).permute(1, 2, 0, 3).reshape(Hk, -1, hd)
        seen = keys[None] <= at[:, None]
        if W:
            seen &= (keys[None] > at[:, None] - W) | (keys[None] < c["sinks"])
        s = torch.matmul(x, kv[:, 0].permute(1, 2, 0).contiguous()) * hd ** -0.5
        s = s.view(Hk, -1, R, keys.numel()).masked_fill_(~seen, -math.inf)
        e = torch.exp(s - s.amax(-1, keepdim=True))
        e = (e / e.sum(-1, keepdim=True)).view(Hk, -1, keys.numel())
        o = torch.matmul(e, kv[:, 1].transpose(0, 1).contiguous())
        outs.append(o.view(Hk, -1, R, hd).permute(2, 0, 1, 3).reshape(R, Hq * hd))
        r0 += R
    return torch.cat(outs).to(q.dtype)


def _run_accept(st, c):
    B, N, V, D = c["batch"], c["nodes"], c["vocab"], st["depth"]
    logits, draft = st["logits"], st["draft"]
    new = torch.empty(B, D + 1, dtype=torch.int32, device="cuda")
    count = torch.empty(B, dtype=torch.int32, device="cuda")
    path = torch.empty(B, D + 1, dtype=torch.int32, device="cuda")
    if own:
        st["B"].chimera_accept(st["dt"], logits.data_ptr(), V, None if draft is None else draft.data_ptr(), V, V,
                               st["tokens"].data_ptr(), st["parent"], N, B, c["temperature"], st["u"].data_ptr(),
                               new.data_ptr(), count.data_ptr(), path.data_ptr(), st["ws"].data_ptr(), st["wsb"],
                               torch.cuda.current_stream().cuda_stream)
        return new, count, path
    # all sequences walk together, on the device, one tested node at a time
    rows, dev = torch.arange(B, device="cuda"), "cuda"
    p = _softmax64(logits, c["temperature"]).view(B, N, V)
    q = None if draft is None else _softmax64(draft, c["temperature"]).view(B, N, V)
    tokens = st["tokens"].long()
    u = st["u"]
    cur = torch.zeros(B, dtype=torch.long, device=dev)  # the node the walk has reached
    gone = torch.zeros(B, dtype=torch.float64, device=dev)  # mass of the siblings rejected there
    w = p[:, 0].clone()  # the next token's weights there
    new.fill_(-1)
    path.fill_(-1)
    path[:, 0] = 0
    depth = torch.zeros(B, dtype=torch.long, device=dev)
    for x in range(1, N):  # breadth-first ids: a node's children follow it in order
        par = st["parents"][x]
        here = cur == par
        t = tokens[:, x]
        px = p[rows, par, t] if q is not None else w[rows, t]
        if q is None:
            ok = here & (u[:, x] * (1 - gone) < px)
            lost = here & ~ok
            gone = torch.where(lost, gone + px, gone)
            w[rows, t] = torch.where(lost, 0.0, w[rows, t])
        else:
            ok = here & (u[:, x] * q[rows, par, t] < px)
            lost = here & ~ok
            w = torch.where(lost[:, None], (p[:, par] - q[:, par]).clamp(min=0), w)
        cur = torch.where(ok, x, cur)
        gone = torch.where(ok, 0.0, gone)
        w = torch.where(ok[:, None], p[:, x], w)
        new[rows, depth] = torch.where(ok, t, new[rows, depth].long()).int()
        depth = depth + ok
        path[rows, depth] = torch.where(ok, x, path[rows, depth].long()).int()
    run_sum = torch.cumsum(w, -1)
    new[rows, depth] = (run_sum <= u[:, :1] * run_sum[:, -1:]).sum(-1).int()
    return new, (depth + 1).int(), path


def _softmax64(x, temperature):
    z = x.double() / temperature
    e = torch.exp(z - z.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _seen(c):
    """Pairs of a query and a key it sees (of one head), and the positions some query sees."""
    pairs = held = 0
    for n, r in zip(_lens(c), _rows(c)):
        W, S = c["window"], c["sinks"]
        if not W:
            pairs += r * n + r * (r + 1) // 2
            held += n + r
            continue
        for p in range(n, n + r):
            pairs += min(p + 1, W + min(S, max(0, p + 1 - W)))
        first = max(0, n - W + 1)
        held += n + r - first + min(S, first)
    return pairs, held


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "append":
        hs = 2 if c["held"] == "bf16" else 4
        rows, wide = c["batch"] * c["rows"], (c["heads"] + 2 * c["kv_heads"]) * c["hd"]
        return {"bytes": rows * (wide * (es + hs) + 4 * _rot(c) + 8), "flops": 8.0 * rows * wide}
    if c["op"] == "attn":
        pairs, held = _seen(c)
        return {"bytes": held * 2 * c["kv_heads"] * c["hd"] * es + 2 * sum(_rows(c)) * c["heads"] * c["hd"] * es,
                "flops": 4.0 * pairs * c["heads"] * c["hd"]}
    # the rows on the path: a node's children are accepted at the case's rate
    visited = sum(c["rate"] ** d for d in range(_depth(c) + 1))
    rows = c["batch"] * (visited + (min(visited, _depth(c)) if c["drawn"] else 0))
    return {"bytes": rows * c["vocab"] * es + 12 * c["batch"] * c["nodes"], "flops": 4.0 * rows * c["vocab"]}


# ---- the definition in 64 bits ----------------------------------------------------
def exact(case, seed):
    c = case
    return {"append": _exact_append, "attn": _exact_attn, "accept": _exact_accept}[c["op"]](c, seed)


def _exact_append(c, seed):
    qkv, seq, pos, table, n_pages, gains = _append_inputs(c, seed)
    H, Hk, hd, page = c["heads"], c["kv_heads"], c["hd"], c["page"]
    rows = qkv.shape[0]
    x = qkv.double().view(rows, -1, hd)
    if c["norm"]:
        for lo, hi, g in ((0, H, gains[0]), (H, H + Hk, gains[1])):
            part = x[:, lo:hi]
            x[:, lo:hi] = part / torch.sqrt(part.pow(2).sum(-1, keepdim=True) / hd + EPS) * g.double()
    th, gain = _theta(c)
    P = th.numel()
    # rotation as a complex product
    turn = torch.polar(torch.full((rows, P), gain, dtype=torch.float64, device="cuda"), pos.double()[:, None] * th)
    first, second = (slice(0, P), slice(P, 2 * P)) if ROPES[c["rope"]]["layout"] == "half" else (
        slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    y = torch.complex(x[:, :H + Hk, first].contiguous(), x[:, :H + Hk, second].contiguous()) * turn[:, None]
    x[:, :H + Hk, first], x[:, :H + Hk, second] = y.real, y.imag
    pool = torch.zeros(n_pages * page, 2, Hk, hd, dtype=torch.float64, device="cuda")
    at = table[seq.long(), pos.long() // page].long() * page + pos.long() % page
    pool[at, 0], pool[at, 1] = x[:, H:H + Hk], x[:, H + Hk:]
    pool = pool.view(n_pages, page, 2, Hk, hd).permute(0, 2, 3, 1, 4).contiguous()
    return x[:, :H].reshape(rows, H * hd), pool


def _exact_attn(c, seed):
    q, pool, table, n_pages, lens, rows = _attn_inputs(c, seed)
    Hq, Hk, hd, page = c["heads"], c["kv_heads"], c["hd"], c["page"]
    out = torch.empty(q.shape[0], Hq, hd, dtype=torch.float64, device="cuda")
    r0 = 0
    for b, (n, R) in enumerate(zip(lens, rows)):
        for i in range(0, R, 256):  # queries at a time, over what any of them may see
            m = min(256, R - i)
            last = n + i + m
            first = max(0, n + i - c["window"] + 1) if c["window"] else 0
            lead = min(first, c["sinks"]) if c["window"] else 0
            keys = torch.cat((torch.arange(lead, device="cuda"), torch.arange(first, last, device="cuda")))
            held = pool[table[b, keys // page].long(), :, :, keys % page].double()
            p = torch.arange(n + i, last, device="cuda")[:, None]
            hidden = keys[None] > p
            if c["window"]:
                hidden |= (p - keys[None] >= c["window"]) & (keys[None] >= c["sinks"])
            for h in range(Hq):
                k, v = held[:, 0, h * Hk // Hq], held[:, 1, h * Hk // Hq]
                x = q[r0 + i:r0 + i + m].view(m, Hq, hd)[:, h].double()
                s = torch.matmul(x, k.t().contiguous()) / math.sqrt(hd)
                w = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
                out[r0 + i:r0 + i + m, h] = torch.matmul(w, v.contiguous())
        r0 += R
    return out.view(-1, Hq * hd)


def _exact_accept(c, seed):
    logits, draft, tokens, u = _accept_inputs(c, seed)
    B, N, T, D = c["batch"], c["nodes"], c["temperature"], _depth(c)
    parents = _parents(c)
    tok, uu = tokens.tolist(), u.tolist()
    new = torch.full((B, D + 1), -1, dtype=torch.int32)
    path = torch.full((B, D + 1), -1, dtype=torch.int32)
    count = torch.zeros(B, dtype=torch.int32)
    for b in range(B):
        node, d = 0, 0
        while True:
            path[b, d] = node
            w = torch.softmax(logits[b * N + node].double() / T, -1)
            r = None if draft is None else torch.softmax(draft[b * N + node].double() / T, -1)
            kids, taken, left = [i for i in range(N) if parents[i] == node], None, 1.0
            for k in kids:
                x = tok[b][k]
                if (uu[b][k] * left if r is None else uu[b][k] * float(r[x])) < float(w[x]):
                    taken = k
                    break
                if r is None:
                    left -= float(w[x])
                    w[x] = 0.0
                else:
                    w = torch.relu(w - r)
            if taken is None:
                total = torch.cumsum(w, 0)
                new[b, d] = int(torch.searchsorted(total, total[-1] * uu[b][0], right=True))
                count[b] = d + 1
                break
            new[b, d] = tok[b][taken]
            node, d = taken, d + 1
    return new.cuda(), count.cuda(), path.cuda()
