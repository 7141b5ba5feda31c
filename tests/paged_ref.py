"""Plain forms in float64 of the operators over a plain paged cache and of the
verification of drafted tokens, for tests: no code of the library's."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


# ---- rotation and norms ------------------------------------------------------------
def theta(rot, base, scaling="none", factor=1.0, original=0, low=0.0, high=0.0):
    out = []
    for i in range(rot // 2):
        th = f32(base) ** (-2.0 * i / rot)
        if scaling == "linear":
            th /= f32(factor)
        elif scaling == "ramp":
            turns = original * th / (2 * math.pi)
            w = min(max((turns - f32(low)) / (f32(high) - f32(low)), 0.0), 1.0)
            th *= w + (1 - w) / f32(factor)
        out.append(th)
    return torch.tensor(out, dtype=torch.float64)


def norm(x, gain, eps):
    x = x.double()
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + f32(eps)) * gain.double()


def turn(x, pos, th, layout, gain=1.0):
    """x [rows][heads][hd] turned by pos; and the sum of magnitudes behind each value."""
    y, mag = x.double().clone(), x.double().abs().clone()
    n = th.numel()
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    ang = pos.double()[:, None] * th
    c, s = (torch.cos(ang) * f32(gain))[:, None], (torch.sin(ang) * f32(gain))[:, None]
    u, v = x.double()[..., a], x.double()[..., b]
    y[..., a], y[..., b] = u * c - v * s, u * s + v * c
    # a table's value is off by a rounding of 1, not of itself
    mag[..., a] = mag[..., b] = (u.abs() + v.abs()) * abs(f32(gain))
    return y, mag


# ---- attention ---------------------------------------------------------------------
def sees(p, keys, window, sinks):
    ok = keys <= p
    if window:
        ok = ok & ((keys > p - window) | (keys < sinks))
    return ok


def attention(q, pool, table, lens, rows, scale, window=0, sinks=0):
    """q [sum rows][Hq][hd], pool [pages][2][H][ps][hd] (NaN past what is written is
    fine).  Values, and for each the bound's pieces: sum of weights times |v|, and the
    largest sum of |q k| scale behind a score."""
    n_pages, _, H, ps, hd = pool.shape
    Hq = q.shape[1]
    out = torch.zeros(q.shape[0], Hq, hd, dtype=torch.float64)
    mag, big = torch.zeros_like(out), torch.zeros(q.shape[0], Hq, 1, dtype=torch.float64)
    r0 = 0
    for b, (n, R) in enumerate(zip(lens, rows)):
        if n < 0:
            r0 += R
            continue
        keys = torch.arange(min(n + R, table.shape[1] * ps))
        page = table[b][keys // ps].long()
        there = (page >= 0) & (page < n_pages)
        keys, page = keys[there], page[there]
        kv = pool[page, :, :, keys % ps].double()  # [keys][2][H][hd]
        for r in range(R):
            ok = sees(n + r, keys, window, sinks)
            if not bool(ok.any()):
                continue
            k, v = kv[ok, 0], kv[ok, 1]
            for h in range(Hq):
                c = h * H // Hq
                x = q[r0 + r, h].double()
                s = (k[:, c] @ x) * scale
                w = torch.softmax(s, 0)
                out[r0 + r, h] = (w[:, None] * v[:, c]).sum(0)
                mag[r0 + r, h] = (w[:, None] * v[:, c].abs()).sum(0)
                big[r0 + r, h] = ((k[:, c].abs() @ x.abs()) * abs(scale)).max()
        r0 += R
    return out, mag, big


def attention_bound(dtype, ref, mag, big, n, hd):
    """|error| of a result: its own rounding; a score's hd products and sums, the
    scaling and the exponential (in base 2, whose argument's rounding is relative to the
    score) to 2^-23 each of the sum of magnitudes, in numerator and denominator; n
    weights summed, each rounded once to bf16 (2^-8) where the cache is."""
    e = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype]
    weights = 2 * (hd + 8) * 2.0 ** -23 * big + 2 * (n + 16) * 2.0 ** -23
    return e * ref.abs() + mag * (weights + (2.0 ** -8 if dtype == "bf16" else 0.0)) * (1 + e) + 1e-37


# ---- verification ------------------------------------------------------------------
def softmax(row, temperature):
    z = row.double() / f32(temperature)
    return torch.softmax(z, 0)


def accept(logits, draft, tokens, parents, u, temperature):
    """One sequence: logits [N][V], draft [N][V] or None, tokens [N], u [N].  New
    tokens, path, and the least distance of a decision to its border."""
    V, node, new, path, margin = logits.shape[1], 0, [], [0], 1.0
    if tokens[0] < 0:
        return [], [], 1.0
    while True:
        row = logits[node].double()
        if bool(torch.isnan(row).any()) or bool((row == math.inf).any()) or bool((row == -math.inf).all()):
            return new + [-1], path, margin
        w = softmax(logits[node], temperature)
        kids = [c for c in range(len(parents)) if parents[c] == node and 0 <= tokens[c] < V]
        q = None
        if draft is not None and kids:
            q = softmax(draft[node], temperature)
            if bool(torch.isnan(q).any()):
                return new + [-1], path, margin
        left, taken = 1.0, None
        for c in kids:
            p = float(w[tokens[c]])
            t = u[c] * (left if q is None else float(q[tokens[c]]))
            margin = min(margin, abs(p - t))
            if t < p:
                taken = c
                break
            if q is None:
                left -= p
                w = w.clone()
                w[tokens[c]] = 0.0
            else:
                w = (w - q).clamp(min=0)
        if taken is None:
            run = torch.cumsum(w, 0)
            t = run[-1] * u[0]
            v = int((run <= t).sum())
            margin = min(margin, float((run - t).abs().min()))
            return new + [v], path, margin
        new.append(int(tokens[taken]))
        node = taken
        path.append(node)
