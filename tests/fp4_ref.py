"""The 4-bit format in float64, from its definition, and plain forms of the
4-bit operators for tests: no code of the library's."""
import math

import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def held(x):
    """The values 4 bits hold of x, groups of 32 along the last axis (float64)."""
    v = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = v.abs().amax(-1, keepdim=True)
    mant, ex = torch.frexp(torch.where(torch.isfinite(top), top, torch.ones_like(top)))
    ex = (ex - 3 + (mant > 0.875).to(ex.dtype)).clamp(-126, 125)
    ex = torch.where(top == 0, torch.full_like(ex, -126), ex)
    unit = torch.ldexp(torch.ones_like(top), ex)
    r = v.abs() / unit
    step = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0)).double()
    r = (torch.round(r / step) * step).clamp(max=6.0)
    out = torch.sign(v) * r * unit
    return torch.where(torch.isfinite(top), out, torch.full_like(out, math.nan)).reshape(x.shape)


def encode(x):
    """Code bytes (even element in the low half) and scale bytes of x, bit for bit."""
    v = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = v.abs().amax(-1, keepdim=True)
    fin = torch.isfinite(top)
    mant, ex = torch.frexp(torch.where(fin, top, torch.ones_like(top)))
    s = (ex - 3 + (mant > 0.875).to(ex.dtype)).clamp(-126, 125) + 127
    s = torch.where(top == 0, torch.ones_like(s), s)
    h = held(x).reshape(v.shape)
    r = h.abs() / torch.ldexp(torch.ones_like(top), s - 127)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
    code = (r.unsqueeze(-1) == grid).int().argmax(-1) + 8 * torch.signbit(v).int()
    code = torch.where(fin, code, torch.zeros_like(code)).flatten(-2).to(torch.uint8)
    s = torch.where(fin, s, torch.full_like(s, 255)).squeeze(-1).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), s


class Cache:
    """A 4-bit paged cache filled on the host: kv [positions] per sequence in a
    shuffled page order, every other byte 0xFF."""

    def __init__(self, lens, extra, heads, hd, page, dtype, seed, gap=1):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.hd, self.page = heads, hd, page
        per = -(-(max(lens) + extra) // page) + gap
        self.n_pages = per * len(lens) + 1
        order = torch.randperm(self.n_pages, generator=g)[: per * len(lens)]
        self.table = order.view(len(lens), per).to(torch.int32)
        self.kv = []  # [positions][2][heads][hd] as written
        codes = torch.full((self.n_pages, 2, heads, page, hd // 2), 0xFF, dtype=torch.uint8)
        scales = torch.full((self.n_pages, 2, heads, page, hd // 32), 0xFF, dtype=torch.uint8)
        for b, n in enumerate(lens):
            x = (torch.randn(max(n, 0) + extra, 2, heads, hd, generator=g)
                 * torch.exp(0.5 * torch.randn(hd, generator=g))).to(TYPES[dtype])
            self.kv.append(x)
            p = torch.arange(x.shape[0])
            pg, slot = self.table[b][p // page].long(), p % page
            codes[pg, :, :, slot], scales[pg, :, :, slot] = encode(x)
        self.pool = torch.cat((codes.flatten(), scales.flatten()))

    def to(self, device):
        self.pool, self.table = self.pool.to(device), self.table.to(device)
        return self

    def struct(self):
        from paper_2402_15758_amd import binding as B
        return B.chimera_kv4(self.pool.data_ptr(), self.pool.numel(), self.table.data_ptr(), self.table.shape[0],
                             self.table.shape[1], self.n_pages, self.page, self.heads, self.hd)


def paths(parents):
    out = []
    for u, p in enumerate(parents):
        out.append((out[p] if p >= 0 else []) + [u])
    return out


def attention(q, kv, lens, parents, scale, seen=None):
    """q [B][N][Hq][hd], kv per sequence [positions][2][H][hd] as written:
    (out, tolerance), float64.  seen(b, p): whether the cache has position p.

    Tolerance: the output's own rounding (half a step of its type, and the
    quotient's), and in float32 the scores' dot products (hd products and sums,
    an MFMA's internal sums counted at 2^-23), which move each weight by twice
    the largest score error; weights held to 16 bits or more (2^-16), and the
    sums over T keys; all relative to the largest |v|."""
    B, N, Hq, hd = q.shape
    out = torch.zeros(B, N, Hq, hd, dtype=torch.float64)
    tol = torch.zeros_like(out)
    eps = torch.finfo(q.dtype).eps / 2
    for b in range(B):
        if lens[b] < 0:
            continue
        h = held(kv[b])
        for u, path in enumerate(paths(parents)):
            keys = [p for p in list(range(lens[b])) + [lens[b] + w for w in path] if seen is None or seen(b, p)]
            if not keys:
                continue
            H = h.shape[2]
            k = h[keys, 0].repeat_interleave(Hq // H, 1).transpose(0, 1)  # [Hq][T][hd]
            v = h[keys, 1].repeat_interleave(Hq // H, 1).transpose(0, 1)
            qu = q[b, u].double()
            s = torch.einsum("hd,htd->ht", qu, k) * scale
            out[b, u] = torch.einsum("ht,htd->hd", torch.softmax(s, -1), v)
            ds = (hd + 8) * 2.0 ** -23 * abs(scale) * torch.einsum("hd,htd->ht", qu.abs(), k.abs()).amax(-1)
            rel = 2 * ds + 2.0 ** -16 + (len(keys) + 64) * 2.0 ** -23
            tol[b, u] = eps * 1.01 * out[b, u].abs() + 2 * (rel * v.abs().amax((1, 2)))[:, None]
    return out, tol


def tree(nodes, arity):
    """Breadth-first parents; arity 1 is a chain."""
    return np.array([-1] + [(i - 1) // arity for i in range(1, nodes)], dtype=np.int32)
