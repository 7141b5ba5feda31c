"""The 4-bit attention's weights: their precision, and scores at the ends of the
float's range."""
import pytest
import torch

import fp4_ref as R
from paper_2402_15758_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": B.CHIMERA_BF16, "f32": B.CHIMERA_F32}


def stream():
    return torch.cuda.current_stream().cuda_stream


class Filled:
    """A cache whose first positions hold k and v ([positions][H][hd], of one sequence)."""

    def __init__(self, k, v, page=16, table=0):
        T, H, hd = k.shape
        pages = -(-T // page)
        self.H, self.hd, self.page, self.pages = H, hd, page, pages
        ids = torch.arange(pages).flip(0).to(torch.int32)
        self.table = torch.cat((ids, torch.full((max(table - pages, 0),), -1, dtype=torch.int32))).view(1, -1).cuda()
        self.pool = torch.full((B.chimera_kv4_bytes(pages, page, H, hd),), 0xFF, dtype=torch.uint8, device="cuda")
        kd, vd = k.cuda().contiguous(), v.cuda().contiguous()
        seq = torch.zeros(T, dtype=torch.int32, device="cuda")
        pos = torch.arange(T, dtype=torch.int32, device="cuda")
        B.chimera_kv4_append(self.struct(), DT["bf16" if k.dtype == torch.bfloat16 else "f32"], kd.data_ptr(),
                             vd.data_ptr(), H * hd, seq.data_ptr(), pos.data_ptr(), T, stream())
        torch.cuda.synchronize()

    def struct(self):
        return B.chimera_kv4(self.pool.data_ptr(), self.pool.numel(), self.table.data_ptr(), 1, self.table.shape[1],
                             self.pages, self.page, self.H, self.hd)

    def attend(self, q, n, scale):
        """q [Hq][hd] of one token at position n."""
        Hq = q.shape[0]
        qd, out = q.cuda().contiguous(), torch.full_like(q, 55.0, device="cuda")
        nb = B.chimera_kv4_attn_bytes(self.struct(), Hq, 1)
        ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
        nd = torch.tensor([n], dtype=torch.int32, device="cuda")
        B.chimera_kv4_attn(self.struct(), DT["bf16" if q.dtype == torch.bfloat16 else "f32"], qd.data_ptr(),
                           Hq * self.hd, nd.data_ptr(), Hq, None, 1, scale, out.data_ptr(), Hq * self.hd, ws.data_ptr(),
                           nb, stream())
        return out.cpu()


# one launch; groups; supers (16 blocks of queries a sequence: from 16 supers on)
@pytest.mark.parametrize("n,first,table", [(40, 0, 0), (200, 100, 40), (1300, 700, 0), (17000, 9000, 0)])
@pytest.mark.parametrize("hd", [64, 128])
def test_weights_keep_all_bits_of_a_float(hd, n, first, table):
    """out = (p_b - p_c) / (1 + p_b + p_c), p_b and p_c 2^-13 apart: what either loses
    shows whole.

    Tolerance: the scores are exact; their product with scale log2(e) takes two
    roundings of a number below 1 and the exponential one of 2^-23, so each weight
    (below 0.8) is within 1.3 2^-23; six sums of three terms a weight, each of at most
    0.8, add 4.7 2^-23; over a denominator above 2.2 that is below 4 2^-23.  Then the
    output's rounding.  Weights of 16 bits miss it: up to 2^-18 each."""
    H, Hq = 1, 256
    g = torch.Generator().manual_seed(n)
    k, v = torch.zeros(n + 1, H, hd), torch.zeros(n + 1, H, hd)
    k[:, :, 32] = -6.0  # everything else: a score of -768, a weight of 0
    for i, p in enumerate((first, first + 1, first + 2)):
        k[p] = 0
        k[p, :, 1] = float(i > 0)
        k[p, :, 2] = float(i > 1)
        v[p] = (0.0, 1.0, -1.0)[i]
    q = torch.zeros(Hq, hd)
    q[:, 1] = -0.25 - 0.25 * torch.rand(Hq, generator=g)
    q[:, 2] = -(1 + torch.rand(Hq, generator=g)) * 2.0 ** -13
    q[:, 32] = 128.0
    q = q.bfloat16()
    out = Filled(k.bfloat16(), v.bfloat16(), table=table).attend(q, n, 1.0).double()
    b, c = torch.exp(q[:, 1].double()), torch.exp(q[:, 1].double() + q[:, 2].double())
    want = ((b - c) / (1 + b + c)).unsqueeze(1)
    tol = torch.finfo(torch.bfloat16).eps / 2 * want.abs() + 4 * 2.0 ** -23
    assert bool(((out - want).abs() <= tol).all()), float(((out - want).abs() / tol).max())


def rows(n, low, high, dtype, seed):
    """Keys whose score with queries() passes the float's range downwards (low)
    or upwards (high), positions of them; the others have ordinary scores."""
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(n + 1, 1, 64, generator=g) for _ in range(2))
    k[:, :, :32] = 0
    k[low, :, 0], k[high, :, 0] = -6.0, 6.0
    return k.to(dtype), v.to(dtype)


def queries(first, dtype, seed):
    q = torch.randn(8, 64, generator=torch.Generator().manual_seed(seed)) * 0.7
    q[:, 0] = first
    return q.to(dtype)


def without(q, k, v, n, gone, scale):
    """The formula over the keys that are not `gone` (fp4_ref's form and tolerance)."""
    kv = torch.stack((k, v), 1)
    k0 = kv.clone()
    k0[:, 0, :, 0] = 0  # the others' share of the first dimension: nothing
    q0 = q.clone()
    q0[:, 0] = 0
    gone = set(gone)
    want, tol = R.attention(q0.view(1, 1, *q.shape), [k0], [n], [-1], scale, seen=lambda b, p: p not in gone)
    return want[0, 0], tol[0, 0]


# tokens, table, copies of the eight queries: one launch, groups, supers
SIZES = [(200, 0, 1), (700, 0, 1), (1500, 200, 1), (18750, 0, 32)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,table,copies", SIZES)
@pytest.mark.parametrize("first,scale", [(2.0 ** 127, 0.125), (2.0 ** 60, 2.0 ** 80), (-(2.0 ** 127), -0.125)])
def test_scores_of_minus_infinity_weigh_nothing(dtype, n, table, copies, first, scale):
    """A key, a chunk, several of them, a stretch up to the window and some of the
    window's keys, whose score (or scaled score) is below the float's range."""
    q = queries(first, dtype, 1)
    if scale > 1:  # the others' scaled scores stay ordinary
        q[:, 1:] = (q[:, 1:].float() * 2.0 ** -80).to(dtype)
    for stretch in ([7], range(64), range(64, 128), range(192), range(0, n - 15), range(n - 5, n - 2), range(3, n)):
        low = list(stretch)
        k, v = rows(n, low, [], dtype, n)
        if scale < 0:
            k[:, :, 0] = -k[:, :, 0].abs()  # q < 0 and scale < 0: the same scores
        want, tol = without(q, k, v, n, low, scale)
        out = Filled(k, v, table=table).attend(q.repeat(copies, 1), n, scale).double().view(copies, 8, 64)
        assert bool(((out - want).abs() <= tol + 1e-30).all()), (low[0], len(low))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,table,copies", SIZES)
@pytest.mark.parametrize("first,scale", [(2.0 ** 127, 0.125), (2.0 ** 60, 2.0 ** 80)])
def test_scores_past_the_range_are_never_dropped_in_silence(dtype, n, table, copies, first, scale):
    """A positive one, or nothing but negative ones: NaN."""
    q = queries(first, dtype, 2)
    for low, high in (([], [5]), ([], range(64)), (range(64), [70]), ([], [n - 3]), (range(n + 1), []),
                      (range(n - 20), range(n - 20, n + 1)), (range(200), range(100, 101))):
        k, v = rows(n, list(low), list(high), dtype, n)
        out = Filled(k, v, table=table).attend(q.repeat(copies, 1), n, scale)
        assert bool(torch.isnan(out).all()), (len(low), len(high))
