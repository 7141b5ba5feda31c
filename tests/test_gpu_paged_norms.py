"""Norms of the rows into the paged cache whose squares or whose sum with eps leave the
float's range, against float64."""
import pytest
import torch

import paged_ref as R
from paper_2402_15758_amd import binding as B
from test_gpu_paged import DT, HALF, cache_of, stream

pytestmark = pytest.mark.gpu


def norms(x, eps, held, seed=1):
    """x [rows][heads][hd] as queries and as keys, without a rotation, against float64."""
    rows, H, hd = x.shape
    dtype = "bf16" if x.dtype == torch.bfloat16 else "f32"
    g = torch.Generator().manual_seed(seed)
    gains = (1 + 0.3 * torch.randn(2, hd, generator=g)).cuda()
    qkv = torch.cat((x, x, torch.zeros_like(x)), 1).cuda().contiguous()
    table = torch.arange(-(-rows // 16)).int().view(1, -1).cuda()
    pool = torch.zeros(table.shape[1], 2, H, 16, hd, dtype=R.TYPES[held], device="cuda")
    out = torch.zeros(rows, H, hd, dtype=R.TYPES[held], device="cuda")
    seq, pos = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.arange(rows).int().cuda()
    p, es = qkv.data_ptr(), qkv.element_size()
    B.chimera_paged_append(cache_of(pool, table, held), DT[dtype], p, p + H * hd * es, p + 2 * H * hd * es, 3 * H * hd,
                           H, seq.data_ptr(), pos.data_ptr(), rows, None, None, gains[0].data_ptr(),
                           gains[1].data_ptr(), eps, out.data_ptr(), H * hd, stream())
    k = pool[:, 0].permute(0, 2, 1, 3).reshape(-1, H, hd)[:rows]
    for got, gain in ((out, gains[0]), (k, gains[1])):
        ref = R.norm(x, gain.cpu(), eps)
        # the sum of hd squares (half of it through the root), the mean, eps, root, quotient
        # and three products; two of them and the result may be subnormal: those are multiples
        # of 2^-149, and of 2^-133 as bf16, whose rounding is off by 2^-134 whatever the value
        small = 2.0 ** -145 + (2.0 ** -134 if held == "bf16" else 0.0)
        bound = HALF[held] * ref.abs() + ((hd + 4) / 2 + 7) * 2.0 ** -24 * ref.abs() * (1 + HALF[held]) + small
        err = (got.double().cpu() - ref).abs()
        assert bool((err <= bound).all()), (float(err.max()), int((~(err <= bound)).sum()))


def rows_of(hd, seed):
    return torch.randn(6, 3, hd, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype,held", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("hd", [64, 128])
def test_largest_rows(dtype, held, hd):
    """Every finite value: heads of nothing but 1e38 and 3e38, one such value among small
    ones, heads beside ordinary ones; and an eps of the mean's size."""
    x = rows_of(hd, hd)
    x[0] = 1e38 * torch.sign(x[0])
    x[1] = 3.38e38 * torch.sign(x[1])
    x[2] = (x[2] * 6e37).clamp(-3.3e38, 3.3e38)
    x[3, 0] *= 1e20
    x[3, 1, 5] = -3.3e38
    x[3, 2, hd - 1] = 2e38
    x[4] *= 2.0 ** 60 * torch.tensor([1.0, 2.0, 16.0])[:, None]  # on either side of the range
    x = x.to(R.TYPES[dtype])
    for eps in (1e-5, 1e30, 3e38):
        norms(x, eps, held)


@pytest.mark.parametrize("dtype,held", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("hd", [64, 128])
def test_smallest_rows(dtype, held, hd):
    """Squares and an eps below the least normal float, down to subnormal values; zeros."""
    x = rows_of(hd, hd + 1)
    x[0] *= 1e-20
    x[1] *= 1e-22
    x[2] *= 1e-30
    x[3] *= torch.tensor([2.0 ** -46, 2.0 ** -50, 2.0 ** -54])[:, None]  # on either side of where sums are scaled
    x[4] *= 1e-40
    x[5, 0] = 0.0
    x = x.to(R.TYPES[dtype])
    for eps in (1e-5, 1e-31, 1e-38, 1e-41, 2.0 ** -149):
        norms(x, eps, held)
