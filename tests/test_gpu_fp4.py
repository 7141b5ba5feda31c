"""The 4-bit operators on the GPU against float64 references (fp4_ref), at the
sizes, types, strides and masks where they can go wrong."""
import math

import numpy as np
import pytest
import torch

import fp4_ref as R
from paper_2402_15758_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": B.CHIMERA_BF16, "f32": B.CHIMERA_F32}


def stream():
    return torch.cuda.current_stream().cuda_stream


# ---- weights ---------------------------------------------------------------------
def pack(w, dtype, ldw=None):
    K, N = w.shape
    nb = B.chimera_fp4_bytes(N, K)
    p = torch.full((nb,), 0xAB, dtype=torch.uint8, device="cuda")
    B.chimera_fp4_pack(DT[dtype], w.data_ptr(), w.stride(0), N, K, p.data_ptr(), nb, stream())
    return p


def unpack(p, N, K, dtype):
    w = torch.empty(K, N, dtype=R.TYPES[dtype], device="cuda")
    B.chimera_fp4_unpack(DT[dtype], p.data_ptr(), N, K, w.data_ptr(), N, stream())
    return w


def weights(K, N, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(K, N, generator=g) * torch.exp(torch.randn(K // 32, 1, generator=g)).repeat_interleave(32, 0)
            * 0.05).to(R.TYPES[dtype])


def held_w(w):
    return R.held(w.t().contiguous()).t()


def same(a, b):
    """Equal values, NaN with NaN."""
    a, b = a.double().cpu(), b.double()
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,N", [(32, 16), (96, 48), (544, 64), (1088, 256), (4096, 80), (160, 8208)])
def test_pack_holds_the_format(dtype, K, N):
    w = weights(K, N, dtype, K + N)
    w[: K // 2, 3] = 0
    w[0, 1], w[31, 2], w[5, 7] = math.inf, math.nan, -math.inf
    w[-1, 5], w[-2, 5] = 3e38, 1e-39
    w[-32:, 6] = 1e-40
    assert same(unpack(pack(w.cuda(), dtype), N, K, dtype), held_w(w))


def test_pack_reads_strided_unaligned_columns():
    w = weights(64, 100, "bf16", 5).cuda()
    part = w[:, 33:33 + 48]
    assert same(unpack(pack(part, "bf16"), 48, 64, "bf16"), held_w(part.cpu()))
    out = torch.full((64, 61), 7.0, dtype=torch.float32, device="cuda")
    B.chimera_fp4_unpack(B.CHIMERA_F32, pack(part, "bf16").data_ptr(), 48, 64, out[:, 5:].data_ptr(), 61, stream())
    assert same(out[:, 5:53], held_w(part.cpu())) and (out[:, :5] == 7).all() and (out[:, 53:] == 7).all()


def product(x, p, N, dtype, ldy=None, ws=None):
    M, K = x.shape
    y = torch.full((M, ldy or N), 123.0, device="cuda")
    nb = B.chimera_gemm_fp4_bytes(DT[dtype], M, N, K)
    if ws is None:
        ws = torch.full((nb + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    B.chimera_gemm_fp4(DT[dtype], x.data_ptr(), x.stride(0), p.data_ptr(), M, N, K, y.data_ptr(), y.stride(0),
                       ws.data_ptr(), nb, stream())
    return y


def check_product(x, w, y):
    """|error| within K + 16 float32 roundings (an MFMA's inner sums counted at
    2^-23) of the sum of magnitudes."""
    h = held_w(w)
    ref = x.double() @ h
    bound = (x.shape[1] + 16) * 2.0 ** -23 * (x.double().abs() @ h.abs())
    err = (y.double().cpu() - ref).abs()
    assert bool((err <= bound).all()), float((err / bound.clamp(min=1e-300)).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(1, 16, 32), (1, 1024, 256), (1, 4096, 4096), (2, 48, 96), (5, 80, 544),
                                   (16, 512, 1088), (17, 64, 64), (33, 208, 2080), (64, 768, 256), (65, 4096, 512),
                                   (129, 320, 1024), (300, 1040, 288), (130, 8256, 160),
                                   # up to 16 rows: whole rows in LDS or a slice of them, one workgroup a column
                                   # block or not, and rows too long for it
                                   (1, 64, 8192), (7, 80, 2048), (16, 320, 4096), (13, 8256, 2048), (16, 8256, 4128)])
def test_product(dtype, M, N, K):
    g = torch.Generator().manual_seed(M * 7 + N + K)
    x = (torch.randn(M, K, generator=g) * torch.exp(torch.randn(K, generator=g))).to(R.TYPES[dtype])
    w = weights(K, N, dtype, M)
    check_product(x, w, product(x.cuda(), pack(w.cuda(), dtype), N, dtype))


def test_largest_row_count():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(4096, 64, generator=g).bfloat16()
    for N in (64, 48):  # the bf16 kernels' route, and its own
        w = weights(64, N, "bf16", N)
        check_product(x, w, product(x.cuda(), pack(w.cuda(), "bf16"), N, "bf16"))


@pytest.mark.parametrize("dtype,N,K", [("bf16", 1024, 2048), ("bf16", 8192, 512), ("bf16", 48, 1088),
                                       ("f32", 512, 1024)])
def test_a_row_does_not_depend_on_the_others(dtype, N, K):
    g = torch.Generator().manual_seed(N)
    x = torch.randn(300, K, generator=g).to(R.TYPES[dtype]).cuda()
    p = pack(weights(K, N, dtype, K).cuda(), dtype)
    alone = torch.cat([product(x[r:r + 1], p, N, dtype) for r in (0, 15, 16, 63, 100, 299)])
    for M in (16, 17, 64, 65, 128, 129, 300):
        y = product(x[:M], p, N, dtype)
        for i, r in enumerate((0, 15, 16, 63, 100, 299)):
            if r < M:
                assert torch.equal(y[r], alone[i]), (M, r)


@pytest.mark.parametrize("M,N,K", [(1, 1024, 2048), (9, 4096, 512), (64, 256, 4096), (200, 1024, 1024)])
def test_bits_of_the_bf16_product_of_the_unpacked_matrix(M, N, K):
    g = torch.Generator().manual_seed(N + M)
    x = torch.randn(M, K, generator=g).bfloat16().cuda()
    p = pack(weights(K, N, "bf16", 3).cuda(), "bf16")
    w = unpack(p, N, K, "bf16")
    ref = torch.empty(M, N, device="cuda")
    B.chimera_gemm_static(B.CHIMERA_BF16, x.data_ptr(), w.data_ptr(), M, N, K, ref.data_ptr(), stream())
    assert torch.equal(product(x, p, N, "bf16"), ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 3, 40, 150])
def test_product_strides_and_alignment(dtype, M):
    N, K = 192, 96
    g = torch.Generator().manual_seed(M)
    big = torch.randn(M, K + 13, generator=g).to(R.TYPES[dtype]).cuda()
    w = weights(K, N, dtype, 9)
    p = pack(w.cuda(), dtype)
    want = product(big[:, 3:3 + K].contiguous(), p, N, dtype)
    y = product(big[:, 3:3 + K], p, N, dtype, ldy=N + 5)  # rows at odd elements
    assert torch.equal(y[:, :N], want) and (y[:, N:] == 123).all()


def test_product_of_special_values():
    x = torch.zeros(3, 64)
    x[0, 0], x[1, 40], x[2] = math.inf, math.nan, 1.0
    w = weights(64, 32, "bf16", 1)
    w[0, 4] = math.inf  # column 4: all its first group is NaN
    y = product(x.bfloat16().cuda(), pack(w.cuda(), "bf16"), 32, "bf16").cpu()
    h = held_w(w)
    assert torch.isnan(y[1]).all() and torch.isnan(y[:, 4]).all()
    for n in range(32):
        if n != 4:
            assert y[0, n] == math.copysign(math.inf, h[0, n]) if h[0, n] != 0 else torch.isnan(y[0, n])
            assert abs(y[2, n] - h[:, n].sum()) <= 80 * 2.0 ** -23 * h[:, n].abs().sum()


# ---- the cache -------------------------------------------------------------------
@pytest.mark.parametrize("dtype,heads,hd,page", [("bf16", 4, 128, 16), ("f32", 3, 64, 1), ("bf16", 1, 64, 256),
                                                 ("f32", 8, 128, 7)])
def test_append_writes_the_rows_and_nothing_else(dtype, heads, hd, page):
    g = torch.Generator().manual_seed(heads)
    lens = [40, 0, 23]
    c = R.Cache(lens, 0, heads, hd, page, dtype, 11)
    D = heads * hd
    rows = 37
    qkv = (torch.randn(rows, 3 * D + 1, generator=g) * torch.exp(torch.randn(3 * D + 1, generator=g))
           ).to(R.TYPES[dtype])
    qkv[4, D + 5], qkv[5, 2 * D + 9], qkv[6] = math.inf, math.nan, 0
    seq = torch.tensor([0, 2] * 18 + [0], dtype=torch.int32)
    pos = torch.arange(rows, dtype=torch.int32)
    cap = c.table.shape[1] * page
    seq[7], seq[8], pos[9], pos[10] = -1, 3, -1, cap      # rows the cache does not have
    c.table[2, min(21, cap - 1) // page] = c.n_pages if page < 256 else c.table[2, 0]
    bad_page = [r for r in range(rows) if int(seq[r]) == 2 and 0 <= int(pos[r]) < cap
                and not 0 <= int(c.table[2, int(pos[r]) // page]) < c.n_pages]
    want = c.pool.clone()
    cut = c.n_pages * 2 * heads * page * hd // 2
    codes = want[:cut].view(c.n_pages, 2, heads, page, hd // 2)
    scales = want[cut:].view(c.n_pages, 2, heads, page, hd // 32)
    skip = {7, 8, 9, 10} | set(bad_page)
    kv = qkv[:, D:3 * D].reshape(rows, 2, heads, hd)
    code, s = R.encode(kv)
    for r in range(rows):
        if r not in skip:
            pg, slot = int(c.table[seq[r], pos[r] // page]), int(pos[r]) % page
            codes[pg, :, :, slot], scales[pg, :, :, slot] = code[r], s[r]
    c.to("cuda")
    x, sd, pd = qkv.cuda(), seq.cuda(), pos.cuda()
    es = x.element_size()
    B.chimera_kv4_append(c.struct(), DT[dtype], x.data_ptr() + D * es, x.data_ptr() + 2 * D * es, 3 * D + 1,
                         sd.data_ptr(), pd.data_ptr(), rows, stream())
    assert torch.equal(c.pool.cpu(), want)
    out = torch.full((2, rows, D + 3), 9.0, dtype=R.TYPES[dtype], device="cuda")
    B.chimera_kv4_read(c.struct(), DT[dtype], sd.data_ptr(), pd.data_ptr(), rows, out[0].data_ptr(), out[1].data_ptr(),
                       D + 3, stream())
    h = R.held(kv)
    for r in range(rows):
        for t in range(2):
            got = out[t, r, :D].view(heads, hd)
            assert (got == 9).all() if r in skip else same(got, h[r, t]), r
    assert (out[:, :, D:] == 9).all()
    B.chimera_kv4_append(c.struct(), DT[dtype], x.data_ptr(), x.data_ptr(), 3 * D, sd.data_ptr(), pd.data_ptr(), 0,
                         stream())
    assert torch.equal(c.pool.cpu(), want)


def attend(c, q, lens, parents, scale, ldo=None, ldq=None, out=None, ws=None):
    Bn, N, Hq, hd = q.shape
    dtype = "bf16" if q.dtype == torch.bfloat16 else "f32"
    qq = torch.zeros(Bn * N, ldq or Hq * hd, dtype=q.dtype, device="cuda")
    qq[:, :Hq * hd] = q.reshape(Bn * N, -1)
    if out is None:
        out = torch.full((Bn * N, ldo or Hq * hd), 55.0, dtype=q.dtype, device="cuda")
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    nb = B.chimera_kv4_attn_bytes(c.struct(), Hq, N)
    if ws is None:
        ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
    B.chimera_kv4_attn(c.struct(), DT[dtype], qq.data_ptr(), qq.shape[1], n.data_ptr(), Hq, parents, N, scale,
                       out.data_ptr(), out.shape[1], ws.data_ptr(), nb, stream())
    return out


def queries(Bn, N, Hq, hd, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(Bn, N, Hq, hd, generator=g) * 1.3).to(R.TYPES[dtype])


def check_attention(out, want, tol):
    got = out.double().cpu().reshape(want.shape)
    err = (got - want).abs()
    assert bool((err <= tol + 1e-30).all()), float((err / tol.clamp(min=1e-30)).max())


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("nodes,arity", [(1, 1), (7, 1), (16, 1), (8, 3), (17, 2), (32, 4), (64, 4)])
def test_attention_over_ragged_lengths(dtype, hd, nodes, arity):
    """Lengths on both sides of every boundary of the reduction, an empty place
    in the batch, and no committed token at all."""
    lens = [0, 1, 15, 16, 17, 63, 64, -1, 79, 80, 81, 255, 272, 300]
    c = R.Cache(lens, nodes, 2, hd, 16, dtype, nodes + hd).to("cuda")
    q = queries(len(lens), nodes, 2, hd, dtype, nodes)
    parents = R.tree(nodes, arity)
    want, tol = R.attention(q, c.kv, lens, parents, hd ** -0.5)
    out = attend(c, q.cuda(), lens, parents, hd ** -0.5)
    check_attention(out, want, tol)
    assert (out.view(len(lens), -1)[7] == 0).all()


@pytest.mark.parametrize("dtype,Hq,H,hd,page,nodes,arity,lens", [
    ("bf16", 8, 1, 128, 1, 1, 1, [515, 3]),
    ("bf16", 8, 2, 64, 256, 8, 3, [777]),
    ("f32", 12, 4, 64, 5, 3, 1, [200, 31, 64]),
    ("bf16", 16, 1, 128, 16, 64, 4, [130]),       # 1024 query rows a cache head
    ("bf16", 4, 4, 128, 64, 32, 4, [4095, 4112]),
    ("bf16", 2, 1, 64, 16, 1, 1, [4096, 5200, 9000]),
    ("f32", 1, 1, 128, 16, 16, 1, [4200]),
])
def test_attention_heads_pages_and_long_contexts(dtype, Hq, H, hd, page, nodes, arity, lens):
    c = R.Cache(lens, nodes, H, hd, page, dtype, Hq + page).to("cuda")
    q = queries(len(lens), nodes, Hq, hd, dtype, 4)
    parents = R.tree(nodes, arity)
    want, tol = R.attention(q, c.kv, lens, parents, 0.11)
    out = attend(c, q.cuda(), lens, parents, 0.11, ldq=Hq * hd + 16, ldo=Hq * hd + 3)
    check_attention(out[:, :Hq * hd], want, tol)
    assert (out[:, Hq * hd:] == 55).all()


def test_attention_without_a_tree_is_a_chain():
    lens = [33, 70]
    c = R.Cache(lens, 9, 2, 64, 16, "bf16", 2).to("cuda")
    q = queries(2, 9, 2, 64, "bf16", 8).cuda()
    assert torch.equal(attend(c, q, lens, None, 0.125), attend(c, q, lens, R.tree(9, 1), 0.125))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_query_does_not_depend_on_its_company(dtype):
    """Node u of a tree, alone in its place on its path, has the same bits."""
    lens, H, hd = [100, 700, 4500], 2, 128
    parents = R.tree(40, 3)
    c = R.Cache(lens, 40, H, hd, 16, dtype, 21).to("cuda")
    q = queries(3, 40, H, hd, dtype, 5).cuda()
    whole = attend(c, q, lens, parents, 0.09).view(3, 40, H * hd)
    path = R.paths(parents)[39]
    for u in (39, 5, 0):
        path = R.paths(parents)[u]
        # the path's rows as a committed stretch: copied behind the context
        d = R.Cache(lens, 40, H, hd, 16, dtype, 21).to("cuda")
        for b, n in enumerate(lens):
            src = torch.tensor([n + w for w in path], dtype=torch.int32, device="cuda")
            seq = torch.full_like(src, b)
            k = torch.empty(len(path), H * hd, dtype=R.TYPES[dtype], device="cuda")
            v = torch.empty_like(k)
            B.chimera_kv4_read(c.struct(), DT[dtype], seq.data_ptr(), src.data_ptr(), len(path), k.data_ptr(),
                               v.data_ptr(), H * hd, stream())
            dst = n + torch.arange(len(path), dtype=torch.int32, device="cuda")
            B.chimera_kv4_append(d.struct(), DT[dtype], k.data_ptr(), v.data_ptr(), H * hd, seq.data_ptr(),
                                 dst.data_ptr(), len(path), stream())
        one = attend(d, q[:, u:u + 1].contiguous(), [n + len(path) - 1 for n in lens], None, 0.09)
        assert torch.equal(one.view(3, H * hd), whole[:, u]), u


@pytest.mark.parametrize("dtype,hd,n", [("bf16", 128, 40), ("bf16", 128, 200), ("f32", 64, 130), ("bf16", 64, 2500)])
def test_bits_do_not_depend_on_the_table_or_the_batch(dtype, hd, n):
    """The work is dealt by its amount and by the table's length (one launch, groups,
    supers): a short and a long table, one sequence and a batch of 300 of it."""
    H, page, nodes = 2, 16, 3
    parents = R.tree(nodes, 2)
    c = R.Cache([n], nodes, H, hd, page, dtype, 41, gap=0).to("cuda")
    q = queries(1, nodes, 2 * H, hd, dtype, 13).cuda()
    want = attend(c, q, [n], parents, 0.1)
    short = c.table
    c.table = torch.cat((short, torch.full((1, 1000), -1, dtype=torch.int32, device="cuda")), 1)
    assert torch.equal(attend(c, q, [n], parents, 0.1), want)
    for table in (short, c.table):
        c.table = table.repeat(300, 1)
        lens = [n] * 300
        lens[7] = -1
        out = attend(c, q.repeat(300, 1, 1, 1), lens, parents, 0.1).view(300, -1)
        keep = torch.arange(300, device="cuda") != 7
        assert bool((out[keep] == want.view(1, -1)).all()) and bool((out[7] == 0).all())


def test_attention_ignores_what_it_does_not_see():
    """Bad pages, positions past the table, and NaN in rows of other branches and
    behind the sequence."""
    lens, H, hd, page = [150, 90], 2, 64, 16
    parents = np.array([-1, 0, 0, 1], dtype=np.int32)
    c = R.Cache(lens, 4, H, hd, page, "bf16", 31, gap=0)
    c.kv[0][152] = math.nan  # node 2 of sequence 0: seen by node 2 alone
    pg, slot = int(c.table[0, 152 // page]), 152 % page
    cut = c.n_pages * 2 * H * page * hd // 2
    scales = c.pool[cut:].view(c.n_pages, 2, H, page, hd // 32)
    scales[pg, :, :, slot] = 255
    c.table[0, 2] = -1
    c.table[0, 5] = c.n_pages
    c.table[1, 0] = 1 << 30
    bad = {(0, p) for p in list(range(32, 48)) + list(range(80, 96))} | {(1, p) for p in range(16)}
    q = queries(2, 4, H, hd, "bf16", 6)
    want, tol = R.attention(q, c.kv, lens, parents, 0.125, seen=lambda b, p: (b, p) not in bad)
    out = attend(c.to("cuda"), q.cuda(), lens, parents, 0.125).double().cpu().view(2, 4, H, hd)
    assert torch.isnan(out[0, 2]).all()
    keep = torch.ones(2, 4, dtype=torch.bool)
    keep[0, 2] = False
    assert bool(((out - want).abs() <= tol)[keep].all())
    c.table.fill_(-1)
    assert bool((attend(c, q.cuda(), lens, parents, 0.125) == 0).all())


def test_attention_past_the_end_of_the_table():
    """A table that ends inside the new tokens: those past it are not seen; one
    that ends before them: they see what is committed; lengths beyond it."""
    H, hd, page, N = 2, 64, 16, 4
    parents = np.array([-1, 0, 0, 1], dtype=np.int32)
    c = R.Cache([60, 60, 60], N, H, hd, page, "bf16", 12, gap=0).to("cuda")  # 64 positions, all written
    q = queries(3, N, H, hd, "bf16", 16)
    lens = [62, 64, 2 ** 31 - 1]
    want, tol = R.attention(q, c.kv, [62, 64, 64], parents, 0.125, seen=lambda b, p: p < 64)
    check_attention(attend(c, q.cuda(), lens, parents, 0.125), want, tol)


def test_extreme_scores():
    lens, H, hd = [200], 1, 64
    c = R.Cache(lens, 1, H, hd, 16, "f32", 3).to("cuda")
    q = queries(1, 1, H, hd, "f32", 7)
    for scale in (0.0, -0.5, 40.0):
        want, tol = R.attention(q, c.kv, lens, np.array([-1], dtype=np.int32), scale)
        check_attention(attend(c, q.cuda(), lens, None, scale), want, tol)
    q[0, 0, 0, 0] = math.inf
    assert torch.isnan(attend(c, q.cuda(), lens, None, 1.0)).all()


# ---- sizes past 31 and 32 bits, the widest staging, the smallest numbers -------------
@pytest.mark.parametrize("dtype,M,N,K", [("bf16", 14, 320, 4096), ("f32", 7, 336, 4096), ("bf16", 4, 64, 14336)])
def test_product_of_the_longest_staged_rows(dtype, M, N, K):
    """112 KiB of rows in LDS, next to the workgroup's sums."""
    g = torch.Generator().manual_seed(M)
    x = torch.randn(M, K, generator=g).to(R.TYPES[dtype])
    w = weights(K, N, dtype, M + 1)
    check_product(x, w, product(x.cuda(), pack(w.cuda(), dtype), N, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 40])
def test_product_of_the_smallest_weights(dtype, M):
    """Groups at the smallest scale, whose smallest values are subnormal."""
    g = torch.Generator().manual_seed(M)
    x = (torch.randn(M, 64, generator=g) * 2.0 ** 100).to(R.TYPES[dtype])
    w = (torch.randint(-7, 8, (64, 16), generator=g).float() * 2.0 ** -127).to(R.TYPES[dtype])
    check_product(x, w, product(x.cuda(), pack(w.cuda(), dtype), 16, dtype))


def test_product_with_a_matrix_past_32_bits():
    """131072 x 40000: over 2^32 values, 2.8 GB packed; first and last columns."""
    N, K = 40000, 131072
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(K, N, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    x = torch.randn(600, K, generator=g, device="cuda").bfloat16()
    p = pack(w, "bf16")
    cols = [w[:, :16].cpu(), w[:, -16:].cpu()]
    del w
    for M in (1, 40, 600):
        y = product(x[:M], p, N, "bf16")
        check_product(x[:M].cpu(), cols[0], y[:, :16])
        check_product(x[:M].cpu(), cols[1], y[:, -16:])
    u = unpack(p, N, K, "bf16")
    assert same(u[:, -16:], held_w(cols[1]))
    del u, p, x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_pool_past_32_bits(dtype):
    """A cache of 140000 pages, over 2^31 groups of values (39 GB): rows in its
    first and its last pages."""
    lens, nodes, H, hd, page = [700, 90], 4, 8, 128, 256
    n_pages = 140000
    parents = R.tree(nodes, 2)
    assert n_pages * 2 * H * page * hd // 32 > 2 ** 31
    nb = B.chimera_kv4_bytes(n_pages, page, H, hd)
    pool = torch.empty(nb, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2], [n_pages // 2, n_pages - 3, -1]], dtype=torch.int32,
                         device="cuda")
    c = R.Cache(lens, nodes, H, hd, page, dtype, 3)
    kv = c.kv
    c.pool, c.table, c.n_pages = pool, table, n_pages
    for b in range(2):
        x = kv[b].cuda()
        rows, D = x.shape[0], H * hd
        seq = torch.full((rows,), b, dtype=torch.int32, device="cuda")
        pos = torch.arange(rows, dtype=torch.int32, device="cuda")
        B.chimera_kv4_append(c.struct(), DT[dtype], x.data_ptr(), x[:, 1].data_ptr(), 2 * D, seq.data_ptr(),
                             pos.data_ptr(), rows, stream())
        out = torch.empty_like(x)
        B.chimera_kv4_read(c.struct(), DT[dtype], seq.data_ptr(), pos.data_ptr(), rows, out.data_ptr(),
                           out[:, 1].data_ptr(), 2 * D, stream())
        assert same(out, R.held(kv[b]))
    q = queries(2, nodes, 2 * H, hd, dtype, 6)
    want, tol = R.attention(q, kv, lens, parents, 0.1)
    check_attention(attend(c, q.cuda(), lens, parents, 0.1), want, tol)
    del pool
    c.pool = None
    torch.cuda.empty_cache()


@pytest.mark.parametrize("H,n", [(8, 34000), (1, 34000)])
def test_more_partials_than_a_wave_holds(H, n):
    """33 supers of a query, and 133 groups, the last of either cut short; a stretch
    of unknown pages in the middle."""
    hd, page = 64, 64
    kv = (torch.randn(n + 1, 2, H, hd, generator=torch.Generator().manual_seed(H)) * 0.7).bfloat16()
    pages = n // page + 1
    c = R.Cache([1], 1, H, hd, page, "bf16", 1)
    c.n_pages = pages
    c.table = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).to(torch.int32).view(1, -1).cuda()
    c.pool = torch.zeros(B.chimera_kv4_bytes(pages, page, H, hd), dtype=torch.uint8, device="cuda")
    x = kv.cuda()
    seq = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    pos = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    B.chimera_kv4_append(c.struct(), 1, x.data_ptr(), x[:, 1].data_ptr(), 2 * H * hd, seq.data_ptr(), pos.data_ptr(),
                         n + 1, stream())
    q = queries(1, 1, 2 * H, hd, "bf16", 3)
    for lost in (False, True):
        if lost:
            c.table[0, 40:200] = -1  # positions 2560 .. 12799: whole supers and groups
        want, tol = R.attention(q, [kv], [n], [-1], 0.2, seen=lambda b, p: not lost or not 2560 <= p < 12800)
        check_attention(attend(c, q.cuda(), [n], None, 0.2), want, tol)


def test_many_rows_and_many_sequences():
    """More rows than a grid's second dimension holds, and a batch at its limit."""
    H, hd, page, B_ = 1, 64, 4, 65535
    table = torch.arange(B_, dtype=torch.int32, device="cuda").view(B_, 1)
    nb = B.chimera_kv4_bytes(B_, page, H, hd)
    c = R.Cache([1], 1, H, hd, page, "bf16", 1)
    c.pool, c.table, c.n_pages = torch.zeros(nb, dtype=torch.uint8, device="cuda"), table, B_
    rows = 2 * B_
    x = torch.randn(rows, hd, generator=torch.Generator().manual_seed(5)).bfloat16()
    seq = torch.arange(rows, dtype=torch.int32, device="cuda") % B_
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") // B_
    xd = x.cuda()
    B.chimera_kv4_append(c.struct(), 1, xd.data_ptr(), xd.data_ptr(), hd, seq.data_ptr(), pos.data_ptr(), rows,
                         stream())
    out = torch.empty(2, rows, hd, dtype=torch.bfloat16, device="cuda")
    B.chimera_kv4_read(c.struct(), 1, seq.data_ptr(), pos.data_ptr(), rows, out[0].data_ptr(), out[1].data_ptr(), hd,
                       stream())
    h = R.held(x)
    assert same(out[0], h) and same(out[1], h)
    # one committed token and the new one; the two rows' weights by hand
    q = queries(B_, 1, 1, hd, "bf16", 2)
    got = attend(c, q.cuda(), [1] * B_, None, 0.125).double().cpu()
    k = h.view(2, B_, hd)
    s = torch.stack([(q.view(B_, hd).double() * k[i]).sum(-1) * 0.125 for i in range(2)])
    want = (torch.softmax(s, 0).unsqueeze(-1) * k).sum(0)
    ds = (hd + 8) * 2.0 ** -23 * 0.125 * (q.view(B_, hd).double().abs() * k.abs().amax(0)).sum(-1, keepdim=True)
    top = k.abs().amax((0, 2)).unsqueeze(-1)
    assert bool(((got - want).abs() <= 2.0 ** -8 * 1.01 * want.abs() + 2 * (2 * ds + 2.0 ** -15) * top).all())


# ---- together, as a decode step uses them ------------------------------------------
def test_a_layer_step_captured_and_replayed():
    """Projections from 4-bit weights, rows into the cache, attention over it and
    the output projection, captured in two graphs with workspaces of their own
    on two streams, replayed between eager work."""
    torch.manual_seed(0)
    H, hd, D, N, lens = 4, 64, 256, 8, [100, 37]
    parents = R.tree(N, 3)
    wqkv, wo = weights(D, 3 * D, "bf16", 1), weights(D, D, "bf16", 2)
    pq, po = pack(wqkv.cuda(), "bf16"), pack(wo.cuda(), "bf16")
    rows = 2 * N
    seq = torch.arange(2, dtype=torch.int32).repeat_interleave(N).cuda()
    pos = torch.cat([n + torch.arange(N) for n in lens]).to(torch.int32).cuda()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")

    class Side:
        def __init__(self):
            self.c = R.Cache(lens, N, H, hd, 16, "bf16", 4).to("cuda")
            self.x = torch.zeros(rows, D, dtype=torch.bfloat16, device="cuda")
            self.qkv, self.y = torch.empty(rows, 3 * D, device="cuda"), torch.empty(rows, D, device="cuda")
            self.h = torch.empty(rows, 3 * D, dtype=torch.bfloat16, device="cuda")
            self.a = torch.empty(rows, D, dtype=torch.bfloat16, device="cuda")
            self.nw = [B.chimera_gemm_fp4_bytes(1, rows, 3 * D, D), B.chimera_kv4_attn_bytes(self.c.struct(), H, N),
                       B.chimera_gemm_fp4_bytes(1, rows, D, D)]
            self.ws = [torch.empty(max(b, 16), dtype=torch.uint8, device="cuda") for b in self.nw]

        def step(self):
            s, kv = stream(), self.c.struct()
            B.chimera_gemm_fp4(1, self.x.data_ptr(), D, pq.data_ptr(), rows, 3 * D, D, self.qkv.data_ptr(), 3 * D,
                               self.ws[0].data_ptr(), self.nw[0], s)
            self.h.copy_(self.qkv)
            p = self.h.data_ptr()
            B.chimera_kv4_append(kv, 1, p + 2 * D, p + 4 * D, 3 * D, seq.data_ptr(), pos.data_ptr(), rows, s)
            B.chimera_kv4_attn(kv, 1, p, 3 * D, n.data_ptr(), H, parents, N, 0.125, self.a.data_ptr(), D,
                               self.ws[1].data_ptr(), self.nw[1], s)
            B.chimera_gemm_fp4(1, self.a.data_ptr(), D, po.data_ptr(), rows, D, D, self.y.data_ptr(), D,
                               self.ws[2].data_ptr(), self.nw[2], s)

    a, b, e = Side(), Side(), Side()
    graphs = []
    for side in (a, b):
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            side.step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            side.step()
        graphs.append((g, st))
    for i in range(4):
        xs = [torch.randn(rows, D).bfloat16().cuda() for _ in range(2)]
        a.x.copy_(xs[0])
        b.x.copy_(xs[1])
        torch.cuda.synchronize()
        for g, st in graphs:
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for side, x in ((a, xs[0]), (b, xs[1])):
            e.x.copy_(x)
            e.step()
            torch.cuda.synchronize()
            assert torch.equal(side.y, e.y), i
            # the definition, from the rows as they were rounded
            qkv = e.h.cpu()
            kvs = [torch.cat((e.c.kv[j][:lens[j]], qkv[j * N:(j + 1) * N, D:].reshape(N, 2, H, hd)))
                   for j in range(2)]
            want, tol = R.attention(qkv[:, :D].reshape(2, N, H, hd), kvs, lens, parents, 0.125)
            check_attention(e.a, want, tol)
            check_product(x.cpu(), wqkv, e.qkv)
            check_product(e.a.cpu(), wo, e.y)
