"""Routes of the 4-bit operators that depend on the amount of work, on both sides of
their borders: launches that unpack the matrix, with a reduction in slices; the
attention in one launch inside the engine; both formats at 7B width."""
import dataclasses

import numpy as np
import pytest
import torch

import fp4_ref as R
import synth
from paper_2402_15758_amd import Session
from paper_2402_15758_amd import binding as B
from test_gpu_fp4 import check_product, pack, stream, unpack, weights
from test_gpu_fp4_engine import SMALL, greedy, prompts, rounded, run

pytestmark = pytest.mark.gpu


def least_workspace(dtype, M, N, K):
    """The smallest workspace a call accepts: found by refusals alone."""
    lo, hi = 0, B.chimera_gemm_fp4_bytes(dtype, M, N, K)  # hi is accepted
    while lo < hi:
        mid = (lo + hi) // 2
        try:
            B.chimera_gemm_fp4(dtype, 4096, K, 4096, M, N, K, 4096, N, 4096 + 4, mid, None)  # ws not aligned
        except B.ChimeraError as e:
            enough = e.status == B.CHIMERA_EINVAL
        lo, hi = (lo, mid) if enough else (mid + 1, hi)
    return hi


def product(x, p, N, K):
    """x @ the matrix, in a workspace of exactly the bytes the call needs."""
    M = x.shape[0]
    need, guard = least_workspace(1, M, N, K), 1 << 20
    ws = torch.full((need + guard,), 0x5A, dtype=torch.uint8, device="cuda")
    y = torch.full((M + 2, N), 123.0, device="cuda")
    B.chimera_gemm_fp4(1, x.data_ptr(), K, p.data_ptr(), M, N, K, y.data_ptr(), N, ws.data_ptr(), need, stream())
    assert bool((ws[need:] == 0x5A).all()) and bool((y[M:] == 123).all()), "written past the workspace or y"
    return y[:M]


def borders(N, K, top):
    """Row counts where a launch takes another route: around those from which on the
    matrix is unpacked, and where more rows need less (the kernel that sums the slices
    itself)."""
    need = {M: least_workspace(1, M, N, K) for M in [*range(64, top + 1, 64), *range(65, top + 1, 64)]}
    drops = [M for M in range(65, top + 1, 64) if need[M] < need[M - 1]]
    near = [M for M in (384, 385, 512, 513, 600, 768, 769, 2048, 2049) if M <= top]
    return sorted({*near, top} | {M + i for M in drops for i in (-1, 0)})


@pytest.mark.parametrize("N,K", [(1024, 2048), (2048, 4096), (4096, 1024), (64, 1024), (48, 2048), (4096, 4096),
                                 (12288, 1024)])
def test_many_rows_have_the_bits_of_one(N, K):
    top = 3000
    g = torch.Generator().manual_seed(N + K)
    x = torch.randn(top, K, generator=g).bfloat16().cuda()
    w = weights(K, N, "bf16", K)
    p = pack(w.cuda(), "bf16")
    picks = [0, 15, 16, 63, 64, 255, 511, 512, 599, 1279, 1280, 2047, top - 1]
    alone = {r: product(x[r:r + 1], p, N, K)[0] for r in picks}
    for M in borders(N, K, top):
        y = product(x[:M], p, N, K)
        for r in picks:
            if r < M:
                assert torch.equal(y[r], alone[r]), (M, r)
        last = product(x[M - 1:M], p, N, K)[0]
        assert torch.equal(y[M - 1], last), M
    check_product(x[:600].cpu(), w, product(x[:600], p, N, K))


@pytest.mark.parametrize("N,K", [(1024, 2048), (2048, 4096), (64, 1024)])
def test_many_rows_have_the_bits_of_the_bf16_product(N, K):
    """Blocks of 128 rows by the library's bf16 product of the unpacked matrix, whose
    rows do not depend on each other."""
    g = torch.Generator().manual_seed(N)
    top = 1400
    x = torch.randn(top, K, generator=g).bfloat16().cuda()
    p = pack(weights(K, N, "bf16", 3).cuda(), "bf16")
    w = unpack(p, N, K, "bf16")
    ref = torch.empty(top, N, device="cuda")
    for r in range(0, top, 128):
        n = min(128, top - r)
        B.chimera_gemm_static(B.CHIMERA_BF16, x[r:].data_ptr(), w.data_ptr(), n, N, K, ref[r:].data_ptr(), stream())
        torch.cuda.synchronize()
    for M in borders(N, K, top):
        assert torch.equal(product(x[:M], p, N, K), ref[:M]), M


@pytest.mark.parametrize("lens,tree,batch", [([900, 40, 700, 513], "T64", 4), ([30 + 7 * i for i in range(26)], "T32", 26)])
def test_engine_unpacks_with_split_reductions(lens, tree, batch):
    """Prefill chunks of over 768 rows, and a verify pass of 832, over unpacked
    matrices: the bits of the rounded model."""
    cfg = dataclasses.replace(SMALL, d_model=1280, n_heads=10, d_ffn=4096, n_layers=2)
    w = synth.make_weights(cfg, std=0.04)
    ps = prompts(lens, cfg.vocab, 5)
    outs = []
    for weights_, fmt in ((w, "fp4"), (rounded(w), "native")):
        s = Session(cfg, weights_, synth.TREES[tree], max_batch=batch, max_len=1024, weight_format=fmt)
        outs.append(run(s, ps, 3))
        s.close()
    assert np.array_equal(outs[0][0], outs[1][0])
    for i in range(1, 4):
        for a, b in zip(outs[0][i], outs[1][i]):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("cfg,tree", [(synth.TINY, "T8"), (SMALL, "T64"), (SMALL, "none")])
@pytest.mark.parametrize("wfmt", ["native", "fp4"])
def test_engine_attention_in_one_launch(cfg, tree, wfmt):
    """Tables of at most 256 positions: the bits of the same steps over a longer one,
    and the stream of greedy decoding."""
    w = synth.make_weights(cfg, std=0.06)
    tr = () if tree == "none" else synth.TREES[tree]
    ps = prompts([60, 9, 25], cfg.vocab, 6)
    got = []
    for max_len in (160, 1024):
        s = Session(cfg, w, tr, max_batch=3, max_len=max_len, weight_format=wfmt, kv_format="fp4")
        got.append(run(s, ps, 8))
        s.close()
    for i in range(4):
        for a, b in zip(got[0][i], got[1][i]):
            assert np.array_equal(a, b)
    s = Session(cfg, w, tr, max_batch=3, max_len=160, weight_format=wfmt, kv_format="fp4")
    assert s.generate(ps, 30)[0] == greedy(cfg, w, ps, 30, weight_format=wfmt, kv_format="fp4")
    s.close()


def test_engine_at_7b_width():
    """Two layers of the 7B shape: 4-bit weights have the bits of the rounded model in
    prefill chunks of 64 to 900 rows and in steps; over both formats speculative steps
    give the stream of greedy ones."""
    cfg = dataclasses.replace(synth.LLAMA7B, n_layers=2)
    w = synth.make_weights(cfg, device="cuda")
    r = dict(w)
    for name, t in w.items():
        if name.startswith("layers.") and t.dim() == 2:
            K, N = t.shape
            r[name] = unpack(pack(t, "bf16"), N, K, "bf16")
    some = "layers.1.w_down"
    assert torch.equal(r[some][:, :64].double().cpu(), R.held(w[some][:, :64].t().contiguous().cpu()).t())
    ps = prompts([900, 64], cfg.vocab, 7)
    outs = []
    for weights_, fmt in ((w, "fp4"), (r, "native")):
        s = Session(cfg, weights_, synth.TREES["T64"], max_batch=2, max_len=1024, weight_format=fmt)
        outs.append(run(s, ps, 3))
        s.close()
    del r
    for i in range(4):
        for a, b in zip(outs[0][i], outs[1][i]):
            assert np.array_equal(a, b)
    kw = dict(weight_format="fp4", kv_format="fp4")
    want = greedy(cfg, w, ps, 24, **kw)
    s = Session(cfg, w, synth.TREES["T64"], max_batch=2, max_len=1024, **kw)
    assert s.generate(ps, 24)[0] == want
    s.close()


def test_profiled_products_count_the_unpacking():
    """640 verify rows at 7B width: with 4-bit weights the products' time holds the
    unpacking (0.8 GB written over two layers, 0.1 ms at the card's peak rate next to
    some 0.5 ms of products), which the same kernels over bf16 weights do not have."""
    cfg = dataclasses.replace(synth.LLAMA7B, n_layers=2)
    w = synth.make_weights(cfg, device="cuda")
    ps = prompts([20] * 20, cfg.vocab, 7)
    ms = {}
    for fmt in ("fp4", "native"):
        s = Session(cfg, w, synth.TREES["T32"], max_batch=20, max_len=128, weight_format=fmt)
        s.set_graph(False)
        s.profile(True)
        s.prefill(ps)
        times = []
        for _ in range(8):
            s.step()
            times.append(s.profile_read().ms_gemm_verify)
            s.profile(True)
        ms[fmt] = sorted(times)[len(times) // 2]
        s.close()
    assert ms["fp4"] > ms["native"] + 0.08, ms


@pytest.mark.parametrize("dtype,N,K", [("bf16", 4096, 7168), ("bf16", 4096, 34816), ("bf16", 8176, 1536),
                                       ("bf16", 5120, 4096), ("bf16", 2048, 8192), ("bf16", 16, 4096),
                                       ("bf16", 16, 2048), ("f32", 4096, 7168), ("f32", 256, 1024),
                                       ("f32", 4112, 1024)])
def test_a_workgroup_a_column_block_has_the_bits_of_slices(dtype, N, K):
    """Row counts on both sides of the choice (8 and 4 rows of 7168 values are the
    most that LDS holds), with and without room between the rows."""
    g = torch.Generator().manual_seed(K)
    t = R.TYPES[dtype]
    big = torch.randn(17, K + 8, generator=g).to(t).cuda()
    w = weights(K, N, dtype, 5)
    p = pack(w.cuda(), dtype)
    d = 1 if dtype == "bf16" else 0
    for src in (big[:, :K].contiguous(), big[:, :K]):
        ref = None
        for M in (17, 16, 12, 9, 8, 7, 5, 4, 3, 2, 1):
            need = B.chimera_gemm_fp4_bytes(d, M, N, K)
            ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
            y = torch.full((M + 1, N), 123.0, device="cuda")
            B.chimera_gemm_fp4(d, src.data_ptr(), src.stride(0), p.data_ptr(), M, N, K, y.data_ptr(), N, ws.data_ptr(),
                               need, stream())
            ref = y[:M].clone() if ref is None else ref
            assert torch.equal(y[:M], ref[:M]) and bool((y[M] == 123).all()), M
    check_product(big[:, :K].cpu(), w, ref)
