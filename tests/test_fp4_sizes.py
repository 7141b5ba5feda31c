"""The 4-bit operators' limits and sizes, on the host: nothing is launched."""
import subprocess

import numpy as np
import pytest

from paper_2402_15758_amd import binding as B

P = 4096  # stands for an aligned device pointer


def cache(**kw):
    a = dict(pool=P, pool_bytes=1 << 50, page_table=P, batch=2, max_pages=4, n_pages=8, page_size=16, n_heads=4,
             head_dim=64)
    a.update(kw)
    return B.chimera_kv4(**a)


@pytest.mark.parametrize("scale", [2.0 ** 127 * 1.01, -3.3e38])
def test_a_scale_that_log2e_takes_past_the_float_is_refused(scale):
    with pytest.raises(B.ChimeraError) as e:
        B.chimera_kv4_attn(cache(), 1, P, 256, P, 4, None, 1, scale, P, 256, P, 1 << 40, None)
    assert e.value.status == B.CHIMERA_EINVAL and "2^127" in str(e.value)


def size_passes(status, what, f, *args):
    """The call gets past its check of the workspace's size, to a later refusal."""
    with pytest.raises(B.ChimeraError) as e:
        f(*args)
    assert e.value.status == B.CHIMERA_EINVAL and "aligned" in str(e.value), (what, str(e.value))


@pytest.mark.parametrize("dtype,N,K", [(1, 4096, 4096), (1, 2048, 2048), (1, 1024, 7168), (1, 5120, 13824),
                                       (1, 48, 4096), (1, 12288, 4096), (0, 1024, 2048)])
def test_a_products_workspace_holds_for_fewer_rows(dtype, N, K):
    last = 0
    for M in list(range(1, 4097, 61)) + [16, 17, 32, 33, 64, 65, 512, 513, 768, 769, 1280, 1281, 2816, 2817, 4096]:
        assert B.chimera_gemm_fp4_bytes(dtype, M, N, K) >= B.chimera_gemm_fp4_bytes(dtype, max(1, M - 1), N, K)
    most = [B.chimera_gemm_fp4_bytes(dtype, M, N, K) for M in (700, 1300, 2900, 4096)]
    assert most == sorted(most)
    for top, ws in zip((700, 1300, 2900, 4096), most):
        for M in range(1, top + 1):
            size_passes(B.CHIMERA_EINVAL, M, B.chimera_gemm_fp4, dtype, P + 4, K, P, M, N, K, P, N, P + 4, ws, None)


@pytest.mark.parametrize("H,Hq,pages,page", [(32, 32, 256, 16), (8, 32, 512, 64), (1, 1, 4096, 16), (4, 64, 40, 256)])
def test_an_attentions_workspace_holds_for_fewer_queries(H, Hq, pages, page):
    def c(b):
        return cache(batch=b, max_pages=pages, n_pages=4096, page_size=page, n_heads=H, head_dim=128)

    batches = [1, 2, 3, 5, 7, 8, 9, 31, 64, 255, 256, 257, 300]
    w = Hq * 128
    size = {(b, n): B.chimera_kv4_attn_bytes(c(b), Hq, n) for b in batches for n in range(1, 65)}
    for (b, n), ws in size.items():
        assert n == 1 or ws >= size[b, n - 1]
        assert b == 1 or ws >= size[batches[batches.index(b) - 1], n]
    tree = [-1] + [0] * 63
    for top_b, top_n in ((8, 49), (9, 64), (300, 33), (1, 64)):
        for b in range(1, top_b + 1):
            for n in (1, 2, 15, 16, 17, 32, 33, 48, 49, 64):
                if n <= top_n:
                    size_passes(B.CHIMERA_EINVAL, (b, n), B.chimera_kv4_attn, c(b), 1, P + 2, w, P, Hq,
                                np.array(tree[:n], dtype=np.int32), n, 0.1, P, w, P, size[top_b, top_n], None)


def test_the_error_message_is_the_librarys_own():
    """Its name is none that a program or another library could take over."""
    names = subprocess.run(["nm", "-D", "--defined-only", B.LIB_PATH], capture_output=True, text=True,
                           check=True).stdout
    assert "chimera_last_error" in names and "g_err" not in names
