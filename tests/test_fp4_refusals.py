"""Checks of the 4-bit operators that happen on the host: sizes and refusals.
No call here passes its checks, so nothing is launched; pointers are never read."""
import os
import re

import numpy as np
import pytest

from paper_2402_15758_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096  # stands for an aligned device pointer


def refused(status, what, f, *args):
    with pytest.raises(B.ChimeraError) as e:
        f(*args)
    assert e.value.status == status and what in str(e.value), str(e.value)


def test_every_declared_name_is_exported_and_bound():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "chimera.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(chimera_[a-z0-9_]+)\s*\(", src))
    assert {"chimera_gemm_fp4", "chimera_kv4_attn", "chimera_kv4_append"} <= names
    for n in names:
        assert hasattr(B.lib(), n) and hasattr(B, n), n


def test_the_format_in_float64():
    """The tests' own reference: the format's corners, spelled out."""
    import torch
    import fp4_ref
    x = torch.zeros(6, 32)
    x[0, :10] = torch.tensor([6, 0.25, 0.26, 0.75, -1.25, 1.75, 2.5, 3.5, 5, -5.1])
    x[1, :2] = torch.tensor([7.0, 0.5])    # 1.75 x 4: stays, saturates
    x[2, :2] = torch.tensor([7.01, 0.5])   # above: the scale doubles
    x[3, 0] = 2.0 ** -140
    x[4, 0] = float("inf")
    h = fp4_ref.held(x)
    assert h[0, :10].tolist() == [6, 0, 0.5, 1, -1, 2, 2, 4, 4, -6]
    assert h[1, :2].tolist() == [6, 0.5] and h[2, :2].tolist() == [8, 0]
    assert h[3].abs().sum() == 0 and torch.isnan(h[4]).all() and h[5].abs().sum() == 0
    big = torch.full((1, 32), 3.3e38)
    assert fp4_ref.held(big)[0, 0] == 6 * 2.0 ** 125
    code, s = fp4_ref.encode(x)
    assert s[:, 0].tolist() == [127, 127, 128, 1, 255, 1]
    again = fp4_ref.held(h[:4])
    assert torch.equal(again, h[:4])  # values of the format are its own


def test_matrix_sizes():
    for N, K in [(8, 32), (24, 32), (16, 16), (0, 32), (16, 0), (-16, 32)]:
        refused(B.CHIMERA_EINVAL, "N must be a multiple of 16", B.chimera_fp4_bytes, N, K)
    for N, K in [((1 << 20) + 16, 32), (16, (1 << 20) + 32)]:
        refused(B.CHIMERA_EINVAL, "2^20", B.chimera_fp4_bytes, N, K)
    assert B.chimera_fp4_bytes(4096, 4096) == 4096 * 4096 * 17 // 32
    # classes of a slice are padded to whole units of four k-blocks
    assert B.chimera_fp4_bytes(16, 32) == 4 * (1024 + 64)


def test_pack_and_product_refusals():
    E = B.CHIMERA_EINVAL
    nb = B.chimera_fp4_bytes(64, 64)
    refused(E, "dtype", B.chimera_fp4_pack, 7, P, 64, 64, 64, P, nb, None)
    refused(E, "null", B.chimera_fp4_pack, 1, None, 64, 64, 64, P, nb, None)
    refused(E, "ldw", B.chimera_fp4_pack, 1, P, 63, 64, 64, P, nb, None)
    refused(E, "aligned", B.chimera_fp4_pack, 1, P, 64, 64, 64, P + 8, nb, None)
    refused(B.CHIMERA_ENOMEM, "packed", B.chimera_fp4_pack, 1, P, 64, 64, 64, P, nb - 1, None)
    refused(E, "ldw", B.chimera_fp4_unpack, 1, P, 64, 64, P, 10, None)
    for M in (0, -1, 4097):
        refused(E, "M in", B.chimera_gemm_fp4_bytes, 1, M, 64, 64)
        refused(E, "M in", B.chimera_gemm_fp4, 1, P, 64, P, M, 64, 64, P, 64, P, 1 << 30, None)
    refused(E, "ldx", B.chimera_gemm_fp4, 1, P, 63, P, 1, 64, 64, P, 64, P, 1 << 30, None)
    refused(E, "ldy", B.chimera_gemm_fp4, 1, P, 64, P, 1, 64, 64, P, 63, P, 1 << 30, None)
    refused(E, "null", B.chimera_gemm_fp4, 1, P, 64, P, 1, 64, 64, None, 64, P, 1 << 30, None)
    refused(E, "packed", B.chimera_gemm_fp4, 1, P, 64, P + 4, 1, 64, 64, P, 64, P, 1 << 30, None)
    need = B.chimera_gemm_fp4_bytes(1, 64, 4096, 4096)
    assert need >= 64 * 4096 * 2
    refused(B.CHIMERA_ENOMEM, "workspace", B.chimera_gemm_fp4, 1, P, 4096, P, 64, 4096, 4096, P, 4096, P, need - 1,
            None)
    refused(E, "null workspace", B.chimera_gemm_fp4, 1, P, 4096, P, 64, 4096, 4096, P, 4096, None, need, None)
    refused(E, "aligned", B.chimera_gemm_fp4, 1, P, 4096, P, 64, 4096, 4096, P, 4096, P + 4, need, None)


def cache(**kw):
    a = dict(pool=P, pool_bytes=1 << 40, page_table=P, batch=2, max_pages=4, n_pages=8, page_size=16, n_heads=4,
             head_dim=64)
    a.update(kw)
    return B.chimera_kv4(**a)


@pytest.mark.parametrize("bad", [dict(pool=None), dict(page_table=None), dict(head_dim=96), dict(n_heads=0),
                                 dict(n_heads=1025), dict(page_size=0), dict(page_size=257), dict(n_pages=0),
                                 dict(batch=0), dict(batch=65536), dict(max_pages=0),
                                 dict(max_pages=1 << 24, page_size=256), dict(pool=P + 8)])
def test_cache_refusals(bad):
    c = cache(**bad)
    with pytest.raises(B.ChimeraError) as e:
        B.chimera_kv4_append(c, 1, P, P, 256, P, P, 1, None)
    assert e.value.status == B.CHIMERA_EINVAL
    with pytest.raises(B.ChimeraError) as e:
        B.chimera_kv4_attn_bytes(c, 4, 1)
    assert e.value.status == B.CHIMERA_EINVAL


def test_row_refusals():
    E = B.CHIMERA_EINVAL
    assert B.chimera_kv4_bytes(8, 16, 4, 64) == 8 * 2 * 4 * 16 * 34
    refused(B.CHIMERA_ENOMEM, "pool", B.chimera_kv4_append, cache(pool_bytes=8 * 2 * 4 * 16 * 34 - 1), 1, P, P, 256, P,
            P, 1, None)
    for f, lead in ((B.chimera_kv4_append, True), (B.chimera_kv4_read, False)):
        def call(c=None, dt=1, k=P, v=P, ld=256, seq=P, pos=P, rows=1):
            c = c or cache()
            if lead:
                f(c, dt, k, v, ld, seq, pos, rows, None)
            else:
                f(c, dt, seq, pos, rows, k, v, ld, None)
        refused(E, "dtype", lambda: call(dt=2))
        refused(E, "rows", lambda: call(rows=-1))
        refused(E, "stride", lambda: call(ld=255))
        for n in ("k", "v", "seq", "pos"):
            refused(E, "null", lambda: call(**{n: None}))


def test_attention_refusals():
    E = B.CHIMERA_EINVAL
    need = B.chimera_kv4_attn_bytes(cache(), 4, 64)

    def call(c=None, dt=1, q=P, ldq=256, n=P, heads=4, parent=None, nodes=1, scale=0.125, out=P, ldo=256, ws=P,
             nb=1 << 40):
        B.chimera_kv4_attn(c or cache(), dt, q, ldq, n, heads, parent, nodes, scale, out, ldo, ws, nb, None)

    refused(E, "dtype", lambda: call(dt=3))
    refused(E, "n_heads", lambda: call(heads=6))
    refused(E, "n_heads", lambda: call(heads=0))
    for nodes in (0, 65):
        refused(E, "n_nodes", lambda: call(nodes=nodes))
    for n in ("q", "n", "out", "ws"):
        refused(E, "null", lambda: call(**{n: None}))
    refused(E, "stride", lambda: call(ldq=248))
    refused(E, "stride", lambda: call(ldo=255))
    refused(E, "multiples of 16", lambda: call(ldq=257))
    refused(E, "aligned", lambda: call(q=P + 2))
    refused(E, "aligned", lambda: call(ws=P + 4))
    refused(E, "finite", lambda: call(scale=float("inf")))
    refused(E, "finite", lambda: call(scale=float("nan")))
    refused(B.CHIMERA_ENOMEM, "workspace", lambda: call(nodes=64, parent=np.array([-1] + [0] * 63, dtype=np.int32),
                                                        nb=need - 1))
    refused(E, "deeper", lambda: call(nodes=17))  # a chain of 17 nodes
    refused(E, "root", lambda: call(nodes=2, parent=np.array([0, 0], dtype=np.int32)))
    refused(E, "root", lambda: call(nodes=2, parent=np.array([-1, 1], dtype=np.int32)))
    refused(E, "root", lambda: call(nodes=3, parent=np.array([-1, 0, -1], dtype=np.int32)))
    with pytest.raises(ValueError):
        call(nodes=3, parent=np.array([-1, 0], dtype=np.int32))
