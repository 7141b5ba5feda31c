"""Checks of the operators over a plain paged cache that happen on the host: sizes and
refusals.  No call here passes its checks, so nothing is launched; pointers are never
read."""
import numpy as np
import pytest

from paper_2402_15758_amd import binding as B

P = 4096  # stands for an aligned device pointer
E, NOMEM = B.CHIMERA_EINVAL, B.CHIMERA_ENOMEM


def refused(status, what, f, *args):
    with pytest.raises(B.ChimeraError) as e:
        f(*args)
    assert e.value.status == status and what in str(e.value), str(e.value)


def cache(**kw):
    a = dict(pool=P, pool_bytes=1 << 40, page_table=P, batch=2, max_pages=4, n_pages=8, page_size=16, n_heads=4,
             head_dim=64, dtype=1)
    a.update(kw)
    return B.chimera_paged(**a)


def rope(**kw):
    a = dict(rot_dim=64, layout=0, max_positions=100, base=1e4, scaling=0, factor=1.0, original_positions=0, low=0.0,
             high=0.0, gain=1.0)
    a.update(kw)
    return B.chimera_rope(**a)


def append(c=None, dt=1, q=P, k=P, v=P, ld=768, heads=4, seq=P, pos=P, rows=1, r=None, table=None, gq=None, gk=None,
           eps=1e-5, out=2 * P, ldo=256):
    B.chimera_paged_append(c or cache(), dt, q, k, v, ld, heads, seq, pos, rows, r, table, gq, gk, eps, out, ldo, None)


def attn(c=None, q=P, ldq=256, heads=4, row0=P, n=P, rows=8, window=0, sinks=0, scale=0.125, out=P, ldo=256, ws=P,
         nb=1 << 40):
    B.chimera_paged_attn(c or cache(), q, ldq, heads, row0, n, rows, window, sinks, scale, out, ldo, ws, nb, None)


@pytest.mark.parametrize("bad", [dict(pool=None), dict(page_table=None), dict(head_dim=96), dict(n_heads=0),
                                 dict(n_heads=1025), dict(page_size=0), dict(page_size=257), dict(n_pages=0),
                                 dict(batch=0), dict(batch=65536), dict(max_pages=0), dict(dtype=2),
                                 dict(max_pages=1 << 24, page_size=256), dict(pool=P + 8),
                                 dict(n_pages=1 << 24, page_size=256)])
def test_cache_refusals(bad):
    for f in (append, attn):
        with pytest.raises(B.ChimeraError) as e:
            f(cache(**bad))
        assert e.value.status == E


def test_sizes():
    assert B.chimera_paged_bytes(8, 16, 4, 64, 1) == 8 * 2 * 4 * 16 * 64 * 2
    assert B.chimera_paged_bytes(8, 16, 4, 64, 0) == 8 * 2 * 4 * 16 * 64 * 4
    refused(NOMEM, "pool", append, cache(pool_bytes=8 * 2 * 4 * 16 * 64 * 2 - 1))
    refused(E, "head_dim", B.chimera_paged_bytes, 8, 16, 4, 32, 1)
    refused(E, "dtype", B.chimera_paged_bytes, 8, 16, 4, 64, 5)
    assert B.chimera_rope_bytes(rope()) == 100 * 32 * 8


@pytest.mark.parametrize("bad,what", [(dict(rot_dim=0), "rot_dim"), (dict(rot_dim=63), "rot_dim"),
                                      (dict(rot_dim=130), "rot_dim"), (dict(layout=2), "layout"),
                                      (dict(max_positions=0), "max_positions"),
                                      (dict(max_positions=(1 << 24) + 1), "max_positions"), (dict(base=1.0), "base"),
                                      (dict(base=float("inf")), "base"), (dict(gain=float("nan")), "gain"),
                                      (dict(scaling=3), "scaling"), (dict(scaling=1, factor=0.0), "factor"),
                                      (dict(scaling=2, factor=2.0, original_positions=0, low=1.0, high=2.0), "ramp"),
                                      (dict(scaling=2, factor=2.0, original_positions=9, low=2.0, high=2.0), "ramp"),
                                      (dict(scaling=2, factor=2.0, original_positions=9, low=-1.0, high=2.0), "ramp")])
def test_rope_refusals(bad, what):
    refused(E, what, B.chimera_rope_bytes, rope(**bad))
    refused(E, what, B.chimera_rope_table, rope(**bad), P, 1 << 40, None)
    refused(E, what, lambda: append(r=rope(**bad), table=P))


def test_rope_table_refusals():
    refused(E, "null", B.chimera_rope_table, rope(), None, 1 << 40, None)
    refused(E, "aligned", B.chimera_rope_table, rope(), P + 4, 1 << 40, None)
    refused(NOMEM, "table", B.chimera_rope_table, rope(), P, 100 * 32 * 8 - 1, None)


def test_append_refusals():
    refused(E, "dtype", lambda: append(dt=2))
    refused(E, "rows", lambda: append(rows=-1))
    refused(E, "rows", lambda: append(rows=(1 << 30) + 1))
    for n in ("k", "v", "seq", "pos", "out"):
        refused(E, "null", lambda: append(**{n: None}))
    refused(E, "stride", lambda: append(ld=255))
    refused(E, "stride", lambda: append(ldo=255))
    refused(E, "multiple", lambda: append(heads=6))
    refused(E, "multiple", lambda: append(heads=0))
    refused(E, "without q", lambda: append(q=None))
    refused(E, "without q", lambda: append(q=None, heads=0))
    refused(E, "without q", lambda: append(q=None, heads=0, out=None, gq=P))
    refused(E, "q_out", lambda: append(out=P))             # another stride
    refused(E, "q_out", lambda: append(out=P, ldo=768, dt=0))  # another type
    refused(E, "rot_dim", lambda: append(r=rope(rot_dim=66), table=P))
    refused(E, "null table", lambda: append(r=rope()))
    refused(E, "aligned", lambda: append(r=rope(), table=P + 8))
    refused(E, "without its rope", lambda: append(table=P))
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        refused(E, "eps", lambda: append(gq=P, eps=eps))
        refused(E, "eps", lambda: append(gk=P, eps=eps))


def test_attention_refusals():
    need = B.chimera_paged_attn_bytes(cache(), 4, 8)
    refused(E, "multiple", lambda: attn(heads=6))
    refused(E, "multiple", lambda: attn(heads=0))
    refused(E, "2^26", lambda: attn(rows=-1))
    refused(E, "2^26", lambda: attn(rows=1 << 25))
    refused(E, "2^23", lambda: attn(cache(batch=65535), heads=256, ldq=1 << 20, ldo=1 << 20))
    refused(E, "without row0", lambda: attn(row0=None))
    for n in ("q", "n", "out"):
        refused(E, "null", lambda: attn(**{n: None}))
    refused(E, "null workspace", lambda: attn(ws=None))
    refused(E, "aligned", lambda: attn(ws=P + 4))
    refused(NOMEM, "workspace", lambda: attn(nb=need - 1))
    refused(E, "stride", lambda: attn(ldq=248))
    refused(E, "stride", lambda: attn(ldo=255))
    refused(E, "multiples of 16", lambda: attn(ldq=257))
    refused(E, "aligned", lambda: attn(q=P + 2))
    for w in (-1, (1 << 30) + 1):
        refused(E, "window", lambda: attn(window=w))
        refused(E, "window", lambda: attn(sinks=w))
    for s in (float("inf"), float("nan"), 2.0 ** 127 * 1.01):
        refused(E, "scale", lambda: attn(scale=s))


def test_a_workspace_holds_for_smaller_calls():
    """Fewer rows, and fewer sequences with the same rows."""
    for heads, H, pages, ps in ((4, 4, 4, 16), (32, 8, 2048, 16), (7, 1, 513, 64), (32, 32, 256, 16)):
        last = 0
        for rows in (0, 1, 2, 5, 8, 9, 31, 64, 65, 200, 511, 2044, 5000, 20000):
            now = B.chimera_paged_attn_bytes(cache(n_heads=H, max_pages=pages, page_size=ps, batch=64), heads, rows)
            assert now >= last
            last = now
            few = B.chimera_paged_attn_bytes(cache(n_heads=H, max_pages=pages, page_size=ps, batch=3), heads, rows)
            assert few <= now
    last = 0
    for nodes in (1, 2, 7, 64):
        now = B.chimera_accept_bytes(8, nodes, 32000, 1)
        assert now >= last and now >= B.chimera_accept_bytes(8, nodes, 32000, 0)
        assert now >= B.chimera_accept_bytes(7, nodes, 32000, 1)
        last = now


def accept(dt=1, logits=P, ld=100, draft=None, ldd=0, vocab=100, tokens=P, parent=None, nodes=4, batch=2, T=1.0, u=P,
           new=P, n=P, path=P, ws=P, nb=1 << 40):
    B.chimera_accept(dt, logits, ld, draft, ldd, vocab, tokens, parent, nodes, batch, T, u, new, n, path, ws, nb, None)


def test_accept_refusals():
    refused(E, "dtype", lambda: accept(dt=9))
    for nodes in (0, 65):
        refused(E, "n_nodes", lambda: accept(nodes=nodes))
        refused(E, "n_nodes", B.chimera_accept_bytes, 1, nodes, 100, 0)
    for b in (0, 65536):
        refused(E, "batch", lambda: accept(batch=b))
    for v in (0, (1 << 24) + 1):
        refused(E, "vocab", lambda: accept(vocab=v, ld=1 << 25))
    for name in ("logits", "tokens", "u", "new", "n", "ws"):
        refused(E, "null", lambda: accept(**{name: None}))
    refused(E, "stride", lambda: accept(ld=99))
    refused(E, "stride", lambda: accept(draft=P, ldd=99))
    for t in (0.0, -1.0, float("inf"), float("nan")):
        refused(E, "temperature", lambda: accept(T=t))
    refused(E, "root", lambda: accept(nodes=2, parent=np.array([0, 0], dtype=np.int32)))
    refused(E, "root", lambda: accept(nodes=2, parent=np.array([-1, 1], dtype=np.int32)))
    refused(E, "chain", lambda: accept(nodes=3, draft=P, ldd=100, parent=np.array([-1, 0, 0], dtype=np.int32)))
    refused(E, "aligned", lambda: accept(ws=P + 8))
    refused(NOMEM, "workspace", lambda: accept(nb=B.chimera_accept_bytes(2, 4, 100, 0) - 1))
    with pytest.raises(ValueError):
        accept(nodes=3, parent=np.array([-1, 0], dtype=np.int32))
