"""The 4-bit operators' limits and sizes, on the host: nothing is launched."""
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
