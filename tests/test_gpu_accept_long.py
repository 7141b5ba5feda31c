"""Verification over rows whose weights reach the end of the range."""
import math

import pytest
import torch

import paged_ref as R
from test_gpu_accept import run

pytestmark = pytest.mark.gpu
LAST = 1 - 2.0 ** -53


@pytest.mark.parametrize("low,high,first", [(-57.0, 130.0, 1024 + 77), (-50.0, 130.0, 0), (127.0, 190.0, 0),
                                            (100.0, 300.0, 1024 + 77)])
def test_weights_at_the_end_of_the_range(low, high, first):
    """1024 equal logits, then a part of far larger ones: the draw at 0 goes to the first
    token whose weight is above 0 in 64 bits, also where a part's weights have a sum and are
    no numbers themselves, in calls large enough for the table of exponentials and in small
    ones."""
    V = 2048
    row = torch.full((V,), -math.inf)
    row[:1024], row[1024 + 77], row[1024 + 300] = low, high, high - 2.0
    row = row.bfloat16()
    want = [R.accept(row[None], None, [0], [-1], [x], 0.25)[0] for x in (0.0, 0.5, LAST)]
    assert want == [[first], [1024 + 77], [1024 + 300]]
    for batch in (3, 5200):
        u = torch.tensor([0.0, 0.5, LAST], dtype=torch.float64).repeat(-(-batch // 3))[:batch, None]
        got = run(row.expand(batch, V).contiguous(), None, torch.zeros(batch, 1, dtype=torch.int64), [-1], u, 0.25, V)
        assert all(o == (want[i % 3], [0]) for i, o in enumerate(got)), got[:3]
