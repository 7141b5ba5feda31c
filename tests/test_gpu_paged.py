"""Operators over a plain paged cache on the GPU against float64 references
(paged_ref), at the sizes, types, strides and masks where they can go wrong."""
import math

import pytest
import torch

import paged_ref as R
from paper_2402_15758_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": B.CHIMERA_BF16, "f32": B.CHIMERA_F32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step, relative


def stream():
    return torch.cuda.current_stream().cuda_stream


def cache_of(pool, table, dtype):
    n_pages, _, H, ps, hd = pool.shape
    return B.chimera_paged(pool.data_ptr(), pool.numel() * pool.element_size(), table.data_ptr(), table.shape[0],
                           table.shape[1], n_pages, ps, H, hd, DT[dtype])


def table_of(g, batch, positions, page, spare=2):
    per = -(-positions // page)
    return torch.randperm(batch * per + spare, generator=g)[:batch * per].view(batch, per).int(), batch * per + spare


# ---- rows into the cache -------------------------------------------------------------
ROPES = {
    "none": None,
    "half": dict(rot=1.0, layout="half", base=10000.0),
    "pairs": dict(rot=1.0, layout="pairs", base=10000.0),
    "part": dict(rot=0.25, layout="half", base=10000.0),
    "pairs6": dict(rot=6, layout="pairs", base=100.0),    # rows of three pairs
    "half10": dict(rot=10, layout="half", base=10000.0),  # runs of five: no vector form
    "linear": dict(rot=1.0, layout="half", base=10000.0, scaling="linear", factor=3.5),
    "ramp": dict(rot=0.5, layout="pairs", base=500000.0, scaling="ramp", factor=8.0, original=512, low=1.0, high=4.0,
                 gain=1.25),
}
SCALING = {"none": B.CHIMERA_ROPE_NONE, "linear": B.CHIMERA_ROPE_LINEAR, "ramp": B.CHIMERA_ROPE_RAMP}


def rope_of(spec, hd, positions):
    rot = spec["rot"] if isinstance(spec["rot"], int) else int(spec["rot"] * hd)
    r = B.chimera_rope(rot, B.CHIMERA_ROPE_HALF if spec["layout"] == "half" else B.CHIMERA_ROPE_PAIRS, positions,
                       spec["base"], SCALING[spec.get("scaling", "none")], spec.get("factor", 1.0),
                       spec.get("original", 0), spec.get("low", 0.0), spec.get("high", 0.0), spec.get("gain", 1.0))
    th = R.theta(rot, spec["base"], spec.get("scaling", "none"), spec.get("factor", 1.0), spec.get("original", 0),
                 spec.get("low", 0.0), spec.get("high", 0.0))
    nb = B.chimera_rope_bytes(r)
    assert nb == positions * rot // 2 * 8
    table = torch.full((nb + 16,), 0xEE, dtype=torch.uint8, device="cuda")
    B.chimera_rope_table(r, table.data_ptr(), nb, stream())
    assert (table[nb:] == 0xEE).all()
    return r, table, th


@pytest.mark.parametrize("name", [n for n in ROPES if n != "none"])
def test_rope_table(name):
    spec = ROPES[name]
    r, table, th = rope_of(spec, 128, 2000)
    t = table[:2000 * th.numel() * 8].view(torch.float32).view(2000, -1, 2).double().cpu()
    ang = torch.arange(2000).double()[:, None] * th
    gain = R.f32(spec.get("gain", 1.0))
    # a rounding of the value, and the angle's in 64 bits (theta to a few steps)
    for i, f in enumerate((torch.cos, torch.sin)):
        assert bool(((t[..., i] - f(ang) * gain).abs() <= 2.0 ** -24 * abs(gain) + ang * 2.0 ** -49).all())


def append_case(dtype, held, Hq, H, hd, page, spec, normed, rows, seed, shift=0, pos_from=0, big=False):
    g = torch.Generator().manual_seed(seed)
    batch, positions = 3, pos_from + rows + 5
    table, n_pages = table_of(g, batch, positions, page)
    width = (Hq + 2 * H) * hd + 3 * shift
    x = torch.randn(rows, width, generator=g) * torch.exp(0.7 * torch.randn(width, generator=g))
    if big:
        x[0] *= 1e37 if held == "f32" or dtype == "bf16" else 1e30
        x[1] *= 1e-30
    x = x.to(R.TYPES[dtype]).cuda()
    seq = torch.randint(0, batch, (rows,), generator=g).int()
    pos = (pos_from + torch.arange(rows)).int()
    bad = []
    if rows >= 6:  # padding, positions and sequences that are not there, a page that is not there
        seq[1], pos[2], seq[3] = -1, positions + page, batch
        pos[4] = -1
        lost = int(seq[5])
        table[lost, int(pos[5]) // page] = n_pages
        bad = sorted({1, 2, 3, 4} | {r for r in range(rows) if seq[r] == lost and pos[r] // page == pos[5] // page})
        if rows > 6 and spec is not None:
            pos[6] = positions + 1  # may lie in the table of pages, not in the rotation's
            bad.append(6)
    gains = (1 + 0.3 * torch.randn(2, hd, generator=g)).cuda() if normed else None
    pool = torch.randn(n_pages, 2, H, page, hd, generator=g).to(R.TYPES[held]).cuda()
    before = pool.clone()
    out = torch.full((rows, Hq * hd + shift), 3.0, dtype=R.TYPES[held], device="cuda")
    rope, rt, th = rope_of(spec, hd, positions + 1) if spec is not None else (None, None, None)
    es = x.element_size()
    dt, ds, dp = table.cuda(), seq.cuda(), pos.cuda()
    p = x.data_ptr() + shift * es
    B.chimera_paged_append(cache_of(pool, dt, held), DT[dtype], p if Hq else None, p + Hq * hd * es,
                           p + (Hq + H) * hd * es, width, Hq, ds.data_ptr(), dp.data_ptr(), rows, rope,
                           rt.data_ptr() if rope else None, gains[0].data_ptr() if normed and Hq else None,
                           gains[1].data_ptr() if normed else None, 1e-5,
                           out.data_ptr() + shift * out.element_size() if Hq else None, out.stride(0), stream())
    torch.cuda.synchronize()
    # the reference
    xs = x.cpu()[:, shift:shift + (Hq + 2 * H) * hd].double().view(rows, -1, hd)
    qk, v = xs[:, :Hq + H], xs[:, Hq + H:]
    if normed:
        gg = gains.cpu()
        qk = torch.cat((R.norm(qk[:, :Hq], gg[0], 1e-5), R.norm(qk[:, Hq:], gg[1], 1e-5)), 1)
    y, mag = R.turn(qk, pos.clamp(0, positions), th, spec["layout"], spec.get("gain", 1.0)) if spec else (
        qk, qk.abs())
    # two products and a sum; a table entry (to a rounding of its gain); the norm's sum of
    # hd squares (half of it through the root), root, quotient and two products
    steps = (4 if spec else 0) + ((hd + 4) / 2 + 6 if normed else 0)
    bound = HALF[held] * y.abs() + steps * 2.0 ** -24 * mag * (1 + HALF[held]) + 1e-37
    good = [r for r in range(rows) if r not in bad]
    got_q = out.double().cpu()[:, shift:shift + Hq * hd].view(rows, Hq, hd)
    assert bool(((got_q - y[:, :Hq]).abs() <= bound[:, :Hq])[good].all())
    assert bool((got_q[bad] == 3).all())
    if shift:
        assert bool((out[:, :shift] == 3).all())
    got, want = pool.double().cpu(), before.double().cpu()
    for r in good:
        page_id, slot = int(table[int(seq[r]), int(pos[r]) // page]), int(pos[r]) % page
        assert bool(((got[page_id, 0, :, slot] - y[r, Hq:]).abs() <= bound[r, Hq:]).all()), r
        assert bool((got[page_id, 1, :, slot] == v[r].to(R.TYPES[held]).double()).all()), r
        got[page_id, :, :, slot] = want[page_id, :, :, slot]
    assert torch.equal(got, want)  # nothing else was written


@pytest.mark.parametrize("dtype,held", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rope", sorted(ROPES))
@pytest.mark.parametrize("normed", [False, True])
def test_append(dtype, held, rope, normed):
    for i, (Hq, H, hd, page, rows, at) in enumerate([(4, 4, 64, 16, 9, 0), (7, 1, 128, 5, 23, 1000), (0, 3, 128, 1, 7, 3),
                                                     (14, 2, 64, 256, 40, 90), (32, 8, 128, 16, 1, 37)]):
        append_case(dtype, held, Hq, H, hd, page, ROPES[rope], normed, rows, 100 * i + len(rope), pos_from=at)


@pytest.mark.parametrize("dtype,held", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("shift", [1, 2, 4])
def test_append_unaligned_rows(dtype, held, shift):
    append_case(dtype, held, 6, 2, 128, 16, ROPES["half"], True, 11, shift, shift=shift)
    append_case(dtype, held, 6, 2, 64, 16, ROPES["pairs6"], False, 11, shift, shift=shift)


def test_append_norms_of_extreme_rows():
    """Squares past the float's range, and rows far below eps."""
    append_case("f32", "f32", 4, 2, 128, 16, ROPES["half"], True, 5, 9, big=True)
    append_case("bf16", "bf16", 4, 2, 64, 16, None, True, 5, 9, big=True)


def test_append_infinities_stay_in_their_head():
    H, hd, rows = 2, 64, 3
    g = torch.Generator().manual_seed(4)
    x = torch.randn(rows, 3 * H * hd, generator=g)
    x[1, 5], x[1, hd + 7], x[2, 2 * H * hd + 1] = math.inf, math.nan, math.inf
    x = x.cuda()
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    pool = torch.zeros(1, 2, H, 16, hd, device="cuda")
    gain = torch.ones(hd, device="cuda")
    seq, pos = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.arange(rows).int().cuda()
    out = torch.empty(rows, H * hd, device="cuda")
    p = x.data_ptr()
    B.chimera_paged_append(cache_of(pool, table, "f32"), 0, p, p + 4 * H * hd, p + 8 * H * hd, 3 * H * hd, H,
                           seq.data_ptr(), pos.data_ptr(), rows, None, None, gain.data_ptr(), gain.data_ptr(), 1e-6,
                           out.data_ptr(), H * hd, stream())
    o = out.cpu().view(rows, H, hd)
    assert torch.isnan(o[1, 0, 5]) and (o[1, 0, :5] == 0).all() and torch.isnan(o[1, 1]).all()
    assert torch.isfinite(o[[0, 2]]).all() and torch.isinf(pool[0, 1, 0, 2, 1]) and torch.isfinite(pool[0, 0]).all()


def test_append_in_place_and_many_rows():
    """Queries turned where they lie, and more rows than a grid's second dimension."""
    g = torch.Generator().manual_seed(1)
    rows, H, hd = 70001, 1, 64
    x = torch.randn(rows, 3 * hd, generator=g).bfloat16().cuda()
    table = torch.randperm(274, generator=g).int().view(1, -1).cuda()
    seq, pos = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.arange(rows).int().cuda()
    rope, rt, _ = rope_of(ROPES["half"], hd, rows)
    outs = []
    for inplace in (False, True):
        y = x.clone()
        pool = torch.zeros(274, 2, H, 256, hd, dtype=torch.bfloat16, device="cuda")
        q_out = y if inplace else torch.empty_like(x)
        p = y.data_ptr()
        B.chimera_paged_append(cache_of(pool, table, "bf16"), 1, p, p + 2 * hd, p + 4 * hd, 3 * hd, H, seq.data_ptr(),
                               pos.data_ptr(), rows, rope, rt.data_ptr(), None, None, 0.0, q_out.data_ptr(), 3 * hd,
                               stream())
        outs.append((q_out[:, :hd].clone(), pool, y[:, hd:].clone()))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert torch.equal(outs[1][2], x[:, hd:])
    last = outs[0][1][table[0, 70000 // 256], 1, 0, 70000 % 256]
    assert torch.equal(last, x[70000, 2 * hd:])


# ---- attention -----------------------------------------------------------------------
def attend(q, pool, table, lens, rows, dtype, scale, window=0, sinks=0, row0="starts", ldo=None, behind=2, ws=None,
           far=False):
    """The operator's rows, and those behind the last sequence.  far: a table of so many
    pages that the work is dealt as for a long cache, 128 queries at once."""
    total, Hq, hd = q.shape
    if far:
        cap = int(1e10 / (4 * total * Hq * hd)) + 1
        wide = torch.full((table.shape[0], table.shape[1] + cap // pool.shape[3]), -1, dtype=torch.int32)
        wide[:, :table.shape[1]] = table
        table = wide
    dq = torch.zeros(total + behind, Hq * hd, dtype=R.TYPES[dtype], device="cuda")
    dq[:total] = q.reshape(total, -1).cuda()
    ldo = ldo or Hq * hd
    out = torch.full((total + behind, ldo), 7.0, dtype=R.TYPES[dtype], device="cuda")
    dt, dp = table.cuda(), pool.cuda()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    starts = torch.cat((torch.zeros(1), torch.tensor(rows).cumsum(0))).int().cuda() if row0 == "starts" else None
    c = cache_of(dp, dt, dtype)
    given = total + behind if starts is not None else total
    nb = B.chimera_paged_attn_bytes(c, Hq, given)
    ws = torch.full((nb + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    B.chimera_paged_attn(c, dq.data_ptr(), Hq * hd, Hq, None if starts is None else starts.data_ptr(), n.data_ptr(),
                         given, window, sinks, scale, out.data_ptr(), ldo, ws.data_ptr(), nb, stream())
    torch.cuda.synchronize()
    assert (ws[nb:] == 0xFF).all()
    assert (out[total:] == 7).all() and (out[:, Hq * hd:] == 7).all()
    return out[:total, :Hq * hd].view(total, Hq, hd).double().cpu()


def attn_inputs(dtype, lens, rows, Hq, H, hd, page, seed, poison=True):
    g = torch.Generator().manual_seed(seed)
    ends = [max(n, 0) + r for n, r in zip(lens, rows)]
    table, n_pages = table_of(g, len(lens), max(max(ends), 1), page)
    pool = torch.randn(n_pages, 2, H, page, hd, generator=g)
    pool[:, 0] *= torch.exp(0.5 * torch.randn(hd, generator=g))
    if poison:  # what nobody has written
        seen = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, e in enumerate(ends):
            p = torch.arange(e)
            seen[table[b][p // page].long(), p % page] = True
        pool.permute(0, 3, 1, 2, 4)[~seen] = math.nan
    q = torch.randn(sum(rows), Hq, hd, generator=g)
    return q.to(R.TYPES[dtype]), pool.to(R.TYPES[dtype]), table


def check(dtype, lens, rows, Hq, H, hd, page, seed, window=0, sinks=0, scale=None, **kw):
    q, pool, table = attn_inputs(dtype, lens, rows, Hq, H, hd, page, seed)
    scale = R.f32(hd ** -0.5 if scale is None else scale)
    got = attend(q, pool, table, lens, rows, dtype, scale, window, sinks, **kw)
    ref, mag, big = R.attention(q, pool, table, lens, rows, scale, window, sinks)
    bound = R.attention_bound(dtype, ref, mag, big, max(n + r for n, r in zip(lens, rows)), hd)
    err = (got - ref).abs()
    assert bool((err <= bound).all()), (float((err / bound).nan_to_num(9e9).max()), int((~(err <= bound)).sum()))


SHAPES = [  # lens, rows, query heads, cache heads, page
    ([0], [1], 4, 4, 16), ([1], [1], 1, 1, 1), ([31], [1], 8, 2, 16), ([32], [1], 7, 1, 8), ([700], [1], 4, 4, 64),
    ([0], [37], 4, 2, 16), ([5], [64], 2, 2, 3), ([63], [65], 2, 1, 256), ([100, 0, 33], [1, 40, 2], 6, 3, 16),
    ([300, 7, -1, 40], [3, 0, 5, 17], 4, 1, 5), ([0], [200], 5, 1, 16), ([129], [150], 2, 2, 16),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_attention(dtype, hd, case):
    lens, rows, Hq, H, page = SHAPES[case]
    check(dtype, lens, rows, Hq, H, hd, page, 10 * case + hd)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (33, 40), (64, 0), (100, 31), (127, 64), (5, 1000),
                                          (1 << 30, 3), (128, 129)])
def test_window(dtype, window, sinks):
    check(dtype, [0, 300, 61], [70, 1, 35], 4, 2, 64, 16, window + sinks, window, sinks)
    check(dtype, [500, 129], [1, 1], 6, 2, 128, 8, window + sinks, window, sinks, row0=None, behind=0)
    check(dtype, [250], [180], 2, 2, 128, 16, window + sinks, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_single_tokens_of_many_sequences(dtype):
    lens = [(37 * i) % 290 - 1 for i in range(150)]
    check(dtype, lens, [1] * 150, 4, 2, 64, 16, 3, row0=None, behind=0)
    check(dtype, lens, [1] * 150, 4, 2, 64, 16, 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [65, 300, 5000])
def test_ragged_rows_of_many_sequences(dtype, batch):
    """Most sequences without rows, some with one or a few, three with a chunk; where the
    cache is long the work is dealt in another way."""
    g = torch.Generator().manual_seed(batch)
    for far in (False, True):
        rows, lens = [0] * batch, torch.randint(0, 60, (batch,), generator=g).tolist()
        for i in torch.randint(0, batch, (60,), generator=g).tolist():
            rows[i] = 1 + i % 5
        rows[0], rows[batch // 2], rows[-1] = 40, 33, 150
        q, pool, table = attn_inputs(dtype, lens, rows, 4, 2, 64, 16, batch)
        got = attend(q, pool, table, lens, rows, dtype, 0.125, far=far)
        ref, mag, big = R.attention(q, pool, table, lens, rows, 0.125)
        assert bool(((got - ref).abs() <= R.attention_bound(dtype, ref, mag, big, 210, 64)).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales(dtype, scale):
    check(dtype, [90, 3], [1, 70], 4, 2, 64, 16, 5, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unaligned_output(dtype):
    check(dtype, [90, 3], [2, 70], 4, 2, 64, 16, 5, ldo=4 * 64 + 3)


def test_long_context_is_split():
    check("bf16", [5000], [1], 4, 1, 128, 16, 6)
    check("f32", [3000, 10], [2, 1], 4, 2, 64, 64, 6)
    check("bf16", [2500], [40], 2, 1, 128, 16, 7)
    check("bf16", [4000], [3], 4, 2, 64, 16, 7, 1500, 70)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, bad):
    """An infinity or NaN in K and V of one position, seen by some rows of a tile and
    not by others."""
    for lens, rows, at, window in (([40], [60], 70, 0), ([200], [9], 204, 0), ([100], [50], 100, 20), ([7], [3], 8, 2),
                                   ([300], [140], 310, 64)):
        q, pool, table = attn_inputs(dtype, lens, rows, 2, 1, 64, 16, 8)
        for kv in (0, 1):
            spoilt = pool.clone()
            spoilt[table[0, at // 16], kv, :, at % 16, 3] = bad
            got = attend(q, spoilt, table, lens, rows, dtype, 0.125, window)
            ref, mag, big = R.attention(q, spoilt, table, lens, rows, 0.125, window)
            p = lens[0] + torch.arange(rows[0])
            free = (p < at) | ((p >= at + window) if window else torch.zeros_like(p, dtype=torch.bool))
            assert bool(free.any()) and not bool(free.all())
            # The tile that holds it is summed in another way than it would be without it,
            # so its rows keep their values to the bound of any way of summing (the
            # reference sums what a row sees) and not to the bit.
            near = (got - ref).abs() <= R.attention_bound(dtype, ref, mag, big, 500, 64)
            assert bool(near[free].all())
            if kv == 1:  # a value: only its dimension, as the sum has it
                assert bool(near[~free][..., :3].all()) and bool(near[~free][..., 4:].all())
                assert bool((got[~free][..., 3].isnan() if math.isnan(bad) else got[~free][..., 3] == bad).all())
            elif math.isnan(bad):
                assert bool(got[~free].isnan().all())
            else:  # a score of -inf weighs nothing, one of +inf makes the row NaN
                up = q[~free][..., 3].double() * bad > 0
                assert bool(got[~free][up].isnan().all())
                ok = ~up & (q[~free][..., 3] != 0)
                bound = R.attention_bound(dtype, ref, mag, torch.zeros_like(big) + 60, 500, 64)[~free]
                assert bool(((got[~free] - ref[~free]).abs() <= bound)[ok].all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_attention_far(dtype, hd, case):
    lens, rows, Hq, H, page = SHAPES[case]
    check(dtype, lens, rows, Hq, H, hd, page, 10 * case + hd, far=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 1150), (64, 1086), (500, 650), (1000, 150), (1200, 128), (1 << 30, 3)])
def test_window_far(dtype, window, sinks):
    """Blocks of 128 queries whose first tiles and last ones lie apart, meet or overlap."""
    check(dtype, [800, 0, 1300], [600, 3, 90], 24, 3, 128, 16, window + sinks, window, sinks, far=True)
    check(dtype, [1200], [693], 24, 6, 128, 64, window + sinks, window, sinks, far=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_of_blocks_of_128(dtype):
    """Blocks whole, in two to eight parts and in more."""
    check(dtype, [4100], [40], 2, 1, 128, 16, 6, far=True)
    check(dtype, [3000, 900], [130, 1], 4, 2, 64, 64, 6, far=True)
    check(dtype, [2500], [500], 16, 16, 64, 16, 7, far=True)
    check(dtype, [2000, 0, 700], [20, 1, 300], 16, 16, 128, 16, 7, far=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_rows_than_positions_before_them(dtype):
    check(dtype, [100], [1000], 24, 8, 128, 16, 8)
    check(dtype, [30, 0, 5], [500, 700, 200], 64, 32, 64, 32, 8)
    check(dtype, [0], [1100], 40, 40, 64, 16, 8, 600, 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [17, 64])
def test_single_tokens_of_many_query_heads(dtype, heads):
    """More query heads a cache head than a block of 16 has rows."""
    for far in (False, True):
        check(dtype, [900, 0, 33], [1, 1, 1], heads, 1, 64, 16, heads, row0=None, behind=0, far=far)
        check(dtype, [900, 33], [2, 1], heads, 1, 128, 16, heads, far=far)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales_and_unaligned_output_far(dtype, scale):
    check(dtype, [90, 3], [1, 70], 4, 2, 64, 16, 5, scale=scale, far=True, ldo=4 * 64 + 3)
    check(dtype, [90], [70], 4, 2, 128, 16, 5, scale=scale, far=True, ldo=4 * 128 + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_reach_it_far(dtype, bad):
    """A value that is no number, behind the mask of some rows of a tile of 128."""
    for lens, rows, at in (([40], [160], 70), ([200], [9], 204), ([300], [140], 310), ([0], [200], 63)):
        for hd in (64, 128):
            q, pool, table = attn_inputs(dtype, lens, rows, 2, 1, hd, 16, 8)
            pool[table[0, at // 16], 1, :, at % 16, 3] = bad
            got = attend(q, pool, table, lens, rows, dtype, 0.125, far=True)
            ref, mag, big = R.attention(q, pool, table, lens, rows, 0.125)
            free = lens[0] + torch.arange(rows[0]) < at
            assert bool(free.any()) and not bool(free.all())
            near = (got - ref).abs() <= R.attention_bound(dtype, ref, mag, big, 500, hd)
            assert bool(near[free].all()) and bool(near[~free][..., :3].all()) and bool(near[~free][..., 4:].all())
            assert bool((got[~free][..., 3].isnan() if math.isnan(bad) else got[~free][..., 3] == bad).all())


def test_scores_past_the_range():
    """All scores -inf: NaN; some: they weigh nothing."""
    for rows in (1, 70):
        lens = [70]
        q, pool, table = attn_inputs("f32", lens, [rows], 2, 2, 64, 16, 9)
        q[..., 0] = 3e38
        pool[:, 0, :, :, 0] = -3e38
        got = attend(q, pool, table, lens, [rows], "f32", 0.125)
        assert bool(got.isnan().all())
        keep = int(table[0, 2])
        pool[keep, 0, :, :, 0] = 0.0
        got = attend(q, pool, table, lens, [rows], "f32", 0.125)
        assert bool(got.isfinite().all())
        part = pool[keep, 1].double().amax(1)
        assert bool((got.amax(0) <= part + 1e-5).all())


def test_positions_and_pages_that_are_not_there():
    lens, rows = [50, 20], [30, 1]
    for hd in (64, 128):
        q, pool, table = attn_inputs("f32", lens, rows, 4, 2, hd, 16, 11)
        pool = pool.nan_to_num(0.5)
        table[0, 1], table[0, 2], table[1, 0] = -1, 1 << 30, pool.shape[0]
        ref, mag, big = R.attention(q, pool, table, lens, rows, 0.125)
        for far in (False, True):
            got = attend(q, pool, table, lens, rows, "f32", 0.125, far=far)
            assert bool(((got - ref).abs() <= R.attention_bound("f32", ref, mag, big, 80, hd)).all())
        # a sequence with no page at all, and one past its table
        table[1] = -5
        got = attend(q, pool, table, [10000, 20], rows, "f32", 0.125, 5, 0)
        assert bool((got == 0).all())
        got = attend(q, pool, table, [10000, 20], rows, "f32", 0.125, 5, 7)
        assert bool((got[:30].abs().sum(-1) > 0).all()) and bool((got[30:] == 0).all())


def test_starts_that_leave_rows_out():
    """Rows before the first sequence and behind the last, empty sequences."""
    q, pool, table = attn_inputs("bf16", [20, 30, 5], [4, 0, 3], 2, 2, 64, 16, 12)
    dq = torch.zeros(20, 128, dtype=torch.bfloat16, device="cuda")
    dq[6:13] = q.reshape(7, -1).cuda()
    out = torch.full((20, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    starts = torch.tensor([6, 10, 10, 13], dtype=torch.int32, device="cuda")
    n = torch.tensor([20, 30, 5], dtype=torch.int32, device="cuda")
    dp, dt = pool.cuda(), table.cuda()
    c = cache_of(dp, dt, "bf16")
    nb = B.chimera_paged_attn_bytes(c, 2, 20)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    B.chimera_paged_attn(c, dq.data_ptr(), 128, 2, starts.data_ptr(), n.data_ptr(), 20, 0, 0, 0.125, out.data_ptr(),
                         128, ws.data_ptr(), nb, stream())
    ref, mag, big = R.attention(q, pool, table, [20, 30, 5], [4, 0, 3], 0.125)
    assert bool(((out[6:13].double().cpu().view(7, 2, 64) - ref).abs() <=
                 R.attention_bound("bf16", ref, mag, big, 40, 64)).all())
    assert bool((out[:6] == 7).all()) and bool((out[13:] == 7).all())


def test_equal_calls_give_equal_bits():
    q, pool, table = attn_inputs("bf16", [3000, 900], [70, 1], 4, 2, 128, 16, 13)
    a = attend(q, pool, table, [3000, 900], [70, 1], "bf16", 0.09)
    b = attend(q, pool, table, [3000, 900], [70, 1], "bf16", 0.09, far=True)
    for _ in range(3):
        assert torch.equal(a, attend(q, pool, table, [3000, 900], [70, 1], "bf16", 0.09))
        assert torch.equal(b, attend(q, pool, table, [3000, 900], [70, 1], "bf16", 0.09, far=True))


def test_offsets_past_32_bits():
    """The last pages of a pool of 5 GiB of bf16: element offsets past 2^31, byte
    offsets past 2^32."""
    n_pages, H, page, hd = 40960, 2, 128, 128
    pool = torch.empty(n_pages, 2, H, page, hd, dtype=torch.bfloat16, device="cuda")
    lens, rows = [200, 130], [3, 70]
    q, small, order = attn_inputs("bf16", lens, rows, 4, H, hd, page, 14)
    table = (n_pages - 1 - order).int()
    pool[table.flatten().long().cuda()] = small[order.flatten().long()].cuda()
    dq = q.reshape(73, -1).cuda()
    out = torch.empty_like(dq)
    starts = torch.tensor([0, 3, 73], dtype=torch.int32, device="cuda")
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    dt = table.cuda()
    c = cache_of(pool, dt, "bf16")
    nb = B.chimera_paged_attn_bytes(c, 4, 73)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    B.chimera_paged_attn(c, dq.data_ptr(), 512, 4, starts.data_ptr(), n.data_ptr(), 73, 0, 0, 0.088, out.data_ptr(), 512,
                         ws.data_ptr(), nb, stream())
    ref, mag, big = R.attention(q, small, order, lens, rows, R.f32(0.088))
    assert bool(((out.double().cpu().view(73, 4, hd) - ref).abs() <=
                 R.attention_bound("bf16", ref, mag, big, 203, hd)).all())
    # rows into them
    x = torch.randn(2, 3 * H * hd, device="cuda").bfloat16()
    seq, pos = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([5, 131], dtype=torch.int32,
                                                                                    device="cuda")
    p = x.data_ptr()
    B.chimera_paged_append(c, 1, None, p + 2 * H * hd, p + 4 * H * hd, 3 * H * hd, 0, seq.data_ptr(), pos.data_ptr(), 2,
                           None, None, None, None, 0.0, None, 0, stream())
    for r, (b, at) in enumerate([(0, 5), (1, 131)]):
        held = pool[int(table[b, at // page]), :, :, at % page]
        assert torch.equal(held.reshape(-1), x[r, H * hd:])


def test_numbers_at_the_ends_of_their_range():
    """Lengths, sequences and positions far outside: rows of zeros, rows left out."""
    lo, hi = -(1 << 31), (1 << 31) - 1
    q, pool, table = attn_inputs("bf16", [40, 3], [1, 1], 4, 2, 64, 16, 21, poison=False)
    for window, sinks in ((0, 0), (1 << 30, 0), (7, 1 << 30)):
        for rows in ([1, 1], [3, 40]):
            got = attend(q[:1].expand(sum(rows), 4, 64).contiguous(), pool, table, [lo, -7], rows, "bf16", 0.125, window,
                         sinks)
            assert bool((got == 0).all())
    # past the table: all that it has is seen
    for far in (False, True):
        got = attend(q, pool, table, [1 << 30, 3], [1, 1], "bf16", 0.125, far=far)
        cap = table.shape[1] * 16
        ref, mag, big = R.attention(q, pool, table, [cap - 1, 3], [1, 1], 0.125)
        assert bool(((got - ref).abs() <= R.attention_bound("bf16", ref, mag, big, cap, 64)).all())
    dp, dt = pool.cuda(), table.cuda()
    before, x = dp.clone(), torch.randn(6, 8 * 64, device="cuda").bfloat16()
    out = torch.full((6, 256), 3.0, dtype=torch.bfloat16, device="cuda")
    seq = torch.tensor([lo, hi, 0, 0, 2, -1], dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 0, lo, hi, 0, 5], dtype=torch.int32, device="cuda")
    p = x.data_ptr()
    for rope in (None, "half"):
        r, rt, _ = rope_of(ROPES[rope], 64, 50) if rope else (None, None, None)
        B.chimera_paged_append(cache_of(dp, dt, "bf16"), B.CHIMERA_BF16, p, p + 512, p + 768, 512, 4, seq.data_ptr(),
                               pos.data_ptr(), 6, r, rt.data_ptr() if rope else None, None, None, 0.0, out.data_ptr(),
                               256, stream())
        assert torch.equal(dp, before) and bool((out == 3).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_thousand_query_heads(dtype):
    check(dtype, [50, 0], [1, 1], 1024, 1, 64, 16, 22, row0=None, behind=0)
    check(dtype, [50, 9], [1, 2], 1000, 8, 128, 16, 22)
    check(dtype, [30], [2], 1024, 1024, 64, 4, 22)


def test_a_captured_call_follows_the_device():
    """Lengths, rows and pages change between replays; the call's shape does not."""
    for dtype, hd, total, cap in (("bf16", 128, 300, 600), ("f32", 64, 40, 200), ("bf16", 64, 7, 5000)):
        g = torch.Generator().manual_seed(total)
        page, batch, Hq, H = 16, 5, 4, 2
        table, n_pages = table_of(g, batch, cap, page)
        pool = torch.randn(n_pages, 2, H, page, hd, generator=g).to(R.TYPES[dtype])
        dq = torch.zeros(total, Hq * hd, dtype=R.TYPES[dtype], device="cuda")
        out = torch.zeros_like(dq)
        dt, dp = table.cuda(), pool.cuda()
        n = torch.zeros(batch, dtype=torch.int32, device="cuda")
        starts = torch.zeros(batch + 1, dtype=torch.int32, device="cuda")
        c = cache_of(dp, dt, dtype)
        nb = B.chimera_paged_attn_bytes(c, Hq, total)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")

        def call():
            B.chimera_paged_attn(c, dq.data_ptr(), Hq * hd, Hq, starts.data_ptr(), n.data_ptr(), total, 0, 0, 0.1,
                                 out.data_ptr(), Hq * hd, ws.data_ptr(), nb, stream())

        graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            call()
        for i in range(4):
            cuts = sorted(torch.randint(0, total + 1, (batch - 1,), generator=g).tolist())
            rows = [b - a for a, b in zip([0] + cuts, cuts + [total])]
            lens = [int(torch.randint(0, max(cap - r, 1), (1,), generator=g)) for r in rows]
            order = torch.randperm(n_pages, generator=g)[:table.numel()].view(table.shape).int()
            q = torch.randn(total, Hq, hd, generator=g).to(R.TYPES[dtype])
            dq.copy_(q.reshape(total, -1))
            dt.copy_(order)
            n.copy_(torch.tensor(lens))
            starts.copy_(torch.tensor([0] + cuts + [total]))
            out.fill_(7.0)
            ws.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            ref, mag, big = R.attention(q, pool, order, lens, rows, R.f32(0.1))
            bound = R.attention_bound(dtype, ref, mag, big, cap + total, hd)
            assert bool(((got.double().cpu().view(total, Hq, hd) - ref).abs() <= bound).all())
            call()
            torch.cuda.synchronize()
            assert torch.equal(got, out)
