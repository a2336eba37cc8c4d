"""Rotary positions against the plain 64-bit form."""
import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import U, inside, rope_frequencies, rope_plain, starts_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
SCALINGS = {"none": {}, "linear": dict(factor=4.0), "bands": dict(factor=8.0, low=1.0, high=4.0, original=8192),
            "ramp": dict(factor=16.0, low=1.0, high=32.0, original=4096, amplitude=1.2772588722239782)}


def draw(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def doc_positions(starts, n):
    pos, rows = torch.arange(n), torch.zeros(n, dtype=torch.bool)
    for lo, hi in zip(starts[:-1], starts[1:]):
        pos[lo:hi] = torch.arange(hi - lo)
        rows[lo:hi] = True
    return pos, rows


def check(got, x, pos, d, rot, layout, scaling, inverse, rows=None, fill=None, base=5e5):
    kw = SCALINGS[scaling]
    y, bound = rope_plain(x.double(), pos, rot, layout, rope_frequencies(rot, base, scaling, **kw),
                          kw.get("amplitude", 1.0), inverse)
    if x.dtype == BF16:
        bound = bound * (1 + U) + U * y.abs()
    rows = torch.ones(x.shape[0], dtype=torch.bool) if rows is None else rows
    got = got.cpu()
    inside("y", got[rows], y[rows], bound[rows])
    assert torch.equal(got[..., rot:][rows], x[..., rot:][rows])
    if fill is not None:
        assert bool((got[~rows] == fill).all())


CASES = [  # n, heads, kv, d, rot, layout, scaling, dtype, inverse
    (1, 1, 1, 64, 64, "half", "none", BF16, False),
    (3, 4, 2, 128, 128, "half", "bands", BF16, True),
    (65, 32, 8, 128, 128, "interleaved", "bands", BF16, False),
    (50, 5, 3, 128, 48, "half", "ramp", BF16, False),
    (50, 5, 3, 128, 48, "interleaved", "ramp", F32, True),
    (130, 2, 1, 64, 2, "half", "linear", F32, False),
    (17, 3, 1, 80, 20, "half", "none", BF16, False),       # no multiple of 16
    (17, 3, 1, 66, 66, "interleaved", "linear", BF16, True),
    (9, 2, 2, 512, 512, "half", "none", F32, False),       # the largest head
    (2050, 16, 4, 64, 32, "half", "bands", BF16, False),
    (2, 8192, 1, 512, 2, "half", "none", BF16, False),     # the most units per row, in pairs and single elements
]


@pytest.mark.parametrize("n,a,g,d,rot,layout,scaling,dtype,inverse", CASES)
def test_matches_the_plain_form(n, a, g, d, rot, layout, scaling, dtype, inverse):
    q, k = draw((n, a, d), n, dtype), draw((n, g, d), n + 1, dtype)
    starts = starts_of([n // 3, 0, n // 2 - n // 3], n // 9)
    pos, rows = doc_positions(starts, n)
    far = torch.randint(-(1 << 20), 1 << 20, (n,), generator=torch.Generator().manual_seed(n))
    rope = L.make_rope(d, rot, layout, 5e5, scaling, **SCALINGS[scaling])
    call = L.rope_bwd if inverse else L.rope_fwd
    pk = L.make_packing(torch.tensor(starts, device="cuda"), n)
    for packing, positions, at, inside_rows in ((pk, None, pos, rows), (None, None, torch.arange(n), None),
                                                (None, far, far, None), (pk, far, far, rows)):
        qo, ko = torch.full_like(q, 3.0).cuda(), torch.full_like(k, 3.0).cuda()
        call(rope, q.cuda(), qo, k.cuda(), ko, positions=None if positions is None else positions.cuda(),
             packing=packing)
        check(qo, q, at, d, rot, layout, scaling, inverse, inside_rows, 3.0)
        check(ko, k, at, d, rot, layout, scaling, inverse, inside_rows, 3.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_in_place_on_columns_of_a_fused_array(dtype, offset):
    """q and k as columns of one array at any alignment; what is beside them stays."""
    n, a, g, d, rot = 70, 4, 2, 64, 32
    wide = draw((n, (a + 2 * g) * d + 8 + offset), 5, dtype)
    dev = wide.cuda()
    views = [t[:, offset:offset + (a + g) * d].unflatten(1, (a + g, d)) for t in (wide, dev)]
    rope = L.make_rope(d, rot, "half", 5e5)
    L.rope_fwd(rope, views[1][:, :a], None, views[1][:, a:])
    check(views[1], views[0], torch.arange(n), d, rot, "half", "none", False)
    left = torch.ones(wide.shape[1], dtype=torch.bool)
    left[offset:offset + (a + g) * d] = False
    assert torch.equal(dev.cpu()[:, left], wide[:, left])


def test_backward_undoes_and_is_the_transpose():
    n, a, d = 40, 3, 128
    rope = L.make_rope(d, 96, "interleaved", 5e5, "ramp", **SCALINGS["ramp"])
    x, y = draw((n, a, d), 1, F32).cuda(), draw((n, a, d), 2, F32).cuda()
    fx, by = torch.empty_like(x), torch.empty_like(y)
    L.rope_fwd(rope, x, fx)
    L.rope_bwd(rope, y, by)
    left, right = (fx.double() * y.double()).sum(), (x.double() * by.double()).sum()
    # <R x, y> = <x, R' y>: each product within 8 F A (|x0| + |x1|) of the exact one
    assert abs(float(left - right)) <= 2 ** -20 * float((fx.abs().double() * y.abs().double()).sum() * 2)


def test_bad_rows_stay_where_they_are():
    n, a, d = 12, 2, 64
    x = draw((n, a, d), 3, BF16)
    x[5] = float("nan")
    rope = L.make_rope(d)
    out = torch.zeros_like(x).cuda()
    L.rope_fwd(rope, x.cuda(), out, packing=L.make_packing(torch.tensor([0, 5], device="cuda"), n))
    assert bool((out[5:] == 0).all()) and bool(torch.isfinite(out[:5]).all())


def test_captured_and_replayed_on_a_side_stream():
    n, a, d = 100, 4, 128
    x, out = draw((n, a, d), 3, BF16).cuda(), torch.zeros(n, a, d, dtype=BF16, device="cuda")
    rope, graph = L.make_rope(d, 64), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        L.rope_fwd(rope, x, out)
    for seed in (4, 5, 6):
        new = draw((n, a, d), seed, BF16)
        x.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        check(out, new, torch.arange(n), d, 64, "half", "none", False, base=1e4)
