"""Norms of heads at the ends of the number range: squares and products that pass fp32."""
import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import inside, rope_frequencies
from test_gpu_qk_norm import BASE, arena, make, norm_plain, step_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def run(x, gain, dy, eps=1e-6):
    n, _, d = x.shape
    y, dx, dg = torch.full_like(x, 7.0), torch.full_like(x, 7.0), torch.zeros(d, device="cuda")
    rope = L.make_rope(d, base=BASE)
    L.qk_norm_rope_fwd(rope, x, gain, y, eps=eps)
    L.qk_norm_rope_bwd(rope, x, gain, dy, dx, dg, arena(n, d), eps=eps)
    return y, dx, dg


@pytest.mark.parametrize("d", [128, 50, 198])            # whole vectors, single pairs, two of them a lane
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_heads_whose_squares_pass_fp32_give_zeros(d, dtype):
    """r is 0 there: so are y and dx, and the gain's gradient is that of the other heads."""
    n, a = 20, 3
    x = make(n, a, 1, d, dtype, 5)
    gain, dy = x["gq"].cuda(), x["dq"].cuda() * 3
    rows = {3: torch.finfo(dtype).max, 9: -2.0 ** 100, 11: 2.0 ** 64}        # 2^64 squared is 2^128, the first that passes
    many = x["q"].cuda()
    for row, v in rows.items():
        many[row] = v
    many[15, 1, 0] = 1e30                                                    # one element of a head
    y, dx, dg = run(many, gain, dy)
    assert bool(torch.isfinite(dg).all())
    for row in rows:
        assert bool((y[row] == 0).all()) and bool((dx[row] == 0).all()), row
    assert bool((y[15, 1] == 0).all()) and bool((dx[15, 1] == 0).all())
    # the same without those heads' part: ordinary x under dy = 0
    plain, none = x["q"].cuda(), dy.clone()
    none[list(rows)] = 0.0
    none[15, 1] = 0.0
    want = run(plain, gain, none)
    keep = torch.ones((n, a), dtype=torch.bool)
    keep[list(rows)] = False
    keep[15, 1] = False
    keep = keep.cuda()
    assert torch.equal(y[keep], want[0][keep]) and torch.equal(dx[keep], want[1][keep]) and torch.equal(dg, want[2])


@pytest.mark.parametrize("d", [128, 50])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size,grad", [(1e16, 1e26), (1e-9, 1e26), (1e16, 1e-10)])
def test_products_of_large_values_and_gradients(d, dtype, size, grad):
    """x dy passes fp32 (1e42), or x is far below the root of eps: the gradients are those of the formula."""
    n, a, eps = 30, 4, 1e-20
    x = make(n, a, 1, d, dtype, 6)
    q, dy, gain = (x["q"] * size), (x["dq"] * grad), x["gq"]
    table, pos = [(0, f) for f in rope_frequencies(d, BASE)], torch.arange(n)[None]
    y, dx, dg = run(q.cuda(), gain.cuda(), dy.cuda(), eps)
    want = norm_plain(q.double(), gain.double(), table, pos, d, "half", eps, dy.double())
    s = step_of(dtype)
    assert float(want["dx"].abs().max()) < 1e37 and float(want["dg"].abs().max()) < 1e37
    inside("y", y.cpu(), want["y"], (1 + s) * want["_y"] + s * want["y"].abs())
    inside("dx", dx.cpu(), want["dx"], (1 + s) * want["_dx"] + s * want["dx"].abs())
    inside("dg", dg.cpu(), want["dg"], want["_dg"])
