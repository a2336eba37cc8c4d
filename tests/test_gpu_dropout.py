"""Dropout in front of the residual sum against a plain form: the mask exactly, the values within one rounding."""
import math

import numpy as np
import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import F, U, inside

BF16, F32 = torch.bfloat16, torch.float32
MASK = 0xffffffff


def philox(counter, key):
    """Philox4x32-10 in Python integers: four 32-bit words of a 128-bit counter and a 64-bit key."""
    x, k = [counter >> 32 * i & MASK for i in range(4)], [key & MASK, key >> 32 & MASK]
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [b >> 32 ^ x[1] ^ k[0], b & MASK, a >> 32 ^ x[3] ^ k[1], a & MASK]
        k = [k[0] + 0x9E3779B9 & MASK, k[1] + 0xBB67AE85 & MASK]
    return x


def kept(rows, cols, p, seed, offset, first_row=0):
    """The mask [rows][cols], element by element."""
    out = np.zeros(rows * cols, dtype=bool)
    first, t, last, words = first_row * cols, round(p * 2 ** 32), -1, None
    for i in range(rows * cols):
        if (first + i) // 4 != last:
            last = (first + i) // 4
            words = philox(last | (offset & 2 ** 64 - 1) << 64, seed & 2 ** 64 - 1)
        out[i] = words[(first + i) % 4] >= t
    return torch.from_numpy(out).view(rows, cols)


def test_the_plain_generator_gives_the_published_words():
    """The known answers that its authors publish for counter and key of all zeros, all ones, and digits of pi."""
    assert philox(0, 0) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert philox(2 ** 128 - 1, 2 ** 64 - 1) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    counter = 0x243f6a88 | 0x85a308d3 << 32 | 0x13198a2e << 64 | 0x03707344 << 96
    assert philox(counter, 0xa4093822 | 0x299f31d0 << 32) == [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def words(seed, offset):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def draw(rows, cols, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((rows, cols), generator=g).to(dtype) for _ in range(3)]


def check(got, x, res, keep, p, dtype):
    s = U if dtype == BF16 else F
    part = torch.where(keep, x.double() / (1 - p), torch.zeros((), dtype=torch.float64))
    want = part if res is None else part + res.double()
    # the scale, the product and the sum in fp32, then one rounding
    bound = 3 * F * (part.abs() + want.abs())
    inside("y", got, want, (1 + s) * bound + s * want.abs())
    dropped = (torch.zeros_like(x) if res is None else res)[~keep]
    assert torch.equal(got.cpu()[~keep], dropped)


CASES = [  # rows, cols, dtype, p, first row, seed, offset
    (1, 1, BF16, 0.5, 0, 0, 0),
    (1, 8, BF16, 0.1, 0, 1, 2),
    (3, 5, F32, 0.5, 0, 5, 1),
    (3, 5, BF16, 0.5, 7, -5, -1),                       # a counter shared by rows, and cut by the first one
    (33, 256, BF16, 0.1, 0, 1 << 62, 1 << 40),
    (33, 256, F32, 0.0, 0, 3, 0),
    (20, 136, F32, 0.9, 3, -(1 << 63), (1 << 63) - 1),
    (7, 1023, F32, 0.35, 0, 9, 9),
    (7, 1023, BF16, 0.35, 1 << 33, 9, 9),
    (64, 4, BF16, 0.5, 1, 9, 9),
    (33, 101, F32, 0.5, 1, 9, 9),                       # units that start 1, 2 and 3 places into a counter
    (33, 102, BF16, 0.5, 1, 9, 9),
    (33, 103, BF16, 0.5, 1, 9, 9),
    (5, 1000, BF16, 1.0 - 2.0 ** -31, 0, 9, 9),         # all but one in 2^31 dropped
    (3, 2048, BF16, 0.25, (1 << 38) - 1, 11, 4),        # counters of more than 32 bits
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,dtype,p,first,seed,offset", CASES)
def test_matches_the_plain_form(rows, cols, dtype, p, first, seed, offset):
    x, res, dy = draw(rows, cols, dtype, rows * cols)
    keep = kept(rows, cols, p, seed, offset, first)
    rng = words(seed, offset)
    for r in (res, None):
        y = torch.full((rows, cols), 7.0, dtype=dtype, device="cuda")
        L.dropout_add_fwd(x.cuda(), None if r is None else r.cuda(), y, rng, p, first_row=first)
        check(y, x, r, keep, p, dtype)
    dx = torch.full((rows, cols), 7.0, dtype=dtype, device="cuda")
    L.dropout_add_bwd(dy.cuda(), dx, rng, p, first_row=first)
    check(dx, dy, None, keep, p, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("cols,pad,shift", [(64, 8, 0), (64, 3, 0), (72, 0, 1), (7, 2, 0), (4096, 64, 0)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_rows_and_odd_addresses_have_the_same_mask(cols, pad, shift, dtype):
    rows, p, rng = 19, 0.3, words(4, 5)
    x, res, _ = draw(rows, cols, dtype, 2)
    want = torch.zeros((rows, cols), dtype=dtype, device="cuda")
    L.dropout_add_fwd(x.cuda(), res.cuda(), want, rng, p)

    def place(t):
        flat = torch.full((rows * (cols + pad) + shift,), 7.0, dtype=dtype, device="cuda")[shift:]
        flat.view(rows, cols + pad)[:, :cols].copy_(t)
        return flat.view(rows, cols + pad)

    y = place(torch.zeros_like(x))
    L.dropout_add_fwd(place(x)[:, :cols], place(res)[:, :cols], y[:, :cols], rng, p)
    assert torch.equal(y[:, :cols], want) and bool((y[:, cols:] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [64, 37])
def test_parts_of_the_rows_draw_from_one_mask(cols):
    """Ranks that hold parts of the rows: together the whole call."""
    x, res, _ = (t.cuda() for t in draw(50, cols, BF16, 3))
    rng, whole, parts = words(8, 1), torch.zeros_like(x), torch.zeros_like(x)
    L.dropout_add_fwd(x, res, whole, rng, 0.5)
    for lo, hi in ((0, 13), (13, 14), (14, 14), (14, 50)):
        L.dropout_add_fwd(x[lo:hi], res[lo:hi], parts[lo:hi], rng, 0.5, first_row=lo)
    assert torch.equal(whole, parts)


@pytest.mark.gpu
def test_dropped_elements_are_not_used_and_in_place_calls_agree():
    rows, cols, p, rng = 40, 128, 0.5, words(1, 2)
    x, res, dy = draw(rows, cols, BF16, 7)
    keep = kept(rows, cols, p, 1, 2)
    clean = torch.zeros((rows, cols), dtype=BF16, device="cuda")
    L.dropout_add_fwd(x.cuda(), res.cuda(), clean, rng, p)
    for bad in (math.nan, math.inf, -math.inf):
        xb = x.clone()
        xb[~keep] = bad
        y = torch.zeros_like(clean)
        L.dropout_add_fwd(xb.cuda(), res.cuda(), y, rng, p)
        assert torch.equal(y, clean)
    on_x, on_res = x.cuda(), res.cuda()
    L.dropout_add_fwd(on_x, res.cuda(), on_x, rng, p)
    L.dropout_add_fwd(x.cuda(), on_res, on_res, rng, p)
    assert torch.equal(on_x, clean) and torch.equal(on_res, clean)
    dx, on_dy = torch.zeros_like(clean), dy.cuda()
    L.dropout_add_bwd(dy.cuda(), dx, rng, p)
    L.dropout_add_bwd(on_dy, on_dy, rng, p)
    assert torch.equal(dx, on_dy)


@pytest.mark.gpu
def test_the_share_kept_and_other_offsets():
    """Of 2^22 elements the share kept is p off by less than 6 standard deviations; other offsets are other masks."""
    n, cols = 1 << 22, 1024
    x = torch.ones((n // cols, cols), device="cuda")
    masks = []
    for offset in (0, 1):
        y = torch.zeros_like(x)
        L.dropout_add_fwd(x, None, y, words(3, offset), 0.2)
        masks.append(y != 0)
        share = float(masks[-1].double().mean())
        assert abs(share - 0.8) <= 6 * math.sqrt(0.2 * 0.8 / n), share
    both = float((masks[0] & masks[1]).double().mean())
    assert abs(both - 0.64) <= 6 * math.sqrt(0.64 * 0.36 / n), both


@pytest.mark.gpu
def test_the_gradient_is_that_of_the_forward():
    """The forward is linear in x: <fwd(x), dy> = <x, bwd(dy)>, to the rounding of its terms."""
    rows, cols, p, rng = 33, 520, 0.4, words(12, 1)
    x, _, dy = (t.cuda() for t in draw(rows, cols, F32, 1))
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    L.dropout_add_fwd(x, None, y, rng, p)
    L.dropout_add_bwd(dy, dx, rng, p)
    a, b = (y.double() * dy.double()), (x.double() * dx.double())
    # each term is off by two roundings on either side
    assert float((a.sum() - b.sum()).abs()) <= 4 * F * float(a.abs().sum())


@pytest.mark.gpu
def test_captured_and_replayed_with_other_offsets():
    x, res, dy = (t.cuda() for t in draw(70, 256, BF16, 1))
    rng, y, dx = words(3, 0), torch.zeros((70, 256), dtype=BF16, device="cuda"), torch.zeros((70, 256), dtype=BF16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    L.dropout_add_fwd(x, res, y, rng, 0.5)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        L.dropout_add_fwd(x, res, y, rng, 0.5)
        L.dropout_add_bwd(dy, dx, rng, 0.5)
    seen = []
    for offset in (5, 6, 7):
        rng[1] = offset
        graph.replay()
        torch.cuda.synchronize()
        want, wx = torch.zeros_like(y), torch.zeros_like(dx)
        L.dropout_add_fwd(x, res, want, words(3, offset), 0.5)
        L.dropout_add_bwd(dy, wx, words(3, offset), 0.5)
        assert torch.equal(y, want) and torch.equal(dx, wx)
        seen.append(y.clone())
    assert not torch.equal(seen[0], seen[1])


@pytest.mark.gpu
def test_more_than_2_to_32_elements_of_counters():
    """The last rows of an array whose places pass 2^32 have the words of those places."""
    rows, cols = 1 << 17, 1 << 15
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 18 GB")
    x = torch.ones((rows + 1, cols), dtype=BF16, device="cuda")
    y = torch.zeros_like(x)
    rng = words(2, 3)
    L.dropout_add_fwd(x, None, y, rng, 0.5)
    last = torch.zeros((2, cols), dtype=BF16, device="cuda")
    L.dropout_add_fwd(x[rows - 1:], None, last, rng, 0.5, first_row=rows - 1)
    assert torch.equal(y[rows - 1:], last)
    assert torch.equal((last[1:, :64] != 0).cpu(), kept(1, cols, 0.5, 2, 3, rows)[:, :64])
