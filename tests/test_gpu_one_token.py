"""The block around the attention over documents of one token: the kernels' gradients of q, k and the gains.

One visible key has probability 1 whatever q and k are, so their exact gradients are 0, and what
the kernels return is rounding alone, bounded here."""
import math

import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import F, U
from test_gpu_attention_block import A, D, EPS, G, Step
from test_gpu_qk_norm import pair_sum

pytestmark = pytest.mark.gpu


def rotated_bounds(q, k, v, o, g):
    """Bounds on dq [n][A][D] and dk [n][G][D] of documents of one token: all float64, o as stored."""
    scale, group = 1.0 / math.sqrt(D), A // G
    ke, ve = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    # the score in fp32 (products, sum, scale, base 2) in both passes, and the stored log-sum-exp: |1 - P|
    s, size = (q * ke).sum(-1).abs() * scale, (q * ke).abs().sum(-1) * scale
    e_s = (D + 8) * F * size + 4 * F * s
    e_p = 2 * (2 * e_s + 9 * F) + e_s + 9 * F + 4 * F * s
    # dP and delta = sum dO o: products and sums in fp32; o is v off by P's error and rounding, and its own
    e_dp = (D + 2) * F * (g * ve).abs().sum(-1)
    e_delta = (D + 2) * F * (g * o).abs().sum(-1)
    apart = (g * ve - g * o).abs().sum(-1) + e_dp + e_delta                  # dP - delta
    # the dQ pass adds P (dP - delta) to delta: what is left is (1 - P) of it and three roundings
    left = apart * (e_p + 3 * F)
    ds = (1 + e_p) * left
    dq = (scale * (1 + U) * (1 + U) * (1 + 4 * F) * ds)[..., None] * ke.abs()
    # dK/dV forms dP again and reads the corrected delta
    ds = (1 + e_p) * (2 * e_dp + left + 2 * F * (g * ve).abs().sum(-1) + 2 * F * (g * o).abs().sum(-1))
    dk = (scale * (1 + U) * (1 + U) * (1 + (4 + group) * F) * ds)[..., None] * q.abs()
    return dq, dk.unflatten(1, (G, group)).sum(2)


@pytest.mark.parametrize("n,starts", [(1, [0, 1]), (5, [0, 1, 1, 2, 3, 4]), (70, list(range(71)))])
def test_gradients_of_q_k_and_the_gains(n, starts):
    s = Step(n, 3, starts)
    s.run()
    rows = starts[-1]

    def f64(t, i, j):
        return s.heads(t, i, j)[:rows].cpu().double()

    q, k, v = f64(s.rot, 0, A), f64(s.rot, A, A + G), f64(s.qkv, A + G, A + 2 * G)
    o, g = (t.unflatten(1, (A, D))[:rows].cpu().double() for t in (s.o, s.d_o))
    bounds = rotated_bounds(q, k, v, o, g)
    size = float((g * v.repeat_interleave(A // G, 1)).sum(-1).abs().max()) / math.sqrt(D)      # dP without delta
    for name, b, (i, j), gain, dg in (("q", bounds[0], (0, A), s.gq, s.dgq), ("k", bounds[1], (A, A + G), s.gk, s.dgk)):
        assert float(b.max()) < 2e-3 * size                                  # far below a gradient that does not cancel
        got = f64(s.d_rot, i, j)
        assert bool((got.abs() <= b).all()), name
        # behind the norm: dx = r (dn g - x r mean(dn g x r)), dn the rotated-back gradient
        x, w = f64(s.qkv, i, j), gain.cpu().double().abs()
        r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
        dn, xr = (1 + 8 * F) * pair_sum(b, D, "half"), (x * r).abs()
        dx = (1 + U) * (1 + 4 * (D + 10) * F) * r * (dn * w + xr * (dn * w * xr).mean(-1, keepdim=True))
        assert bool((f64(s.d_qkv, i, j).abs() <= dx).all()), name
        sums = (1 + (D + 10 + x.shape[0] * x.shape[1]) * F) * (dn * xr).sum((0, 1))
        assert bool((dg.cpu().double().abs() <= sums).all()), name
        assert not s.heads(s.d_qkv, i, j)[rows:].any()
