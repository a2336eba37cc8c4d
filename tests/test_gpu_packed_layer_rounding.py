"""The packed layer's attention gradients: rounded to bf16 once, after they are turned back,
and right where some blocks of keys are cut and others are not."""
import math

import numpy as np
import pytest
import torch

import paper_2411_06465_amd as L
import test_gpu_packed_layer as P
import workloads as W
from gpu_common import Buffers, host_f64
from oracle.bf16 import from_bits, round_bf16
from packed_common import starts_of

pytestmark = pytest.mark.gpu

# Documents of at most 7 rows: every row has a probability of at least 1/7, so P and dS enter
# the products in two bf16 parts.
LENS = [7, 5, 1, 6, 3, 7, 2, 4, 6, 7, 5, 3, 7, 1]

CASES = {   # slices of the query heads (the sum of their parts stores dK) and whole ones, both head sizes
    "d64-slices": W.TINY,
    "d64": W.LayerWorkload("packed-mha64", 256, 4, 4, 688, 0),
    "d128-slices": W.LayerWorkload("packed-d128", 1024, 8, 2, 1376, 0, rope_base=5e5),
    "d128": W.LayerWorkload("packed-mha", 512, 4, 4, 768, 0),
}


def attention_gradients(q, k, v, d_o, starts, base):
    """float64 gradients of causal attention within documents with respect to q and k before
    their rotation (half layout, plain angles) and to v; [rows][heads][d]."""
    (n, a, d), g = q.shape, k.shape[1]
    out = [np.zeros_like(x) for x in (q, k, v)]
    angle = np.concatenate([np.arange(hi - lo) for lo, hi in zip(starts[:-1], starts[1:])])[:, None] * \
        base ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    for lo, hi in zip(starts[:-1], starts[1:]):
        for h in range(a):
            Q, K, V, G = q[lo:hi, h], k[lo:hi, h * g // a], v[lo:hi, h * g // a], d_o[lo:hi, h]
            score = np.where(np.tri(hi - lo, dtype=bool), Q @ K.T / math.sqrt(d), -np.inf)
            p = np.exp(score - score.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            dp = G @ V.T
            ds = p * (dp - (p * dp).sum(-1, keepdims=True)) / math.sqrt(d)
            out[0][lo:hi, h] = ds @ K
            out[1][lo:hi, h * g // a] += ds.T @ Q
            out[2][lo:hi, h * g // a] += p.T @ G
    for x in out[:2]:
        x0, x1 = x[..., :d // 2].copy(), x[..., d // 2:].copy()
        x[..., :d // 2], x[..., d // 2:] = x0 * c + x1 * s, x1 * c - x0 * s
    return out


@pytest.mark.parametrize("name", list(CASES))
def test_one_rounding_of_the_gradients_of_q_k_and_v(name):
    """The gradient of [Q|K|V] is read back from the layer's weight gradient (dQKV^T xn1, with fewer rows
    than columns and so solvable for dQKV; the gradient of the attention's output the same way from the
    output projection's) and compared with the rounding of the 64-bit gradients.

    Rounded once, an element differs only where its own error before the rounding, relative e, takes
    it across the middle of two bf16 values: for a fraction of e / 2^-9 at most.  P and dS in two parts leave
    2^-16, fp32 sums of 7 and scores of 128 products 2^-17 each, a few elements of the attention's output
    gradient rounded the other way 2^-14 on average: under 2^-13 altogether, 1/16 of the elements.
    A second rounding is off by a quarter of a step on average, which is a quarter of them."""
    starts = starts_of(LENS)
    n = starts[-1]
    w = CASES[name].replace(name=f"{name}-rounding", seq=n)
    buf = Buffers(w)
    a, g, d = w.a_t, w.k_t, w.d_h
    pk = L.make_packing(torch.tensor(starts, device="cuda"), n)
    st = L.llama_layer_packed_fwd(buf.model, buf.par, buf.weights, buf.x, buf.y, buf.arena, pk)
    x = {t: host_f64(buf.stash_view(st, t, (n, cols)))
         for t, cols in (("xn1", w.hidden), ("q", a * d), ("k", g * d), ("v", g * d), ("ctx", a * d))}
    L.llama_layer_packed_bwd(buf.model, buf.par, buf.weights, st, buf.dy, buf.dx, buf.grads, buf.arena, pk)
    torch.cuda.synchronize()
    got = (host_f64(buf.grads["qkv"]) @ np.linalg.pinv(x["xn1"])).T
    d_h1 = round_bf16((host_f64(buf.grads["o"]) @ np.linalg.pinv(x["ctx"])).T)
    d_ctx = round_bf16(d_h1 @ from_bits(buf.wbits["o"]).reshape(w.hidden, a * d))
    want = attention_gradients(*(x[t].reshape(n, -1, d) for t in "qkv"), d_ctx.reshape(n, a, d), starts, w.rope_base)
    assert got.shape == (n, (a + 2 * g) * d)
    at, off = 0, {}
    for t, y in zip("qkv", want):
        y = y.reshape(n, -1)
        mine = got[:, at:at + y.shape[1]]
        at += y.shape[1]
        assert np.linalg.norm(mine - y) <= 2.0 ** -8 * np.linalg.norm(y), t
        some = np.abs(y) > 1e-2 * np.sqrt((y ** 2).mean())       # smaller ones are lost in the solution
        off[t] = float((round_bf16(mine) != round_bf16(y))[some].mean())
    print({t: round(v, 4) for t, v in off.items()}, flush=True)
    assert all(v <= 0.1 for v in off.values()), off


MIXED = {   # enough blocks that only those with many tiles are cut: one document's first ones; 20 query heads per kv head
    "cut-and-whole": (W.LayerWorkload("packed-mixed", 512, 8, 4, 688, 0), [1300] + [1, 5, 3, 0, 2] * 26, 9),
    "20-1": (W.LayerWorkload("packed-20-1", 1280, 20, 1, 688, 0), [100] * 9 + [0] * 520, 3),
}


@pytest.mark.parametrize("name", list(MIXED))
def test_blocks_cut_and_whole(name, monkeypatch):
    monkeypatch.setitem(P.CASES, name, MIXED[name])
    P.test_documents_match_the_oracle(name, 1.0)
