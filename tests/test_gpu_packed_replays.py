"""Packed operators captured once and replayed with other documents in the array of starts,
and the rounding of gradients of short documents."""
import math

import numpy as np
import pytest
import torch

import paper_2411_06465_amd as L
import workloads as W
from gpu_common import Buffers
from oracle.bf16 import round_bf16
from packed_common import starts_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def many_starts(n, docs, seed):
    """Documents that fill n rows or less, in very different ways."""
    g = torch.Generator().manual_seed(seed)
    cut = torch.sort(torch.randint(0, n + 1, (docs - 1,), generator=g))[0].tolist()
    yield [0] + cut + [n]                                                 # as they fall
    short = [1 + i % 3 for i in range(docs - 1)]
    long = n - 7 - sum(short)
    yield starts_of(short[:docs // 2] + [long] + short[docs // 2:], 5)    # one with nearly all rows
    yield starts_of([n // docs] * docs, n % docs)                         # equal ones, rows before the first
    yield [n // 3] * docs + [2 * n // 3]                                  # only the last holds rows
    yield [n // 2] * (docs + 1)                                           # none does


ATTENTION = {  # rows, documents, heads, kv heads, d: below and above 64 documents, all blocks cut, some cut
    "few": (700, 5, 8, 2, 128),
    "63": (900, 63, 4, 2, 64),
    "64": (900, 64, 4, 2, 64),
    "some-cut": (2600, 48, 16, 8, 64),
    "some-cut-many": (5000, 560, 4, 1, 64),
    "20-1": (2500, 520, 20, 1, 64),
}


@pytest.mark.parametrize("name", list(ATTENTION))
def test_attention_replayed_with_other_documents(name):
    n, docs, a, g, d = ATTENTION[name]
    gen = torch.Generator().manual_seed(n)
    q, k, v, do = (torch.randn((n, h, d), generator=gen).to(BF16).cuda() for h in (a, g, g, a))
    plans = list(many_starts(n, docs, 3))
    pk = L.make_packing(torch.tensor(plans[0], device="cuda"), n)
    size = L.l4d_attn_packed_workspace_bytes(n, a, g, d) + 256
    ar = [L.Arena.on(torch.zeros(size, dtype=torch.uint8, device="cuda")) for _ in range(2)]
    out, want = ({t: torch.empty(s, dtype=dt, device="cuda") for t, s, dt in
                  (("o", q.shape, BF16), ("lse", (a, n), F32), ("dq", q.shape, BF16), ("dk", k.shape, BF16),
                   ("dv", k.shape, BF16))} for _ in range(2))

    def step(x, arena, packing):
        L.attn_packed_fwd(q, k, v, x["o"], x["lse"], packing)
        L.attn_packed_bwd(q, k, v, x["o"], x["lse"], do, x["dq"], x["dk"], x["dv"], packing, arena)

    for x in (out, want):
        for t in x.values():
            t.fill_(7.0)
        step(x, ar[0], pk)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(out, ar[0], pk)
    for i, starts in enumerate(plans + plans[::-1]):
        pk.starts.copy_(torch.tensor(starts))
        for x in (out, want):
            for t in x.values():
                t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        step(want, ar[1], L.make_packing(torch.tensor(starts, device="cuda"), n))
        torch.cuda.synchronize()
        for t in want:
            assert torch.equal(out[t], want[t]), (i, t)
        outside = torch.ones(n, dtype=torch.bool)
        outside[starts[0]:starts[-1]] = False
        for t in ("o", "dq", "dk", "dv"):
            assert bool((out[t].cpu()[outside] == 7).all()) and not bool((out[t].cpu()[~outside] == 7).all(-1).any()), (i, t)


@pytest.mark.parametrize("docs", [4, 70])
def test_the_layer_replayed_with_other_documents(docs):
    w = W.TINY.replace(name="packed-replay", seq=300)
    buf = Buffers(w)
    plans = list(many_starts(w.seq, docs, 5))
    pk = L.make_packing(torch.tensor(plans[0], device="cuda"), w.seq)

    def step(packing):
        st = L.llama_layer_packed_fwd(buf.model, buf.par, buf.weights, buf.x, buf.y, buf.arena, packing)
        L.llama_layer_packed_bwd(buf.model, buf.par, buf.weights, st, buf.dy, buf.dx, buf.grads, buf.arena, packing)

    step(pk)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for t in buf.grads.values():
            t.zero_()
        step(pk)
    results = lambda: [t.clone() for t in (buf.y, buf.dx, *buf.grads.values())]      # noqa: E731
    for i, starts in enumerate(plans + plans[::-1]):
        pk.starts.copy_(torch.tensor(starts))
        graph.replay()
        torch.cuda.synchronize()
        got = results()
        for t in buf.grads.values():
            t.zero_()
        step(L.make_packing(torch.tensor(starts, device="cuda"), w.seq))
        torch.cuda.synchronize()
        for x, y in zip(got, results()):
            assert torch.equal(x, y) and bool(torch.isfinite(x).all()), i


@pytest.mark.parametrize("a,g,d", [(4, 2, 64), (4, 4, 64), (8, 2, 128), (3, 3, 128)])
def test_gradients_of_short_documents_are_rounded_once(a, g, d):
    """Documents of at most 7 rows: every row has a probability of 1/7 or more, so P and dS enter the
    products in two bf16 parts, which leave 2^-16 of an element, and fp32 sums of 7 and scores of 128
    products 2^-17 each.  The result is the rounding of the 64-bit gradient but for a fraction of
    2^-14 / 2^-9 of the elements; with one part a fifth of them would differ."""
    lens = [7, 5, 1, 6, 3, 7, 2, 4] * 6
    starts = starts_of(lens)
    n = starts[-1]
    gen = torch.Generator().manual_seed(d + a)
    q, k, v, do = (torch.randn((n, h, d), generator=gen).to(BF16) for h in (a, g, g, a))
    dev = [t.cuda() for t in (q, k, v, do)]
    pk = L.make_packing(torch.tensor(starts, device="cuda"), n)
    ar = L.Arena.on(torch.empty(L.l4d_attn_packed_workspace_bytes(n, a, g, d) + 256, dtype=torch.uint8, device="cuda"))
    o, lse = torch.empty_like(dev[0]), torch.empty((a, n), dtype=F32, device="cuda")
    grads = [torch.empty_like(t) for t in dev[:3]]
    L.attn_packed_fwd(*dev[:3], o, lse, pk)
    L.attn_packed_bwd(*dev[:3], o, lse, dev[3], *grads, pk, ar)
    x = [t.double().numpy() for t in (q, k, v, do)]
    want = [np.zeros(t.shape) for t in x[:3]]
    for lo, hi in zip(starts[:-1], starts[1:]):
        for h in range(a):
            hk = h * g // a
            Q, K, V, G = x[0][lo:hi, h], x[1][lo:hi, hk], x[2][lo:hi, hk], x[3][lo:hi, h]
            s = np.where(np.tri(hi - lo, dtype=bool), Q @ K.T / math.sqrt(d), -np.inf)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            dp = G @ V.T
            ds = p * (dp - (p * dp).sum(-1, keepdims=True)) / math.sqrt(d)
            want[0][lo:hi, h] = ds @ K
            want[1][lo:hi, hk] += ds.T @ Q
            want[2][lo:hi, hk] += p.T @ G
    off = []
    for t, y in zip(grads, want):
        some = np.abs(y) > 1e-3 * np.sqrt((y ** 2).mean())      # the others are sums that cancel
        off.append(float((t.cpu().double().numpy() != round_bf16(y))[some].mean()))
    print(off, flush=True)
    assert max(off) <= 2.0 ** -5
