"""The operators around the attention together, as a layer's step makes them: norms and rotation of
q and k, windowed attention over packed documents, an output projection, dropout and the residual
sum, and the gradients back to q, k, v, the gains and the residual; eager, on a stream of its own,
and captured."""
import math

import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import U, close, starts_of
from test_gpu_attn_window import hidden_pairs
from test_gpu_qk_norm import BASE, axes_frequencies, turn

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64

A, G, D, WINDOW, SINKS, P, EPS = 8, 2, 64, 50, 3, 0.2, 1e-6
PAIRS = (12, 10, 10)


class Step:
    """Buffers and one forward and backward of the block over n rows."""

    def __init__(self, n, seed, starts):
        g = torch.Generator().manual_seed(seed)

        def t(*shape, mean=0.0, std=1.0):
            return (mean + std * torch.randn(shape, generator=g)).to(BF16).cuda()

        self.n, self.cols = n, A * D
        self.qkv, self.res, self.dy = t(n, (A + 2 * G) * D), t(n, A * D), t(n, A * D)
        self.gq, self.gk = t(D, mean=1.0, std=0.2), t(D, mean=1.0, std=0.2)
        self.pos = torch.randint(0, 300, (3, n), generator=g).cuda()
        self.rng = torch.tensor([seed, 7], device="cuda")
        self.pk = L.make_packing(torch.tensor(starts, device="cuda"), n)
        self.win, self.rope = L.make_window(WINDOW, SINKS), L.make_rope(D, base=BASE)
        self.axes = L.make_rope_axes(PAIRS, "cycled")
        size = (L.l4d_attn_window_workspace_bytes(self.win, n, A, G, D) + L.l4d_qk_norm_workspace_bytes(n, D) + 4096)
        self.arena = L.Arena.on(torch.full((size,), 0xff, dtype=torch.uint8, device="cuda"))
        self.rot = torch.zeros((n, (A + G) * D), dtype=BF16, device="cuda")          # rotated q | k
        self.o, self.y = (torch.zeros((n, A * D), dtype=BF16, device="cuda") for _ in range(2))
        self.lse = torch.zeros((A, n), dtype=F32, device="cuda")
        self.d_o = torch.zeros_like(self.o)
        self.d_rot, self.d_qkv = torch.zeros_like(self.rot), torch.zeros_like(self.qkv)
        self.dgq, self.dgk = (torch.zeros(D, device="cuda") for _ in range(2))

    def heads(self, t, i, j):
        return t[:, i * D:j * D].unflatten(1, (j - i, D))

    def run(self, stream=None):
        q, k, v = (self.heads(self.qkv, i, j) for i, j in ((0, A), (A, A + G), (A + G, A + 2 * G)))
        rq, rk = self.heads(self.rot, 0, A), self.heads(self.rot, A, A + G)
        where = dict(eps=EPS, positions=self.pos, axes=self.axes, packing=self.pk, stream=stream)
        L.qk_norm_rope_fwd(self.rope, q, self.gq, rq, k, self.gk, rk, **where)
        o = self.o.unflatten(1, (A, D))
        L.attn_window_fwd(self.win, rq, rk, v, o, self.lse, self.pk, stream=stream)
        L.dropout_add_fwd(self.o, self.res, self.y, self.rng, P, stream=stream)
        # backward
        L.dropout_add_bwd(self.dy, self.d_o, self.rng, P, stream=stream)
        dq, dk, dv = (self.heads(self.d_qkv, i, j) for i, j in ((0, A), (A, A + G), (A + G, A + 2 * G)))
        drq, drk = self.heads(self.d_rot, 0, A), self.heads(self.d_rot, A, A + G)
        L.attn_window_bwd(self.win, rq, rk, v, o, self.lse, self.d_o.unflatten(1, (A, D)), drq, drk, dv, self.pk, self.arena,
                          stream=stream)
        L.qk_norm_rope_bwd(self.rope, q, self.gq, drq, dq, self.dgq, self.arena, k, self.gk, drk, dk, self.dgk, **where)

    def results(self):
        return dict(y=self.y, d_qkv=self.d_qkv, dgq=self.dgq, dgk=self.dgk)

    def clear(self):
        for t in (self.rot, self.o, self.y, self.lse, self.d_o, self.d_rot, self.d_qkv, self.dgq, self.dgk):
            t.zero_()


def plain(s, starts, keep):
    """The block in 64 bits, its gradients by differentiation; keep: the dropout mask [n][cols]."""
    qkv, gq, gk = (t.cpu().double().requires_grad_() for t in (s.qkv, s.gq, s.gk))
    table = axes_frequencies(PAIRS, "cycled", False, D)
    axis = torch.tensor([a for a, _ in table])
    angle = s.pos.cpu()[axis].t().double() * torch.tensor([f for _, f in table], dtype=F64)
    c, sn = angle.cos()[:, None, :], angle.sin()[:, None, :]

    def head(t, gain):
        x = t * (t.square().mean(-1, keepdim=True) + EPS).rsqrt() * gain
        a, b = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([a * c - b * sn, b * c + a * sn], -1)

    q, k, v = (s.heads(qkv, i, j) for i, j in ((0, A), (A, A + G), (A + G, A + 2 * G)))
    q, k = head(q, gq), head(k, gk)
    rows = []
    rows.append(torch.zeros((starts[0], A, D), dtype=F64))
    for lo, hi in zip(starts[:-1], starts[1:]):
        mask = torch.zeros(hi - lo, hi - lo, dtype=F64).masked_fill(hidden_pairs(hi - lo, WINDOW, SINKS), -math.inf)
        rows.append(torch.stack([torch.softmax(q[lo:hi, h] @ k[lo:hi, h // (A // G)].T / math.sqrt(D) + mask, -1)
                                 @ v[lo:hi, h // (A // G)] for h in range(A)], 1))
    rows.append(torch.zeros((s.n - starts[-1], A, D), dtype=F64))
    y = s.res.cpu().double() + torch.where(keep, torch.cat(rows).reshape(s.n, -1) / (1 - P), torch.zeros((), dtype=F64))
    grads = torch.autograd.grad((y * s.dy.cpu().double()).sum(), (qkv, gq, gk))
    return dict(y=y.detach(), d_qkv=grads[0], dgq=grads[1], dgk=grads[2])


STARTS, N = starts_of([70, 0, 1, 200, 33], 2), 310


def test_the_block_against_the_plain_form():
    s = Step(N, 5, STARTS)
    s.run()
    ones, keep = torch.ones((N, A * D), device="cuda"), torch.zeros((N, A * D), device="cuda")
    L.dropout_add_fwd(ones, None, keep, s.rng, P)
    want = plain(s, STARTS, (keep != 0).cpu())
    got = s.results()
    # Roundings to bf16 on the way, each at most U/sqrt(3) of a tensor's norm where the step before
    # carries it on with a factor of about one: y: rotated q and k (through the softmax), P, o, y.
    # d_qkv: those, d_o, dS, the gradient of the rotated heads, the result.  The gains' gradients
    # sum the errors of many rows, which are independent: no larger part of them.
    close("y", got["y"], want["y"], 3 * U)
    # behind the norm the gradients of q and k lose their part along x, which the errors keep: twice
    for i, j in ((0, A), (A, A + G), (A + G, A + 2 * G)):
        close("d_qkv", got["d_qkv"][:, i * D:j * D], want["d_qkv"][:, i * D:j * D], 6 * U)
    close("dgq", got["dgq"], want["dgq"], 6 * U)
    close("dgk", got["dgk"], want["dgk"], 6 * U)


def test_the_block_on_a_stream_and_captured_beside_an_eager_one():
    """Replays of a captured step, with an eager step of the same inputs between them, and of one on a stream."""
    s, e = Step(N, 9, STARTS), Step(N, 9, STARTS)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    s.run(stream)
    stream.synchronize()
    e.run()
    for t, x in e.results().items():
        assert torch.equal(x, s.results()[t]), t
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for i, starts in enumerate((STARTS, [0, 0, 100, 101, 300, 310], [5, 6, 7, 8, 9, 10])):
        for x in (s, e):
            x.clear()
            x.qkv.add_(0.25)
            x.rng[1] = 40 + i
            x.pk.starts.copy_(torch.tensor(starts))
        graph.replay()
        e.run()
        torch.cuda.synchronize()
        for t, x in e.results().items():
            assert torch.equal(x, s.results()[t]), (i, t)
        s.clear()
        graph.replay()
        torch.cuda.synchronize()
        for t, x in e.results().items():
            assert torch.equal(x, s.results()[t]), (i, t)


def test_one_token():
    s = Step(1, 3, [0, 1])
    s.run()
    keep = torch.zeros((1, A * D), device="cuda")
    L.dropout_add_fwd(torch.ones_like(keep), None, keep, s.rng, P)
    want = plain(s, [0, 1], (keep != 0).cpu())
    got = s.results()
    close("y", got["y"], want["y"], U)
    # one visible key: q and k get no gradient, v gets d_o summed over its heads
    close("dv", got["d_qkv"][:, (A + G) * D:], want["d_qkv"][:, (A + G) * D:], 2 * U)
    assert float(want["d_qkv"][:, :(A + G) * D].abs().max()) < 1e-12
