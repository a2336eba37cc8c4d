"""The layer over packed documents against the float64 oracle of each document,
and a training step that uses the packed operators together."""
import numpy as np
import pytest
import torch

import paper_2411_06465_amd as L
import workloads as W
from gpu_common import REL_FROB, Buffers, check, compare_layer, host_f64, oracle_layer
from oracle import layer as OL
from oracle.bf16 import from_bits
from packed_common import starts_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
GRADS = ("norm1", "qkv", "o", "norm2", "gate_up", "down")

CASES = {  # workload (its sequence is replaced by the packed row), document lengths, rows behind them
    "d64": (W.TINY, [50, 1, 77], 8),
    "d64-one": (W.TINY, [128], 0),
    "d128-gqa4": (W.LayerWorkload("packed-d128", 1024, 8, 2, 1376, 0, rope_base=5e5), [130, 0, 200, 31], 23),
    "d128-mha": (W.LayerWorkload("packed-mha", 512, 4, 4, 768, 0), [3] * 20 + [170], 2),
}


class ScaledShard(OL.Shard):
    """Positions divided by a factor (linear scaling)."""
    factor = 1.0

    def positions(self):
        own, rem = super().positions()
        return own / self.factor, rem


def packing(starts, n):
    return L.make_packing(torch.tensor(starts, dtype=torch.int64, device="cuda"), n)


def run_packed(buf, pk, rope=None):
    w = buf.w
    st = L.llama_layer_packed_fwd(buf.model, buf.par, buf.weights, buf.x, buf.y, buf.arena, pk, rope,
                                  peers=buf.peers, sends=buf.sends)
    saved = {n: buf.stash_view(st, n, (1, w.s_c, c)).clone() for n, c in
             (("q", w.a_t * w.d_h), ("k", w.k_t * w.d_h), ("v", w.k_t * w.d_h), ("ctx", w.a_t * w.d_h))}
    L.llama_layer_packed_bwd(buf.model, buf.par, buf.weights, st, buf.dy, buf.dx, buf.grads, buf.arena, pk, rope,
                             peers=buf.peers, sends=buf.sends)
    torch.cuda.synchronize()
    return saved


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("factor", [1.0, 4.0])
def test_documents_match_the_oracle(name, factor):
    base, lens, tail = CASES[name]
    starts = starts_of(lens)
    n = starts[-1] + tail
    w = base.replace(name=f"{base.name}-packed", seq=n)
    buf = Buffers(w)
    buf.dy[:, starts[-1]:] = 0                  # padding has no gradient
    rope = None if factor == 1.0 else L.make_rope(w.d_h, base=w.rope_base, scaling="linear", factor=factor)
    saved = run_packed(buf, packing(starts, n), rope)
    x, dy = from_bits(buf.abits["x"]), from_bits(buf.abits["dy"])
    wts = {k: from_bits(v) for k, v in buf.wbits.items()}
    got = dict(y=host_f64(buf.y), dx=host_f64(buf.dx), **{k: host_f64(t) for k, t in saved.items()})
    want = {k: [] for k in got}
    grads = {g: 0.0 for g in GRADS}
    for lo, hi in zip(starts[:-1], starts[1:]):
        if hi == lo:
            continue
        sh = ScaledShard(**w.replace(seq=hi - lo).shard_kwargs())
        sh.factor = factor
        fw = OL.layer_forward(sh, wts, x[:, lo:hi], {})
        bw = OL.layer_backward(sh, wts, fw, dy[:, lo:hi], {})
        for k in want:
            want[k].append((bw if k == "dx" else fw)[k])
        for g in GRADS:
            grads[g] = grads[g] + bw["d_" + g]
    ok = True
    for k in got:
        ok &= check(k, got[k][:, :starts[-1]], np.concatenate(want[k], axis=1))
    for g in GRADS:
        ok &= check("d_" + g, host_f64(buf.grads[g]), grads[g], bf16=False)
    assert ok
    assert np.all(got["ctx"][:, starts[-1]:] == 0) and np.all(np.isfinite(got["y"]))


def test_tensor_parallel_rank_matches_the_oracle():
    """TP2 with sequence parallelism: gathered rows, receipts and sends, one document over the whole row."""
    w = W.TINY.replace(name="packed-tp2", tp=2, tp_rank=1, n_gpus=2)
    buf = Buffers(w)
    st = L.llama_layer_packed_fwd(buf.model, buf.par, buf.weights, buf.x, buf.y, buf.arena, packing([0, w.seq], w.seq),
                                  peers=buf.peers, sends=buf.sends)
    shapes = dict(x=w.hidden, xn1=w.hidden, h1=w.hidden, xn2=w.hidden, q=w.a_t * w.d_h, ctx=w.a_t * w.d_h,
                  k=w.k_t * w.d_h, v=w.k_t * w.d_h, gate=w.f_t, up=w.f_t, act=w.f_t, prod=w.f_t)
    saved = {n: buf.stash_view(st, n, (1, w.s_sp if n in ("x", "xn1", "h1", "xn2") else w.s_c, c)).clone()
             for n, c in shapes.items()}
    saved["lse"] = buf.stash_view(st, "lse", (1, w.a_t, w.s_c), F32).clone()
    saved.update({n: buf.sends[n].clone() for n in ("o_partial", "ffn_partial")})
    L.llama_layer_packed_bwd(buf.model, buf.par, buf.weights, st, buf.dy, buf.dx, buf.grads, buf.arena,
                             packing([0, w.seq], w.seq), peers=buf.peers, sends=buf.sends)
    fw, bw = oracle_layer(w, buf.wbits, buf.abits)
    ok, rep = compare_layer(w, buf, saved, fw, bw)
    assert ok, "\n".join(rep)


def test_refusals():
    w = W.TINY
    buf = Buffers(w)
    pk = packing([0, 60, 128], 128)

    def refused(call):
        with pytest.raises(L.L4DError) as e:
            call()
        assert e.value.code == L.L4D_EINVAL
        assert buf.arena.stats()["in_use"] == held

    held = 0

    def fwd(par=buf.par, pk=pk, rope=None):
        return L.llama_layer_packed_fwd(buf.model, par, buf.weights, buf.x, buf.y, buf.arena, pk, rope)

    refused(lambda: fwd(pk=packing([0, 60], 60)))
    refused(lambda: fwd(pk=packing([0], 128)))
    refused(lambda: fwd(par=L.make_parallel(64, micro_batch=2)))
    refused(lambda: fwd(par=L.make_parallel(256, cp=2)))
    refused(lambda: fwd(rope=L.make_rope(128)))
    refused(lambda: fwd(rope=L.make_rope(64, 32)))
    refused(lambda: fwd(rope=L.make_rope(64, layout="interleaved")))
    packed, plain = fwd(), L.llama_layer_fwd(buf.model, buf.par, buf.weights, buf.x, buf.y, buf.arena)
    held = buf.arena.stats()["in_use"]
    refused(lambda: L.llama_layer_bwd(buf.model, buf.par, buf.weights, packed, buf.dy, buf.dx, buf.grads, buf.arena))
    refused(lambda: L.llama_layer_packed_bwd(buf.model, buf.par, buf.weights, plain, buf.dy, buf.dx, buf.grads,
                                             buf.arena, pk))
    packed.release()
    plain.release()
    torch.cuda.synchronize()


# ------------------------------------------------------------------ the operators together

class Step:
    """One training step on packed documents: embedding, two layers, the loss, and back."""

    def __init__(self, lens, tail):
        self.w = w = W.TINY
        self.starts = starts_of(lens)
        self.n = n = self.starts[-1] + tail
        g = torch.Generator().manual_seed(5)
        self.v = 1000
        self.model = L.make_model(**dict(w.model(), vocab=self.v))
        self.weights = {k: torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).cuda().view(BF16)
                        for k, b in W.layer_weights(w).items()}
        self.w_emb = torch.randn((self.v, w.hidden), generator=g).to(BF16).cuda()
        self.w_lm = (0.05 * torch.randn((self.v, w.hidden), generator=g)).to(BF16).cuda()
        self.ids = torch.randint(0, self.v, (n,), generator=g).cuda()
        self.targets = torch.roll(self.ids, -1)
        self.targets[torch.tensor(self.starts[1:], device="cuda") - 1] = -1      # a document's last token predicts nothing
        self.targets[self.starts[-1]:] = -1
        self.valid = int((self.targets >= 0).sum())
        self.arena = L.Arena.on(torch.empty(256 << 20, dtype=torch.uint8, device="cuda"))

    def buffers(self, n):
        h = self.w.hidden
        x = [torch.empty((n, h), dtype=BF16, device="cuda") for _ in range(3)]
        d = [torch.empty((n, h), dtype=BF16, device="cuda") for _ in range(3)]
        return x, d, torch.empty(n, dtype=F32, device="cuda"), torch.empty(n, dtype=F32, device="cuda")

    def grads(self):
        h = self.w.hidden
        out = {k: torch.zeros(t.shape, dtype=F32, device="cuda") for k, t in self.weights.items()}
        out["emb"], out["lm"] = (torch.zeros((self.v, h), dtype=F32, device="cuda") for _ in range(2))
        return out

    def run(self, ids, targets, grads, bufs, packing=None):
        x, d, loss, lse = bufs
        par = L.make_parallel(ids.numel())
        emb = L.embedding_fwd(self.model, par, ids, self.w_emb, x[0], self.arena)
        st = []
        for i in range(2):
            a = (self.model, par, self.weights, x[i], x[i + 1], self.arena)
            st.append(L.llama_layer_packed_fwd(*a, packing) if packing else L.llama_layer_fwd(*a))
        L.lm_loss_fwd(x[2], self.w_lm, targets, loss, lse, self.arena)
        L.lm_loss_bwd(x[2], self.w_lm, targets, lse, d[2], grads["lm"], self.arena, grad_scale=1.0 / self.valid)
        for i in (1, 0):
            a = (self.model, par, self.weights, st[i], d[i + 1], d[i], grads, self.arena)
            if packing:
                L.llama_layer_packed_bwd(*a, packing)
            else:
                L.llama_layer_bwd(*a)
        L.embedding_bwd(self.model, par, emb, d[0], grads["emb"], self.arena)
        return loss


@pytest.mark.parametrize("lens,tail", [([40, 7, 100, 1, 60], 16), ([300], 0)])
def test_a_training_step_on_packed_documents(lens, tail):
    """Losses and every gradient as when each document goes through the unpacked layer alone."""
    s = Step(lens, tail)
    got, want = s.grads(), s.grads()
    bufs = s.buffers(s.n)
    loss = s.run(s.ids, s.targets, got, bufs, packing(s.starts, s.n))
    # a document of which no token counts still runs: its gradients are zero
    one = [s.run(s.ids[lo:hi].contiguous(), s.targets[lo:hi].contiguous(), want, s.buffers(hi - lo))
           for lo, hi in zip(s.starts[:-1], s.starts[1:])]
    ok = check("loss", host_f64(loss)[:s.starts[-1]], host_f64(torch.cat(one)), bf16=False, abs_bound=2e-2)
    for k in got:
        # both paths are held to REL_FROB of the oracle
        e = float((got[k] - want[k]).norm() / want[k].norm())
        print(f"{k:>8s}: {e:.2e}", flush=True)
        ok &= e <= 2 * REL_FROB
    assert ok
    assert bool((loss[s.starts[-1]:] == 0).all())


def test_the_step_captured_and_replayed():
    s = Step([40, 7, 100, 1, 60], 16)
    pk, bufs, grads = packing(s.starts, s.n), s.buffers(s.n), s.grads()
    s.run(s.ids, s.targets, grads, bufs, pk)          # warms up
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for t in grads.values():
            t.zero_()
        loss = s.run(s.ids, s.targets, grads, bufs, pk)
    for seed in range(3):
        new = torch.randint(0, s.v, (s.n,), generator=torch.Generator().manual_seed(seed)).cuda()
        keep = s.targets >= 0
        s.ids.copy_(new)
        s.targets.copy_(torch.where(keep, torch.roll(new, -1), s.targets))
        graph.replay()
        torch.cuda.synchronize()
        eager = s.grads()
        want = s.run(s.ids, s.targets, eager, s.buffers(s.n), pk)
        assert torch.equal(loss, want)
        for k in grads:
            if k == "emb":      # atomic adds in no fixed order
                assert float((grads[k] - eager[k]).norm() / eager[k].norm()) <= 1e-6
            else:
                assert torch.equal(grads[k], eager[k]), (seed, k)
