"""Cross-entropy without stored logits against the plain 64-bit form."""
import math

import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import U, close, inside, loss_plain

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def draw(n, h, v, tp=1, seed=0, std=0.05, ignored=0.2):
    """A shard of v rows of a vocabulary of v * tp, the middle one when there are several."""
    g = torch.Generator().manual_seed(seed + 31 * n + v)
    c = dict(hidden=torch.randn((n, h), generator=g).to(BF16), w=(std * torch.randn((v, h), generator=g)).to(BF16),
             v0=(tp // 2) * v, peer_lse=None, peer_z=None)
    c["targets"] = torch.randint(0, v * tp, (n,), generator=g)
    c["targets"][torch.rand(n, generator=g) < ignored] = -100
    if tp > 1:
        c["peer_lse"] = (math.log(v * (tp - 1)) + torch.randn(n, generator=g)).float()
        c["peer_z"] = torch.randn(n, generator=g).float()
    c["d_loss"] = torch.rand(n, generator=g).float() / n
    return c


def arena(n, h, v):
    return L.Arena.on(torch.empty(max(L.l4d_lm_loss_workspace_bytes(n, h, v)) + 256, dtype=torch.uint8, device="cuda"))


def run(c, ar=None, d_w0=0.0, d_loss=True, grad_scale=1.0):
    dev = {k: t.cuda() if torch.is_tensor(t) else t for k, t in c.items()}
    n, h, v = *c["hidden"].shape, c["w"].shape[0]
    ar = ar or arena(n, h, v)
    out = {k: torch.full((n,), 5.0, dtype=F32, device="cuda") for k in ("loss", "lse", "target_logit")}
    L.lm_loss_fwd(dev["hidden"], dev["w"], dev["targets"], out["loss"], out["lse"], ar, vocab_start=c["v0"],
                  peer_lse=dev["peer_lse"], peer_target_logit=dev["peer_z"], target_logit=out["target_logit"])
    out["d_hidden"] = torch.full_like(dev["hidden"], 5.0)
    out["d_w"] = torch.full(c["w"].shape, d_w0, dtype=F32, device="cuda")
    L.lm_loss_bwd(dev["hidden"], dev["w"], dev["targets"], out["lse"], out["d_hidden"], out["d_w"], ar,
                  d_loss=dev["d_loss"] if d_loss else None, grad_scale=grad_scale, vocab_start=c["v0"])
    return out


def compare(out, c, weights=None):
    d = {k: t.double() if torch.is_tensor(t) and t.is_floating_point() else t for k, t in c.items()}
    want = loss_plain(d["hidden"], d["w"], d["targets"], c["v0"], d["peer_lse"], d["peer_z"],
                      d["d_loss"] if weights is None else weights)
    inside("logit", out["target_logit"], want["target_logit"], want["_loss"] + want["_lse"])
    for t in ("lse", "loss", "d_hidden", "d_w"):
        inside(t, out[t], want[t], want["_" + t])
    close("d_hidden", out["d_hidden"], want["d_hidden"], U)     # two independent roundings of U/sqrt(3)
    close("d_w", out["d_w"], want["d_w"], 2.0 ** -15)           # what two bf16 parts leave
    return want


CASES = [  # n, h, v, tp
    (1, 8, 1, 1), (1, 64, 9, 1), (3, 8, 40, 1), (130, 256, 1000, 1), (64, 128, 64, 4), (257, 72, 333, 2),
    (777, 512, 1003, 1), (100, 1024, 5000, 1),       # several pieces of the vocabulary
    (33, 2048, 129, 8),
]


@pytest.mark.parametrize("n,h,v,tp", CASES)
def test_matches_the_plain_form(n, h, v, tp):
    c = draw(n, h, v, tp)
    compare(run(c), c)


def test_pieces_of_a_long_vocabulary():
    """So many tokens that the vocabulary is taken in pieces, with targets at the borders."""
    c = draw(8300, 16, 8203, seed=7, std=0.2)
    c["targets"][:4] = torch.tensor([0, 8191, 8192, 8202])
    compare(run(c), c)


def test_confident_rows_and_large_logits():
    """Probabilities next to 1 (the gradient a small difference) and logits of hundreds."""
    c = draw(96, 256, 500, std=0.5, seed=3, ignored=0.0)
    c["hidden"][:32] = (4 * c["w"][:32].float()).to(BF16)
    c["targets"][:32] = torch.arange(32)
    c["hidden"][32:64] *= 40
    compare(run(c), c)


def test_all_ignored_and_none_weighted():
    c = draw(50, 128, 300)
    c["targets"][:] = -1
    out = run(c, d_w0=2.5)
    assert bool((out["loss"] == 0).all()) and bool((out["d_hidden"] == 0).all()) and bool((out["d_w"] == 2.5).all())
    assert bool((out["target_logit"] == -math.inf).all()) and bool(torch.isfinite(out["lse"]).all())
    c = draw(50, 128, 300)
    compare(run(c, d_loss=False, grad_scale=0.25), c, torch.full((50,), 0.25, dtype=torch.float64))


def test_an_ignored_row_of_nan_reaches_no_other_row():
    c = draw(70, 128, 260, ignored=0.0)
    c["targets"][11] = -1
    want = run(c)
    c["hidden"][11] = math.nan
    out = run(c)
    keep = torch.arange(70) != 11
    for t in ("loss", "lse", "d_hidden"):
        assert torch.equal(out[t].cpu()[keep], want[t].cpu()[keep]), t
    assert bool((out["d_hidden"][11] == 0).all())


def test_weight_gradient_is_added():
    c = draw(65, 64, 200)
    base, out = run(c), run(c, d_w0=1.0)
    assert torch.allclose(out["d_w"] - 1.0, base["d_w"], rtol=0, atol=2 * 2.0 ** -24 * 2)   # two roundings near 1
    for t in ("loss", "d_hidden"):
        assert torch.equal(base[t], out[t])


def test_shards_make_the_whole_loss():
    """Two ranks' shards, each given the other's statistics, against the whole vocabulary."""
    c = draw(90, 128, 400, ignored=0.1)
    whole = run(c)
    halves = [dict(c, w=c["w"][i:i + 200].contiguous(), v0=i) for i in (0, 200)]
    alone = [run(h) for h in halves]
    got = []
    for h, other in zip(halves, alone[::-1]):
        got.append(run(dict(h, peer_lse=other["lse"].cpu(), peer_z=other["target_logit"].cpu())))
    want = compare(whole, c)
    for g in got:
        inside("loss", g["loss"], want["loss"], want["_loss"] + 8 * 2.0 ** -24 * (1 + want["lse"].abs()))
    d_w = torch.cat([g["d_w"] for g in got])
    close("d_w", d_w, want["d_w"], 2.0 ** -15)
    total = got[0]["d_hidden"].float() + got[1]["d_hidden"].float()
    close("d_hidden", total, want["d_hidden"], 2 * U)


def test_captured_and_replayed():
    n, h, v = 150, 256, 700
    c = draw(n, h, v)
    ar = arena(n, h, v)
    dev = {k: t.cuda() for k, t in c.items() if torch.is_tensor(t)}
    out = run(c, ar)
    d_w = torch.zeros_like(out["d_w"])

    def step():
        d_w.zero_()
        L.lm_loss_fwd(dev["hidden"], dev["w"], dev["targets"], out["loss"], out["lse"], ar)
        L.lm_loss_bwd(dev["hidden"], dev["w"], dev["targets"], out["lse"], out["d_hidden"], d_w, ar, d_loss=dev["d_loss"])

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2, 3):
        new = draw(n, h, v, seed=seed)
        for k, t in dev.items():
            t.copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        want = run(new)
        assert torch.equal(out["loss"], want["loss"]) and torch.equal(out["d_hidden"], want["d_hidden"])
        assert torch.equal(d_w, want["d_w"])


def test_a_full_arena_is_refused_before_any_launch():
    c = draw(40, 64, 100)
    small = L.Arena.on(torch.empty(512, dtype=torch.uint8, device="cuda"))
    with pytest.raises(L.L4DError) as e:
        run(c, small)
    assert e.value.code == L.L4D_ENOMEM
