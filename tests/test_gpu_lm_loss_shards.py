"""Cross-entropy without stored logits where shards and pieces of the vocabulary are
joined: values that are not numbers, and a forward in several pieces."""
import math

import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import F, inside, loss_plain

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def forward(hidden, w, targets, v0=0, peer_lse=None, peer_z=None):
    n, h = hidden.shape
    size = L.l4d_lm_loss_workspace_bytes(n, h, w.shape[0])[0]
    ar = L.Arena.on(torch.empty(size + 256, dtype=torch.uint8, device="cuda"))
    loss, lse, z = (torch.full((n,), 5.0, dtype=F32, device="cuda") for _ in range(3))
    L.lm_loss_fwd(hidden, w, targets, loss, lse, ar, vocab_start=v0, peer_lse=peer_lse, peer_target_logit=peer_z,
                  target_logit=z)
    return loss, lse, z


@pytest.mark.parametrize("bad", ["own", "peer", "both"])
def test_a_shard_that_is_not_a_number_shows_in_every_loss(bad):
    """One row of a shard's head is NaN: both ranks' log-sum-exp and the losses of all counted tokens are."""
    n, h, v = 90, 64, 200
    g = torch.Generator().manual_seed(3)
    hidden = torch.randn((n, h), generator=g).to(BF16).cuda()
    w = (0.05 * torch.randn((2 * v, h), generator=g)).to(BF16).cuda()
    targets = torch.randint(0, 2 * v, (n,), generator=g).cuda()
    targets[::7] = -1
    if bad != "peer":
        w[17] = math.nan
    if bad != "own":
        w[v + 40] = math.nan
    shards = [(w[:v].contiguous(), 0), (w[v:].contiguous(), v)]
    alone = [forward(hidden, x, targets, v0) for x, v0 in shards]
    for (x, v0), other, own_bad in zip(shards, alone[::-1], (bad != "peer", bad != "own")):
        loss, lse, _ = forward(hidden, x, targets, v0, other[1], other[2])
        assert bool(torch.isnan(lse).all()), (v0, own_bad)
        assert torch.equal(torch.isnan(loss), targets >= 0) and bool((loss[targets < 0] == 0).all())
    # the shard without it keeps its own statistics
    for (loss, lse, _), own_bad in zip(alone, (bad != "peer", bad != "own")):
        assert bool(torch.isnan(lse).all() if own_bad else torch.isfinite(lse).all())


def test_one_row_that_is_not_a_number_reaches_no_other():
    n, h, v = 70, 64, 300
    g = torch.Generator().manual_seed(4)
    hidden = torch.randn((n, h), generator=g).to(BF16).cuda()
    w = (0.05 * torch.randn((v, h), generator=g)).to(BF16).cuda()
    targets = torch.randint(0, 2 * v, (n,), generator=g).cuda()
    peer_lse, peer_z = (torch.randn(n, generator=g).cuda() + 5 for _ in range(2))
    want = forward(hidden, w, targets, 0, peer_lse, peer_z)
    hidden[13] = math.nan
    peer_lse[29] = math.nan
    got = forward(hidden, w, targets, 0, peer_lse, peer_z)
    keep = torch.ones(n, dtype=torch.bool)
    keep[[13, 29]] = False
    for x, y in zip(got[:2], want[:2]):
        assert torch.equal(x.cpu()[keep], y.cpu()[keep]) and bool(torch.isnan(x.cpu()[~keep]).all())


def test_the_forward_in_pieces_of_the_vocabulary():
    """33000 tokens take 65536 columns at a time: two pieces, with targets at their border."""
    n, h, v = 33000, 8, 65800
    g = torch.Generator().manual_seed(5)
    hidden = torch.randn((n, h), generator=g).to(BF16).cuda()
    w = torch.randn((v, h), generator=g).to(BF16).cuda()
    targets = torch.randint(0, v, (n,), generator=g)
    at = torch.arange(0, n, 173)                                # the rows compared with the plain form
    targets[at[:6]] = torch.tensor([0, 65535, 65536, 65799, -1, 65537])
    targets = targets.cuda()
    size = L.l4d_lm_loss_workspace_bytes(n, h, v)[0]
    assert size < n * (v + 63) // 64 * 8                        # the statistics of fewer than all columns
    got = [x.cpu() for x in forward(hidden, w, targets)]
    print("the plain form", flush=True)
    want = loss_plain(hidden[at.cuda()].cpu().double(), w.cpu().double(), targets[at.cuda()].cpu())
    for t, x in zip(("loss", "lse"), got):
        inside(t, x[at], want[t], want["_" + t])
    inside("logit", got[2][at], want["target_logit"], want["_loss"] + want["_lse"])
    # every row: two shards of one piece each, joined by the peers' statistics
    parts = [(w[:65536].contiguous(), 0), (w[65536:].contiguous(), 65536)]
    first, second = (forward(hidden, x, targets, v0) for x, v0 in parts)
    loss, lse, _ = (x.cpu() for x in forward(hidden, *parts[0][:1], targets, 0, second[1], second[2]))
    here = torch.isfinite(first[2]).cpu()
    assert torch.equal(got[2], torch.where(here, first[2].cpu(), second[2].cpu()))       # the same products
    # Two orders of adding the same 65800 exponentials, each term off by a few F and each sum by F per
    # addition: 64 in a block of columns, then 1029 blocks, and the logarithms' own roundings.
    bound = (2 * (64 + 1029) + 32) * F * torch.ones(n, dtype=torch.float64) + 16 * F * lse.double().abs()
    inside("lse", got[1], lse.double(), bound)
    inside("loss", got[0], loss.double(), bound + 4 * F * (lse.double().abs() + got[2].double().nan_to_num(neginf=0.0).abs()))
