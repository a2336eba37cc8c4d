"""What loss gradients owe to their targets, where every other element of G is exactly zero.

Each token's logits are 256 at column HOT and below 60 elsewhere, so its softmax is 1
there and underflows to 0 in every other column: G is -w at the target, w at HOT and 0
in between, with w = d_loss.  The rows of d_w at the targets and d_hidden then come from
the targets alone, and known values make every sum exact."""
import numpy as np
import pytest
import torch

import paper_2411_06465_amd as L
from oracle.bf16 import round_bf16
from packed_common import F

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
N, H, V, HOT = 2060, 64, 33000, 17          # two pieces of the vocabulary in the backward: 32512 columns and 488
BORDER = 32512
MANY = 20                                   # the target of most tokens


def inputs(seed):
    g = torch.Generator().manual_seed(seed)
    hidden = torch.randint(0, 2, (N, H), generator=g).float() * 2 - 1
    hidden[:, 0] = 4
    w = 0.25 * torch.randn((V, H), generator=g)
    w[:, 0] = 0
    w[HOT] = 0
    w[HOT, 0] = 64
    targets = torch.full((N,), MANY)
    # pairs and single ones, on both sides of 1024 tokens and of the border of the pieces
    for i, t in enumerate((BORDER - 1, BORDER, V - 1, 0, 9000)):
        targets[[1023 - i, 1024 + i]] = t
    targets[5], targets[2050] = 500, 500
    targets[2047], targets[2048], targets[0] = 32600, 700, 701
    targets[::9] = torch.where(targets[::9] == MANY, torch.tensor(-1), targets[::9])
    return hidden.to(BF16), w.to(BF16), targets


def gradients(hidden, w, targets, d_loss):
    h = [t.cuda() for t in (hidden, w, targets, d_loss)]
    ar = L.Arena.on(torch.empty(max(L.l4d_lm_loss_workspace_bytes(N, H, V)) + 256, dtype=torch.uint8, device="cuda"))
    loss, lse = (torch.empty(N, dtype=F32, device="cuda") for _ in range(2))
    L.lm_loss_fwd(*h[:3], loss, lse, ar)
    assert bool((lse == 256).all())
    d_hidden, d_w = torch.full_like(h[0], 5.0), torch.zeros((V, H), dtype=F32, device="cuda")
    L.lm_loss_bwd(*h[:3], lse, d_hidden, d_w, ar, d_loss=h[3])
    return d_hidden.cpu().double().numpy(), d_w.cpu().double().numpy()


def test_the_weight_gradient_is_completed_at_its_targets():
    """w = 1 + 2^-9 + b 2^-20 with b in 0 .. 3: its bf16 parts are 1 and 2^-9, and leave b 2^-20.  With hidden
    of +-1 the sums of the parts are multiples of 2^-9 below 2^12 and those of the rest multiples
    of 2^-20 below 2^-6: exact in fp32 in any order.  Only their last addition rounds, by F of the result."""
    hidden, w, targets = inputs(1)
    b = torch.randint(0, 4, (N,), generator=torch.Generator().manual_seed(2)).double()
    d_loss = (1 + 2.0 ** -9 + b * 2.0 ** -20).float()
    _, d_w = gradients(hidden, w, targets, d_loss)
    x, weight, t = hidden.double().numpy()[:, 1:], d_loss.double().numpy(), targets.numpy()
    lost = 0
    for col in sorted(set(t[t >= 0])):
        rows = t == col
        want = -(weight[rows, None] * x[rows]).sum(0)
        assert np.all(np.abs(d_w[col, 1:] - want) <= F * np.abs(want)), col
        parts = -((1 + 2.0 ** -9) * x[rows]).sum(0)               # what two parts alone give
        lost += int((np.abs(parts - want) > F * np.abs(want)).sum())
    assert lost > 300                                             # the comparison sees the completion
    others = np.ones(V, dtype=bool)
    others[t[t >= 0]] = others[HOT] = False
    assert not d_w[others].any()


def test_the_hidden_gradient_is_completed_at_its_targets():
    """Without column 0 d_hidden is -w W[target], rounded once: the nearest bf16 value, but for what a
    product and an addition in fp32 move."""
    hidden, w, targets = inputs(3)
    d_loss = 1 + torch.rand(N, generator=torch.Generator().manual_seed(4)).float()
    d_hidden, _ = gradients(hidden, w, targets, d_loss)
    t = targets.numpy()
    rows = t >= 0
    want = -d_loss.double().numpy()[rows, None] * w.double().numpy()[t[rows]][:, 1:]
    assert not d_hidden[~rows].any()
    best = np.abs(round_bf16(want) - want)
    got = d_hidden[rows][:, 1:]
    assert np.all(np.abs(got - want) <= best + 2 * F * np.abs(want))
    one = round_bf16(d_loss.double().numpy()[rows, None]) * -w.double().numpy()[t[rows]][:, 1:]     # one part alone
    assert int((np.abs(round_bf16(one) - want) > best + 2 * F * np.abs(want)).sum()) > 10000
