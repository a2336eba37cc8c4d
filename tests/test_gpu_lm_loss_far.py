"""The loss's gradient pieces past 2^32 elements."""
import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import U

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def gradients(hidden, w, targets, d_loss):
    n, h = hidden.shape
    v = w.shape[0]
    ar = L.Arena.on(torch.empty(max(L.l4d_lm_loss_workspace_bytes(n, h, v)) + 256, dtype=torch.uint8, device="cuda"))
    loss, lse = (torch.empty(n, dtype=F32, device="cuda") for _ in range(2))
    d_hidden, d_w = torch.empty_like(hidden), torch.zeros((v, h), dtype=F32, device="cuda")
    L.lm_loss_fwd(hidden, w, targets, loss, lse, ar)
    L.lm_loss_bwd(hidden, w, targets, lse, d_hidden, d_w, ar, d_loss=d_loss)
    return loss, d_hidden.float(), d_w


def test_many_tokens_as_two_halves():
    """280000 tokens x 8192 columns, twice 2.3e9 elements of G, against the same tokens in two calls.  A
    loss is the same sum in another order at most; d_hidden may round the other way (2 U of the larger of
    two neighbours); the halves of d_w add up to the whole within what two bf16 parts leave (2^-15 in norm)."""
    n, h, v = 280000, 16, 8192
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 20 GB")
    g = torch.Generator(device="cuda").manual_seed(2)
    hidden = torch.randn((n, h), generator=g, device="cuda").to(BF16)
    w = (0.3 * torch.randn((v, h), generator=g, device="cuda")).to(BF16)
    targets = torch.randint(0, v, (n,), generator=g, device="cuda")
    targets[::5] = -1
    d_loss = torch.rand(n, generator=g, device="cuda")
    whole = gradients(hidden, w, targets, d_loss)
    half = n // 2
    parts = [gradients(*(t[i:i + half] if t is not w else t for t in (hidden, w, targets, d_loss))) for i in (0, half)]
    loss, d_hidden = (torch.cat([p[i] for p in parts]) for i in (0, 1))
    assert float((whole[0] - loss).abs().max()) <= 1e-5                      # of about 10: a few fp32 steps
    assert bool((whole[1][targets < 0] == 0).all()) and bool((whole[1][targets >= 0] != 0).any(-1).all())
    norm = float(d_hidden.abs().max())
    assert bool(((whole[1] - d_hidden).abs() <= 2 * U * torch.maximum(whole[1].abs(), d_hidden.abs()) + 1e-6 * norm).all())
    d_w = parts[0][2] + parts[1][2]
    assert float((whole[2] - d_w).norm()) <= 2.0 ** -15 * float(d_w.norm())
