"""Packed attention with many query heads per key head, against the plain 64-bit form."""
import random

import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import U, attention_plain, close, inside, starts_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def log_normal(docs, tokens, seed):
    rng = random.Random(seed)
    share = [rng.lognormvariate(0.0, 1.0) for _ in range(docs)]
    return [max(1, round(tokens * s / sum(share))) for s in share]


CASES = {  # document lengths, heads, kv heads, d; blocks enough that only long ones are cut
    "22-1": (log_normal(390, 16000, 1), 22, 1, 64),
    "48-1": (log_normal(390, 16000, 2), 48, 1, 64),
    "64-2": (log_normal(300, 16000, 3), 64, 2, 64),
    "64-2-short": ([65] * 60 + [0] * 200, 64, 2, 128),
    "18-1-around-128": ([127, 128, 129, 33, 97] * 30 + [0] * 400, 18, 1, 128),
    "48-1-equal": ([40] * 450, 48, 1, 64),          # all short: more second slices than windows, were they cut
}


@pytest.mark.parametrize("name", list(CASES))
def test_gradients_of_many_query_heads(name):
    lens, a, g, d = CASES[name]
    starts = starts_of(lens, 5)
    n = starts[-1] + 9
    gen = torch.Generator().manual_seed(n)
    q, k, v, do = (torch.randn((n, h, d), generator=gen).to(BF16) for h in (a, g, g, a))
    dev = [t.cuda() for t in (q, k, v, do)]
    pk = L.make_packing(torch.tensor(starts, device="cuda"), n)
    ar = L.Arena.on(torch.empty(L.l4d_attn_packed_workspace_bytes(n, a, g, d) + 256, dtype=torch.uint8, device="cuda"))
    out = dict(o=torch.full_like(dev[0], 7.0), lse=torch.full((a, n), 7.0, dtype=F32, device="cuda"),
               dq=torch.full_like(dev[0], 7.0), dk=torch.full_like(dev[1], 7.0), dv=torch.full_like(dev[2], 7.0))
    L.attn_packed_fwd(*dev[:3], out["o"], out["lse"], pk)
    L.attn_packed_bwd(*dev[:3], out["o"], out["lse"], dev[3], out["dq"], out["dk"], out["dv"], pk, ar)
    torch.cuda.synchronize()
    print("the plain form", flush=True)
    rows = slice(starts[0], starts[-1])
    for hk in range(g):      # a kv head and its query heads at a time
        hq, kk = slice(hk * (a // g), (hk + 1) * (a // g)), slice(hk, hk + 1)
        want = attention_plain(q[:, hq].double(), k[:, kk].double(), v[:, kk].double(), starts, None, do[:, hq].double())
        for t in ("o", "lse", "dq", "dk", "dv"):
            got = out[t].cpu().double()
            assert bool((got[:, starts[-1]:] == 7).all() if t == "lse" else (got[starts[-1]:] == 7).all()), t
            if t == "lse":
                inside(t, got[hq, rows], want[t][:, rows], want["_" + t][:, rows])
                continue
            got = got[rows, hq if t in ("o", "dq") else kk]
            inside(t, got, want[t][rows], want["_" + t][rows])
            close(t, got, want[t][rows], U)      # at most three roundings of U/sqrt(3) each
