"""Calls around the attention over no tokens at all, whose arrays have no address: nothing is
launched and nothing refused.  The shapes are checked as ever."""
import ctypes as C
import os

import pytest
import torch

import paper_2411_06465_amd as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libl4d.so not built")
H, G, D = 4, 2, 64


@pytest.mark.parametrize("direction", ["fwd", "bwd"])
@pytest.mark.parametrize("axes", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_rotary_calls_and_norms(direction, axes, packed):
    rope, ax = L.make_rope(D), L.make_rope_axes((16, 16))
    pk = C.byref(L.PackingC(0, 0, None)) if packed else None
    turn = [C.byref(L.RopeHeads(None, None, h, h * D, h * D)) for h in (H, G)]
    head = [C.byref(rope)] + ([C.byref(ax)] if axes else [])
    name = "rope_axes_" if axes else "rope_"
    assert getattr(L.lib(), name + direction)(*head, 0, 0, pk, None, *turn, None) == L.L4D_OK, L.lib().l4d_last_error().decode()
    args = [C.byref(rope), C.byref(ax) if axes else None, 0, 0, pk, None, 1e-6]
    if direction == "fwd":
        t = [C.byref(L.NormHeads(None, 1 << 20, None, h, h * D, h * D)) for h in (H, G)]
        assert L.lib().qk_norm_rope_fwd(*args, *t, None) == L.L4D_OK, L.lib().l4d_last_error().decode()
    else:
        t = [C.byref(L.NormHeadsGrad(None, 1 << 20, None, None, 1 << 21, h, h * D, h * D, h * D)) for h in (H, G)]
        assert L.lib().qk_norm_rope_bwd(*args, *t, None, None) == L.L4D_OK, L.lib().l4d_last_error().decode()


def test_rotary_calls_still_check_their_arguments():
    t = C.byref(L.RopeHeads(None, None, H, H * D, H * D))
    ax = L.make_rope_axes((16, 15))
    assert L.lib().rope_fwd(C.byref(L.make_rope(D, 63)), 0, 0, None, None, t, None, None) == L.L4D_EINVAL
    assert L.lib().rope_axes_fwd(C.byref(L.make_rope(D)), C.byref(ax), 0, 0, None, None, t, None, None) == L.L4D_EINVAL


@pytest.mark.parametrize("window", [False, True])
def test_attention(window):
    pk, lib = C.byref(L.PackingC(0, 0, None)), L.lib()
    win = [C.byref(L.make_window(5, 1))] if window else []
    name = "attn_window_" if window else "attn_packed_"

    def rows(*heads):
        return [x for h in heads for x in (None, h * D)]

    def both(attn, win):
        f = getattr(lib, name + "fwd")(*win, C.byref(attn), pk, *rows(H, G, G, H), None, None)
        b = getattr(lib, name + "bwd")(*win, C.byref(attn), pk, *rows(H, G, G, H), None, *rows(H, H, G, G), None, None)
        return f, b

    assert both(L.Attn(H, G, D, 0.0), win) == (L.L4D_OK, L.L4D_OK), lib.l4d_last_error().decode()
    assert both(L.Attn(H, G, 96, 0.0), win) == (L.L4D_EINVAL, L.L4D_EINVAL)
    if window:
        assert both(L.Attn(H, G, D, 0.0), [C.byref(L.make_window(0, 1))]) == (L.L4D_EINVAL, L.L4D_EINVAL)


@pytest.mark.gpu
def test_empty_tensors_through_the_binding():
    q, k = (torch.empty((0, h, D), dtype=torch.bfloat16, device="cuda") for h in (H, G))
    gain, dg = torch.ones(D, dtype=torch.bfloat16, device="cuda"), torch.full((D,), 3.0, device="cuda")
    pk, rope = L.make_packing(torch.zeros(1, dtype=torch.int64, device="cuda"), 0), L.make_rope(D)
    axes, pos = L.make_rope_axes((16, 16)), torch.empty((2, 0), dtype=torch.int64, device="cuda")
    arena = L.Arena.on(torch.empty(256, dtype=torch.uint8, device="cuda"))
    L.rope_fwd(rope, q, k=k)
    L.rope_axes_bwd(rope, axes, q, pos, dk=k, packing=pk)
    L.qk_norm_rope_fwd(rope, q, gain, None, k, gain, positions=pos, axes=axes, packing=pk)
    L.qk_norm_rope_bwd(rope, q, gain, q.clone(), q.clone(), dg, arena, positions=pos, axes=axes)
    lse, win = torch.empty((H, 0), device="cuda"), L.make_window(3)
    L.attn_window_fwd(win, q, k, k, q.clone(), lse, pk)
    L.attn_window_bwd(win, q, k, k, q, lse, q, q.clone(), k.clone(), k.clone(), pk, arena)
    x = torch.empty((0, 8), device="cuda")
    L.dropout_add_fwd(x, x, x, torch.zeros(2, dtype=torch.int64, device="cuda"), 0.5)
    torch.cuda.synchronize()
    assert bool((dg == 3.0).all())
