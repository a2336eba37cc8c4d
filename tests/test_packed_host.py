"""Argument checks of the packed-document operators (no GPU needed).

Every refused call returns before any HIP call, so fake addresses are safe.
"""
import ctypes as C
import math
import os

import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import rope_frequencies

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libl4d.so not built")
BASE = 1 << 40


def at(i, off=0):
    return C.c_void_p(BASE + (i << 30) + off)


def message():
    return L.lib().l4d_last_error().decode()


def pack(tokens=64, n_seqs=2, starts=BASE):
    return L.PackingC(tokens, n_seqs, starts)


# ------------------------------------------------------------------ rotary positions

def rope_rc(rope=None, dtype=0, tokens=64, packing=None, positions=None, q=None, k=None, **kw):
    rope = L.make_rope(**{**dict(head_dim=64), **kw}) if rope is None else rope
    q = L.RopeHeads(BASE, BASE + (1 << 30), 4, 256, 256) if q is None else q
    return L.lib().rope_fwd(C.byref(rope), dtype, tokens, None if packing is None else C.byref(packing), positions,
                            C.byref(q), None if k is None else C.byref(k), None)


def heads(x=BASE, y=BASE + (1 << 30), n=4, x_ld=256, y_ld=256):
    return L.RopeHeads(x, y, n, x_ld, y_ld)


@pytest.mark.parametrize("bad", [
    dict(head_dim=0), dict(head_dim=514), dict(rot_dim=63), dict(rot_dim=0), dict(rot_dim=66), dict(base=1.0),
    dict(base=math.inf), dict(base=math.nan), dict(amplitude=0.0), dict(amplitude=math.nan), dict(amplitude=1e39),
    dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=math.nan),
    dict(scaling="bands", factor=2.0, low=4.0, high=4.0), dict(scaling="bands", factor=2.0, low=0.0),
    dict(scaling="ramp", factor=2.0, original=0.0), dict(scaling="ramp", factor=2.0, high=math.inf)])
def test_rope_refuses_parameters(bad):
    assert rope_rc(**bad) == L.L4D_EINVAL and "rope" in message()


def test_rope_refuses_one_output_for_both():
    assert rope_rc(q=heads(), k=heads()) == L.L4D_EINVAL and "same output" in message()


def test_rope_refuses_arguments():
    r = L.make_rope(64)
    r.layout = 2
    assert rope_rc(r) == L.L4D_EINVAL
    r = L.make_rope(64)
    r.scaling = 4
    assert rope_rc(r) == L.L4D_EINVAL
    assert rope_rc(dtype=2) == L.L4D_EINVAL
    assert rope_rc(tokens=-1) == L.L4D_EINVAL
    assert rope_rc(tokens=(1 << 25) + 1) == L.L4D_EINVAL
    assert rope_rc(packing=pack(63)) == L.L4D_EINVAL
    assert rope_rc(packing=pack(64, 2, None)) == L.L4D_EINVAL
    assert rope_rc(packing=pack(64, -1)) == L.L4D_EINVAL
    assert rope_rc(positions=C.c_void_p(BASE + 4)) == L.L4D_EINVAL
    for q in (heads(x=None), heads(y=None), heads(n=0), heads(n=8193, x_ld=1 << 20, y_ld=1 << 20), heads(x_ld=255), heads(y_ld=255),
              heads(x=BASE + 1), heads(y=BASE + 1), heads(y=BASE + 512), heads(y=BASE, y_ld=512)):
        assert rope_rc(q=q) == L.L4D_EINVAL
        assert rope_rc(k=q) == L.L4D_EINVAL
    assert "overlap" in message()
    assert L.lib().rope_fwd(None, 0, 4, None, None, C.byref(heads()), None, None) == L.L4D_EINVAL
    assert L.lib().rope_bwd(C.byref(L.make_rope(64)), 0, 4, None, None, None, None, None) == L.L4D_EINVAL
    assert rope_rc(tokens=0) == L.L4D_OK                          # nothing to do, nothing launched
    assert rope_rc(packing=pack(64, 0, None)) == L.L4D_OK


def test_the_ramp_is_a_ramp():
    """The plain form the GPU tests use: pairs of many turns keep their angle, slow ones are divided."""
    f, g = rope_frequencies(128, 5e5), rope_frequencies(128, 5e5, "ramp", 8.0, 1.0, 32.0, 8192)
    keep = [(b / a - 1 / 8) / (1 - 1 / 8) for a, b in zip(f, g)]
    assert keep[0] == 1.0 and abs(keep[-1]) < 1e-12 and all(x >= y - 1e-12 for x, y in zip(keep, keep[1:]))


# ------------------------------------------------------------------ packed attention

def attn_rc(backward, attn=(8, 2, 64, 0.0), packing=None, over=None, lse=BASE + (20 << 30), arena=None):
    """over: {tensor index: (pointer, ld)} of q k v o | d_o dq dk dv."""
    a, g, d, scale = attn
    rows = [(BASE + (i << 30), (a if i in (0, 3, 4, 5) else g) * d) for i in range(8)]
    for i, r in (over or {}).items():
        rows[i] = r
    at_ = L.Attn(a, g, d, scale)
    pk = pack() if packing is None else packing
    flat = [x for p, ld in rows[:4] for x in (p, ld)]
    if not backward:
        return L.lib().attn_packed_fwd(C.byref(at_), C.byref(pk), *flat, lse, None)
    tail = [x for p, ld in rows[4:] for x in (p, ld)]
    return L.lib().attn_packed_bwd(C.byref(at_), C.byref(pk), *flat, lse, *tail, arena, None)


@pytest.mark.parametrize("backward", [False, True])
def test_attention_refuses(backward):
    ar = C.c_void_p()
    assert L.lib().l4d_arena_create(C.c_void_p(BASE), 256, C.byref(ar)) == L.L4D_OK

    def rc(**kw):
        return attn_rc(backward, arena=ar, **kw)

    for attn in ((8, 2, 96, 0.0), (8, 3, 64, 0.0), (0, 1, 64, 0.0), (8, 0, 64, 0.0), (1 << 17, 1, 64, 0.0),
                 (8, 2, 64, -1.0), (8, 2, 64, math.nan), (8, 2, 64, math.inf)):
        assert rc(attn=attn) == L.L4D_EINVAL, attn
    for pk in (pack(-1), pack((1 << 30) + 1), pack(64, -1), pack(64, (1 << 30) + 1), pack(64, 2, None),
               pack(64, 2, BASE + 4)):
        assert rc(packing=pk) == L.L4D_EINVAL
    for i in range(8 if backward else 4):
        ld = 512 if i in (0, 3, 4, 5) else 128
        for bad in ((None, ld), (BASE + (9 << 30) + 2, ld), (BASE + (9 << 30), ld - 8), (BASE + (9 << 30), ld + 4),
                    (BASE + (9 << 30), (1 << 22) + 8)):
            assert rc(over={i: bad}) == L.L4D_EINVAL, (i, bad)
    assert rc(lse=None) == L.L4D_EINVAL and rc(lse=BASE + 2) == L.L4D_EINVAL
    out = 5 if backward else 3
    assert rc(over={out: (BASE, 512)}) == L.L4D_EINVAL and "same array" in message()
    # 2^24 blocks and more do not fit a launch
    assert rc(packing=pack(1 << 30)) == L.L4D_EINVAL and "too large" in message()
    assert rc(packing=pack(64, 1 << 24)) == L.L4D_EINVAL
    assert rc(packing=pack(0)) == L.L4D_OK and rc(packing=pack(64, 0, None)) == L.L4D_OK
    if backward:
        assert attn_rc(True, arena=None) == L.L4D_EINVAL
        assert rc() == L.L4D_ENOMEM                       # 256 bytes do not hold the workspace
    L.lib().l4d_arena_destroy(ar)


def test_attention_workspace():
    n = L.l4d_attn_packed_workspace_bytes(4096, 32, 8, 128)
    assert n >= 4096 * 32 * 4
    # 128 blocks of keys of one kv head: its 8 query heads go into slices with fp32 partial sums
    assert L.l4d_attn_packed_workspace_bytes(16384, 8, 1, 128) >= 2 * 2 * 16384 * 128 * 4
    assert L.l4d_attn_packed_workspace_bytes(0, 8, 1, 64) == 0
    with pytest.raises(L.L4DError):
        L.l4d_attn_packed_workspace_bytes(16, 8, 3, 64)
    with pytest.raises(L.L4DError):
        L.l4d_attn_packed_workspace_bytes(-1, 8, 1, 64)


# ------------------------------------------------------------------ loss without stored logits

def loss_rc(backward, n=64, h=64, v=100, v0=0, over=None, peers=(None, None), scale=1.0, arena=None):
    ptr = [at(i) for i in range(6)]      # hidden w targets | loss lse ; lse d_hidden d_w
    for i, p in (over or {}).items():
        ptr[i] = p
    if backward:
        return L.lib().lm_loss_bwd(n, h, v, v0, *ptr[:4], None, scale, ptr[4], ptr[5], arena, None)
    return L.lib().lm_loss_fwd(n, h, v, v0, *ptr[:3], *peers, ptr[3], ptr[4], None, arena, None)


@pytest.mark.parametrize("backward", [False, True])
def test_loss_refuses(backward):
    ar = C.c_void_p()
    assert L.lib().l4d_arena_create(C.c_void_p(BASE), 256, C.byref(ar)) == L.L4D_OK
    for bad in (dict(n=-1), dict(h=0), dict(h=12), dict(h=8200), dict(v=0), dict(v0=-1), dict(n=(1 << 20) + 1),
                dict(v=(1 << 24) + 1)):
        assert loss_rc(backward, arena=ar, **bad) == L.L4D_EINVAL, bad
    align = [16, 16, 8, 4, 16, 4] if backward else [16, 16, 8, 4, 4]
    for i, a in enumerate(align):
        assert loss_rc(backward, arena=ar, over={i: None}) == L.L4D_EINVAL, i
        assert loss_rc(backward, arena=ar, over={i: at(i, a // 2)}) == L.L4D_EINVAL, i
    if backward:
        assert loss_rc(True, arena=ar, scale=math.nan) == L.L4D_EINVAL
    else:
        assert loss_rc(False, arena=ar, peers=(at(8), None)) == L.L4D_EINVAL
        assert loss_rc(False, arena=ar, peers=(None, at(8))) == L.L4D_EINVAL
    assert loss_rc(backward, arena=None) == L.L4D_EINVAL
    assert loss_rc(backward, n=0, arena=ar) == L.L4D_OK
    assert loss_rc(backward, arena=ar) == L.L4D_ENOMEM
    L.lib().l4d_arena_destroy(ar)


def test_loss_gradient_is_no_input():
    ar = C.c_void_p()
    assert L.lib().l4d_arena_create(C.c_void_p(BASE), 256, C.byref(ar)) == L.L4D_OK
    for i in (0, 1):
        assert loss_rc(True, arena=ar, over={4: at(i)}) == L.L4D_EINVAL and "d_hidden" in message()
    L.lib().l4d_arena_destroy(ar)


def test_loss_workspace_does_not_grow_with_the_logits():
    n, v = 65536, 128256
    f, b = L.l4d_lm_loss_workspace_bytes(n, 4096, v)
    # 8192 columns of gradient in two parts, fp32 d_hidden, hidden twice; bf16 logits would be 2 n v = 16.8 GB
    assert f < n * v / 4 and b <= n * (8192 * 4 + 4096 * 8 + 4) + 4096
    for bad in ((-1, 64, 8), (4, 12, 8), (4, 64, 0)):
        with pytest.raises(L.L4DError):
            L.l4d_lm_loss_workspace_bytes(*bad)


# ------------------------------------------------------------------ the binding's own checks

def test_the_binding_refuses_other_layouts():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        L.make_packing(torch.zeros(2, dtype=torch.int32), 4)
    with pytest.raises(ValueError):
        L.make_packing(torch.zeros(2, 2, dtype=torch.int64), 4)
    pk, lse = L.make_packing(torch.zeros(2, dtype=torch.int64), 4), torch.zeros(2, 4)
    with pytest.raises(ValueError):
        L.attn_packed_fwd(x, x, x, x.transpose(1, 2), lse, pk)
    with pytest.raises(TypeError):
        L.attn_packed_fwd(x, x, x.float(), x.clone(), lse, pk)
    with pytest.raises(ValueError):
        L.attn_packed_fwd(x, x[:3], x[:3], x.clone(), lse, pk)
    with pytest.raises(ValueError):
        L.attn_packed_fwd(x, x, x, x.clone(), lse.t().contiguous(), pk)
    with pytest.raises(TypeError):
        L.rope_fwd(L.make_rope(64), x.half())
    with pytest.raises(ValueError):
        L.rope_fwd(L.make_rope(128), x)
    with pytest.raises(ValueError):
        L.rope_fwd(L.make_rope(64), x, x.clone(), positions=torch.zeros(3, dtype=torch.int64))
    h, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(5, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        L.lm_loss_fwd(h, w, torch.zeros(3, dtype=torch.int64), torch.zeros(4), torch.zeros(4), None)
    with pytest.raises(TypeError):
        L.lm_loss_fwd(h, w, torch.zeros(4, dtype=torch.int32), torch.zeros(4), torch.zeros(4), None)
    with pytest.raises(ValueError):
        L.lm_loss_fwd(h, w.repeat(1, 2)[:, ::2], torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(4), None)
