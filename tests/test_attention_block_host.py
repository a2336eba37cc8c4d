"""Argument checks of the norms of heads, rotary axes, window attention and dropout (no GPU needed).

Every refused call returns before any HIP call, so fake addresses are safe.
"""
import ctypes as C
import math
import os

import pytest
import torch

import paper_2411_06465_amd as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libl4d.so not built")
BASE = 1 << 40


def at(i, off=0):
    return BASE + (i << 30) + off


def message():
    return L.lib().l4d_last_error().decode()


def pack(tokens=64, n_seqs=2, starts=BASE + (60 << 30)):
    return L.PackingC(tokens, n_seqs, starts)


@pytest.fixture
def arena():
    ar = C.c_void_p()
    assert L.lib().l4d_arena_create(C.c_void_p(BASE), 256, C.byref(ar)) == L.L4D_OK
    yield ar
    L.lib().l4d_arena_destroy(ar)


# ------------------------------------------------------------------ window attention

def window_rc(backward, window=(10, 2), attn=(8, 2, 64, 0.0), packing=None, over=None, lse=at(20), arena=None, none=False):
    a, g, d, scale = attn
    rows = [(at(i), (a if i in (0, 3, 4, 5) else g) * d) for i in range(8)]
    for i, r in (over or {}).items():
        rows[i] = r
    win = None if none else C.byref(L.make_window(*window))
    at_, pk = L.Attn(a, g, d, scale), pack() if packing is None else packing
    flat = [x for p, ld in rows[:4] for x in (p, ld)]
    if not backward:
        return L.lib().attn_window_fwd(win, C.byref(at_), C.byref(pk), *flat, lse, None)
    tail = [x for p, ld in rows[4:] for x in (p, ld)]
    return L.lib().attn_window_bwd(win, C.byref(at_), C.byref(pk), *flat, lse, *tail, arena, None)


@pytest.mark.parametrize("backward", [False, True])
def test_window_attention_refuses(backward, arena):
    def rc(**kw):
        return window_rc(backward, arena=arena, **kw)

    assert rc(none=True) == L.L4D_EINVAL
    for window in ((0, 0), (-5, 0), (10, -1), (10, 4097), (1 << 40, 4097)):
        assert rc(window=window) == L.L4D_EINVAL, window
    for attn in ((8, 2, 96, 0.0), (8, 3, 64, 0.0), (0, 1, 64, 0.0), (8, 2, 64, -1.0), (8, 2, 64, math.nan)):
        assert rc(attn=attn) == L.L4D_EINVAL, attn
    for pk in (pack(-1), pack((1 << 30) + 1), pack(64, -1), pack(64, 2, None)):
        assert rc(packing=pk) == L.L4D_EINVAL
    for i in range(8 if backward else 4):
        ld = 512 if i in (0, 3, 4, 5) else 128
        for bad in ((None, ld), (at(9, 2), ld), (at(9), ld - 8), (at(9), ld + 4), (at(9), (1 << 22) + 8)):
            assert rc(over={i: bad}) == L.L4D_EINVAL, (i, bad)
    assert rc(lse=None) == L.L4D_EINVAL
    assert rc(over={5 if backward else 3: (at(0), 512)}) == L.L4D_EINVAL and "same array" in message()
    assert rc(packing=pack((1 << 28) + 1), attn=(1, 1, 64, 0.0)) == L.L4D_EINVAL and "too large" in message()
    assert rc(packing=pack(0)) == L.L4D_OK and rc(packing=pack(64, 0, None)) == L.L4D_OK
    if backward:
        assert window_rc(True, arena=None) == L.L4D_EINVAL
        assert rc() == L.L4D_ENOMEM                       # 256 bytes do not hold the workspace


def test_window_workspace():
    def size(window, sinks, tokens, *heads):
        return L.l4d_attn_window_workspace_bytes(L.make_window(window, sinks), tokens, *heads)

    plain = L.l4d_attn_packed_workspace_bytes(4096, 32, 8, 128)
    assert size(4096, 4, 4096, 32, 8, 128) == plain                    # hides nothing
    assert size(100, 0, 4096, 32, 8, 128) >= plain
    # parts of the first tokens' sums: no more than the sums of all rows would take
    for sinks in (1, 16, 128, 4096):
        more = size(100, sinks, 40000, 8, 8, 64) - size(100, 0, 40000, 8, 8, 64)
        assert 0 < more <= 1.1 * 2 * 40000 * 8 * 64 * 4 + (1 << 20), sinks
    assert size(10, 2, 0, 8, 1, 64) == 0
    for bad in ((0, 0, 16, 8, 1, 64), (4, -1, 16, 8, 1, 64), (4, 0, -1, 8, 1, 64), (4, 0, 16, 8, 3, 64)):
        with pytest.raises(L.L4DError):
            size(*bad)


# ------------------------------------------------------------------ rotary axes

def axes_rc(pairs=(16, 16), order="sections", frequencies="shared", positions=at(50), rope=None, change=None, call="rope_axes_fwd",
            none=False, tokens=64):
    rope = L.make_rope(64) if rope is None else rope
    axes = L.make_rope_axes(pairs, order, frequencies)
    for name, v in (change or {}).items():
        setattr(axes, name, v)
    q = L.RopeHeads(at(0), at(1), 4, 256, 256)
    return getattr(L.lib(), call)(C.byref(rope), None if none else C.byref(axes), 0, tokens, C.byref(pack(tokens, 0, None)),
                                  positions, C.byref(q), None, None)


@pytest.mark.parametrize("call", ["rope_axes_fwd", "rope_axes_bwd"])
def test_axes_refuse(call):
    def rc(**kw):
        return axes_rc(call=call, **kw)

    assert rc() == L.L4D_OK
    assert rc(none=True) == L.L4D_EINVAL and rc(positions=None) == L.L4D_EINVAL and rc(positions=at(50, 4)) == L.L4D_EINVAL
    for pairs in ((16, 15), (32, 0), (33, -1), (0, 32), (16, 16, 16)):
        assert rc(pairs=pairs) == L.L4D_EINVAL, pairs
    for change in (dict(n_axes=0), dict(n_axes=5), dict(n_axes=1), dict(order=2), dict(order=-1), dict(frequencies=2)):
        assert rc(change=change) == L.L4D_EINVAL, change
    # dealt in turn: the last of an axis' pairs would lie behind the head's
    assert rc(pairs=(10, 11, 11), order="cycled") == L.L4D_EINVAL and "dealt" in message()
    assert rc(pairs=(11, 11, 10), order="cycled") == L.L4D_OK and rc(pairs=(24, 4, 4), order="cycled") == L.L4D_OK
    assert rc(pairs=(32,), order="cycled", frequencies="own") == L.L4D_OK
    assert rc(rope=L.make_rope(64, 32)) == L.L4D_EINVAL and rc(rope=L.make_rope(64, base=1.0)) == L.L4D_EINVAL


# ------------------------------------------------------------------ norms of heads

def norm_rc(backward, arena=None, rope=None, dtype=0, tokens=64, packing=None, positions=None, eps=1e-6, q=None, k=None, axes=None):
    rope = L.make_rope(64) if rope is None else rope
    fn = L.lib().qk_norm_rope_bwd if backward else L.lib().qk_norm_rope_fwd
    args = [C.byref(rope), None if axes is None else C.byref(axes), dtype, tokens, None if packing is None else C.byref(packing),
            positions, eps]
    return fn(*args, *[None if t is None else C.byref(t) for t in (heads(backward) if q is None else q, k)],
              *([arena] if backward else []), None)


def heads(backward, **over):
    """q with four heads of 64: x at 0, gain at 1, dy at 2, the output at 3, d_gain at 4."""
    v = dict(x=at(0), gain=at(1), dy=at(2), out=at(3), d_gain=at(4), heads=4, x_ld=256, dy_ld=256, out_ld=256)
    v.update(over)
    if backward:
        return L.NormHeadsGrad(v["x"], v["gain"], v["dy"], v["out"], v["d_gain"], v["heads"], v["x_ld"], v["dy_ld"], v["out_ld"])
    return L.NormHeads(v["x"], v["gain"], v["out"], v["heads"], v["x_ld"], v["out_ld"])


@pytest.mark.parametrize("backward", [False, True])
def test_norm_refuses(backward, arena):
    none = pack(64, 0, None)

    def rc(**kw):
        return norm_rc(backward, arena, packing=kw.pop("packing", none), **kw)

    def h(**over):
        return heads(backward, **over)

    assert rc() == L.L4D_OK and rc(k=h(x=at(10), gain=at(11), dy=at(12), out=at(13), d_gain=at(14))) == L.L4D_OK
    assert rc(k=h(x=at(10), dy=at(12), out=at(13), d_gain=at(14))) == L.L4D_OK            # one gain for both
    for rope in (L.make_rope(65, 64), L.make_rope(514), L.make_rope(64, 63), L.make_rope(64, base=0.5)):
        assert rc(rope=rope) == L.L4D_EINVAL
    for bad in (dict(dtype=2), dict(tokens=-1), dict(tokens=(1 << 25) + 1), dict(packing=pack(63)), dict(packing=pack(64, 2, None)),
                dict(positions=at(50, 4)), dict(axes=L.make_rope_axes((16, 16)))):
        assert rc(**bad) == L.L4D_EINVAL, bad
    for eps in (0.0, -1e-6, math.nan, math.inf, 1e-31):
        assert rc(eps=eps) == L.L4D_EINVAL and "eps" in message(), eps
    wrong = [dict(x=None), dict(out=None), dict(gain=None), dict(heads=0), dict(heads=8193, x_ld=1 << 20, out_ld=1 << 20, dy_ld=1 << 20),
             dict(x_ld=255), dict(out_ld=255), dict(x=at(0, 1)), dict(out=at(3, 1)), dict(gain=at(1, 1)), dict(x_ld=(1 << 31) + 2)]
    if backward:
        wrong += [dict(dy=None), dict(d_gain=None), dict(dy_ld=255), dict(dy=at(2, 1)), dict(d_gain=at(4, 2))]
    for over in wrong:
        assert rc(q=h(**over)) == L.L4D_EINVAL, over
        assert rc(k=h(**over)) == L.L4D_EINVAL, over
    # an output on an input of its own tensor, with the same rows, and on nothing else
    assert rc(q=h(out=at(0))) == L.L4D_OK
    assert rc(q=h(out=at(0), out_ld=512)) == L.L4D_EINVAL and rc(q=h(out=at(0, 512))) == L.L4D_EINVAL
    assert rc(q=h(out=at(1))) == L.L4D_EINVAL and rc(q=h(gain=at(3, 64))) == L.L4D_EINVAL
    other = dict(x=at(10), gain=at(11), dy=at(12), out=at(13), d_gain=at(14))
    for over in (dict(out=at(0)), dict(out=at(3)), dict(x=at(3)), dict(out=at(1)), dict(out=at(3, 128))):
        assert rc(k=h(**{**other, **over})) == L.L4D_EINVAL and "overlap" in message(), over
    # columns of one array
    assert rc(q=h(out=at(0), x_ld=512, out_ld=512), k=h(**{**other, "x": at(0, 512), "out": at(0, 512), "heads": 2, "x_ld": 512, "out_ld": 512})) == L.L4D_OK
    assert rc(q=h(out=at(0), x_ld=512, out_ld=512), k=h(**{**other, "x": at(0, 384), "out": at(0, 384), "heads": 2, "x_ld": 512, "out_ld": 512})) == L.L4D_EINVAL
    if backward:
        assert rc(q=h(out=at(2))) == L.L4D_OK
        for over in (dict(dy=at(3)), dict(out=at(2)), dict(d_gain=at(4)), dict(out=at(4)), dict(gain=at(4))):
            assert rc(k=h(**{**other, **over})) == L.L4D_EINVAL, over
        for over in (dict(d_gain=at(1)), dict(d_gain=at(0, 512)), dict(d_gain=at(2, 4)), dict(d_gain=at(3))):
            assert rc(q=h(**over)) == L.L4D_EINVAL, over
        assert norm_rc(True, None, packing=none) == L.L4D_EINVAL and "arena" in message()
        assert norm_rc(True, arena) == L.L4D_ENOMEM
    fn = L.lib().qk_norm_rope_bwd if backward else L.lib().qk_norm_rope_fwd
    assert fn(C.byref(L.make_rope(64)), None, 0, 4, None, None, 1e-6, None, None, *([arena] if backward else []), None) == L.L4D_EINVAL
    assert norm_rc(backward, arena, tokens=0, q=h(x=None, out=None)) == L.L4D_OK      # an empty array may have no address


def test_norm_workspace():
    assert L.l4d_qk_norm_workspace_bytes(0, 64) == 0
    assert 8 * 128 <= L.l4d_qk_norm_workspace_bytes(1, 128) <= L.l4d_qk_norm_workspace_bytes(1 << 25, 128) <= 1 << 20
    for bad in ((-1, 64), (4, 0), (4, 514), ((1 << 25) + 1, 64)):
        with pytest.raises(L.L4DError):
            L.l4d_qk_norm_workspace_bytes(*bad)


# ------------------------------------------------------------------ dropout

def drop_rc(backward=False, dtype=0, rows=8, cols=16, x=at(0), x_ld=None, res=at(1), r_ld=None, y=at(2), y_ld=None, p=0.1, rng=at(3),
            first=0):
    x_ld, r_ld, y_ld = (cols if v is None else v for v in (x_ld, r_ld, y_ld))
    if backward:
        return L.lib().dropout_add_bwd(dtype, rows, cols, x, x_ld, y, y_ld, p, rng, first, None)
    return L.lib().dropout_add_fwd(dtype, rows, cols, x, x_ld, res, r_ld, y, y_ld, p, rng, first, None)


@pytest.mark.parametrize("backward", [False, True])
def test_dropout_refuses(backward):
    def rc(**kw):
        return drop_rc(backward, **kw)

    for bad in (dict(dtype=2), dict(rows=-1), dict(cols=-1), dict(rows=(1 << 31) + 1), dict(cols=(1 << 24) + 1),
                dict(rows=1 << 20, cols=1 << 15), dict(p=-0.1), dict(p=1.0), dict(p=math.nan), dict(p=1.0 - 2.0 ** -40), dict(p=2.0),
                dict(first=-1), dict(first=(1 << 38) + 1), dict(x=None), dict(y=None), dict(rng=None), dict(rng=at(3, 4)),
                dict(x=at(0, 1)), dict(y=at(2, 1)), dict(x_ld=15), dict(y_ld=15), dict(x_ld=(1 << 31) + 1), dict(dtype=1, x=at(0, 2)),
                dict(y=at(0, 2)), dict(y=at(0), y_ld=32), dict(y=at(3)), dict(y=at(3, 16 - 256))):
        assert rc(**bad) == L.L4D_EINVAL and "dropout" in message(), bad
    if not backward:
        for bad in (dict(res=at(1, 1)), dict(r_ld=15), dict(y=at(1), y_ld=32), dict(y=at(1, 2))):
            assert rc(**bad) == L.L4D_EINVAL, bad
    assert rc(rows=0, x=None, y=None) == L.L4D_OK and rc(cols=0, x=None, y=None) == L.L4D_OK


# ------------------------------------------------------------------ the binding's own checks

def test_the_binding_refuses_other_layouts():
    bf, f32, i64 = torch.bfloat16, torch.float32, torch.int64
    x = torch.zeros(4, 2, 64, dtype=bf)
    pk, lse = L.make_packing(torch.zeros(2, dtype=i64), 4), torch.zeros(2, 4)
    win, rope, axes, gain = L.make_window(2, 1), L.make_rope(64), L.make_rope_axes((16, 16)), torch.ones(64, dtype=bf)
    for args, error in (((x, x, x, x.transpose(1, 2), lse, pk), ValueError), ((x, x, x.float(), x.clone(), lse, pk), TypeError),
                        ((x, x[:3], x[:3], x.clone(), lse, pk), ValueError), ((x, x, x, x.clone(), lse.t(), pk), ValueError)):
        with pytest.raises(error):
            L.attn_window_fwd(win, *args)
    pos = torch.zeros(2, 4, dtype=i64)
    for args, error in (((x, pos[0]), ValueError), ((x, pos.to(torch.int32)), TypeError), ((x.half(), pos), TypeError),
                        ((x[:3], pos), ValueError), ((x, None), ValueError), ((torch.zeros(4, 2, 32, dtype=bf), pos), ValueError)):
        with pytest.raises(error):
            L.rope_axes_fwd(rope, axes, *args)
    for pairs in ((), (1, 2, 3, 4, 5)):
        with pytest.raises(ValueError):
            L.make_rope_axes(pairs)
    with pytest.raises(KeyError):
        L.make_rope_axes((4, 4), "turned")
    for kw, error in ((dict(q_gain=None), ValueError), (dict(q_gain=gain.float()), TypeError), (dict(q_gain=gain[:32]), ValueError),
                      (dict(q=x.half()), TypeError), (dict(q_out=x.float()), TypeError), (dict(k=x), ValueError),
                      (dict(k=x[:3], k_gain=gain), ValueError), (dict(axes=axes), ValueError), (dict(positions=pos), ValueError)):
        with pytest.raises(error):
            L.qk_norm_rope_fwd(rope, **{**dict(q=x, q_gain=gain), **kw})
    dg = torch.zeros(64)
    for kw, error in ((dict(d_q_gain=None), ValueError), (dict(d_q_gain=dg.to(bf)), TypeError), (dict(dq=x[:3]), ValueError),
                      (dict(dq_out=x.float()), TypeError)):
        with pytest.raises(error):
            L.qk_norm_rope_bwd(rope, **{**dict(q=x, q_gain=gain, dq_out=x.clone(), dq=x.clone(), d_q_gain=dg, arena=None), **kw})
    m, rng = torch.zeros(4, 8), torch.zeros(2, dtype=i64)
    for args, error in (((m[0], None, m[0], rng), ValueError), ((m.double(), None, m.double(), rng), TypeError),
                        ((m, m[:3], m.clone(), rng), ValueError), ((m, m.to(bf), m.clone(), rng), TypeError),
                        ((m, None, torch.zeros(8, 4).t(), rng), ValueError), ((m, None, m.clone(), rng[:1]), ValueError),
                        ((m, None, m.clone(), rng.to(torch.int32)), TypeError), ((m, None, torch.zeros(1, 8).expand(4, 8), rng), ValueError)):
        with pytest.raises(error):
            L.dropout_add_fwd(*args, 0.5)
