"""Rotary and norm calls whose outputs lie on the positions or the documents' starts that the same
launch reads (no GPU needed): every accepted call here is over a packing without documents, which
launches nothing."""
import ctypes as C
import os

import pytest

import paper_2411_06465_amd as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libl4d.so not built")
BASE, N, H, D = 1 << 40, 64, 4, 64
ROW = 2 * H * D                          # bytes of a row


def place(i, off=0):
    return BASE + (i << 30) + off


@pytest.fixture
def arena():
    ar = C.c_void_p()
    assert L.lib().l4d_arena_create(C.c_void_p(1 << 20), 256, C.byref(ar)) == L.L4D_OK
    yield ar
    L.lib().l4d_arena_destroy(ar)


def rc(call, arena, positions, starts, n_seqs=0, out=place(1), ld=H * D, axes=None, second=None):
    """second: the output of a k beside q."""
    rope, pk = L.make_rope(D), L.PackingC(N, n_seqs, starts)
    ax = L.make_rope_axes((16, 16)) if axes else None
    ax = None if ax is None else C.byref(ax)
    if call.startswith("rope"):
        t = [L.RopeHeads(place(0), out, H, H * D, ld), L.RopeHeads(place(2), second, H, H * D, H * D)]
        extra = [ax] if axes else []
        return getattr(L.lib(), call)(C.byref(rope), *extra, 0, N, C.byref(pk), positions, C.byref(t[0]),
                                      C.byref(t[1]) if second else None, None)
    head = [C.byref(rope), ax, 0, N, C.byref(pk), positions, 1e-6]
    if call == "qk_norm_rope_fwd":
        t = [L.NormHeads(place(0), place(5), out, H, H * D, ld), L.NormHeads(place(2), place(6), second, H, H * D, H * D)]
        return L.lib().qk_norm_rope_fwd(*head, C.byref(t[0]), C.byref(t[1]) if second else None, None)
    t = [L.NormHeadsGrad(place(0), place(5), place(7), out, place(9), H, H * D, H * D, ld),
         L.NormHeadsGrad(place(2), place(6), place(8), second, place(10), H, H * D, H * D, H * D)]
    return L.lib().qk_norm_rope_bwd(*head, C.byref(t[0]), C.byref(t[1]) if second else None, arena, None)


CALLS = [("rope_fwd", 0), ("rope_bwd", 0), ("rope_axes_fwd", 2), ("rope_axes_bwd", 2), ("qk_norm_rope_fwd", 0),
         ("qk_norm_rope_fwd", 2), ("qk_norm_rope_bwd", 0), ("qk_norm_rope_bwd", 2)]


@pytest.mark.parametrize("call,axes", CALLS)
def test_an_output_on_positions_or_starts_is_refused(call, axes, arena):
    def refused(**kw):
        got = rc(call, arena, axes=axes, **{**dict(positions=place(20), starts=place(21)), **kw})
        return got == L.L4D_EINVAL and "overlap" in L.lib().l4d_last_error().decode()

    def taken(**kw):
        return rc(call, arena, axes=axes, **{**dict(positions=place(20), starts=place(21)), **kw}) == L.L4D_OK

    size = 8 * N * max(1, axes)                                  # of the positions
    assert taken() and taken(second=place(3)) and taken(positions=place(21))          # inputs may share
    for where in (dict(out=place(15)), dict(second=place(15))):
        assert refused(positions=place(15, N * ROW - 8), **where) and refused(positions=place(15, 8 - size), **where)
        assert taken(positions=place(15, N * ROW), **where) and taken(positions=place(15, -size), **where)
        assert refused(starts=place(15, N * ROW - 8), **where) and refused(starts=place(15), **where)
        assert taken(starts=place(15, N * ROW), **where) and taken(starts=place(15, -8), **where)
    # the documents' starts between the rows of a strided output, which they are no part of
    assert taken(starts=place(15, ROW), out=place(15), ld=H * D + 4)
    assert refused(starts=place(15, ROW - 8), out=place(15), ld=H * D + 4)
    if not axes:
        assert taken(positions=None)
    if call == "qk_norm_rope_bwd":
        assert refused(positions=place(9)) and refused(starts=place(9, 4 * D - 8)) and taken(starts=place(9, 4 * D))


@pytest.mark.parametrize("call,axes", CALLS)
def test_all_starts_count(call, axes, arena):
    """Three documents: four starts, of which the last lies on the output."""
    got = rc(call, arena, place(20), place(1, -24), n_seqs=3, axes=axes)
    assert got == L.L4D_EINVAL and "overlap" in L.lib().l4d_last_error().decode()
