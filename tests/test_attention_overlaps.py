"""Which arrays one call of the packed or window attention takes together (no GPU needed): every
accepted call here is over a packing without documents, which launches nothing."""
import ctypes as C
import os
import random

import pytest

import paper_2411_06465_amd as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libl4d.so not built")
BASE, N, A, G, D = 1 << 40, 64, 4, 2, 64
NAMES = ("q", "k", "v", "o", "d_o", "dq", "dk", "dv")
HEADS = dict(zip(NAMES, (A, G, G, A, A, A, G, G)))


def place(i, off=0):
    return BASE + (i << 30) + off


@pytest.fixture
def arena():
    ar = C.c_void_p()
    assert L.lib().l4d_arena_create(C.c_void_p(1 << 20), 256, C.byref(ar)) == L.L4D_OK
    yield ar
    L.lib().l4d_arena_destroy(ar)


def rc(call, arena, tokens=N, heads=(A, G), lse=None, starts=None, n_seqs=0, **over):
    """over: name -> (address, row stride)."""
    at = dict(zip(NAMES, [(place(i), HEADS[n] * D) for i, n in enumerate(NAMES)]), **over)
    attn, pk = L.Attn(*heads, D, 0.0), L.PackingC(tokens, n_seqs, starts)
    lse = place(20) if lse is None else lse
    win = [C.byref(L.make_window(10, 2))] if "window" in call else []
    names = NAMES[:4] if call.endswith("fwd") else NAMES
    rows = [x for n in names for x in at[n]]
    fn = getattr(L.lib(), call)
    if call.endswith("fwd"):
        return fn(*win, C.byref(attn), C.byref(pk), *rows, lse, None)
    return fn(*win, C.byref(attn), C.byref(pk), *rows[:8], lse, *rows[8:], arena, None)


def refused(*args, **kw):
    got = rc(*args, **kw)
    return got == L.L4D_EINVAL and "overlap" in L.lib().l4d_last_error().decode()


CALLS = ["attn_packed_fwd", "attn_packed_bwd", "attn_window_fwd", "attn_window_bwd"]


@pytest.mark.parametrize("call", CALLS)
def test_an_output_that_shares_elements_with_another_array_is_refused(call, arena):
    outs = ("o",) if call.endswith("fwd") else ("dq", "dk", "dv")
    names = NAMES[:4] if call.endswith("fwd") else NAMES
    assert rc(call, arena) == L.L4D_OK
    for out in outs:
        for other in names:
            if other == out:
                continue
            p, ld = place(NAMES.index(other)), HEADS[other] * D
            mine = HEADS[out] * D
            for off, stride in ((16, mine), (2 * ld * (N - 1), mine), (16, 512), (-2 * mine * (N - 1), mine)):
                assert refused(call, arena, **{out: (p + off, stride)}), (out, other, off, stride)
            # one behind the other
            assert rc(call, arena, **{out: (p + 2 * ld * N, mine)}) == L.L4D_OK, (out, other)
    lse_bytes, starts = 4 * A * N, place(40)
    for out in outs:
        p, ld = place(NAMES.index(out)), HEADS[out] * D
        assert refused(call, arena, lse=p + 2 * ld * N - 4) and refused(call, arena, lse=p + 4 - lse_bytes)
        assert rc(call, arena, lse=p + 2 * ld * N) == L.L4D_OK and rc(call, arena, lse=p - lse_bytes) == L.L4D_OK
        assert refused(call, arena, starts=p + 8)
        # more documents than a launch holds would be refused for that; a few, on an output
        assert refused(call, arena, n_seqs=5, starts=p - 40)
    if call.endswith("fwd"):
        assert refused(call, arena, lse=place(0, 4)) and refused(call, arena, lse=starts, starts=starts + 8)
    else:
        assert rc(call, arena, lse=place(0, 4)) == L.L4D_OK                  # two inputs


@pytest.mark.parametrize("call", CALLS)
def test_columns_of_fused_arrays_are_taken(call, arena):
    ld = (A + 2 * G) * D
    cols = {n: 2 * D * i for n, i in (("q", 0), ("k", A), ("v", A + G), ("dq", 0), ("dk", A), ("dv", A + G))}
    over = {n: (place(10 if n[0] != "d" else 11, c), ld) for n, c in cols.items()}
    over["o"], over["d_o"] = (place(12), (A + 1) * D), (place(12, 2 * (A + 1) * D * N), (A + 1) * D)
    assert rc(call, arena, **over) == L.L4D_OK, L.lib().l4d_last_error().decode()
    # o in the columns behind v of a wider fused array, q and o in alternate rows of one
    wide = {n: (p, ld + A * D) for n, (p, _) in over.items()}
    wide["o"] = (place(10, 2 * ld), ld + A * D)
    assert rc(call, arena, **wide) == L.L4D_OK
    assert rc(call, arena, **{**over, "q": (place(13), 2 * A * D), "o": (place(13, 2 * A * D), 2 * A * D)}) == L.L4D_OK
    if call.endswith("bwd"):       # dk and dv by a head too far to the left
        assert refused(call, arena, **{**over, "dk": (place(11, 2 * D * (A - 1)), ld)})
        assert refused(call, arena, **{**over, "dv": (place(11, 2 * D * (A + G - 1)), ld)})


@pytest.mark.parametrize("same", [True, False])
def test_the_rule_against_the_elements(same):
    """Small layouts at random, equal and different strides, against the sets of 16-byte units."""
    rng, seen = random.Random(1), [0, 0]
    for _ in range(20000):
        n = rng.randrange(1, 6)
        ld = [8 * rng.randrange(8, 40) for _ in range(2)]
        if same:
            ld[1] = ld[0]
        at = [1 << 16, (1 << 16) + rng.randrange(-160, 161)]           # units of 16 bytes
        if at[0] == at[1]:
            continue
        units = [{p + i * s // 8 + j for i in range(n) for j in range(D // 8)} for p, s in zip(at, ld)]
        bad = bool(units[0] & units[1])
        got = rc("attn_window_fwd", None, tokens=n, heads=(1, 1), q=(BASE + 16 * at[0], ld[0]), o=(BASE + 16 * at[1], ld[1]),
                 k=(place(5), D), v=(place(6), D))
        assert got == (L.L4D_EINVAL if bad else L.L4D_OK), (n, ld, at)
        seen[bad] += 1
    assert min(seen) > 2000
