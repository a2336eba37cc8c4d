"""Which arrays of q and k one rotary call takes together (no GPU needed): every accepted
call here is over a packing without documents, which launches nothing."""
import ctypes as C
import os
import random

import pytest

import paper_2411_06465_amd as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libl4d.so not built")
BASE = 1 << 40


def rc(n, q, k, call="rope_fwd", d=64):
    """q, k: (x, y, heads, x_ld, y_ld) with x and y as bf16 elements from one address on."""
    heads = [L.RopeHeads(BASE + 2 * x, BASE + 2 * y, h, x_ld, y_ld) for x, y, h, x_ld, y_ld in (q, k)]
    return getattr(L.lib(), call)(C.byref(L.make_rope(d)), 0, n, C.byref(L.PackingC(n, 0, None)), None,
                                  C.byref(heads[0]), C.byref(heads[1]), None)


A, B, G, D = 0, 1 << 24, 1 << 25, 1 << 26      # four arrays apart


@pytest.mark.parametrize("call", ["rope_fwd", "rope_bwd"])
@pytest.mark.parametrize("q,k", [
    ((A, B, 4, 256, 256), (B, G, 4, 256, 256)),              # q's output is k's input
    ((A, B, 4, 256, 256), (G, A, 4, 256, 256)),              # k's output is q's input
    ((A, A, 4, 256, 256), (A, B, 4, 256, 256)),              # q in place where k is read
    ((A, B, 4, 256, 256), (G, B + 64, 4, 256, 256)),         # outputs that overlap in part
    ((A, B, 4, 256, 256), (G, B + 128, 2, 512, 512)),        # other strides, ranges that meet
    ((A, B, 4, 256, 256), (G, B + 256 * 63, 1, 64, 64)),     # the last row only
    ((A, A, 4, 512, 512), (A + 192, A + 192, 2, 512, 512)),  # columns of one array that share a head
])
def test_an_output_that_is_the_other_tensors_is_refused(call, q, k):
    assert rc(64, q, k, call) == L.L4D_EINVAL and "overlap" in L.lib().l4d_last_error().decode()


@pytest.mark.parametrize("q,k", [
    ((A, B, 4, 256, 256), (G, D, 2, 128, 128)),
    ((A, B, 4, 256, 256), (A, G, 4, 256, 256)),              # one input for both
    ((A, A, 4, 512, 512), (A + 256, A + 256, 2, 512, 512)),  # columns of one fused array, in place
    ((A + 256, A + 256, 4, 512, 512), (A + 128, A + 128, 2, 512, 512)),
    ((A, B, 4, 512, 512), (A + 256, B + 256, 2, 512, 512)),  # from one fused array into another
    ((A, B, 4, 256, 256), (G, B + 64 * 256, 2, 128, 128)),   # one behind the other
])
def test_arrays_that_share_nothing_written_are_taken(q, k):
    assert rc(64, q, k) == L.L4D_OK, L.lib().l4d_last_error().decode()


def test_the_rule_against_the_elements():
    """Small layouts at random, against the sets of elements that a call reads and writes."""
    rng, seen = random.Random(1), [0, 0]
    for _ in range(20000):
        n, ld = rng.randrange(1, 5), rng.randrange(4, 14)
        hq, hk = rng.randrange(1, 3), rng.randrange(1, 3)
        ld = max(ld, 2 * max(hq, hk))
        qx, kx = 1000, 1000 + rng.randrange(-50, 51)         # in place, d = 2, one stride
        sets = [{x + i * ld + j for i in range(n) for j in range(2 * h)} for x, h in ((qx, hq), (kx, hk))]
        bad = bool(sets[0] & sets[1])
        got = rc(n, (qx, qx, hq, ld, ld), (kx, kx, hk, ld, ld), d=2)
        assert got == (L.L4D_EINVAL if bad else L.L4D_OK), (n, ld, hq, hk, kx)
        seen[bad] += 1
    assert min(seen) > 2000
