"""The dK/dV pass of packed attention replayed on the host (no GPU needed): the cut of
the key blocks that attn_packed_plan picks, the list of blocks, the launch's places and
the pass that adds the slices.  attn_packed_plan and attn_packed_places of kernels.h,
by their C++ names."""
import ctypes as C
import os
import random

import pytest

import paper_2411_06465_amd as L
from packed_common import starts_of

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libl4d.so not built")


class PackedAttn(C.Structure):
    _fields_ = [("starts", C.c_void_p), ("n_seqs", C.c_int32), ("tokens", C.c_int32)] + \
               [(n, C.c_int32) for n in ("heads", "kv_heads", "d_h", "hpb", "n_slots")] + [("scale", C.c_float)] + \
               [(n, C.c_int64) for n in ("q", "k", "v", "q_ld", "k_ld", "v_ld", "o", "o_ld", "lse", "dout", "do_ld",
                                         "dq", "dk", "dv", "dq_ld", "dk_ld", "dv_ld", "delta", "lse2")] + \
               [("n_split", C.c_int32), ("cut_rows", C.c_int32), ("list_steps", C.c_int32), ("rope", C.c_int64),
                ("items", C.c_int64), ("dkv_partial", C.c_int64)]


def plan(starts, tokens, heads, kv):
    lib = L.lib()
    make, places = lib._ZN3l4d16attn_packed_planEPNS_10PackedAttnE, lib._ZN3l4d18attn_packed_placesERKNS_10PackedAttnE
    make.argtypes, make.restype = [C.POINTER(PackedAttn)], None
    places.argtypes, places.restype = [C.POINTER(PackedAttn)], C.c_int64
    p = PackedAttn(n_seqs=len(starts) - 1, tokens=tokens, heads=heads, kv_heads=kv, d_h=64)
    make(C.byref(p))
    return p, places(C.byref(p))


def replay(starts, tokens, heads, kv):
    p, places = plan(starts, tokens, heads, kv)
    group = heads // kv
    assert p.n_split >= 1 and group % p.n_split == 0
    blocks = [(row0, hi) for lo, hi in zip(starts[:-1], starts[1:]) for row0 in range(lo, hi, 128)]
    # the listing workgroup's 256 threads take the documents in turn, and none stops early
    for thread in range(256):
        docs = range(thread, len(starts) - 1, 256)
        assert sum(-(-(starts[i + 1] - starts[i]) // 128) for i in docs) <= p.list_steps
    if p.cut_rows == 0:        # all cut alike: a place per block and slice
        assert len(blocks) * p.n_split <= places
        return 0
    cut = [b for b in blocks if p.n_split > 1 and b[1] - b[0] >= p.cut_rows]
    assert len(blocks) + len(cut) <= places
    assert places <= tokens + (tokens + 127) // 128          # the room of the list
    # the pass that adds the slices looks at the block of every 128th row
    found = set()
    for row in range(0, tokens, 128):
        for lo, hi in zip(starts[:-1], starts[1:]):
            if lo <= row < hi:
                found.add((lo + (row - lo) // 128 * 128, hi))
    assert set(cut) <= found
    return len(cut)


def documents(rng, docs, mean, spread, empty):
    return [0 if rng.random() < empty else max(1, round(mean * rng.lognormvariate(0.0, spread))) for _ in range(docs)]


@pytest.mark.parametrize("group", range(1, 65))
def test_every_cut_block_is_listed_launched_and_added_up(group):
    rng, cut = random.Random(group), 0
    for docs, mean, spread, empty, kv in ((400, 40, 1.0, 0.0, 1), (450, 40, 0.0, 0.0, 1), (700, 36, 0.3, 0.1, 1),
                                          (520, 100, 1.3, 0.5, 1), (130, 65, 0.0, 0.0, 4), (60, 300, 1.0, 0.2, 32)):
        starts = starts_of(documents(rng, docs, mean, spread, empty), rng.randrange(200))
        cut += replay(starts, starts[-1] + rng.randrange(300), group * kv, kv)
    assert cut > 0 if group % 2 == 0 else cut == 0


@pytest.mark.parametrize("lens,heads,kv", [([65] * 60 + [0] * 200, 64, 2), ([36] * 900, 128, 1), ([40] * 450, 48, 1),
                                           ([127] * 500, 32, 1), ([128] * 500, 32, 1), ([129] * 500, 32, 1)])
def test_short_documents_of_many_query_heads(lens, heads, kv):
    starts = starts_of(lens)
    cut = replay(starts, starts[-1], heads, kv)
    assert cut == (0 if max(lens) < 128 else len(lens))


@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 1), (2, 2), (8, 1), (32, 8)])
def test_counts_of_the_list_stay_in_32_bits(heads, kv):
    """Starts out of order (0, tokens, 0, tokens, ..) make every other document hold all rows: the
    listing workgroup counts list_steps blocks per thread, each in up to two slices, and no sum
    of them passes 2^31, over all packings that a launch takes."""
    fits = L.lib()._ZN3l4d16attn_packed_fitsERKNS_10PackedAttnE
    fits.argtypes, fits.restype = [C.POINTER(PackedAttn)], C.c_bool
    largest = 0
    for t in range(31):
        for s in range(25):
            for tokens, n_seqs in (((1 << t) - 1, (1 << s) - 1), (1 << t, 1 << s), (3 << t >> 1, 3 << s >> 1)):
                p = PackedAttn(n_seqs=n_seqs, tokens=tokens, heads=heads, kv_heads=kv, d_h=64)
                if tokens < 1 or n_seqs < 1 or not fits(C.byref(p)):
                    continue
                L.lib()._ZN3l4d16attn_packed_planEPNS_10PackedAttnE(C.byref(p))
                assert p.list_steps >= 1
                per_block = p.n_split if p.cut_rows else 1
                assert 256 * p.list_steps * per_block < 1 << 31, (tokens, n_seqs)
                largest = max(largest, tokens)
    assert largest >= 1 << 23
