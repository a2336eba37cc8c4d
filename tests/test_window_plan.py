"""The dK/dV pass of window attention replayed on the host (no GPU needed): the chunks of rows
far from first tokens, the list of blocks, the launch's places, and which part of the sums each
takes.  attn_window_chunks, attn_window_plan and attn_window_places of kernels.h, by their C++ names."""
import ctypes as C
import os
import random

import pytest

import paper_2411_06465_amd as L
from packed_common import starts_of

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libl4d.so not built")


class WindowAttn(C.Structure):
    _fields_ = [("starts", C.c_void_p), ("n_seqs", C.c_int32), ("tokens", C.c_int32)] + \
               [(n, C.c_int32) for n in ("heads", "kv_heads", "d_h", "hpb", "n_slots")] + [("scale", C.c_float)] + \
               [(n, C.c_int64) for n in ("q", "k", "v", "q_ld", "k_ld", "v_ld", "o", "o_ld", "lse", "dout", "do_ld",
                                         "dq", "dk", "dv", "dq_ld", "dk_ld", "dv_ld", "delta", "lse2")] + \
               [("n_split", C.c_int32), ("cut_rows", C.c_int32), ("list_steps", C.c_int32), ("rope", C.c_int64),
                ("items", C.c_int64), ("dkv_partial", C.c_int64)] + \
               [(n, C.c_int32) for n in ("window", "sinks", "far_rows", "far_chunk", "far_parts", "cut_mask")] + \
               [("sink_partial", C.c_int64)]


def plan(starts, tokens, heads, kv, d, window, sinks):
    lib = L.lib()
    chunks, make = lib._ZN3l4d18attn_window_chunksEPNS_10WindowAttnE, lib._ZN3l4d16attn_window_planEPNS_10WindowAttnE
    places = lib._ZN3l4d18attn_window_placesERKNS_10WindowAttnE
    for f in (chunks, make, places):
        f.argtypes, f.restype = [C.POINTER(WindowAttn)], None
    places.restype = C.c_int64
    p = WindowAttn(n_seqs=len(starts) - 1, tokens=tokens, heads=heads, kv_heads=kv, d_h=d, window=window, sinks=sinks)
    chunks(C.byref(p))
    make(C.byref(p))
    return p, places(C.byref(p))


def slices(p, row0, rows):
    return p.n_split if rows >= p.cut_rows and not row0 >> 7 & p.cut_mask else 1


def replay(starts, tokens, heads, kv, d, window, sinks):
    p, places = plan(starts, tokens, heads, kv, d, window, sinks)
    assert p.n_split >= 1 and heads // kv % p.n_split == 0
    assert p.n_split <= L.lib()._ZN3l4d23attn_packed_most_splitsElll(C.c_long(tokens), C.c_long(heads), C.c_long(kv))
    n_items, parts, steps, seen = 0, {}, [0] * 256, {}
    for i, (lo, hi) in enumerate(zip(starts[:-1], starts[1:])):
        for row0 in range(lo, hi, 128):
            first = row0 - lo < sinks
            end = min(hi, lo + p.far_rows) if first else min(hi, row0 + 127 + window)
            steps[i % 256] += 1
            cut = slices(p, row0, end - row0)
            n_items += cut if p.cut_rows else 1
            if p.cut_rows and cut > 1:
                assert hi - row0 >= 128              # found from its 128-row window by the pass that adds the slices
            # every row that sees a key of the block is covered by it or by far chunks
            need = hi if first else min(hi, min(row0 + 127, hi - 1) + window)
            assert end >= min(need, lo + p.far_rows) if first else end >= need
            if first and hi - lo > p.far_rows:
                part = (lo + p.far_rows) // p.far_chunk - 1
                assert 0 <= part < p.far_parts
                assert parts.setdefault(part, (i, "own")) == (i, "own")
        q0 = lo + p.far_rows
        while q0 < hi and sinks:
            end = min(hi, (q0 // p.far_chunk + 1) * p.far_chunk)
            part = q0 // p.far_chunk
            assert part < p.far_parts and part not in parts
            parts[part] = (i, "far")
            blocks = -(-sinks // 128)
            assert lo + 128 * blocks <= lo + p.far_rows          # the blocks of first rows are whole
            steps[i % 256] += blocks
            n_items += blocks
            q0 = end
        if hi - lo > p.far_rows and sinks:
            # the pass that joins the parts finds the document from its own part, and no other one there
            part0 = (lo + p.far_rows) // p.far_chunk - 1
            base = (part0 + 1) * p.far_chunk
            at = base + p.far_chunk - 1 - p.far_rows
            found = max((j for j, s in enumerate(starts[:-1]) if s <= at), default=-1)
            assert found == i and starts[found] + p.far_rows >= base
            assert part0 not in seen
            seen[part0] = i
            assert all(parts[c] == (i, "far") for c in range(part0 + 1, (hi - 1) // p.far_chunk + 1))
    assert max(steps) <= p.list_steps
    room = tokens + (tokens + 127) // 128 + p.far_parts * -(-sinks // 128)
    per = 1 if p.cut_rows else p.n_split
    assert n_items <= room and n_items * per <= places and places <= room * per
    return len(seen)


def test_the_chunks_of_far_rows():
    """Every part has one owner, whatever the documents, windows and first tokens."""
    rng, far = random.Random(3), 0
    for _ in range(600):
        tokens = rng.choice([200, 1500, 5000, 40000])
        docs = rng.choice([1, 2, 3, 5, 20, 300])
        cut = sorted(rng.randrange(tokens + 1) for _ in range(docs - 1))
        starts = [0] + cut + [tokens] if rng.random() < 0.7 else starts_of([tokens // docs] * docs, tokens % docs)
        heads, kv = rng.choice([(4, 2), (8, 1), (32, 8), (64, 32), (20, 1), (5, 5)])
        window, sinks = rng.choice([1, 7, 128, 500, 1024, 4096]), rng.choice([0, 1, 4, 16, 100, 128, 129, 600, 4096])
        if window < tokens:
            far += replay(starts, tokens, heads, kv, rng.choice([64, 128]), window, sinks)
    assert far > 100


def test_every_eighth_block_is_cut_where_a_round_is_part_empty():
    starts = [0, 2000, 4000, 6000]
    p, _ = plan(starts, 6000, 32, 8, 128, 1024, 4)
    assert p.cut_mask == 7 and p.n_split == 2
    replay(starts, 6000, 32, 8, 128, 1024, 4)
    assert plan([0, 8192], 8192, 32, 8, 128, 1024, 4)[0].n_split == 1


def test_documents_at_the_border_of_the_far_rows():
    for window, sinks in ((1, 1), (128, 4), (600, 130), (64, 1000)):
        p, _ = plan([0, 40000], 40000, 8, 1, 64, window, sinks)
        assert p.far_rows >= 2 * p.far_chunk and p.far_rows >= window and p.far_chunk % 128 == 0
        for more in (-1, 0, 1, 2, p.far_chunk):
            starts = starts_of([p.far_rows + more] * 4 + [3, p.far_rows + 5 * p.far_chunk], 11)
            replay(starts, starts[-1] + 7, 8, 1, 64, window, sinks)


def test_a_window_without_first_tokens_or_far_rows_has_no_parts():
    for tokens, window, sinks in ((40000, 100, 0), (256, 100, 4)):      # far rows begin 128 + 128 behind the first one
        p, _ = plan([0, tokens], tokens, 8, 2, 128, window, sinks)
        assert p.far_parts == 0
    assert plan([0, 257], 257, 8, 2, 128, 100, 4)[0].far_parts > 0
