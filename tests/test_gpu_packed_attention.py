"""Causal attention over packed documents against the plain 64-bit form."""
import math

import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import U, attention_plain, close, inside, starts_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# A tensor's rounding errors are independent: their Frobenius norm is at most U/sqrt(3) of the
# tensor's for each of the at most three roundings on the way (P or dS, o inside delta, the output).
FROB = U


def draw(n, a, g, d, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    t = [torch.randn((n, h, d), generator=gen) * s for h, s in ((a, scale), (g, 1.0), (g, 1.0), (a, 1.0))]
    return [x.to(BF16) for x in t]


def packing(starts, n):
    return L.make_packing(torch.tensor(starts, dtype=torch.int64, device="cuda"), n)


def arena(n, a, g, d):
    return L.Arena.on(torch.empty(L.l4d_attn_packed_workspace_bytes(n, a, g, d) + 256, dtype=torch.uint8, device="cuda"))


def run(q, k, v, g, pk, scale=0.0, fill=0.0, ar=None):
    """Forward and backward into arrays that hold `fill`."""
    n, a, d = q.shape
    out = dict(o=torch.full_like(q, fill), lse=torch.full((a, n), fill, dtype=F32, device="cuda"),
               dq=torch.full_like(q, fill), dk=torch.full_like(k, fill), dv=torch.full_like(v, fill))
    L.attn_packed_fwd(q, k, v, out["o"], out["lse"], pk, scale)
    L.attn_packed_bwd(q, k, v, out["o"], out["lse"], g, out["dq"], out["dk"], out["dv"], pk,
                      ar or arena(n, a, k.shape[1], d), scale)
    return out


def compare(out, q, k, v, g, starts, scale=None, fill=0.0, norms=("o", "dq", "dk", "dv")):
    want = attention_plain(*(t.cpu().double() for t in (q, k, v)), starts, scale, g.cpu().double())
    n = q.shape[0]
    rows = torch.zeros(n, dtype=torch.bool)
    rows[starts[0]:max(starts[0], starts[-1])] = True
    for t in ("o", "lse", "dq", "dk", "dv"):
        got = out[t].cpu().double()
        at = (slice(None), rows) if t == "lse" else rows
        inside(t, got[at], want[t][at], want["_" + t][at])
        if t in norms and any(hi - lo > 1 for lo, hi in zip(starts[:-1], starts[1:])):
            close(t, got[at], want[t][at], FROB)
        outside = got[:, ~rows] if t == "lse" else got[~rows]
        assert bool((outside == fill).all()), f"{t}: rows of no document were written"


CASES = [  # lens, first row, rows behind, heads, kv heads, d
    ([1], 0, 0, 1, 1, 64),
    ([1, 1, 1], 0, 5, 4, 2, 128),
    ([2], 0, 0, 2, 1, 128),
    ([31, 0, 33, 1, 0, 0, 64], 0, 3, 4, 4, 64),
    ([127, 129, 1, 128], 0, 0, 4, 1, 64),
    ([100, 3, 260], 7, 40, 8, 2, 128),
    ([0, 0, 5, 0], 0, 9, 6, 2, 128),
    ([700], 0, 1, 5, 5, 128),
    ([513, 64, 65], 0, 0, 12, 2, 64),
    ([17] * 40, 0, 8, 14, 2, 64),
    ([300, 77], 3, 0, 16, 2, 128),      # query heads of a kv head in slices
]


@pytest.mark.parametrize("lens,first,tail,a,g,d", CASES)
def test_matches_the_plain_form(lens, first, tail, a, g, d):
    starts = starts_of(lens, first)
    n = starts[-1] + tail
    q, k, v, do = (t.cuda() for t in draw(n, a, g, d, 11 * n + a))
    # rows of no document hold NaN: nothing of them may be used
    for t in (q, k, v, do):
        t[:first], t[starts[-1]:] = math.nan, math.nan
    out = run(q, k, v, do, packing(starts, n), fill=7.0)
    compare(out, q, k, v, do, starts, fill=7.0)


def test_more_documents_than_a_wave_probes_at_once():
    lens = [(i * 7) % 4 for i in range(5000)]      # 0 .. 3 tokens, many empty
    starts = starts_of(lens)
    n = starts[-1]
    q, k, v, do = (t.cuda() for t in draw(n, 2, 1, 64, 5))
    compare(run(q, k, v, do, packing(starts, n)), q, k, v, do, starts)


@pytest.mark.parametrize("d", [64, 128])
def test_long_blocks_cut_among_many_short_ones(d):
    """Enough blocks that only those of the long document are cut; four of the 32 kv heads are compared."""
    starts, a, g = starts_of([40, 1600, 3, 0, 300] + [1] * 9 + [100], 10), 64, 32
    n = starts[-1] + 47
    q, k, v, do = (t.cuda() for t in draw(n, a, g, d, 31))
    out = run(q, k, v, do, packing(starts, n), fill=7.0)
    again = run(q, k, v, do, packing(starts, n), fill=7.0)
    for t in out:
        assert torch.equal(out[t], again[t]), t       # whatever the order of the blocks
    for h in (0, 1, 17, 31):
        hq, hk = slice(2 * h, 2 * h + 2), slice(h, h + 1)
        part = {t: x[hq] if t == "lse" else x[:, hk if t in ("dk", "dv") else hq] for t, x in out.items()}
        compare(part, q[:, hq], k[:, hk], v[:, hk], do[:, hq], starts, fill=7.0)


@pytest.mark.parametrize("docs", [2, 62, 63, 64, 65])
def test_documents_around_a_wave(docs):
    lens = [(i * 37) % 71 for i in range(docs)]
    lens[docs // 2] = 333
    starts = starts_of(lens, 3)
    n = starts[-1] + 2
    q, k, v, do = (t.cuda() for t in draw(n, 4, 2, 64, docs))
    compare(run(q, k, v, do, packing(starts, n), fill=7.0), q, k, v, do, starts, fill=7.0)


@pytest.mark.parametrize("scale,spread", [(0.5, 4.0), (1e-3, 1.0), (1.0, 30.0)])
def test_scales_and_large_scores(scale, spread):
    starts = starts_of([90, 210])
    q, k, v, do = (t.cuda() for t in draw(300, 4, 2, 128, 3, spread))
    # Where one p of a row is nearly 1, dS = p (dP - delta) is a small difference of equal
    # numbers: with p = 1 - e it is e (dP_1 - dP_2), while o's rounding leaves an error of
    # delta of up to U sum |d_o o| whatever e is.  dq and dk then have no relative norm bound,
    # only the element-wise one, which carries that error.
    compare(run(q, k, v, do, packing(starts, 300), scale), q, k, v, do, starts, scale, norms=("o", "dv"))


def test_columns_of_fused_arrays():
    """q, k, v as columns of one array, the gradients as columns of another, o and d_o with a longer row."""
    starts, n, a, g, d = starts_of([150, 0, 77]), 230, 6, 2, 64
    gen = torch.Generator().manual_seed(9)
    qkv = torch.randn((n, (a + 2 * g) * d), generator=gen).to(BF16).cuda()
    wide = torch.randn((n, (a + 1) * d), generator=gen).to(BF16).cuda()

    def split(t):
        return [t[:, i * d:j * d].unflatten(1, (j - i, d)) for i, j in ((0, a), (a, a + g), (a + g, a + 2 * g))]

    q, k, v = split(qkv)
    do = wide[:, d:].unflatten(1, (a, d))
    grads = torch.zeros_like(qkv)
    o = torch.zeros_like(wide)[:, :a * d].unflatten(1, (a, d))
    lse = torch.zeros((a, n), dtype=F32, device="cuda")
    pk = packing(starts, n)
    L.attn_packed_fwd(q, k, v, o, lse, pk)
    dq, dk, dv = split(grads)
    L.attn_packed_bwd(q, k, v, o, lse, do, dq, dk, dv, pk, arena(n, a, g, d))
    compare(dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv), q, k, v, do, starts)


def test_a_bad_document_reaches_no_other():
    starts, n = starts_of([40, 50, 37]), 127
    q, k, v, do = (t.cuda() for t in draw(n, 4, 1, 128, 21))
    pk = packing(starts, n)
    clean = run(q, k, v, do, pk)
    for bad in (math.nan, math.inf, torch.finfo(BF16).max, torch.finfo(BF16).min):
        qb, kb, vb, gb = (t.clone() for t in (q, k, v, do))
        for t in (qb, kb, vb, gb):
            t[45:80] = bad
        out = run(qb, kb, vb, gb, pk)
        for t in out:
            x, y = (out[t], clean[t]) if t != "lse" else (out[t].t(), clean[t].t())
            assert torch.equal(x[:40], y[:40]) and torch.equal(x[90:], y[90:]), (t, bad)


def test_far_rows_pass_32_bit_offsets():
    """A row stride that puts the last rows behind 2^32 elements."""
    n, a, g, d, ld = 1100, 2, 1, 64, 1 << 22
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 10 GB")
    starts = starts_of([1000, 100])
    q, k, v, do = (t.cuda() for t in draw(n, a, g, d, 2))
    big = torch.zeros((n - 1) * ld + a * d, dtype=BF16, device="cuda")
    qs = big.as_strided((n, a, d), (ld, d, 1))
    qs.copy_(q)
    pk = packing(starts, n)
    near, far = run(q, k, v, do, pk), run(qs, k, v, do, pk)
    for t in near:
        assert torch.equal(near[t], far[t]), t


def test_another_stream_and_an_unordered_table_of_calls():
    """Calls on a side stream, two arenas on two streams, the same results as one after another."""
    starts, n = starts_of([65, 200, 20]), 290
    sets = [[t.cuda() for t in draw(n, 8, 2, 64, s)] for s in (1, 2)]
    pk = packing(starts, n)
    want = [run(*s, pk) for s in sets]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    arenas = [arena(n, 8, 2, 64) for _ in sets]
    torch.cuda.synchronize()
    for s, st, ar in zip(sets, streams, arenas):
        with torch.cuda.stream(st):
            got.append(run(*s, pk, ar=ar))
    torch.cuda.synchronize()
    for w, x in zip(want, got):
        for t in w:
            assert torch.equal(w[t], x[t]), t


def test_captured_and_replayed():
    starts, n = starts_of([33, 150, 0, 90]), 280
    q, k, v, do = (t.cuda() for t in draw(n, 8, 1, 128, 4))
    pk, ar = packing(starts, n), arena(n, 8, 1, 128)
    eager = run(q, k, v, do, pk, ar=ar)
    out = {t: torch.zeros_like(x) for t, x in eager.items()}

    def step():
        L.attn_packed_fwd(q, k, v, out["o"], out["lse"], pk)
        L.attn_packed_bwd(q, k, v, out["o"], out["lse"], do, out["dq"], out["dk"], out["dv"], pk, ar)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        for x in out.values():
            x.zero_()
        new = draw(n, 8, 1, 128, 40 + i)
        for t, x in zip((q, k, v, do), new):
            t.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        want = run(q, k, v, do, pk)
        for t in want:
            assert torch.equal(out[t], want[t]), (i, t)


def test_gradients_against_differences():
    """A directional difference of sum(o * d_o) in each input, by the 64-bit form."""
    starts, n, a, g, d = starts_of([20, 45]), 65, 4, 2, 64
    q, k, v, do = draw(n, a, g, d, 8)
    out = run(*(t.cuda() for t in (q, k, v, do)), packing(starts, n))
    x = [t.double() for t in (q, k, v)]
    for i, name in enumerate(("dq", "dk", "dv")):
        way = torch.randn(x[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64)
        h = 1e-5
        val = []
        for s in (h, -h):
            y = list(x)
            y[i] = x[i] + s * way
            val.append(float((attention_plain(*y, starts)["o"] * do.double()).sum()))
        slope = (val[0] - val[1]) / (2 * h)
        got = float((out[name].cpu().double() * way).sum())
        # the gradient's own relative error (FROB) times the norms of what is multiplied
        assert abs(got - slope) <= 4 * FROB * float(out[name].cpu().double().norm()) + 1e-6 * abs(slope), (name, got, slope)
