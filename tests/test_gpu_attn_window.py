"""Attention over packed documents with a sliding window and first tokens, against the plain 64-bit form."""
import math

import pytest
import torch

import paper_2411_06465_amd as L
from packed_common import F, U, close, inside, starts_of

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64

# A tensor's rounding errors are independent: their Frobenius norm is at most U/sqrt(3) of the
# tensor's for each of the at most three roundings on the way (P or dS, o inside delta, the output).
FROB = U


def hidden_pairs(n, window, sinks):
    i = torch.arange(n)
    back = i[:, None] - i[None, :]
    return (back < 0) | ((back >= window) & (i[None, :] >= sinks))


def plain(q, k, v, starts, window, sinks, scale=None, d_o=None):
    """q [n][a][d], k, v [n][g][d] float64 -> results and, under "_" + name, element-wise error
    bounds that count roundings (of P, dS and the outputs to bf16; fp32 products and sums)."""
    n, a, d = q.shape
    group = a // k.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = {t: torch.zeros_like(q) for t in ("o", "_o", "dq", "_dq")}
    out.update({t: torch.zeros_like(k) for t in ("dk", "_dk", "dv", "_dv")})
    out["lse"], out["_lse"] = torch.zeros(a, n, dtype=F64), torch.zeros(a, n, dtype=F64)
    for lo, hi in zip(starts[:-1], starts[1:]):
        if hi <= lo:
            continue
        at, add = slice(lo, hi), (hi - lo + 8) * F
        mask = hidden_pairs(hi - lo, window, sinks)
        for h in range(a):
            g = h // group
            Q, K, V = q[at, h], k[at, g], v[at, g]
            s = (Q @ K.T * scale).masked_fill(mask, -math.inf)
            lse = torch.logsumexp(s, -1)
            P = torch.exp(s - lse[:, None])
            # a score: its products, the scale, its exponent (base 2) next to the maximum's
            e_s = ((d + 8) * F * scale * (Q.abs() @ K.abs().T) + 4 * F * s.abs()).masked_fill(mask, 0.0)
            e_p = e_s.amax(-1, keepdim=True) + e_s + add                    # relative error of P in fp32
            out["o"][at, h], out["lse"][h, at] = P @ V, lse
            e_lse = e_s.amax(-1) + add + 4 * F * lse.abs()
            out["_lse"][h, at] = e_lse
            e_o = (P * (U + e_p)) @ V.abs() * (1 + U) + add * (P @ V.abs())   # before its own rounding
            e_o = U * (P @ V).abs() + (1 + U) * e_o
            out["_o"][at, h] = e_o
            if d_o is None:
                continue
            G = d_o[at, h]
            dP = G @ V.T
            go = G * (P @ V)
            delta = go.sum(-1, keepdim=True)
            dS = P * (dP - delta)
            # delta from the rounded output; dP from fp32 products; P from the rounded lse
            e_delta = (G.abs() * e_o).sum(-1, keepdim=True) + (d + 2) * F * go.abs().sum(-1, keepdim=True)
            e_dp = (d + 2) * F * (G.abs() @ V.abs().T)
            e_pb = 2 * e_p + e_lse[:, None]
            e_ds = U * dS.abs() + (1 + U) * (P * (e_dp + e_delta) + e_pb * dS.abs() + 4 * F * P * (dP.abs() + delta.abs()))
            e_ds = e_ds.masked_fill(mask, 0.0)
            out["dq"][at, h] = scale * dS @ K
            out["_dq"][at, h] = scale * (e_ds @ K.abs() + add * (dS.abs() @ K.abs()))
            out["dk"][at, g] += scale * dS.T @ Q
            out["_dk"][at, g] += scale * (e_ds.T @ Q.abs() + (add + group * F) * (dS.abs().T @ Q.abs()))
            out["dv"][at, g] += P.T @ G
            out["_dv"][at, g] += (P * (U + e_pb)).T @ G.abs() * (1 + U) + (add + group * F) * (P.T @ G.abs())
    for t in ("dq", "dk", "dv"):
        out["_" + t] = (1 + U) * out["_" + t] + U * out[t].abs()
    return out


def draw(n, a, g, d, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    t = [torch.randn((n, h, d), generator=gen) * s for h, s in ((a, scale), (g, 1.0), (g, 1.0), (a, 1.0))]
    return [x.to(BF16) for x in t]


def packing(starts, n):
    return L.make_packing(torch.tensor(starts, dtype=torch.int64, device="cuda"), n)


def arena(win, n, a, g, d, fill=0xff):
    """Workspace that holds NaN: what is not written must not be read."""
    size = L.l4d_attn_window_workspace_bytes(win, n, a, g, d) + 256
    return L.Arena.on(torch.full((size,), fill, dtype=torch.uint8, device="cuda"))


def run(win, q, k, v, g, pk, scale=0.0, fill=0.0, ar=None):
    """Forward and backward into arrays that hold `fill`."""
    n, a, d = q.shape
    out = dict(o=torch.full_like(q, fill), lse=torch.full((a, n), fill, dtype=F32, device="cuda"),
               dq=torch.full_like(q, fill), dk=torch.full_like(k, fill), dv=torch.full_like(v, fill))
    L.attn_window_fwd(win, q, k, v, out["o"], out["lse"], pk, scale)
    L.attn_window_bwd(win, q, k, v, out["o"], out["lse"], g, out["dq"], out["dk"], out["dv"], pk,
                      ar or arena(win, n, a, k.shape[1], d), scale)
    return out


def compare(out, q, k, v, g, starts, window, sinks, scale=None, fill=0.0, norms=("o", "dq", "dk", "dv")):
    want = plain(*(t.cpu().double() for t in (q, k, v)), starts, window, sinks, scale, g.cpu().double())
    rows = torch.zeros(q.shape[0], dtype=torch.bool)
    rows[starts[0]:max(starts[0], starts[-1])] = True
    for t in ("o", "lse", "dq", "dk", "dv"):
        got = out[t].cpu().double()
        at = (slice(None), rows) if t == "lse" else rows
        inside(t, got[at], want[t][at], want["_" + t][at])
        # one visible key leaves no gradient of q and k: its exact value is 0
        if t in norms and any(hi - lo > 1 for lo, hi in zip(starts[:-1], starts[1:])) and (window + sinks > 1 or t in ("o", "dv")):
            close(t, got[at], want[t][at], FROB)
        outside = got[:, ~rows] if t == "lse" else got[~rows]
        assert bool((outside == fill).all()), f"{t}: rows of no document were written"


CASES = [  # lens, first row, rows behind, heads, kv heads, d, window, sinks
    ([1], 0, 1, 1, 1, 64, 1, 0),
    ([1, 1, 2], 0, 5, 4, 2, 128, 1, 1),
    ([40], 0, 0, 2, 1, 128, 1, 0),                  # every row sees itself alone
    ([31, 0, 33, 1, 0, 0, 64], 0, 3, 4, 4, 64, 7, 0),
    ([127, 129, 1, 128], 0, 0, 4, 1, 64, 33, 2),
    ([200], 3, 7, 4, 2, 64, 63, 5),
    ([200], 3, 7, 4, 2, 128, 64, 64),
    ([200], 3, 7, 8, 2, 64, 65, 63),
    ([100, 3, 260], 7, 40, 8, 2, 128, 128, 65),
    ([0, 0, 5, 0], 0, 9, 6, 2, 128, 2, 1),
    ([700], 0, 1, 5, 5, 128, 96, 130),              # first tokens in two blocks of keys
    ([513, 64, 65], 0, 0, 12, 2, 64, 300, 1),
    ([17] * 40, 0, 8, 14, 2, 64, 5, 3),
    ([300, 77], 3, 0, 16, 2, 128, 50, 40),          # query heads of a kv head in slices
    ([300, 77], 3, 0, 4, 1, 64, 299, 0),            # the window hides one pair
    ([300, 77], 3, 0, 4, 1, 64, 100, 500),          # more first tokens than rows: all is visible
    ([1500, 20, 1300, 0, 1200], 5, 9, 2, 1, 64, 100, 3),     # rows far from first tokens, in chunks
    ([2600], 0, 0, 2, 2, 128, 17, 200),             # and first tokens in two blocks
    ([2700, 10], 1, 3, 4, 1, 64, 1400, 600),        # chunks of more than 512 rows
    ([1153, 1152, 1154], 0, 0, 2, 1, 128, 1, 1),    # one row, none, two of them far
]


@pytest.mark.parametrize("lens,first,tail,a,g,d,window,sinks", CASES)
def test_matches_the_plain_form(lens, first, tail, a, g, d, window, sinks):
    starts = starts_of(lens, first)
    n = starts[-1] + tail
    q, k, v, do = (t.cuda() for t in draw(n, a, g, d, 11 * n + a))
    # rows of no document hold NaN: nothing of them may be used
    for t in (q, k, v, do):
        t[:first], t[starts[-1]:] = math.nan, math.nan
    out = run(L.make_window(window, sinks), q, k, v, do, packing(starts, n), fill=7.0)
    compare(out, q, k, v, do, starts, window, sinks, fill=7.0)


def test_more_documents_than_a_wave_probes_at_once():
    lens = [(i * 7) % 4 for i in range(2000)] + [1400] + [2] * 500      # many empty, one with far rows
    starts = starts_of(lens)
    n = starts[-1]
    q, k, v, do = (t.cuda() for t in draw(n, 2, 1, 64, 5))
    compare(run(L.make_window(2, 1), q, k, v, do, packing(starts, n)), q, k, v, do, starts, 2, 1)


@pytest.mark.parametrize("d,window,sinks", [(64, 700, 4), (128, 900, 140)])
def test_long_blocks_cut_among_many_short_ones(d, window, sinks):
    """Enough blocks that only those of the long document are cut; three of the 32 kv heads are compared."""
    starts, a, g = starts_of([40, 1900, 3, 0, 300] + [1] * 9 + [100], 10), 64, 32
    n, win = starts[-1] + 47, L.make_window(window, sinks)
    q, k, v, do = (t.cuda() for t in draw(n, a, g, d, 31))
    out = run(win, q, k, v, do, packing(starts, n), fill=7.0)
    again = run(win, q, k, v, do, packing(starts, n), fill=7.0)
    for t in out:
        assert torch.equal(out[t], again[t]), t       # whatever the order of the blocks
    for h in (0, 1, 31):
        hq, hk = slice(2 * h, 2 * h + 2), slice(h, h + 1)
        part = {t: x[hq] if t == "lse" else x[:, hk if t in ("dk", "dv") else hq] for t, x in out.items()}
        compare(part, q[:, hq], k[:, hk], v[:, hk], do[:, hq], starts, window, sinks, fill=7.0)


@pytest.mark.parametrize("sinks", [0, 200])
def test_every_eighth_block_cut(sinks):
    """As many blocks as fill the chip once and a part: every eighth is cut; two of the 16 kv heads are compared."""
    starts, a, g, d = starts_of([1400, 30, 1530], 0), 32, 16, 128
    n, win = starts[-1] + 5, L.make_window(512, sinks)
    q, k, v, do = (t.cuda() for t in draw(n, a, g, d, 33))
    out = run(win, q, k, v, do, packing(starts, n), fill=7.0)
    for h in (0, 9):
        hq, hk = slice(2 * h, 2 * h + 2), slice(h, h + 1)
        part = {t: x[hq] if t == "lse" else x[:, hk if t in ("dk", "dv") else hq] for t, x in out.items()}
        compare(part, q[:, hq], k[:, hk], v[:, hk], do[:, hq], starts, 512, sinks, fill=7.0)


@pytest.mark.parametrize("window", [500, 501, 1 << 40])
def test_a_window_of_all_rows_is_no_window(window):
    starts, n = starts_of([90, 210, 0, 150]), 500
    q, k, v, do = (t.cuda() for t in draw(n, 8, 2, 128, 3))
    pk = packing(starts, n)
    got = run(L.make_window(window, 3), q, k, v, do, pk)
    o, lse, dq, dk, dv = (torch.zeros_like(got[t]) for t in ("o", "lse", "dq", "dk", "dv"))
    L.attn_packed_fwd(q, k, v, o, lse, pk)
    size = L.l4d_attn_packed_workspace_bytes(n, 8, 2, 128) + 256
    L.attn_packed_bwd(q, k, v, o, lse, do, dq, dk, dv, pk, L.Arena.on(torch.zeros(size, dtype=torch.uint8, device="cuda")))
    for t, x in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert torch.equal(got[t], x), t


@pytest.mark.parametrize("scale,spread", [(0.5, 4.0), (1e-3, 1.0), (1.0, 30.0)])
def test_scales_and_large_scores(scale, spread):
    starts = starts_of([90, 210])
    q, k, v, do = (t.cuda() for t in draw(300, 4, 2, 128, 3, spread))
    # where one p of a row is nearly 1, dq and dk are small differences of equal numbers and have
    # no relative norm bound, only the element-wise one
    compare(run(L.make_window(70, 2), q, k, v, do, packing(starts, 300), scale), q, k, v, do, starts, 70, 2, scale,
            norms=("o", "dv"))


def test_columns_of_fused_arrays():
    """q, k, v as columns of one array, the gradients as columns of another, o and d_o with a longer row."""
    starts, n, a, g, d, win = starts_of([150, 0, 77]), 230, 6, 2, 64, L.make_window(40, 4)
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
    L.attn_window_fwd(win, q, k, v, o, lse, pk)
    dq, dk, dv = split(grads)
    L.attn_window_bwd(win, q, k, v, o, lse, do, dq, dk, dv, pk, arena(win, n, a, g, d))
    compare(dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv), q, k, v, do, starts, 40, 4)


def test_keys_that_no_row_of_a_block_sees_are_not_read():
    """Not-finite rows between a document's first tokens and a late block's window leave the block as it is."""
    n, win = 1000, L.make_window(100, 4)
    q, k, v, do = (t.cuda() for t in draw(n, 4, 1, 128, 21))
    pk = packing([0, n], n)
    clean = run(win, q, k, v, do, pk)
    for bad in (math.nan, math.inf, torch.finfo(BF16).min):
        kb, vb = k.clone(), v.clone()
        kb[300:500], vb[300:500] = bad, bad
        out = run(win, q, kb, vb, do, pk)
        for t in ("o", "dq"):
            assert torch.equal(out[t][768:], clean[t][768:]) and torch.equal(out[t][:256], clean[t][:256]), (t, bad)
        assert torch.equal(out["lse"][:, 768:], clean["lse"][:, 768:]), bad


def test_a_bad_document_reaches_no_other():
    starts, n, win = starts_of([40, 50, 37]), 127, L.make_window(20, 2)
    q, k, v, do = (t.cuda() for t in draw(n, 4, 1, 128, 21))
    pk = packing(starts, n)
    clean = run(win, q, k, v, do, pk)
    for bad in (math.nan, math.inf, torch.finfo(BF16).max, torch.finfo(BF16).min):
        qb, kb, vb, gb = (t.clone() for t in (q, k, v, do))
        for t in (qb, kb, vb, gb):
            t[45:80] = bad
        out = run(win, qb, kb, vb, gb, pk)
        for t in out:
            x, y = (out[t], clean[t]) if t != "lse" else (out[t].t(), clean[t].t())
            assert torch.equal(x[:40], y[:40]) and torch.equal(x[90:], y[90:]), (t, bad)


def test_far_rows_pass_32_bit_offsets():
    """A row stride that puts the last rows behind 2^32 elements."""
    n, a, g, d, ld, win = 1400, 2, 1, 64, 1 << 22, L.make_window(60, 3)
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 13 GB")
    starts = starts_of([1300, 100])
    q, k, v, do = (t.cuda() for t in draw(n, a, g, d, 2))
    big = torch.zeros((n - 1) * ld + a * d, dtype=BF16, device="cuda")
    qs = big.as_strided((n, a, d), (ld, d, 1))
    qs.copy_(q)
    pk = packing(starts, n)
    near, far = run(win, q, k, v, do, pk), run(win, qs, k, v, do, pk)
    for t in near:
        assert torch.equal(near[t], far[t]), t


def test_two_streams_with_arenas_of_their_own():
    starts, n, win = starts_of([65, 1400, 20]), 1500, L.make_window(70, 4)
    sets = [[t.cuda() for t in draw(n, 8, 2, 64, s)] for s in (1, 2)]
    pk = packing(starts, n)
    want = [run(win, *s, pk) for s in sets]
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    arenas = [arena(win, n, 8, 2, 64) for _ in sets]
    torch.cuda.synchronize()
    for s, st, ar in zip(sets, streams, arenas):
        with torch.cuda.stream(st):
            got.append(run(win, *s, pk, ar=ar))
    torch.cuda.synchronize()
    for w, x in zip(want, got):
        for t in w:
            assert torch.equal(w[t], x[t]), t


REPLAYS = {  # rows, heads, kv heads, d, window, sinks, the documents of each replay
    "few": (2700, 8, 2, 128, 90, 4, ([0, 900, 1000, 2700], [0, 2600, 2650, 2690], [5, 5, 5, 1400], [9, 9, 9, 9])),
    "64": (1700, 4, 1, 64, 33, 130, ([26 * i for i in range(65)] + [1700], [3] * 60 + [4, 5, 1600, 1601, 1602, 1700])),
    "some-cut": (2600, 64, 32, 64, 700, 4, ([0, 100, 2600], [0, 1300, 2600], [2600, 2600, 2600])),
}


@pytest.mark.parametrize("name", list(REPLAYS))
def test_captured_and_replayed_with_other_documents(name):
    n, a, g, d, window, sinks, plans = REPLAYS[name]
    win = L.make_window(window, sinks)
    q, k, v, do = (t.cuda() for t in draw(n, a, g, d, 4))
    pk, ar = packing(plans[0], n), arena(win, n, a, g, d)
    out = dict(o=torch.zeros_like(q), lse=torch.zeros((a, n), dtype=F32, device="cuda"), dq=torch.zeros_like(q),
               dk=torch.zeros_like(k), dv=torch.zeros_like(v))

    def step():
        L.attn_window_fwd(win, q, k, v, out["o"], out["lse"], pk)
        L.attn_window_bwd(win, q, k, v, out["o"], out["lse"], do, out["dq"], out["dk"], out["dv"], pk, ar)

    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(2):
        for plan in plans:
            new = draw(n, a, g, d, 40 + i)
            for t, x in zip((q, k, v, do), new):
                t.copy_(x)
            for x in out.values():
                x.fill_(7.0)
            pk.starts.copy_(torch.tensor(plan))
            graph.replay()
            torch.cuda.synchronize()
            want = run(win, q, k, v, do, packing(plan, n), fill=7.0)
            for t in want:
                assert torch.equal(out[t], want[t]), (i, plan[:6], t)


def test_gradients_against_differences():
    """A directional difference of sum(o * d_o) in each input, by the 64-bit form."""
    starts, n, a, g, d = starts_of([20, 45]), 65, 4, 2, 64
    q, k, v, do = draw(n, a, g, d, 8)
    out = run(L.make_window(9, 2), *(t.cuda() for t in (q, k, v, do)), packing(starts, n))
    x = [t.double() for t in (q, k, v)]
    for i, name in enumerate(("dq", "dk", "dv")):
        way = torch.randn(x[i].shape, generator=torch.Generator().manual_seed(i), dtype=F64)
        h = 1e-5
        val = []
        for s in (h, -h):
            y = list(x)
            y[i] = x[i] + s * way
            val.append(float((plain(*y, starts, 9, 2)["o"] * do.double()).sum()))
        slope = (val[0] - val[1]) / (2 * h)
        got = float((out[name].cpu().double() * way).sum())
        # the gradient's own relative error (FROB) times the norms of what is multiplied
        assert abs(got - slope) <= 4 * FROB * float(out[name].cpu().double().norm()) + 1e-6 * abs(slope), (name, got, slope)
