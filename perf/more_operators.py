"""Operators around the attention of a layer that trains on packed documents, and their plain forms.

Norms of the query and key heads with the rotation in the same pass, rotary positions with
several axes, attention with a sliding window and a few first tokens that stay visible, and
dropout in front of the residual sum with a mask that is never stored.  Every case is one call,
or a forward and the backward that follows it, as a training or evaluation step makes it.

With `own` false, `run` computes the operators in their plain form: elementary torch operations
in 32 bits (angles in 64, random words in whole numbers), rounded once at the end.  With `own`
true it calls the library.  A case is a dict of plain values; `draw` gives more cases of the
same ranges.

Documents have log-normal lengths; with many of them some are empty; `tail` rows behind the
last one are padding.  Queries, keys, values and gradients are N(0, 1) rows, gains 1 + N(0, 0.1),
positions of several axes those of images' patches among text.
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DTYPES = {"bf16": BF16, "f32": F32}
FORWARD, BACKWARD = 4, 10    # attention flops per pair, head and channel: two products forward, five backward
EPS = 1e-6
WORD = 0xffffffff


# ------------------------------------------------------------------ the cases

def _norm(tokens, heads, kv, d, rot, layout, dtype, train, docs, tail=0, pairs="", **name):
    return dict(name, kind="norm", tokens=tokens, heads=heads, kv=kv, d=d, rot=rot, layout=layout, dtype=dtype, train=train,
                docs=docs, tail=tail, pairs=pairs, order="sections", frequencies="shared", spread=1.0)


def _axes(tokens, heads, kv, d, layout, dtype, direction, pairs, order, frequencies, docs, tail=0, **name):
    return dict(name, kind="axes", tokens=tokens, heads=heads, kv=kv, d=d, rot=2 * sum(_pairs_of(pairs)), layout=layout,
                dtype=dtype, direction=direction, pairs=pairs, order=order, frequencies=frequencies, docs=docs, tail=tail,
                spread=1.0)


def _window(tokens, heads, kv, d, window, sinks, docs, train, tail=0, spread=1.0, **name):
    return dict(name, kind="window", tokens=tokens, heads=heads, kv=kv, d=d, window=window, sinks=sinks, docs=docs,
                train=train, tail=tail, spread=spread)


def _dropout(rows, cols, p, dtype, train, first_row=0, **name):
    return dict(name, kind="dropout", rows=rows, cols=cols, p=p, dtype=dtype, train=train, first_row=first_row)


def _pairs_of(text):
    return [int(x) for x in text.split("+")] if text else []


def listed():
    return [
        # the heads of a small model on a handful of tokens, evaluation: the call's latency is what counts
        _norm(48, 4, 2, 64, 64, "half", "bf16", False, 3, name="norm-tiny"),
        # Llama-3-8B's heads over a packed row of 8192 tokens
        _norm(8192, 32, 8, 128, 128, "half", "bf16", True, 23, tail=100, name="norm-8b-train"),
        # interleaved pairs on half of each head, fp32, an odd token count, positions of two axes
        _norm(4099, 16, 16, 128, 64, "interleaved", "f32", True, 1, pairs="16+16", name="norm-axes-f32-train"),
        # text with images: time, height and width in sections of a head's pairs
        _axes(8000, 32, 8, 128, "half", "bf16", "forward", "16+24+24", "sections", "shared", 11, tail=50, name="axes-8b"),
        # an image's patches: height and width with frequencies of their own, backward in fp32
        _axes(4900, 16, 16, 64, "interleaved", "f32", "backward", "16+16", "sections", "own", 4, name="axes-image-f32-bwd"),
        # the smallest training call: head size 64, three short documents, a window within them
        _window(128, 4, 2, 64, 16, 2, 3, True, name="window-tiny-train"),
        # many short documents (chat turns) on heads of size 64, most within the window
        _window(16384, 16, 4, 64, 128, 4, 100, True, spread=0.8, name="window-short-docs-train"),
        # Llama-3-8B's heads on a packed row, windows of 1024 tokens
        _window(8192, 32, 8, 128, 1024, 4, 5, True, tail=61, name="window-8b-train"),
        # Llama-3-70B's heads at TP8, one long document next to a shorter one
        _window(32768, 8, 1, 128, 4096, 4, 2, True, spread=0.7, name="window-70b-tp8-long-train"),
        # the test model's hidden size: latency counts
        _dropout(128, 256, 0.1, "bf16", False, name="dropout-tiny"),
        # Llama-3-8B's residual, the second sequence-parallel rank's rows
        _dropout(8192, 4096, 0.1, "bf16", True, first_row=8192, name="dropout-8b-train"),
        # odd rows of odd length in fp32
        _dropout(3001, 1023, 0.35, "f32", True, name="dropout-odd-f32-train"),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _cost(case):
    w = work(case)
    return w["flops"] / 1e15 + w["bytes"] / 5e12


def _split(rng, pairs):
    n = rng.choice([2, 3, 3, 4])
    if pairs < n:
        return str(pairs)
    cuts = sorted(rng.sample(range(1, pairs), n - 1))
    return "+".join(str(b - a) for a, b in zip([0] + cuts, cuts + [pairs]))


def draw(rng):
    largest = {}
    for c in listed():
        largest[c["kind"]] = max(largest.get(c["kind"], 0.0), _cost(c))
    while True:
        kind = rng.choice(["norm", "norm", "axes", "window", "window", "window", "dropout"])
        heads, kv = rng.choice([(4, 2), (8, 1), (16, 4), (32, 8), (32, 32), (12, 4), (5, 5), (14, 2)])
        tokens = max(1, round(_log_uniform(rng, 1, 32768 if kind == "window" else 16384)))
        docs = max(1, min(tokens, round(_log_uniform(rng, 1, 200))))
        tail = rng.choice([0, 0, rng.randrange(300)])
        dtype, layout = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["half", "interleaved"])
        if kind == "dropout":
            case = _dropout(tokens, rng.choice([256, 512, 1024, 4096, 8192, round(_log_uniform(rng, 1, 8192))]),
                            rng.choice([0.0, 0.05, 0.1, 0.5, 0.9]), dtype, rng.random() < 0.6,
                            first_row=rng.choice([0, rng.randrange(1 << 34)]))
        elif kind == "window":
            # documents of one token alone would have no gradient of q and k to compare
            case = _window(tokens, heads, kv, rng.choice([64, 128, 128]), max(2, round(_log_uniform(rng, 2, 8192))),
                           rng.choice([0, 1, 4, 4, 16, rng.randrange(300)]), docs, tokens >= 2 * docs and rng.random() < 0.8,
                           tail=tail, spread=rng.choice([0.3, 1.0, 1.5]))
        elif kind == "norm":
            d = rng.choice([64, 128, 128, 256, 80, 2 * rng.randrange(2, 100)])
            rot = rng.choice([d, d, d // 4 * 2])
            case = _norm(tokens, heads, kv, d, rot, layout, dtype, rng.random() < 0.7, docs, tail=tail,
                         pairs=rng.choice(["", "", _split(rng, rot // 2)]))
        else:
            d = rng.choice([64, 128, 128, 96, 2 * rng.randrange(4, 100)])
            pairs = _split(rng, rng.choice([d // 2, d // 2, max(2, d // 4)]))
            many = _pairs_of(pairs)
            dealt = all(a + len(many) * (n - 1) < sum(many) for a, n in enumerate(many) if a)
            case = _axes(tokens, heads, kv, d, layout, dtype, rng.choice(["forward", "backward"]), pairs,
                         rng.choice(["sections", "cycled"]) if dealt else "sections", rng.choice(["shared", "own"]), docs,
                         tail=tail)
        if _cost(case) <= largest[kind]:
            return case


def _lens(c):
    """Document lengths: log-normal shares of the tokens, every fifth of many documents empty."""
    rng = random.Random(1000003 * c["docs"] + c["tokens"])
    n, docs = c["tokens"], c["docs"]
    share = [0.0 if docs >= 10 and i % 5 == 3 else rng.lognormvariate(0.0, c["spread"]) for i in range(docs)]
    ends = [round(n * s / sum(share)) for s in np.cumsum(share)]
    return [b - a for a, b in zip([0] + ends, ends)]


def _visible(c):
    """Visible pairs of queries and keys: min(i + 1, window) in the window, the first tokens in front of it."""
    total, w, s = 0, c["window"], c["sinks"]
    for n in _lens(c):
        m = min(n, w)
        total += m * (m + 1) // 2 + (n - m) * w
        if n > w:                       # query i >= w sees min(i + 1 - w, s) more
            k = min(n - w, s)
            total += k * (k + 1) // 2 + (n - w - k) * s
    return total


def work(case):
    c = case
    size = 2 if c.get("dtype", "bf16") == "bf16" else 4
    if c["kind"] in ("norm", "axes"):
        n = c["tokens"] * (c["heads"] + c["kv"]) * c["d"]
        pos = 8 * c["tokens"] * len(_pairs_of(c["pairs"]))
        if c["kind"] == "axes":
            return {"bytes": 2 * n * size + pos, "flops": 3 * n}
        train = c["train"]                                       # x read, y written; x and dy read, dx written
        return {"bytes": (5 if train else 2) * n * size + pos * (2 if train else 1), "flops": (6 + (14 if train else 0)) * n}
    if c["kind"] == "dropout":
        n = c["rows"] * c["cols"]                                # x and residual read, y written; dy read, dx written
        return {"bytes": n * size * (5 if c["train"] else 3), "flops": 2 * n}
    q, kv = c["tokens"] * c["heads"] * c["d"] * 2, c["tokens"] * c["kv"] * c["d"] * 2
    lse = c["tokens"] * c["heads"] * 4
    forward = 2 * q + 2 * kv + lse                               # q, k, v read, o and lse written
    backward = 4 * q + 4 * kv + lse if c["train"] else 0         # q, o, dO, k, v read, dQ, dK, dV written
    pair = _visible(c) * c["heads"] * c["d"]
    return {"bytes": forward + backward, "flops": pair * (FORWARD + (BACKWARD if c["train"] else 0))}


# ------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype=BF16, std=1.0, mean=0.0):
    return (mean + torch.randn(shape, generator=g, device="cuda", dtype=F32) * std).to(dtype)


_BASE = 500000.0


def _inputs(c, seed):
    """The tensors of a case, the same for every side."""
    g = _generator(seed)
    x = {}
    if c["kind"] == "dropout":
        dt, shape = DTYPES[c["dtype"]], (c["rows"], c["cols"])
        x["x"], x["residual"] = _normal(g, shape, dt), _normal(g, shape, dt)
        x["rng"] = torch.randint(-(1 << 62), 1 << 62, (2,), generator=g, device="cuda", dtype=torch.int64)   # seed, offset
        if c["train"]:
            x["d_y"] = _normal(g, shape, dt)
        return x
    rows = c["tokens"] + c["tail"]
    x["starts"] = torch.tensor([0] + list(np.cumsum(_lens(c))), dtype=torch.int64, device="cuda")
    dt = DTYPES[c.get("dtype", "bf16")]
    q, kv = (rows, c["heads"], c["d"]), (rows, c["kv"], c["d"])
    x["q"], x["k"] = _normal(g, q, dt), _normal(g, kv, dt)
    if c["kind"] == "window":
        x["v"] = _normal(g, kv)
        if c["train"]:
            x["d_o"] = _normal(g, q)
        return x
    n_axes = len(_pairs_of(c["pairs"]))
    # a patch's time or text position, then its places in the image
    x["positions"] = torch.stack(
        [torch.randint(0, 1 << (15 if a == 0 else 7), (rows,), generator=g, device="cuda", dtype=torch.int64)
         for a in range(n_axes)]) if n_axes else None
    if c["kind"] == "norm":
        x["q_gain"], x["k_gain"] = (_normal(g, (c["d"],), dt, 0.1, 1.0) for _ in range(2))
        if c["train"]:
            x["d_q"], x["d_k"] = _normal(g, q, dt), _normal(g, kv, dt)
    return x


def prepare(case, seed):
    c = case
    state = dict(_inputs(c, seed), case=c)
    if c["kind"] == "dropout":
        state["y"] = torch.zeros_like(state["x"])
        if c["train"]:
            state["d_x"] = torch.zeros_like(state["x"])
        return state
    state["lens"] = _lens(c)
    state["q_out"], state["k_out"] = torch.zeros_like(state["q"]), torch.zeros_like(state["k"])
    if c["kind"] == "norm" and c["train"]:
        state["dx_q"], state["dx_k"] = torch.zeros_like(state["q"]), torch.zeros_like(state["k"])
        state["d_q_gain"], state["d_k_gain"] = (torch.zeros((c["d"],), dtype=F32, device="cuda") for _ in range(2))
    if c["kind"] == "window":
        state["v_out"], state["o"] = torch.zeros_like(state["v"]), torch.zeros_like(state["q"])
        state["lse"] = torch.zeros((c["heads"], state["q"].shape[0]), dtype=F32, device="cuda")
    if own:                                   # the plan, the handles and the workspace that a program keeps
        import paper_2411_06465_amd as L
        size = 0
        state["packing"] = L.make_packing(state["starts"], state["q"].shape[0])
        if c["kind"] == "window":
            state["win"] = L.make_window(c["window"], c["sinks"])
            if c["train"]:
                size = L.l4d_attn_window_workspace_bytes(state["win"], state["q"].shape[0], c["heads"], c["kv"], c["d"])
        else:
            state["rope"] = L.make_rope(c["d"], c["rot"], c["layout"], _BASE)
            pairs = _pairs_of(c["pairs"])
            state["axes"] = L.make_rope_axes(pairs, c["order"], c["frequencies"]) if pairs else None
            if c["kind"] == "norm" and c["train"]:
                size = L.l4d_qk_norm_workspace_bytes(state["q"].shape[0], c["d"])
        if size:
            state["arena"] = L.Arena.on(torch.empty(size + 4096, dtype=torch.uint8, device="cuda"))
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    c = state["case"]
    if own:
        return _OWN[c["kind"]](c, state)
    return _PLAIN[c["kind"]](c, state)


def _own_norm(c, s):
    import paper_2411_06465_amd as L
    where = dict(positions=s["positions"], axes=s["axes"], packing=s["packing"])
    L.qk_norm_rope_fwd(s["rope"], s["q"], s["q_gain"], s["q_out"], s["k"], s["k_gain"], s["k_out"], eps=EPS, **where)
    out = {"q": s["q_out"], "k": s["k_out"]}
    if c["train"]:
        s["d_q_gain"].zero_()     # the gradient accumulators of a step's first micro-batch
        s["d_k_gain"].zero_()
        L.qk_norm_rope_bwd(s["rope"], s["q"], s["q_gain"], s["d_q"], s["dx_q"], s["d_q_gain"], s["arena"], s["k"],
                           s["k_gain"], s["d_k"], s["dx_k"], s["d_k_gain"], eps=EPS, **where)
        out.update(dq=s["dx_q"], dk=s["dx_k"], d_q_gain=s["d_q_gain"], d_k_gain=s["d_k_gain"])
    return out


def _own_axes(c, s):
    import paper_2411_06465_amd as L
    call = L.rope_axes_fwd if c["direction"] == "forward" else L.rope_axes_bwd
    call(s["rope"], s["axes"], s["q"], s["positions"], s["q_out"], s["k"], s["k_out"], packing=s["packing"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_window(c, s):
    import paper_2411_06465_amd as L
    L.attn_window_fwd(s["win"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["packing"])
    out = {"o": s["o"], "lse": s["lse"]}
    if c["train"]:
        L.attn_window_bwd(s["win"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["d_o"], s["q_out"], s["k_out"], s["v_out"],
                          s["packing"], s["arena"])
        out.update(dq=s["q_out"], dk=s["k_out"], dv=s["v_out"])
    return out


def _own_dropout(c, s):
    import paper_2411_06465_amd as L
    L.dropout_add_fwd(s["x"], s["residual"], s["y"], s["rng"], c["p"], first_row=c["first_row"])
    out = {"y": s["y"]}
    if c["train"]:
        L.dropout_add_bwd(s["d_y"], s["d_x"], s["rng"], c["p"], first_row=c["first_row"])
        out["d_x"] = s["d_x"]
    return out


_OWN = {"norm": _own_norm, "axes": _own_axes, "window": _own_window, "dropout": _own_dropout}


# ------------------------------------------------------------------ the plain forms

def _pair_axes(c):
    """(axis, rank within it, pairs of it) of every pair, as vectors."""
    pairs = _pairs_of(c["pairs"])
    n, total = len(pairs), sum(pairs)
    j = np.arange(total)
    if c["order"] == "sections":
        axis = np.repeat(np.arange(n), pairs)
    else:
        axis = np.where(j < n * np.asarray(pairs)[j % n], j % n, 0)
    rank = (np.cumsum(axis[:, None] == np.arange(n), axis=0) - 1)[j, axis]
    return axis, rank, np.asarray(pairs)[axis]


def _positions(s, rows):
    """Each row's distance from its document's start; -1 behind the last document."""
    starts = s["starts"]
    row = torch.arange(rows, dtype=torch.int64, device="cuda")
    doc = torch.searchsorted(starts, row, right=True) - 1
    return torch.where(row < starts[-1], row - starts[doc], torch.full_like(row, -1))


def _angles(c, s):
    """Angle of every row and pair, in 64 bits."""
    half = c["rot"] // 2
    if not c["pairs"]:
        j = torch.arange(half, dtype=F64, device="cuda")
        pos = _positions(s, s["q"].shape[0]).to(F64)[:, None]
        return pos * torch.pow(torch.tensor(_BASE, dtype=F64, device="cuda"), -2.0 * j / c["rot"])[None, :]
    axis, rank, many = _pair_axes(c)
    share = rank / many if c["frequencies"] == "own" else np.arange(half) / half
    f = torch.pow(torch.tensor(_BASE, dtype=F64, device="cuda"), -torch.from_numpy(share).cuda())
    return s["positions"].to(F64)[torch.from_numpy(axis).cuda()].t() * f[None, :]


def _turn(c, y, cos, sin):
    """The pairs of every head of y turned, in 32 bits."""
    rot, half = c["rot"], c["rot"] // 2
    if c["layout"] == "half":
        a, b = y[..., :half], y[..., half:rot]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., rot:]], -1)
    a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), y[..., rot:]], -1)


def _plain_axes(c, s):
    inside = (_positions(s, s["q"].shape[0]) >= 0)[:, None, None]
    angle = _angles(c, s)
    cos, sin = torch.cos(angle).to(F32)[:, None, :], torch.sin(angle).to(F32)[:, None, :]
    if c["direction"] == "backward":
        sin = -sin
    return {t: torch.where(inside, _turn(c, s[t].to(F32), cos, sin), 0.0).to(s[t].dtype) for t in ("q", "k")}


def _plain_norm(c, s):
    inside = (_positions(s, s["q"].shape[0]) >= 0)[:, None, None]
    angle = _angles(c, s)
    cos, sin = torch.cos(angle).to(F32)[:, None, :], torch.sin(angle).to(F32)[:, None, :]
    out = {}

    def one(t, gain):
        x, g = s[t].to(F32), s[gain].to(F32)
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        xhat = x * rstd
        out[t] = torch.where(inside, _turn(c, xhat * g, cos, sin), 0.0).to(s[t].dtype)
        if not c["train"]:
            return
        dn = torch.where(inside, _turn(c, s["d_" + t].to(F32), cos, -sin), 0.0)
        dxhat = dn * g
        out["d" + t] = (rstd * (dxhat - xhat * (dxhat * xhat).mean(-1, keepdim=True))).to(s[t].dtype)
        out["d_" + gain] = (dn * xhat).sum((0, 1))

    one("q", "q_gain")
    one("k", "k_gain")
    return {t: out[t] for t in ("q", "k", "dq", "dk", "d_q_gain", "d_k_gain") if t in out}


def _plain_window(c, s):
    """Document by document: blocks of queries against the keys of their window and the first
    tokens, each group of query heads under one another."""
    group, scale, d, kv = c["heads"] // c["kv"], 1.0 / math.sqrt(c["d"]), c["d"], c["kv"]
    out = {"o": torch.zeros_like(s["q"]), "lse": torch.zeros_like(s["lse"])}
    if c["train"]:
        out.update(dq=torch.zeros_like(s["q"]), dk=torch.zeros_like(s["k"]), dv=torch.zeros_like(s["v"]))
    first = 0
    for n in s["lens"]:
        at = slice(first, first + n)
        first += n
        if n == 0:
            continue
        front = min(c["window"] - 1, n - 1)                  # keys in front of a block that its rows may see
        b = min(n, max(128, min(c["window"], 1024)))         # rows of a block
        nb, sinks = -(-n // b), min(c["sinks"], n)
        rows = nb * b
        qi = torch.arange(rows, device="cuda").view(nb, b, 1)
        ki = (torch.arange(nb, device="cuda") * b - front)[:, None, None] + torch.arange(front + b, device="cuda")
        si = torch.arange(sinks, device="cuda")
        seen = torch.cat([(ki >= 0) & (ki < n) & (ki <= qi) & (qi - ki < c["window"]),
                          (qi - si >= c["window"]).expand(nb, b, sinks)], -1)[:, None, None]
        take = ki.view(nb, -1).clamp(0, n - 1)

        def blocks(x, count):                                # [nb * kv][group * b][d]
            y = torch.zeros((rows, count, d), dtype=F32, device="cuda")
            y[:n] = x[at]
            return y.view(nb, b, kv, count // kv, d).permute(0, 2, 3, 1, 4).reshape(nb * kv, -1, d)

        def keys(x):                                         # [nb * kv][front + b + sinks][d]
            y = x[at].to(F32)
            y = torch.cat([y[take], y[:sinks].expand(nb, sinks, kv, d)], 1)
            return y.transpose(1, 2).reshape(nb * kv, -1, d)

        q, k, v = blocks(s["q"], c["heads"]), keys(s["k"]), keys(s["v"])
        many = k.shape[1]
        p = (torch.bmm(q, k.transpose(1, 2).contiguous()) * scale).view(nb, kv, group, b, many)
        p.masked_fill_(~seen, float("-inf"))
        top = p.amax(-1, keepdim=True).clamp_min(-3e38)      # rows behind the document see nothing
        p.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        p.div_(total)
        lse = (top + total.log()).view(nb, kv * group, b).transpose(0, 1).reshape(c["heads"], rows)
        out["lse"][:, at] = lse[:, :n]
        pg = p.view(nb * kv, group * b, many).nan_to_num_(0.0)
        o = torch.bmm(pg, v)

        def rows_of(x):                                      # back to [n][heads][d]
            return x.view(nb, kv, group, b, d).permute(0, 3, 1, 2, 4).reshape(rows, c["heads"], d)[:n].to(BF16)

        out["o"][at] = rows_of(o)
        if not c["train"]:
            continue

        def keys_of(x):                                      # the sums of the blocks' parts
            x = x.view(nb, kv, many, d).transpose(1, 2)
            y = torch.zeros((n, kv, d), dtype=F32, device="cuda")
            y.index_add_(0, take.reshape(-1), x[:, :front + b].reshape(-1, kv, d))
            y[:sinks] += x[:, front + b:].sum(0)
            return y.to(BF16)

        do = blocks(s["d_o"], c["heads"])
        out["dv"][at] = keys_of(torch.bmm(pg.transpose(1, 2).contiguous(), do))
        ds = torch.bmm(do, v.transpose(1, 2).contiguous())
        ds.sub_((do * o).sum(-1, keepdim=True)).mul_(pg).mul_(scale)
        out["dq"][at] = rows_of(torch.bmm(ds, k))
        out["dk"][at] = keys_of(torch.bmm(ds.transpose(1, 2).contiguous(), q))
    return out


def _words(c, rng):
    """The random 32-bit word of every element: word e % 4 of Philox4x32-10 at counter e / 4 of the
    element's place e in the whole array, its upper half the offset, its key the seed."""
    rows, cols = c["rows"], c["cols"]
    first = c["first_row"] * cols
    b0, n = first // 4, (first + rows * cols + 3) // 4 - first // 4
    block = torch.arange(n, dtype=torch.int64, device="cuda") + b0
    x0, x1 = block & WORD, block >> 32
    x2, x3 = (rng[1] & WORD).expand(n), (rng[1] >> 32 & WORD).expand(n)
    k0, k1 = rng[0] & WORD, rng[0] >> 32 & WORD
    for i in range(10):
        p, q = x0 * 0xD2511F53, x2 * 0xCD9E8D57               # the products modulo 2^64
        a, b = (k0 + i * 0x9E3779B9) & WORD, (k1 + i * 0xBB67AE85) & WORD
        x0, x1, x2, x3 = (q >> 32 & WORD) ^ x1 ^ a, q & WORD, (p >> 32 & WORD) ^ x3 ^ b, p & WORD
    return torch.stack([x0, x1, x2, x3], -1).view(-1)[first - 4 * b0:][:rows * cols].view(rows, cols)


def _plain_dropout(c, s):
    keep = _words(c, s["rng"]) >= round(c["p"] * 2 ** 32)
    scale = 1.0 / (1.0 - c["p"])
    out = {"y": (s["residual"].to(F32) + torch.where(keep, s["x"].to(F32) * scale, 0.0)).to(s["x"].dtype)}
    if c["train"]:
        out["d_x"] = torch.where(keep, s["d_y"].to(F32) * scale, 0.0).to(s["x"].dtype)
    return out


_PLAIN = {"norm": _plain_norm, "axes": _plain_axes, "window": _plain_window, "dropout": _plain_dropout}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    return _EXACT[case["kind"]](case, _inputs(case, seed))


def _rotor(c, x):
    """exp(i angle) of every row and pair, and which rows belong to a document."""
    lens, half = _lens(c), c["rot"] // 2
    pairs = _pairs_of(c["pairs"])
    if pairs:
        owner, left = [], list(pairs)
        for j in range(half):                                # deal the pairs out
            if c["order"] == "sections":
                a = next(i for i, n in enumerate(left) if n > 0)
            else:
                a = j % len(pairs) if j // len(pairs) < pairs[j % len(pairs)] else 0
            owner.append((a, pairs[a] - left[a]))
            left[a] -= 1
        own_count = c["frequencies"] == "own"
        f = [_BASE ** (-(i / pairs[a] if own_count else j / half)) for j, (a, i) in enumerate(owner)]
        pos = torch.stack([x["positions"][a] for a, _ in owner], 1).double()
    else:
        f = [_BASE ** (-j / half) for j in range(half)]
        pos = torch.tensor(np.concatenate([np.arange(n) for n in lens] + [np.zeros(c["tail"])]), dtype=F64, device="cuda")[:, None]
    angle = pos * torch.tensor(f, dtype=F64, device="cuda")
    return torch.polar(torch.ones_like(angle), angle)[:, None, :], sum(lens)


def _complex_turn(c, t, turn):
    rot, half = c["rot"], c["rot"] // 2
    parts = [slice(0, half), slice(half, rot)] if c["layout"] == "half" else [slice(0, rot, 2), slice(1, rot, 2)]
    z = torch.complex(t[..., parts[0]].contiguous(), t[..., parts[1]].contiguous()) * turn
    y = torch.cat([z.real, z.imag], -1) if c["layout"] == "half" else torch.view_as_real(z).flatten(-2)
    return torch.cat([y, t[..., rot:]], -1)


def _exact_axes(c, x):
    turn, n = _rotor(c, x)
    if c["direction"] == "backward":
        turn = turn.conj()
    out = {t: _complex_turn(c, x[t].double(), turn) for t in ("q", "k")}
    for y in out.values():
        y[n:] = 0.0
    return out


def _exact_norm(c, x):
    """The gradients by differentiation."""
    turn, n = _rotor(c, x)
    out = {}
    for t, gain in (("q", "q_gain"), ("k", "k_gain")):
        a, g = x[t].double().requires_grad_(c["train"]), x[gain].double().requires_grad_(c["train"])
        y = _complex_turn(c, a / torch.sqrt(a.square().sum(-1, keepdim=True) / c["d"] + EPS) * g, turn)[:n]
        out[t] = torch.cat([y.detach(), torch.zeros_like(a.detach()[n:])])
        if c["train"]:
            out["d" + t], out["d_" + gain] = torch.autograd.grad(y, (a, g), x["d_" + t][:n].double())
    return {t: out[t] for t in ("q", "k", "dq", "dk", "d_q_gain", "d_k_gain") if t in out}


def _exact_window(c, x):
    """Softmax attention of every document and head under the whole mask, the gradients by differentiation."""
    lens, group = _lens(c), c["heads"] // c["kv"]
    if sum(n * n for n in lens) * c["heads"] * c["d"] > 3e12:
        return None
    out = {"o": torch.zeros_like(x["q"], dtype=F64),
           "lse": torch.zeros((c["heads"], x["q"].shape[0]), dtype=F64, device="cuda")}
    if c["train"]:
        out.update(dq=torch.zeros_like(out["o"]), dk=torch.zeros_like(x["k"], dtype=F64),
                   dv=torch.zeros_like(x["v"], dtype=F64))
    for end, n in zip(np.cumsum(lens), lens):
        if n == 0:
            continue
        at = slice(int(end) - n, int(end))
        i = torch.arange(n, device="cuda")
        back = i[:, None] - i[None, :]
        hidden = (back < 0) | ((back >= c["window"]) & (i[None, :] >= c["sinks"]))
        mask = torch.zeros((n, n), dtype=F64, device="cuda").masked_fill_(hidden, float("-inf"))
        for h in range(c["heads"]):
            q, k, v = (x[t][at, i].double().requires_grad_(c["train"])
                       for t, i in (("q", h), ("k", h // group), ("v", h // group)))
            scores = q @ k.t() / math.sqrt(c["d"]) + mask
            o = torch.softmax(scores, -1) @ v
            out["o"][at, h] = o.detach()
            out["lse"][h, at] = torch.logsumexp(scores.detach(), -1)
            if c["train"]:
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), x["d_o"][at, h].double())
                out["dq"][at, h] = dq
                out["dk"][at, h // group] += dk
                out["dv"][at, h // group] += dv
    return out


def _exact_dropout(c, x):
    """The words in unsigned 64-bit arithmetic on the host."""
    rows, cols = c["rows"], c["cols"]
    e = np.arange(rows * cols, dtype=np.uint64) + np.uint64(c["first_row"] * cols)
    block = np.arange(int(e[0]) >> 2, (int(e[-1]) >> 2) + 1, dtype=np.uint64)
    at = ((e >> np.uint64(2)) - block[0]).astype(np.int64)
    seed, offset = (int(v) & (1 << 64) - 1 for v in x["rng"].tolist())
    low, s32 = np.uint64(WORD), np.uint64(32)
    r = [block & low, block >> s32, np.full_like(block, offset & WORD), np.full_like(block, offset >> 32)]
    key = [seed & WORD, seed >> 32]
    for _ in range(10):
        p, q = r[0] * np.uint64(0xD2511F53), r[2] * np.uint64(0xCD9E8D57)
        r = [(q >> s32) ^ r[1] ^ np.uint64(key[0]), q & low, (p >> s32) ^ r[3] ^ np.uint64(key[1]), p & low]
        key = [(key[0] + 0x9E3779B9) & WORD, (key[1] + 0xBB67AE85) & WORD]
    words = np.stack(r, -1)[at, (e & np.uint64(3)).astype(np.int64)]
    keep = torch.from_numpy(words >= np.uint64(round(c["p"] * 2 ** 32))).cuda().view(rows, cols).double()
    out = {"y": x["residual"].double() + keep * x["x"].double() / (1.0 - c["p"])}
    if c["train"]:
        out["d_x"] = keep * x["d_y"].double() / (1.0 - c["p"])
    return out


_EXACT = {"norm": _exact_norm, "axes": _exact_axes, "window": _exact_window, "dropout": _exact_dropout}
