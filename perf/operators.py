"""The operators that train on packed documents, and their plain forms.

Rotary positions counted from each document's start, causal attention that
stops at document borders, and the cross-entropy of the LM head without stored
logits.  Every case is one call, or a forward and the backward that follows it,
as a training or evaluation step over one packed micro-batch makes it.

With `own` false, `run` computes the operators in their plain form: elementary
torch operations in 32 bits (angles in 64), rounded once at the end.  With
`own` true it calls the library.  A case is a dict of plain values; `draw` gives
more cases of the same ranges.

Documents of a micro-batch have log-normal lengths (text is heavy-tailed); with
many of them some are empty; `tail` rows behind the last one are padding.
Queries and keys are N(0, 1) rows, values and gradients N(0, 1), weights
N(0, 0.02), targets uniform with a share of them ignored (document ends,
padding), the other vocabulary shards' statistics what such a head gives.
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DTYPES = {"bf16": BF16, "f32": F32}
FORWARD, BACKWARD = 4, 10    # attention flops per pair, head and channel: two products forward, five backward


# ------------------------------------------------------------------ the cases

def _rope(tokens, heads, kv, d, rot, layout, scaling, dtype, direction, docs, tail=0, far=False, **name):
    return dict(name, kind="rope", tokens=tokens, heads=heads, kv=kv, d=d, rot=rot, layout=layout, scaling=scaling,
                dtype=dtype, direction=direction, docs=docs, tail=tail, far=far, spread=1.0)


def _attn(tokens, heads, kv, d, docs, train, tail=0, spread=1.0, **name):
    return dict(name, kind="attn", tokens=tokens, heads=heads, kv=kv, d=d, docs=docs, train=train, tail=tail,
                spread=spread)


def _loss(tokens, hidden, vocab, tp, train, ignored=0.05, **name):
    return dict(name, kind="loss", tokens=tokens, hidden=hidden, vocab=vocab, tp=tp, train=train, ignored=ignored)


def listed():
    return [
        # the heads of a small model on a handful of tokens: the call's latency is what counts
        _rope(48, 4, 2, 64, 64, "half", "none", "bf16", "forward", 3, name="rope-tiny"),
        # Llama-3-8B's heads over a packed row of 8192 tokens, frequencies scaled by wavelength
        _rope(8192, 32, 8, 128, 128, "half", "bands", "bf16", "forward", 23, tail=100, name="rope-8b"),
        # interleaved pairs on half of each head, fp32, an odd token count at far positions, backward
        _rope(4099, 16, 16, 128, 64, "interleaved", "ramp", "f32", "backward", 1, far=True, name="rope-far-f32-bwd"),
        # the smallest training call: head size 64, three short documents
        _attn(128, 4, 2, 64, 3, True, name="attn-tiny-train"),
        # Llama-2-7B's heads, evaluation of a packed row with padding behind it
        _attn(4000, 32, 32, 128, 7, False, tail=200, name="attn-7b-eval"),
        # Llama-3-8B's heads on a packed row of 8192 tokens
        _attn(8192, 32, 8, 128, 23, True, tail=61, name="attn-8b-train"),
        # many short documents (chat turns) on heads of size 64
        _attn(16384, 16, 4, 64, 160, True, spread=0.6, name="attn-short-docs-train"),
        # Llama-3-70B's heads at TP8 on a long row: a few long documents carry nearly all pairs
        _attn(32768, 8, 1, 128, 6, True, spread=1.3, name="attn-70b-tp8-long-train"),
        # the test model's head: launches and latency count
        _loss(128, 256, 1000, 1, True, name="loss-tiny-train"),
        # an odd vocabulary and an odd token count
        _loss(777, 1024, 32003, 1, True, ignored=0.3, name="loss-odd-train"),
        # Llama-3-8B's whole vocabulary, evaluation
        _loss(2000, 4096, 128256, 1, False, name="loss-8b-eval"),
        # Llama-3-8B at TP4, training
        _loss(8192, 4096, 128256, 4, True, name="loss-8b-tp4-train"),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _cost(case):
    w = work(case)
    return w["flops"] / 1e15 + w["bytes"] / 5e12


def draw(rng):
    largest = {}
    for c in listed():
        largest[c["kind"]] = max(largest.get(c["kind"], 0.0), _cost(c))
    while True:
        kind = rng.choice(["rope", "attn", "attn", "loss", "loss"])
        if kind == "loss":
            vocab = rng.choice([32000, 128256, round(_log_uniform(rng, 40, 64000))])
            case = _loss(max(1, round(_log_uniform(rng, 1, 8192))), rng.choice([256, 512, 1024, 2048, 4096, 8192]),
                         vocab, rng.choice([t for t in (1, 2, 4, 8) if vocab % t == 0]), rng.random() < 0.7,
                         ignored=rng.choice([0.0, 0.05, 0.5]))
        else:
            heads, kv = rng.choice([(4, 2), (8, 1), (16, 4), (32, 8), (32, 32), (12, 4), (5, 5), (14, 2)])
            d = rng.choice([64, 128, 128])
            tokens = max(1, round(_log_uniform(rng, 1, 32768 if kind == "attn" else 16384)))
            docs = max(1, min(tokens, round(_log_uniform(rng, 1, 200))))
            tail = rng.choice([0, 0, rng.randrange(300)])
            if kind == "attn":
                # documents of one token alone would have no gradient of q and k to compare
                case = _attn(tokens, heads, kv, d, docs, tokens >= 2 * docs and rng.random() < 0.8, tail=tail,
                             spread=rng.choice([0.3, 1.0, 1.5]))
            else:
                case = _rope(tokens, heads, kv, d, rng.choice([d, d, d // 2, 16 * rng.randrange(1, d // 16 + 1)]),
                             rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "bands", "ramp"]),
                             rng.choice(["bf16", "bf16", "f32"]), rng.choice(["forward", "backward"]), docs, tail=tail,
                             far=rng.random() < 0.3)
        if _cost(case) <= largest[kind]:
            return case


def _lens(c):
    """Document lengths: log-normal shares of the tokens, every fifth of many documents empty."""
    rng = random.Random(1000003 * c["docs"] + c["tokens"])
    n, docs = c["tokens"], c["docs"]
    share = [0.0 if docs >= 10 and i % 5 == 3 else rng.lognormvariate(0.0, c["spread"]) for i in range(docs)]
    ends = [round(n * s / sum(share)) for s in np.cumsum(share)]
    return [b - a for a, b in zip([0] + ends, ends)]


def _pairs(c):
    return sum(n * (n + 1) // 2 for n in _lens(c))


def work(case):
    c = case
    if c["kind"] == "rope":
        n = c["tokens"] * (c["heads"] + c["kv"]) * c["d"]
        return {"bytes": 2 * n * (2 if c["dtype"] == "bf16" else 4) + 8 * c["tokens"], "flops": 3 * n}
    if c["kind"] == "attn":
        q, kv = c["tokens"] * c["heads"] * c["d"] * 2, c["tokens"] * c["kv"] * c["d"] * 2
        lse = c["tokens"] * c["heads"] * 4
        forward = 2 * q + 2 * kv + lse                       # q, k, v read, o and lse written
        backward = 4 * q + 4 * kv + lse if c["train"] else 0   # q, o, dO, k, v read, dQ, dK, dV written
        pair = _pairs(c) * c["heads"] * c["d"]
        return {"bytes": forward + backward, "flops": pair * (FORWARD + (BACKWARD if c["train"] else 0))}
    n, h, v = c["tokens"], c["hidden"], c["vocab"] // c["tp"]
    x, w = n * h * 2, v * h * 2
    forward, backward = x + w + 16 * n, (2 * x + w + 4 * v * h + 16 * n if c["train"] else 0)
    return {"bytes": forward + backward, "flops": 2.0 * n * h * v * (4 if c["train"] else 1)}


# ------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype=BF16, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=F32) * std).to(dtype)


_SCALING = {  # a context stretched eightfold from 8192 positions
    "none": {}, "linear": dict(factor=8.0),
    "bands": dict(factor=8.0, low=1.0, high=4.0, original=8192),
    "ramp": dict(factor=8.0, low=1.0, high=32.0, original=8192, amplitude=0.1 * math.log(8.0) + 1.0),
}
_BASE = 500000.0


def _inputs(c, seed):
    """The tensors of a case, the same for every side."""
    g = _generator(seed)
    x = {}
    if c["kind"] in ("rope", "attn"):
        rows = c["tokens"] + c["tail"]
        x["starts"] = torch.tensor([0] + list(np.cumsum(_lens(c))), dtype=torch.int64, device="cuda")
    if c["kind"] == "rope":
        dt = DTYPES[c["dtype"]]
        x["q"], x["k"] = _normal(g, (rows, c["heads"], c["d"]), dt), _normal(g, (rows, c["kv"], c["d"]), dt)
        x["positions"] = (torch.randint(0, 1 << 20, (rows,), generator=g, device="cuda", dtype=torch.int64)
                          if c["far"] else None)
    elif c["kind"] == "attn":
        q, kv = (rows, c["heads"], c["d"]), (rows, c["kv"], c["d"])
        x["q"], x["k"], x["v"] = _normal(g, q), _normal(g, kv), _normal(g, kv)
        if c["train"]:
            x["d_o"] = _normal(g, q)
    else:
        n, h, v, t = c["tokens"], c["hidden"], c["vocab"] // c["tp"], c["tp"]
        x["hidden"], x["w_lm"] = _normal(g, (n, h)), _normal(g, (v, h), std=0.02)
        tg = torch.randint(0, c["vocab"], (n,), generator=g, device="cuda", dtype=torch.int64)
        skip = torch.rand((n,), generator=g, device="cuda") < c["ignored"]
        x["targets"] = torch.where(skip, torch.full_like(tg, -1), tg)
        z_std = 0.02 * math.sqrt(h)
        x["peer_lse"] = x["peer_z"] = None
        if t > 1:
            x["peer_lse"] = math.log(v * (t - 1)) + z_std ** 2 / 2 + 0.01 * _normal(g, (n,), F32)
            x["peer_z"] = z_std * _normal(g, (n,), F32)
        if c["train"]:   # each token's weight in the mean loss
            x["d_loss"] = torch.rand((n,), generator=g, device="cuda", dtype=F32) / n
    return x


def prepare(case, seed):
    c = case
    state = dict(_inputs(c, seed), case=c)
    if c["kind"] in ("rope", "attn"):
        state["lens"] = _lens(c)
        state["q_out"] = torch.zeros_like(state["q"])
        state["k_out"] = torch.zeros_like(state["k"])
    if c["kind"] == "attn":
        state["v_out"] = torch.zeros_like(state["v"])
        state["o"] = torch.zeros_like(state["q"])
        state["lse"] = torch.zeros((c["heads"], state["q"].shape[0]), dtype=F32, device="cuda")
    if c["kind"] == "loss":
        n = c["tokens"]
        state["loss"], state["lse"] = (torch.zeros((n,), dtype=F32, device="cuda") for _ in range(2))
        if c["train"]:
            state["d_hidden"] = torch.zeros_like(state["hidden"])
            state["d_w"] = torch.zeros(state["w_lm"].shape, dtype=F32, device="cuda")
    if own:
        import paper_2411_06465_amd as L
        size = 0
        if c["kind"] == "rope":
            state["rope"] = L.make_rope(c["d"], c["rot"], c["layout"], _BASE, c["scaling"], **_SCALING[c["scaling"]])
        elif c["kind"] == "attn" and c["train"]:
            size = L.l4d_attn_packed_workspace_bytes(state["q"].shape[0], c["heads"], c["kv"], c["d"])
        elif c["kind"] == "loss":
            size = max(L.l4d_lm_loss_workspace_bytes(c["tokens"], c["hidden"], state["w_lm"].shape[0]))
        if c["kind"] in ("rope", "attn"):
            state["packing"] = L.make_packing(state["starts"], state["q"].shape[0])
        if size:
            state["arena"] = L.Arena.on(torch.empty(size + 4096, dtype=torch.uint8, device="cuda"))
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    c = state["case"]
    if own:
        return _OWN[c["kind"]](c, state)
    return _PLAIN[c["kind"]](c, state)


def _own_rope(c, s):
    import paper_2411_06465_amd as L
    call = L.rope_fwd if c["direction"] == "forward" else L.rope_bwd
    call(s["rope"], s["q"], s["q_out"], s["k"], s["k_out"], positions=s["positions"], packing=s["packing"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_attn(c, s):
    import paper_2411_06465_amd as L
    L.attn_packed_fwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["packing"])
    out = {"o": s["o"], "lse": s["lse"]}
    if c["train"]:
        L.attn_packed_bwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["d_o"], s["q_out"], s["k_out"], s["v_out"],
                          s["packing"], s["arena"])
        out.update(dq=s["q_out"], dk=s["k_out"], dv=s["v_out"])
    return out


def _own_loss(c, s):
    import paper_2411_06465_amd as L
    L.lm_loss_fwd(s["hidden"], s["w_lm"], s["targets"], s["loss"], s["lse"], s["arena"], peer_lse=s["peer_lse"],
                  peer_target_logit=s["peer_z"])
    out = {"loss": s["loss"], "lse": s["lse"]}
    if c["train"]:
        s["d_w"].zero_()      # the gradient accumulator of a step's first micro-batch
        L.lm_loss_bwd(s["hidden"], s["w_lm"], s["targets"], s["lse"], s["d_hidden"], s["d_w"], s["arena"],
                      d_loss=s["d_loss"])
        out.update(d_hidden=s["d_hidden"], d_w=s["d_w"])
    return out


_OWN = {"rope": _own_rope, "attn": _own_attn, "loss": _own_loss}


# ------------------------------------------------------------------ the plain forms

def _frequencies(c):
    """Angle per position of each pair, in 64 bits."""
    rot, s = c["rot"], _SCALING[c["scaling"]]
    j = torch.arange(rot // 2, dtype=F64, device="cuda")
    f = torch.pow(torch.tensor(_BASE, dtype=F64, device="cuda"), -2.0 * j / rot)
    if c["scaling"] == "none":
        return f
    if c["scaling"] == "linear":
        return f / s["factor"]
    if c["scaling"] == "bands":
        turns = s["original"] * f / (2 * math.pi)             # rotations over the original context
        keep = ((turns - s["low"]) / (s["high"] - s["low"])).clamp(0.0, 1.0)
    else:
        def pair(r):
            return rot * math.log(s["original"] / (2 * math.pi * r)) / (2 * math.log(_BASE))
        lo, hi = max(math.floor(pair(s["high"])), 0), min(math.ceil(pair(s["low"])), rot - 1)
        keep = 1.0 - ((j - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
    return f * (keep + (1.0 - keep) / s["factor"])


def _positions(s, rows):
    """Each row's distance from its document's start; -1 behind the last document."""
    starts = s["starts"]
    row = torch.arange(rows, dtype=torch.int64, device="cuda")
    doc = torch.searchsorted(starts, row, right=True) - 1
    return torch.where(row < starts[-1], row - starts[doc], torch.full_like(row, -1))


def _plain_rope(c, s):
    rows = s["q"].shape[0]
    inside = _positions(s, rows) >= 0
    pos = s["positions"] if s["positions"] is not None else _positions(s, rows)
    angle = pos.to(F64)[:, None] * _frequencies(c)[None, :]
    amp = _SCALING[c["scaling"]].get("amplitude", 1.0)
    cos, sin = (amp * torch.cos(angle)).to(F32)[:, None, :], (amp * torch.sin(angle)).to(F32)[:, None, :]
    if c["direction"] == "backward":
        sin = -sin
    rot, half = c["rot"], c["rot"] // 2

    def turn(x):
        y = x.to(F32)
        if c["layout"] == "half":
            a, b = y[..., :half], y[..., half:rot]
            z = torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., rot:]], -1)
        else:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            z = torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), y[..., rot:]], -1)
        return torch.where(inside[:, None, None], z, torch.zeros_like(z)).to(x.dtype)

    return {"q": turn(s["q"]), "k": turn(s["k"])}


def _plain_attn(c, s):
    group, scale = c["heads"] // c["kv"], 1.0 / math.sqrt(c["d"])
    out = {"o": torch.zeros_like(s["q"]), "lse": torch.zeros_like(s["lse"])}
    if c["train"]:
        out.update(dq=torch.zeros_like(s["q"]), dk=torch.zeros_like(s["k"]), dv=torch.zeros_like(s["v"]))
    first = 0
    for n in s["lens"]:
        at = slice(first, first + n)
        first += n
        if n == 0:
            continue

        def heads(x):                                        # [heads][n][d]
            return x[at].to(F32).transpose(0, 1).contiguous()

        q, k, v = heads(s["q"]), heads(s["k"]), heads(s["v"])
        q = q.view(c["kv"], group * n, c["d"])               # the query heads of a kv-head, one under another
        p = (torch.bmm(q, k.transpose(1, 2).contiguous()) * scale).view(c["heads"], n, n)
        later = torch.ones((n, n), dtype=torch.bool, device="cuda").triu_(1)
        p.masked_fill_(later, float("-inf"))
        top = p.amax(-1, keepdim=True)
        p.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        p.div_(total)
        out["lse"][:, at] = (top + total.log())[..., 0]
        pg = p.view(c["kv"], group * n, n)
        o = torch.bmm(pg, v)

        def back(x, count):                                  # to [n][heads][d]
            return x.view(count, n, c["d"]).transpose(0, 1).to(BF16)

        out["o"][at] = back(o, c["heads"])
        if c["train"]:
            do = heads(s["d_o"]).view(c["kv"], group * n, c["d"])
            out["dv"][at] = back(torch.bmm(pg.transpose(1, 2).contiguous(), do), c["kv"])
            ds = torch.bmm(do, v.transpose(1, 2).contiguous())
            ds.sub_((do * o).sum(-1, keepdim=True)).mul_(pg).mul_(scale)
            out["dq"][at] = back(torch.bmm(ds, k), c["heads"])
            out["dk"][at] = back(torch.bmm(ds.transpose(1, 2).contiguous(), q), c["kv"])
    return out


def _plain_loss(c, s):
    hidden, w, targets = s["hidden"].to(F32), s["w_lm"].to(F32), s["targets"]
    n, v = hidden.shape[0], w.shape[0]
    logits = hidden @ w.t()
    top = logits.amax(-1)
    lse = top + (logits - top[:, None]).exp().sum(-1).log()
    here = (targets >= 0) & (targets < v)
    row = torch.arange(n, device="cuda")
    z = logits[row, targets.clamp(0, v - 1)]
    if s["peer_lse"] is not None:
        big = torch.maximum(lse, s["peer_lse"])
        lse = big + ((lse - big).exp() + (s["peer_lse"] - big).exp()).log()
        z = torch.where(here, z, s["peer_z"])
    loss = torch.where(targets >= 0, lse - z, torch.zeros_like(lse))
    out = {"loss": loss, "lse": lse}
    if c["train"]:
        g = (logits - lse[:, None]).exp()
        g[row, targets.clamp(0, v - 1)] -= here.to(F32)
        g *= torch.where(targets >= 0, s["d_loss"], torch.zeros_like(lse))[:, None]
        out.update(d_hidden=(g @ w).to(BF16), d_w=g.t() @ hidden)
    return out


_PLAIN = {"rope": _plain_rope, "attn": _plain_attn, "loss": _plain_loss}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    return _EXACT[case["kind"]](case, _inputs(case, seed))


def _exact_rope(c, x):
    """Each pair a complex number, turned by exp(i angle)."""
    lens, rows, rot, amp = _lens(c), x["q"].shape[0], c["rot"], 1.0
    s = _SCALING[c["scaling"]]
    freq = []
    for j in range(rot // 2):
        f = math.exp(-2.0 * j / rot * math.log(_BASE))
        if c["scaling"] == "linear":
            f /= s["factor"]
        elif c["scaling"] == "bands":
            length = 2 * math.pi / f
            if length > s["original"] / s["low"]:
                f /= s["factor"]
            elif length >= s["original"] / s["high"]:
                m = (s["original"] / length - s["low"]) / (s["high"] - s["low"])
                f = (1 - m) * f / s["factor"] + m * f
        elif c["scaling"] == "ramp":
            amp = s["amplitude"]
            edge = [rot * math.log(s["original"] / (2 * math.pi * r)) / (2 * math.log(_BASE))
                    for r in (s["high"], s["low"])]
            lo, hi = max(math.floor(edge[0]), 0), min(math.ceil(edge[1]), rot - 1)
            m = min(max((j - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = m * f / s["factor"] + (1 - m) * f
        freq.append(f)
    pos = np.concatenate([np.arange(n) for n in lens] + [np.zeros(c["tail"])])
    pos = torch.tensor(pos, dtype=F64, device="cuda") if x["positions"] is None else x["positions"].double()
    angle = torch.outer(pos, torch.tensor(freq, dtype=F64, device="cuda"))
    turn = torch.polar(torch.full_like(angle, amp), angle if c["direction"] == "forward" else -angle)[:, None, :]
    n, half = sum(lens), rot // 2

    def rotate(t):
        y = t.double().clone()
        pair = [(0, half, 1), (half, rot, 1)] if c["layout"] == "half" else [(0, rot, 2), (1, rot, 2)]
        parts = [slice(*p) for p in pair]
        z = torch.complex(y[..., parts[0]].contiguous(), y[..., parts[1]].contiguous()) * turn
        y[..., parts[0]], y[..., parts[1]] = z.real, z.imag
        y[n:rows] = 0.0
        return y

    return {"q": rotate(x["q"]), "k": rotate(x["k"])}


def _exact_attn(c, x):
    """Softmax attention of every document and head, the gradients by differentiation."""
    lens, group = _lens(c), c["heads"] // c["kv"]
    if sum(n * n for n in lens) * c["heads"] * c["d"] > 3e12:
        return None
    out = {"o": torch.zeros_like(x["q"], dtype=F64),
           "lse": torch.zeros((c["heads"], x["q"].shape[0]), dtype=F64, device="cuda")}
    if c["train"]:
        out.update(dq=torch.zeros_like(out["o"]), dk=torch.zeros_like(x["k"], dtype=F64),
                   dv=torch.zeros_like(x["v"], dtype=F64))
    ends = np.cumsum(lens)
    for end, n in zip(ends, lens):
        if n == 0:
            continue
        at = slice(int(end) - n, int(end))
        mask = torch.full((n, n), float("-inf"), dtype=F64, device="cuda").triu_(1)
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


def _exact_loss(c, x):
    """Negative log-probability of the target, weighted and differentiated."""
    v, valid = x["w_lm"].shape[0], x["targets"] >= 0
    hidden, w = (x[t].double().requires_grad_(c["train"]) for t in ("hidden", "w_lm"))
    logits = torch.mm(hidden, w.t())
    mine = valid & (x["targets"] < v)
    z = torch.gather(logits, 1, torch.where(mine, x["targets"], torch.zeros_like(x["targets"]))[:, None])[:, 0]
    lse = torch.logsumexp(logits, 1)
    if x["peer_lse"] is not None:
        lse = torch.logaddexp(lse, x["peer_lse"].double())
        z = torch.where(mine, z, x["peer_z"].double())
    loss = torch.where(valid, lse - z, torch.zeros_like(lse))
    out = {"loss": loss.detach(), "lse": lse.detach()}
    if c["train"]:
        out["d_hidden"], out["d_w"] = torch.autograd.grad((loss * x["d_loss"].double()).sum(), (hidden, w))
    return out


_EXACT = {"rope": _exact_rope, "attn": _exact_attn, "loss": _exact_loss}
