"""Plain 64-bit forms of the packed-document operators, written from their
formulas, and element-wise bounds on what the kernels may be off.

Every bound counts roundings.  One rounding to bf16 is off by at most U = 2^-8
of the value (half a step); one fp32 operation by F = 2^-24.  Sums of fp32
products of length n are off by at most (n + 2) F times the sum of the absolute
products.
"""
import math

import torch

U, F = 2.0 ** -8, 2.0 ** -24
F64 = torch.float64


def starts_of(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


# ------------------------------------------------------------------ rotary positions

def rope_frequencies(rot, base, scaling="none", factor=1.0, low=1.0, high=4.0, original=8192, **_):
    f = [base ** (-2.0 * j / rot) for j in range(rot // 2)]
    if scaling == "linear":
        return [x / factor for x in f]
    out = []
    for j, x in enumerate(f):
        g = 1.0
        if scaling == "bands":
            g = min(max((original * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
        elif scaling == "ramp":
            at = [rot * math.log(original / (2 * math.pi * t)) / (2 * math.log(base)) for t in (high, low)]
            j0, j1 = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
            g = 1.0 - min(max((j - j0) / (j1 - j0 if j1 > j0 else 0.001), 0.0), 1.0)
        out.append(x * ((1 - g) / factor + g))
    return out


def rope_plain(x, positions, rot, layout, freq, amplitude=1.0, inverse=False):
    """x [n][heads][d] float64, positions [n] -> (y, bound on |error| of an fp32 result)."""
    a = positions.to(F64)[:, None] * torch.tensor(freq, dtype=F64)
    c, s = amplitude * torch.cos(a)[:, None, :], amplitude * torch.sin(a)[:, None, :]
    if inverse:
        s = -s
    half = rot // 2
    i0, i1 = (slice(0, half), slice(half, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y, bound = x.clone(), torch.zeros_like(x)
    x0, x1 = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = x0 * c - x1 * s, x1 * c + x0 * s
    # the angle as a fraction of a turn in fp32 (pi F), sine and cosine (2 F), the
    # amplitude, the products and their sum (3 F): below 8 F of |x0| + |x1|
    bound[..., i0] = bound[..., i1] = 8 * F * amplitude * (x0.abs() + x1.abs())
    return y, bound


# ------------------------------------------------------------------ packed attention

def attention_plain(q, k, v, starts, scale=None, d_o=None):
    """q [n][a][d], k, v [n][g][d] float64 -> dict of results and, under "_" + name,
    element-wise error bounds.  Rows outside every document are zero."""
    n, a, d = q.shape
    group = a // k.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = {t: torch.zeros_like(q) for t in ("o", "_o")}
    out["lse"], out["_lse"] = torch.zeros(a, n, dtype=F64), torch.zeros(a, n, dtype=F64)
    if d_o is not None:
        out.update({t: torch.zeros_like(q) for t in ("dq", "_dq")})
        out.update({t: torch.zeros_like(k) for t in ("dk", "_dk", "dv", "_dv")})
    for lo, hi in zip(starts[:-1], starts[1:]):
        if hi <= lo:
            continue
        at = slice(lo, hi)
        later = torch.ones(hi - lo, hi - lo, dtype=torch.bool).triu(1)
        for h in range(a):
            Q, K, V = q[at, h], k[at, h // group], v[at, h // group]
            s = (Q @ K.T * scale).masked_fill(later, -math.inf)
            lse = torch.logsumexp(s, -1)
            P = torch.exp(s - lse[:, None])
            # a score: its products, the scale, its exponent (base 2) next to the maximum's
            e_s = ((d + 8) * F * scale * (Q.abs() @ K.abs().T)).masked_fill(later, 0.0)
            e_s = e_s + 4 * F * s.masked_fill(later, 0.0).abs()
            e_p = e_s.amax(-1, keepdim=True) + e_s + (hi - lo + 8) * F      # relative error of P in fp32
            out["o"][at, h], out["lse"][h, at] = P @ V, lse
            out["_lse"][h, at] = e_s.amax(-1) + (hi - lo + 8) * F + 4 * F * lse.abs()
            e_o = (P * (U + e_p)) @ V.abs() * (1 + U) + (hi - lo + 8) * F * (P @ V.abs())   # before its own rounding
            out["_o"][at, h] = U * (P @ V).abs() + (1 + U) * e_o
            if d_o is None:
                continue
            G = d_o[at, h]
            dP = G @ V.T
            delta = (G * (P @ V)).sum(-1, keepdim=True)
            dS = P * (dP - delta)
            # delta from the rounded output; dP from fp32 products; P from the rounded lse
            e_delta = (G.abs() * out["_o"][at, h]).sum(-1, keepdim=True) + (d + 2) * F * (G * (P @ V)).abs().sum(-1, keepdim=True)
            e_dp = (d + 2) * F * (G.abs() @ V.abs().T)
            e_pb = 2 * e_p + out["_lse"][h, at][:, None]
            e_ds = U * dS.abs() + (1 + U) * (P * (e_dp + e_delta) + e_pb * dS.abs() + 4 * F * P * (dP.abs() + delta.abs()))
            e_ds = e_ds.masked_fill(later, 0.0)
            add = (hi - lo + 8) * F
            g = h // group
            out["dq"][at, h] = scale * dS @ K
            out["_dq"][at, h] = scale * (e_ds @ K.abs() + add * (dS.abs() @ K.abs()))
            out["dk"][at, g] += scale * dS.T @ Q
            out["_dk"][at, g] += scale * (e_ds.T @ Q.abs() + (add + group * F) * (dS.abs().T @ Q.abs()))
            out["dv"][at, g] += P.T @ G
            out["_dv"][at, g] += (P * (U + e_pb)).T @ G.abs() * (1 + U) + (add + group * F) * (P.T @ G.abs())
    for t in ("dq", "dk", "dv"):
        if d_o is not None:
            out["_" + t] = (1 + U) * out["_" + t] + U * out[t].abs()
    return out


# ------------------------------------------------------------------ loss without stored logits

def loss_plain(hidden, w, targets, v0=0, peer_lse=None, peer_z=None, d_loss=None):
    """hidden [n][h], w [v][h] float64 -> dict of results and, under "_" + name, error bounds."""
    n, h = hidden.shape
    v = w.shape[0]
    z = hidden @ w.T
    e_z = (h + 2) * F * (hidden.abs() @ w.abs().T)
    lse = torch.logsumexp(z, -1)
    here = (targets >= v0) & (targets < v0 + v)
    row = torch.arange(n)
    col = (targets - v0).clamp(0, v - 1)
    zt = torch.where(here, z[row, col], torch.full((n,), -math.inf, dtype=F64))
    out = dict(shard_lse=lse, target_logit=zt)
    # exponentials (a few F of the exponent's size each) and their fp32 sum, then the logarithm
    e_lse = e_z.amax(-1) + (v + 16) * F + 8 * F * (z - z.amax(-1, keepdim=True)).abs().amax(-1) + 4 * F * lse.abs()
    if peer_lse is not None:
        lse = torch.logaddexp(lse, peer_lse)
        e_lse = e_lse + 8 * F * (1 + lse.abs())
        zt = torch.where(here, zt, peer_z)
    valid = targets >= 0
    out.update(lse=lse, loss=torch.where(valid, lse - zt, torch.zeros(n, dtype=F64)), _lse=e_lse)
    out["_loss"] = torch.where(valid, e_lse + e_z.amax(-1) + 2 * F * (lse.abs() + torch.where(valid, zt, lse).abs()), torch.zeros(n, dtype=F64))
    if d_loss is not None:
        p = torch.exp(z - lse[:, None])
        hot = torch.zeros_like(p)
        hot[row, col] = here.to(F64)
        wt = torch.where(valid, d_loss, torch.zeros(n, dtype=F64))[:, None]
        G = wt * (p - hot)
        # p in fp32: logits, the given lse, the exponential of an argument of this size
        e_g = wt.abs() * (p * (e_z + e_lse[:, None] + 8 * F + 4 * F * (z - lse[:, None]).abs()) + 4 * F * (p + hot))
        out["d_hidden"] = G @ w
        e = (U * G.abs() + (1 + U) * e_g) @ w.abs() + (v + 8) * F * (G.abs() @ w.abs())
        out["_d_hidden"] = (1 + U) * e + U * out["d_hidden"].abs()
        out["d_w"] = G.T @ hidden
        # two bf16 parts: what is left is U of the second one, itself at most U of the value
        out["_d_w"] = (U * U * G.abs() + 2 * e_g).T @ hidden.abs() + (2 * n + 8) * F * (G.abs().T @ hidden.abs())
    return out


def inside(name, got, want, bound):
    """Every element of got within its bound of want (and finite where want is)."""
    got, bound = got.detach().cpu().double(), bound + 1e-30
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), f"{name}: not finite in other places"
    assert torch.equal(got[~finite], want[~finite]), name
    off = (got - want).abs()[finite] / bound[finite] if bound.dim() else (got - want).abs()[finite] / bound
    worst = float(off.max()) if off.numel() else 0.0
    print(f"{name:>10s}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, f"{name}: {worst} times the bound"


def close(name, got, want, rel):
    """Relative Frobenius error."""
    got = got.detach().cpu().double()
    norm = float(want.norm())
    off = float((got - want).norm()) / norm if norm else float(got.norm())
    print(f"{name:>10s}: relative Frobenius error {off:.2e}", flush=True)
    assert off <= rel, f"{name}: {off}"
