"""Plain 64-bit forms of the operators around the scan: causal convolution, selective state space scan, norm and rotation of
heads, each with its gradients by formula.

Beside every value stands its magnitude: the same sums with every term's absolute value.  An error of e relative to each term is at
most e times the magnitude of the result, which is what the tests' tolerances are made of.
"""
import torch

F64 = torch.float64
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def f64(t):
    return None if t is None else t.detach().to("cpu", F64)


def silu(v):
    return v * torch.sigmoid(v)


def silu_slope(v):
    s = torch.sigmoid(v)
    return s * (1 + v * (1 - s))


def rows_of(lens):
    at, out = 0, []
    for n in lens:
        out.append(slice(at, at + n))
        at += n
    return out


def close(got, want, mag, relative, name=""):
    """|got - want| <= half a step of the type at `want` + relative * magnitude, everywhere; NaN where NaN is wanted."""
    got = got.detach().cpu()
    g, tol = got.to(F64), HALF_STEP[got.dtype] * want.abs() + relative * mag + 1e-30
    # (a value that rounds to the neighbour of the wanted one's rounding is half a step of its own off)
    tol = tol * (1 + 2.0 ** -7) if got.dtype is torch.bfloat16 else tol
    bad = ~((g - want).abs() <= tol) & ~(torch.isnan(g) & torch.isnan(want)) & ~(g == want)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float(((g - want).abs() / tol)[bad].max())} tolerances"


# ---- convolution --------------------------------------------------------------------------------------------------------
def conv_row(x, w, b, init, act, mag=False):
    """One row: x [len, C], w [C, W], init [W - 1, C]: pre-activation, out, last inputs.  mag: their magnitudes."""
    if mag:
        x, w, b, init = x.abs(), w.abs(), None if b is None else b.abs(), init.abs()
    W, seen = w.shape[1], torch.cat((init, x))
    pre = torch.stack([seen[j : j + len(x)] * w[:, j] for j in range(W)]).sum(0) if len(x) else x.clone()
    if b is not None:
        pre = pre + b
    return pre, (silu(pre) if act and not mag else pre), seen[len(x) :]


def conv_row_grad(x, w, b, init, act, dout, dfinal, mag=False):
    """Gradients of a row's x, w, b, init."""
    W = w.shape[1]
    pre = conv_row(x, w, b, init, act)[0]
    seen = torch.cat((init, x))
    dpre = dout * silu_slope(pre) if act else dout.clone()
    if mag:
        # silu' is at most 1.1, and 0.5 of an error of the pre-activation more
        dpre = dout.abs() * (1.1 + 0.5 * conv_row(x, w, b, init, act, mag=True)[0])
        seen, w, dfinal = seen.abs(), w.abs(), dfinal.abs()
    dseen = torch.zeros_like(seen)
    dw = torch.zeros_like(w)
    for j in range(W):
        dseen[j : j + len(x)] += dpre * w[:, j]
        dw[:, j] = (dpre * seen[j : j + len(x)]).sum(0)
    dseen[len(x) :] += dfinal
    return dseen[W - 1 :], dw, dpre.sum(0), dseen[: W - 1]


# ---- state space scan -----------------------------------------------------------------------------------------------------
def ssm_row(t, S, mag=False):
    """One row; t: dict of its x, delta, A, B, C [len, D, N], D, z (fp64).  out, last state, and what the gradients need."""
    a = (lambda v: None if v is None else v.abs()) if mag else (lambda v: v)
    x, B, C, A = a(t["x"]), a(t["B"]), a(t["C"]), t["A"]
    S = a(S).clone()
    prev, ys = [], []
    for i in range(len(x)):
        prev.append(S.clone())
        S = torch.exp(t["delta"][i][:, None] * A) * S + (t["delta"][i].abs() * x[i] if mag else t["delta"][i] * x[i])[:, None] * B[i]
        ys.append((S * C[i]).sum(-1))
    y = torch.stack(ys) if ys else torch.zeros_like(x)
    if t["D"] is not None:
        y = y + x * a(t["D"])
    return (y if t["z"] is None else y * a(silu(t["z"]))), S, prev, y


def ssm_row_grad(t, S, dout, dS, mag=False):
    """Gradients of a row: dx, ddelta, dA, dB, dC [len, D, N], dD, dz, dS0; with mag their magnitudes."""
    a = (lambda v: None if v is None else v.abs()) if mag else (lambda v: v)
    out, last, prev, y = ssm_row(t, S, mag)
    x, B, C, delta = a(t["x"]), a(t["B"]), a(t["C"]), a(t["delta"])
    dout, adj = a(dout), a(dS).clone()
    dz = None if t["z"] is None else dout * y * a(silu_slope(t["z"])) if not mag else dout * y * 1.1
    dy = dout if t["z"] is None else dout * a(silu(t["z"]))
    dx, dd, dB, dC = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(B), torch.zeros_like(C)
    dA = torch.zeros_like(t["A"])
    for i in range(len(x) - 1, -1, -1):
        e = torch.exp(t["delta"][i][:, None] * t["A"])
        u = (delta[i] * x[i])[:, None]
        h = e * prev[i] + u * B[i]
        adj = adj + dy[i][:, None] * C[i]
        dC[i], dB[i] = dy[i][:, None] * h, adj * u
        sB, moved = (adj * B[i]).sum(-1), adj * e * prev[i]
        dx[i] = delta[i] * sB
        dd[i] = x[i] * sB + (moved * a(t["A"])).sum(-1)
        dA += moved * delta[i][:, None]
        adj = e * adj
    dD = None
    if t["D"] is not None:
        dx, dD = dx + dy * a(t["D"]), (dy * x).sum(0)
    return dict(x=dx, delta=dd, A=dA, B=dB, C=dC, D=dD, z=dz, S_init=adj)


def ssm(case, lens, S0, dout=None, dS=None, mag=False):
    """All rows; case: dict of x, dt, A, B, C [T, G, N], D, z, dt_bias, softplus.  Forward: out, S.  With dout: gradients too."""
    A, G = f64(case["A"]), case["B"].shape[1]
    x = f64(case["x"])
    raw = f64(case["dt"]) + (0 if case["dt_bias"] is None else f64(case["dt_bias"]))
    delta = torch.nn.functional.softplus(raw, threshold=1e9) if case["softplus"] else raw
    rep = x.shape[1] // G
    B, C = (f64(case[k]).repeat_interleave(rep, 1) for k in ("B", "C"))
    z = f64(case["z"])
    out, S = torch.zeros_like(x), f64(S0).clone()
    g = dict(x=torch.zeros_like(x), dt=torch.zeros_like(x), A=torch.zeros_like(A), B=torch.zeros_like(f64(case["B"])), C=torch.zeros_like(f64(case["C"])),
             D=None if case["D"] is None else torch.zeros(x.shape[1], dtype=F64), z=None if z is None else torch.zeros_like(x), S_init=torch.zeros_like(S))
    for i, r in enumerate(rows_of(lens)):
        t = dict(x=x[r], delta=delta[r], A=A, B=B[r], C=C[r], D=f64(case["D"]), z=None if z is None else z[r])
        if dout is not None:
            d = ssm_row_grad(t, S[i], f64(dout)[r], f64(dS)[i], mag)
            g["x"][r], g["A"], g["S_init"][i] = d["x"], g["A"] + d["A"], d["S_init"]
            g["dt"][r] = d["delta"] * (torch.sigmoid(raw[r]) if case["softplus"] else 1)
            for k in ("B", "C"):
                g[k][r] = d[k].unflatten(1, (G, rep)).sum(2)
            if g["D"] is not None:
                g["D"] += d["D"]
            if z is not None:
                g["z"][r] = d["z"]
        out[r], S[i] = ssm_row(t, S[i], mag)[:2]
    g["dt_bias"] = None if case["dt_bias"] is None else g["dt"].sum(0)
    return out, S, g


# ---- norm and rotation of heads ---------------------------------------------------------------------------------------------
def head_norm(x, w, norm, eps, scale, rot, interleaved, cos, sin):
    """x [T, H, d] fp64; cos, sin [T, rot / 2] of the tokens' positions.  Differentiable."""
    d = x.shape[-1]
    if norm != "none":
        ss = (x * x).sum(-1, keepdim=True)
        x = x / torch.sqrt((ss / d if norm == "rms" else ss) + eps)
        if w is not None:
            x = x * w
    if rot:
        h = rot // 2
        i, j = (torch.arange(0, rot, 2), torch.arange(1, rot, 2)) if interleaved else (torch.arange(h), torch.arange(h, rot))
        u, v, c, s = x[..., i], x[..., j], cos[:, None], sin[:, None]
        turned = torch.zeros_like(x[..., :rot])
        turned = turned.index_copy(-1, i, u * c - v * s).index_copy(-1, j, v * c + u * s)
        x = torch.cat((turned, x[..., rot:]), -1)
    return x * scale
