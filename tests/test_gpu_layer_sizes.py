"""The operators around the scan at sizes whose kernels take other forms and longer walks than small ones: two or four channels a lane and
long stretches in the state space scan, many items a warp in the norm of heads, long runs in the convolution.  Against 64 bits on the GPU.

Tolerances: those of the operators' own tests, element by element, and beside them a bound on the norm of what is off, which errors that
cancel stay far below and a lost bit does not.  Every token of the scan multiplies a state by a decay that is 5e-8 off at random and
under 4e-9 on average, and rounds once; a state that remembers n tokens holds sqrt(n / 2) of the former and n of the latter: 1.5e-6 for
n of 300.  A gradient goes through two of them, its step sizes 2.8e-7 more: 5e-6.  (A state kept in 11 bits is 1e-4 off and more.)
"""
import random
from unittest import mock

import pytest
import torch

import layer_reference as ref
import paper_2608_15533_b200 as dl
import test_gpu_ssm as small

DEV = "cuda"
DT = {torch.float32: dl.F32, torch.bfloat16: dl.BF16}
NORMWISE = 5e-6


def _off(got, want):
    got, want = got.detach().double(), want.double().to(got.device)
    return float((got - want).norm() / want.norm())


def _close(got, want, mag, relative, name):
    """layer_reference.close without leaving the GPU."""
    with mock.patch.object(torch.Tensor, "cpu", lambda t: t):
        ref.close(got, want, mag, relative, name)


def _ssm64(*args, **kw):
    with mock.patch.object(ref, "f64", lambda t: None if t is None else t.detach().double()), torch.device(DEV):
        return ref.ssm(*args, **kw)


def _lens(total, seed, longest=300):
    r, lens = random.Random(seed), [0, 1]
    while sum(lens) < total:
        lens.append(min(r.choice((r.randint(1, 9), r.randint(1, longest), 0)), total - sum(lens)))
    return lens + [0]


# Channels, groups, tokens; channels of a CTA in the wide form, tokens of a stretch: 148 CTAs and more, so that the wide form is taken.
WIDE = [(8, 1304, 1, 2050, 128, 128, dict()), (16, 776, 1, 1950, 64, 128, dict(wide=True)), (32, 336, 2, 1950, 32, 128, dict(gate=False)),
        (64, 304, 1, 1950, 32, 128, dict(skip=False)), (16, 4488, 1, 2000, 64, 256, dict(wide=True)), (8, 2640, 2, 1300, 128, 128, dict(softplus=False, bias=False)),
        (8, 16384, 1, 900, 64, 128, dict(gate=False))]  # with fp32 the narrow form in several stretches: the wide one has 128 CTAs


@pytest.mark.gpu
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,D,G,T,cols,span,kw", WIDE)
def test_state_space_scan_with_many_ctas(io, N, D, G, T, cols, span, kw):
    assert -(-(D // G) // cols) * G * -(-T // span) >= 148
    lens = _lens(T, N) if span == 128 else [700] + _lens(T - 700, N)
    n = len(lens)
    c = small._case(T, D, N, G, io, **kw)
    g = torch.Generator().manual_seed(N)
    S0, dS = (torch.randn(n, D, N, generator=g).to(DEV) for _ in range(2))
    dout = torch.randn(T, D, generator=g).to(io).to(DEV)
    desc, plan = dl.SsmDesc(D, N, G, DT[io], c["softplus"]), small._plan(lens)
    work = dl.ssm_workspace(desc, n, T, train=True, device=DEV)
    work.fill_(0xff)                                    # NaN in whatever is read before it is written
    out, S = dl.ssm_forward(desc, plan, *small._args(c), S_init=S0, workspace=work, save=True)
    d = dl.ssm_backward(desc, plan, *small._args(c), dout, S_init=S0, dS_final=dS, workspace=work, saved=True)
    want, mag = (_ssm64(c, lens, S0, dout, dS, mag=m) for m in (False, True))
    rel = small._rel(c, lens)
    _close(out, want[0], mag[0], rel, "out")
    _close(S, want[1], mag[1], rel, "S")
    assert _off(S, want[1]) < NORMWISE and (io is torch.bfloat16 or _off(out, want[0]) < NORMWISE)
    many = rel + T * 2.0 ** -24
    for k, e in (("x", rel), ("dt", rel), ("A", many), ("B", rel), ("C", rel), ("D", many), ("z", rel), ("dt_bias", many), ("S_init", rel)):
        got = getattr(d, k)
        assert (got is None) == (want[2][k] is None)
        if got is not None:
            _close(got, want[2][k], mag[2][k] + want[2][k].abs(), 2 * e, "d" + k)
            if got.dtype is torch.float32:
                assert _off(got, want[2][k]) < NORMWISE, k
    again = dl.ssm_backward(desc, plan, *small._args(c), dout, S_init=S0, dS_final=dS)
    for k in ("x", "dt", "A", "B", "C", "S_init"):
        assert torch.equal(getattr(d, k), getattr(again, k)), k


@pytest.mark.gpu
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,D,G,T,cols,span,kw", WIDE[:5])
def test_state_space_prompts_with_many_ctas(io, N, D, G, T, cols, span, kw):
    lens = _lens(T, N + 1) if span == 128 else [700] + _lens(T - 700, N)
    n = len(lens)
    c = small._case(T, D, N, G, io, **kw)
    r = random.Random(N)
    slots = r.sample(range(n + 5), n)
    for i in r.sample(range(n), n // 6):
        slots[i] = r.choice((-1, n + 5))              # padding, and slots that do not exist
    rows = ref.rows_of(lens)
    skipped = [i for i in range(n) if not 0 <= slots[i] < n + 5]
    for i in skipped:                                  # whose tokens may hold anything
        for k in ("x", "dt", "B", "C", "z"):
            if c[k] is not None:
                c[k][rows[i]] = float("nan")
    fresh = torch.tensor([r.randrange(2) for _ in range(n)], dtype=torch.int32, device=DEV)
    desc = dl.SsmDesc(D, N, G, DT[io], c["softplus"], num_slots=n + 5)
    pool = torch.randn(n + 5, D, N, device=DEV)
    state, mark = dl.SsmState(desc, pool.clone()), torch.full((T, D), 3.0, dtype=io, device=DEV)
    work = dl.ssm_workspace(desc, n, T, device=DEV)
    work.fill_(0xff)
    dl.ssm_prefill(desc, state, small._plan(lens, slots), *small._args(c), fresh=fresh, out=mark, workspace=work)
    live = [i for i in range(n) if i not in skipped]
    cut = {k: v if k in ("A", "D", "dt_bias", "softplus") or v is None else torch.cat([v[rows[i]] for i in live]) for k, v in c.items()}
    start = torch.stack([pool[slots[i]] * (1 - int(fresh[i])) for i in live])
    want, mag = (_ssm64(cut, [lens[i] for i in live], start, mag=m) for m in (False, True))
    rel = small._rel(cut, [lens[i] for i in live])
    _close(torch.cat([mark[rows[i]] for i in live]), want[0], mag[0], rel, "out")
    expect = pool.clone()
    for j, i in enumerate(live):
        if lens[i]:
            _close(state.S[slots[i]], want[1][j], mag[1][j], rel, f"row {i}")
            expect[slots[i]] = state.S[slots[i]]
    assert torch.equal(state.S, expect)                # slots that no row names, and those of rows without tokens
    for i in skipped:
        assert (mark[rows[i]] == 3.0).all()


def test_a_state_of_eleven_bits_would_be_seen():
    g = torch.Generator().manual_seed(0)
    T, D, N = 300, 8, 16
    A, x, B = -torch.rand(D, N, generator=g) * 4 - 0.02, torch.randn(T, D, generator=g), torch.randn(T, N, generator=g)
    delta = torch.nn.functional.softplus(torch.randn(T, D, generator=g) - 2)
    A, x, B, delta = (t.double() for t in (A, x, B, delta))
    exact = torch.zeros(D, N, dtype=torch.float64)
    short = exact.clone()
    for t in range(T):
        a, b = torch.exp(delta[t][:, None] * A), (delta[t] * x[t])[:, None] * B[t]
        exact, short = a * exact + b, (a * short + b).half().double()
    assert _off(short, exact) > 10 * NORMWISE


@pytest.mark.gpu
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,Hq,Hk,d,norm,rot,interleaved", [(9001, 8, 2, 128, "rms", 128, False), (12000, 12, 4, 64, "rms", 32, True),
                                                            (5003, 9, 5, 256, "l2", 96, False), (20011, 5, 3, 40, "rms", 0, False)])
def test_norm_of_many_heads_a_warp(io, T, Hq, Hk, d, norm, rot, interleaved):
    g = torch.Generator().manual_seed(d)
    proj = torch.randn(T, Hq + 2 * Hk, d, generator=g).to(io).to(DEV)
    q, k = proj[:, :Hq], proj[:, Hq : Hq + Hk]
    wq, wk = ((1 + 0.3 * torch.randn(d, generator=g)).to(DEV) if norm == "rms" else None for _ in range(2))
    cos = sin = pos = None
    live = torch.ones(T, dtype=torch.bool, device=DEV)
    if rot:
        angle = torch.arange(500, dtype=torch.float64)[:, None] * torch.pow(10000.0, -torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))
        cos, sin = angle.cos().float().to(DEV), angle.sin().float().to(DEV)
        pos = torch.randint(0, 500, (T,), generator=g).to(torch.int32).to(DEV)
        live[torch.randint(0, T, (T // 20,), generator=g).to(DEV)] = False
        pos[~live] = -1
        proj[~live] = float("nan")                     # a padding token may hold anything
    desc = dl.NormDesc(Hq, Hk, d, DT[io], {"rms": dl.NORM_RMS, "l2": dl.NORM_L2}[norm], 1e-5, rot, interleaved, q_scale=0.37)
    doq, dok = (torch.randn(T, h, d, generator=g).to(io).to(DEV) for h in (Hq, Hk))
    got = dl.head_norm_forward(desc, q, k, wq, wk, cos, sin, pos)
    grads = dl.head_norm_backward(desc, q, k, wq, wk, cos, sin, pos, doq, dok)
    with torch.device(DEV):
        c, s = (t.double()[pos[live].long()] if rot else None for t in (cos, sin))
        for x, w, scale, out, do, dx, dw, name in ((q, wq, 0.37, got[0], doq, grads.q, grads.w_q, "q"), (k, wk, 1.0, got[1], dok, grads.k, grads.w_k, "k")):
            X, Wt, G0 = x[live].double().requires_grad_(), None if w is None else w.double().requires_grad_(), do[live].double()
            want = ref.head_norm(X, Wt, norm, 1e-5, scale, rot, interleaved, c, s)
            n = ref.head_norm(X, Wt, norm, 1e-5, scale, 0, False, None, None).detach().abs()
            _close(out[live], want.detach(), n.amax(-1, keepdim=True).expand_as(n), 2.0 ** -19, name)
            assert not out[~live].any() and not dx[~live].any()
            (want * G0).sum().backward()
            G, wmax, cc, V = G0.abs().amax(-1, keepdim=True) * 1.5 * scale, 1.0 if w is None else w.abs().max(), 1 / d if norm == "rms" else 1.0, X.detach()
            r = 1 / torch.sqrt(cc * (V ** 2).sum(-1, keepdim=True) + 1e-5)
            gm = r * (G * wmax + V.abs() * cc * r * r * (G * wmax * V.abs()).sum(-1, keepdim=True))
            _close(dx[live], X.grad, gm, 2.0 ** -18, "d" + name)
            if w is not None:
                # a thread's sums over its few items and a fixed tree over the rest: their roundings are a few of 2^-24, the values' own 2^-18
                assert _off(dw, Wt.grad) < NORMWISE, "dw of " + name


def _conv64(x, w, b, init, lens, act, dout, dfinal, mag=False):
    """out, final, dx, dw, db, dinit of all rows at once, in 64 bits; mag: their magnitudes."""
    x, w, init, dout, dfinal = (t.double().abs() if mag else t.double() for t in (x, w, init, dout, dfinal))
    T, C = x.shape
    W, n = w.shape[1], len(lens)
    ln = torch.tensor(lens, device=DEV)
    first = torch.cumsum(ln, 0) - ln
    row = torch.repeat_interleave(torch.arange(n, device=DEV), ln)
    at = torch.arange(T, device=DEV) - first[row]
    taps = []
    for back in range(W):                              # the input `back` tokens in front, of the row or of its window
        tap = torch.cat((torch.zeros_like(x[:back]), x[: T - back])) if back else x.clone()
        early = torch.nonzero(at < back)[:, 0]
        tap[early] = init[row[early], W - 1 + at[early] - back]
        taps.append(tap)
    pre = (0 if b is None else (b.double().abs() if mag else b.double())) + sum(w[:, W - 1 - back] * taps[back] for back in range(W))
    out = ref.silu(pre) if act and not mag else pre
    dpre = dout * (1.1 + 0.5 * pre) if mag else dout * ref.silu_slope(pre) if act else dout
    dx, dinit, dw, final = torch.zeros_like(x), torch.zeros_like(init), torch.zeros_like(w), torch.zeros_like(init)
    for back in range(W):
        part, late = w[:, W - 1 - back] * dpre, at >= back
        dx[: T - back] += (part * late[:, None])[back:]
        early = torch.nonzero(~late)[:, 0]
        dinit.index_put_((row[early], W - 1 + at[early] - back), part[early], accumulate=True)
        dw[:, W - 1 - back] = (dpre * taps[back]).sum(0)
    for j in range(W - 1):
        p = ln - (W - 1) + j                           # the window behind a row: its token p, or what was in the window in front
        own, old = torch.nonzero(p >= 0)[:, 0], torch.nonzero(p < 0)[:, 0]
        final[own, j], final[old, j] = x[first[own] + p[own]], init[old, W - 1 + p[old]]
        dx[first[own] + p[own]] += dfinal[own, j]
        dinit[old, W - 1 + p[old]] += dfinal[old, j]
    return out, final, dx, dw, dpre.sum(0), dinit


@pytest.mark.gpu
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("T,act", [(17_000, True), (67_003, True), (67_003, False)])
def test_convolution_in_long_runs(io, W, T, act):
    C = 2120                                           # 17 blocks of channels, the last one with 72: runs of 32 and of 128 tokens
    r = random.Random(T + W)
    lens = _lens(T // 3, W, longest=40) + [T // 2]
    lens += _lens(T - sum(lens), W + 1, longest=500)
    n = len(lens)
    assert sum(lens) == T and 17 * T // (60 * 148) >= (128 if T > 60_000 else 32)
    g = torch.Generator(DEV).manual_seed(T + W)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)
    x, w, b = rnd(T, C + 16).to(io)[:, 8 : 8 + C], rnd(C, W) * W ** -0.5, rnd(C) * 0.3 if act else None
    init, dfinal, dout = rnd(n, W - 1, C).to(io), rnd(n, W - 1, C).to(io), rnd(T, C).to(io)
    desc, plan = dl.ConvDesc(C, W, DT[io], act, num_slots=n + 5), small._plan(lens)
    out, final = dl.conv_forward(desc, plan, x, w, b, init=init)
    d = dl.conv_backward(desc, plan, x, w, b, dout, init=init, dfinal=dfinal)
    want, mag = (_conv64(x, w, b, init, lens, act, dout, dfinal, mag=m) for m in (False, True))
    rel = 2.0 ** -19
    _close(out, want[0], mag[0], rel, "out")
    assert torch.equal(final.double(), want[1])
    _close(d.x, want[2], mag[2], rel, "dx")
    _close(d.init, want[5], mag[5], rel, "dinit")
    # sums of T terms that mostly cancel: what is off is some 1e-6 of the terms' own errors
    assert _off(d.weight, want[3]) < NORMWISE and (b is None or _off(d.bias, want[4]) < NORMWISE)
    # a pool: the same bits for the rows that it has, nothing of the others
    slots = r.sample(range(n + 5), n)
    for i in r.sample(range(n), n // 6):
        slots[i] = r.choice((-1, n + 5))
    ok = [i for i in range(n) if 0 <= slots[i] < n + 5]
    state = dl.ConvState(desc, torch.zeros(n + 5, W - 1, C, dtype=io, device=DEV))
    at = torch.tensor([slots[i] for i in ok], device=DEV)
    state.window[at] = init[torch.tensor(ok, device=DEV)]
    before = state.window.clone()
    got = dl.conv_prefill(desc, state, small._plan(lens, slots), x, w, b)
    alive = torch.repeat_interleave(torch.tensor([i in set(ok) for i in range(n)], device=DEV), torch.tensor(lens, device=DEV))
    assert torch.equal(got[alive], out[alive]) and not got[~alive].any()
    some = [i for i in ok if lens[i]]
    before[torch.tensor([slots[i] for i in some], device=DEV)] = final[torch.tensor(some, device=DEV)]
    assert torch.equal(state.window, before) and int(state.status) == dl.STATUS_BAD_SLOT
