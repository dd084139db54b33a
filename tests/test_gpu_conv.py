"""The short causal convolution on the GPU against its 64-bit form.

Tolerances: half a step of the output's type, and W + 1 products and sums of fp32 with a sigmoid of 2^-21 behind them: 2^-19 of the
magnitude (the same sums of absolute values).  A gradient of the weights sums T of them: 2^-19 + T 2^-24.
"""
import pytest
import torch

import layer_reference as ref
import paper_2608_15533_b200 as dl

pytestmark = pytest.mark.gpu
DEV = "cuda"
REL = 2.0 ** -19
DT = {torch.float32: dl.F32, torch.bfloat16: dl.BF16}


def _inputs(lens, C, W, io, bias=True, wide=False, seed=0, spare=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    T = sum(lens) + spare
    x = rnd(T, C + (16 if wide else 0)).to(io).to(DEV)
    if wide:
        x = x[:, 8 : 8 + C]
    return x, (rnd(C, W) * W ** -0.5).to(DEV), (rnd(C) * 0.3).to(DEV) if bias else None


def _plan(lens, slots=None, token_map=True, room=0, rows=None):
    plan = dl.Plan(len(lens), sum(lens) + room, device=DEV, token_map=token_map)
    s = None if slots is None else torch.tensor(slots, dtype=torch.int32, device=DEV)
    return dl.build_plan(torch.tensor(lens, dtype=torch.int32, device=DEV), plan, slots=s)


def _check_forward(out, final, x, w, b, init, lens, act):
    x, w, b = ref.f64(x), ref.f64(w), ref.f64(b)
    for i, r in enumerate(ref.rows_of(lens)):
        _, want, last = ref.conv_row(x[r], w, b, init[i], act)
        mag = ref.conv_row(x[r], w, b, init[i], act, mag=True)[0]
        ref.close(out[r], want, mag, REL, f"row {i}")
        assert torch.equal(ref.f64(final[i]), last), f"window of row {i}"


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C,W,lens,wide,act,bias,token_map", [
    (64, 4, (1,), False, True, True, True),
    (8, 2, (2, 1, 0, 3), False, False, False, True),
    (136, 3, (0, 0, 5, 1, 2, 0, 40), True, True, False, False),
    (1096, 4, (3, 2, 1, 130, 0, 65), True, True, True, True),
    (512, 4, (700,), False, True, True, False),
    (128, 4, tuple(range(12)), False, True, True, True),
])
def test_forward_and_gradients(io, C, W, lens, wide, act, bias, token_map):
    x, w, b = _inputs(lens, C, W, io, bias, wide)
    n, T = len(lens), sum(lens)
    g = torch.Generator().manual_seed(1)
    init, dfinal = (torch.randn(n, W - 1, C, generator=g).to(io).to(DEV) for _ in range(2))
    dout = torch.randn(T, C, generator=g).to(io).to(DEV)
    desc, plan = dl.ConvDesc(C, W, DT[io], act), _plan(lens, token_map=token_map)
    out, final = dl.conv_forward(desc, plan, x, w, b, init=init)
    _check_forward(out, final, x, w, b, ref.f64(init), lens, act)
    # without a start: zeros
    out0, final0 = dl.conv_forward(desc, plan, x, w, b)
    _check_forward(out0, final0, x, w, b, torch.zeros(n, W - 1, C, dtype=ref.F64), lens, act)
    for start, df in ((init, dfinal), (None, None)):
        d = dl.conv_backward(desc, plan, x, w, b, dout, init=start, dfinal=df)
        again = dl.conv_backward(desc, plan, x, w, b, dout, init=start, dfinal=df, workspace=dl.conv_workspace(desc, T, DEV))
        X, Wt, Bt, DO = ref.f64(x), ref.f64(w), ref.f64(b), ref.f64(dout)
        S = torch.zeros(n, W - 1, C, dtype=ref.F64) if start is None else ref.f64(start)
        DF = torch.zeros_like(S) if df is None else ref.f64(df)
        dw, dwm, db, dbm = torch.zeros_like(Wt), torch.zeros_like(Wt), torch.zeros(C, dtype=ref.F64), torch.zeros(C, dtype=ref.F64)
        for i, r in enumerate(ref.rows_of(lens)):
            want, mag = (ref.conv_row_grad(X[r], Wt, Bt, S[i], act, DO[r], DF[i], mag=m) for m in (False, True))
            ref.close(d.x[r], want[0], mag[0], REL, f"dx of row {i}")
            ref.close(d.init[i], want[3], mag[3], REL, f"dinit of row {i}")
            dw, dwm, db, dbm = dw + want[1], dwm + mag[1], db + want[2], dbm + mag[2]
        ref.close(d.weight, dw, dwm, REL + T * 2.0 ** -24, "dw")
        if bias:
            ref.close(d.bias, db, dbm, REL + T * 2.0 ** -24, "db")
        for k in ("x", "weight", "init") + (("bias",) if bias else ()):
            assert torch.equal(getattr(d, k), getattr(again, k)), f"{k} differs from run to run"


def test_gradients_against_differences():
    lens, C, W = (5, 2, 9), 16, 4
    x, w, b = _inputs(lens, C, W, torch.float32)
    desc, plan = dl.ConvDesc(C, W, dl.F32), _plan(lens)
    leaf = [t.clone().requires_grad_() for t in (x, w, b, torch.randn(3, W - 1, C, device=DEV))]
    out, final = dl.conv(desc, plan, *leaf[:3], init=leaf[3])
    do, df = torch.randn_like(out), torch.randn_like(final)
    grads = torch.autograd.grad((out, final), leaf, (do, df))

    def value(args):
        total = 0
        for i, r in enumerate(ref.rows_of(lens)):
            _, o, f = ref.conv_row(args[0][r], args[1], args[2], args[3][i], True)
            total = total + (o * ref.f64(do)[r]).sum() + (f * ref.f64(df)[i]).sum()
        return float(total)

    base = [ref.f64(t) for t in leaf]
    for i, g in enumerate(grads):
        v = torch.randn(base[i].shape, dtype=ref.F64)
        move = lambda h: [t + h * v if j == i else t for j, t in enumerate(base)]
        want = (value(move(1e-6)) - value(move(-1e-6))) / 2e-6
        # a sum of g v: each term is 2^-19 of its magnitude off at most, and silu' magnitudes are at most 1.1 + 0.5 |pre|
        tol = 2.0 ** -17 * float((ref.f64(g).abs() * v.abs()).sum()) + 2.0 ** -17 * v.abs().sum().item()
        assert abs(float((ref.f64(g) * v).sum()) - want) < tol


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
def test_prefill_of_a_pool(io):
    lens, C, W = (4, 0, 1, 2, 30, 3, 5, 2), 72, 4
    slots = [5, 2, 0, -1, 7, 9, 1, 3]  # row 3 is padding, slot 9 does not exist
    x, w, b = _inputs(lens, C, W, io, spare=6)
    desc = dl.ConvDesc(C, W, DT[io], num_slots=8)
    pool = torch.randn(8, W - 1, C).to(io).to(DEV)
    fresh = torch.tensor([0, 1, 1, 0, 0, 0, 1, 0], dtype=torch.int32, device=DEV)
    x[4 + 1 : 4 + 1 + 2] = float("nan")      # the padding row's tokens may hold anything
    x[sum(lens) :] = float("nan")
    for mine in (False, True):
        state = dl.ConvState(desc, pool.clone())
        plan = _plan(lens, slots, room=4)
        mark = torch.full_like(x, 3.0).contiguous()
        out = dl.conv_prefill(desc, state, plan, x, w, b, fresh=fresh, out=mark if mine else None)
        assert int(state.status) == dl.STATUS_BAD_SLOT
        want_pool = ref.f64(pool)
        X = ref.f64(x)
        for i, r in enumerate(ref.rows_of(lens)):
            if slots[i] in (-1, 9) or lens[i] == 0:
                assert (out[r] == (3.0 if mine else 0.0)).all()
                continue
            init = want_pool[slots[i]] * (0 if fresh[i] else 1)
            _, want, last = ref.conv_row(X[r], ref.f64(w), ref.f64(b), init, True)
            ref.close(out[r], want, ref.conv_row(X[r], ref.f64(w), ref.f64(b), init, True, mag=True)[0], REL, f"row {i}")
            want_pool[slots[i]] = last
        assert (out[sum(lens) :] == (3.0 if mine else 0.0)).all()   # behind the last sequence
        assert torch.equal(ref.f64(state.window), want_pool)


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,W,listed", [(1, 8, 2, False), (3, 200, 4, True), (70, 64, 3, True), (9, 1160, 4, False)])
def test_steps(io, B, C, W, listed):
    x, w, b = _inputs((B,), C, W, io, wide=True)
    desc = dl.ConvDesc(C, W, DT[io], num_slots=B + 3)
    state = dl.ConvState(desc, torch.randn(B + 3, W - 1, C).to(io).to(DEV))
    slots = torch.randperm(B + 3)[:B].to(torch.int32) if listed else None
    if listed:
        slots[B // 2] = -1
        slots[B - 1] = B + 3
    before, mark = ref.f64(state.window), torch.full((B, C), 2.0, dtype=io, device=DEV)
    out = dl.conv_step(desc, state, x, w, b, slot_idx=None if slots is None else slots.to(DEV), out=mark)
    assert out is mark and int(state.status) == (dl.STATUS_BAD_SLOT if listed else 0)
    want_pool = before.clone()
    for i in range(B):
        s = i if slots is None else int(slots[i])
        if s < 0 or s >= B + 3:
            assert (out[i] == 2.0).all()
            continue
        _, want, last = ref.conv_row(ref.f64(x)[i : i + 1], ref.f64(w), ref.f64(b), before[s], True)
        ref.close(out[i : i + 1], want, ref.conv_row(ref.f64(x)[i : i + 1], ref.f64(w), ref.f64(b), before[s], True, mag=True)[0], REL, f"row {i}")
        want_pool[s] = last
    assert torch.equal(ref.f64(state.window), want_pool)


def test_a_prompt_in_parts_and_token_by_token_is_the_prompt():
    C, W, T = 320, 4, 45
    x, w, b = _inputs((T,), C, W, torch.bfloat16)
    desc = dl.ConvDesc(C, W, num_slots=1)
    whole = dl.ConvState(desc, device=DEV)
    out = dl.conv_prefill(desc, whole, _plan((T,)), x, w, b)
    part, got = dl.ConvState(desc, device=DEV), []
    for lo, hi in ((0, 1), (1, 3), (3, 30)):
        got.append(dl.conv_prefill(desc, part, _plan((hi - lo,)), x[lo:hi].contiguous(), w, b))
    for t in range(30, T):
        got.append(dl.conv_step(desc, part, x[t : t + 1], w, b))
    assert torch.equal(torch.cat(got), out) and torch.equal(part.window, whole.window)


def test_values_that_are_not_finite_stay_in_their_window():
    lens, C = (6, 6), 64
    x, w, b = _inputs(lens, C, 4, torch.float32)
    x[2, 5], x[3, 7] = float("nan"), float("inf")
    out, final = dl.conv_forward(dl.ConvDesc(C, 4, dl.F32), _plan(lens), x, w, b)
    X = ref.f64(x)
    for i, r in enumerate(ref.rows_of(lens)):
        want = ref.conv_row(X[r], ref.f64(w), ref.f64(b), torch.zeros(3, C, dtype=ref.F64), True)[1]
        assert torch.equal(torch.isnan(out[r]).cpu(), torch.isnan(want))


def test_offsets_beyond_32_bits():
    C, T = 8192, 280_000                     # 2.3e9 elements
    x = torch.zeros(T, C, dtype=torch.bfloat16, device=DEV)
    tail = torch.randn(9, C).bfloat16().to(DEV)
    x[-9:] = tail
    w, b = torch.randn(C, 4, device=DEV), torch.randn(C, device=DEV)
    desc = dl.ConvDesc(C, 4, num_slots=90_000)
    plan = _plan((T - 9, 9), [3, 89_999])
    state = dl.ConvState(desc, device=DEV)   # 2.2e9 elements
    out = dl.conv_prefill(desc, state, plan, x, w, b)
    small = dl.ConvState(dl.ConvDesc(C, 4), device=DEV)
    want = dl.conv_prefill(small.desc, small, _plan((9,)), tail, w, b)
    assert torch.equal(out[-9:], want) and torch.equal(state.window[89_999], tail[-3:]) and not state.window[89_998].any()
    step = dl.conv_step(desc, state, tail[:1], w, b, slot_idx=torch.tensor([89_999], dtype=torch.int32, device=DEV))
    assert torch.equal(step, dl.conv_step(small.desc, small, tail[:1], w, b)) and torch.equal(state.window[89_999], small.window[0])
    del x, out, state
    torch.cuda.empty_cache()


def test_a_plan_for_many_more_tokens():
    rows, C, bound = 500, 64, 3000
    lens = [0] * rows
    lens[7], lens[499] = 2, 90
    x, w, b = _inputs((bound + 5,), C, 4, torch.float32)
    x[92:] = float("nan")
    plan = dl.Plan(rows, bound, device=DEV)
    dl.build_plan(torch.tensor(lens, dtype=torch.int32, device=DEV), plan)
    desc = dl.ConvDesc(C, 4, dl.F32)
    out, final = dl.conv_forward(desc, plan, x, w, b)
    _check_forward(out[:92], final[[7, 499]], x[:92], w, b, torch.zeros(2, 3, C, dtype=ref.F64), (2, 90), True)
    d = dl.conv_backward(desc, plan, x, w, b, torch.where(torch.isnan(x), x, torch.ones_like(x)))
    assert not out[92:].any() and not d.x[92:].any() and torch.isfinite(d.weight).all() and torch.isfinite(d.x).all()
    assert not final[[0, 250, 498]].any() and not d.init[[0, 250, 498]].any()


def test_streams_and_replays():
    lens, C = (20, 7), 256
    x, w, b = _inputs(lens, C, 4, torch.bfloat16)
    desc, plan = dl.ConvDesc(C, 4, num_slots=2), _plan(lens)
    want = dl.conv_prefill(desc, dl.ConvState(desc, device=DEV), plan, x, w, b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a, c = dl.ConvState(desc, device=DEV), dl.ConvState(desc, device=DEV)
    torch.cuda.synchronize()
    got = dl.conv_prefill(desc, a, plan, x, w, b, stream=side)       # two calls at once
    here = dl.conv_prefill(desc, c, plan, x, w, b)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(here, want)
    token, out = torch.zeros(2, C, dtype=torch.bfloat16, device=DEV), torch.zeros(2, C, dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dl.conv_step(desc, a, token, w, b, out=out)
    for t in range(5):
        token.copy_(x[t : t + 2])
        graph.replay()
        assert torch.equal(out, dl.conv_step(desc, c, token, w, b))
    assert torch.equal(a.window, c.window)


def test_no_rows_and_a_rebuilt_plan():
    desc = dl.ConvDesc(64, 4)
    plan = dl.Plan(0, 0, device=DEV)
    x, w, b = _inputs((4,), 64, 4, torch.bfloat16)
    out, final = dl.conv_forward(desc, plan, x, w, b)
    assert not out.any() and final.shape == (0, 3, 64)
    d = dl.conv_backward(desc, plan, x, w, b, x.clone())
    assert not d.x.any() and not d.weight.any() and not d.bias.any()
    plan = _plan((4,))
    out, _ = dl.conv(desc, plan, x.requires_grad_(), w, b)
    dl.build_plan(torch.tensor([3], dtype=torch.int32, device=DEV), plan)
    with pytest.raises(RuntimeError, match="rebuilt"):
        out.float().sum().backward()
