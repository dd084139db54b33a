"""The selective state space scan on the GPU against its 64-bit form.

Tolerances.  One step multiplies the state by a decay whose exponent carries the relative error of the step size (2^-21) times itself and
whose power of two is 2^-22 off, and rounds twice: e = 2^-21 (1 + max |delta A|) of its magnitude, and a state that went through t
steps t of them, in front of and behind a token alike.  So half a step of the output's type and (T + 16) e of the magnitude, T the
longest row; sums over all tokens add their number of roundings of 2^-24.
"""
import pytest
import torch

import layer_reference as ref
import paper_2608_15533_b200 as dl

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {torch.float32: dl.F32, torch.bfloat16: dl.BF16}


def _case(T, D, N, G, io, gate=True, skip=True, bias=True, softplus=True, wide=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    c = dict(x=rnd(T, D).to(io), A=-torch.rand(D, N, generator=g) * 4 - 0.02, D=1 + 0.3 * rnd(D) if skip else None, dt_bias=rnd(D) - 2 if bias else None, softplus=softplus)
    c["dt"] = (rnd(T, D) if softplus else torch.rand(T, D, generator=g) * 0.3 + 0.001).to(io)
    z = rnd(T, 2 * D if wide else D).to(io).to(DEV)
    bc = rnd(T, 2 * G * N + 8).to(io).to(DEV)
    c = {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    c["z"] = (z[:, D:] if wide else z) if gate else None
    if wide:   # columns of wider projections
        c["B"], c["C"] = bc[:, 8 : 8 + G * N].unflatten(1, (G, N)), bc[:, 8 + G * N :].unflatten(1, (G, N))
        c["x"] = torch.cat((c["x"], c["x"]), 1)[:, :D]
    else:
        c["B"], c["C"] = bc[:, : G * N].reshape(T, G, N).contiguous(), bc[:, G * N : 2 * G * N].reshape(T, G, N).contiguous()
    return c


def _args(c):
    return [c[k] for k in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias")]


def _rel(c, lens):
    raw = ref.f64(c["dt"]) + (0 if c["dt_bias"] is None else ref.f64(c["dt_bias"]))
    delta = torch.nn.functional.softplus(raw) if c["softplus"] else raw.abs()
    return (max(lens, default=0) + 16) * 2.0 ** -21 * (1 + float(delta.max() * c["A"].abs().max()) if delta.numel() else 1)


def _plan(lens, slots=None, token_map=True, room=0):
    plan = dl.Plan(len(lens), sum(lens) + room, device=DEV, token_map=token_map)
    s = None if slots is None else torch.tensor(slots, dtype=torch.int32, device=DEV)
    return dl.build_plan(torch.tensor(lens, dtype=torch.int32, device=DEV), plan, slots=s)


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D,N,G,lens,kw", [
    (8, 16, 1, (1,), dict()),
    (64, 16, 1, (3, 0, 1, 8, 9), dict(gate=False, skip=False, bias=False)),
    (72, 8, 1, (17, 40, 0, 2), dict(wide=True)),
    (48, 32, 2, (33, 5, 64), dict(softplus=False, bias=False)),
    (80, 64, 2, (0, 31, 7), dict(wide=True, skip=False)),
    (136, 16, 1, (300, 2, 150), dict()),               # rows that several stretches share
    (32, 16, 4, (129, 127, 1), dict(gate=False)),
    (24, 8, 1, (520,), dict(bias=False)),
    (40, 64, 1, (200,), dict(wide=True)),
])
def test_forward_and_gradients(io, D, N, G, lens, kw):
    T, n = sum(lens), len(lens)
    c = _case(T, D, N, G, io, **kw)
    g = torch.Generator().manual_seed(5)
    S0, dS = (torch.randn(n, D, N, generator=g).to(DEV) for _ in range(2))
    dout = torch.randn(T, D, generator=g).to(io).to(DEV)
    desc, plan = dl.SsmDesc(D, N, G, DT[io], c["softplus"]), _plan(lens, token_map=D != 136)
    rel = _rel(c, lens)
    work = dl.ssm_workspace(desc, n, T, train=True, device=DEV)
    work.fill_(0xff)                                    # NaN in whatever is read before it is written
    want, mag = (ref.ssm(c, lens, S0, dout, dS, mag=m) for m in (False, True))
    out, S = dl.ssm_forward(desc, plan, *_args(c), S_init=S0, workspace=work, save=True)
    ref.close(out, want[0], mag[0], rel, "out")
    ref.close(S, want[1], mag[1], rel, "S")
    d = dl.ssm_backward(desc, plan, *_args(c), dout, S_init=S0, dS_final=dS, workspace=work, saved=True)
    many = rel + T * 2.0 ** -24
    for k, e in (("x", rel), ("dt", rel), ("A", many), ("B", rel), ("C", rel), ("D", many), ("z", rel), ("dt_bias", many), ("S_init", rel)):
        got = getattr(d, k)
        assert (got is None) == (want[2][k] is None)
        if got is not None:
            ref.close(got, want[2][k], mag[2][k] + want[2][k].abs(), 2 * e, "d" + k)
    # computed again instead of kept, and bit for bit the same
    again = dl.ssm_backward(desc, plan, *_args(c), dout, S_init=S0, dS_final=dS)
    for k in ("x", "dt", "A", "B", "C", "S_init"):
        assert torch.equal(getattr(d, k), getattr(again, k)), k
    # without a start, without a gradient behind
    out0, S00 = dl.ssm_forward(desc, plan, *_args(c))
    zero = torch.zeros_like(S0)
    want0, mag0 = (ref.ssm(c, lens, zero, dout, zero, mag=m) for m in (False, True))
    ref.close(out0, want0[0], mag0[0], rel, "out from zeros")
    ref.close(S00, want0[1], mag0[1], rel, "S from zeros")
    d0 = dl.ssm_backward(desc, plan, *_args(c), dout)
    for k in ("x", "dt", "B", "C", "S_init"):
        ref.close(getattr(d0, k), want0[2][k], mag0[2][k] + want0[2][k].abs(), 2 * rel, "d" + k + " from zeros")


def test_gradients_against_differences():
    lens, D, N = (5, 3, 12), 16, 16
    c = _case(sum(lens), D, N, 1, torch.float32)
    desc, plan = dl.SsmDesc(D, N, 1, dl.F32), _plan(lens)
    names = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias")
    leaf = {k: c[k].detach().clone().requires_grad_() for k in names} | {"S_init": torch.randn(3, D, N, device=DEV).requires_grad_()}
    out, S = dl.ssm(desc, plan, *[leaf[k] for k in names], S_init=leaf["S_init"])
    do, dS = torch.randn_like(out), torch.randn_like(S)
    grads = dict(zip(leaf, torch.autograd.grad((out, S), list(leaf.values()), (do, dS))))
    base = {k: ref.f64(t) for k, t in leaf.items()}

    def value(**kw):
        t = base | kw
        o, s, _ = ref.ssm({**t, "softplus": True}, lens, t["S_init"])
        return float((o * ref.f64(do)).sum() + (s * ref.f64(dS)).sum())

    mag = ref.ssm({**base, "softplus": True}, lens, base["S_init"], do, dS, mag=True)[2]
    rel = _rel(c, lens)
    for k, g in grads.items():
        v = torch.randn(base[k].shape, dtype=ref.F64)
        want = (value(**{k: base[k] + 1e-6 * v}) - value(**{k: base[k] - 1e-6 * v})) / 2e-6
        tol = 4 * rel * float((mag[k] * v.abs()).sum()) + 1e-6 * abs(want)
        assert abs(float((ref.f64(g) * v).sum()) - want) < tol, k


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
def test_prefill_of_a_pool(io):
    lens, D, N = (140, 0, 1, 2, 300, 3, 5, 9), 72, 16
    slots = [5, 2, 0, -1, 7, 9, 1, 3]  # row 3 is padding, slot 9 does not exist
    T = sum(lens)
    c = _case(T + 6, D, N, 1, io)
    rows = ref.rows_of(lens)
    for k in ("x", "dt", "B", "C", "z"):   # skipped tokens may hold anything
        c[k][rows[3]] = float("nan")
        c[k][rows[5]] = float("inf")
        c[k][T:] = float("nan")
    desc = dl.SsmDesc(D, N, 1, DT[io], num_slots=8)
    pool = torch.randn(8, D, N, device=DEV)
    fresh = torch.tensor([0, 1, 1, 0, 0, 0, 1, 0], dtype=torch.int32, device=DEV)
    live = {k: v if k in ("A", "D", "dt_bias", "softplus") else torch.cat([v[r] for i, r in enumerate(rows) if i not in (3, 5)]) for k, v in c.items()}
    kept = [n for i, n in enumerate(lens) if i not in (3, 5)]
    start = torch.stack([pool[s] * (0 if fresh[i] else 1) for i, s in enumerate(slots) if i not in (3, 5)])
    want, mag = (ref.ssm(live, kept, start, mag=m) for m in (False, True))
    rel = _rel(live, kept)
    for mine in (False, True):
        state = dl.SsmState(desc, pool.clone())
        plan = _plan(lens, slots, room=4, token_map=mine)
        mark = torch.full((T + 6, D), 3.0, dtype=io, device=DEV)
        work = dl.ssm_workspace(desc, len(lens), T + 4, device=DEV)
        work.fill_(0xff)
        out = dl.ssm_prefill(desc, state, plan, *_args(c), fresh=fresh, out=mark if mine else None, workspace=work)
        assert int(state.status) == dl.STATUS_BAD_SLOT
        still = 3.0 if mine else 0.0
        assert (out[rows[3]] == still).all() and (out[rows[5]] == still).all() and (out[T:] == still).all()
        ref.close(torch.cat([out[r] for i, r in enumerate(rows) if i not in (3, 5)]), want[0], mag[0], rel, "out")
        j = 0
        for i, s in enumerate(slots):
            if i in (3, 5):
                continue
            if lens[i]:
                ref.close(state.S[s], want[1][j], mag[1][j], rel, f"slot {s}")
            else:
                assert torch.equal(state.S[s], pool[s])
            j += 1
        for s in (4, 6):
            assert torch.equal(state.S[s], pool[s])


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,D,N,G,listed,kw", [(1, 8, 16, 1, False, dict()), (3, 200, 8, 1, True, dict(gate=False)), (70, 64, 32, 2, True, dict(wide=True)),
                                               (9, 72, 64, 1, False, dict(softplus=False, bias=False, skip=False))])
def test_steps(io, B, D, N, G, listed, kw):
    c = _case(B, D, N, G, io, **kw)
    desc = dl.SsmDesc(D, N, G, DT[io], c["softplus"], num_slots=B + 3)
    state = dl.SsmState(desc, torch.randn(B + 3, D, N, device=DEV))
    slots = torch.randperm(B + 3)[:B].to(torch.int32) if listed else None
    if listed:
        slots[B // 2] = -1
        slots[B - 1] = B + 3
    before, mark = state.S.clone(), torch.full((B, D), 2.0, dtype=io, device=DEV)
    out = dl.ssm_step(desc, state, *_args(c), slot_idx=None if slots is None else slots.to(DEV), out=mark)
    assert out is mark and int(state.status) == (dl.STATUS_BAD_SLOT if listed else 0)
    at = [i if slots is None else int(slots[i]) for i in range(B)]
    ok = [i for i in range(B) if 0 <= at[i] < B + 3]
    start = torch.zeros(B, D, N, device=DEV)
    for i in ok:
        start[i] = before[at[i]]
    want, mag = (ref.ssm(c, [1] * B, start, mag=m) for m in (False, True))
    rel = _rel(c, (1,))
    want_pool, mag_pool = ref.f64(before), torch.zeros_like(ref.f64(before))
    for i in range(B):
        if i not in ok:
            assert (out[i] == 2.0).all()
            continue
        ref.close(out[i], want[0][i], mag[0][i], rel, f"row {i}")
        want_pool[at[i]], mag_pool[at[i]] = want[1][i], mag[1][i]
    ref.close(state.S, want_pool, mag_pool, rel, "pool")


def test_a_prompt_in_parts_and_token_by_token_is_the_prompt():
    D, N, T = 96, 16, 460
    c = _case(T, D, N, 1, torch.float32)
    cut = lambda lo, hi: [v if k in ("A", "D", "dt_bias") else v[lo:hi] for k, v in ((k, c[k]) for k in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias"))]
    desc = dl.SsmDesc(D, N, 1, dl.F32, num_slots=1)
    whole, part, got = dl.SsmState(desc, device=DEV), dl.SsmState(desc, device=DEV), []
    out = dl.ssm_prefill(desc, whole, _plan((T,)), *_args(c))
    for lo, hi in ((0, 1), (1, 200), (200, 420)):
        got.append(dl.ssm_prefill(desc, part, _plan((hi - lo,)), *cut(lo, hi)))
    for t in range(420, T):
        got.append(dl.ssm_step(desc, part, *cut(t, t + 1)))
    mag = ref.ssm(c, (T,), torch.zeros(1, D, N), mag=True)
    rel = 2 * _rel(c, (T,))
    ref.close(torch.cat(got), ref.f64(out), mag[0], rel, "out")
    ref.close(part.S, ref.f64(whole.S), mag[1], rel, "S")


def test_a_plan_for_many_more_tokens_and_rows_without_any():
    # a captured step's plan: its bounds are fixed, this step brings few tokens; what lies behind them may be anything
    rows, D, N, bound = 3000, 40, 16, 4000
    lens = [0] * rows
    for i, n in ((5, 3), (700, 150), (2999, 20)):
        lens[i] = n
    T = sum(lens)
    c = _case(bound + 9, D, N, 1, torch.float32)
    for k in ("x", "dt", "B", "C", "z"):
        c[k][T:] = float("nan")
    desc, plan = dl.SsmDesc(D, N, 1, dl.F32), dl.Plan(rows, bound, device=DEV)
    dl.build_plan(torch.tensor(lens, dtype=torch.int32, device=DEV), plan)
    S0, dS = torch.randn(rows, D, N, device=DEV), torch.randn(rows, D, N, device=DEV)
    work = dl.ssm_workspace(desc, rows, bound + 9, train=True, device=DEV)
    work.fill_(0xff)
    out, S = dl.ssm_forward(desc, plan, *_args(c), S_init=S0, workspace=work, save=True)
    dout = torch.randn(bound + 9, D, device=DEV)
    dout[T:] = float("nan")
    d = dl.ssm_backward(desc, plan, *_args(c), dout, S_init=S0, dS_final=dS, workspace=work, saved=True)
    cut = {k: v[:T] if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items()}
    live = [5, 700, 2999]
    want, mag = (ref.ssm(cut, [3, 150, 20], S0[live], dout[:T], dS[live], mag=m) for m in (False, True))
    rel = _rel(cut, [150])
    ref.close(out[:T], want[0], mag[0], rel, "out")
    ref.close(S[live], want[1], mag[1], rel, "S")
    dead = torch.ones(rows, dtype=torch.bool, device=DEV)
    dead[live] = False
    assert not out[T:].any() and torch.equal(S[dead], S0[dead]) and torch.equal(d.S_init[dead], dS[dead])
    for k in ("x", "dt", "B", "C", "z"):
        got = getattr(d, k)
        assert not got[T:].any()
        ref.close(got[:T], want[2][k], mag[2][k] + want[2][k].abs(), 2 * rel, "d" + k)
    for k in ("A", "D", "dt_bias"):
        ref.close(getattr(d, k), want[2][k], mag[2][k], 2 * rel + T * 2.0 ** -24, "d" + k)
    ref.close(d.S_init[live], want[2]["S_init"], mag[2]["S_init"], 2 * rel, "dS_init")


def test_step_sizes_at_their_ends():
    # delta = 0 leaves the state as it is, a large one replaces it; both without NaN
    D, N = 16, 16
    c = _case(4, D, N, 1, torch.float32, bias=False)
    c["dt"] = torch.tensor([-1e30, -200.0, 200.0, 60.0], device=DEV)[:, None].expand(4, D).contiguous()
    c["A"] = torch.full((D, N), -1.0, device=DEV)
    desc = dl.SsmDesc(D, N, 1, dl.F32)
    S0 = torch.randn(1, D, N, device=DEV)
    one = {k: v[:2] if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items()}
    out, S = dl.ssm_forward(desc, _plan((2,)), *_args(one), S_init=S0)
    assert torch.equal(S, S0)
    out, S = dl.ssm_forward(desc, _plan((4,)), *_args(c), S_init=S0)
    want = 60.0 * c["x"][3][:, None] * c["B"][3]
    assert torch.allclose(S[0], want, rtol=1e-6, atol=0) and torch.isfinite(out).all()


def test_values_that_are_not_finite_stay_in_their_row_and_channel():
    lens, D, N = (40, 30, 20), 64, 16
    c = _case(sum(lens), D, N, 1, torch.float32)
    c["x"][45, 3], c["dt"][50, 9] = float("nan"), float("nan")
    desc = dl.SsmDesc(D, N, 1, dl.F32)
    out, S = dl.ssm_forward(desc, _plan(lens), *_args(c))
    bad = torch.zeros(90, D, dtype=torch.bool)
    bad[45:70, 3], bad[50:70, 9] = True, True
    assert torch.equal(torch.isnan(out).cpu(), bad)
    assert torch.isnan(S[1, 3]).all() and torch.isnan(S[1, 9]).all() and int(torch.isnan(S).sum()) == 2 * N
    c["A"][5, 2] = float("nan")
    out, S = dl.ssm_forward(desc, _plan(lens), *_args(c))
    assert torch.isnan(out[:, 5]).all() and torch.isnan(S[:, 5, 2]).all() and not torch.isnan(S[:, 5, :2]).any()


def test_offsets_beyond_32_bits():
    D, N, slots = 4096, 64, 8400             # 2.2e9 states
    desc = dl.SsmDesc(D, N, num_slots=slots)
    state = dl.SsmState(desc, torch.zeros(slots, D, N, device=DEV))
    c = _case(3, D, N, 1, torch.bfloat16)
    last = torch.tensor([slots - 1], dtype=torch.int32, device=DEV)
    small = dl.SsmState(dl.SsmDesc(D, N), device=DEV)
    one = {k: v[:1] if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items()}
    got = dl.ssm_step(desc, state, *_args(one), slot_idx=last)
    assert torch.equal(got, dl.ssm_step(small.desc, small, *_args(one))) and torch.equal(state.S[-1], small.S[0]) and not state.S[-2].any()
    got = dl.ssm_prefill(desc, state, _plan((3,), [slots - 1]), *_args(c))
    assert torch.equal(got, dl.ssm_prefill(small.desc, small, _plan((3,)), *_args(c))) and torch.equal(state.S[-1], small.S[0])
    del state
    torch.cuda.empty_cache()
    D, T = 8192, 270_000                      # 2.2e9 inputs
    x = torch.zeros(T, D, dtype=torch.bfloat16, device=DEV)
    bc = torch.zeros(T, 1, 8, dtype=torch.bfloat16, device=DEV)
    tail = _case(5, D, 8, 1, torch.bfloat16, gate=False)
    x[-5:], bc[-5:] = tail["x"], tail["B"]
    desc = dl.SsmDesc(D, 8)
    out, S = dl.ssm_forward(desc, _plan((T - 5, 5)), x, x, tail["A"], bc, bc)
    want, S1 = dl.ssm_forward(desc, _plan((5,)), tail["x"], tail["x"], tail["A"], tail["B"], tail["B"])
    assert torch.equal(out[-5:], want) and torch.equal(S[1:], S1) and not out[:-5].any()
    del x, bc, out
    torch.cuda.empty_cache()


def test_streams_and_replays():
    lens, D, N = (200, 7), 256, 16
    c = _case(sum(lens), D, N, 1, torch.bfloat16)
    desc, plan = dl.SsmDesc(D, N, num_slots=2), _plan(lens)
    want = dl.ssm_prefill(desc, dl.SsmState(desc, device=DEV), plan, *_args(c))
    a, b = dl.SsmState(desc, device=DEV), dl.SsmState(desc, device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = dl.ssm_prefill(desc, a, plan, *_args(c), stream=side)      # two calls at once, a workspace each
    here = dl.ssm_prefill(desc, b, plan, *_args(c))
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(here, want) and torch.equal(a.S, b.S)
    token = {k: v[:2].clone() if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items()}
    out = torch.zeros(2, D, dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dl.ssm_step(desc, a, *_args(token), out=out)
    for t in range(4):
        for k in ("x", "dt", "B", "C", "z"):
            token[k].copy_(c[k][t : t + 2])
        graph.replay()
        assert torch.equal(out, dl.ssm_step(desc, b, *_args(token)))
    assert torch.equal(a.S, b.S)


def test_training_step_in_a_graph():
    lens, D, N = (150, 30), 64, 16
    c = _case(sum(lens), D, N, 1, torch.float32)
    desc, plan = dl.SsmDesc(D, N, 1, dl.F32), _plan(lens)
    names = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        leaf = {k: c[k].detach().clone().contiguous().requires_grad_() for k in names}
        for _ in range(2):
            out, S = dl.ssm(desc, plan, *leaf.values())
            torch.autograd.grad(out.square().sum() + S.sum(), list(leaf.values()))
        del out, S
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, S = dl.ssm(desc, plan, *leaf.values())
        grads = torch.autograd.grad(out.square().sum() + S.sum(), list(leaf.values()))
    with torch.no_grad():
        leaf["x"].mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    eager = {k: v.detach().clone().requires_grad_() for k, v in leaf.items()}
    o, s = dl.ssm(desc, plan, *eager.values())
    want = torch.autograd.grad(o.square().sum() + s.sum(), list(eager.values()))
    for g, w, k in zip(grads, want, names):
        assert torch.equal(g, w), k


def test_capture_beside_an_eager_graph_is_refused():
    lens, D = (4,), 64
    c = _case(4, D, 16, 1, torch.float32)
    desc, plan = dl.SsmDesc(D, 16, 1, dl.F32), _plan(lens)
    c["x"] = c["x"].clone().requires_grad_()
    out, _ = dl.ssm(desc, plan, *_args(c))
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="eager|default stream"):
        with torch.cuda.graph(graph):
            dl.ssm(desc, plan, *_args(c))
    out.sum().backward()
    assert torch.isfinite(c["x"].grad).all()


def test_no_rows_and_a_rebuilt_plan():
    desc = dl.SsmDesc(64)
    c = _case(4, 64, 16, 1, torch.bfloat16)
    plan = dl.Plan(0, 0, device=DEV)
    out, S = dl.ssm_forward(desc, plan, *_args(c))
    assert not out.any() and S.shape == (0, 64, 16)
    d = dl.ssm_backward(desc, plan, *_args(c), c["x"].contiguous())
    assert not any(getattr(d, k).any() for k in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias"))
    plan = _plan((0, 0))                      # rows without tokens hand their states on
    S0 = torch.randn(2, 64, 16, device=DEV)
    empty = {k: v[:0] if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items()}
    out, S = dl.ssm_forward(desc, plan, *_args(empty), S_init=S0)
    assert torch.equal(S, S0) and out.shape == (0, 64)
    d = dl.ssm_backward(desc, plan, *_args(empty), empty["x"], S_init=S0, dS_final=S0)
    assert torch.equal(d.S_init, S0) and not d.A.any() and not d.D.any()
    plan = _plan((4,))
    c["x"] = c["x"].clone().requires_grad_()
    out, _ = dl.ssm(desc, plan, *_args(c))
    dl.build_plan(torch.tensor([3], dtype=torch.int32, device=DEV), plan)
    with pytest.raises(RuntimeError, match="rebuilt"):
        out.float().sum().backward()


def _lowest(io):
    return torch.finfo(io).min


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", ["-inf", "lowest", "-2.4e38"])
@pytest.mark.parametrize("N,lens", [(16, (9, 40)), (8, (300,)), (64, (33, 140))])
def test_tokens_masked_by_their_step_size(io, value, N, lens):
    # softplus is 0 there: the token leaves the state as it is, and no gradient passes through its step size
    D, T = 72, sum(lens)
    c = _case(T, D, N, 1, io, wide=True)
    masked = torch.zeros(T, dtype=torch.bool, device=DEV)
    masked[::3], masked[-1], masked[140:142] = True, True, True
    whole = c["dt"].clone()
    c["dt"][masked] = _lowest(io) if value == "lowest" else float(value)
    live = {**c, "dt": torch.where(masked[:, None], torch.full_like(whole, -1e30), whole)}   # a softplus of 0 for the 64-bit form
    desc, plan = dl.SsmDesc(D, N, 1, DT[io], num_slots=len(lens)), _plan(lens)
    g = torch.Generator().manual_seed(7)
    S0, dS = (torch.randn(len(lens), D, N, generator=g).to(DEV) for _ in range(2))
    dout = torch.randn(T, D, generator=g).to(io).to(DEV)
    out, S = dl.ssm_forward(desc, plan, *_args(c), S_init=S0)
    d = dl.ssm_backward(desc, plan, *_args(c), dout, S_init=S0, dS_final=dS)
    want, mag = (ref.ssm(live, lens, S0, dout, dS, mag=m) for m in (False, True))
    rel = _rel(live, lens)
    ref.close(out, want[0], mag[0], rel, "out")
    ref.close(S, want[1], mag[1], rel, "S")
    many = rel + T * 2.0 ** -24
    for k, e in (("x", rel), ("dt", rel), ("A", many), ("B", rel), ("C", rel), ("D", many), ("z", rel), ("dt_bias", many), ("S_init", rel)):
        ref.close(getattr(d, k), want[2][k], mag[2][k] + want[2][k].abs(), 2 * e, "d" + k)
    assert not d.dt[masked].any()
    state = dl.SsmState(desc, S0.clone())
    assert torch.equal(dl.ssm_prefill(desc, state, plan, *_args(c)), out) and torch.equal(state.S, S)
    # nothing but masked tokens, of a prompt and one by one: the bits of the state stay
    c["dt"][:] = c["dt"][0].clone()
    state = dl.SsmState(desc, S0.clone())
    dl.ssm_prefill(desc, state, plan, *_args(c))
    assert torch.equal(state.S, S0)
    token = {k: v[: len(lens)] if k in ("x", "dt", "B", "C", "z") else v for k, v in c.items()}
    out = dl.ssm_step(desc, state, *_args(token))
    assert torch.equal(state.S, S0) and torch.isfinite(out).all()


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
def test_step_sizes_as_large_as_they_get(io):
    # softplus is its argument there: the old state is gone, the new one delta x B; infinite where delta is
    D, N = 16, 16
    c = _case(3, D, N, 1, io, bias=False, gate=False)
    c["A"] = torch.full((D, N), -1.0, device=DEV)
    c["x"], c["B"] = torch.full_like(c["x"], 0.5), torch.full_like(c["B"], 0.25)
    c["dt"][2] = float("nan")
    for value in (2.4e38, 3e38, float("inf")):
        c["dt"][:2] = value
        delta = float(c["dt"][0, 0])
        one = {k: v[:2] if k in ("x", "dt", "B", "C") else v for k, v in c.items()}
        S0 = torch.randn(1, D, N, device=DEV)
        S = dl.ssm_forward(dl.SsmDesc(D, N, 1, DT[io]), _plan((2,)), *_args(one), S_init=S0)[1]
        if value < float("inf"):
            assert torch.equal(S, torch.full_like(S, delta * 0.125))
            state = dl.SsmState(dl.SsmDesc(D, N, 1, DT[io], num_slots=2), S0.repeat(2, 1, 1))
            dl.ssm_step(state.desc, state, *_args(one))
            assert torch.equal(state.S, torch.full_like(state.S, delta * 0.125))
        state = dl.SsmState(dl.SsmDesc(D, N, 1, DT[io], num_slots=3), S0.repeat(3, 1, 1))
        dl.ssm_step(state.desc, state, *_args(c))
        assert bool((state.S[:2] == delta * 0.125).all()) and torch.isnan(state.S[2]).all()   # (a step size that is no number stays none)


def test_step_sizes_keep_their_relative_accuracy():
    # The step size alone as a state, its derivative alone as a gradient, over all that is no denormal number.  A power of two is 2^-22 off,
    # its correction's sum rounds once (2^-24), the polynomial's last sums and the product with e three times more, and its own error is 2^-27:
    # 2^-21 together.  The derivative: the same e, 1 + e, a reciprocal of 2^-23 and a product.
    B, D, N = 2048, 256, 8
    v = torch.linspace(-85, 80, B * D, dtype=torch.float64).to(torch.float32).view(B, D).to(DEV)
    one = torch.zeros(B, 1, N, device=DEV)
    one[..., 0] = 1
    A = torch.full((D, N), -1.0, device=DEV)
    desc = dl.SsmDesc(D, N, 1, dl.F32, num_slots=B)
    args = (torch.ones(B, D, device=DEV), v, A, one, torch.zeros_like(one))
    state, V = dl.SsmState(desc, device=DEV), v.double()
    dl.ssm_step(desc, state, *args)
    want = V.clamp(min=0) + torch.log1p(torch.exp(-V.abs()))
    assert float((state.S[..., 0].double() / want - 1).abs().max()) < 2.0 ** -21
    plan = _plan((1,) * B)
    dS = torch.zeros(B, D, N, device=DEV)
    dS[..., 0] = 1
    S = dl.ssm_forward(desc, plan, *args)[1]
    assert torch.equal(S, state.S)
    d = dl.ssm_backward(desc, plan, *args, None, None, None, torch.zeros(B, D, device=DEV), dS_final=dS)
    assert float((d.dt.double() * (1 + torch.exp(-V)) - 1).abs().max()) < 2.0 ** -21


@pytest.mark.parametrize("known", [True, False])
def test_slow_channels_forget_at_their_rate(known):
    # A state without input is the product of its decays.  Their roundings to fp32 cancel over thousands of channels; what does not is a
    # mean error, which a state that remembers 1000 tokens holds 1000 times.  Under a sixteenth of half a step of fp32 a token (2^-28)
    # is asked for, where the bias says what the step sizes are like or every token is looked at, and under an eighth otherwise: the
    # channels' mean is itself known to 2e-10 (1e-7 a token of a channel, 128 tokens, 4096 channels and states).
    D, N, T = 256, 16, 128
    g = torch.Generator().manual_seed(11)
    A = -(0.5 + 0.5 * torch.rand(D, N, generator=g)).to(DEV)
    bias = torch.log(torch.expm1(0.0005 + 0.0015 * torch.rand(D, generator=g))).to(DEV) if known else None
    dt = (0.5 * torch.randn(T, D, generator=g) if known else 0.0005 + 0.0015 * torch.rand(T, D, generator=g)).to(DEV)
    delta = torch.log1p(torch.exp(dt.double() + bias.double())) if known else dt.double()
    zero, bc = torch.zeros(T, D, device=DEV), torch.zeros(T, 1, N, device=DEV)
    desc, plan = dl.SsmDesc(D, N, 1, dl.F32, softplus=known, num_slots=1), _plan((T,))
    ones = torch.ones(1, D, N, device=DEV)
    want = torch.exp(delta.sum(0)[:, None] * A.double())

    def mean_error(S):
        return abs(float((S[0].double() / want - 1).mean())) / T

    S = dl.ssm_forward(desc, plan, zero, dt, A, bc, bc, dt_bias=bias, S_init=ones)[1]
    assert mean_error(S) < (2.0 ** -28 if known else 2.0 ** -27)
    d = dl.ssm_backward(desc, plan, zero, dt, A, bc, bc, None, None, bias, zero, S_init=ones, dS_final=ones)
    assert mean_error(d.S_init) < (2.0 ** -28 if known else 2.0 ** -27)
    state = dl.SsmState(desc, ones.clone())
    for t in range(T):
        dl.ssm_step(desc, state, zero[t : t + 1], dt[t : t + 1], A, bc[t : t + 1], bc[t : t + 1], dt_bias=bias)
    assert mean_error(state.S) < 2.0 ** -28
