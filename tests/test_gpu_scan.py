"""Scan over packed sequences, its gradients, prefill into the slot pool and the step plan against plain references in
64 bits, at the lengths, head groups, gates and slots where they can go wrong.

Tolerances (max |x - ref| / max |ref|): a sum in fp32 over a contraction of up to 128 channels, 64 tokens of a chunk and
64 more through the triangular inverse makes at most 256 additions, each off by at most one unit 2^-23 of the largest
partial sum: 256 * 2^-23 = 3.1e-5.  A bf16 result adds half a step, 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

import paper_2608_15533_b200 as dl
import scan_reference as ref
from paper_2608_15533_b200 import binding

pytestmark = pytest.mark.gpu

TOL_F32 = 256 * 2.0 ** -23
TOL = {torch.float32: TOL_F32, torch.bfloat16: TOL_F32 + 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16


def err(x, y):
    x, y = x.double().cpu(), y.double().cpu()
    assert x.shape == y.shape
    assert torch.isfinite(x).all()
    m = y.abs().max().item() if y.numel() else 0.0
    return (x - y).abs().max().item() / m if m > 0 else (x.abs().max().item() if x.numel() else 0.0)


def make_desc(op, H, Hq, dk, dv, io, scale=0.7, num_slots=1, cap=8, base=None):
    return dl.Desc(op=op, num_slots=num_slots, H=H, H_qk=Hq, d_k=dk, d_v=dv, cap=cap, io_dtype=dl.F32 if io == F32 else dl.BF16,
                   scale=1.0 if op == ref.RWKV6 else scale, base_dtype=dl.F32 if base is None else base)


def make_plan(lens, slots=None, tail=0, **kw):
    plan = dl.Plan(len(lens), sum(lens) + tail, device="cuda")
    s = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
    return dl.build_plan(torch.tensor(lens, dtype=torch.int32, device="cuda"), plan, slots=s, **kw)


LENS = [17, 0, 1, 64, 2, 129, 63, 65, 16, 200]


@pytest.mark.parametrize("op", sorted(ref.OPS.values()))
@pytest.mark.parametrize("io,H,Hq,dk,dv", [(BF16, 4, 2, 128, 128), (F32, 3, 3, 64, 64), (BF16, 3, 1, 64, 128), (F32, 2, 1, 128, 64),
                                           (F32, 2, 2, 128, 128), (BF16, 2, 2, 64, 64)])
def test_forward(op, io, H, Hq, dk, dv):
    t, S0 = ref.inputs(op, LENS, H, Hq, dk, dv, io, seed=op)
    desc, plan = make_desc(op, H, Hq, dk, dv, io), make_plan(LENS)
    out, S = dl.scan_forward(desc, plan, **t, S_init=S0)
    want, S_want = ref.scan(op, desc.scale, LENS, t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], S0)
    assert err(out, want) < TOL[io]
    assert err(S, S_want) < TOL_F32
    assert torch.equal(S[1], S0[1])  # a sequence without tokens keeps its state
    zero, S = dl.scan_forward(desc, plan, **t)
    want, S_want = ref.scan(op, desc.scale, LENS, t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], torch.zeros_like(S0))
    assert err(zero, want) < TOL[io] and err(S, S_want) < TOL_F32


def grads_of(op, scale, lens, t, S0, dout, dS):
    leaf = {x: None if y is None else y.double().requires_grad_() for x, y in t.items()}
    s0 = S0.double().requires_grad_()
    out, S = ref.scan(op, scale, lens, leaf["q"], leaf["k"], leaf["v"], leaf["g"], leaf["beta"], leaf["u_bonus"], s0)
    names = [x for x in leaf if leaf[x] is not None]
    n = out.shape[0]
    got = torch.autograd.grad((out, S), [*(leaf[x] for x in names), s0], (dout[:n].double(), dS.double()), allow_unused=True)
    return dict(zip([*names, "S_init"], got))


def check_grads(d, want, io):
    for name, w in want.items():
        x = getattr(d, name)
        assert err(x, w) < (TOL[io] if name in ("q", "k", "v") else TOL_F32), name


@pytest.mark.parametrize("op", sorted(ref.OPS.values()))
@pytest.mark.parametrize("io,H,Hq,dk,dv", [(BF16, 4, 2, 128, 128), (F32, 3, 3, 64, 64), (BF16, 3, 1, 64, 128), (F32, 2, 1, 128, 64),
                                           (F32, 2, 2, 128, 128)])
def test_backward(op, io, H, Hq, dk, dv):
    lens = [17, 0, 1, 64, 2, 129, 63, 16]
    t, S0 = ref.inputs(op, lens, H, Hq, dk, dv, io, seed=op + 10, tail=5)
    desc, plan = make_desc(op, H, Hq, dk, dv, io), make_plan(lens, tail=5)
    gen = torch.Generator().manual_seed(3)
    dout = torch.randn(t["v"].shape, generator=gen).to(io).cuda()
    dS = (torch.randn(S0.shape, generator=gen) * 0.1).cuda()
    want = grads_of(op, desc.scale, lens, t, S0, dout, dS)
    d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, dS_final=dS)
    check_grads(d, want, io)
    T = sum(lens)
    for x in (d.q, d.k, d.v, d.g, d.beta):
        assert x is None or not x[T:].any()   # rows behind the last sequence
    # with the states that a forward pass kept, and without dS_final / S_init
    ws = dl.scan_workspace(desc, len(lens), plan.max_tokens, train=True)
    dl.scan_forward(desc, plan, **t, S_init=S0, workspace=ws, save=True)
    again = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, dS_final=dS, workspace=ws, saved=True)
    for name in want:
        assert torch.equal(getattr(d, name), getattr(again, name)), name
    plain = dl.scan_backward(desc, plan, **t, dout=dout)
    check_grads(plain, grads_of(op, desc.scale, lens, t, torch.zeros_like(S0), dout, torch.zeros_like(dS)), io)


@pytest.mark.parametrize("op", sorted(ref.OPS.values()))
def test_gradients_against_differences(op):
    """<gradient, direction> against the central difference of the fp64 loss: step 1e-4, so the difference itself is good
    to 1e-8 of its curvature; the direction's norm is spread over all inputs, so fp32 gradients give TOL_F32 of the
    largest term."""
    lens, H, dk, dv = [37, 70], 2, 64, 64
    t, S0 = ref.inputs(op, lens, H, H, dk, dv, F32, seed=op + 20)
    desc, plan = make_desc(op, H, H, dk, dv, F32), make_plan(lens)
    gen = torch.Generator().manual_seed(4)
    dout, dS = torch.randn(t["v"].shape, generator=gen).cuda(), torch.randn(S0.shape, generator=gen).cuda() * 0.1
    d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, dS_final=dS)
    for name in ("q", "k", "v", "g", "beta", "u_bonus", "S_init"):
        x = S0 if name == "S_init" else t[name]
        if x is None:
            continue
        way = torch.randn(x.shape, generator=gen).cuda().double()

        def loss(e):
            y = {a: None if b is None else b.double() for a, b in t.items()} | {"S0": S0.double()}
            y["S0" if name == "S_init" else name] = x.double() + e * way
            out, S = ref.scan(op, desc.scale, lens, y["q"], y["k"], y["v"], y["g"], y["beta"], y["u_bonus"], y["S0"])
            return (out * dout).sum() + (S * dS).sum()

        want = ((loss(1e-4) - loss(-1e-4)) / 2e-4).item()
        terms = getattr(d, name).double() * way
        assert abs(terms.sum().item() - want) < TOL_F32 * terms.abs().sum().item() + 1e-6 * abs(want), name


@pytest.mark.parametrize("op", [ref.GDN, ref.RETNET, ref.KDA, ref.RWKV6, ref.GLA])
@pytest.mark.parametrize("gates", ["none", "strong", "reset", "mixed"])
def test_extreme_gates(op, gates):
    """Gates of zero, gates that empty the state within a block of tokens, resets (-inf), and all of them by turns."""
    lens, H, dk, dv = [150, 40], 2, 64, 64
    t, S0 = ref.inputs(op, lens, H, H, dk, dv, F32, seed=op + 30)
    g = t["g"]
    gen = torch.Generator().manual_seed(5)
    pick = torch.rand(g.shape, generator=gen).cuda()
    if gates == "none":
        g = torch.zeros_like(g)
    elif gates == "strong":
        g = g * 40 - 3
    elif gates == "reset":
        g = torch.where(pick < 0.1, -torch.inf, g)
    else:
        g = torch.where(pick < 0.05, -torch.inf, torch.where(pick < 0.2, -50.0, torch.where(pick < 0.5, 0.0, g)))
    t["g"] = g.contiguous()
    desc, plan = make_desc(op, H, H, dk, dv, F32), make_plan(lens)
    out, S = dl.scan_forward(desc, plan, **t, S_init=S0)
    want, S_want = ref.scan(op, desc.scale, lens, t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], S0)
    assert err(out, want) < TOL_F32 and err(S, S_want) < TOL_F32
    dout, dS = torch.randn(t["v"].shape, generator=gen).cuda(), torch.randn(S0.shape, generator=gen).cuda() * 0.1
    d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, dS_final=dS)
    check_grads(d, grads_of(op, desc.scale, lens, t, S0, dout, dS), F32)


@pytest.mark.parametrize("op", [ref.GDN, ref.KDA])
@pytest.mark.parametrize("case", ["beta0", "beta1", "same_key", "tiny_beta"])
def test_delta_rule_edges(op, case):
    """beta of 0, 1 and below fp32's normal numbers' square, and one key for every token (the inverse at its worst)."""
    lens, H, dk, dv = [100], 2, 64, 64
    t, S0 = ref.inputs(op, lens, H, H, dk, dv, F32, seed=op + 40)
    if case == "beta0":
        t["beta"][::2] = 0.0
    elif case == "beta1":
        t["beta"].fill_(1.0)
    elif case == "tiny_beta":
        t["beta"][::3] = 1e-25
    else:
        t["k"] = t["k"][:1].expand_as(t["k"]).contiguous()
        t["beta"].fill_(1.0)
        t["g"] = t["g"] * 0.01
    desc, plan = make_desc(op, H, H, dk, dv, F32), make_plan(lens)
    out, S = dl.scan_forward(desc, plan, **t, S_init=S0)
    want, S_want = ref.scan(op, desc.scale, lens, t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], S0)
    assert err(out, want) < TOL_F32 and err(S, S_want) < TOL_F32
    gen = torch.Generator().manual_seed(6)
    dout, dS = torch.randn(t["v"].shape, generator=gen).cuda(), torch.randn(S0.shape, generator=gen).cuda() * 0.1
    d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, dS_final=dS)
    check_grads(d, grads_of(op, desc.scale, lens, t, S0, dout, dS), F32)


def pool(desc, seed, poison=False):
    gen = torch.Generator().manual_seed(seed)
    S = (torch.randn(desc.num_slots, desc.H, desc.d_k, desc.d_v, generator=gen) * 0.1).cuda()
    return dl.State(desc, S.to(torch.bfloat16) if desc.base_dtype == dl.BF16 else S)


@pytest.mark.parametrize("op", sorted(ref.OPS.values()))
@pytest.mark.parametrize("base", [dl.F32, dl.BF16])
def test_prefill_then_decode(op, base):
    """Prompts into slots (one continuing a state with pending log entries, one fresh over a poisoned slot, a padding row, a
    slot outside the pool, a row without tokens), then decode steps and a merge: the whole run against the recurrence."""
    H, Hq, dk, dv, cap = 4, 2, 64, 128, 8
    lens, slots = [70, 33, 20, 9, 0, 1], [5, 2, -1, 11, 0, 7]
    desc = make_desc(op, H, Hq, dk, dv, BF16, num_slots=9, cap=cap, base=base)
    state = pool(desc, 1)
    # a few decode steps leave entries in the logs of slots 5 and 0
    pre, _ = ref.inputs(op, [6], H, Hq, dk, dv, BF16, seed=50)
    only = torch.tensor([5, 0], dtype=torch.int32, device="cuda")
    start = state.S_base[[5, 0]].float()

    def rows(d, i):
        return {x: None if y is None else (y if x == "u_bonus" else y[i].contiguous()) for x, y in d.items()}

    bonus = pre["u_bonus"]
    steps = 3
    for s in range(steps):
        dl.decode_step(desc, state, **rows(pre, slice(2 * s, 2 * s + 2)), slot_idx=only)
    assert (state.log_len[5] == steps).all()
    state.S_base[2] = float("nan")
    state.K_log[2], state.U_log[2], state.decay_log[2] = float("nan"), float("nan"), float("nan")
    state.log_len[2] = 4
    keep = {i: state.S_base[i].clone() for i in (0, 1, 3, 4, 6, 8)}
    t, _ = ref.inputs(op, lens, H, Hq, dk, dv, BF16, seed=51)
    t["u_bonus"] = bonus
    fresh = torch.tensor([0, 1, 0, 0, 1, 1], dtype=torch.int32, device="cuda")
    plan = make_plan(lens, slots)
    out = torch.full((sum(lens), H, dv), 7.0, dtype=BF16, device="cuda")
    got = dl.prefill(desc, state, plan, **t, fresh=fresh, out=out)
    assert got is out and state.status.item() == dl.STATUS_BAD_SLOT
    at = np.cumsum([0] + lens)
    skipped = slice(at[2], at[4])
    assert (out[skipped] == 7.0).all()
    for i, S in keep.items():
        assert torch.equal(state.S_base[i], S), i
    assert state.log_len[0].tolist() == [steps] * H and not state.log_len[[5, 2, 7]].any()
    # the continuing slot: its three decoded tokens and the prompt in one go
    def joined(first, second, sl):
        return {x: None if y is None else (y if x == "u_bonus" else torch.cat((y[first], second[x][sl]))) for x, y in pre.items()}

    whole = joined(slice(0, 2 * steps, 2), t, slice(at[0], at[1]))
    want, S_want = ref.scan(op, desc.scale, [steps + lens[0]], whole["q"], whole["k"], whole["v"], whole["g"], whole["beta"], bonus, start[:1])
    # a 16-bit base is rounded when the pending entries are folded, and once more at the end: two half steps
    tol_state = TOL_F32 if base == dl.F32 else TOL_F32 + 2 * 2.0 ** -8
    assert err(out[at[0]:at[1]], want[steps:]) < TOL[BF16] + (0 if base == dl.F32 else 2.0 ** -8)
    assert err(state.S_base[5], S_want[0]) < tol_state
    zeros = torch.zeros_like(start[:1])
    for row in (1, 5):
        part = rows(t, slice(at[row], at[row + 1]))
        want, S_want = ref.scan(op, desc.scale, [lens[row]], part["q"], part["k"], part["v"], part["g"], part["beta"], bonus, zeros)
        assert err(out[at[row]:at[row + 1]], want) < TOL[BF16]
        assert err(state.S_base[slots[row]], S_want[0]) < (TOL_F32 if base == dl.F32 else TOL_F32 + 2.0 ** -8)
    # decode on from the prefilled state
    more, _ = ref.inputs(op, [5], H, Hq, dk, dv, BF16, seed=52)
    more["u_bonus"] = bonus
    S_from = state.S_base[5].float().clone()[None]
    one = torch.tensor([5], dtype=torch.int32, device="cuda")
    outs = [dl.decode_step(desc, state, **rows(more, slice(s, s + 1)), slot_idx=one) for s in range(5)]
    dl.merge(desc, state, one)
    want, S_want = ref.scan(op, desc.scale, [5], more["q"], more["k"], more["v"], more["g"], more["beta"], bonus, S_from)
    assert err(torch.cat(outs), want) < 2e-2 and err(state.S_base[5], S_want[0]) < (1e-4 if base == dl.F32 else 1e-4 + 2.0 ** -8)


def test_prefill_in_pieces():
    """A prompt in two calls leaves what it leaves in one (the pieces end inside a chunk, so only to rounding)."""
    op, H, dk = ref.KDA, 2, 128
    desc = make_desc(op, H, H, dk, dk, BF16, num_slots=2)
    t, _ = ref.inputs(op, [300], H, H, dk, dk, BF16, seed=60)
    one, two = pool(desc, 2), pool(desc, 2)
    out1 = dl.prefill(desc, one, make_plan([300], [1]), **t)
    parts = []
    for a, b in ((0, 101), (101, 300)):
        piece = {x: None if y is None else y[a:b].contiguous() for x, y in t.items()}
        parts.append(dl.prefill(desc, two, make_plan([b - a], [1]), **piece))
    assert err(torch.cat(parts), out1) < 2 * TOL[BF16] and err(two.S_base, one.S_base) < 2 * TOL_F32


def test_more_sequences_than_a_wave_and_every_cta_shape():
    """The chain kernels take 8, 4 or 2 warps per CTA by the number of units: the same bits from each."""
    op, H, dk = ref.GDN, 32, 128
    t, S0 = ref.inputs(op, [130], H, H, dk, dk, BF16, seed=61)
    desc = make_desc(op, H, H, dk, dk, BF16)
    base, S = dl.scan_forward(desc, make_plan([130]), **t, S_init=S0)
    for n in (3, 5, 11):
        big = {x: None if y is None else y.repeat(n, *[1] * (y.dim() - 1)) for x, y in t.items()}
        out, Sn = dl.scan_forward(desc, make_plan([130] * n), **big, S_init=S0.repeat(n, 1, 1, 1))
        assert torch.equal(out, base.repeat(n, 1, 1)) and torch.equal(Sn, S.repeat(n, 1, 1, 1))


def test_same_bits_again_and_on_another_stream():
    op, H, dk = ref.KDA, 4, 64
    lens = [130, 77]
    t, S0 = ref.inputs(op, lens, H, 2, dk, dk, BF16, seed=62)
    desc, plan = make_desc(op, H, 2, dk, dk, BF16), make_plan(lens)
    dout = torch.randn(t["v"].shape, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    first = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        second = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0)
    s.synchronize()
    for name in ("q", "k", "v", "g", "beta", "S_init"):
        assert torch.equal(getattr(first, name), getattr(second, name)), name


def test_autograd():
    op, H, dk = ref.GDN, 2, 64
    lens = [70, 3]
    t, S0 = ref.inputs(op, lens, H, 1, dk, dk, F32, seed=63)
    desc, plan = make_desc(op, H, 1, dk, dk, F32), make_plan(lens)
    leaf = {x: None if y is None else y.clone().requires_grad_() for x, y in t.items()}
    s0 = S0.clone().requires_grad_()
    out, S = dl.scan(desc, plan, **leaf, S_init=s0)
    ((out ** 2).sum() + S.sum()).backward()
    want = grads_of(op, desc.scale, lens, t, S0, 2 * out.detach(), torch.ones_like(S))
    for x in ("q", "k", "v", "g", "beta"):
        assert err(leaf[x].grad, want[x]) < TOL_F32 * 2, x     # dout itself comes from the fp32 output
    assert err(s0.grad, want["S_init"]) < TOL_F32 * 2
    # only v asks for a gradient; the state's output goes unused
    v = t["v"].clone().requires_grad_()
    out, _ = dl.scan(desc, plan, t["q"], t["k"], v, t["g"], t["beta"])
    out.sum().backward()
    assert v.grad is not None and torch.isfinite(v.grad).all()
    out, _ = dl.scan(desc, plan, t["q"], t["k"], v, t["g"], t["beta"])
    dl.build_plan(torch.tensor(lens, dtype=torch.int32, device="cuda"), plan)
    with pytest.raises(RuntimeError, match="rebuilt"):
        out.sum().backward()


def plan_reference(lens, slots, log_len, cap, decode_rows, max_tokens):
    starts, chunks, token_seq, chunk_seq, eff = [0], [0], [], [], []
    full = False
    for i, n in enumerate(lens):
        n = max(int(n), 0)
        if n and (full or starts[-1] + n > max_tokens):
            full, n = True, 0
        eff.append(n)
        token_seq += [i] * n
        chunk_seq += [i] * ((n + 63) // 64)
        starts.append(starts[-1] + n)
        chunks.append(chunks[-1] + (n + 63) // 64)
    scan, app, mrg = [], [], []
    for i, n in enumerate(eff):
        s = slots[i] if slots is not None else i
        one = decode_rows and n == 1
        done = one and log_len is not None and 0 <= s < len(log_len) and log_len[s] >= cap
        scan.append(s if n > 0 and not one else -1)
        app.append(s if one and not done else -1)
        mrg.append(s if one and done else -1)
    token_seq += [-1] * (max_tokens - len(token_seq))
    chunk_seq += [-1] * (max_tokens // 64 + len(lens) - len(chunk_seq))
    dec = sum(1 for n in eff if decode_rows and n == 1)
    return dict(starts=starts, chunk_starts=chunks, token_seq=token_seq, chunk_seq=chunk_seq, scan_slots=scan, append_slots=app, merge_slots=mrg,
                totals=[starts[-1], chunks[-1], sum(1 for n in eff if n) - dec, dec])


def check_plan(plan, want):
    for name, w in want.items():
        x = getattr(plan, name)
        if x is None:
            assert not w
            continue
        assert x.cpu().tolist() == w, name


@pytest.mark.parametrize("n,hi,most", [(0, 1, 10), (1, 1, 1), (1, 70, 70), (7, 130, 1000), (513, 5, 900), (600, 300, 20000), (5000, 9, 40003),
                                       (24576, 3, 50000), (24577, 3, 50000), (40000, 4, 30000)])
@pytest.mark.parametrize("decode_rows", [False, True])
def test_plan(n, hi, most, decode_rows):
    """Row counts around the thread and shared-memory limits; budgets that the rows do and do not fit into."""
    rng = np.random.default_rng(n + hi)
    lens = rng.integers(-2, hi + 1, n)
    num_slots = n + 3
    slots = rng.permutation(num_slots + 4)[:n] - 2          # some negative, some outside the pool
    log = rng.integers(0, 9, (num_slots, 2)).astype(np.int32)
    plan = dl.Plan(n, most, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    dl.build_plan(torch.tensor(lens, **i32), plan, slots=torch.tensor(slots, **i32), log_len=torch.tensor(log, **i32), cap=6, decode_rows=decode_rows)
    check_plan(plan, plan_reference(lens, slots.tolist(), log[:, 0].tolist(), 6, decode_rows, most))
    bare = dl.Plan(n, most, device="cuda", token_map=False)
    dl.build_plan(torch.tensor(lens, **i32), bare, decode_rows=decode_rows)
    want = plan_reference(lens, None, None, 0, decode_rows, most)
    want.pop("token_seq")
    check_plan(bare, want)


def test_plan_lengths_that_pass_32_bits():
    """The lengths' sum passes 2^31 and 2^32; what fits is planned, the rest is dropped."""
    big = 2 ** 31 - 1
    lens = [3, big, big, big, 2, 0, 1]
    plan = make_plan([0] * 7, tail=100)
    dl.build_plan(torch.tensor(lens, dtype=torch.int32, device="cuda"), plan)
    check_plan(plan, plan_reference(lens, None, None, 0, False, 100))


def test_step_of_a_serving_loop_captured_once():
    """Plan, prefill and the two decode calls of a mixed batch in one graph; every replay takes new lengths and tokens.  The
    rows' results equal those of the same calls made one by one."""
    op, H, dk, cap, n, most = ref.GDN, 2, 64, 2, 6, 200
    desc = make_desc(op, H, H, dk, dk, BF16, num_slots=n, cap=cap)
    ws = dl.scan_workspace(desc, n, most)
    plan = dl.Plan(n, most, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    lens, slots = torch.zeros(n, **i32), torch.arange(n, **i32)
    t, _ = ref.inputs(op, [most], H, H, dk, dk, BF16, seed=70)
    dec, _ = ref.inputs(op, [n], H, H, dk, dk, BF16, seed=71)
    out, out_d = torch.zeros(most, H, dk, dtype=BF16, device="cuda"), torch.zeros(n, H, dk, dtype=BF16, device="cuda")

    def step(state):
        dl.build_plan(lens, plan, slots=slots, log_len=state.log_len, cap=cap, decode_rows=True)
        dl.prefill(desc, state, plan, **t, out=out, workspace=ws)
        dl.decode_merge_step(desc, state, **dec, slot_idx=plan.merge_slots, out=out_d)
        dl.decode_step(desc, state, **dec, slot_idx=plan.append_slots, out=out_d)

    graphed, eager = pool(desc, 3), pool(desc, 3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(pool(desc, 4))
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    seen = [False, False]
    for i, ln in enumerate(([64, 1, 1, 0, 30, 1], [1, 1, 1, 90, 1, 1], [1] * 6, [1, 1, 1, 0, 1, 1], [2, 1, 1, 1, 1, 190], [1] * 6)):
        lens.copy_(torch.tensor(ln, **i32))
        gen = torch.Generator().manual_seed(80 + i)
        t["v"].copy_(torch.randn(t["v"].shape, generator=gen))
        dec["v"].copy_(torch.randn(dec["v"].shape, generator=gen))
        out.zero_(), out_d.zero_()
        graph.replay()
        a, b = out.clone(), out_d.clone()
        out.zero_(), out_d.zero_()
        step(eager)
        assert torch.equal(a, out) and torch.equal(b, out_d), i
        assert torch.equal(graphed.S_base, eager.S_base) and torch.equal(graphed.log_len, eager.log_len), i
        seen = [seen[0] or bool(a.any()), seen[1] or bool(b.any())]
    assert eager.status.item() == 0 and all(seen)


def test_training_step_captured():
    op, H, dk = ref.GLA, 2, 64
    lens = [70, 129]
    t, S0 = ref.inputs(op, lens, H, 1, dk, dk, BF16, seed=72)
    desc, plan = make_desc(op, H, 1, dk, dk, BF16), make_plan(lens)
    ws = dl.scan_workspace(desc, 2, sum(lens), train=True)
    dout = torch.randn(t["v"].shape, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()

    def step():
        o, _ = dl.scan_forward(desc, plan, **t, S_init=S0, workspace=ws, save=True)
        return o, dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, workspace=ws, saved=True)

    want = step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    graph.replay()
    assert torch.equal(got[0], want[0]) and all(torch.equal(getattr(got[1], x), getattr(want[1], x)) for x in ("q", "k", "v", "g", "S_init"))


def test_offsets_beyond_32_bits():
    """Token tensors of more than 2^31 elements: the last head of the last tokens equals the same head run alone (to rounding:
    one head alone is cut into segments)."""
    op, H, dk, T = ref.RETNET, 160, 128, 110_000
    assert T * H * dk > 2 ** 31
    gen = torch.Generator("cuda").manual_seed(1)

    def rand(*shape):
        return torch.empty(*shape, dtype=BF16, device="cuda").normal_(generator=gen)

    q, k, v = rand(T, 1, dk) * 0.1, rand(T, 1, dk) * 0.1, rand(T, H, dk)
    g = torch.full((T, H), -0.05, device="cuda")
    plan = make_plan([T])
    out, S = dl.scan_forward(make_desc(op, H, 1, dk, dk, BF16), plan, q, k, v, g)
    one, S1 = dl.scan_forward(make_desc(op, 1, 1, dk, dk, BF16), plan, q, k, v[:, -1:].contiguous(), g[:, -1:].contiguous())
    assert err(out[-4096:, -1:], one[-4096:]) < 2 * TOL[BF16] and err(S[:, -1:], S1) < 2 * TOL_F32


def test_launches_are_the_librarys():
    before = dl.launch_count()
    t, S0 = ref.inputs(ref.GDN, [10], 2, 2, 64, 64, BF16)
    dl.scan_forward(make_desc(ref.GDN, 2, 2, 64, 64, BF16), make_plan([10]), **t)
    assert dl.launch_count() == before + 3   # plan, per-chunk matrices, chain


def test_status_of_a_bad_slot_only():
    desc = make_desc(ref.GDN, 2, 2, 64, 64, BF16, num_slots=2)
    state = pool(desc, 5)
    t, _ = ref.inputs(ref.GDN, [5, 5], 2, 2, 64, 64, BF16)
    before = state.S_base.clone()
    dl.prefill(desc, state, make_plan([5, 5], [2, -3]), **t)
    assert state.status.item() == binding.STATUS_BAD_SLOT and torch.equal(state.S_base, before)


@pytest.mark.parametrize("op", [ref.GDN, ref.KDA, ref.RWKV6])
def test_bits_do_not_depend_on_what_the_memory_held(op):
    """More units than the device holds at once, again and again over workspaces and outputs full of other patterns."""
    H, dk, lens = 32, 128, [300, 64, 7, 1, 190, 90, 129, 65]
    t, S0 = ref.inputs(op, lens, H, H, dk, dk, BF16, seed=op + 90)
    desc, plan = make_desc(op, H, H, dk, dk, BF16), make_plan(lens)
    ws = dl.scan_workspace(desc, len(lens), plan.max_tokens, train=True)
    dout = torch.randn(t["v"].shape, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    first = None
    for i in range(8):
        ws.random_(generator=torch.Generator("cuda").manual_seed(i))
        out = torch.full_like(t["v"], float("nan"))
        out, S = dl.scan_forward(desc, plan, **t, S_init=S0, out=out, workspace=ws, save=True)
        d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, workspace=ws, saved=True)
        got = [out, S, d.q, d.k, d.v, d.g, d.S_init]
        first = first or got
        assert all(torch.equal(x, y) for x, y in zip(first, got)), i
    assert all(torch.isfinite(x).all() for x in first) and plan.status.item() == 0


def stream_of_memory(t):
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]


def test_buffers_belong_to_the_stream_asked_for():
    """A call on another stream than the current one: its results' memory is that stream's, so that no work queued on the
    current one, in front or behind, shares it; the same for its workspace, which is free again when the call returns."""
    op, H, dk, lens = ref.GDN, 2, 64, [70, 9]
    t, S0 = ref.inputs(op, lens, H, 2, dk, dk, BF16, seed=64)
    desc, plan = make_desc(op, H, 2, dk, dk, BF16, num_slots=2), make_plan(lens)
    dout, state = torch.ones_like(t["v"]), pool(desc, 6)
    want, S_want = dl.scan_forward(desc, plan, **t, S_init=S0)
    torch.cuda.synchronize()
    for stream in (torch.cuda.Stream(), torch.cuda.Stream().cuda_stream):
        handle = stream if isinstance(stream, int) else stream.cuda_stream
        out, S = dl.scan_forward(desc, plan, **t, S_init=S0, stream=stream)
        d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, stream=stream)
        served = dl.prefill(desc, state, plan, **t, stream=stream)
        torch.cuda.synchronize()
        dl.build_plan(torch.tensor(lens, dtype=torch.int32, device="cuda"), plan, stream=0)
        torch.cuda.synchronize()
        assert torch.cuda.current_stream() == torch.cuda.default_stream()
        assert {stream_of_memory(x) for x in (out, S, d.q, d.k, d.v, d.g, d.beta, d.S_init, served)} == {handle}
        assert torch.equal(out, want) and torch.equal(S, S_want)


@pytest.mark.parametrize("dk,op", [(128, ref.GDN), (64, ref.RWKV6)])
def test_early_decode_steps_behind_a_prefill(dk, op):
    """Decode steps that may start ahead of the kernel in front: the second one, on the prefilled state, keeps its promise (the
    first one writes another state) and must still see the bases that the prefill writes."""
    H, lens = 32, [1900, 30, 64, 500]
    t, _ = ref.inputs(op, lens, H, H, dk, dk, BF16, seed=65)
    desc = make_desc(op, H, H, dk, dk, BF16, num_slots=4)
    early = make_desc(op, H, H, dk, dk, BF16, num_slots=4)
    early.hints = dl.HINT_BASE_UNTOUCHED | dl.HINT_SLOTS_STABLE
    plan = make_plan(lens)
    step, _ = ref.inputs(op, [4], H, H, dk, dk, BF16, seed=66)
    ws = dl.scan_workspace(desc, 4, sum(lens))
    results = []
    for hinted in (False, True, True, True):
        a, b = pool(desc, 7), pool(desc, 8)
        torch.cuda.synchronize()
        dl.prefill(desc, a, plan, **t, workspace=ws)
        for state in (b, a):
            if not hinted:
                torch.cuda.synchronize()
            got = dl.decode_step(early if hinted else desc, state, **step)
        results.append((got, a.S_base.clone(), b.K_log.clone()))
    for r in results[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, results[0]))


def test_captured_autograd():
    """Forward and backward of the differentiable scan in one graph, replayed over changed inputs."""
    op, H, dk, lens = ref.KDA, 2, 64, [70, 129, 1]
    t, S0 = ref.inputs(op, lens, H, 1, dk, dk, F32, seed=67)
    other, _ = ref.inputs(op, lens, H, 1, dk, dk, F32, seed=68)
    desc, plan = make_desc(op, H, 1, dk, dk, F32), make_plan(lens)
    names = [x for x, y in t.items() if y is not None]
    fixed = {x: y.clone().requires_grad_() if y is not None else None for x, y in t.items()}

    def grads(leaf):
        out, S = dl.scan(desc, plan, **leaf, S_init=S0)
        return [out, *torch.autograd.grad((out ** 2).sum() + S.sum(), [leaf[x] for x in names])]

    kept = dl.scan(desc, plan, **fixed, S_init=S0)      # an eager graph of the same leaves
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="same leaves"):
        with torch.cuda.graph(graph):
            grads(fixed)
    del kept
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        grads(fixed)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = grads(fixed)
    for values in (t, other, t):
        with torch.no_grad():
            for x in names:
                fixed[x].copy_(values[x])
        graph.replay()
        torch.cuda.synchronize()
        want = grads({x: None if y is None else y.clone().requires_grad_() for x, y in values.items()})
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    with torch.no_grad():
        out, _ = dl.scan(desc, plan, **fixed, S_init=S0)
    assert not out.requires_grad and torch.equal(out, got[0])


# A row that is cut into s segments passes s - 2 joins, each a contraction over 128 channels more: 128 additions of at most one
# unit 2^-23 of the largest partial sum.
def tol_joined(segments):
    return TOL_F32 + max(0, segments - 2) * 128 * 2.0 ** -23


SPLIT_LENS = [1900, 3, 0, 1100, 512, 1537]   # with 6 rows of one head up to 13 segments of 8 chunks: 3, 1, 1, 1 (17 chunks), 1, 3


@pytest.mark.parametrize("op", sorted(ref.OPS.values()))
@pytest.mark.parametrize("io,dk", [(BF16, 128), (F32, 128), (BF16, 64), (F32, 64)])
def test_rows_cut_into_segments(op, io, dk):
    H, dv = 1, 128
    t, S0 = ref.inputs(op, SPLIT_LENS, H, H, dk, dv, io, seed=op + 110, tail=3)
    desc, plan = make_desc(op, H, H, dk, dv, io), make_plan(SPLIT_LENS, tail=3)
    want, S_want = ref.scan(op, desc.scale, SPLIT_LENS, t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], S0)
    out = torch.full(t["v"].shape, 7.0, dtype=io, device="cuda")
    out, S = dl.scan_forward(desc, plan, **t, S_init=S0, out=out)
    at = np.cumsum([0] + SPLIT_LENS)
    more = tol_joined(3) - TOL_F32
    for i, n in enumerate(SPLIT_LENS):   # row by row: a row's error is measured against its own size
        assert err(out[at[i]:at[i + 1]], want[at[i]:at[i + 1]]) < TOL[io] + more, i
        assert err(S[i], S_want[i]) < TOL_F32 + more, i
    assert (out[at[-1]:] == 7.0).all()
    again, S2 = dl.scan_forward(desc, plan, **t, S_init=S0)
    assert torch.equal(again[:at[-1]], out[:at[-1]]) and torch.equal(S, S2) and plan.status.item() == 0


@pytest.mark.parametrize("op", [ref.GDN, ref.KDA, ref.GLA])
@pytest.mark.parametrize("gates", ["as drawn", "none", "mixed"])
def test_one_long_row_in_many_segments(op, gates):
    """4100 tokens, 65 chunks, 8 segments; gates that are drawn, absent (nothing is forgotten) or strong and reset by turns."""
    lens, H, dk = [4100], 2, 128
    t, S0 = ref.inputs(op, lens, H, 1, dk, dk, F32, seed=op + 120)
    gen = torch.Generator().manual_seed(7)
    pick = torch.rand(t["g"].shape, generator=gen).cuda()
    if gates == "none":
        t["g"] = torch.zeros_like(t["g"])
    elif gates == "mixed":
        t["g"] = torch.where(pick < 0.01, -torch.inf, torch.where(pick < 0.1, -50.0, torch.where(pick < 0.5, 0.0, t["g"]))).contiguous()
    desc, plan = make_desc(op, H, 1, dk, dk, F32), make_plan(lens)
    want, S_want = ref.scan(op, desc.scale, lens, t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], S0)
    out, S = dl.scan_forward(desc, plan, **t, S_init=S0)
    assert err(out, want) < tol_joined(8) and err(S, S_want) < tol_joined(8)


@pytest.mark.parametrize("op,io", [(ref.GDN, BF16), (ref.KDA, F32), (ref.RETNET, BF16)])
def test_gradients_of_rows_cut_into_segments(op, io):
    lens, H, dk = [1600, 70], 1, 128
    t, S0 = ref.inputs(op, lens, H, H, dk, dk, io, seed=op + 130)
    desc, plan = make_desc(op, H, H, dk, dk, io), make_plan(lens)
    gen = torch.Generator().manual_seed(8)
    dout, dS = torch.randn(t["v"].shape, generator=gen).to(io).cuda(), torch.randn(S0.shape, generator=gen).cuda() * 0.1
    ws = dl.scan_workspace(desc, len(lens), plan.max_tokens, train=True)
    ws.random_(generator=torch.Generator("cuda").manual_seed(1))
    dl.scan_forward(desc, plan, **t, S_init=S0, workspace=ws, save=True)
    d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, dS_final=dS, workspace=ws, saved=True)
    for name, w in grads_of(op, desc.scale, lens, t, S0, dout, dS).items():
        tol = TOL[io] if name in ("q", "k", "v") else TOL_F32
        assert err(getattr(d, name), w) < tol + tol_joined(3) - TOL_F32, name


@pytest.mark.parametrize("base", [dl.F32, dl.BF16])
def test_prefill_of_rows_cut_into_segments(base):
    """Slots of the pool: a row that continues, one that starts afresh over a poisoned slot, padding, one outside the pool."""
    op, H, dk = ref.GDN, 2, 128
    lens, slots = [1700, 1600, 1540, 1540, 9], [3, 0, -1, 17, 2]
    desc = make_desc(op, H, 1, dk, dk, BF16, num_slots=5, base=base)
    state = pool(desc, 9)
    start = state.S_base.float().clone()
    keep = state.S_base[[1, 4]].clone()
    state.S_base[0] = float("nan")
    state.log_len[0] = 2
    t, _ = ref.inputs(op, lens, H, 1, dk, dk, BF16, seed=140)
    out = torch.full(t["v"].shape, 7.0, dtype=BF16, device="cuda")
    fresh = torch.tensor([0, 1, 1, 1, 0], dtype=torch.int32, device="cuda")
    dl.prefill(desc, state, make_plan(lens, slots), **t, fresh=fresh, out=out)
    at = np.cumsum([0] + lens)
    assert state.status.item() == dl.STATUS_BAD_SLOT and (out[at[2]:at[4]] == 7.0).all()
    assert torch.equal(state.S_base[[1, 4]], keep) and not state.log_len.any()
    more = tol_joined(3) - TOL_F32
    for row, S0 in ((0, start[3]), (1, torch.zeros_like(start[0])), (4, start[2])):
        part = {x: None if y is None else y[at[row]:at[row + 1]].contiguous() for x, y in t.items()}
        want, S_want = ref.scan(op, desc.scale, [lens[row]], part["q"], part["k"], part["v"], part["g"], part["beta"], None, S0[None])
        assert err(out[at[row]:at[row + 1]], want) < TOL[BF16] + more
        assert err(state.S_base[slots[row]], S_want[0]) < TOL_F32 + more + (0 if base == dl.F32 else 2.0 ** -8)
