"""Sequence operators where a call's documentation allows more than its everyday use: output rows that nothing writes, gates inside
a block of tokens, gradients that arrive off a 16-byte boundary, capture beside live graphs, and the kernel variants that
only some shapes take.

Tolerances as in ``test_gpu_scan``, whose helpers are used: 256 units 2^-23 for a sum in fp32, half a step more for a bf16 result.
"""
import numpy as np
import pytest
import torch

import paper_2608_15533_b200 as dl
import scan_reference as ref
from test_gpu_scan import BF16, F32, TOL, TOL_F32, check_grads, err, grads_of, make_desc, make_plan, pool

pytestmark = pytest.mark.gpu


def poison(shape, dtype):
    """Memory of this size full of NaN goes back to the allocator, so that the next tensor of the size finds it."""
    x = torch.full(shape, float("nan"), dtype=dtype, device="cuda")
    torch.cuda.synchronize()
    del x


@pytest.mark.parametrize("op,io,H,Hq,dk,dv", [(ref.GDN, BF16, 4, 2, 128, 128), (ref.KDA, F32, 1, 1, 64, 128), (ref.RWKV6, BF16, 2, 2, 64, 64),
                                              (ref.RETNET, F32, 3, 1, 128, 64)])
@pytest.mark.parametrize("tail", [0, 5, 700])
def test_rows_of_a_new_output_that_nothing_writes_are_zero(op, io, H, Hq, dk, dv, tail):
    """A mixed step: prompts, rows that decode, padding, a slot outside the pool, no tokens, rows dropped by the plan, and more
    rows in the tensors than the plan reaches.  What the call writes is what it writes into the caller's tensor."""
    lens, slots = [70, 1, 0, 130, 1, 64, 200, 1, 3], [4, 0, 1, -1, 2, 3, 99, 5, 6]
    rows = sum(lens) + tail + 3
    desc = make_desc(op, H, Hq, dk, dv, io, num_slots=8)
    t, _ = ref.inputs(op, lens, H, Hq, dk, dv, io, seed=op + 200, tail=tail + 3)
    at = np.cumsum([0] + lens)
    for decode_rows, most in ((True, sum(lens) + tail), (False, sum(lens) + tail), (True, int(at[6]) + 30)):
        plan = dl.Plan(len(lens), most, device="cuda")
        i32 = dict(dtype=torch.int32, device="cuda")
        dl.build_plan(torch.tensor(lens, **i32), plan, slots=torch.tensor(slots, **i32), decode_rows=decode_rows)
        runs = [i for i, s in enumerate(plan.scan_slots.tolist()) if 0 <= s < 8]
        own = torch.full(t["v"].shape, 7.0, dtype=io, device="cuda")
        dl.prefill(desc, pool(desc, 1), plan, **t, out=own)
        poison(t["v"].shape, io)
        got = dl.prefill(desc, pool(desc, 1), plan, **t)
        written = torch.zeros(rows, dtype=torch.bool)
        for i in runs:
            written[at[i]:at[i + 1]] = True
        assert runs and torch.equal(got[written], own[written])
        assert not got[~written].any() and (own[~written] == 7.0).all()
    # the scan without a pool: every row runs, the tail is zero
    plan = make_plan(lens, tail=tail)
    own, S = dl.scan_forward(desc, plan, **t, out=torch.full(t["v"].shape, 7.0, dtype=io, device="cuda"))
    leaf = {x: None if y is None else y.clone().requires_grad_() for x, y in t.items()}
    for call in (lambda: dl.scan_forward(desc, plan, **t), lambda: dl.scan(desc, plan, **t), lambda: dl.scan(desc, plan, **leaf)):
        poison(t["v"].shape, io)
        out, S_again = call()
        assert torch.equal(out[:at[-1]], own[:at[-1]]) and torch.equal(S, S_again) and not out[at[-1]:].any()
    assert (own[at[-1]:] == 7.0).all()


def test_new_outputs_without_rows_or_tokens_are_zero():
    op, H, d = ref.GDN, 2, 64
    t, _ = ref.inputs(op, [], H, H, d, d, BF16, tail=9)
    desc = make_desc(op, H, H, d, d, BF16, num_slots=3)
    for lens, most in (([], 9), ([0, 0], 9), ([0, 0], 0), ([], 0)):
        plan = dl.Plan(len(lens), most, device="cuda")
        dl.build_plan(torch.tensor(lens, dtype=torch.int32, device="cuda"), plan)
        for call in (lambda: dl.prefill(desc, pool(desc, 1), plan, **t), lambda: dl.scan_forward(desc, plan, **t)[0]):
            poison(t["v"].shape, BF16)
            assert not call().any()


# Weights of pairs inside a block of 16 tokens.  A pair's weight is the product of the gates' exponentials between its tokens, made
# of the block's prefix and suffix products and the reciprocal of the whole: up to 15 exponentials of the pair, two units 2^-23
# each, 16 products of half a unit in the prefix, in the suffix and in the whole, three half units joining them and q, k: 30
# + 24 + 1.5 units.  The matrix product adds eight: one per sum of the six plane products, one for the others' zeros, one for scale.
TOL_PAIR = 64 * 2.0 ** -23


def relative(x, want):
    x, want = x.double().cpu(), want.double().cpu()
    live = want != 0
    assert x.shape == want.shape and not x[~live].any()
    return ((x - want).abs()[live] / want.abs()[live]).max().item()


@pytest.mark.parametrize("op", [ref.GLA, ref.RWKV6, ref.KDA])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128)])
@pytest.mark.parametrize("depth", [1.0, 20.0, 40.0, 59.0])
def test_weights_of_pairs_inside_a_block(op, dk, dv, depth):
    """Every pair's weight by itself: one channel is live in each run, v_j is the j-th unit vector, so that out_ij is the weight
    of pair (i, j); for the gradients one token's k (or q) is live, so that dq (dk) is the weight of one pair per channel."""
    T, H = 16, 1
    gen = torch.Generator().manual_seed(int(depth) + dk)
    g = -torch.rand(T, H, dk, generator=gen, dtype=torch.float64) - 0.05
    g = (g * (depth / -g.sum(0).min())).float()                     # the deepest channel's block decays by e^-depth
    G = g.double().cumsum(0)[:, 0]
    before = G - g[:, 0].double() if op == ref.RWKV6 else G         # what a readout sees
    low = torch.ones(T, T, dtype=torch.bool).tril(-1 if op == ref.RWKV6 else 0)
    desc, plan = make_desc(op, H, H, dk, dv, F32, scale=1.0), make_plan([T])
    ones = torch.ones(T, H, dk)
    more = dict(beta=torch.ones(T, H).cuda() if op == ref.KDA else None, u_bonus=torch.zeros(H, dk).cuda() if op == ref.RWKV6 else None)
    v = torch.eye(T, dv)[:, None].contiguous()
    S0 = torch.zeros(1, H, dk, dv, device="cuda")

    def weights(c):
        return torch.exp(before[:, None, c] - G[None, :, c]).masked_fill(~low, 0.0)

    if op != ref.KDA:       # the delta rule's outputs mix the pairs; its gradients' weights are looked at below
        for c in (0, 1, dk // 2 + 3, dk - 1):
            one = torch.zeros(T, H, dk)
            one[..., c] = 1.0
            out, _ = dl.scan_forward(desc, plan, one.cuda(), one.cuda(), v.cuda(), g.cuda(), **more, S_init=S0)
            assert relative(out[:, 0, :T], weights(c)) < TOL_PAIR
    # one live token: with k = 0 but for token j the delta rule has nothing to remove, and u_j = v_j
    for j in (0, 5, 14):
        k = torch.zeros(T, H, dk)
        k[j] = 1.0
        dout = torch.zeros(T, H, dv)
        dout[:, 0, j] = 1.0
        d = dl.scan_backward(desc, plan, ones.cuda(), k.cuda(), v.cuda(), g.cuda(), more["beta"], more["u_bonus"], dout.cuda(), S_init=S0)
        want = torch.exp(before - G[j]) * low[:, j, None]
        assert relative(d.q[:, 0], want) < TOL_PAIR
    # with q = 0 but for token i, dk_j is the weight of (i, j) (RWKV6, GLA)
    if op != ref.KDA:
        for i in (15, 7):
            q = torch.zeros(T, H, dk)
            q[i] = 1.0
            dout = torch.zeros(T, H, dv)
            dout[i, 0] = 1.0
            vv = torch.zeros(T, H, dv)
            vv[:, 0, 0] = 1.0
            d = dl.scan_backward(desc, plan, q.cuda(), ones.cuda(), vv.cuda(), g.cuda(), None, more["u_bonus"], dout.cuda(), S_init=S0)
            assert relative(d.k[:, 0], torch.exp(before[i] - G) * low[i, :, None]) < TOL_PAIR


@pytest.mark.parametrize("op,io,d", [(ref.GDN, BF16, 128), (ref.RWKV6, BF16, 64), (ref.GLA, F32, 64)])
def test_gradients_that_arrive_off_a_16_byte_boundary(op, io, d):
    """Flattened outputs joined behind a single number: their gradients are contiguous views that start in between."""
    H, lens = 2, [70, 9]
    t, S0 = ref.inputs(op, lens, H, H, d, d, io, seed=op + 210)
    desc, plan = make_desc(op, H, H, d, d, io), make_plan(lens)
    names = [x for x, y in t.items() if y is not None]
    gen = torch.Generator().manual_seed(2)
    w_out, w_S = torch.randn(t["v"].numel(), generator=gen).to(io).cuda(), torch.randn(S0.numel(), generator=gen).cuda()

    def grads(offset):
        leaf = {x: None if y is None else y.clone().requires_grad_() for x, y in t.items()}
        out, S = dl.scan(desc, plan, **leaf, S_init=S0)
        front = torch.zeros(offset, dtype=io, device="cuda"), torch.zeros(offset, device="cuda")
        loss = (torch.cat((front[0], out.flatten()))[offset:] * w_out).sum() + (torch.cat((front[1], S.flatten()))[offset:] * w_S).sum()
        return torch.autograd.grad(loss, [leaf[x] for x in names])

    for x, y in zip(grads(1), grads(0)):
        assert torch.equal(x, y)


def test_capture_of_a_layer_beside_an_eager_graph_of_its_weights():
    """q, k and v are computed from weights, which are the leaves: refused while an eager graph of them lives, fine afterwards."""
    op, H, d, lens = ref.RETNET, 2, 64, [40, 9]
    T = sum(lens)
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(T, 32, generator=gen).cuda()
    w = {n: (torch.randn(32, H * d, generator=gen) * 0.1).cuda().requires_grad_() for n in "qkv"}
    g = torch.full((T, H), -0.05, device="cuda")
    desc, plan = make_desc(op, H, H, d, d, F32), make_plan(lens)

    def layer():
        out, S = dl.scan(desc, plan, *(torch.matmul(x, w[n]).view(T, H, d) for n in "qkv"), g)
        return [out, *torch.autograd.grad((out ** 2).sum() + S.sum(), list(w.values()))]

    def forward():
        return dl.scan(desc, plan, *(torch.matmul(x, w[n]).view(T, H, d) for n in "qkv"), g)

    kept = forward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="same leaves"):
        with torch.cuda.graph(graph):
            forward()
    del kept
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer()
    x.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, layer()):
        assert torch.equal(a, b)


# bf16 tensors with d_v = 128: the gradients' products over d_v take states, U and dV as two bf16 planes, each off by at most 2^-18 of
# its value.  A sum of 128 products of random sign is about 1 / sqrt(128) of the sum of their sizes, so a gate's or beta's
# gradient is off by 2 * 2^-18 * sqrt(128) of itself on top of the fp32 sums.
TOL_TWO_PLANES = TOL_F32 + 128 ** 0.5 * 2.0 ** -17


def check_all(op, io, lens, H, Hq, dk, dv, t, S0, seed, saved=True):
    """Forward and every gradient of one batch against the fp64 recurrence."""
    desc, plan = make_desc(op, H, Hq, dk, dv, io), make_plan(lens)
    gen = torch.Generator().manual_seed(seed)
    dout, dS = torch.randn(t["v"].shape, generator=gen).to(io).cuda(), torch.randn(S0.shape, generator=gen).cuda() * 0.1
    want, S_want = ref.scan(op, desc.scale, lens, t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], S0)
    ws = dl.scan_workspace(desc, len(lens), plan.max_tokens, train=True)
    out, S = dl.scan_forward(desc, plan, **t, S_init=S0, workspace=ws, save=True)
    assert err(out, want) < TOL[io] and err(S, S_want) < TOL_F32
    d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, dS_final=dS, workspace=ws, saved=True)
    two = io == BF16 and dv == 128
    for name, w in grads_of(op, desc.scale, lens, t, S0, dout, dS).items():
        tol = TOL[io] if name in ("q", "k", "v") else TOL_TWO_PLANES if two and name in ("g", "beta", "u_bonus") else TOL_F32
        assert err(getattr(d, name), w) < tol, name
    served, S = dl.scan_forward(desc, plan, **t, S_init=S0)      # serving's kernels, which keep nothing
    assert err(served, want) < TOL[io] and err(S, S_want) < TOL_F32
    assert plan.status.item() == 0


@pytest.mark.parametrize("op", sorted(ref.OPS.values()))
@pytest.mark.parametrize("io,H,Hq,dk,dv", [(BF16, 2, 2, 64, 64), (BF16, 4, 2, 128, 64), (F32, 2, 1, 64, 128)])
def test_forward_and_gradients_of_the_other_shapes(op, io, H, Hq, dk, dv):
    lens = [17, 0, 1, 64, 2, 129, 63, 16, 200]
    t, S0 = ref.inputs(op, lens, H, Hq, dk, dv, io, seed=op + 220)
    check_all(op, io, lens, H, Hq, dk, dv, t, S0, 11)


SHAPES = [(BF16, 128, 128), (BF16, 64, 128), (F32, 128, 128), (BF16, 128, 64)]


@pytest.mark.parametrize("op", [ref.GDN, ref.RETNET, ref.KDA, ref.RWKV6, ref.GLA])
@pytest.mark.parametrize("gates", ["none", "slow", "strong", "reset", "mixed", "some channels"])
@pytest.mark.parametrize("io,dk,dv", SHAPES)
def test_gates_of_every_strength(op, gates, io, dk, dv):
    """No decay, that of trained layers (-0.001 to -0.1), gates that empty the state within a block, resets, all by turns; and, per
    channel, a tenth of the channels that forget fast beside ordinary ones."""
    lens, H = [150, 40], 2
    t, S0 = ref.inputs(op, lens, H, 1, dk, dv, io, seed=op + 230)
    g = t["g"]
    gen = torch.Generator().manual_seed(5)
    pick = torch.rand(g.shape, generator=gen).cuda()
    if gates == "none":
        g = torch.zeros_like(g)
    elif gates == "slow":
        g = -0.001 - 0.099 * pick
    elif gates == "strong":
        g = g * 40 - 3
    elif gates == "reset":
        g = torch.where(pick < 0.1, -torch.inf, g)
    elif gates == "mixed":
        g = torch.where(pick < 0.05, -torch.inf, torch.where(pick < 0.2, -50.0, torch.where(pick < 0.5, 0.0, g)))
    else:
        g = torch.where(torch.arange(g.shape[-1], device="cuda") % 10 == 3, g - 5.0, g)
    t["g"] = g.contiguous()
    check_all(op, io, lens, H, 1, dk, dv, t, S0, 12)


@pytest.mark.parametrize("op", [ref.GDN, ref.KDA])
@pytest.mark.parametrize("case", ["beta0", "beta1", "same_key", "tiny_beta", "all_beta0"])
@pytest.mark.parametrize("io,dk,dv", SHAPES)
def test_delta_rule_at_its_edges(op, case, io, dk, dv):
    lens, H = [100, 7], 2
    t, S0 = ref.inputs(op, lens, H, H, dk, dv, io, seed=op + 240)
    if case == "beta0":
        t["beta"][::2] = 0.0
    elif case == "all_beta0":
        t["beta"].zero_()
    elif case == "beta1":
        t["beta"].fill_(1.0)
    elif case == "tiny_beta":
        t["beta"][::3] = 1e-25
    else:
        t["k"] = t["k"][:1].expand_as(t["k"]).contiguous()
        t["beta"].fill_(1.0)
        t["g"] = t["g"] * 0.01
    check_all(op, io, lens, H, H, dk, dv, t, S0, 13)


@pytest.mark.parametrize("op,io,dk", [(ref.GDN, BF16, 64), (ref.GDN, F32, 128), (ref.KDA, BF16, 128), (ref.RWKV6, BF16, 64), (ref.GLA, F32, 64)])
def test_head_size_64_on_both_sides_of_a_wave(op, io, dk):
    """The chain kernels for d_v = 64 take two warps per CTA while the units do not fill the device, four beyond: the same bits, forward and
    backward, and those of the recurrence."""
    H, dv, n0 = 32, 64, 130
    t, S0 = ref.inputs(op, [n0], H, H, dk, dv, io, seed=op + 250)
    desc = make_desc(op, H, H, dk, dv, io)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    gen = torch.Generator().manual_seed(14)
    dout, dS = torch.randn(t["v"].shape, generator=gen).to(io).cuda(), torch.randn(S0.shape, generator=gen).cuda() * 0.1
    want, S_want = ref.scan(op, desc.scale, [n0], t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], S0)
    grads = grads_of(op, desc.scale, [n0], t, S0, dout, dS)
    sides, first = set(), None
    for n in (1, 4, 5, 11):
        sides.add(n * H < sms)

        def rep(x):
            return None if x is None else x.repeat(n, *[1] * (x.dim() - 1))

        big = {x: y if x == "u_bonus" else rep(y) for x, y in t.items()}
        plan = make_plan([n0] * n)
        out, S = dl.scan_forward(desc, plan, **big, S_init=rep(S0))
        d = dl.scan_backward(desc, plan, **big, dout=rep(dout), S_init=rep(S0), dS_final=rep(dS))
        rows = [x.view(n, -1) for x in (out, S, d.q, d.k, d.v, d.S_init, *(y for y in (d.g, d.beta) if y is not None))]
        assert all(torch.equal(x[i], x[0]) for x in rows for i in range(n))
        first = first or [x[0] for x in rows]
        assert all(torch.equal(x[0], y) for x, y in zip(rows, first))
        if n in (4, 5):
            assert err(out[-n0:], want) < TOL[io] and err(S[-1], S_want[0]) < TOL_F32
            for name, w in grads.items():
                x = getattr(d, name)
                x = x / n if name == "u_bonus" else x[-1:] if name == "S_init" else x[-n0:]
                assert err(x, w) < (TOL[io] if name in ("q", "k", "v") else TOL_F32), name
    assert sides == {True, False}


@pytest.mark.parametrize("op", sorted(ref.OPS.values()))
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (64, 128)])
def test_prefill_fp32(op, dk, dv):
    """fp32 token tensors into the pool: a slot with pending log entries goes on, a fresh row over NaN, a padding row, a slot
    outside the pool; then a decode step."""
    H, Hq, cap, steps = 2, 1, 8, 3
    lens, slots = [70, 129, 20, 9, 0, 1], [5, 2, -1, 11, 0, 7]
    desc = make_desc(op, H, Hq, dk, dv, F32, num_slots=9, cap=cap)
    state = pool(desc, 1)
    S5, S7 = state.S_base[5].clone(), state.S_base[7].clone()
    pre, _ = ref.inputs(op, [steps], H, Hq, dk, dv, F32, seed=op + 260)
    t, _ = ref.inputs(op, lens, H, Hq, dk, dv, F32, seed=op + 261)
    t["u_bonus"] = bonus = pre["u_bonus"]

    def rows(x, sl):
        return {n: y if y is None or n == "u_bonus" else y[sl].clone() for n, y in x.items()}   # (16-byte boundaries)

    five = torch.tensor([5], dtype=torch.int32, device="cuda")
    for s in range(steps):
        dl.decode_step(desc, state, **rows(pre, slice(s, s + 1)), slot_idx=five)
    state.S_base[2], state.log_len[2] = float("nan"), 4
    keep = state.S_base[[0, 1, 3, 4, 6, 8]].clone()
    fresh = torch.tensor([0, 1, 0, 0, 1, 0], dtype=torch.int32, device="cuda")
    out = dl.prefill(desc, state, make_plan(lens, slots), **t, fresh=fresh)
    at = np.cumsum([0] + lens)
    assert state.status.item() == dl.STATUS_BAD_SLOT and torch.equal(state.S_base[[0, 1, 3, 4, 6, 8]], keep)
    assert not out[at[2]:at[4]].any() and not state.log_len[[5, 2, 7]].any()
    for row, front, S0 in ((0, pre, S5), (1, None, torch.zeros_like(S5)), (5, None, S7)):
        x = rows(t, slice(at[row], at[row + 1]))
        if front:
            x = {n: y if y is None or n == "u_bonus" else torch.cat((front[n], y)) for n, y in x.items()}
        n = lens[row] + (steps if front else 0)
        want, S_want = ref.scan(op, desc.scale, [n], x["q"], x["k"], x["v"], x["g"], x["beta"], bonus, S0[None])
        assert err(out[at[row]:at[row + 1]], want[n - lens[row]:]) < TOL_F32
        assert err(state.S_base[slots[row]], S_want[0]) < TOL_F32
    more, _ = ref.inputs(op, [1], H, Hq, dk, dv, F32, seed=op + 262)
    more["u_bonus"] = bonus
    S_from = state.S_base[5].clone()[None]
    got = dl.decode_step(desc, state, **more, slot_idx=five)
    want, _ = ref.scan(op, desc.scale, [1], more["q"], more["k"], more["v"], more["g"], more["beta"], bonus, S_from)
    assert err(got, want) < TOL_F32


@pytest.mark.parametrize("op,io", [(ref.GDN, BF16), (ref.KDA, BF16), (ref.GDN, F32), (ref.GLA, BF16)])
@pytest.mark.parametrize("lens,H", [([1900, 3, 0, 1537], 1), ([4100], 2)])
def test_segments_of_rows_that_forget_slowly(op, io, lens, H):
    """Gates of -0.001 to -0.02 and small betas: what a segment's map carries over its 500 tokens and more is a good part of the
    state, so the join counts (with gates of -0.7 the map is zero to working precision)."""
    dk = 128
    t, S0 = ref.inputs(op, lens, H, 1, dk, dk, io, seed=op + 270)
    gen = torch.Generator().manual_seed(15)
    t["g"] = (-0.001 - 0.019 * torch.rand(t["g"].shape, generator=gen) ** 4).cuda()   # mean -0.005
    if t["beta"] is not None:
        t["beta"] *= 0.1
    desc, plan = make_desc(op, H, 1, dk, dk, io), make_plan(lens)
    want, S_want = ref.scan(op, desc.scale, lens, t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], S0)
    out, S = dl.scan_forward(desc, plan, **t, S_init=S0)
    at = np.cumsum([0] + lens)
    for i, n in enumerate(lens):
        chunks = (n + 63) // 64
        segments = chunks // 8 if chunks >= 24 else 1
        more = max(0, segments - 2) * 128 * 2.0 ** -23      # a contraction over 128 channels more for each join
        assert err(out[at[i]:at[i + 1]], want[at[i]:at[i + 1]]) < TOL[io] + more, i
        assert err(S[i], S_want[i]) < TOL_F32 + more, i
        if segments > 1:    # the last segment behind a segment that starts from nothing, as if its map were zero: told apart
            last, before = (64 * (chunks * (segments - x) // segments) for x in (1, 2))
            part = [None if t[x] is None else t[x][at[i] + before:at[i + 1]] for x in ("q", "k", "v", "g", "beta")]
            cold, _ = ref.scan(op, desc.scale, [n - before], *part, None, torch.zeros_like(S0[i:i + 1]))
            first = slice(last - before, last - before + 64)
            assert err(cold[first], want[at[i] + before:at[i + 1]][first]) > 4 * (TOL[io] + more)


@pytest.mark.parametrize("io", [BF16, F32])
def test_new_output_of_a_captured_prefill(io):
    """The output's place is the graph's own and is written again by every replay: rows that ran in one replay and do not in the
    next are zero then."""
    op, H, d, n, most = ref.GDN, 2, 64, 5, 210
    desc = make_desc(op, H, H, d, d, io, num_slots=n)
    i32 = dict(dtype=torch.int32, device="cuda")
    lens, slots, plan, state = torch.zeros(n, **i32), torch.arange(n, **i32), dl.Plan(n, most, device="cuda"), pool(desc, 1)
    ws = dl.scan_workspace(desc, n, most)
    t, _ = ref.inputs(op, [most + 7], H, H, d, d, io, seed=280)

    def step(out=None):
        dl.build_plan(lens, plan, slots=slots, decode_rows=True)
        return dl.prefill(desc, state, plan, **t, out=out, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    start = state.S_base.clone()
    for ln in ([64, 1, 70, 0, 30], [1, 90, 0, 0, 1], [1] * 5, [0] * 5, [2, 200, 5, 3, 1], [1, 1, 1, 1, 206]):
        lens.copy_(torch.tensor(ln, **i32))
        slots.copy_(torch.tensor([0, 1, -1, 3, 4], **i32))
        out.fill_(float("nan"))
        state.S_base.copy_(start)
        graph.replay()
        got, S = out.clone(), state.S_base.clone()
        state.S_base.copy_(start)
        want = step(out=torch.zeros_like(out))
        assert torch.equal(got, want) and torch.equal(S, state.S_base), ln


@pytest.mark.parametrize("op,io,H,Hq,dk,dv,lens,tail", [
    (ref.GDN, BF16, 4, 2, 128, 128, [17, 0, 1, 64, 200], 5), (ref.KDA, BF16, 2, 1, 128, 128, [129, 63], 0), (ref.RWKV6, BF16, 2, 2, 64, 64, [65, 3, 190], 1),
    (ref.KDA, F32, 2, 1, 64, 128, [70, 64], 64), (ref.GLA, F32, 3, 3, 128, 64, [5, 127], 0), (ref.RETNET, F32, 2, 1, 64, 64, [64], 0),
    (ref.LINATTN, BF16, 1, 1, 64, 128, [1537, 9], 70), (ref.GDN, BF16, 1, 1, 128, 128, [1700], 0)])
def test_nothing_is_written_beside_the_tensors(op, io, H, Hq, dk, dv, lens, tail):
    """The workspace at its very size, the output and the plan's tables lie in larger buffers whose other bytes stay as they were."""
    room = 4096

    def inside(shape, dtype):
        size = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        whole = torch.full((size + 2 * room,), 0x5A, dtype=torch.uint8, device="cuda")
        return whole, whole[room:room + size].view(dtype).view(shape)

    wholes = []

    def place(like_shape, dtype):
        whole, view = inside(like_shape, dtype)
        wholes.append((whole, view.numel() * view.element_size()))
        return view

    n, most = len(lens), sum(lens) + tail
    t, S0 = ref.inputs(op, lens, H, Hq, dk, dv, io, seed=op + 290, tail=tail)
    desc = make_desc(op, H, Hq, dk, dv, io, num_slots=n)
    plan = dl.Plan(n, most, device="cuda")
    for name in ("starts", "chunk_starts", "chunk_seq", "token_seq", "scan_slots", "append_slots", "merge_slots", "totals"):
        setattr(plan, name, place((getattr(plan, name).numel(),), torch.int32))
    dl.build_plan(torch.tensor(lens, dtype=torch.int32, device="cuda"), plan)
    out = place(tuple(t["v"].shape), io)
    dout = torch.ones_like(t["v"])
    serve, train = ((place((dl.scan_workspace(desc, n, most, train=x).numel(),), torch.uint8)) for x in (False, True))
    dl.prefill(desc, pool(desc, 1), plan, **t, out=out, workspace=serve)
    dl.scan_forward(desc, plan, **t, S_init=S0, out=out, workspace=serve)
    dl.scan_forward(desc, plan, **t, S_init=S0, out=out, workspace=train, save=True)
    dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, workspace=train, saved=True)
    torch.cuda.synchronize()
    for whole, size in wholes:
        assert (whole[:room] == 0x5A).all() and (whole[room + size:] == 0x5A).all()
    want, S_want = ref.scan(op, desc.scale, lens, t["q"], t["k"], t["v"], t["g"], t["beta"], t["u_bonus"], S0)
    assert err(out[:sum(lens)], want) < TOL[io] + 128 * 2.0 ** -23 and (out[sum(lens):].contiguous().view(torch.uint8) == 0x5A).all()


# The tensor cores cut an accumulator's last bits: every addition into a sum loses half a unit 2^-23 of the partial sum on average,
# always towards zero.  A contraction over 128 channels takes eight additions of the operands' leading planes, whose partial
# sums are half of the sum on average: two units.  The lower planes' products have to come first, where the sums are still small
# (behind the leading ones they were forty more additions).  Twice that is allowed, for the sums are made of several contractions.
MEAN_CUT = 4 * 2.0 ** -23


def mean_relative(x, want):
    want = want.double().cpu()
    return ((x.double().cpu() - want) / want).mean().item()


@pytest.mark.parametrize("op", [ref.LINATTN, ref.RETNET])
@pytest.mark.parametrize("dk", [64, 128])
def test_fp32_sums_are_not_cut_on_tcgen05(op, dk):
    """One chunk of positive numbers, so that nothing averages out: the mean error of states, outputs and their gradients."""
    H, dv, T = 2, 128, 64
    gen = torch.Generator().manual_seed(16)

    def rand(*shape):
        return (0.5 + torch.rand(*shape, generator=gen)).cuda()

    t = dict(q=rand(T, H, dk), k=rand(T, H, dk), v=rand(T, H, dv), g=None if op == ref.LINATTN else -0.01 * rand(T, H), beta=None, u_bonus=None)
    S0, dS, dout = rand(1, H, dk, dv), rand(1, H, dk, dv), rand(T, H, dv)
    desc, plan = make_desc(op, H, H, dk, dv, F32, scale=1.0), make_plan([T])
    want, S_want = ref.scan(op, 1.0, [T], t["q"], t["k"], t["v"], t["g"], None, None, S0)
    grads = grads_of(op, 1.0, [T], t, S0, dout, dS)
    out, S = dl.scan_forward(desc, plan, **t, S_init=S0)
    d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, dS_final=dS)
    got = dict(out=mean_relative(out, want), S=mean_relative(S, S_want), dv=mean_relative(d.v, grads["v"]), dS=mean_relative(d.S_init, grads["S_init"]))
    assert all(abs(x) < MEAN_CUT for x in got.values()), got


@pytest.mark.parametrize("op", [ref.LINATTN, ref.RETNET, ref.GLA])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 64), (128, 128)])
def test_fp32_sums_are_not_cut(op, dk, dv):
    """The same for every output and gradient, head size 64 and per-channel gates among them."""
    H, T = 2, 64
    gen = torch.Generator().manual_seed(17)

    def rand(*shape):
        return (0.5 + torch.rand(*shape, generator=gen)).cuda()

    gate = (T, H, dk) if op == ref.GLA else (T, H)
    t = dict(q=rand(T, H, dk), k=rand(T, H, dk), v=rand(T, H, dv), g=None if op == ref.LINATTN else -0.01 * rand(*gate), beta=None, u_bonus=None)
    S0, dS, dout = rand(1, H, dk, dv), rand(1, H, dk, dv), rand(T, H, dv)
    desc, plan = make_desc(op, H, H, dk, dv, F32, scale=1.0), make_plan([T])
    want, S_want = ref.scan(op, 1.0, [T], t["q"], t["k"], t["v"], t["g"], None, None, S0)
    grads = grads_of(op, 1.0, [T], t, S0, dout, dS)
    out, S = dl.scan_forward(desc, plan, **t, S_init=S0)
    d = dl.scan_backward(desc, plan, **t, dout=dout, S_init=S0, dS_final=dS)
    got = dict(out=mean_relative(out, want), S=mean_relative(S, S_want)) | {n: mean_relative(getattr(d, n), grads[n]) for n in ("q", "k", "v", "S_init")}
    assert all(abs(x) < MEAN_CUT for x in got.values()), got


@pytest.mark.parametrize("op,io,H,Hq,dk,dv", [(ref.GDN, BF16, 4, 2, 128, 128), (ref.KDA, F32, 2, 1, 128, 128), (ref.RWKV6, BF16, 2, 2, 64, 64),
                                              (ref.GLA, F32, 2, 2, 64, 64), (ref.KDA, BF16, 2, 2, 64, 128)])
def test_what_no_row_runs_may_hold_anything(op, io, H, Hq, dk, dv):
    """NaN and infinities in the tokens of padding rows, of a slot outside the pool and behind the last sequence reach nothing: the same
    bits as with zeros there, forward and backward."""
    lens, slots, tail = [70, 33, 64, 9, 130], [2, -1, 0, 50, 1], 21
    t, S0 = ref.inputs(op, lens, H, Hq, dk, dv, io, seed=op + 300, tail=tail)
    desc = make_desc(op, H, Hq, dk, dv, io, num_slots=4)
    at = np.cumsum([0] + lens)
    skipped = torch.zeros(t["v"].shape[0], dtype=torch.bool)
    skipped[at[1]:at[2]] = skipped[at[3]:at[4]] = skipped[at[5]:] = True
    behind = torch.zeros_like(skipped)
    behind[at[5]:] = True
    gen = torch.Generator().manual_seed(18)
    dout = torch.randn(t["v"].shape, generator=gen).to(io).cuda()

    def filled(x, rows, value):
        x = x.clone()
        x[rows.cuda()] = value
        return x

    def run(value):
        def put(rows):
            return {n: y if y is None or n == "u_bonus" else filled(y, rows, value) for n, y in t.items()}

        state = pool(desc, 1)
        served = dl.prefill(desc, state, make_plan(lens, slots, tail=tail), **put(skipped))
        plan = make_plan(lens, tail=tail)
        ws = dl.scan_workspace(desc, len(lens), plan.max_tokens, train=True)
        out, S = dl.scan_forward(desc, plan, **put(behind), S_init=S0, workspace=ws, save=True)
        d = dl.scan_backward(desc, plan, **put(behind), dout=filled(dout, behind, value), S_init=S0, workspace=ws, saved=True)
        return [served, state.S_base, out, S, *(x for x in (d.q, d.k, d.v, d.g, d.beta, d.u_bonus, d.S_init) if x is not None)]

    clean = run(0.0)
    assert all(torch.isfinite(x).all() for x in clean)
    for value in (float("nan"), float("inf"), -float("inf")):
        for x, y in zip(clean, run(value)):
            assert torch.equal(x, y)


def test_two_scans_at_once():
    """One plan, two streams, a workspace each: both give what they give alone."""
    op, H, d, lens = ref.GDN, 8, 128, [900, 64, 3, 400]
    desc, plan = make_desc(op, H, H, d, d, BF16), make_plan(lens)
    sets = [ref.inputs(op, lens, H, H, d, d, BF16, seed=310 + i) for i in range(2)]
    spaces = [dl.scan_workspace(desc, len(lens), plan.max_tokens, train=True) for _ in sets]

    def run(i, stream=None):
        t, S0 = sets[i]
        out, S = dl.scan_forward(desc, plan, **t, S_init=S0, workspace=spaces[i], save=True, stream=stream)
        g = dl.scan_backward(desc, plan, **t, dout=t["v"], S_init=S0, workspace=spaces[i], saved=True, stream=stream)
        return out, S, g.q, g.k, g.v, g.g, g.beta, g.S_init

    alone = [run(0), run(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        both = [run(i, streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        for got, want in zip(both, alone):
            assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert plan.status.item() == 0
