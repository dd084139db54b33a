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
