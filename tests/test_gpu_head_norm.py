"""Norm and rotation of query and key heads on the GPU against their 64-bit form.

Tolerances: half a step of the output's type, and of fp32: d / 16 + 6 roundings in a sum of squares over lanes, a reciprocal square root
of 2^-22, the weight, the scale and two products and a sum of the rotation, under 2^-19 of the largest value of a pair for d <= 256.  A
gradient takes the same of two sums: 2^-18 of r (|g w| + |x| c r^2 sum |g w x|); the weights' sum over T H values adds their roundings.
"""
import pytest
import torch

import layer_reference as ref
import paper_2608_15533_b200 as dl

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {torch.float32: dl.F32, torch.bfloat16: dl.BF16}
NORM = {"l2": dl.NORM_L2, "rms": dl.NORM_RMS, "none": dl.NORM_NONE}


def _table(rows, rot):
    a = torch.arange(rows, dtype=ref.F64)[:, None] * torch.pow(10000.0, -torch.arange(rot // 2, dtype=ref.F64) / max(rot // 2, 1))
    return a.cos().float().to(DEV), a.sin().float().to(DEV)


def _setup(T, Hq, Hk, d, io, norm, rot, weights, wide=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    proj = torch.randn(T, Hq + Hk + 1, d, generator=g).to(io).to(DEV)
    q, k = proj[:, :Hq], proj[:, Hq : Hq + Hk]
    if not wide:
        q, k = q.contiguous(), k.contiguous()
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(DEV) if weights else None for _ in range(2)]
    cos = sin = pos = None
    if rot:
        cos, sin = _table(500, rot)
        pos = torch.randint(0, 500, (T,), generator=g).to(torch.int32).to(DEV)
    return q, k if Hk else None, w[0], w[1] if Hk else None, cos, sin, pos


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,Hq,Hk,d,norm,rot,interleaved,weights", [
    (1, 1, 1, 64, "l2", 0, False, False),
    (5, 3, 2, 128, "rms", 128, False, True),
    (7, 16, 4, 128, "rms", 64, True, True),
    (33, 5, 1, 96, "l2", 48, False, False),
    (9, 1, 3, 256, "rms", 256, True, True),
    (130, 7, 0, 40, "rms", 32, False, True),
    (4, 2, 2, 8, "rms", 0, False, True),
    (6, 9, 9, 32, "none", 16, True, False),
    (3, 33, 17, 72, "rms", 16, False, False),
    (700, 8, 2, 128, "rms", 128, False, True),
])
def test_forward_and_gradients(io, T, Hq, Hk, d, norm, rot, interleaved, weights):
    q, k, wq, wk, cos, sin, pos = _setup(T, Hq, Hk, d, io, norm, rot, weights)
    desc = dl.NormDesc(Hq, Hk, d, DT[io], NORM[norm], 1e-5, rot, interleaved, q_scale=0.37)
    g = torch.Generator().manual_seed(3)
    doq, dok = (torch.randn(T, h, d, generator=g).to(io).to(DEV) for h in (Hq, Hk))
    got = dl.head_norm_forward(desc, q, k, wq, wk, cos, sin, pos)
    grads = dl.head_norm_backward(desc, q, k, wq, wk, cos, sin, pos, doq, dok if Hk else None)
    again = dl.head_norm_backward(desc, q, k, wq, wk, cos, sin, pos, doq, dok if Hk else None)
    c, s = (ref.f64(cos)[pos.cpu().long()], ref.f64(sin)[pos.cpu().long()]) if rot else (None, None)
    for x, w, scale, out, do, dx, dw, name in ((q, wq, 0.37, got[0], doq, grads.q, grads.w_q, "q"), (k, wk, 1.0, got[1], dok, grads.k, grads.w_k, "k")):
        if x is None:
            assert out is None and dx is None and dw is None
            continue
        X, Wt = ref.f64(x).requires_grad_(), None if w is None else ref.f64(w).requires_grad_()
        want = ref.head_norm(X, Wt, norm, 1e-5, scale, rot, interleaved, c, s)
        n = ref.head_norm(X, Wt, norm, 1e-5, scale, 0, False, None, None).detach().abs()
        mag = n.amax(-1, keepdim=True).expand_as(n)
        ref.close(out, want.detach(), mag, 2.0 ** -19, name)
        (want * ref.f64(do)).sum().backward()
        # the gradient's magnitude: pairs mix under the rotation, so the largest of a head
        G = ref.f64(do).abs().amax(-1, keepdim=True) * 1.5 * scale
        wmax = 1.0 if Wt is None else Wt.detach().abs().max()
        if norm == "none":
            gm = G.expand_as(X)
        else:
            cc = 1 / d if norm == "rms" else 1.0
            r = 1 / torch.sqrt(cc * (X.detach() ** 2).sum(-1, keepdim=True) + 1e-5)
            gm = r * (G * wmax + X.detach().abs() * cc * r * r * (G * wmax * X.detach().abs()).sum(-1, keepdim=True))
        ref.close(dx, X.grad, gm, 2.0 ** -18, "d" + name)
        if w is not None:
            wm = (G * X.detach().abs() * r).sum((0, 1))
            ref.close(dw, Wt.grad, wm, 2.0 ** -18 + T * x.shape[1] * 2.0 ** -24, "dw of " + name)
            assert torch.equal(dw, again.w_q if name == "q" else again.w_k)


def test_positions_outside_of_the_table():
    T, d = 6, 64
    q, k, wq, wk, cos, sin, pos = _setup(T, 2, 1, d, torch.bfloat16, "rms", d, True)
    pos[1], pos[4] = -1, 500
    q[1] = float("nan")              # a padding token may hold anything
    desc = dl.NormDesc(2, 1, d, norm=dl.NORM_RMS, rot=d)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    oq, ok = dl.head_norm_forward(desc, q, k, wq, wk, cos, sin, pos, status=status)
    assert int(status) == dl.STATUS_BAD_POSITION
    do = torch.randn(T, 2, d, device=DEV).bfloat16(), torch.randn(T, 1, d, device=DEV).bfloat16()
    g = dl.head_norm_backward(desc, q, k, wq, wk, cos, sin, pos, *do)
    for t in (oq, ok, g.q, g.k):
        assert not t[1].any() and not t[4].any() and torch.isfinite(t).all()
    good = [0, 2, 3, 5]
    sub = [t[good].contiguous() for t in (q, k)]
    want = dl.head_norm_forward(desc, *sub, wq, wk, cos, sin, pos[good])
    assert torch.equal(oq[good], want[0]) and torch.equal(ok[good], want[1])
    gw = dl.head_norm_backward(desc, *sub, wq, wk, cos, sin, pos[good], do[0][good], do[1][good])
    assert torch.allclose(g.w_q, gw.w_q, rtol=1e-5, atol=1e-6) and torch.isfinite(g.w_k).all()
    status.zero_()
    pos[4] = -7                      # negative alone: no complaint
    dl.head_norm_forward(desc, q, k, wq, wk, cos, sin, pos, status=status)
    assert int(status) == 0


def test_zeros_infinities_and_nan():
    d = 128
    x = torch.randn(5, 1, d, device=DEV)
    x[0] = 0
    x[2, 0, 3], x[3, 0, 7] = float("nan"), float("inf")
    desc = dl.NormDesc(1, 0, d, dl.F32, dl.NORM_L2, 1e-6)
    out, none = dl.head_norm_forward(desc, x, None)
    assert none is None and not out[0].any()
    want = ref.head_norm(ref.f64(x), None, "l2", 1e-6, 1.0, 0, False, None, None)
    assert torch.equal(torch.isnan(out).cpu(), torch.isnan(want))
    assert torch.isfinite(out[[0, 1, 4]]).all()
    g = dl.head_norm_backward(desc, x[:2].contiguous(), None, None, None, None, None, None, torch.ones(2, 1, d, device=DEV), None)
    assert torch.isfinite(g.q).all()


def test_in_place_streams_and_replays():
    T, d = 40, 128
    q, k, wq, wk, cos, sin, pos = _setup(T, 8, 2, d, torch.bfloat16, "rms", d, True, wide=False)
    desc = dl.NormDesc(8, 2, d, norm=dl.NORM_RMS, rot=d)
    want = dl.head_norm_forward(desc, q, k, wq, wk, cos, sin, pos)
    a, b = q.clone(), k.clone()
    dl.head_norm_forward(desc, a, b, wq, wk, cos, sin, pos, out_q=a, out_k=b)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = dl.head_norm_forward(desc, q, k, wq, wk, cos, sin, pos, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0])
    oq, ok = torch.zeros_like(q), torch.zeros_like(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dl.head_norm_forward(desc, q, k, wq, wk, cos, sin, pos, out_q=oq, out_k=ok)
    pos.add_(1).remainder_(500)
    graph.replay()
    want = dl.head_norm_forward(desc, q, k, wq, wk, cos, sin, pos)
    assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])


def test_autograd_and_no_tokens():
    q, k, wq, wk, cos, sin, pos = _setup(12, 3, 1, 64, torch.float32, "rms", 32, True)
    desc = dl.NormDesc(3, 1, 64, dl.F32, dl.NORM_RMS, rot=32)
    leaf = [t.detach().clone().requires_grad_() for t in (q, k, wq, wk)]
    oq, ok = dl.head_norm(desc, *leaf, cos, sin, pos)
    grads = torch.autograd.grad(oq.square().sum(), leaf, allow_unused=True)     # keys without a gradient
    assert not grads[1].any() and not grads[3].any() and grads[0].any() and grads[2].any()
    empty = [t[:0] for t in (q, k)]
    oq, ok = dl.head_norm_forward(desc, *empty, wq, wk, cos, sin, pos[:0])
    assert oq.shape == (0, 3, 64) and ok.shape == (0, 1, 64)
    g = dl.head_norm_backward(desc, *empty, wq, wk, cos, sin, pos[:0], oq, ok)
    assert not g.w_q.any() and not g.w_k.any() and g.q.shape == (0, 3, 64)


def test_offsets_beyond_32_bits():
    T, H, d = 530_000, 32, 128               # 2.2e9 values
    q = torch.zeros(T, H, d, dtype=torch.bfloat16, device=DEV)
    q[-3:] = torch.randn(3, H, d).bfloat16().to(DEV)
    desc = dl.NormDesc(H, 0, d)
    out, _ = dl.head_norm_forward(desc, q, None)
    want, _ = dl.head_norm_forward(desc, q[-3:].clone(), None)
    assert torch.equal(out[-3:], want) and not out[:-3].any()
    g = dl.head_norm_backward(desc, q, None, None, None, None, None, None, out, None)
    assert torch.isfinite(g.q[-3:]).all()
    del q, out, g
    torch.cuda.empty_cache()
