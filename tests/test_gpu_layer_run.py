"""The operators together, as layers use them: a delta rule layer (convolution, norm of heads, scan or decode) and a state space
layer (convolution, state space scan): a prompt and then single tokens against the longer prompt, and a training step."""
import pytest
import torch

import paper_2608_15533_b200 as dl

pytestmark = pytest.mark.gpu
DEV = "cuda"
H, HQ, DK, DV, W = 4, 2, 64, 64, 4
CH = 2 * HQ * DK + H * DV


class DeltaLayer:
    """q, k, v of one convolution; q and k to unit length and rotated; the gated delta rule."""

    def __init__(self, slots, io=torch.float32):
        g = torch.Generator().manual_seed(0)
        self.io, dt = io, dl.F32 if io is torch.float32 else dl.BF16
        self.w, self.b = (torch.randn(CH, W, generator=g) * 0.5).to(DEV), (torch.randn(CH, generator=g) * 0.1).to(DEV)
        a = torch.arange(200, dtype=torch.float64)[:, None] * torch.pow(10000.0, -torch.arange(16, dtype=torch.float64) / 16)
        self.cos, self.sin = a.cos().float().to(DEV), a.sin().float().to(DEV)
        self.conv = dl.ConvDesc(CH, W, dt, num_slots=slots)
        self.norm = dl.NormDesc(HQ, HQ, DK, dt, dl.NORM_L2, 1e-6, rot=32, q_scale=DK ** -0.5)
        self.scan = dl.Desc(dl.GDN, slots, H, DK, DV, 8, dt, H_qk=HQ)
        self.window = dl.ConvState(self.conv, device=DEV)
        self.state = dl.State(self.scan, torch.zeros(slots, H, DK, DV, device=DEV))

    def heads(self, y, pos, norm):
        split = y[:, : HQ * DK].unflatten(1, (HQ, DK)), y[:, HQ * DK : 2 * HQ * DK].unflatten(1, (HQ, DK))
        q, k = norm(self.norm, *split, None, None, self.cos, self.sin, pos)
        return q, k, y[:, 2 * HQ * DK :].unflatten(1, (H, DV)).contiguous()

    def prefill(self, plan, x, pos, g, beta):
        y = dl.conv_prefill(self.conv, self.window, plan, x, self.w, self.b)
        return dl.prefill(self.scan, self.state, plan, *self.heads(y, pos, dl.head_norm_forward), g, beta)

    def step(self, x, pos, g, beta, slots):
        y = dl.conv_step(self.conv, self.window, x, self.w, self.b, slot_idx=slots)
        return dl.decode_step(self.scan, self.state, *self.heads(y, pos, dl.head_norm_forward), g, beta, slot_idx=slots)


def _tokens(T, width, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, width, generator=g).to(DEV), -torch.nn.functional.softplus(torch.randn(T, H, generator=g)).to(DEV),
            torch.sigmoid(torch.randn(T, H, generator=g)).to(DEV))


def _plan(lens, slots):
    plan = dl.Plan(len(lens), sum(lens), device=DEV)
    return dl.build_plan(torch.tensor(lens, dtype=torch.int32, device=DEV), plan, slots=torch.tensor(slots, dtype=torch.int32, device=DEV))


def _positions(lens, at=0):
    return torch.cat([torch.arange(n) + at for n in lens]).to(torch.int32).to(DEV)


def test_delta_layer_prompt_then_tokens_is_the_longer_prompt():
    lens, more, slots = (30, 1, 77), 5, [2, 0, 3]
    rows = [_tokens(n + more, CH, i) for i, n in enumerate(lens)]
    whole, served = DeltaLayer(4), DeltaLayer(4)
    cat = lambda cut: [torch.cat([r[j][cut(n)] for r, n in zip(rows, lens)]).contiguous() for j in range(3)]
    long = [n + more for n in lens]
    want = whole.prefill(_plan(long, slots), cat(lambda n: slice(0, n + more))[0], _positions(long), *cat(lambda n: slice(0, n + more))[1:])
    x, g, beta = cat(lambda n: slice(0, n))
    got = [served.prefill(_plan(lens, slots), x, _positions(lens), g, beta)]
    idx = torch.tensor(slots, dtype=torch.int32, device=DEV)
    steps = []
    for t in range(more):
        x, g, beta = (torch.stack([r[j][n + t] for r, n in zip(rows, lens)]) for j in range(3))
        steps.append(served.step(x, torch.tensor([n + t for n in lens], dtype=torch.int32, device=DEV), g, beta, idx))
    dl.merge(served.scan, served.state)
    at, first = 0, 0
    for i, n in enumerate(lens):
        mine = torch.cat([got[0][first : first + n]] + [s[i : i + 1] for s in steps])
        err = (mine - want[at : at + n + more]).abs().max() / want.abs().max()
        assert err < 1e-4, (i, float(err))      # the bar of the fp32 states and outputs
        at, first = at + n + more, first + n
    assert (served.state.S_base - whole.state.S_base).abs().max() / whole.state.S_base.abs().max() < 1e-4
    assert torch.equal(served.window.window, whole.window.window)


def test_delta_layer_trains():
    layer = DeltaLayer(1)
    lens = (20, 9)
    x, g, beta = _tokens(sum(lens), CH, 7)
    plan = _plan(lens, [0, 0])
    leaf = [t.clone().requires_grad_() for t in (x, layer.w, layer.b, g, beta)]

    def run(x, w, b, g, beta):
        y, _ = dl.conv(layer.conv, plan, x, w, b)
        q, k, v = layer.heads(y, _positions(lens), dl.head_norm)
        return dl.scan(layer.scan, plan, q, k, v, g, beta)[0]

    out = run(*leaf)
    do = torch.randn_like(out)
    grads = torch.autograd.grad((out * do).sum(), leaf)
    for i, gr in enumerate(grads):
        # a central difference of the fp32 layer in the gradient's own direction: the step moves the loss by about 1e-3 of sum |out do|,
        # whose evaluation is good to 1e-5 of it (fp32 outputs, 1e-4 of their largest at worst), and the cubic term is of the step squared
        v = gr / gr.norm()
        h = 2e-3 * float((out * do).abs().sum()) / float(gr.norm())
        h = min(h, 0.05)
        move = lambda s: [t.detach() + s * v if j == i else t.detach() for j, t in enumerate(leaf)]
        with torch.no_grad():
            num = float(((run(*move(h)) * do).double().sum() - (run(*move(-h)) * do).double().sum()) / (2 * h))
        assert abs(num - float(gr.norm())) < 0.05 * float(gr.norm()), i


def test_state_space_layer_prompt_then_tokens_is_the_longer_prompt():
    D, N, R = 128, 16, 8
    lens, more, slots = (40, 3, 200), 4, [1, 3, 0]
    g = torch.Generator().manual_seed(4)
    rnd = lambda *s: torch.randn(*s, generator=g).to(DEV)
    w, b, A, skip, bias = rnd(D, W) * 0.5, rnd(D) * 0.1, -torch.arange(1, N + 1, device=DEV).float().expand(D, N).contiguous(), rnd(D), rnd(D) - 3
    xz, proj = [rnd(n + more, 2 * D) for n in lens], [rnd(n + more, D + R + 2 * N) for n in lens]
    conv, ssm = dl.ConvDesc(D, W, dl.F32, num_slots=4), dl.SsmDesc(D, N, 1, dl.F32, num_slots=4)

    class Layer:
        def __init__(self):
            self.window, self.state = dl.ConvState(conv, device=DEV), dl.SsmState(ssm, device=DEV)

        def args(self, y, xz, p):
            # B and C are columns of one projection, the gate is the second half of the input's
            return y, p[:, :D], A, p[:, D + R : D + R + N].unflatten(1, (1, N)), p[:, D + R + N :].unflatten(1, (1, N)), skip, xz[:, D:], bias

        def prefill(self, plan, xz, p):
            y = dl.conv_prefill(conv, self.window, plan, xz[:, :D], w, b)
            return dl.ssm_prefill(ssm, self.state, plan, *self.args(y, xz, p))

        def step(self, xz, p, idx):
            y = dl.conv_step(conv, self.window, xz[:, :D], w, b, slot_idx=idx)
            return dl.ssm_step(ssm, self.state, *self.args(y, xz, p), slot_idx=idx)

    whole, served = Layer(), Layer()
    want = whole.prefill(_plan([n + more for n in lens], slots), torch.cat(xz), torch.cat(proj))
    got = served.prefill(_plan(lens, slots), torch.cat([t[:n] for t, n in zip(xz, lens)]), torch.cat([t[:n] for t, n in zip(proj, lens)]))
    idx = torch.tensor(slots, dtype=torch.int32, device=DEV)
    steps = [served.step(torch.stack([t[n + i] for t, n in zip(xz, lens)]), torch.stack([t[n + i] for t, n in zip(proj, lens)]), idx) for i in range(more)]
    at = first = 0
    for i, n in enumerate(lens):
        mine = torch.cat([got[first : first + n]] + [s[i : i + 1] for s in steps])
        assert (mine - want[at : at + n + more]).abs().max() / want.abs().max() < 1e-4, i
        at, first = at + n + more, first + n
    assert (served.state.S - whole.state.S).abs().max() / whole.state.S.abs().max() < 1e-4 and torch.equal(served.window.window, whole.window.window)
    assert int(served.window.status) == 0 and int(served.state.status) == 0


def _small(which):
    """A differentiable call and its leaves, on the device."""
    g = torch.Generator().manual_seed(5)
    lens = (40, 3)
    T, plan = sum(lens), _plan(lens, [0, 1])

    def new(*shape):
        return torch.randn(*shape, generator=g).to(DEV)

    if which == "conv":
        desc = dl.ConvDesc(64, 4, dl.F32)
        return [new(T, 64), new(64, 4), new(64)], lambda x, w, b: dl.conv(desc, plan, x, w, b)
    if which == "norm":
        desc = dl.NormDesc(2, 1, 64, dl.F32, dl.NORM_RMS)
        return [new(T, 2, 64), new(T, 1, 64), new(64), new(64)], lambda q, k, wq, wk: dl.head_norm(desc, q, k, wq, wk)
    desc = dl.SsmDesc(64, 16, 1, dl.F32)
    return [new(T, 64), new(T, 64), -new(64, 16).exp(), new(T, 1, 16), new(T, 1, 16)], lambda *a: dl.ssm(desc, plan, *a)


def _gradients(call, leaves):
    a, b = call(*leaves)
    return torch.autograd.grad(a.square().sum() + b.sum(), leaves)


@pytest.mark.parametrize("which", ["conv", "norm"])
def test_gradients_in_a_graph(which):
    values, call = _small(which)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        leaves = [v.clone().requires_grad_() for v in values]
        _gradients(call, leaves)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = _gradients(call, leaves)
    with torch.no_grad():
        leaves[0].mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    for got, want in zip(grads, _gradients(call, [v.detach().clone().requires_grad_() for v in leaves])):
        assert torch.equal(got, want)


@pytest.mark.parametrize("which", ["conv", "norm"])
def test_capture_beside_an_eager_graph_is_refused(which):
    values, call = _small(which)
    values[0].requires_grad_()
    out, _ = call(*values)
    with pytest.raises(RuntimeError, match="eager|default stream"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            call(*values)
    out.sum().backward()
    assert torch.isfinite(values[0].grad).all()


@pytest.mark.parametrize("which", ["conv", "norm", "ssm"])
def test_gradients_on_two_streams_at_once(which):
    values, call = _small(which)
    want = _gradients(call, [v.clone().requires_grad_() for v in values])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(_gradients(call, [v.clone().requires_grad_() for v in values]))
    torch.cuda.synchronize()
    for grads in got:
        for g, w in zip(grads, want):
            assert torch.equal(g, w)
