"""Packed-sequence entry points without a GPU: every refusal comes back from the host before anything is launched, the
workspace sizes follow their formula, and the Python layer names the argument it refuses."""
import ctypes

import pytest
import torch

import paper_2608_15533_b200 as dl
from paper_2608_15533_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return dl.load_library()


def _desc(**kw):
    return dl.Desc(**(dict(op=dl.GDN, num_slots=4, H=2, d_k=64, d_v=64, cap=8, io_dtype=dl.BF16) | kw))


def _plan(**kw):
    # fake, aligned, never dereferenced
    names = ("starts", "chunk_starts", "chunk_seq", "token_seq", "scan_slots", "append_slots", "merge_slots", "totals", "status")
    vals = {"n": 3, "max_tokens": 100} | {x: 0x1000 * (i + 1) for i, x in enumerate(names)} | kw
    return binding._Plan(**vals)


def _state():
    return binding._State(**{n: 0x100000 * (i + 1) for i, n in enumerate(("S_base", "K_log", "U_log", "decay_log", "log_len", "status"))})


P = dict(q=0x10000, k=0x20000, v=0x30000, g=0x40000, beta=0x50000, bonus=None)
BIG = 1 << 40


def _prefill(lib, d, plan, state=None, out=0x60000, ws=0x70000, size=BIG, **kw):
    a = P | kw
    return lib.deltalog_prefill(ctypes.byref(d.c_struct()), ctypes.byref(_state() if state is None else state), ctypes.byref(plan), a["q"], a["k"],
                                a["v"], a["g"], a["beta"], a["bonus"], None, out, ws, size, None)


def _forward(lib, d, plan, out=0x60000, save=0, ws=0x70000, size=BIG, **kw):
    a = P | kw
    return lib.deltalog_scan_forward(ctypes.byref(d.c_struct()), ctypes.byref(plan), None, a["q"], a["k"], a["v"], a["g"], a["beta"], a["bonus"], out,
                                     None, save, ws, size, None)


def _backward(lib, d, plan, dout=0x80000, rows=100, ws=0x70000, size=BIG, grads=None, **kw):
    a = P | kw
    g = {"q": 0x90000, "k": 0xa0000, "v": 0xb0000, "g": 0xc0000, "beta": 0xd0000, "u_bonus": None, "S_init": None} | (grads or {})
    return lib.deltalog_scan_backward(ctypes.byref(d.c_struct()), ctypes.byref(plan), None, a["q"], a["k"], a["v"], a["g"], a["beta"], a["bonus"],
                                      dout, None, 0, ctypes.byref(binding._ScanGrads(**g)), rows, ws, size, None)


def test_scan_refusals(lib):
    before = dl.launch_count()
    INV, SHAPE, CAP = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED_SHAPE, binding.ERR_CAP_RANGE
    for call in (_prefill, _forward, _backward):
        assert call(lib, _desc(op=9), _plan()) == INV
        assert call(lib, _desc(d_k=96), _plan()) == SHAPE
        assert call(lib, _desc(d_v=256), _plan()) == SHAPE
        assert call(lib, _desc(cap=0), _plan()) == CAP
        assert call(lib, _desc(H=3, H_qk=2), _plan()) == INV
        assert call(lib, _desc(), _plan(n=-1)) == INV
        assert call(lib, _desc(), _plan(max_tokens=-1)) == INV
        assert call(lib, _desc(), _plan(max_tokens=2 ** 31 - 1)) == SHAPE
        assert call(lib, _desc(H=2 ** 20), _plan()) == SHAPE
        for name in ("starts", "chunk_starts", "chunk_seq", "scan_slots"):
            assert call(lib, _desc(), _plan(**{name: None})) == INV
        for name in ("q", "k", "v", "g", "beta"):
            assert call(lib, _desc(), _plan(), **{name: None}) == INV
        for name in ("q", "k", "v", "g"):
            assert call(lib, _desc(), _plan(), **{name: 0x10008}) == INV      # misaligned
        assert call(lib, _desc(op=dl.RWKV6), _plan()) == INV                  # no bonus
        assert call(lib, _desc(), _plan(), ws=None) == INV
        assert call(lib, _desc(), _plan(), ws=0x70004) == INV
        need = lib.deltalog_scan_workspace_bytes(ctypes.byref(_desc().c_struct()), 3, 100, 1 if call is _backward else 0)
        assert call(lib, _desc(), _plan(), size=need - 1) == INV
        assert call(lib, _desc(), _plan(n=0)) == binding.OK                   # no rows: nothing to launch
    need = lib.deltalog_scan_workspace_bytes(ctypes.byref(_desc().c_struct()), 3, 100, 0)
    assert _forward(lib, _desc(), _plan(), save=1, size=need) == INV          # save wants the larger workspace
    assert _prefill(lib, _desc(), _plan(), out=None) == INV and _forward(lib, _desc(), _plan(), out=0x60008) == INV
    bad = _state()
    bad.log_len = None
    assert _prefill(lib, _desc(), _plan(), state=bad) == INV
    assert _backward(lib, _desc(), _plan(), dout=None) == INV and _backward(lib, _desc(), _plan(), rows=99) == INV
    for name in ("q", "k", "v", "g", "beta"):
        assert _backward(lib, _desc(), _plan(), grads={name: None}) == INV
    assert _backward(lib, _desc(op=dl.RWKV6), _plan(), bonus=0xe0000) == INV  # u_bonus' gradient is missing
    assert dl.launch_count() == before


def test_plan_refusals(lib):
    def call(plan, lens=0x9000, log=None, H=2, cap=8, num=4):
        return lib.deltalog_build_plan(lens, None, log, H, cap, num, 1, ctypes.byref(plan), None)

    before = dl.launch_count()
    assert lib.deltalog_build_plan(0x9000, None, None, 0, 0, 0, 0, None, None) == binding.ERR_INVALID_ARG
    assert call(_plan(), lens=None) == binding.ERR_INVALID_ARG
    assert call(_plan(n=-1)) == binding.ERR_INVALID_ARG
    for name in ("starts", "chunk_starts", "chunk_seq", "scan_slots", "totals"):
        assert call(_plan(**{name: None})) == binding.ERR_INVALID_ARG
    assert call(_plan(token_seq=0x4004)) == binding.ERR_INVALID_ARG
    assert call(_plan(), log=0xa000, H=0) == binding.ERR_INVALID_ARG
    assert call(_plan(), log=0xa000, cap=0) == binding.ERR_CAP_RANGE and call(_plan(), log=0xa000, cap=65) == binding.ERR_CAP_RANGE
    assert dl.launch_count() == before


def test_workspace_sizes(lib):
    def size(n, tokens, train, **kw):
        return lib.deltalog_scan_workspace_bytes(ctypes.byref(_desc(**kw).c_struct()), n, tokens, train)

    units = (640 // 64 + 3) * 2
    assert size(3, 640, 0) == units * (2 * 3 * 64 * 64 * 2 + 2 * 64 * 4) + 256
    assert size(3, 640, 0, op=dl.RETNET) == units * (3 * 64 * 64 * 2 + 2 * 64 * 4) + 256
    assert size(3, 640, 1) == size(3, 640, 0) + units * (2 * 64 * 64 * 4 + 2 * 64 * 64 * 4)
    assert size(3, 640, 1, H_qk=1) == size(3, 640, 1) + 2 * 640 * 2 * 64 * 4
    assert size(-1, 640, 0) == 0 and size(3, -1, 0) == 0 and size(3, 640, 0, d_k=32) == 0
    assert size(1000, 2 ** 30, 1) > 2 ** 40   # 64-bit arithmetic


def test_python_layer_names_what_it_refuses():
    plan = dl.Plan(2, 10, device="cpu")
    d = _desc()
    T, bf = 10, torch.bfloat16
    good = dict(q=torch.zeros(T, 2, 64, dtype=bf), k=torch.zeros(T, 2, 64, dtype=bf), v=torch.zeros(T, 2, 64, dtype=bf), g=torch.zeros(T, 2),
                beta=torch.zeros(T, 2))
    lens = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="no path but the GPU"):
        dl.build_plan(lens, plan)
    with pytest.raises(ValueError, match="lens"):
        dl.build_plan(lens.long(), plan)
    with pytest.raises(ValueError, match="lens"):
        dl.build_plan(lens[:1], plan)
    with pytest.raises(ValueError, match="slots"):
        dl.build_plan(lens, plan, slots=torch.zeros(4, dtype=torch.int32)[::2])
    with pytest.raises(ValueError):
        dl.Plan(-1, 10, device="cpu")
    for name, bad in (("q", good["q"].float()), ("k", good["k"][:, :1]), ("v", good["v"].transpose(0, 1).contiguous().transpose(0, 1)),
                      ("g", good["g"][:9]), ("beta", None), ("beta", good["beta"].to(bf))):
        with pytest.raises(ValueError, match=name):
            dl.scan_forward(d, plan, **(good | {name: bad}))
        with pytest.raises(ValueError, match=name):
            dl.scan_backward(d, plan, **(dict(u_bonus=None) | good | {name: bad}), dout=good["v"])
    with pytest.raises(ValueError, match="reaches over"):
        dl.scan_forward(d, dl.Plan(2, 11, device="cpu"), **good)
    with pytest.raises(ValueError, match="no path but the GPU"):
        dl.scan_forward(d, plan, **good)
    with pytest.raises(ValueError, match="save"):
        dl.scan_forward(d, plan, **good, save=True)
    with pytest.raises(ValueError, match="saved"):
        dl.scan_backward(d, plan, **good, u_bonus=None, dout=good["v"], saved=True)
    with pytest.raises(ValueError, match="S_init"):
        dl.scan_forward(d, plan, **good, S_init=torch.zeros(2, 2, 64, 64, dtype=bf))
    with pytest.raises(ValueError, match="dout"):
        dl.scan_backward(d, plan, **good, u_bonus=None, dout=good["v"].float())
    with pytest.raises(ValueError, match="u_bonus"):
        dl.scan_forward(_desc(op=dl.RWKV6), plan, **(good | dict(g=torch.zeros(T, 2, 64))))
    with pytest.raises(ValueError):
        dl.scan_workspace(_desc(d_k=32), 1, 10, device="cpu")
    n, H, cap = 4, 2, 8
    state = [torch.zeros(n, H, 64, 64), torch.zeros(n, H, cap, 64, dtype=bf), torch.zeros(n, H, cap, 64), torch.zeros(n, H, cap, 1),
             torch.zeros(n, H, dtype=torch.int32)]
    assert dl.State.wrap(d, *state).S_base is state[0]
    for i, name in enumerate(("S_base", "K_log", "U_log", "decay_log", "log_len")):
        bad = list(state)
        bad[i] = bad[i][:3]
        with pytest.raises(ValueError, match=name):
            dl.State.wrap(d, *bad)


def test_prefill_refuses_a_state_of_another_shape():
    plan, d, T, bf = dl.Plan(2, 10, device="cpu"), _desc(), 10, torch.bfloat16
    tokens = dict(q=torch.zeros(T, 2, 64, dtype=bf), k=torch.zeros(T, 2, 64, dtype=bf), v=torch.zeros(T, 2, 64, dtype=bf), g=torch.zeros(T, 2),
                  beta=torch.zeros(T, 2))
    import dataclasses
    for other in (dict(num_slots=d.num_slots - 1), dict(cap=d.cap - 1), dict(H=1, H_qk=1), dict(d_k=128), dict(ulog_dtype=dl.BF16)):
        od = dataclasses.replace(d, **other)
        state = dl.State(od, torch.zeros(od.num_slots, od.H, od.d_k, od.d_v))
        with pytest.raises(ValueError, match="another descriptor"):
            dl.prefill(d, state, plan, **tokens)
    same = dl.State(dataclasses.replace(d), torch.zeros(d.num_slots, 2, 64, 64))
    with pytest.raises(ValueError, match="no path but the GPU"):   # an equal descriptor passes this check
        dl.prefill(d, same, plan, **tokens)


def test_scan_names_what_it_refuses():
    plan, d, T, bf = dl.Plan(2, 10, device="cpu"), _desc(), 10, torch.bfloat16
    tokens = dict(q=torch.zeros(T, 2, 64, dtype=bf, requires_grad=True), k=torch.zeros(T, 2, 64, dtype=bf), v=torch.zeros(T, 2, 64, dtype=bf),
                  g=torch.zeros(T, 2), beta=torch.zeros(T, 2))
    with pytest.raises(ValueError, match="beta"):
        dl.scan(d, plan, **(tokens | dict(beta=None)))
    with pytest.raises(ValueError, match="no path but the GPU"):
        dl.scan(d, plan, **tokens)


@pytest.mark.parametrize("name", ["q", "k", "v", "g", "beta", "S_init"])
def test_scan_refuses_forward_mode(name):
    """A dual tensor does not require a gradient: its tangent must not be dropped without a word."""
    from torch.autograd import forward_ad

    plan, d, T, bf = dl.Plan(2, 10, device="cpu"), _desc(), 10, torch.bfloat16
    tokens = dict(q=torch.zeros(T, 2, 64, dtype=bf), k=torch.zeros(T, 2, 64, dtype=bf), v=torch.zeros(T, 2, 64, dtype=bf), g=torch.zeros(T, 2),
                  beta=torch.zeros(T, 2), S_init=torch.zeros(2, 2, 64, 64))
    with forward_ad.dual_level():
        with pytest.raises(ValueError, match="no path but the GPU"):
            dl.scan(d, plan, **tokens)
        for grad in (True, False):
            with torch.set_grad_enabled(grad), pytest.raises(RuntimeError, match="forward-mode"):
                dl.scan(d, plan, **(tokens | {name: forward_ad.make_dual(tokens[name], torch.ones_like(tokens[name]))}))


def test_wrap_refuses_a_status_word_that_the_kernels_cannot_set():
    d, bf, n, H, cap = _desc(), torch.bfloat16, 4, 2, 8
    state = [torch.zeros(n, H, 64, 64), torch.zeros(n, H, cap, 64, dtype=bf), torch.zeros(n, H, cap, 64), torch.zeros(n, H, cap, 1),
             torch.zeros(n, H, dtype=torch.int32)]
    word = torch.zeros(1, dtype=torch.int32)
    assert dl.State.wrap(d, *state, status=word).status is word
    for bad in (torch.zeros(1, dtype=torch.int64), torch.zeros(1), torch.zeros(0, dtype=torch.int32), torch.zeros(1, dtype=torch.int32, device="meta")):
        with pytest.raises(ValueError, match="status"):
            dl.State.wrap(d, *state, status=bad)


@pytest.mark.parametrize("H,dv", [(1, 128), (2, 64), (8, 128), (32, 128), (49, 128), (50, 128)])
@pytest.mark.parametrize("train", [0, 1])
def test_a_workspace_serves_every_smaller_plan(lib, H, dv, train):
    """A program that allocates once for its largest step passes the same workspace with every smaller plan."""
    def size(n, tokens):
        return lib.deltalog_scan_workspace_bytes(ctypes.byref(_desc(H=H, d_k=128, d_v=dv).c_struct()), n, tokens, train)

    ns, tokens = (1, 2, 3, 4, 7, 13, 49, 50, 148, 149), (0, 1, 64, 1400, 1408, 1471, 1472, 1535, 1536, 1600, 5000, 16384)
    sizes = {(n, t): size(n, t) for n in ns for t in tokens}
    for (n, t), most in sizes.items():
        for (m, u), less in sizes.items():
            assert less <= most or m > n or u > t, ((m, u), (n, t))


def test_capture_check_sees_leaves_behind_computed_inputs():
    """The leaves that a live eager graph shares with a captured one need not be arguments of the scan: weights are not."""
    from paper_2608_15533_b200 import sequence

    class Node(torch.autograd.Function):
        @staticmethod
        def forward(ctx, *x):
            return sum(x)

        @staticmethod
        def backward(ctx, d):
            return d, d

    w, u, other = (torch.ones(3, requires_grad=True) for _ in range(3))
    x = torch.ones(3)
    out = Node.apply((w * x).exp() + w, u)
    assert {id(t) for t in sequence._leaves([out.grad_fn])} == {id(w), id(u)}
    sequence._eager.add(out.grad_fn)
    for mine in ([w], [u], [x, w * 2], [other * w], [None, (u + other).sum()]):
        with pytest.raises(RuntimeError, match="same leaves"):
            sequence._refuse_capture_beside_eager(mine)
    for mine in ([], [None], [x], [other], [other * 2, x], [w.detach()]):
        sequence._refuse_capture_beside_eager(mine)
    del out     # the graph is gone
    sequence._refuse_capture_beside_eager([w, u, w * 2])
