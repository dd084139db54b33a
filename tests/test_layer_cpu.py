"""The operators around the scan without a GPU: refusals of the C ABI and of the Python layer, workspace sizes, and the
64-bit references against derivatives by differences."""
import ctypes

import pytest
import torch

import layer_reference as ref
import paper_2608_15533_b200 as dl
from paper_2608_15533_b200 import binding, build

INV, SHAPE, OK = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED_SHAPE, binding.OK
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return dl.load_library()


def _plan(**kw):
    # fake, aligned, never dereferenced
    names = ("starts", "chunk_starts", "chunk_seq", "token_seq", "scan_slots", "append_slots", "merge_slots", "totals", "status")
    return binding._Plan(**({"n": 3, "max_tokens": 100} | {x: 0x1000 * (i + 1) for i, x in enumerate(names)} | kw))


def _conv(call, lib, plan=None, desc=None, **kw):
    d = binding._ConvDesc(*({"channels": 64, "width": 4, "io_dtype": dl.BF16, "silu": 1, "num_slots": 4, "hints": 0} | (desc or {})).values())
    p = ctypes.byref(plan or _plan())
    a = dict(window=0x100000, x=0x200000, stride=64, w=0x300000, b=0x400000, out=0x500000, init=0x600000, final=0x700000, dout=0x800000,
             dfinal=0x900000, ws=0xa00000, size=BIG, rows=100, B=2, slots=0x4) | kw
    if call == "step":
        return lib.deltalog_conv_step(ctypes.byref(d), a["window"], a["x"], a["stride"], a["w"], a["b"], a["slots"], a["B"], a["out"], None, None)
    if call == "prefill":
        return lib.deltalog_conv_prefill(ctypes.byref(d), a["window"], p, a["x"], a["stride"], a["w"], a["b"], None, a["out"], None, None)
    if call == "forward":
        return lib.deltalog_conv_forward(ctypes.byref(d), p, a["init"], a["x"], a["stride"], a["w"], a["b"], a["out"], a["final"], None)
    g = binding._ConvGrads(*({"x": 0xb00000, "weight": 0xc00000, "bias": 0xd00000, "init": 0xe00000} | kw.get("grads", {})).values())
    return lib.deltalog_conv_backward(ctypes.byref(d), p, a["init"], a["x"], a["stride"], a["w"], a["b"], a["dout"], a["dfinal"], ctypes.byref(g), a["rows"],
                                      a["ws"], a["size"], None)


def test_conv_refusals(lib):
    before = dl.launch_count()
    for call in ("step", "prefill", "forward", "backward"):
        for desc, code in ((dict(channels=0), INV), (dict(channels=60), SHAPE), (dict(width=1), SHAPE), (dict(width=5), SHAPE), (dict(io_dtype=2), INV)):
            assert _conv(call, lib, desc=desc) == code, (call, desc)
        for kw in (dict(x=None), dict(w=None), dict(x=0x200008), dict(w=0x300004), dict(b=0x400008), dict(stride=56), dict(stride=68)):
            assert _conv(call, lib, **kw) == INV, (call, kw)
    for call in ("prefill", "forward", "backward"):
        for plan, code in ((_plan(n=-1), INV), (_plan(max_tokens=-1), INV), (_plan(starts=None), INV), (_plan(max_tokens=2 ** 31 - 1), SHAPE)):
            assert _conv(call, lib, plan=plan) == code
        assert _conv(call, lib, plan=_plan(n=0)) == OK  # no rows: nothing to launch
    for call in ("step", "prefill"):
        for kw in (dict(window=None), dict(window=0x100008), dict(out=None), dict(out=0x500004), dict(desc=dict(num_slots=0))):
            assert _conv(call, lib, **kw) == INV
    assert _conv("step", lib, B=-1) == INV and _conv("step", lib, B=0) == OK
    assert _conv("step", lib, B=5, slots=None) == INV       # more rows than the pool has slots, and no list
    assert _conv("forward", lib, out=None) == INV and _conv("forward", lib, init=0x600004) == INV and _conv("forward", lib, final=0x700004) == INV
    for kw in (dict(dout=None), dict(rows=99), dict(ws=None), dict(ws=0xa00008), dict(size=0), dict(dfinal=0x900002), dict(grads=dict(x=None)), dict(grads=dict(weight=None)),
               dict(grads=dict(x=0xb00004))):
        assert _conv("backward", lib, **kw) == INV, kw
    for call in ("prefill", "forward"):   # a run reads what its neighbour owns: never in place
        for out in (0x200000, 0x200010, 0x200000 - 99 * 128):
            assert _conv(call, lib, out=out) == INV
        assert _conv(call, lib, out=0x200000 - 100 * 128, plan=_plan(n=0)) == OK
    assert _conv("backward", lib, grads=dict(x=0x200000)) == INV and _conv("backward", lib, grads=dict(x=0x800000)) == INV
    need = lib.deltalog_conv_workspace_bytes(ctypes.byref(binding._ConvDesc(64, 4, dl.BF16, 1, 4, 0)), 100)
    assert need > 0 and _conv("backward", lib, size=need - 1) == INV
    assert dl.launch_count() == before


def _ssm(call, lib, plan=None, desc=None, **kw):
    d = binding._SsmDesc(*({"channels": 64, "d_state": 16, "groups": 1, "io_dtype": dl.BF16, "softplus": 1, "num_slots": 4, "hints": 0} | (desc or {})).values())
    p = ctypes.byref(plan or _plan())
    a = dict(S=0x100000, out=0x500000, S_init=0x600000, S_final=0x700000, dout=0x800000, dS=0x900000, ws=0xa00000, size=BIG, rows=100, B=2, slots=0x4, save=1) | kw
    i = {"x": 0x200000, "dt": 0x210000, "B": 0x220000, "C": 0x230000, "z": 0x240000, "x_stride": 64, "dt_stride": 64, "B_stride": 16, "C_stride": 16,
         "z_stride": 128, "A": 0x250000, "D": 0x260000, "dt_bias": 0x270000} | kw.get("inputs", {})
    inp = None if kw.get("inputs") == "none" else ctypes.byref(binding._SsmInputs(*i.values()))
    if call == "step":
        return lib.deltalog_ssm_step(ctypes.byref(d), a["S"], inp, a["slots"], a["B"], a["out"], None, None)
    if call == "prefill":
        return lib.deltalog_ssm_prefill(ctypes.byref(d), a["S"], p, inp, None, a["out"], None, a["ws"], a["size"], None)
    if call == "forward":
        return lib.deltalog_ssm_forward(ctypes.byref(d), p, a["S_init"], inp, a["out"], a["S_final"], a["save"], a["ws"], a["size"], None)
    names = ("x", "dt", "B", "C", "z", "A", "D", "dt_bias", "S_init")
    g = binding._SsmGrads(*({n: 0x1000000 * (k + 1) for k, n in enumerate(names)} | kw.get("grads", {})).values())
    return lib.deltalog_ssm_backward(ctypes.byref(d), p, a["S_init"], inp, a["dout"], a["dS"], 0, ctypes.byref(g), a["rows"], a["ws"], a["size"], None)


def test_ssm_refusals(lib):
    before = dl.launch_count()
    for call in ("step", "prefill", "forward", "backward"):
        for desc, code in ((dict(channels=0), INV), (dict(channels=60), SHAPE), (dict(groups=0), INV), (dict(groups=3), SHAPE), (dict(groups=16), SHAPE),
                           (dict(d_state=12), SHAPE), (dict(d_state=128), SHAPE), (dict(io_dtype=7), INV), (dict(channels=1 << 28), SHAPE)):
            assert _ssm(call, lib, desc=desc) == code, (call, desc)
        for name in ("x", "dt", "A", "B", "C"):
            assert _ssm(call, lib, inputs={name: None}) == INV
        for name in ("x", "dt", "A", "B", "C", "z", "D", "dt_bias"):
            assert _ssm(call, lib, inputs={name: 0x200004}) == INV
        for name, bad in (("x_stride", 56), ("dt_stride", 65), ("B_stride", 8), ("C_stride", 17), ("z_stride", 0)):
            assert _ssm(call, lib, inputs={name: bad}) == INV
        assert _ssm(call, lib, inputs={"x_stride": (1 << 25) + 8}) == SHAPE
    for call in ("prefill", "forward", "backward"):
        for plan, code in ((_plan(n=-1), INV), (_plan(starts=None), INV), (_plan(max_tokens=2 ** 31 - 1), SHAPE)):
            assert _ssm(call, lib, plan=plan) == code
        for kw in (dict(ws=None), dict(ws=0xa00004), dict(size=0)):
            assert _ssm(call, lib, **kw) == INV
        assert _ssm(call, lib, plan=_plan(n=0)) == OK
    for call in ("step", "prefill"):
        for kw in (dict(S=None), dict(S=0x100008), dict(out=None), dict(out=0x500004), dict(desc=dict(num_slots=0))):
            assert _ssm(call, lib, **kw) == INV
    assert _ssm("step", lib, S=0x100010) == INV and _ssm("step", lib, inputs={"A": 0x250010}) == INV   # 32-byte accesses
    assert _ssm("step", lib, B=-1) == INV and _ssm("step", lib, B=0) == OK and _ssm("step", lib, B=5, slots=None) == INV
    assert _ssm("forward", lib, out=None) == INV and _ssm("forward", lib, S_init=0x600004) == INV and _ssm("forward", lib, S_final=0x700004) == INV
    for kw in (dict(dout=None), dict(rows=99), dict(dS=0x900004)):
        assert _ssm("backward", lib, **kw) == INV
    for name in ("x", "dt", "B", "C", "z", "A", "D", "dt_bias"):
        assert _ssm("backward", lib, grads={name: None}) == INV
    assert dl.launch_count() == before


def test_ssm_workspaces_grow_with_tokens(lib):
    for ch, n in ((64, 16), (4096, 16), (512, 64), (136, 8)):
        d = binding._SsmDesc(ch, n, 1, dl.BF16, 1, 4, 0)
        for train in (0, 1):
            sizes = [lib.deltalog_ssm_workspace_bytes(ctypes.byref(d), 5, t, train) for t in (0, 1, 127, 128, 129, 500, 1000, 1001, 5000, 20000)]
            assert all(0 < x <= y for x, y in zip(sizes, sizes[1:]))
    assert lib.deltalog_ssm_workspace_bytes(ctypes.byref(d), -1, 5, 0) == 0 and lib.deltalog_ssm_workspace_bytes(ctypes.byref(d), 1, -5, 0) == 0


def _norm(call, lib, desc=None, **kw):
    d = {"H_q": 2, "H_k": 1, "d": 64, "io_dtype": dl.BF16, "norm": dl.NORM_RMS, "rot": 64, "interleaved": 0, "table_rows": 9, "eps": 1e-6, "q_scale": 1.0} | (desc or {})
    a = dict(q=0x100000, qs=128, k=0x200000, ks=64, wq=0x300000, wk=0x400000, cos=0x500000, sin=0x600000, pos=0x700000, tokens=3, oq=0x800000, ok=0x900000,
             dq=0xa00000, dk=0xb00000, dwq=0xc00000, dwk=0xd00000, ws=0xe00000, size=BIG) | kw
    head = (ctypes.byref(binding._NormDesc(*d.values())), a["q"], a["qs"], a["k"], a["ks"], a["wq"], a["wk"], a["cos"], a["sin"], a["pos"], a["tokens"])
    if call == "forward":
        return lib.deltalog_head_norm_forward(*head, a["oq"], a["ok"], None, None)
    return lib.deltalog_head_norm_backward(*head, a["oq"], a["ok"], a["dq"], a["dk"], a["dwq"], a["dwk"], a["ws"], a["size"], None)


def test_head_norm_refusals(lib):
    before = dl.launch_count()
    for call in ("forward", "backward"):
        for desc, code in ((dict(H_q=0), INV), (dict(H_k=-1), INV), (dict(d=60), SHAPE), (dict(d=264), SHAPE), (dict(rot=24), SHAPE), (dict(rot=80), SHAPE), (dict(rot=-16), SHAPE),
                           (dict(norm=3), INV), (dict(io_dtype=5), INV), (dict(eps=-1.0), INV), (dict(eps=float("nan")), INV), (dict(q_scale=float("inf")), INV),
                           (dict(table_rows=0), INV), (dict(norm=dl.NORM_L2), INV)):     # (weights with a norm that has none)
            assert _norm(call, lib, desc=desc) == code, desc
        for kw in (dict(q=None), dict(q=0x100008), dict(qs=120), dict(qs=132), dict(k=None), dict(ks=32), dict(wq=None), dict(wk=None), dict(wq=0x300004), dict(cos=None), dict(sin=None),
                   dict(pos=None), dict(cos=0x500004), dict(tokens=-1), dict(oq=None), dict(ok=None), dict(oq=0x800008)):
            assert _norm(call, lib, **kw) == INV, kw
    assert _norm("forward", lib, tokens=0) == OK
    for kw in (dict(dq=None), dict(dk=0xb00004), dict(dwq=None), dict(dwk=None), dict(ws=None), dict(ws=0xe00008), dict(size=16)):
        assert _norm("backward", lib, **kw) == INV, kw
    assert _norm("backward", lib, tokens=1 << 30, desc=dict(H_q=64, H_k=64, d=256, rot=0), qs=64 * 256, ks=64 * 256) == SHAPE
    assert dl.launch_count() == before


def test_python_layer_names_what_it_refuses():
    d = torch.device("cpu")
    conv, ssm = dl.ConvDesc(64, 4, num_slots=3), dl.SsmDesc(64, 16, num_slots=3)
    cs, ss = dl.ConvState(conv, device=d), dl.SsmState(ssm, device=d)
    x, w = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(64, 4)
    step = lambda **kw: dl.conv_step(*[{**dict(desc=conv, state=cs, x=x, weight=w), **kw}[k] for k in ("desc", "state", "x", "weight")],
                                     **{k: v for k, v in kw.items() if k in ("bias", "slot_idx", "out")})
    for kw, name in ((dict(x=x.float()), "x:"), (dict(x=x[:, :32]), "x:"), (dict(x=None), "x:"), (dict(x=torch.zeros(2, 128, dtype=torch.bfloat16)[:, ::2]), "x:"),
                     (dict(x=torch.zeros(2, 68, dtype=torch.bfloat16)[:, :64]), "x:"), (dict(x=x[:1].expand(2, 64)), "x:"), (dict(weight=w[:, :3]), "weight:"),
                     (dict(weight=w.t().contiguous().t()), "weight:"), (dict(bias=torch.zeros(63)), "bias:"), (dict(slot_idx=torch.zeros(2)), "slot_idx:"),
                     (dict(x=torch.zeros(4, 64, dtype=torch.bfloat16)), "slot_idx:"), (dict(out=torch.zeros(2, 64)), "out:"), (dict(desc=dl.ConvDesc(64, 3, num_slots=3), weight=w[:, :3].contiguous()), "state:"),
                     (dict(), "cpu")):  # all well: there is no path but the GPU's
        with pytest.raises(ValueError, match=name):
            step(**kw)
    plan = dl.Plan(2, 10, device=d)
    t = torch.zeros(10, 64, dtype=torch.bfloat16)
    bc, A = torch.zeros(10, 1, 16, dtype=torch.bfloat16), torch.zeros(64, 16)
    for call in (lambda **kw: dl.ssm_prefill(ssm, ss, plan, **{**good, **kw}), lambda **kw: dl.ssm_forward(ssm, plan, **{**good, **kw}),
                 lambda **kw: dl.ssm_backward(ssm, plan, **{**good, "D": None, "z": None, "dt_bias": None, "dout": t, **kw})):
        good = dict(x=t, dt=t, A=A, B=bc, C=bc)
        for kw, name in ((dict(x=t[:9]), "x:"), (dict(dt=t[:9]), "dt:"), (dict(A=A[:8]), "A:"), (dict(B=bc[:, 0]), "B:"), (dict(C=bc.float()), "C:"), (dict(z=t.float()), "z:"),
                         (dict(D=torch.zeros(8)), "D:"), (dict(dt_bias=torch.zeros(64, 1)), "dt_bias:"), (dict(), "cpu")):
            with pytest.raises(ValueError, match=name):
                call(**kw)
    odd = torch.zeros(64 * 16 + 8)
    odd = odd[next(i for i in range(8) if (odd.data_ptr() + 4 * i) % 32 == 16):][: 64 * 16].view(64, 16)
    with pytest.raises(ValueError, match="32-byte"):
        dl.ssm_step(ssm, ss, t[:2], t[:2], odd, bc[:2], bc[:2])
    with pytest.raises(ValueError, match="workspace"):
        dl.ssm_forward(ssm, plan, t, t, A, bc, bc, save=True)
    with pytest.raises(ValueError, match="workspace"):
        dl.ssm_backward(ssm, plan, t, t, A, bc, bc, None, None, None, t, saved=True)
    nd = dl.NormDesc(2, 1, 64)
    q, k = torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 1, 64, dtype=torch.bfloat16)
    cos = torch.zeros(7, 32)
    rot = dl.NormDesc(2, 1, 64, norm=dl.NORM_RMS, rot=64)
    pos = torch.zeros(5, dtype=torch.int32)
    for args, name in (((nd, q[:, :1], k), "q:"), ((nd, q, k[:4]), "k:"), ((nd, q, None), "k:"), ((nd, q, k, torch.ones(64), torch.ones(64)), "w_q, w_k"),
                       ((rot, q, k, torch.ones(64), None, cos, cos, pos), "w_q, w_k"), ((rot, q, k, torch.ones(32), torch.ones(64), cos, cos, pos), "w_q:"),
                       ((rot, q, k, None, None, None, cos, pos), "cos:"), ((rot, q, k, None, None, cos, cos[:6], pos), "sin:"), ((rot, q, k, None, None, cos, cos, pos[:4]), "positions:"),
                       ((rot, q, k, None, None, cos, cos, pos.long()), "positions:"), ((dl.NormDesc(2, 0, 64), q, k), "k:"), ((nd, q, k), "cpu")):
        with pytest.raises(ValueError, match=name):
            dl.head_norm_forward(*args)
    with pytest.raises(ValueError, match="gradient"):
        dl.head_norm(rot, q, k, None, None, cos.requires_grad_(), cos, pos)


def test_tangents_are_refused():
    plan = dl.Plan(1, 4, device="cpu")
    t = torch.zeros(4, 64, dtype=torch.bfloat16)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(t, torch.ones_like(t))
        with pytest.raises(RuntimeError, match="forward-mode"):
            dl.conv(dl.ConvDesc(64), plan, dual, torch.zeros(64, 4))
        with pytest.raises(RuntimeError, match="forward-mode"):
            dl.ssm(dl.SsmDesc(64), plan, dual, t, torch.zeros(64, 16), t, t)
        with pytest.raises(RuntimeError, match="forward-mode"):
            dl.head_norm(dl.NormDesc(1, 0, 64), dual.unflatten(1, (1, 64)), None)


def test_a_changed_descriptor_is_seen():
    d = dl.ConvDesc(64, 4)
    assert d.c_struct().silu == 1 and d.c_struct(True).hints == dl.HINT_ZERO_UNWRITTEN and d.c_struct() is d.c_struct()
    d.silu = False
    assert d.c_struct().silu == 0 and d.c_struct(True).silu == 0
    n = dl.NormDesc(1, 1, 64)
    assert n.c_struct(5).table_rows == 5 and n.c_struct(7).table_rows == 7
    n.q_scale = 0.5
    assert n.c_struct(7).q_scale == 0.5


# ---- the references themselves, against differences -----------------------------------------------------------------------
def _difference(f, x, v, h=1e-6):
    return float((f(x + h * v) - f(x - h * v)) / (2 * h))


def test_reference_gradients_against_differences():
    gen = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=gen, dtype=ref.F64)
    lens, D, N, G = (3, 0, 5), 16, 8, 2
    T = sum(lens)
    case = dict(x=rnd(T, D), dt=rnd(T, D), A=-torch.rand(D, N, generator=gen, dtype=ref.F64) - 0.1, B=rnd(T, G, N), C=rnd(T, G, N), D=rnd(D), z=rnd(T, D), dt_bias=rnd(D), softplus=True)
    S0, dout, dS = rnd(3, D, N), rnd(T, D), rnd(3, D, N)
    grads = ref.ssm(case, lens, S0, dout, dS)[2]

    def loss(**kw):
        c = case | {k: v for k, v in kw.items() if k != "S_init"}
        out, S, _ = ref.ssm(c, lens, kw.get("S_init", S0))
        return (out * dout).sum() + (S * dS).sum()

    for name in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "S_init"):
        at = S0 if name == "S_init" else case[name]
        v = rnd(*at.shape)
        want = _difference(lambda t: loss(**{name: t}), at, v)
        assert abs(float((grads[name] * v).sum()) - want) < 1e-7 * max(1, abs(want)), name
    for act in (False, True):
        for n in (0, 1, 2, 7):
            x, w, b, init, do, df = rnd(n, 8), rnd(8, 4), rnd(8), rnd(3, 8), rnd(n, 8), rnd(3, 8)
            args = [x, w, b, init]
            for i, g in enumerate(ref.conv_row_grad(x, w, b, init, act, do, df)):
                v = rnd(*args[i].shape)

                def value(t):
                    _, out, final = ref.conv_row(*[t if j == i else args[j] for j in range(4)], act)
                    return (out * do).sum() + (final * df).sum()

                assert abs(float((g * v).sum()) - _difference(value, args[i], v)) < 1e-7


def test_pools_of_a_changed_descriptor_are_refused():
    """A descriptor that grows behind its pool's back would send slots past the pool's end."""
    def conv(desc, state):
        x = torch.zeros(1, 64, dtype=torch.bfloat16)
        return dl.conv_step(desc, state, x, torch.zeros(64, 4))

    def ssm(desc, state):
        x, bc = torch.zeros(1, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 16, dtype=torch.bfloat16)
        return dl.ssm_step(desc, state, x, x, torch.zeros(64, 16), bc, bc)

    for desc, pool, call in ((dl.ConvDesc(64, num_slots=4), dl.ConvState, conv), (dl.SsmDesc(64, num_slots=4), dl.SsmState, ssm)):
        state = pool(desc, device="cpu")
        desc.num_slots = 5
        with pytest.raises(ValueError, match="another descriptor"):
            call(desc, state)
        desc.num_slots = 4
        with pytest.raises(ValueError, match="GPU"):  # it fits again: the device is what is wrong now
            call(desc, state)


@pytest.mark.parametrize("pool,desc,name", [(dl.ConvState, dl.ConvDesc(64), "window"), (dl.SsmState, dl.SsmDesc(64), "S")])
def test_pool_tensors_are_not_replaced(pool, desc, name):
    state = pool(desc, device="cpu")
    for field in (name, "status"):  # the calls would go on with the old one
        with pytest.raises(AttributeError):
            setattr(state, field, getattr(state, field).clone())


def test_more_rows_than_31_bits_are_refused(lib):
    most = 2 ** 31 - 64
    assert _conv("backward", lib, x=1 << 44, grads=dict(x=1 << 50), dout=1 << 47, rows=most) == SHAPE
    desc, weight = dl.ConvDesc(8), torch.zeros(8, 4)
    x = torch.empty(1, 8, dtype=torch.bfloat16).expand(most, 8)  # (no such memory is needed to be asked)
    with pytest.raises(ValueError, match="x: .* rows"):
        dl.conv_step(desc, dl.ConvState(desc, device="cpu"), x, weight)


def test_head_norm_of_host_tensors_is_refused():
    q = torch.zeros(3, 1, 16, requires_grad=True)
    with pytest.raises(ValueError, match="GPU"):
        dl.head_norm(dl.NormDesc(1, 0, 16, io_dtype=dl.F32), q, None)
