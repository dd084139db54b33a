"""Cases of the operators that a recurrent layer runs around and beside its scan: the short causal convolution, the selective
state space scan, and the norm of query and key heads with their rotation; packed prompts, training steps and single tokens.

``own`` false: the plain form, elementary torch operations in fp32.  ``own`` true: the calls a user makes of this package.
``exact`` is the definition in fp64: token by token for the scan, row by row for the convolution, complex numbers for the
rotation.
"""
import math
import random

import torch

own = False

BLOCK = 1 << 27  # elements of one [tokens, channels, states] tensor of the plain scan


# ---------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one request's next token through the convolution in front of a small layer: call latency
        dict(name="conv_step_small", kind="conv_step", dtype="bf16", n=2, C=1024, W=4, silu=True, bias=True),
        # a decode batch, queries, keys and values of 32 heads of 128 in one convolution
        dict(name="conv_step_batch", kind="conv_step", dtype="bf16", n=250, C=12288, W=4, silu=True, bias=False),
        # a serving step's prompts, ragged, half of them continuing a conversation
        dict(name="conv_prefill_ragged", kind="conv_prefill", dtype="bf16", n=48, lo=1, hi=1500, C=8192, W=4, silu=True, bias=False, lens=1),
        # a training step's documents: forward and gradients
        dict(name="conv_train", kind="conv_train", dtype="bf16", n=11, lo=500, hi=2800, C=4096, W=4, silu=True, bias=True, lens=2),
        # a decode batch of a state space layer
        dict(name="ssm_step_batch", kind="ssm_step", dtype="bf16", n=125, D=4096, N=16, G=1, gate=True, skip=True, softplus=True),
        # one short prompt of a small fp32 layer: call latency
        dict(name="ssm_prefill_fp32_small", kind="ssm_prefill", dtype="fp32", n=1, lo=67, hi=67, D=128, N=16, G=1, gate=True, skip=True, softplus=True, lens=3),
        # a serving step's prompts, ragged, half of them continuing
        dict(name="ssm_prefill_ragged", kind="ssm_prefill", dtype="bf16", n=24, lo=1, hi=1500, D=4096, N=16, G=1, gate=True, skip=True, softplus=True, lens=4),
        # one long document: the chain over its tokens counts
        dict(name="ssm_prefill_long", kind="ssm_prefill", dtype="bf16", n=1, lo=16384, hi=16384, D=2048, N=16, G=1, gate=True, skip=True, softplus=True, lens=5),
        # training steps: forward and gradients of packed documents
        dict(name="ssm_train", kind="ssm_train", dtype="bf16", n=4, lo=2048, hi=2048, D=4096, N=16, G=1, gate=True, skip=True, softplus=True, lens=6),
        dict(name="ssm_train_ragged", kind="ssm_train", dtype="bf16", n=9, lo=30, hi=900, D=2560, N=32, G=2, gate=False, skip=True, softplus=True, lens=7),
        # a decode batch's queries and keys on their way into a delta rule step: unit length, no rotation
        dict(name="norm_step", kind="norm", train=False, dtype="bf16", T=250, Hq=16, Hk=16, d=128, mode="l2", rot=0, pairs="half", far=1),
        # training tokens of a layer with normalised and rotated heads, few key heads
        dict(name="norm_train", kind="norm", train=True, dtype="bf16", T=16383, Hq=32, Hk=8, d=128, mode="rms", rot=128, pairs="half", far=40000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("conv_step", "conv_prefill", "conv_train", "ssm_step", "ssm_prefill", "ssm_prefill", "ssm_train", "ssm_train", "norm", "norm"))
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    lens = rng.randrange(1 << 30)
    if kind == "norm":
        d = rng.choice((32, 64, 96, 128, 256))
        Hq, Hk = rng.choice((1, 2, 3, 4, 8, 12, 16, 24, 32)), rng.choice((1, 2, 3, 4, 8, 16))
        T = _log(rng, 1, min(16000, 60_000_000 // ((Hq + Hk) * d * 4)))
        rot = rng.choice((0, d // 32 * 16, d))
        return dict(kind=kind, train=rng.random() < 0.5, dtype=dtype, T=T, Hq=Hq, Hk=Hk, d=d, mode=rng.choice(("l2", "rms", "none") if rot else ("l2", "rms")),
                    rot=rot, pairs=rng.choice(("half", "interleaved")), far=_log(rng, 1, 200000))
    step = kind.endswith("step")
    n = _log(rng, 1, 250) if step else _log(rng, 1, 48)
    if kind.startswith("conv"):
        C = 8 * _log(rng, 4, 1500 if step else 1000)
        case = dict(kind=kind, dtype=dtype, n=n, C=C, W=rng.choice((2, 3, 4, 4)), silu=rng.random() < 0.8, bias=rng.random() < 0.5)
        most = 150_000_000 if kind == "conv_prefill" else 50_000_000
    else:
        G = rng.choice((1, 1, 1, 2, 4))
        D, N = 8 * G * _log(rng, 8, 512 // G), rng.choice((8, 16, 16, 32, 64))
        case = dict(kind=kind, dtype=dtype, n=n, D=D, N=N, G=G, gate=rng.random() < 0.7, skip=rng.random() < 0.8, softplus=rng.random() < 0.8)
        C, most = D * N, 350_000_000
        if step:
            case["n"] = max(1, min(n, 8_000_000 // C))
    if step:
        return case
    hi = max(1, min(_log(rng, 1, 8000), most // (n * C)))
    return dict(case, lo=rng.randint(0 if kind.endswith("prefill") else 1, hi), hi=hi, lens=lens)


def _lens(case):
    """Row lengths of a case, from the case alone."""
    r = random.Random(case["lens"])
    lens = [r.randint(case["lo"], case["hi"]) for _ in range(case["n"])]
    lens[0] = case["hi"]
    return lens


# ---------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    io = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    kind = case["kind"]

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    st = dict(case=case)
    if kind == "norm":
        T, Hq, Hk, d = case["T"], case["Hq"], case["Hk"], case["d"]
        # queries and keys are columns of one projection, in front of the values
        proj = randn(T, Hq + 2 * Hk, d).to(io)
        st |= dict(q=proj[:, :Hq], k=proj[:, Hq : Hq + Hk], wq=None, wk=None, cos=None, sin=None, positions=None, q_scale=d ** -0.5)
        if case["mode"] == "rms":
            st |= dict(wq=1 + 0.2 * randn(d), wk=1 + 0.2 * randn(d))
        if case["rot"]:
            half, far = case["rot"] // 2, case["far"]
            angle = torch.arange(far, dtype=torch.float64, device="cuda")[:, None] * torch.pow(10000.0, -torch.arange(half, dtype=torch.float64, device="cuda") / half)
            st |= dict(cos=angle.cos().float(), sin=angle.sin().float(), positions=torch.randint(0, far, (T,), generator=gen, device="cuda", dtype=torch.int32))
        if case["train"]:
            st |= dict(dq=randn(T, Hq, d).to(io), dk=randn(T, Hk, d).to(io))
        return st

    n = case["n"]
    if kind.endswith("step"):
        T = n
    else:
        lens = _lens(case)
        T = sum(lens)
        ln = torch.tensor(lens, device="cuda")
        st |= dict(lens_host=lens, lens=ln.to(torch.int32), first=torch.cumsum(ln, 0) - ln, row=torch.repeat_interleave(torch.arange(n, device="cuda"), ln, output_size=T))
        st["at"] = torch.arange(T, device="cuda") - st["first"][st["row"]]  # a token's place in its row
    st["T"] = T
    if not kind.endswith("train"):
        slots = n + 1 + n // 8
        st["slots"] = torch.randperm(slots, generator=gen, device="cuda")[:n].to(torch.int32)
    if kind.endswith("prefill"):
        st["fresh"] = (torch.arange(n, device="cuda") % 2).to(torch.int32)
    if kind.startswith("conv"):
        C, W = case["C"], case["W"]
        st["x"] = randn(T, C).to(io)
        st["w"], st["b"] = randn(C, W) * W ** -0.5, randn(C) * 0.1 if case["bias"] else None
        if kind == "conv_train":
            st |= dict(init=randn(n, W - 1, C).to(io), dout=randn(T, C).to(io), dfinal=randn(n, W - 1, C).to(io))
        else:
            st["pool"] = randn(slots, W - 1, C).to(io)
        return st
    D, N, G = case["D"], case["N"], case["G"]
    R = 8 * ((D // 32 + 7) // 8)
    st["x"] = torch.nn.functional.silu(randn(T, D)).to(io)
    # the gate is the second half of the layer's input projection; B and C follow the low-rank step size in another one
    st["z"] = randn(T, 2 * D).to(io)[:, D:] if case["gate"] else None
    bc = randn(T, R + 2 * G * N).to(io)
    st["B"], st["C"] = bc[:, R : R + G * N].unflatten(1, (G, N)), bc[:, R + G * N :].unflatten(1, (G, N))
    st["A"] = -torch.arange(1, N + 1, device="cuda") * torch.exp(0.2 * randn(D, N))
    st["skip"] = 1 + 0.1 * randn(D) if case["skip"] else None
    step = torch.exp(rand(D) * math.log(100.0) + math.log(1e-3))  # step sizes from 0.001 to 0.1
    if case["softplus"]:
        st["bias"] = step + torch.log(-torch.expm1(-step))
        st["dt"] = (randn(T, D) * 0.5).to(io)
    else:
        st["bias"] = None
        st["dt"] = (step * torch.exp(0.5 * randn(T, D))).to(io)
    if kind == "ssm_train":
        st |= dict(S0=randn(n, D, N) * 0.1, dout=randn(T, D).to(io), dS=randn(n, D, N) * 0.1)
    else:
        st["pool"] = randn(slots, D, N) * 0.1
    return st


# ---------------------------------------------------------------------------------------------------- plain forms
def _plain_conv(x, w, b, init, st, silu):
    """out [T, C] and the last W - 1 inputs of each row, fp32."""
    W, T = w.shape[1], x.shape[0]
    at, row, ln, first = st["at"], st["row"], st["lens"].long(), st["first"]
    out = x * w[:, W - 1]
    for back in range(1, W):
        inside = (at >= back)[:, None]
        past = torch.cat((torch.zeros_like(x[:back]), x[: T - back]))[:T] * inside
        early = torch.nonzero(at < back)[:, 0]
        past = past.index_add(0, early, init[row[early], W - 1 + at[early] - back])
        out = out + past * w[:, W - 1 - back]
    if b is not None:
        out = out + b
    if silu:
        out = out / (1 + torch.exp(-out))
    final = []
    for i in range(W - 1):
        p = ln - (W - 1) + i
        old = init[torch.arange(len(ln), device="cuda"), (W - 1 + p).clamp(0, W - 2)]
        final.append(torch.where((p >= 0)[:, None], x[(first + p).clamp(0, max(T - 1, 0))], old) if T else old)
    return out, torch.stack(final, 1)


def _plain_conv_step(st):
    c, slots = st["case"], st["slots"].long()
    seen = torch.cat((st["pool"][slots], st["x"][:, None]), 1)
    out = (seen.float() * st["w"].t()).sum(1)
    if st["b"] is not None:
        out = out + st["b"]
    if c["silu"]:
        out = out / (1 + torch.exp(-out))
    st["pool"][slots] = seen[:, 1:]
    return out.to(st["x"].dtype), st["pool"]


def _plain_conv_prefill(st):
    io, slots = st["x"].dtype, st["slots"].long()
    init = st["pool"][slots].float() * (st["fresh"] == 0)[:, None, None]
    out, final = _plain_conv(st["x"].float(), st["w"], st["b"], init, st, st["case"]["silu"])
    some = st["lens"] > 0
    st["pool"][slots[some]] = final[some].to(io)
    return out.to(io), st["pool"]


def _plain_conv_train(st):
    io = st["x"].dtype
    leaf = [t if t is None else t.float().detach().requires_grad_() for t in (st["x"], st["w"], st["b"], st["init"])]
    out, final = _plain_conv(*leaf, st, st["case"]["silu"])
    g = list(torch.autograd.grad((out, final), [t for t in leaf if t is not None], (st["dout"].float(), st["dfinal"].float())))
    res = dict(out=out.detach().to(io), final=final.detach().to(io), dx=g[0].to(io), dw=g[1], dinit=g[-1].to(io))
    return res | (dict(db=g[2]) if st["b"] is not None else {})


def _plain_delta(dt, bias, softplus):
    v = dt.float() if bias is None else dt.float() + bias
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs())) if softplus else v


def _running(a, b, most):
    """h_t = a_t h_(t-1) + b_t along the first axis, over stretches of at most `most` tokens (a is zero where one begins)."""
    s = 1
    while s < most:
        b = torch.cat((b[:s], torch.addcmul(b[s:], a[s:], b[:-s])))
        a = torch.cat((a[:s], a[s:] * a[:-s]))
        s *= 2
    return b


def _plain_ssm(st, S0, grads=False):
    c, T = st["case"], st["T"]
    D, N, G = c["D"], c["N"], c["G"]
    row, at, ln = st["row"], st["at"], st["lens"].long()
    most = max(st["lens_host"])
    begins, rows = torch.nonzero(at == 0)[:, 0], torch.nonzero(ln > 0)[:, 0]
    ends = begins + ln[rows] - 1
    out, S = torch.empty(T, D, device="cuda"), S0.clone()
    res = {}
    if grads:
        io = st["x"].dtype
        res = dict(dx=torch.empty(T, D, dtype=io, device="cuda"), ddt=torch.empty(T, D, dtype=io, device="cuda"), dA=torch.empty(D, N, device="cuda"),
                   dB=torch.zeros(T, G, N, device="cuda"), dC=torch.zeros(T, G, N, device="cuda"), dS0=st["dS"].clone())
        res |= dict(dz=torch.empty(T, D, dtype=io, device="cuda")) if st["z"] is not None else {}
        res |= dict(dD=torch.empty(D, device="cuda")) if st["skip"] is not None else {}
        res |= dict(dbias=torch.empty(D, device="cuda")) if st["bias"] is not None else {}
    per = D // G
    width = max(1, min(per, BLOCK // max(1, T * N)))
    for lo in [g * per + i for g in range(G) for i in range(0, per, width)]:
        g = lo // per
        cut = slice(lo, min(lo + width, (g + 1) * per))
        x, A = st["x"][:, cut].float(), st["A"][cut]
        B, C = st["B"][:, g, None].float(), st["C"][:, g, None].float()
        bias = None if st["bias"] is None else st["bias"][cut]
        delta = _plain_delta(st["dt"][:, cut], bias, c["softplus"])
        a = torch.exp(delta[..., None] * A)
        b = (delta * x)[..., None] * B
        keep = a.clone()
        b[begins] += a[begins] * S0[rows][:, cut]
        keep[begins] = 0
        h = _running(keep, b, most)
        S[rows[:, None], torch.arange(cut.start, cut.stop, device="cuda")] = h[ends]
        y = (h * C).sum(-1)
        if st["skip"] is not None:
            y = y + x * st["skip"][cut]
        if st["z"] is not None:
            z = st["z"][:, cut].float()
            sig = 1 / (1 + torch.exp(-z))
        out[:, cut] = y * z * sig if st["z"] is not None else y
        if not grads:
            continue
        dy = st["dout"][:, cut].float()
        if st["z"] is not None:
            res["dz"][:, cut] = (dy * y * sig * (1 + z * (1 - sig))).to(io)
            dy = dy * z * sig
        e = dy[..., None] * C
        e[ends] += st["dS"][rows][:, cut]
        nxt = torch.cat((keep[1:], torch.zeros_like(keep[:1])))       # the decay into the next token of the row
        dh = _running(nxt.flip(0), e.flip(0), most).flip(0)
        prev = torch.cat((torch.zeros_like(h[:1]), h[:-1]))
        prev[begins] = S0[rows][:, cut]
        res["dC"][:, g] += (dy[..., None] * h).sum(1)
        res["dB"][:, g] += (dh * (delta * x)[..., None]).sum(1)
        sB = (dh * B).sum(-1)
        dx = delta * sB
        if st["skip"] is not None:
            dx = dx + dy * st["skip"][cut]
            res["dD"][cut] = (dy * x).sum(0)
        res["dx"][:, cut] = dx.to(io)
        w = dh * prev * a
        res["dA"][cut] = (w * delta[..., None]).sum(0)
        ddt = (w * A).sum(-1) + x * sB
        if c["softplus"]:
            v = st["dt"][:, cut].float() if bias is None else st["dt"][:, cut].float() + bias
            ddt = ddt / (1 + torch.exp(-v))
        res["ddt"][:, cut] = ddt.to(io)
        if bias is not None:
            res["dbias"][cut] = ddt.sum(0)
        res["dS0"][rows[:, None], torch.arange(cut.start, cut.stop, device="cuda")] = a[begins] * dh[begins]
    if grads:
        res["dB"], res["dC"] = res["dB"].to(io), res["dC"].to(io)
    return out, S, res


def _plain_ssm_step(st):
    c, slots = st["case"], st["slots"].long()
    x = st["x"].float()
    B, C = (t.float().repeat_interleave(c["D"] // c["G"], 1) for t in (st["B"], st["C"]))
    delta = _plain_delta(st["dt"], st["bias"], c["softplus"])
    S = torch.exp(delta[..., None] * st["A"]) * st["pool"][slots] + (delta * x)[..., None] * B
    y = (S * C).sum(-1)
    if st["skip"] is not None:
        y = y + x * st["skip"]
    if st["z"] is not None:
        z = st["z"].float()
        y = y * z / (1 + torch.exp(-z))
    st["pool"][slots] = S
    return y.to(st["x"].dtype), st["pool"]


def _plain_ssm_prefill(st):
    slots = st["slots"].long()
    S0 = st["pool"][slots] * (st["fresh"] == 0)[:, None, None]
    out, S, _ = _plain_ssm(st, S0)
    some = st["lens"] > 0
    st["pool"][slots[some]] = S[some]
    return out.to(st["x"].dtype), st["pool"]


def _plain_ssm_train(st):
    out, S, res = _plain_ssm(st, st["S0"], grads=True)
    return dict(out=out.to(st["x"].dtype), S=S) | res


def _plain_heads(x, w, scale, st):
    c = st["case"]
    rot, half = c["rot"], c["rot"] // 2
    if c["mode"] == "rms":
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
    elif c["mode"] == "l2":
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) + 1e-6)
    if rot:
        p = st["positions"].long()
        cos, sin = st["cos"][p][:, None], st["sin"][p][:, None]
        if c["pairs"] == "half":
            u, v = x[..., :half], x[..., half:rot]
            turned = torch.cat((u * cos - v * sin, v * cos + u * sin), -1)
        else:
            u, v = x[..., 0:rot:2], x[..., 1:rot:2]
            turned = torch.stack((u * cos - v * sin, v * cos + u * sin), -1).flatten(-2)
        x = torch.cat((turned, x[..., rot:]), -1)
    return x * scale


def _norm_train(st, heads, f):
    """Outputs and gradients of both tensors by differentiating `heads` in the type `f`."""
    io, names, leaves = st["q"].dtype, ("q", "k", "wq", "wk"), []
    for name in names:
        leaves.append(None if st[name] is None else st[name].to(f).detach().requires_grad_())
    q, k, wq, wk = leaves
    oq, ok = heads(q, wq, st["q_scale"], st), heads(k, wk, 1.0, st)
    g = torch.autograd.grad((oq, ok), [t for t in leaves if t is not None], (st["dq"].to(f), st["dk"].to(f)))
    res = dict(zip(("d" + name for name, t in zip(names, leaves) if t is not None), g))
    return dict(q=oq.detach(), k=ok.detach()) | res, io


def _plain_norm(st):
    if not st["case"]["train"]:
        io = st["q"].dtype
        return dict(q=_plain_heads(st["q"].float(), st["wq"], st["q_scale"], st).to(io), k=_plain_heads(st["k"].float(), st["wk"], 1.0, st).to(io))
    res, io = _norm_train(st, _plain_heads, torch.float32)
    return {k: v if k in ("dwq", "dwk") else v.to(io) for k, v in res.items()}


# ---------------------------------------------------------------------------------------------------- the package's calls
def _handle(st):
    """What a program keeps between steps: descriptors, the pool, the plan that all layers of a step share, workspaces."""
    if "handle" not in st:
        import paper_2608_15533_b200 as dl

        c = st["case"]
        kind, io = c["kind"], dl.F32 if c["dtype"] == "fp32" else dl.BF16
        h = dict(dl=dl)
        if kind == "norm":
            norm = {"rms": dl.NORM_RMS, "l2": dl.NORM_L2, "none": dl.NORM_NONE}[c["mode"]]
            h["desc"] = dl.NormDesc(H_q=c["Hq"], H_k=c["Hk"], d=c["d"], io_dtype=io, norm=norm, eps=1e-6, rot=c["rot"],
                                    interleaved=c["pairs"] == "interleaved", q_scale=st["q_scale"])
            st["handle"] = h
            return h
        slots = st["pool"].shape[0] if "pool" in st else 1
        if kind.startswith("conv"):
            h["desc"] = dl.ConvDesc(channels=c["C"], width=c["W"], io_dtype=io, silu=c["silu"], num_slots=slots)
            if "pool" in st:
                h["pool"] = dl.ConvState(h["desc"], st["pool"])
        else:
            h["desc"] = dl.SsmDesc(channels=c["D"], d_state=c["N"], groups=c["G"], io_dtype=io, softplus=c["softplus"], num_slots=slots)
            if "pool" in st:
                h["pool"] = dl.SsmState(h["desc"], st["pool"])
        if not kind.endswith("step"):
            h["plan"] = dl.build_plan(st["lens"], dl.Plan(c["n"], st["T"], device="cuda"), slots=st.get("slots"))
            if kind.startswith("ssm"):
                h["work"] = dl.ssm_workspace(h["desc"], c["n"], st["T"], train=kind == "ssm_train", device="cuda")
        st["handle"] = h
    return st["handle"]


def _own_conv_step(st):
    h = _handle(st)
    return h["dl"].conv_step(h["desc"], h["pool"], st["x"], st["w"], st["b"], slot_idx=st["slots"]), st["pool"]


def _own_conv_prefill(st):
    h = _handle(st)
    return h["dl"].conv_prefill(h["desc"], h["pool"], h["plan"], st["x"], st["w"], st["b"], fresh=st["fresh"]), st["pool"]


def _own_conv_train(st):
    h = _handle(st)
    args = (h["desc"], h["plan"], st["x"], st["w"], st["b"])
    out, final = h["dl"].conv_forward(*args, init=st["init"])
    d = h["dl"].conv_backward(*args, st["dout"], init=st["init"], dfinal=st["dfinal"])
    res = dict(out=out, final=final, dx=d.x, dw=d.weight, dinit=d.init)
    return res | (dict(db=d.bias) if st["b"] is not None else {})


def _ssm_args(st):
    return [st[x] for x in ("x", "dt", "A", "B", "C", "skip", "z", "bias")]


def _own_ssm_step(st):
    h = _handle(st)
    return h["dl"].ssm_step(h["desc"], h["pool"], *_ssm_args(st), slot_idx=st["slots"]), st["pool"]


def _own_ssm_prefill(st):
    h = _handle(st)
    return h["dl"].ssm_prefill(h["desc"], h["pool"], h["plan"], *_ssm_args(st), fresh=st["fresh"], workspace=h["work"]), st["pool"]


def _own_ssm_train(st):
    h = _handle(st)
    args = (h["desc"], h["plan"], *_ssm_args(st))
    out, S = h["dl"].ssm_forward(*args, S_init=st["S0"], workspace=h["work"], save=True)
    d = h["dl"].ssm_backward(*args, st["dout"], S_init=st["S0"], dS_final=st["dS"], workspace=h["work"], saved=True)
    res = dict(out=out, S=S, dx=d.x, ddt=d.dt, dA=d.A, dB=d.B, dC=d.C, dS0=d.S_init)
    return res | {k: v for k, v in (("dz", d.z), ("dD", d.D), ("dbias", d.dt_bias)) if v is not None}


def _own_norm(st):
    h = _handle(st)
    args = (h["desc"], st["q"], st["k"], st["wq"], st["wk"], st["cos"], st["sin"], st["positions"])
    q, k = h["dl"].head_norm_forward(*args)
    if not st["case"]["train"]:
        return dict(q=q, k=k)
    d = h["dl"].head_norm_backward(*args, st["dq"], st["dk"])
    res = dict(q=q, k=k, dq=d.q, dk=d.k)
    return res | (dict(dwq=d.w_q, dwk=d.w_k) if st["wq"] is not None else {})


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["kind"]](state)


# ---------------------------------------------------------------------------------------------------- work
def work(case):
    e, kind = 4 if case["dtype"] == "fp32" else 2, case["kind"]
    if kind == "norm":
        T, d, H = case["T"], case["d"], case["Hq"] + case["Hk"]
        table = 4 * case["rot"] * min(T, case["far"]) + (4 * T if case["rot"] else 0)  # the positions' rows of both tables
        # a training step reads its inputs once for both directions, and dq and dk; outputs and gradients go out
        return {"bytes": T * H * d * e * (4 if case["train"] else 2) + table, "flops": T * H * d * (20 if case["train"] else 6)}
    n = case["n"]
    T = n if kind.endswith("step") else sum(_lens(case))
    if kind.startswith("conv"):
        C, W = case["C"], case["W"]
        weights, window = 4 * C * (W + case["bias"]), n * (W - 1) * C * e
        if kind == "conv_train":  # x, init, dout, dfinal in; out, final, dx, dinit, dw out
            return {"bytes": T * C * e * 4 + 4 * window + 2 * weights, "flops": T * C * (6 * W + 12)}
        return {"bytes": T * C * e * 2 + 2 * window + weights, "flops": T * C * (2 * W + 4)}
    D, N, G = case["D"], case["N"], case["G"]
    tokens = T * e * (D * (3 + case["gate"]) + 2 * G * N)  # x, dt, z, B, C in, out out
    weights, pool = 4 * D * (N + case["skip"] + case["softplus"]), 4 * n * D * N
    flops = T * D * (N * 7 + 8)
    if kind == "ssm_train":
        return {"bytes": tokens + T * e * (D * (3 + case["gate"]) + 2 * G * N) + 2 * weights + 4 * pool, "flops": flops * 3}
    return {"bytes": tokens + 2 * pool + weights, "flops": flops}


# ---------------------------------------------------------------------------------------------------- 64 bits
def _exact_heads(x, w, scale, st):
    c = st["case"]
    rot = c["rot"]
    if c["mode"] != "none":
        norm = torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2
        x = x * torch.rsqrt((norm / x.shape[-1] if c["mode"] == "rms" else norm) + 1e-6)
        x = x * w if w is not None else x
    if rot:
        p = st["positions"].long()
        turn = torch.complex(st["cos"].double(), st["sin"].double())[p][:, None]
        pairs = x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if c["pairs"] == "half" else x[..., :rot].unflatten(-1, (rot // 2, 2))
        turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        x = torch.cat(((turned.transpose(-1, -2) if c["pairs"] == "half" else turned).flatten(-2), x[..., rot:]), -1)
    return x * scale


def _exact_conv_row(x, w, b, init, silu):
    """One row: x [len, C], init [W - 1, C], fp64."""
    seen = torch.cat((init, x))
    pre = torch.nn.functional.conv1d(seen.t()[None], w[:, None], b, groups=w.shape[0])[0].t()
    return pre * torch.sigmoid(pre) if silu else pre, seen[len(x) :]


def _exact_conv(case, st):
    f, n = torch.float64, case["n"]
    w, b = st["w"].to(f), None if st["b"] is None else st["b"].to(f)
    x = st["x"].to(f)
    if case["kind"] == "conv_step":
        out, pool = torch.empty_like(x), st["pool"].to(f)
        past = pool[st["slots"].long()]
        pre = torch.einsum("ntc,ct->nc", torch.cat((past, x[:, None]), 1), w) + (0 if b is None else b)
        pool[st["slots"].long()] = torch.cat((past[:, 1:], x[:, None]), 1)
        return pre * torch.sigmoid(pre) if case["silu"] else pre, pool
    first = st["first"].tolist()
    rows = [slice(s, s + ln) for s, ln in zip(first, st["lens_host"])]
    if case["kind"] == "conv_prefill":
        out, pool = torch.empty_like(x), st["pool"].to(f)
        for i, r in enumerate(rows):
            if r.stop > r.start:
                s = int(st["slots"][i])
                out[r], pool[s] = _exact_conv_row(x[r], w, b, pool[s] * (1 - i % 2), case["silu"])
        return out, pool
    res = dict(out=torch.empty_like(x), final=torch.empty_like(st["init"], dtype=f), dx=torch.empty_like(x), dw=torch.zeros_like(w), dinit=torch.empty_like(st["init"], dtype=f))
    if b is not None:
        res["db"] = torch.zeros_like(b)
    for i, r in enumerate(rows):
        leaf = [t.detach().clone().requires_grad_() for t in (x[r], w, st["init"][i].to(f)) + (() if b is None else (b,))]
        out, final = _exact_conv_row(leaf[0], leaf[1], leaf[3] if b is not None else None, leaf[2], case["silu"])
        g = torch.autograd.grad((out, final), leaf, (st["dout"][r].to(f), st["dfinal"][i].to(f)))
        res["out"][r], res["final"][i], res["dx"][r], res["dinit"][i] = out.detach(), final.detach(), g[0], g[2]
        res["dw"] += g[1]
        if b is not None:
            res["db"] += g[3]
    return res


def _exact_ssm(case, st):
    f, n, T = torch.float64, case["n"], st["T"]
    D, N, G = case["D"], case["N"], case["G"]
    lens = [1] * n if case["kind"] == "ssm_step" else st["lens_host"]
    train = case["kind"] == "ssm_train"
    order = sorted(range(n), key=lambda i: -lens[i])
    first = [sum(lens[:i]) for i in range(n)]
    begin = torch.tensor([first[i] for i in order], device="cuda")
    live = [sum(1 for ln in lens if ln > t) for t in range(max(lens))]
    A = st["A"].to(f)
    pick = torch.tensor(order, device="cuda")
    if train:
        S = st["S0"].to(f)[pick]
    else:
        S = st["pool"].to(f)[st["slots"].long()[pick]]
        if case["kind"] == "ssm_prefill":
            S = S * (1 - pick % 2)[:, None, None]
    raw = st["dt"].to(f) + (0 if st["bias"] is None else st["bias"].to(f))
    delta = torch.logaddexp(raw, torch.zeros_like(raw)) if case["softplus"] else raw
    x = st["x"].to(f)

    def wide(t, at):  # [m, G, N] of the tokens `at`, for every channel
        return t[at].to(f)[:, :, None].expand(-1, -1, D // G, -1).reshape(len(at), D, N)

    y = torch.empty(T, D, dtype=f, device="cuda")
    kept = []
    for t, m in enumerate(live):
        at = begin[:m] + t
        if train:
            kept.append(S[:m].clone())
        S[:m] = torch.exp(delta[at][..., None] * A) * S[:m] + (delta[at] * x[at])[..., None] * wide(st["B"], at)
        y[at] = torch.einsum("mdn,mdn->md", S[:m], wide(st["C"], at))
    if st["skip"] is not None:
        y = y + x * st["skip"].to(f)
    z = None if st["z"] is None else st["z"].to(f)
    out = y if z is None else y * z * torch.sigmoid(z)
    if not train:
        pool = st["pool"].to(f)
        for j, i in enumerate(order):
            if lens[i]:
                pool[int(st["slots"][i])] = S[j]
        return out, pool
    back = torch.argsort(pick)
    res = dict(out=out, S=S[back].clone())
    do = st["dout"].to(f)
    if z is not None:
        s = torch.sigmoid(z)
        res["dz"] = do * y * (s + z * s * (1 - s))
        do = do * z * s
    dS = st["dS"].to(f)[pick]
    dx, dd = torch.zeros(T, D, dtype=f, device="cuda"), torch.zeros(T, D, dtype=f, device="cuda")
    dA, dB, dC = torch.zeros_like(A), torch.zeros(T, G, N, dtype=f, device="cuda"), torch.zeros(T, G, N, dtype=f, device="cuda")
    for t in range(max(lens) - 1, -1, -1):
        m = live[t]
        at, prev = begin[:m] + t, kept.pop()
        a, B, u = torch.exp(delta[at][..., None] * A), wide(st["B"], at), (delta[at] * x[at])[..., None]
        h = a * prev + u * B
        adj = dS[:m] + do[at][..., None] * wide(st["C"], at)
        dC[at] = (do[at][..., None] * h).unflatten(1, (G, D // G)).sum(2)
        dB[at] = (adj * u).unflatten(1, (G, D // G)).sum(2)
        through = (adj * B).sum(-1)
        dx[at], moved = delta[at] * through, adj * prev * a
        dd[at] = x[at] * through + (moved * A).sum(-1)
        dA += torch.einsum("mdn,md->dn", moved, delta[at])
        dS[:m] = a * adj
    if st["skip"] is not None:
        dx += do * st["skip"].to(f)
        res["dD"] = (do * x).sum(0)
    if case["softplus"]:
        dd = dd * torch.sigmoid(raw)
    if st["bias"] is not None:
        res["dbias"] = dd.sum(0)
    return res | dict(dx=dx, ddt=dd, dA=dA, dB=dB, dC=dC, dS0=dS[back])


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "norm":
        f = torch.float64
        if case["train"]:
            return _norm_train(st, _exact_heads, f)[0]
        wq, wk = (None if w is None else w.to(f) for w in (st["wq"], st["wk"]))
        return dict(q=_exact_heads(st["q"].to(f), wq, st["q_scale"], st), k=_exact_heads(st["k"].to(f), wk, 1.0, st))
    return (_exact_conv if case["kind"].startswith("conv") else _exact_ssm)(case, st)
