"""Cases of the sequence operators: the scan of a recurrent state over packed prompts, its backward pass, and the
plan (offsets, chunk table, slot maps) that serving builds from request lengths.

``own`` false: the plain form, elementary torch operations in fp32 (log-decay sums in fp64).  ``own`` true: the calls a
user makes of this package.  ``exact`` is the token-by-token definition in fp64.
"""
import math
import random

import torch

own = False

OPS = {"gdn": 0, "kda": 1, "rwkv6": 2, "linattn": 3, "retnet": 4, "gla": 5}
DELTA = ("gdn", "kda")            # u = beta (v - S'^T k), else u = v
VECTOR = ("kda", "rwkv6", "gla")  # one log-decay per key channel
CHUNK = 64                        # tokens per entry of the chunk table
CAP = 16                          # log capacity of the slots


# ---------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one short prompt of the smallest configuration (fp32, two heads of 64): call latency
        dict(name="prefill_gdn_fp32_small", kind="prefill", op="gdn", dtype="fp32", n=1, lo=64, hi=64, H=2, Hq=2, dk=64, dv=64, lens=1),
        # a serving step's prompts, ragged, half of them continuing a conversation, 32 heads of 128
        dict(name="prefill_gdn_ragged", kind="prefill", op="gdn", dtype="bf16", n=48, lo=2, hi=1500, H=32, Hq=32, dk=128, dv=128, lens=2),
        # one long document, few (sequence, head) pairs: the chain over chunks counts
        dict(name="prefill_gdn_long", kind="prefill", op="gdn", dtype="bf16", n=1, lo=16384, hi=16384, H=32, Hq=16, dk=128, dv=128, lens=3),
        # per-channel gates
        dict(name="prefill_kda_ragged", kind="prefill", op="kda", dtype="bf16", n=24, lo=2, hi=1200, H=32, Hq=32, dk=128, dv=128, lens=4),
        # many heads of 64 with the bonus term
        dict(name="prefill_rwkv6", kind="prefill", op="rwkv6", dtype="bf16", n=33, lo=100, hi=900, H=64, Hq=64, dk=64, dv=64, lens=5),
        # training steps: forward and gradients of packed documents
        dict(name="train_retnet_fp32_small", kind="train", op="retnet", dtype="fp32", n=3, lo=1, hi=150, H=4, Hq=2, dk=64, dv=128, lens=6),
        dict(name="train_gdn", kind="train", op="gdn", dtype="bf16", n=4, lo=2048, hi=2048, H=32, Hq=32, dk=128, dv=128, lens=7),
        dict(name="train_gdn_large", kind="train", op="gdn", dtype="bf16", n=19, lo=700, hi=2800, H=32, Hq=16, dk=128, dv=128, lens=8),
        dict(name="train_kda", kind="train", op="kda", dtype="bf16", n=5, lo=300, hi=1300, H=32, Hq=32, dk=128, dv=128, lens=9),
        dict(name="train_rwkv6", kind="train", op="rwkv6", dtype="bf16", n=4, lo=1024, hi=1024, H=64, Hq=64, dk=64, dv=64, lens=10),
        # a decode batch with a few prompts among it: the plan of one serving step
        dict(name="plan_step", kind="plan", n=512, one=0.95, hi=4000, slots=700, lens=11),
        # offline packing of many documents
        dict(name="plan_packing", kind="plan", n=20000, one=0.02, hi=800, slots=25000, lens=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    lens = rng.randrange(1 << 30)
    kind = rng.choice(("prefill", "prefill", "train", "train", "plan"))
    if kind == "plan":
        n = _log(rng, 1, 20000)
        return dict(kind=kind, n=n, one=round(rng.random(), 3), hi=_log(rng, 2, 800), slots=n + rng.randrange(1 + n), lens=lens)
    op = rng.choice(tuple(OPS))
    dk, dv = rng.choice((64, 128)), rng.choice((64, 128))
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    H = rng.choice((1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64))
    Hq = rng.choice([x for x in range(1, H + 1) if H % x == 0])
    # token-heads of a 128 x 128 state; the per-channel gates' plain form needs more memory and time
    most = 250_000 if op in VECTOR else 600_000
    n = _log(rng, 1, 48)
    hi = max(1, min(_log(rng, 1, 12000), int(most / (H * n * dk * dv / 16384))))
    lo = rng.randint(0 if kind == "prefill" else 1, hi)
    return dict(kind=kind, op=op, dtype=dtype, n=n, lo=lo, hi=hi, H=H, Hq=Hq, dk=dk, dv=dv, lens=lens)


def _lens(case):
    """Request lengths of a case, from the case alone."""
    r = random.Random(case["lens"])
    if case["kind"] == "plan":
        return [1 if r.random() < case["one"] else r.randint(0, case["hi"]) for _ in range(case["n"])]
    lens = [r.randint(case["lo"], case["hi"]) for _ in range(case["n"])]
    lens[0] = case["hi"]
    return lens


# ---------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    lens = _lens(case)
    n, T = len(lens), sum(lens)
    i32 = dict(dtype=torch.int32, device="cuda")
    st = dict(case=case, lens=torch.tensor(lens, **i32), T=T)
    if case["kind"] == "plan":
        st["slots"] = torch.randperm(case["slots"], generator=gen, device="cuda")[:n].to(torch.int32)
        st["log_len"] = torch.randint(0, CAP + 1, (case["slots"], 1), generator=gen, **i32).expand(-1, 32).contiguous()
        order = torch.randperm(n, generator=gen, device="cuda")
        st["lens"] = st["lens"][order].contiguous()   # the requests of another seed come in another order
        return st
    op, H, Hq, dk, dv = case["op"], case["H"], case["Hq"], case["dk"], case["dv"]
    io = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    q, k, v = randn(T, Hq, dk), randn(T, Hq, dk), randn(T, H, dv)
    if op == "linattn":
        q, k = torch.nn.functional.elu(q) + 1, torch.nn.functional.elu(k) + 1
    if op != "rwkv6":
        q, k = (x / x.norm(dim=-1, keepdim=True).clamp_min(1e-12) for x in (q, k))
    st |= dict(q=q.to(io), k=k.to(io), v=v.to(io), beta=None, bonus=None, g=None, lens_host=lens)
    if op in ("kda", "gla"):
        st["g"] = -torch.nn.functional.softplus(randn(T, H, dk))
    elif op == "rwkv6":
        st["g"] = -torch.exp(randn(T, H, dk) * 0.5 - 0.5)
        st["bonus"] = randn(H, dk) * 0.1
    elif op == "gdn":
        st["g"] = -torch.nn.functional.softplus(randn(T, H))
    elif op == "retnet":
        st["g"] = torch.log1p(-torch.pow(2.0, -5.0 - torch.arange(H, device="cuda") % 8)).expand(T, H).contiguous()
    if op in DELTA:
        st["beta"] = torch.sigmoid(randn(T, H))
    st["scale"] = 1.0 if op in ("rwkv6", "linattn") else dk ** -0.5
    if case["kind"] == "train":
        st |= dict(S0=randn(n, H, dk, dv) * 0.1, dout=randn(T, H, dv).to(io), dS=randn(n, H, dk, dv) * 0.1)
        return st
    # the slot pool: every other request continues from its slot's state, with entries pending in its log
    slots = n + 1 + n // 8
    st["slots"] = torch.randperm(slots, generator=gen, device="cuda")[:n].to(torch.int32)
    st["fresh"] = (torch.arange(n, device="cuda") % 2).to(torch.int32)
    st["S_base"] = randn(slots, H, dk, dv) * 0.1
    d_lam = dk if op in VECTOR else 1
    st["K_log"] = (randn(slots, H, CAP, dk) * dk ** -0.5).to(io)
    st["U_log"] = randn(slots, H, CAP, dv).to(torch.float32 if op in DELTA else io)
    st["decay_log"] = (-torch.rand(slots, H, CAP, d_lam, generator=gen, device="cuda") * (op != "linattn")).cumsum(2)
    st["log_len"] = torch.randint(0, CAP + 1, (slots, 1), generator=gen, **i32).expand(-1, H).contiguous()
    return st


# ---------------------------------------------------------------------------------------------------- plain forms
def _plain_plan(st):
    """Offsets, chunk table, token map and row-aligned slot lists from the lengths."""
    lens, slots = st["lens"].long(), st["slots"]
    n, T = lens.numel(), st["T"]
    most = T // CHUNK + n
    rows = torch.arange(n, device="cuda", dtype=torch.int32)
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    nch = (lens + CHUNK - 1) // CHUNK
    starts, chunk_starts = (torch.cat((zero, x.cumsum(0))).to(torch.int32) for x in (lens, nch))
    at = torch.arange(most, device="cuda", dtype=torch.int32)
    chunk_seq = torch.where(at < chunk_starts[-1], torch.searchsorted(chunk_starts, at, right=True).to(torch.int32) - 1, -1)
    token_seq = torch.repeat_interleave(rows, lens, output_size=T)
    one = lens == 1
    full = st["log_len"][slots.long(), 0] >= CAP
    scan = torch.where(lens > 1, slots, -1)
    append = torch.where(one & ~full, slots, -1)
    merge = torch.where(one & full, slots, -1)
    totals = torch.stack((starts[-1], chunk_starts[-1], (lens > 1).sum(), one.sum())).to(torch.int32)
    return dict(starts=starts, chunk_starts=chunk_starts, chunk_seq=chunk_seq, token_seq=token_seq, scan_slots=scan,
                append_slots=append, merge_slots=merge, totals=totals)


def _chunks(lens, C):
    """[chunks, C] token index and validity of sequences cut into chunks, longest sequence first, and their order."""
    ln = torch.tensor(lens)
    order = torch.argsort(ln, descending=True, stable=True)
    start = torch.cumsum(ln, 0) - ln
    nch = (ln[order] + C - 1) // C
    row = torch.repeat_interleave(torch.arange(len(lens)), nch)
    base = torch.cumsum(nch, 0) - nch
    tok = (torch.arange(row.numel()) - base[row])[:, None] * C + torch.arange(C)
    ok = tok < ln[order][row][:, None]
    tok = torch.where(ok, tok + start[order][row][:, None], 0)
    return order.cuda(), nch, base, tok.cuda(), ok.cuda()


def _plain_scan(op, scale, q, k, v, g, beta, bonus, S0, lens):
    """Chunked recurrence over packed sequences in fp32: out [T,H,dv] and the last states, in the order of `lens`."""
    H, T, dv = v.shape[1], v.shape[0], v.shape[2]
    C = 16 if op in VECTOR else 32
    order, nch, base, tok, ok = _chunks(lens, C)

    def cut(x):  # [T, h, ...] -> [chunks, H, C, ...]
        x = (x.float() if x.dtype != torch.float64 else x)[tok]
        x = x * ok.view(*ok.shape, *([1] * (x.dim() - 2)))
        return x.repeat_interleave(H // x.shape[2], 2).transpose(1, 2)

    q, k, v = cut(q) * scale, cut(k), cut(v)
    G = (torch.zeros(T, H, dtype=torch.float64, device="cuda") if g is None else g.double())
    gc = cut(G)
    gc = gc if op in VECTOR else gc[..., None]                     # [chunks, H, C, dk or 1]
    G = gc.cumsum(2)
    Gr = G - gc if op == "rwkv6" else G                            # what a readout sees
    low = torch.ones(C, C, dtype=torch.bool, device="cuda").tril(-1 if op == "rwkv6" else 0)
    strict = torch.ones(C, C, dtype=torch.bool, device="cuda").tril(-1)

    def pairs(a, Ga, keep):                                        # sum_c a_ic k_jc exp(Ga_ic - G_jc), masked
        if op in VECTOR:
            e = torch.exp((Ga[..., :, None, :] - G[..., None, :, :]).masked_fill(~keep[:, :, None], -math.inf).float())
            return ((a[..., :, None, :] * k[..., None, :, :]) * e).sum(-1)
        e = torch.exp((Ga - G.transpose(-1, -2)).masked_fill(~keep, -math.inf).float())
        return (a @ k.transpose(-1, -2)) * e

    A = pairs(q, Gr, low)
    if op == "rwkv6":
        A = A + torch.diag_embed((q * k * bonus[:, None]).sum(-1))
    qt, kt, kh, last = q * torch.exp(Gr.float()), k * torch.exp(G.float()), k * torch.exp((G[..., -1:, :] - G).float()), torch.exp(G[..., -1, :, None].float())
    if op in DELTA:
        b = cut(beta)[..., None]
        L = -b * pairs(k, G, strict)
        inv = torch.eye(C, device="cuda") + L                      # (I - L)^-1 = (I + L)(I + L^2)(I + L^4)...
        for _ in range(int(math.log2(C)) - 1):
            L = L @ L
            inv = inv + inv @ L
    S = S0.float()[order]
    ends, outs, at = [], [], []
    n_at = torch.bincount(nch, minlength=int(nch.max()) + 1).flip(0).cumsum(0).flip(0).tolist()  # sequences with >= s chunks
    base = base.cuda()
    for s in range(int(nch.max())):
        m = n_at[s + 1]
        ends.append(S[m:])
        S, c = S[:m], base[:m] + s
        U = v[c]
        if op in DELTA:
            U = inv[c] @ (b[c] * (U - kt[c] @ S))
        outs.append(qt[c] @ S + A[c] @ U)
        at.append(c)
        S = last[c] * S + kh[c].transpose(-1, -2) @ U
    ends.append(S)
    out = torch.zeros(T, H, dv, device="cuda")
    if outs:
        where = torch.cat(at)
        out = out.index_put((tok[where][ok[where]],), torch.cat(outs).transpose(1, 2)[ok[where]])
    return out, torch.cat(ends[::-1])[torch.argsort(order)]


def _plain_prefill(st):
    c, slots = st["case"], st["slots"].long()
    io = st["q"].dtype
    # fold the pending log entries of the requests that continue; the others start from zero
    ln = st["log_len"][slots, 0]
    at = torch.arange(CAP, device="cuda")
    lam = st["decay_log"][slots]
    end = torch.where(ln[:, None, None] > 0, lam[torch.arange(len(ln), device="cuda"), :, (ln - 1).clamp_min(0).long()], 0.0)
    live = (at < ln[:, None])[:, None, :, None]
    w = torch.exp((end[:, :, None] - lam).masked_fill(~live, -math.inf)) * st["K_log"][slots].float()
    S = torch.exp(end)[..., None] * st["S_base"][slots] + w.transpose(-1, -2) @ st["U_log"][slots].float()
    S = S * (st["fresh"] == 0)[:, None, None, None]
    out, S = _plain_scan(c["op"], st["scale"], st["q"], st["k"], st["v"], st["g"], st["beta"], st["bonus"], S, st["lens_host"])
    any_ = st["lens"] > 0
    st["S_base"][slots[any_]] = S[any_]
    st["log_len"][slots[any_]] = 0
    return out.to(io), st["S_base"], st["log_len"]


def _plain_train(st):
    names = [x for x in ("q", "k", "v", "g", "beta", "bonus") if st[x] is not None]
    leaf = {x: st[x].float().detach().requires_grad_() for x in names}
    S0 = st["S0"].detach().requires_grad_()
    args = [leaf.get(x) for x in ("q", "k", "v", "g", "beta", "bonus")]
    out, S = _plain_scan(st["case"]["op"], st["scale"], *args, S0, st["lens_host"])
    grads = torch.autograd.grad((out, S), [*leaf.values(), S0], (st["dout"].float(), st["dS"]))
    res = {"d" + x: d.to(st[x].dtype) for x, d in zip(names, grads)}
    return dict(out=out.detach().to(st["q"].dtype), S=S.detach(), dS0=grads[-1], **res)


# ---------------------------------------------------------------------------------------------------- the package's calls
def _handle(st):
    """What a program keeps between steps: the descriptor, the pool's tensors, the plan's tables and workspaces."""
    if "handle" not in st:
        import paper_2608_15533_b200 as dl

        c = st["case"]
        n, T = st["lens"].numel(), st["T"]
        h = dict(dl=dl, plan=dl.Plan(n, T, device="cuda"))
        if c["kind"] != "plan":
            h["desc"] = dl.Desc(op=OPS[c["op"]], num_slots=n + 1 + n // 8, H=c["H"], H_qk=c["Hq"], d_k=c["dk"], d_v=c["dv"], cap=CAP,
                                io_dtype=dl.F32 if c["dtype"] == "fp32" else dl.BF16, scale=st["scale"])
            h["work"] = dl.scan_workspace(h["desc"], n, T, train=c["kind"] == "train", device="cuda")
        if c["kind"] == "prefill":
            h["pool"] = dl.State.wrap(h["desc"], st["S_base"], st["K_log"], st["U_log"], st["decay_log"], st["log_len"])
        st["handle"] = h
    return st["handle"]


def _own_plan(st):
    h = _handle(st)
    p = h["dl"].build_plan(st["lens"], h["plan"], slots=st["slots"], log_len=st["log_len"], cap=CAP, decode_rows=True)
    return dict(starts=p.starts, chunk_starts=p.chunk_starts, chunk_seq=p.chunk_seq, token_seq=p.token_seq, scan_slots=p.scan_slots,
                append_slots=p.append_slots, merge_slots=p.merge_slots, totals=p.totals)


def _own_prefill(st):
    h = _handle(st)
    plan = h["dl"].build_plan(st["lens"], h["plan"], slots=st["slots"])
    out = h["dl"].prefill(h["desc"], h["pool"], plan, st["q"], st["k"], st["v"], st["g"], st["beta"], st["bonus"], fresh=st["fresh"], workspace=h["work"])
    return out, st["S_base"], st["log_len"]


def _own_train(st):
    h = _handle(st)
    dl, plan = h["dl"], h["dl"].build_plan(st["lens"], h["plan"])
    args = (h["desc"], plan, st["q"], st["k"], st["v"], st["g"], st["beta"], st["bonus"])
    out, S = dl.scan_forward(*args, S_init=st["S0"], workspace=h["work"], save=True)
    d = dl.scan_backward(*args, st["dout"], S_init=st["S0"], dS_final=st["dS"], workspace=h["work"], saved=True)
    res = dict(out=out, S=S, dS0=d.S_init, dq=d.q, dk=d.k, dv=d.v)
    return res | {"d" + x: y for x, y in (("g", d.g), ("beta", d.beta), ("bonus", d.u_bonus)) if y is not None}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"plan": _own_plan, "prefill": _own_prefill, "train": _own_train}[kind](state)
    return {"plan": _plain_plan, "prefill": _plain_prefill, "train": _plain_train}[kind](state)


# ---------------------------------------------------------------------------------------------------- work
def work(case):
    lens = _lens(case)
    n, T = len(lens), sum(lens)
    if case["kind"] == "plan":
        ch = T // CHUNK + n
        # lengths, slots and one length word of the log per row in; offsets, three slot lists, chunk table, token map out
        return {"bytes": 4 * (3 * n + 2 * (n + 1) + 3 * n + ch + T + 4), "flops": 0}
    H, Hq, dk, dv, op = case["H"], case["Hq"], case["dk"], case["dv"], case["op"]
    e = 4 if case["dtype"] == "fp32" else 2
    delta = op in DELTA
    gate = 0 if op == "linattn" else 4 * H * (dk if op in VECTOR else 1)
    small = gate + (4 * H if delta else 0)
    tokens = T * (e * (2 * Hq * dk + 2 * H * dv) + small)                 # q, k, v, g, beta in, out out
    state = 4 * n * H * dk * dv
    bonus = 4 * H * dk if op == "rwkv6" else 0
    flops = T * H * dk * dv * (6 if delta else 4)
    if case["kind"] == "prefill":
        return {"bytes": tokens + 2 * state + bonus, "flops": flops}
    # a step keeps its inputs: they and dout come in, out and a gradient for each input go out
    return {"bytes": tokens + T * (e * (2 * Hq * dk + 2 * H * dv) + small) + 4 * state + 2 * bonus, "flops": flops * 3}


# ---------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    if case["kind"] == "plan":
        return None
    st = prepare(case, seed)
    op, scale, lens = case["op"], st["scale"], st["lens_host"]
    n, T, H, dk, dv = len(lens), st["T"], case["H"], case["dk"], case["dv"]
    rep = H // case["Hq"]
    f64 = torch.float64
    start = [sum(lens[:i]) for i in range(n)]
    order = sorted(range(n), key=lambda i: -lens[i])
    first = torch.tensor([start[i] for i in order], device="cuda")
    live = [sum(1 for x in lens if x > t) for t in range(max(lens) + 1)]

    def row(x, at):  # tokens `at` of x as fp64 [m, H, ...]
        return x[at].to(f64).repeat_interleave(H // x.shape[1], 1)

    def gate(at, m):
        if st["g"] is None:
            return torch.ones(m, H, 1, 1, device="cuda", dtype=f64)
        a = torch.exp(row(st["g"], at))
        return a[..., None] if op in VECTOR else a[..., None, None]

    def read(S, x):   # S^T x
        return torch.einsum("nhkv,nhk->nhv", S, x)

    def step(S, t):
        """One token of the sequences that still run: states before the update (decayed) and after, factors."""
        m = live[t]
        at = first[:m] + t
        Sd = S[:m] * gate(at, m)
        k, e = row(st["k"], at), row(st["v"], at)
        u = e
        if op in DELTA:
            e = e - read(Sd, k)
            u = row(st["beta"], at)[..., None] * e
        return at, Sd, k, e, u, Sd + k[..., None] * u[..., None, :]

    if case["kind"] == "train":
        S = st["S0"].to(f64)[torch.tensor(order, device="cuda")]
    else:
        S = torch.zeros(n, H, dk, dv, dtype=f64, device="cuda")
        ln = st["log_len"][:, 0].tolist()
        for j, i in enumerate(order):
            if i % 2:
                continue  # a fresh request
            s = int(st["slots"][i])
            lam = st["decay_log"][s].to(f64)
            end = lam[:, ln[s] - 1] if ln[s] else torch.zeros_like(lam[:, 0])
            S[j] = torch.exp(end)[..., None] * st["S_base"][s].to(f64)
            for x in range(ln[s]):
                f = torch.exp(end - lam[:, x]) * st["K_log"][s, :, x].to(f64)
                S[j] += f[..., None] * st["U_log"][s, :, x].to(f64)[:, None, :]
    out = torch.zeros(T, H, dv, dtype=f64, device="cuda")
    seg = 64
    marks = []
    for t in range(max(lens)):
        if t % seg == 0:
            marks.append(S.clone() if case["kind"] == "train" else None)
        at, Sd, k, e, u, S_new = step(S, t)
        q = row(st["q"], at)
        if op == "rwkv6":
            out[at] = read(S[: live[t]], q) + (q * st["bonus"].to(f64) * k).sum(-1, keepdim=True) * u
        else:
            out[at] = scale * read(S_new, q)
        S[: live[t]] = S_new
    back = torch.argsort(torch.tensor(order, device="cuda"))
    if case["kind"] == "prefill":
        pool = st["S_base"].to(f64)
        for j, i in enumerate(order):
            if lens[i]:
                pool[int(st["slots"][i])] = S[j]
        return out, pool, None
    # adjoint of the same recurrence, states recomputed segment by segment
    S_last = S[back]
    dS = st["dS"].to(f64)[torch.tensor(order, device="cuda")].clone()
    dq, dk_, dv_ = (torch.zeros(T, H, w, dtype=f64, device="cuda") for w in (dk, dk, dv))
    dg = None if st["g"] is None else torch.zeros(st["g"].shape, dtype=f64, device="cuda")
    dbeta = torch.zeros(T, H, dtype=f64, device="cuda")
    dbonus = torch.zeros(H, dk, dtype=f64, device="cuda")
    for t0 in range((max(lens) - 1) // seg * seg, -1, -seg):
        S = marks.pop()
        kept = []
        for t in range(t0, min(t0 + seg, max(lens))):
            at, Sd, k, e, u, S_new = step(S, t)
            kept.append((at, S[: live[t]].clone(), Sd, k, e, u, S_new))
            S[: live[t]] = S_new
        while kept:
            at, Sp, Sd, k, e, u, S_new = kept.pop()
            m = at.numel()
            q, do = row(st["q"], at), st["dout"][at].to(f64)
            D = dS[:m]
            pre = None
            du = 0.0
            if op == "rwkv6":
                b = st["bonus"].to(f64)
                vd = (u * do).sum(-1, keepdim=True)
                dq[at] = torch.einsum("nhkv,nhv->nhk", Sp, do) + b * k * vd
                dk_[at] += b * q * vd
                dbonus += (q * k * vd).sum(0)
                du = (q * b * k).sum(-1, keepdim=True) * do
                pre = q[..., None] * do[..., None, :]
            else:
                dq[at] = scale * torch.einsum("nhkv,nhv->nhk", S_new, do)
                D = D + scale * q[..., None] * do[..., None, :]
            dk_[at] += torch.einsum("nhkv,nhv->nhk", D, u)
            du = du + read(D, k)
            if op in DELTA:
                dbeta[at] = (du * e).sum(-1)
                du = row(st["beta"], at)[..., None] * du
                dk_[at] -= torch.einsum("nhkv,nhv->nhk", Sd, du)
                D = D - k[..., None] * du[..., None, :]
            dv_[at] = du
            if dg is not None:
                x = D * Sd
                dg[at] = x.sum(-1) if op in VECTOR else x.sum((-1, -2))
            D = D * gate(at, m)
            dS[:m] = D if pre is None else D + pre
    dq, dk_ = (x.view(T, case["Hq"], rep, dk).sum(2) for x in (dq, dk_))
    res = dict(out=out, S=S_last, dS0=dS[back], dq=dq, dk=dk_, dv=dv_)
    return res | {"d" + x: y for x, y in (("g", dg), ("beta", dbeta), ("bonus", dbonus)) if st[x] is not None}
