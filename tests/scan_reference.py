"""Token-by-token fp64 reference of the packed-sequence operators (torch, differentiable), for the tests.

The recurrence is written as it is defined: one token, one dense state, no chunks.
"""
from __future__ import annotations

import torch
import torch.nn.functional as F

GDN, KDA, RWKV6, LINATTN, RETNET, GLA = 0, 1, 2, 3, 4, 5
OPS = {"gdn": GDN, "kda": KDA, "rwkv6": RWKV6, "linattn": LINATTN, "retnet": RETNET, "gla": GLA}
DELTA, VECTOR = (GDN, KDA), (KDA, RWKV6, GLA)


def scan(op, scale, lens, q, k, v, g, beta, bonus, S0):
    """``(out [tokens,H,dv], S [n,H,dk,dv])`` in fp64; differentiable in every tensor."""
    H = v.shape[1]
    rep = H // q.shape[1]
    q, k, v = (x.double() for x in (q, k, v))
    q, k = q.repeat_interleave(rep, 1), k.repeat_interleave(rep, 1)
    outs, states, at = [], [], 0
    for i, n in enumerate(lens):
        S = S0[i].double()
        for t in range(at, at + n):
            Sp = S
            if g is not None:
                a = torch.exp(g[t].double())
                S = S * (a[:, :, None] if op in VECTOR else a[:, None, None])
            u = v[t]
            if op in DELTA:
                u = beta[t].double()[:, None] * (u - torch.einsum("hkv,hk->hv", S, k[t]))
            S = S + k[t][:, :, None] * u[:, None, :]
            if op == RWKV6:
                o = torch.einsum("hkv,hk->hv", Sp, q[t]) + (q[t] * bonus.double() * k[t]).sum(-1, keepdim=True) * u
            else:
                o = scale * torch.einsum("hkv,hk->hv", S, q[t])
            outs.append(o)
        states.append(S)
        at += n
    out = torch.stack(outs) if outs else v[:0]
    return out, torch.stack(states)


def inputs(op, lens, H, Hq, dk, dv, io, seed=0, tail=0, device="cuda"):
    """Token tensors of packed sequences (``tail`` rows behind the last one), with the distributions of the workloads."""
    gen = torch.Generator().manual_seed(seed)
    T = sum(lens) + tail

    def randn(*shape):
        return torch.randn(*shape, generator=gen)

    q, k, v = randn(T, Hq, dk), randn(T, Hq, dk), randn(T, H, dv)
    if op == LINATTN:
        q, k = F.elu(q) + 1, F.elu(k) + 1
    if op != RWKV6:
        q, k = F.normalize(q, dim=-1), F.normalize(k, dim=-1)
    noise = randn(T, H, dk)
    g = None
    if op in (KDA, GLA):
        g = -F.softplus(noise)
    elif op == RWKV6:
        g = -torch.exp(noise * 0.5 - 0.5)
    elif op == GDN:
        g = -F.softplus(noise[:, :, 0])
    elif op == RETNET:
        g = torch.log1p(-torch.pow(2.0, -5.0 - torch.arange(H) % 8)).expand(T, H)
    beta = torch.sigmoid(randn(T, H)) if op in DELTA else None
    bonus = randn(H, dk) * 0.1 if op == RWKV6 else None
    S0 = randn(len(lens), H, dk, dv) * 0.1
    d = dict(q=q.to(io), k=k.to(io), v=v.to(io), g=g, beta=beta, u_bonus=bonus)
    return {x: None if y is None else y.contiguous().to(device) for x, y in d.items()}, S0.to(device)
