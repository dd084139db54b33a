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
