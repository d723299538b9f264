"""Plans that the gradient of attention does not take, in each type: the device status says so and nothing is written.  What a plan
of another shape, or one without the gradient's lists, would hold at this call's offsets is not looked at; the plans lie in
buffers with room for this call all the same.
"""
import pytest
import torch

import paper_2607_01125_gb300 as zo
from test_gpu_attention import DEV, Case, packed, plan_of

pytestmark = pytest.mark.gpu


def with_room(plan, n):
    room = torch.zeros(max(n, plan.numel()), dtype=torch.uint8, device=DEV)
    room[:plan.numel()] = plan
    return room


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_with_plans_of_other_calls_write_nothing(dt, d):
    ctx = zo.Context(0)
    c = Case(ctx, dt, 4, 2, d, packed(40, 90), grad=True)
    c.forward()
    bytes_ = zo.zoact_attention_plan_bytes(ctx, c.shape, grad=True)
    smaller = zo.attention_shape(20, 20, 1, 4, 2, d)
    own, keep = c.plan, c.lse.clone()
    plans = [with_room(plan_of(ctx, smaller, [(0, 20, 0, 20)], True), bytes_),              # a smaller shape
             with_room(plan_of(ctx, c.shape, packed(40, 90), False), bytes_),               # without the gradient's lists
             with_room(plan_of(ctx, zo.attention_shape(130, 130, 2, 4, 2, d, False), packed(40, 90), True), bytes_),   # not causal
             torch.zeros(bytes_, dtype=torch.uint8, device=DEV)]                            # none at all
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    for plan in plans:
        c.plan = plan
        outs = c.grads()
        torch.cuda.synchronize()
        assert ctx.device_status() == -1
        assert all(torch.isnan(t).all() for t in outs) and torch.equal(c.lse, keep)
    # and the call with its own plan is as it was
    c.plan = own
    outs = c.grads()
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    c.check_grads(outs)
    ctx.close()


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
def test_keys_without_any_query_and_queries_without_any_key(dt):
    """No rows of q at all: dk and dv are zeros in the spans.  No rows of k: outputs and dq are zeros."""
    ctx = zo.Context(0)
    c = Case(ctx, dt, 4, 2, 64, [(0, 0, 2, 40), (0, 0, 50, 130)], grad=True, rows_q=0, rows_k=190)
    c.forward()
    dq, dk, dv = c.grads()
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    inside = torch.zeros(190, dtype=torch.bool, device=DEV)
    inside[2:42] = inside[50:180] = True
    for t in (dk, dv):
        assert (t[inside] == 0).all() and torch.isnan(t[~inside]).all()
    c = Case(ctx, dt, 4, 2, 64, [(1, 30, 0, 0), (40, 200, 0, 0)], grad=True, rows_q=250, rows_k=0)
    c.forward()
    c.check_forward()
    dq, dk, dv = c.grads()
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    inside = torch.zeros(250, dtype=torch.bool, device=DEV)
    inside[1:31] = inside[40:240] = True
    assert (dq[inside] == 0).all() and torch.isnan(dq[~inside]).all()
    ctx.close()
