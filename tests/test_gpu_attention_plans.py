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
