"""TokenStep's refusals: calls out of order, and ids that are not those of the forward pass."""
import pytest
import torch

import paper_2607_01125_gb300 as zo
from paper_2607_01125_gb300.model import TokenStep

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_calls_that_have_nothing_to_work_on():
    ctx = zo.Context(0)
    table = torch.randn(50, 64, generator=torch.Generator(DEV).manual_seed(1), device=DEV)
    ids = torch.arange(20, device=DEV)
    model = TokenStep(None, table, ctx=ctx)
    before = ctx.launch_count()
    for call in (lambda: model.loss(ids), lambda: model.ends_grad(ids, ids), lambda: model.step(ids, ids, 1, 0, 0)):
        with pytest.raises(ValueError):
            call()
    assert ctx.launch_count() == before
    model.forward(ids)
    before = ctx.launch_count()
    for n in (19, 21):                                   # a part of the batch, or more than it
        other = torch.arange(n, device=DEV)
        with pytest.raises(ValueError):
            model.ends_grad(other, other)
    with pytest.raises(ValueError):
        model.ends_grad(ids, ids[:19])
    assert ctx.launch_count() == before
    assert torch.equal(model.ends_grad(ids, ids), model.loss(ids))
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    ctx.close()
