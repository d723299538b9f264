"""Arguments of the calls at a language model's ends that concern an output which is not asked for."""
import pytest
import torch

import paper_2607_01125_gb300 as zo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
def test_accumulate_without_the_output_that_it_concerns(dt):
    ctx = zo.Context(0)
    g = torch.Generator(DEV).manual_seed(1)
    H, W = (torch.randn(n, 64, generator=g, device=DEV).to(dt) for n in (20, 300))
    t = torch.randint(0, 300, (20,), generator=g, device=DEV)
    dH, want = torch.empty_like(H), torch.empty_like(H)
    zo.zoact_ce_grad(ctx, H, W, t, dH=want)
    zo.zoact_ce_grad(ctx, H, W, t, dH=dH, accumulate=True)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    assert torch.equal(dH, want)
    if dt != torch.float32:                              # sums over calls are held in fp32
        with pytest.raises(zo.ZoactError) as e:
            zo.zoact_ce_grad(ctx, H, W, t, dH=dH, dW=torch.zeros_like(W), accumulate=True)
        assert e.value.status == -2
    ctx.close()
