"""Closing order of contexts and plans on the GPU: what comes too late is an exception."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_plan_whose_context_is_closed_refuses_its_calls():
    from paper_1811_03617_b200 import gvq
    ctx = gvq.Context(gvq.HostLayout(64, 4, [0, 4096], [4096, 120 * 400]))
    plan = gvq.OrthoPlan(ctx, [64, 120], [64, 400])
    g = torch.randn(ctx.M, device="cuda")
    mo, w = torch.zeros_like(g), torch.zeros_like(g)
    plan.step(g, mo, w, lr=0.1)
    torch.cuda.synchronize()
    ctx.close()
    for call in (lambda: plan.step(g, mo, w, lr=0.1), lambda: plan.orthogonalize(g, w)):
        with pytest.raises(gvq.GvqError) as e:
            call()
        assert e.value.status == 1
    plan.close()
    with pytest.raises(gvq.GvqError):
        plan.orthogonalize(g, w)
    with pytest.raises(gvq.GvqError):
        gvq.OrthoPlan(ctx, [64, 120], [64, 400])
