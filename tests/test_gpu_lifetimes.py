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


@pytest.mark.parametrize("shapes", [[(64, 576)] * 6, [(300, 400), (129, 1000)], [(1024, 1024)] * 7])
def test_a_plan_made_on_a_side_stream_is_ready_for_it_at_once(shapes):
    """Tables are on the device when the calls that make them return: a side stream does not wait for the default one."""
    from paper_1811_03617_b200 import gvq
    lens = [m * n for m, n in shapes]
    off = [sum(lens[:i]) for i in range(len(lens))]
    g = torch.randn(sum(lens), device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(torch.cuda.Stream()):
            ctx = gvq.Context(gvq.HostLayout(64, 4, off, lens))
            plan = gvq.OrthoPlan(ctx, [m for m, _ in shapes], [n for _, n in shapes])
            first = torch.empty(ctx.M, device="cuda")
            plan.orthogonalize(g, first)
            torch.cuda.synchronize()
            later = torch.empty(ctx.M, device="cuda")
            plan.orthogonalize(g, later)
            ctx.device_status()
        assert torch.equal(first, later)
