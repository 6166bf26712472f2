"""Calls that a captured graph would repeat wrongly."""

import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


# ---------------------------------------------------------------- the optimizer
@pytest.mark.parametrize("how,say", [(dict(), "capturable"), (dict(capturable=True), "before the capture"),
                                     (dict(capturable=True, masters=True, bits=8), "before the capture")])
def test_captures_that_would_not_count_on(cuda_ok, how, say):
    """The capture fails with the optimizer's message; a step outside is as if it had not been."""
    from paper_2608_13578_gb300 import optim
    p = torch.nn.Parameter(torch.ones(300, device="cuda", dtype=BF))
    p.grad = torch.ones_like(p)
    opt = optim.AdamW([p], lr=0.1, weight_decay=0.0, **how)
    if not how:
        opt.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match=say):
        with torch.cuda.graph(graph):
            opt.step()
    opt.step()
    torch.cuda.synchronize()
    assert int(opt.state[p]["step"]) == 1 + (not how)
    # a constant gradient moves a weight by lr a step, whatever the betas
    assert abs(float(p.detach()[0]) - (0.8 if not how else 0.9)) <= 2 * 2.0 ** -8
    if how:
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            opt.step()
