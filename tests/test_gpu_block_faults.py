"""The optimizer under capture and the norm that clips its gradients."""

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


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


@pytest.mark.parametrize("dtype", [BF, F])
def test_the_norm_that_clips(cuda_ok, dtype):
    """As on the CPU: a sum of 4121 squares in fp32 is off by at most 4121 * 2^-24, its root by half of
    that; the few other operations are within the rest of 2^-12."""
    from paper_2608_13578_gb300 import gpt
    p, q = (torch.nn.Parameter(torch.zeros(n, dtype=d, device="cuda")) for n, d in ((4121, dtype), (50, F)))
    p.grad, q.grad = torch.full_like(p, 0.01), torch.full_like(q, 1e-3)
    norm = float(p.grad.double().square().sum() + q.grad.double().square().sum()) ** 0.5
    scale = gpt._clip_scale([p, q], 0.5)
    assert scale.dtype == F and scale.is_cuda
    assert abs(float(scale) * (norm + 1e-6) / 0.5 - 1.0) <= 2.0 ** -12
