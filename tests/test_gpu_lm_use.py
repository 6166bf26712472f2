"""The language-model operators as programs use them, beyond their values: what
autograd sees of a state that is written in place, derivatives of derivatives,
arguments in every form that Python takes."""

import pytest
import torch

from tests.test_gpu_lm_ops import F, make, no_wait_ran_out  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------ states written in place
@pytest.mark.parametrize("how", ["step", "step_of_a_view", "state_out", "state_out_in_place"])
def test_autograd_sees_a_state_written_in_place(F, how):
    """The first state of a differentiable call is kept for its backward: a write
    before that must be an error, as it is for torch's own operations in place."""
    T = 1 if how.startswith("step") else 40
    d, _ = make(2, T, 2, 64, "bf16", 31, True)
    q = d["q"].clone().requires_grad_()
    s = d["s0"]
    o, last = F.linear_attention(q, d["k"], d["v"], d["decay"], state=s)
    if how == "step":
        F.linear_attention_step(d["q"], d["k"], d["v"], d["decay"], s)
    elif how == "step_of_a_view":
        F.linear_attention_step(d["q"], d["k"], d["v"], d["decay"], s.detach())
    elif how == "state_out":
        F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], state_out=s)
    else:
        F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], state=s, state_out=s)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.backward(d["do"])


def test_a_state_of_its_own_may_be_written(F):
    """Copies, fresh outputs and states under inference mode take steps as before."""
    d, _ = make(2, 1, 2, 64, "bf16", 32, True)
    q = d["q"].clone().requires_grad_()
    o, last = F.linear_attention(q, d["k"], d["v"], d["decay"], state=d["s0"])
    own = d["s0"].clone()
    version = d["s0"]._version
    F.linear_attention_step(d["q"], d["k"], d["v"], d["decay"], own)
    F.linear_attention_step(d["q"], d["k"], d["v"], d["decay"], d["s0"], state_out=own)
    assert d["s0"]._version == version and torch.equal(own, last.detach())
    o.backward(d["do"])
    assert torch.isfinite(q.grad).all()
    with torch.inference_mode():
        s = d["s0"].clone()
        F.linear_attention_step(d["q"], d["k"], d["v"], d["decay"], s)
        assert torch.equal(s, own)
    F.linear_attention_step(d["q"], d["k"], d["v"], d["decay"], s)   # made there, used here
