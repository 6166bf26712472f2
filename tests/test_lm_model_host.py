"""Host side of the GPT's use of the language-model operators (CPU only): the
operators are replaced by torch forms that record what they are called with."""

import copy

import pytest
import torch
import torch.utils.checkpoint

from paper_2608_13578_gb300 import gpt


def config(**kw):
    base = dict(vocab=31, D=16, H=2, layers=2, mlp=32, L=16, T=12, mixer="dense", dropout=0.25)
    return gpt.GPTConfig(**{**base, **kw})


def model_of(**kw):
    return gpt.build(config(**kw), device="cpu", dtype=torch.float32)


def ids_of(n=8, B=2):
    return torch.randint(0, 31, (B, n), generator=torch.Generator().manual_seed(1))


@pytest.fixture
def drawn(monkeypatch):
    """(offset, step) of every mask that is drawn, in order."""
    calls = []

    def dropout(x, p, seed, offset, residual=None, step=None):
        at = (offset, 0 if step is None else int(step))
        calls.append(at)
        g = torch.Generator().manual_seed(at[0] // (1 << 40) * 1000 + at[1])
        y = x * (torch.rand(x.shape, generator=g) >= p) / (1 - p)
        return y if residual is None else y + residual
    monkeypatch.setattr(gpt.lm_ops, "dropout", dropout)
    return calls


# ------------------------------------------------------------------- masks
def test_every_call_draws_masks_of_its_own(drawn):
    """A loop of the user's own, or gradients accumulated over several calls, trains
    with new masks at every call, not only train_step."""
    model = model_of()
    first, second = model(ids_of()), model(ids_of())
    assert not torch.equal(first, second)
    assert len(drawn) == 10 and len(set(drawn)) == 10      # 5 places a call
    steps = [s for _, s in drawn]
    assert steps == [0] * 5 + [1] * 5
    model.eval()
    assert torch.equal(model(ids_of()), model(ids_of())) and len(drawn) == 10


def test_train_step_draws_once(drawn):
    model = model_of()
    opt = gpt.make_optimizer(model)
    for _ in range(3):
        gpt.train_step(model, opt, ids_of(), ids_of())
    assert [s for _, s in drawn] == [0] * 5 + [1] * 5 + [2] * 5
    assert int(model.drop_step) == 3


def test_a_block_run_anew_draws_the_same_masks(drawn):
    """Activations recomputed in the backward pass have the masks of their forward."""
    grads = []
    for again in (False, True):
        model = model_of()
        if again:
            for blk in model.blocks:
                run = blk.forward
                blk.forward = lambda x, drop, run=run: torch.utils.checkpoint.checkpoint(
                    run, x, drop, use_reentrant=False)
        model(ids_of()).square().sum().backward()
        grads.append(torch.cat([p.grad.reshape(-1) for p in model.parameters()]))
    assert len(drawn) > 10 and torch.equal(grads[0], grads[1])
