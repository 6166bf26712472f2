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


@pytest.fixture
def linear(monkeypatch):
    """Linear attention in float32 torch operations, token by token."""
    def attention(q, k, v, decay, scale=None, lengths=None, state=None):
        B, T, H, d = q.shape
        S = torch.zeros(B, H, d, d) if state is None else state
        n = torch.full((B,), T) if lengths is None else lengths
        rows = []
        for t in range(T):
            on = (t < n).view(B, 1, 1, 1)
            S = torch.where(on, decay.view(1, H, 1, 1) * S + k[:, t, :, :, None] * v[:, t, :, None],
                            S)
            o = torch.einsum("bhij,bhi->bhj", S, q[:, t]) * (scale or d ** -0.5)
            rows.append(torch.where(on[..., 0], o, torch.zeros(())))
        return torch.stack(rows, 1), S
    monkeypatch.setattr(gpt.lm_ops, "linear_attention", attention)


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


# -------------------------------------------------------------- saved models
def test_a_resumed_run_goes_on_with_new_masks(drawn):
    model = model_of()
    model(ids_of()), model(ids_of())
    saved = {k: v.clone() for k, v in model.state_dict().items()}
    resumed = model_of(dropout=0.25)
    resumed.load_state_dict(saved)
    assert torch.equal(resumed(ids_of()), model(ids_of()))
    assert [s for _, s in drawn] == [0] * 5 + [1] * 5 + [2] * 10


@pytest.mark.parametrize("to", [0.0, 0.25])
@pytest.mark.parametrize("frm", [0.0, 0.25])
def test_weights_go_between_models_with_and_without_dropout(drawn, frm, to):
    a, b = model_of(dropout=frm), model_of(dropout=to)
    a(ids_of())
    missing, unexpected = b.load_state_dict(a.state_dict())
    assert not missing and not unexpected
    assert int(b.drop_step) == (1 if frm and to else 0)
    plain = set(model_of(dropout=0.0).state_dict())
    assert "drop_step" not in plain        # files of models without dropout are as they were
    with pytest.raises(RuntimeError):      # other names are still looked at
        b.load_state_dict({**a.state_dict(), "other": torch.zeros(1)})
    with pytest.raises(RuntimeError):
        b.load_state_dict({k: v for k, v in a.state_dict().items() if k != "pos"})


def test_counters_without_an_entry_stay(drawn):
    """A file from before the counter was saved loads, and leaves the counter as it is."""
    model = model_of()
    model(ids_of())
    model.load_state_dict({k: v for k, v in model.state_dict().items() if k != "drop_step"})
    assert int(model.drop_step) == 1


# ---------------------------------------------------------- the recurrent form
def test_recurrent_form_trains_with_dropout(drawn, linear):
    """Training carried from one piece of a sequence to the next has the dropout of a
    whole one: on a whole sequence both forms are the same function."""
    model = model_of(mixer="linear")
    zero = torch.zeros(2, dtype=torch.int64)
    whole = model(ids_of())
    model.drop_step.zero_()
    logits, states = model.recurrent(ids_of(), zero)
    assert torch.equal(logits, whole) and drawn[:5] == drawn[5:]
    model.recurrent(ids_of(), zero, states)                 # the next piece: new masks
    assert len(drawn) == 15 and not set(drawn[10:]) & set(drawn[:10])
    model.eval()
    a, _ = model.recurrent(ids_of(), zero)
    assert torch.equal(a, model(ids_of())) and len(drawn) == 15


# ------------------------------------------------------------------ generation
@pytest.mark.parametrize("new", [0, 1, 4])
def test_generate_gives_as_many_tokens_as_asked(linear, new):
    model = model_of(mixer="linear", dropout=0.0)
    out = gpt.generate(model, ids_of(6), new)
    assert out.shape == (2, new) and out.dtype == torch.int64
    ragged = gpt.generate(model, ids_of(6), new, torch.tensor([6, 2], dtype=torch.int32))
    assert torch.equal(ragged[0], out[0])
    alone = gpt.generate(model, ids_of(6)[1:, :2], new)
    assert torch.equal(ragged[1], alone[0])


@pytest.mark.parametrize("lengths", [[6, 0], [7, 6], [-1, 6], [6], [[6, 6]]])
def test_generate_refuses_lengths_outside_the_prompts(linear, lengths):
    model = model_of(mixer="linear", dropout=0.0)
    with pytest.raises(ValueError, match="lengths"):
        gpt.generate(model, ids_of(6), 3, torch.tensor(lengths, dtype=torch.int32))


def test_generate_refuses_empty_prompts_and_negative_counts(linear):
    model = model_of(mixer="linear", dropout=0.0)
    for ids, new in ((ids_of(0), 3), (ids_of(6), -1)):
        with pytest.raises(ValueError, match="new_tokens"):
            gpt.generate(model, ids, new)
    with pytest.raises(ValueError, match="recurrent"):
        gpt.generate(model_of(mixer="dense"), ids_of(6), 0)
