"""The language-model operators together, as the GPT of gpt.py uses them: training
steps with linear attention, the scaled embedding and dropout, and generation
from the recurrent state."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def config(**kw):
    from paper_2608_13578_gb300 import gpt
    base = dict(vocab=512, D=128, H=2, layers=2, mlp=256, L=32, T=200, mixer="linear",
                embed_scale=1.0)
    return gpt.GPTConfig(**{**base, **kw})


def train(cfg, dtype=torch.bfloat16, steps=8):
    from paper_2608_13578_gb300 import gpt
    model = gpt.build(cfg, dtype=dtype)
    opt = gpt.make_optimizer(model, lr=2e-3)
    g = torch.Generator().manual_seed(3)
    ids = torch.randint(0, cfg.vocab, (2, cfg.T + 1), generator=g).cuda()
    losses = [gpt.train_step(model, opt, ids[:, :-1], ids[:, 1:]).item() for _ in range(steps)]
    return model, losses


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("mixer,p", [("linear", 0.0), ("linear", 0.1), ("bcmt", 0.1)])
def test_training_steps(cuda_ok, mixer, p, dtype):
    from paper_2608_13578_gb300 import bcmt as C
    model, losses = train(config(mixer=mixer, dropout=p), dtype)
    C.bcmt_device_status()
    assert all(l == l and l < 20 for l in losses), losses
    assert losses[-1] < losses[0] - 0.5, losses
    assert int(model.drop_step) == (8 if p > 0 else 0)
    if mixer == "linear":   # near 1 the decays would not survive a cast to bf16
        assert model.blocks[0].mix.decay.dtype == torch.float32
        assert float(model.blocks[0].mix.decay[-1]) == 1 - 2.0 ** -9


def test_training_is_repeatable_and_seeded(cuda_ok):
    a = train(config(dropout=0.2), steps=4)[1]
    assert a == train(config(dropout=0.2), steps=4)[1]
    assert a != train(config(dropout=0.2, dropout_seed=1), steps=4)[1]
    assert a != train(config(), steps=4)[1]


def test_embedding_matches_torch_in_the_model(cuda_ok):
    """embed_scale = 1 is the same model as PyTorch's embedding."""
    import torch.nn.functional as F
    from paper_2608_13578_gb300 import gpt
    grads = []
    for scale in (0.0, 1.0):
        model = gpt.build(config(embed_scale=scale), dtype=torch.float32)
        ids = torch.randint(0, 512, (2, 201), generator=torch.Generator().manual_seed(5)).cuda()
        logits = model(ids[:, :-1])
        F.cross_entropy(logits.reshape(-1, 512), ids[:, 1:].reshape(-1)).backward()
        grads.append(model.tok.weight.grad)
    # both sum the same rows in fp32, in orders of their own
    assert torch.allclose(grads[0], grads[1], rtol=1e-4, atol=1e-7)


@pytest.mark.parametrize("ragged", [False, True])
def test_generation_follows_the_full_forward(cuda_ok, ragged):
    from paper_2608_13578_gb300 import gpt
    model, _ = train(config(), torch.float32, steps=3)
    B, n, new = 3, 90, 12
    ids = torch.randint(0, 512, (B, n), generator=torch.Generator().manual_seed(6)).cuda()
    lengths = [90, 1, 41] if ragged else [n] * B
    lt = torch.tensor(lengths, dtype=torch.int32, device="cuda") if ragged else None
    out = gpt.generate(model, ids, new, lt)
    assert out.shape == (B, new) and model.training
    model.eval()
    for b in range(B):
        seq = torch.cat([ids[b, :lengths[b]], out[b]])[None]
        with torch.no_grad():
            logits = model(seq)[0]
        for i in range(new):   # the greedy choice, up to ties at fp32 rounding
            row = logits[lengths[b] - 1 + i]
            assert row[out[b, i]] >= row.max() - 1e-3 * row.abs().max()
    with pytest.raises(ValueError):
        gpt.generate(gpt.build(config(mixer="dense"), dtype=torch.float32), ids, 2)


def test_recurrent_states_continue(cuda_ok):
    """A sequence read in pieces through its states gives the rows of one pass."""
    model, _ = train(config(), torch.float32, steps=2)
    model.eval()
    ids = torch.randint(0, 512, (2, 150), generator=torch.Generator().manual_seed(7)).cuda()
    zero = torch.zeros(2, dtype=torch.int64, device="cuda")
    with torch.no_grad():
        full = model(ids)
        a, st = model.recurrent(ids[:, :70], zero)
        b, st = model.recurrent(ids[:, 70:149], zero + 70, st)
        c, st = model.recurrent(ids[:, 149:], zero + 149, st)
    got = torch.cat([a, b, c], 1)
    assert (got - full).abs().max() <= 1e-3 * full.abs().max()
