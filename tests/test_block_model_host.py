"""Host side of the GPT's use of the norms around a block, the optimizer and beam search
(CPU only): the operators are replaced by torch forms of them."""

import itertools
import math

import pytest
import torch

from paper_2608_13578_gb300 import gpt
from tests.test_lm_model_host import drawn, linear  # noqa: F401


def config(**kw):
    base = dict(vocab=13, D=16, H=2, layers=2, mlp=32, L=16, T=12, mixer="linear")
    return gpt.GPTConfig(**{**base, **kw})


def model_of(**kw):
    return gpt.build(config(**kw), device="cpu", dtype=torch.float32)


def ids_of(n=8, B=2, vocab=13):
    return torch.randint(0, vocab, (B, n), generator=torch.Generator().manual_seed(1))


@pytest.fixture
def plain(monkeypatch):
    """The operators in torch; the calls of the norms, in order."""
    calls = []

    def norm(z, w, b, kind, eps):
        if kind == "layer":
            z = z - z.mean(-1, keepdim=True)
        z = z / (z.square().mean(-1, keepdim=True) + eps).sqrt() * w
        return z if b is None else z + b

    def residual_norm(branch, x, weight, bias=None, *, post_weight=None, post_bias=None, gate=None,
                      residual_scale=1.0, kind="layer", eps=1e-5):
        calls.append((kind, post_weight is not None, gate is not None, residual_scale, eps))
        z = branch if post_weight is None else norm(branch, post_weight, post_bias, kind, eps)
        h = residual_scale * x + (z if gate is None else gate * z)
        return h, norm(h, weight, bias, kind, eps)

    def select(logits, scores, finished=None, eos=None):
        N, K, V = logits.shape
        lp = logits.double().log_softmax(-1)
        if finished is not None:
            end = torch.full((V,), -math.inf, dtype=lp.dtype)
            end[eos] = 0
            lp = torch.where(finished[..., None], end, lp)
        c = (scores.double()[..., None] + lp).reshape(N, K * V)
        best, at = torch.sort(c, dim=1, descending=True, stable=True)
        at, p = at[:, :K], at[:, :K] // V
        t = at % V
        was = torch.zeros(N, K, dtype=torch.bool) if finished is None else finished.gather(1, p)
        return best[:, :K].float(), p, t, was | (t == (-1 if eos is None else eos))

    def reorder(tensors, parents, out=None):
        N, K = parents.shape
        return [t.view(N, K, -1)[torch.arange(N)[:, None], parents].view(t.shape) for t in tensors]
    monkeypatch.setattr(gpt.norms, "residual_norm", residual_norm)
    monkeypatch.setattr(gpt.beam, "beam_select", select)
    monkeypatch.setattr(gpt.beam, "beam_reorder", reorder)
    return calls


# -------------------------------------------------------------------- norms
def test_layer_norms_are_the_same_model(plain, linear):
    """block_norm="layer" alone computes what the model computes without it, with weights
    of the same names."""
    a, b = model_of(), model_of(block_norm="layer")
    b.load_state_dict(a.state_dict())
    x = ids_of()
    assert torch.allclose(a(x), b(x), atol=1e-5)
    assert len(plain) == 4 and set(plain) == {("layer", False, False, 1.0, 1e-5)}
    pos = torch.zeros(2, dtype=torch.int64)
    for m in (a, b):
        whole, (one, states) = m(x), m.recurrent(x[:, :5], pos)
        two, _ = m.recurrent(x[:, 5:], pos + 5, states)
        assert torch.allclose(torch.cat([one, two], 1), whole, atol=1e-5)


def test_post_norms_gates_and_scales(plain, linear):
    m = model_of(block_norm="rms", post_norm=True, branch_gate=0.25, residual_scale=0.5)
    names = {n for n, _ in m.named_parameters()}
    assert {"blocks.0.post1.weight", "blocks.1.gate2", "ln_f.weight"} <= names
    assert not any(n.endswith(("ln1.bias", "post2.bias", "ln_f.bias")) for n in names)
    assert all(float(b.gate1.detach().sum()) == 4.0 for b in m.blocks)
    m(ids_of()).square().sum().backward()
    assert all(p.grad is not None and torch.isfinite(p.grad).all() for p in m.parameters())
    assert set(plain) == {("rms", True, True, 0.5, 1e-5)}


def test_dropout_before_the_norms(plain, drawn, linear):
    m = model_of(block_norm="layer", dropout=0.25)
    m(ids_of())
    assert len(drawn) == 5 and len(set(drawn)) == 5
    m.drop_step.zero_()
    m.recurrent(ids_of(), torch.zeros(2, dtype=torch.int64))
    assert drawn[5:] == drawn[:5]


def test_what_needs_a_block_norm():
    for kw in (dict(post_norm=True), dict(branch_gate=0.1), dict(residual_scale=0.5), dict(block_norm="batch")):
        with pytest.raises(ValueError, match="block_norm"):
            model_of(**kw)


def test_models_without_a_layer(plain):
    m = model_of(block_norm="layer", layers=0)
    assert m(ids_of()).shape == (2, 8, 13)


# ---------------------------------------------------------------- optimizers
def test_optimizers(plain):
    m = model_of()
    assert type(gpt.make_optimizer(m)) is torch.optim.AdamW
    for bits in (32, 8):
        opt = gpt.make_optimizer(m, lr=1e-2, bits=bits, masters=True)
        assert type(opt) is gpt.optim.AdamW
        assert opt.defaults["bits"] == bits and opt.defaults["masters"] and opt.defaults["weight_decay"] == 0.1
    with pytest.raises(ValueError, match="masters"):
        gpt.make_optimizer(m, masters=True)


def test_clipping(plain, linear, monkeypatch):
    """With the library's optimizer the scale goes into the step; it is clip over the
    gradients' norm, at most 1."""
    got = []
    monkeypatch.setattr(gpt.optim.AdamW, "step", lambda self, closure=None, *, grad_scale=None: got.append(
        (grad_scale, torch.cat([p.grad.reshape(-1) for p in m.parameters()]).norm())))
    m = model_of()
    opt = gpt.make_optimizer(m, bits=32)
    for clip in (0.01, 1e6, 0.0):
        gpt.train_step(m, opt, ids_of(), ids_of(), clip=clip)
    assert torch.allclose(got[0][0], 0.01 / got[0][1], rtol=1e-4)
    assert float(got[1][0]) == 1.0 and got[2][0] is None
    torch_opt = gpt.make_optimizer(m)
    gpt.train_step(m, torch_opt, ids_of(), ids_of(), clip=0.01)


# -------------------------------------------------------------- beam search
def score_of(model, prompt, tokens):
    """Sum of the log probabilities of tokens after the prompt."""
    ids = torch.cat([prompt, tokens])
    lp = model(ids[None]).double().log_softmax(-1)[0]
    n = len(prompt)
    return sum(float(lp[n - 1 + i, t]) for i, t in enumerate(tokens))


@torch.no_grad()
def test_all_continuations(plain, linear):
    """With a beam for every continuation the search is exhaustive."""
    m = model_of(vocab=5)
    prompts = ids_of(4, 2, 5)
    tokens, scores = gpt.beam_search(m, prompts, 2, 25)
    for b in range(2):
        every = sorted(((score_of(m, prompts[b], torch.tensor(t)), t)
                        for t in itertools.product(range(5), repeat=2)), reverse=True)
        assert [tuple(t) for t in tokens[b].tolist()] == [t for _, t in every]
        assert torch.allclose(scores[b].double(), torch.tensor([s for s, _ in every]).double(), atol=1e-5)


@torch.no_grad()
def test_scores_belong_to_their_tokens(plain, linear):
    m = model_of(block_norm="rms")
    prompts, lengths = ids_of(6, 3), torch.tensor([6, 2, 4], dtype=torch.int32)
    tokens, scores = gpt.beam_search(m, prompts, 4, 3, lengths)
    assert tokens.shape == (3, 3, 4) and tokens.dtype == torch.int64
    for b in range(3):
        for k in range(3):
            s = score_of(m, prompts[b, :lengths[b]], tokens[b, k])
            assert abs(s - float(scores[b, k])) < 1e-4
    assert bool((scores.diff(dim=1) <= 0).all())
    alone, s = gpt.beam_search(m, prompts[1:2, :2], 4, 3)
    assert torch.equal(alone[0], tokens[1])


@torch.no_grad()
def test_one_beam_is_greedy(plain, linear):
    m = model_of()
    tokens, _ = gpt.beam_search(m, ids_of(), 5, 1)
    assert torch.equal(tokens[:, 0], gpt.generate(m, ids_of(), 5))


@torch.no_grad()
def test_ends(plain, linear):
    """A beam that has ended keeps its score and goes on with the end token."""
    m = model_of(vocab=5)
    prompts = ids_of(4, 2, 5)
    tokens, scores = gpt.beam_search(m, prompts, 4, 25, eos=3)
    some = 0
    for b in range(2):
        for k in range(25):
            t = tokens[b, k].tolist()
            n = t.index(3) + 1 if 3 in t else 4
            some += n < 4
            assert t[n:] == [3] * (4 - n)
            assert abs(score_of(m, prompts[b], tokens[b, k, :n]) - float(scores[b, k])) < 1e-4
    assert some


@torch.no_grad()
def test_more_beams_than_continuations(plain, linear):
    m = model_of(vocab=5)
    tokens, scores = gpt.beam_search(m, ids_of(4, 1, 5), 1, 7)
    assert torch.isinf(scores[0, 5:]).all() and torch.isfinite(scores[0, :5]).all()
    assert sorted(tokens[0, :5, 0].tolist()) == list(range(5))


def test_beam_search_refusals(plain, linear):
    m = model_of()
    tokens, scores = gpt.beam_search(m, ids_of(), 0, 3)
    assert tokens.shape == (2, 3, 0) and scores.shape == (2, 3)
    for args, kw in (((ids_of(), 3, 0), {}), ((ids_of(), 3, 33), {}), ((ids_of(), -1, 2), {}), ((ids_of(0), 3, 2), {}),
                     ((ids_of(), 3, 2), dict(eos=13)), ((ids_of(), 3, 2), dict(eos=-1)),
                     ((ids_of(), 3, 2), dict(lengths=torch.tensor([0, 8], dtype=torch.int32)))):
        with pytest.raises(ValueError):
            gpt.beam_search(m, *args, **kw)
    with pytest.raises(ValueError, match="recurrent"):
        gpt.beam_search(model_of(mixer="dense"), ids_of(), 3, 2)
    assert m.training


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_norm_that_clips(dtype):
    """The scale is that of the gradients' norm, also for bf16 gradients.  A sum of n squares in
    fp32 is off by at most n 2^-24 in any order, its root by half of that: 2^-13 for 4121; the few
    other operations are far within the rest of 2^-12.  (A norm of 0.6426 rounded to bf16 is off by
    0.3 percent.)"""
    params = [torch.nn.Parameter(torch.zeros(n, dtype=d)) for n, d in ((4121, dtype), (7, dtype), (50, torch.float32))]
    g = torch.Generator().manual_seed(0)
    for p in params:
        p.grad = (torch.full(p.shape, 0.01) if p.numel() > 100 else torch.randn(p.shape, generator=g) * 1e-3).to(p.dtype)
    norm = math.sqrt(sum(float(p.grad.double().square().sum()) for p in params))
    scale = gpt._clip_scale(params, 0.5)
    assert scale.dtype == torch.float32 and scale.shape == ()
    assert abs(float(scale) * (norm + 1e-6) / 0.5 - 1.0) <= 2.0 ** -12
    assert float(gpt._clip_scale(params, 1e9)) == 1.0
