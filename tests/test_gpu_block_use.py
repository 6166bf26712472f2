"""The norms around a block, the optimizer and beam search together, as the GPT of gpt.py
uses them: training steps and the search from the trained weights."""

import pytest
import torch

from tests import block_reference as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def config(**kw):
    from paper_2608_13578_gb300 import gpt
    base = dict(vocab=512, D=128, H=2, layers=2, mlp=256, L=32, T=200, mixer="linear", embed_scale=1.0,
                block_norm="layer")
    return gpt.GPTConfig(**{**base, **kw})


def data(cfg, B=2, n=None):
    g = torch.Generator().manual_seed(3)
    return torch.randint(0, cfg.vocab, (B, (n or cfg.T) + 1), generator=g).cuda()


@pytest.mark.parametrize("dtype,bits,masters", [(BF, 8, True), (BF, 32, False), (F, 8, False), (F, 32, False)])
@pytest.mark.parametrize("kw", [{}, dict(block_norm="rms", post_norm=True, branch_gate=0.5, residual_scale=0.9),
                                dict(mixer="bcmt", post_norm=True), dict(mixer="dense", branch_gate=1.0, dropout=0.1)],
                         ids=["layer", "rms-post-gate", "bcmt", "dense-dropout"])
def test_training_steps(cuda_ok, kw, dtype, bits, masters):
    """Steps run, every weight gets a gradient and moves, and two runs are the same."""
    from paper_2608_13578_gb300 import bcmt as C, gpt
    cfg = config(**kw)
    runs = []
    for _ in range(2):
        model = gpt.build(cfg, dtype=dtype)
        before = [p.detach().clone() for p in model.parameters()]
        opt = gpt.make_optimizer(model, lr=2e-3, bits=bits, masters=masters)
        ids = data(cfg)
        losses = [gpt.train_step(model, opt, ids[:, :-1], ids[:, 1:], clip=1.0).item() for _ in range(4)]
        assert all(x == x and x < 20 for x in losses), losses
        assert all(not torch.equal(a, p) and bool(torch.isfinite(p).all())
                   for a, p in zip(before, model.parameters()))
        runs.append(losses + [float(p.detach().double().sum()) for p in model.parameters()])
    C.bcmt_device_status()
    if cfg.mixer == "linear":       # no operation whose order changes from run to run
        assert runs[0] == runs[1]


@pytest.mark.parametrize("kw", [{}, dict(block_norm="rms", post_norm=True, branch_gate=0.5, residual_scale=0.9)],
                         ids=["layer", "rms-post-gate"])
def test_model_gradients_against_torch(cuda_ok, kw):
    """One fp32 model with the library's norms beside the same model with the norms in
    torch: 4 norms and 2 additions a block differ by their roundings (180 each), which the
    products between them carry on; the largest gradients are of the order of 1."""
    from paper_2608_13578_gb300 import gpt, norms
    cfg = config(**kw)
    model = gpt.build(cfg, dtype=F)
    ids = data(cfg)

    def norm(z, w, b, kind, eps):
        if kind == "layer":
            z = z - z.mean(-1, keepdim=True)
        z = z / (z.square().mean(-1, keepdim=True) + eps).sqrt() * w
        return z if b is None else z + b

    def plain(branch, x, weight, bias=None, *, post_weight=None, post_bias=None, gate=None, residual_scale=1.0,
              kind="layer", eps=1e-5):
        z = branch if post_weight is None else norm(branch, post_weight, post_bias, kind, eps)
        h = residual_scale * x + (z if gate is None else gate * z)
        return h, norm(h, weight, bias, kind, eps)
    grads = []
    own = norms.residual_norm
    allow = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        for f in (own, plain):
            norms.residual_norm = f
            model.zero_grad(set_to_none=True)
            torch.nn.functional.cross_entropy(model(ids[:, :-1]).flatten(0, 1), ids[:, 1:].flatten()).backward()
            grads.append([p.grad.clone() for p in model.parameters()])
    finally:
        norms.residual_norm = own
        torch.backends.cuda.matmul.allow_tf32 = allow
    for (n, _), a, b in zip(model.named_parameters(), *grads):
        assert float((a - b).abs().max()) <= 12 * 180 * R.U * max(1.0, float(b.abs().max())), n


def test_a_captured_training_step(cuda_ok):
    """A whole step, optimizer and all, captured: replays are the steps that follow."""
    from paper_2608_13578_gb300 import gpt, optim
    cfg = config(post_norm=True, branch_gate=0.5)
    losses = []
    for captured in (False, True):
        model = gpt.build(cfg, dtype=BF)
        opt = optim.AdamW(model.parameters(), lr=2e-3, bits=8, masters=True, capturable=True)
        ids = data(cfg)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            out = [gpt.train_step(model, opt, ids[:, :-1], ids[:, 1:], clip=1.0).detach().clone() for _ in range(2)]
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                loss = gpt.train_step(model, opt, ids[:, :-1], ids[:, 1:], clip=1.0)
            for _ in range(3):
                graph.replay()
                out.append(loss.detach().clone())
        else:
            for _ in range(3):
                out.append(gpt.train_step(model, opt, ids[:, :-1], ids[:, 1:], clip=1.0).detach().clone())
        torch.cuda.synchronize()
        losses.append([float(x) for x in out])
    assert losses[0] == losses[1]


@pytest.mark.parametrize("dtype", [BF, F])
def test_beam_search(cuda_ok, dtype):
    """Beams of ragged prompts: scores are those of their tokens, one beam is the greedy
    continuation, ended beams stay as they are, and searches do not disturb one another."""
    from paper_2608_13578_gb300 import bcmt as C, gpt
    cfg = config(block_norm="rms", post_norm=True)
    model = gpt.build(cfg, dtype=dtype)
    ids = data(cfg, 5, 40)[:, :40]
    lengths = torch.tensor([40, 7, 23, 1, 16], dtype=torch.int32, device="cuda")
    one, _ = gpt.beam_search(model, ids, 6, 1, lengths)
    assert torch.equal(one[:, 0], gpt.generate(model, ids, 6, lengths))
    tokens, scores = gpt.beam_search(model, ids, 6, 4, lengths)
    assert bool((scores.diff(dim=1) <= 0).all())
    alone, s = gpt.beam_search(model, ids[2:3, :23], 6, 4)
    if dtype == F:     # in bf16 another batch rounds its products in another order
        assert torch.equal(alone[0], tokens[2])
    # the scores, from one pass over prompt and continuation
    with torch.no_grad():
        model.eval()
        for b in (0, 1):
            n = int(lengths[b])
            rows = torch.cat([ids[b, :n].expand(4, n), tokens[b]], 1)
            lp = model(rows).double().log_softmax(-1)[:, n - 1:-1]
            want = lp.gather(2, tokens[b][..., None]).sum((1, 2))
            # logits differ by the roundings of a model of 2 blocks: each of 6 tokens' log
            # probabilities by 16 half steps of logits below 4
            tol = 6 * 16 * 4 * (R.half_step(BF) if dtype == BF else 40 * R.U)
            assert float((want - scores[b].double()).abs().max()) <= tol
        model.train()
    eos = int(tokens[0, 0, 2])
    ended, se = gpt.beam_search(model, ids, 6, 4, lengths, eos=eos)
    for b in range(5):
        for k in range(4):
            t = ended[b, k].tolist()
            if eos in t:
                assert set(t[t.index(eos):]) == {eos}
    C.bcmt_device_status()
