"""What autograd does with the language-model operators (CPU only): the bare calls
are replaced by float64 forms that, like the library's kernels, return tensors
outside the graph."""

import pytest
import torch

from tests import lm_reference as R


@pytest.fixture
def F(monkeypatch):
    from paper_2608_13578_gb300 import build
    build.build()
    from paper_2608_13578_gb300 import lm_ops

    def linear(q, k, v, decay, scale=None, lengths=None, state=None, state_out=None):
        a = [x.detach().numpy() for x in (q, k, v, decay)]
        s = None if state is None else state.detach().numpy()
        return tuple(map(torch.from_numpy, R.linear_attention(*a, scale, None, s)))

    def linear_back(do, q, k, v, decay, scale=None, lengths=None, state=None, dstate=None,
                    need_dstate=None):
        a = [x.detach().numpy() for x in (do, q, k, v, decay)]
        s, ds = (None if x is None else x.detach().numpy() for x in (state, dstate))
        return tuple(map(torch.from_numpy, R.linear_attention_grads(*a, scale, None, s, ds)))

    def embed(ids, weight, scale=1.0):
        return weight.detach()[ids] * scale

    def embed_back(ids, dout, V, scale=1.0):
        dw, _, _ = R.embedding_grad(ids.reshape(-1).numpy(),
                                    dout.detach().reshape(-1, dout.shape[-1]).numpy(), V, scale)
        return torch.from_numpy(dw)

    def drop(x, p, seed, offset, residual=None, step=None):
        keep = R.dropout_keep(x.numel(), p, seed, offset + (0 if step is None else int(step)))
        y = x.detach() * torch.from_numpy(keep).view(x.shape) / (1 - p)
        return y if residual is None else y + residual.detach()

    def drop_back(dy, p, seed, offset, step=None):
        return drop(dy, p, seed, offset, None, step)
    for name, fn in (("linear_attention_forward", linear), ("linear_attention_backward", linear_back),
                     ("embedding_forward", embed), ("embedding_backward", embed_back),
                     ("dropout_forward", drop), ("dropout_backward", drop_back)):
        monkeypatch.setattr(lm_ops, name, fn)
    return lm_ops


def normal(*shape, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def penalised(out, leaf, target):
    """An ordinary loss and a penalty on its gradient, as one: its gradient of leaf."""
    loss = ((out - target) ** 2).sum()
    g, = torch.autograd.grad(loss, leaf, create_graph=True)
    (loss + (g ** 2).sum()).backward()
    return leaf.grad


def test_penalty_on_the_embedding_gradient(F):
    ids = torch.tensor([[3, 1, 3], [0, 3, 5]])
    target = normal(2, 3, 8, seed=1)
    grads = []
    for fn in (lambda w: F.embedding(ids, w, 1.5), lambda w: w[ids] * 1.5):
        w = normal(7, 8, seed=2).requires_grad_()
        grads.append(penalised(fn(w), w, target))
    # the same sums of six products each, in float64
    assert torch.allclose(grads[0], grads[1], rtol=1e-13, atol=1e-13)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("step", [False, True])
def test_penalty_on_the_dropout_gradient(F, residual, step):
    keep = torch.from_numpy(R.dropout_keep(60, 0.3, 5, 7)).view(6, 10)
    target = normal(6, 10, seed=3)
    counter = torch.tensor([3]) if step else None
    offset = 4 if step else 7
    grads = []
    for fn in (lambda x, r: F.dropout(x, 0.3, 5, offset, residual=r, step=counter),
               lambda x, r: keep * x / (1 - 0.3) + (0 if r is None else r)):
        x = normal(6, 10, seed=4).requires_grad_()
        r = normal(6, 10, seed=5).requires_grad_() if residual else None
        out = fn(x, r)
        if counter is not None:
            counter += 1           # moved on before the derivatives are taken
        grads.append(penalised(out, x, target))
        if counter is not None:
            counter -= 1
    assert torch.allclose(grads[0], grads[1], rtol=1e-13, atol=1e-13)


def test_second_derivative_of_linear_attention_raises(F):
    q, k, v = (normal(1, 5, 2, 8, seed=s) for s in (6, 7, 8))
    s0 = normal(1, 2, 8, 8, seed=9)
    decay = torch.tensor([0.9, 0.5], dtype=torch.float64)
    leaves = [x.requires_grad_() for x in (q, k, v, s0)]
    o, _ = F.linear_attention(q, k, v, decay, 0.3, state=s0)
    first = torch.autograd.grad((o ** 2).sum(), leaves, retain_graph=True)
    again = torch.autograd.grad((o ** 2).sum(), leaves, create_graph=True)
    for a, b in zip(first, again):
        assert torch.equal(a, b)    # the first derivative is as it was
    with pytest.raises(RuntimeError, match="once_differentiable"):
        ((o ** 2).sum() + sum((g ** 2).sum() for g in again)).backward()
