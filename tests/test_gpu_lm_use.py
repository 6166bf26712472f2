"""The language-model operators as programs use them, beyond their values: what
autograd sees of a state that is written in place, derivatives of derivatives,
arguments in every form that Python takes."""

import numpy as np
import pytest
import torch

from tests import lm_reference as R
from tests.test_gpu_lm_ops import F, make, no_wait_ran_out, tolerances  # noqa: F401

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


# ---------------------------------------------------- derivatives of derivatives
def test_penalties_on_gradients(F):
    """Embedding and dropout are linear: a penalty on their gradients reaches the
    leaves, as through torch's own operations in float64.  Tolerance: four passes
    through fp32 arithmetic with sums of up to 40 terms each."""
    ids = torch.randint(0, 9, (4, 10), generator=torch.Generator().manual_seed(5)).cuda()
    target = torch.randn(4, 10, 16, device="cuda")
    w0 = torch.randn(9, 16, device="cuda")
    keep = F.dropout_forward(torch.ones_like(target), 0.25, 3, 8) != 0
    grads = []
    for fn, dt in ((lambda w: F.dropout(F.embedding(ids, w, 1.5), 0.25, 3, 8), torch.float32),
                   (lambda w: w[ids] * 1.5 * keep / 0.75, torch.float64)):
        w = w0.detach().clone().to(dt).requires_grad_()
        loss = ((fn(w) - target.to(dt)) ** 2).sum()
        g, = torch.autograd.grad(loss, w, create_graph=True)
        (loss + (g ** 2).sum()).backward()
        grads.append(w.grad.double())
    assert (grads[0] - grads[1]).abs().max() <= 4 * 48 * 2.0 ** -24 * grads[1].abs().max()


def test_second_derivative_of_linear_attention_raises(F):
    d, _ = make(1, 40, 2, 64, "fp32", 33)
    q = d["q"].clone().requires_grad_()
    o, _ = F.linear_attention(q, d["k"], d["v"], d["decay"])
    g, = torch.autograd.grad((o ** 2).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        ((o ** 2).sum() + (g ** 2).sum()).backward()


# ------------------------------------------------- numbers given as tensors
def test_a_number_held_by_a_tensor_is_read_at_each_call(F):
    """scale and p may be one-element tensors or arrays: each call takes the value of
    then, and a backward that of its forward."""
    d, _ = make(1, 40, 2, 64, "fp32", 34)
    scale = torch.tensor(0.25)
    ids, w = torch.arange(4, device="cuda"), torch.randn(4, 16, device="cuda")
    for value in (0.25, 0.5):
        scale.fill_(value)
        args = (d["q"], d["k"], d["v"], d["decay"])
        assert torch.equal(F.linear_attention_forward(*args, scale)[0],
                           F.linear_attention_forward(*args, value)[0])
        assert torch.equal(F.linear_attention_backward(d["do"], *args, scale)[2],
                           F.linear_attention_backward(d["do"], *args, value)[2])
        assert torch.equal(F.embedding_forward(ids, w, scale), F.embedding_forward(ids, w, value))
        assert torch.equal(F.embedding_backward(ids, w, 4, scale),
                           F.embedding_backward(ids, w, 4, value))
        assert torch.equal(F.dropout_forward(w, scale, 1, 2), F.dropout_forward(w, value, 1, 2))


@pytest.mark.parametrize("op", ["linear_attention", "embedding", "dropout"])
def test_a_backward_takes_the_number_of_its_forward(F, op):
    d, _ = make(1, 40, 2, 64, "fp32", 35)
    ids = torch.arange(4, device="cuda")
    w0 = torch.randn(4, 16, device="cuda")

    def grad(number, after=None):
        x = (d["q"] if op == "linear_attention" else w0).detach().clone().requires_grad_()
        if op == "linear_attention":
            y = F.linear_attention(x, d["k"], d["v"], d["decay"], number)[0]
        elif op == "embedding":
            y = F.embedding(ids, x, number)
        else:
            y = F.dropout(x, number, 1, 2)
        if after is not None:
            number.fill_(after)
        y.sum().backward()
        return x.grad
    assert torch.equal(grad(torch.tensor(0.25), 0.5), grad(0.25))
    with pytest.raises(ValueError, match="gradient"):
        grad(torch.tensor(0.25, requires_grad=True))


# ------------------------------------------------------------ decays out of range
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [1, 20, 300])
@pytest.mark.parametrize("bad", [-0.5, -1e-6, 1.0 + 2.0 ** -23, 2.0, float("inf"), float("nan")])
def test_a_decay_outside_its_range_is_reported(F, bad, T, dtype):
    from paper_2608_13578_gb300 import bcmt as C
    good, worse = torch.tensor([0.9, 0.0, 1.0]).cuda(), torch.tensor([0.9, bad, 1.0]).cuda()
    d, _ = make(2, T, 3, 64, dtype, 36, True)

    def calls(decay):
        yield F.linear_attention_forward(d["q"], d["k"], d["v"], decay, state=d["s0"])
        yield F.linear_attention_backward(d["do"], d["q"], d["k"], d["v"], decay, state=d["s0"],
                                          dstate=d["ds"])
    for right, wrong in zip(calls(good), calls(worse)):
        with pytest.raises(C.BCMTError, match="decay") as e:
            C.bcmt_device_status()
        assert e.value.code == C.BCMT_ERR_ARG
        for x, y in zip(right, wrong):     # the other heads are what they were
            h = 1 if x.shape[1] == 3 and x.shape[2] == 64 else 2
            keep = torch.tensor([0, 2], device="cuda")
            assert torch.equal(x.index_select(h, keep), y.index_select(h, keep))
    list(calls(good))
    C.bcmt_device_status()                 # the ends of the range are in it


def test_a_call_with_the_check_flag_reports_the_decay(F):
    from paper_2608_13578_gb300 import bcmt as C
    x = torch.zeros(1, 4, 2, 8, device="cuda")
    p = C.bcmt_linattn_params(1, 4, 2, 8, C.BCMT_F32, C.BCMT_FLAG_CHECK, 0.5)
    decay = torch.tensor([0.5, 1.5], device="cuda")
    ws = torch.empty(C.bcmt_linattn_workspace_size(p, False), dtype=torch.uint8, device="cuda")
    with pytest.raises(C.BCMTError, match="decay"):
        C.bcmt_linattn_forward(p, x, 16, x, 16, x, 16, decay, None, None, torch.empty_like(x), 16,
                               None, ws)


# ------------------------------------------------------------- dropout near p = 1
@pytest.mark.parametrize("p", [0.1, 0.25, 0.6, 0.75, 0.7777, 0.9, 0.99, 0.999, 0.99997, 0.99999,
                               1 - 2.0 ** -17, 1 - 2.0 ** -30])
def test_dropout_keeps_the_expectation(F, p):
    """The kept elements' scale times the mask's rate is 1 to 2^-15 (and half an ulp of
    fp32), at every p below 1; up to 0.75 the scale is 1 / (1 - p) itself."""
    n = 1 << 20
    t = min(round(65536 * p), 65535)
    keep = R.dropout_keep(n, t / 65536, 77, 5)
    assert keep.any()
    for call in (F.dropout_forward, F.dropout_backward):
        y = call(torch.ones(n, device="cuda"), p, 77, 5).double().cpu().numpy()
        assert ((y != 0) == keep).all()
        scale = y[keep]
        assert (scale == scale[0]).all()
        assert abs(scale[0] * (65536 - t) / 65536 - 1) <= 2.0 ** -15 + 2.0 ** -23
        if p <= 0.75:
            assert scale[0] == np.float32(1 / (1 - p))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [5, 4096, 1000003])
def test_dropout_in_place(F, n, dtype):
    """The C entry point takes x or the residual as y: the bits of a call apart."""
    from paper_2608_13578_gb300 import bcmt as C
    x, r = (torch.randn(n, device="cuda").to(dtype) for _ in range(2))
    p = C.bcmt_dropout_params(n, C.BCMT_BF16 if dtype == torch.bfloat16 else C.BCMT_F32, 0, 0.3,
                              11, 12, None)
    plain = F.dropout_forward(x, 0.3, 11, 12)
    added = F.dropout_forward(x, 0.3, 11, 12, residual=r)
    for y, src, res, want in ((x.clone(), None, None, plain), (x.clone(), None, r, added),
                              (r.clone(), x, "y", added), (x.clone(), None, "y", None)):
        if want is None:    # x, residual and y are one
            want = F.dropout_forward(x, 0.3, 11, 12, residual=x)
        C.bcmt_dropout(p, y if src is None else src, y if isinstance(res, str) else res, y)
        assert torch.equal(y, want)


# --------------------------------------------------------- table gradient, many ids
@pytest.mark.parametrize("N,V,kind", [(2097152, 300, "uniform"), (2097153, 300, "uniform"),
                                      (2500001, 40000, "zipf"), (5000000, 70000, "uniform"),
                                      (3000000, 200, "same")])
def test_table_gradient_of_millions_of_ids(F, N, V, kind):
    """Against float64 sums on the device; tolerance as in test_gpu_lm_ops."""
    g = torch.Generator(device="cuda").manual_seed(N)
    if kind == "same":
        ids = torch.full((N,), V - 1, device="cuda")
    else:
        u = torch.rand(N, generator=g, device="cuda", dtype=torch.float64)
        ids = (V * (u ** 6 if kind == "zipf" else u)).long().clamp(max=V - 1)
    dy = torch.randn(N, 8, generator=g, device="cuda")
    dw = F.embedding_backward(ids, dy, V, 1.5)
    ref = torch.zeros(V, 8, dtype=torch.float64, device="cuda").index_add_(0, ids, 1.5 * dy.double())
    mag = torch.zeros_like(ref).index_add_(0, ids, 1.5 * dy.double().abs())
    cnt = torch.bincount(ids, minlength=V).view(V, 1)
    assert ((dw - ref).abs() <= (cnt + 1) * 2.0 ** -24 * mag + 2.0 ** -23 * ref.abs()).all()
    assert torch.equal(dw, F.embedding_backward(ids, dy, V, 1.5))


def test_table_gradient_time_grows_with_the_ids(F):
    """Eight times the ids take about eight times as long, not 64."""
    def ms(N):
        ids = torch.randint(0, 40000, (N,), device="cuda", dtype=torch.int32)
        dy = torch.zeros(N, 8, device="cuda", dtype=torch.bfloat16)
        best = float("inf")
        for _ in range(4):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            F.embedding_backward(ids, dy, 40000)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        return best
    small, large = ms(1 << 23), ms(1 << 26)
    assert large <= 16 * small, (small, large)


# --------------------------------------------------------- values that are not finite
def same_where_finite(name, got, ref, tol):
    """Finite exactly where the definition is, and within tol of its largest entry there."""
    got = got.detach().double().cpu().numpy()
    ok = np.isfinite(ref)
    assert (np.isfinite(got) == ok).all(), (name, int((np.isfinite(got) != ok).sum()))
    if ok.any():
        assert np.abs(got[ok] - ref[ok]).max() <= tol * np.abs(ref[ok]).max(), name


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("where", ["q", "k", "v", "do"])
@pytest.mark.parametrize("B,H,dh,T,at,dtype,ragged", [
    (1, 2, 64, 300, 150, "bf16", False), (2, 2, 128, 260, 259, "bf16", False),
    (1, 2, 40, 700, 0, "bf16", False), (1, 3, 128, 1500, 1100, "bf16", True),
    (32, 10, 64, 385, 200, "bf16", True), (40, 4, 96, 300, 77, "bf16", False),
    (1, 2, 64, 300, 150, "fp32", False), (1, 2, 64, 20, 11, "bf16", False),
])
@pytest.mark.filterwarnings("ignore::RuntimeWarning")
def test_what_is_not_finite_stays_where_it_belongs(F, B, H, dh, T, at, dtype, ragged, where, value):
    """An infinity or NaN of one entry reaches the rows and channels that the definition
    lets it reach: no earlier row of an output, no later one of a gradient."""
    lengths = [T - 3 * (b % 7) if b else T for b in range(B)] if ragged else None
    d, r = make(B, T, H, dh, dtype, 41, True, lengths)
    for x in (d, r):
        x[where][0, at, H - 1, 5] = value
    some = sorted({0, B - 1})
    r = {x: y if x == "decay" or y is None else y[some] for x, y in r.items()}
    o, S = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], None, d["n"], d["s0"])
    got = F.linear_attention_backward(d["do"], d["q"], d["k"], d["v"], d["decay"], None, d["n"],
                                      d["s0"], d["ds"])
    ro, rS = R.linear_attention(r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, r["n"], r["s0"])
    ref = R.linear_attention_grads(r["do"], r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, r["n"],
                                   r["s0"], r["ds"])
    to, ts = tolerances(dtype, T, dh)
    for name, x, y, t in zip(("o", "state", "dq", "dk", "dv", "d_state"), (o, S, *got),
                             (ro, rS, *ref), (to, ts, to, to, to, ts)):
        same_where_finite(name, x[some], y, t)


def test_rows_before_a_value_that_is_not_finite_keep_their_bits(F):
    """The rows that it does not reach are those of a call without it, where the kernel
    had them finite: other chunks of 128 tokens, and other heads and channels."""
    d, _ = make(2, 700, 2, 64, "bf16", 42)
    want, _ = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"])
    d["v"][1, 300, 0, 7] = float("nan")
    o, _ = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"])
    bad = torch.zeros_like(o, dtype=torch.bool)
    bad[1, 300:, 0, 7] = True
    redone = torch.zeros_like(bad)
    redone[1, 256:300, 0, 7] = True
    assert o[bad].isnan().all() and torch.equal(o[~bad & ~redone], want[~bad & ~redone])
    scale = want.float().abs().max()
    assert (o[redone].float() - want[redone].float()).abs().max() <= 4 * 2.0 ** -9 * scale


# ------------------------------------------------------------------- the model
def test_a_captured_training_forward_draws_new_masks(F):
    """Replays of one captured call of a model with dropout move its counter on."""
    from paper_2608_13578_gb300 import gpt
    c = gpt.GPTConfig(vocab=64, D=64, H=2, layers=1, mlp=64, L=16, T=32, mixer="linear",
                      embed_scale=1.0, dropout=0.3)
    model = gpt.build(c, dtype=torch.float32)
    ids = torch.randint(0, 64, (2, 32), generator=torch.Generator().manual_seed(1)).cuda()
    with torch.no_grad():
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            model(ids)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = model(ids)
        model.drop_step.zero_()
        replayed = []
        for _ in range(3):
            graph.replay()
            replayed.append(out.clone())
        assert int(model.drop_step) == 3
        model.drop_step.zero_()
        for got in replayed:
            assert torch.equal(got, model(ids))
        assert not torch.equal(replayed[0], replayed[1])
