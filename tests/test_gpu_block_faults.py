"""The optimizer under capture, the norm that clips its gradients, norms whose gradients are not all
wanted or whose result takes the place of an input, and beam search's sums over a large background."""

import math

import pytest
import torch

from tests import block_reference as R
from tests import test_gpu_norms as T

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


@pytest.mark.parametrize("capturable", [False, True])
def test_a_file_of_bf16_goes_on_with_masters(cuda_ok, capturable):
    """States of torch's AdamW over bf16 weights, loaded with masters: the steps that follow are those of
    float32 weights that begin where the bf16 ones are (tolerance as in test_gpu_optim)."""
    from paper_2608_13578_gb300 import optim
    g = torch.Generator().manual_seed(0)
    shapes, how = [(40, 7), (300,), (1000,)], dict(lr=1e-3, weight_decay=0.05)
    a = [torch.nn.Parameter((torch.randn(s, generator=g) * 0.1).to(BF).cuda()) for s in shapes]

    def gradients(*lists):
        for ps in zip(*lists):
            d = torch.randn(ps[0].shape, generator=g).to(BF).cuda()
            for p in ps:
                p.grad = d.to(p.dtype)
    old = torch.optim.AdamW(a, **how)
    for _ in range(3):
        gradients(a)
        old.step()
    b = [torch.nn.Parameter(p.detach().clone()) for p in a]
    c = [torch.nn.Parameter(p.detach().float()) for p in a]
    ob, oc = optim.AdamW(b, masters=True, capturable=capturable, **how), torch.optim.AdamW(c, **how)
    file = old.state_dict()
    ob.load_state_dict(file)
    oc.load_state_dict(file)
    for s in oc.state.values():
        assert s["exp_avg"].dtype == F
    for _ in range(3):
        gradients(b, c)
        ob.step()
        oc.step()
    for p, q in zip(b, c):
        w = ob.state[p]["master"]
        assert float((w - q.detach()).abs().max()) <= 3 * 16 * (1e-3 * 2.0 ** -20 + 2 * R.U * float(q.detach().abs().max()))
        assert torch.equal(p.detach(), w.to(BF)) and int(ob.state[p]["step"]) == 6


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


# -------------------------------------------------------------------- norms
NAMES = ["branch", "x", "weight", "bias", "post_weight", "post_bias", "gate"]


def arguments(shape, dtype, post, gate, seed=0):
    g = torch.Generator().manual_seed(seed)
    D = shape[-1]
    sizes = dict(branch=shape, x=shape, weight=(D,), bias=(D,), post_weight=(D,) if post else None,
                 post_bias=(D,) if post else None, gate=gate)
    return {k: None if s is None else torch.randn(s, generator=g).to(dtype).cuda() for k, s in sizes.items()}


def both(norms, t, wanted=None):
    """Gradients of every argument (None where there is none) of sums over h and n."""
    t = {k: None if v is None else v.clone().requires_grad_(wanted is None or wanted[i])
         for i, (k, v) in enumerate(t.items())}
    h, n = norms.residual_norm(t["branch"], t["x"], t["weight"], t["bias"], post_weight=t["post_weight"],
                               post_bias=t["post_bias"], gate=t["gate"], residual_scale=0.7)
    at = torch.linspace(-1, 1, h.numel(), device="cuda", dtype=h.dtype).view(h.shape)
    ((h * at).sum() + (n * at.flip(0)).sum()).backward()
    return [None if v is None else v.grad for v in t.values()]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("D", [40, 264, 1001, 4096])
def test_gradients_that_are_wanted_are_the_same(cuda_ok, D, post, dtype):
    """Each gradient alone, and all but each one, bit for bit as all together; gates of all rows,
    of groups (with several segments, and several groups a worker), of every row, and none."""
    from paper_2608_13578_gb300 import bcmt as C, norms
    for rows, gates in ((2, 0), (700, 1), (700, 2), (700, 350), (330, 330)):
        shape = (gates, rows // gates, D) if gates else (rows, D)
        t = arguments(shape, dtype, post, (gates, 1, D) if gates else None)
        every = both(norms, t)
        for i in range(7):
            for only in (True, False):
                wanted = [(k == i) == only for k in range(7)]
                if not any(w and v is not None for w, v in zip(wanted, t.values())):
                    continue
                for k, (a, b) in enumerate(zip(both(norms, t, wanted), every)):
                    if wanted[k] and b is not None:
                        assert torch.equal(a, b), (NAMES[k], wanted, gates)
                    else:
                        assert a is None
    C.bcmt_device_status()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("over", ["x", "branch"])
@pytest.mark.parametrize("rows,D,gates", [(14600, 257, 0), (7308, 1001, 7), (3656, 2047, 3656), (1832, 4099, 1),
                                          (700, 768, 7)])
def test_result_over_an_input_of_many_rows(cuda_ok, rows, D, gates, over, dtype):
    """h over the residual or the branch where rows come in 16-byte pieces that neighbours share, and
    are requested ahead."""
    from paper_2608_13578_gb300 import bcmt as C, norms
    shape = (gates, rows // gates, D) if gates else (rows, D)
    t = arguments(shape, dtype, True, (gates, 1, D) if gates else None)
    h, n = norms.residual_norm_forward(t["branch"], t["x"], t["weight"], t["bias"], post_weight=t["post_weight"],
                                       post_bias=t["post_bias"], gate=t["gate"], residual_scale=0.5)
    dt = C.BCMT_BF16 if dtype == BF else C.BCMT_F32
    p = C.bcmt_norm_params(rows, D, dt, dt, 0, gates, 0, 0.5, 1e-5)
    for _ in range(3):
        u, m = {k: None if v is None else v.clone() for k, v in t.items()}, torch.empty_like(n)
        C.bcmt_residual_norm_forward(p, u["branch"], u["x"], u["weight"], u["bias"], u["post_weight"],
                                     u["post_bias"], u["gate"], u[over], m, torch.cuda.current_stream().cuda_stream)
        assert torch.equal(u[over], h) and torch.equal(m, n)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("kind,post,gated", [("layer", True, 1), ("rms", True, 8), ("layer", False, 0),
                                             ("rms", False, None)])
@pytest.mark.parametrize("rows,D", [(14600, 257), (14600, 511), (11000, 700), (7304, 1001), (4904, 1500),
                                    (3656, 2047), (1832, 4099), (1224, 6399)])
def test_forward_of_workers_side_by_side(cuda_ok, dtype, kind, post, gated, rows, D):
    """Enough rows of odd widths for the ring with as many workers a CTA as fit (four rows for each
    of 152 CTAs); gated: gates (None: one for every row, 0: without)."""
    from paper_2608_13578_gb300 import norms
    gates = rows if gated is None else gated
    shape = (gates, rows // gates, D) if gates else (rows, D)
    t, _, _ = T.make(shape, dtype, F, kind, post, (gates, 1, D) if gates else None)
    h, n = T.forward(norms, t, 0.9, kind)
    kw = dict(post_weight=t["post_weight"], post_bias=t["post_bias"], gate=t["gate"], kind=kind, alpha=0.9)
    (rh, rn), (bh, bn) = R.norm_forward(t["branch"], t["x"], t["weight"], t["bias"], **kw)
    T.close(h, rh, bh, T.ROUNDINGS, "h")
    T.close(n, rn, bn, T.ROUNDINGS, "n")


def full(D, post):
    """Rows that fill the backward's CTAs with as many workers as registers allow, and some more."""
    R = 32 // (8 if D <= 64 else 16 if D <= 128 else 32)
    one = D <= 512 or (post and D <= 768)      # a warp a row
    warps = 20 if D <= 256 else 12 if one and D > 512 else 16
    wide = 1 if one else (D + 511) // 512      # (J = 2 at the widths below)
    return (warps // (wide * (2 if post else 1))) * 152 * R + 8


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("kind,post,gated", [("layer", True, 1), ("rms", True, 8), ("layer", True, None),
                                             ("layer", False, 0), ("rms", False, 8)])
@pytest.mark.parametrize("D", [64, 100, 200, 256, 511, 512, 768, 1001, 1024, 2048])
def test_backward_of_workers_side_by_side(cuda_ok, D, kind, post, gated, dtype):
    """As many workers a CTA as fit, with and without a post norm."""
    from paper_2608_13578_gb300 import norms
    rows = full(D, post)
    gates = rows if gated is None else gated
    shape = (gates, rows // gates, D) if gates else (rows, D)
    t, dh, dn = T.make(shape, dtype, F, kind, post, (gates, 1, D) if gates else None)
    T.check(norms, t, dh, dn, 0.9, kind)


# -------------------------------------------------------------- beam search
V = 32000


def rows_of(background, dtype=F):
    """Logits [1, beams, V]: a best token of 0, eight tokens in every 4096 above the background,
    which the lists take, and the background itself, which they do not."""
    x = torch.tensor(background)[:, None].expand(-1, V).clone()
    x[:, ::512] += 1.0
    x[:, 77] = 0.0
    return x[None].to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [0.71875, 3.3, 6.71875, 9.828125, 11.3, 15.0])
def test_sums_over_a_large_background(cuda_ok, d, dtype):
    """The log-sum is off by the background's share of it times (3 d + 25) 2^-24 (its argument's three
    roundings, 2^-22 of ex2.approx, 20 additions), the score by a rounding of its own."""
    from paper_2608_13578_gb300 import beam
    x = rows_of([-d, -d - 0.5], dtype)
    got = beam.beam_select(x, torch.zeros(1, 2, device="cuda"))
    lp = x.double().log_softmax(-1)[0]
    for score, parent, token in zip(*[t[0].tolist() for t in got[:3]]):
        z = x[0, parent].double()
        share = float((z == z.min()).sum() * z.min().exp() / z.exp().sum())
        want = float(lp[parent, token])
        bound = share * (3 * float(z.max() - z.min()) + 25) * 2.0 ** -24 + abs(want) * 2.0 ** -24
        assert abs(score - want) <= bound, (score, want, bound)


@pytest.mark.parametrize("d", [6.71875, 9.828125])
def test_beams_that_differ_by_their_backgrounds(cuda_ok, d):
    """Best tokens of equal logits, sums whose backgrounds differ by 2^-14: the difference of the
    scores is more than twice the log-sums' bound, and decides."""
    from paper_2608_13578_gb300 import beam
    bound = 2 * (3 * math.log(V) + 25) * 2.0 ** -24
    for low in (0, 1):
        x = rows_of([-d - (k == low) * 2.0 ** -14 for k in (0, 1)])
        lp = x.double().log_softmax(-1)[0, :, 77]
        assert float(lp[low] - lp[1 - low]) > bound
        got = beam.beam_select(x, torch.zeros(1, 2, device="cuda"))
        assert got[1].tolist() == [[low, 1 - low]] and got[2].tolist() == [[77, 77]]
        got = beam.beam_select(x.repeat(1, 2, 1)[:, 1:3].contiguous(), torch.zeros(1, 2, device="cuda"))
        assert got[1].tolist() == [[1 - low, low]]
