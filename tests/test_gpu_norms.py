"""The norms around a block against their float64 forms: outputs, every gradient, gates of
every broadcast, odd widths, strides, streams, devices, graphs and values that are not
finite.

Tolerances: a quantity passes at most three sums over a row (each at most 32 roundings in
a thread, 5 over a warp's lanes and 16 over its warps) and 20 other operations, so its
error is within 180 roundings of the bound in which all terms count by their magnitude;
sums over the rows of a test add at most 70 (rows of a worker, workers, CTAs); one
rounding to the stored type."""

import pytest
import torch

from tests import block_reference as R

pytestmark = pytest.mark.gpu
ROUNDINGS, COLUMNS = 180, 70
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def N(cuda_ok):
    from paper_2608_13578_gb300 import norms
    return norms


def make(shape, dtype, wtype, kind, post, gate, bias=True, post_bias=True, seed=0):
    """Arguments of a call: a gate of shape ``gate`` (None: without)."""
    g = torch.Generator().manual_seed(seed)

    def rnd(*s, std=1.0, mean=0.0, dt=dtype):
        return (torch.randn(*s, generator=g) * std + mean).to(dt).cuda()
    D = shape[-1]
    t = dict(branch=rnd(*shape), x=rnd(*shape, std=2.0, mean=0.3),
             weight=rnd(D, std=0.2, mean=1.0, dt=wtype), bias=rnd(D, std=0.2, dt=wtype) if bias else None,
             post_weight=rnd(D, std=0.2, mean=0.5, dt=wtype) if post else None,
             post_bias=rnd(D, std=0.2, dt=wtype) if post and post_bias else None,
             gate=rnd(*gate, std=0.5, mean=0.2) if gate is not None else None)
    return t, rnd(*shape), rnd(*shape)


def close(got, ref, bound, roundings, what):
    assert got is not None, what
    tol = roundings * R.U * bound + R.half_step(got.dtype) * ref.abs() + 1e-37
    bad = (got.double().cpu() - ref).abs() / tol
    assert bad.shape == ref.shape and bool((bad <= 1).all()), (what, float(bad.max()))


def forward(N, t, alpha, kind, eps=1e-5):
    return N.residual_norm_forward(t["branch"], t["x"], t["weight"], t["bias"],
                                   post_weight=t["post_weight"], post_bias=t["post_bias"],
                                   gate=t["gate"], residual_scale=alpha, kind=kind, eps=eps)


def check(N, t, dh, dn, alpha, kind, eps=1e-5):
    kw = dict(post_weight=t["post_weight"], post_bias=t["post_bias"], gate=t["gate"], kind=kind, eps=eps)
    h, n = forward(N, t, alpha, kind, eps)
    (rh, rn), (bh, bn) = R.norm_forward(t["branch"], t["x"], t["weight"], t["bias"], alpha=alpha, **kw)
    close(h, rh, bh, ROUNDINGS, "h")
    close(n, rn, bn, ROUNDINGS, "n")
    got = dict(zip(R.NAMES, N.residual_norm_backward(dh, dn, t["branch"], h, t["weight"], t["bias"],
                                                     residual_scale=alpha, **kw)))
    ref, bound = R.norm_backward(dh, dn, t["branch"], h, t["weight"], t["bias"], alpha=alpha, **kw)
    for k in R.NAMES:
        if k not in ref:
            assert got[k] is None, k
            continue
        own = dict(dbranch="branch", dx="x", dgate="gate").get(k, k[1:])
        assert got[k].dtype == t[own].dtype
        summed = k not in ("dbranch", "dx")
        close(got[k], ref[k], bound[k], ROUNDINGS + (COLUMNS if summed else 0), k)


SHAPES = [(1, 1), (1, 7), (3, 8), (1, 2, 16), (2, 33, 64), (5, 3, 100), (2, 64, 128), (4, 9, 129),
          (2, 30, 136), (61, 255), (7, 256), (3, 11, 264), (130, 511), (8, 40, 512), (2, 16, 768),
          (3, 5, 1001), (33, 1024), (9, 1032), (2, 3, 2047), (4, 4, 2048), (17, 2056), (3, 4095),
          (2, 7, 4096), (5, 4104), (2, 8191), (1, 3, 8192)]


@pytest.mark.parametrize("dtype,wtype", [(BF, BF), (BF, F), (F, F), (F, BF)],
                         ids=["bf16", "bf16-w32", "fp32", "fp32-w16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(N, shape, dtype, wtype):
    i = SHAPES.index(shape)
    kind = ("layer", "rms")[i % 2]
    gates = [None, (shape[-1],), shape] + ([(shape[0], 1, shape[-1])] if len(shape) == 3 else [])
    for post, gate in ((True, gates[-1]), (False, gates[i % len(gates)]), (True, gates[1]), (False, None)):
        t, dh, dn = make(shape, dtype, wtype, kind, post, gate, bias=kind == "layer",
                         post_bias=kind == "layer", seed=i)
        check(N, t, dh, dn, 0.7 if i % 3 else 1.0, kind)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("post,post_bias", [(True, True), (True, False), (False, False)])
@pytest.mark.parametrize("gate", [None, (96,), (3, 1, 96), (3, 20, 96), (1, 1, 96), (1, 96)], ids=str)
def test_parts(N, kind, bias, post, post_bias, gate):
    t, dh, dn = make((3, 20, 96), BF, F, kind, post, gate, bias, post_bias)
    check(N, t, dh, dn, 1.0, kind)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rows,D,gates", [(4096, 64, 1), (3000, 96, 50), (1500, 768, 3), (1216, 512, 0),
                                          (997, 520, 997), (700, 2048, 7), (610, 4096, 2), (320, 8192, 5),
                                          (610, 1001, 610), (1400, 201, 2)])
def test_many_rows(N, dtype, rows, D, gates):
    """More rows than workers: segments, and gates whose rows are several segments."""
    shape = (gates, rows // gates, D) if gates else (rows, D)
    t, dh, dn = make(shape, dtype, F, "layer", True, (gates, 1, D) if gates else None)
    check(N, t, dh, dn, 0.9, "layer")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("kind,post,gated", [("layer", True, 1), ("rms", True, 8), ("layer", False, 0),
                                             ("rms", False, None)])
@pytest.mark.parametrize("rows,D", [(9800, 131), (9736, 257), (9728, 511), (4872, 1001), (2440, 2047), (1232, 4095),
                                    (1600, 5001), (1216, 8191)])
def test_forward_over_many_odd_rows(N, dtype, kind, post, gated, rows, D):
    """Rows that come in pieces, the last of which is cut short; gated: gates (None: one for
    every row, 0: without)."""
    gates = rows if gated is None else gated
    shape = (gates, rows // gates, D) if gates else (rows, D)
    t, _, _ = make(shape, dtype, F, kind, post, (gates, 1, D) if gates else None)
    h, n = forward(N, t, 0.9, kind)
    kw = dict(post_weight=t["post_weight"], post_bias=t["post_bias"], gate=t["gate"], kind=kind, alpha=0.9)
    (rh, rn), (bh, bn) = R.norm_forward(t["branch"], t["x"], t["weight"], t["bias"], **kw)
    close(h, rh, bh, ROUNDINGS, "h")
    close(n, rn, bn, ROUNDINGS, "n")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("rows,D,gates", [(3000, 64, 1500), (4100, 100, 2050), (3000, 768, 1500), (900, 1001, 450),
                                          (800, 5000, 400), (480, 7676, 160), (480, 8192, 160)])
def test_more_gates_than_workers(N, dtype, post, rows, D, gates):
    """Workers that walk the segments of several gates, a few rows each."""
    t, dh, dn = make((gates, rows // gates, D), dtype, dtype, "layer", post, (gates, 1, D))
    check(N, t, dh, dn, 1.0, "layer")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("post,post_bias", [(True, True), (True, False), (False, False)])
@pytest.mark.parametrize("rows,D", [(1, 72), (5, 2056), (7, 5001), (160, 6152), (3, 7676), (160, 8191), (157, 8192)])
def test_gates_of_every_row(N, dtype, post, post_bias, rows, D):
    t, dh, dn = make((rows, D), dtype, F, "layer", post, (rows, D), post_bias=post_bias)
    check(N, t, dh, dn, 1.0, "layer")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("D", [40, 321, 1024, 6000])
def test_no_gradient_of_the_sum(N, D, dtype):
    t, _, dn = make((2, 6, D), dtype, dtype, "layer", True, (2, 1, D))
    check(N, t, None, dn, 1.0, "layer")


@pytest.mark.parametrize("D", [16, 100, 768, 4096])
def test_constant_rows_and_offsets(N, D):
    """Rows without variance, and rows whose mean is large against their deviation."""
    t, dh, dn = make((6, D), F, F, "layer", False, None)
    t["branch"].zero_()
    t["x"][0] = 0.0
    t["x"][1] = 3.0
    t["x"][2] += 1000.0
    check(N, t, dh, dn, 1.0, "layer")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("D", [16, 100, 264, 768, 1001, 4096])
def test_rows_whose_first_element_stands_out(N, D, dtype):
    """The backward takes a row's squares less its first element: an outlier there, a row of
    nothing else, and one that hides a small deviation behind a large mean."""
    t, dh, dn = make((3, 5, D), dtype, F, "layer", True, (3, 1, D))
    for y in (t["branch"], t["x"]):
        y[0, 0, 0] = 1e4
        y[1, 2] = 0.0
        y[1, 2, 0] = -3e3
        y[2, 1] = 0.01 * y[2, 1] + 64.0
        y[2, 1, 0] = 0.0
    check(N, t, dh, dn, 1.0, "layer")


@pytest.mark.parametrize("D", [24, 1001])
def test_not_finite_rows_stay_apart(N, D):
    t, dh, dn = make((3, 9, D), BF, BF, "rms", True, (3, 1, D), bias=False, post_bias=False)
    h0, n0 = forward(N, t, 1.0, "rms")
    t["x"][1, 4, 3] = float("inf")
    t["branch"][2, 0, 1] = float("nan")
    h, n = forward(N, t, 1.0, "rms")
    keep = torch.ones(3, 9, dtype=torch.bool)
    keep[1, 4] = keep[2, 0] = False
    assert torch.equal(h[keep], h0[keep]) and torch.equal(n[keep], n0[keep])
    assert torch.isinf(h[1, 4, 3]) and torch.isnan(h[2, 0]).all() and torch.isnan(n[2, 0]).all()
    args = dict(post_weight=t["post_weight"], gate=t["gate"], kind="rms")
    clean = N.residual_norm_backward(dh, dn, t["branch"].nan_to_num(0.0), h0, t["weight"], **args)
    got = N.residual_norm_backward(dh, dn, t["branch"], h, t["weight"], **args)
    for a, b in zip(got[:2], clean[:2]):
        assert torch.equal(a[keep], b[keep])
    assert torch.isfinite(got[6][0]).all()        # a gate whose rows are finite


def test_strides_and_offsets(N):
    """Slices, transposed rows and buffers off the 16-byte grid are copied."""
    g = torch.Generator().manual_seed(1)
    big = torch.randn(4, 10, 3, 72, generator=g).cuda()
    branch, x = big[:, :, 1], big.permute(1, 0, 2, 3)[:, :, 2].transpose(0, 1)
    w = torch.randn(145, generator=g).cuda()
    kw = dict(post_weight=w[73:], gate=big[:, :1, 0])
    h, n = N.residual_norm_forward(branch, x, w[1:73], **kw)
    a, b = N.residual_norm_forward(branch.clone(), x.clone(), w[1:73].clone(), post_weight=w[73:].clone(),
                                   gate=big[:, :1, 0].clone())
    assert torch.equal(h, a) and torch.equal(n, b)
    back = N.residual_norm_backward(x, branch, branch, h, w[1:73], **kw)
    same = N.residual_norm_backward(x.clone(), branch.clone(), branch.clone(), h, w[1:73].clone(),
                                    post_weight=w[73:].clone(), gate=big[:, :1, 0].clone())
    assert all(torch.equal(p, q) for p, q in zip(back, same) if p is not None)


@pytest.mark.parametrize("D", [48, 333])
def test_autograd_against_differences(N, D):
    """The gradient of a function of both results against central differences of the
    float64 form, along random directions."""
    t, dh, dn = make((2, 5, D), F, F, "layer", True, (2, 1, D), seed=3)
    names = ["branch", "x", "weight", "bias", "post_weight", "post_bias", "gate"]
    leaves = {k: t[k].clone().requires_grad_() for k in names}
    h, n = N.residual_norm(leaves["branch"], leaves["x"], leaves["weight"], leaves["bias"],
                           post_weight=leaves["post_weight"], post_bias=leaves["post_bias"],
                           gate=leaves["gate"], residual_scale=0.8)
    ((h * dh).sum() + (n * dn).sum()).backward()

    def value(args):
        (a, b), _ = R.norm_forward(*[args[k] for k in names], alpha=0.8)
        return (a * dh.double().cpu()).sum() + (b * dn.double().cpu()).sum()
    _, bound = R.norm_backward(dh, dn, t["branch"], h.detach(), t["weight"], t["bias"], t["post_weight"],
                               t["post_bias"], t["gate"], alpha=0.8)
    of = dict(zip(["branch", "x"] + names[2:], R.NAMES))
    g = torch.Generator().manual_seed(5)
    for k in names:
        d = torch.randn(t[k].shape, generator=g, dtype=torch.float64)
        e, at = 1e-5, {q: v.double().cpu() for q, v in t.items()}
        up, down = value({**at, k: at[k] + e * d}), value({**at, k: at[k] - e * d})
        slope = (up - down) / (2 * e)
        got = (leaves[k].grad.double().cpu() * d).sum()
        # the gradient: its own roundings and as many again from those of h; the differences:
        # e^2 = 1e-10 times third derivatives and 2^-53 / e = 1e-11 of the value
        tol = 2 * (ROUNDINGS + COLUMNS) * R.U * (bound[of[k]] * d.abs()).sum() + 1e-7 * abs(slope) + 1e-7
        assert abs(got - slope) <= tol, (k, float(got), float(slope), float(tol))


def test_shared_tensors_and_reuse(N):
    """One tensor as branch and residual, one weight for both norms, and a result used
    twice: their gradients add up; the second derivative is refused."""
    x = torch.randn(4, 6, 40, device="cuda", dtype=F).requires_grad_()
    w = torch.ones(40, device="cuda").requires_grad_()
    h, n = N.residual_norm(x, x, w, post_weight=w, kind="rms")
    (g1, gw) = torch.autograd.grad((h + n * 2 + h * n).sum(), (x, w), create_graph=True)
    second = g1.sum()
    xd, wd = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()

    def rms(z):
        return z / (z.square().mean(-1, keepdim=True) + 1e-5).sqrt() * wd
    hd = xd + rms(xd)
    nd = rms(hd)
    r1, rw = torch.autograd.grad((hd + nd * 2 + hd * nd).sum(), (xd, wd))
    # the cotangents h and n are themselves results: twice the roundings of a gradient
    g1, gw = g1.detach(), gw.detach()
    assert float((g1 - r1).abs().max()) <= 2 * ROUNDINGS * R.U * 40
    assert float((gw - rw).abs().max()) <= 2 * (ROUNDINGS + COLUMNS) * R.U * 24 * 40
    with pytest.raises(RuntimeError):
        torch.autograd.grad(second, x)


def test_equal_gradients_are_not_written_twice(N):
    """Without post norm, gate and scale the two row gradients are equal; leaves that share
    them accumulate apart."""
    x, y = (torch.randn(3, 16, device="cuda").requires_grad_() for _ in range(2))
    w = torch.ones(16, device="cuda")
    for _ in range(2):
        h, n = N.residual_norm(x, y, w)
        (h.sum() + (n * n).sum()).backward()
    first = x.grad.clone()
    assert torch.equal(x.grad, y.grad)
    x.grad.zero_()
    assert torch.equal(y.grad, first)


def test_only_one_result_used(N):
    t, dh, dn = make((2, 5, 64), F, F, "layer", True, None)
    for use in ("h", "n"):
        b = t["branch"].clone().requires_grad_()
        h, n = N.residual_norm(b, t["x"], t["weight"], t["bias"], post_weight=t["post_weight"])
        (h if use == "h" else n).backward(dh)
        zero = torch.zeros_like(dh)
        ref, bound = R.norm_backward(dh if use == "h" else zero, dh if use == "n" else zero, t["branch"],
                                     h, t["weight"], post_weight=t["post_weight"])
        close(b.grad, ref["dbranch"], bound["dbranch"], ROUNDINGS, use)


def test_empty(N):
    for shape in ((0, 64), (2, 0, 64)):
        t, dh, dn = make(shape, BF, F, "layer", True, None)
        h, n = forward(N, t, 1.0, "layer")
        assert h.shape == n.shape == shape
        got = N.residual_norm_backward(dh, dn, t["branch"], h, t["weight"], t["bias"],
                                       post_weight=t["post_weight"], post_bias=t["post_bias"])
        assert got[0].shape == shape and all(float(g.abs().sum()) == 0 for g in got[2:6])
    t, dh, dn = make((2, 0, 64), BF, F, "layer", True, (2, 1, 64))
    h, n = forward(N, t, 1.0, "layer")
    got = N.residual_norm_backward(dh, dn, t["branch"], h, t["weight"], t["bias"], gate=t["gate"])
    assert got[6].shape == (2, 1, 64) and float(got[6].float().abs().sum()) == 0


def test_repeatable_on_streams_and_in_graphs(N):
    """The same bits from a call, from two at once on two streams, and from two graphs that
    share nothing but their inputs."""
    t, dh, dn = make((16, 100, 264), BF, F, "layer", True, (16, 1, 264))

    def call():
        h, n = forward(N, t, 1.0, "layer")
        return [h, n, *N.residual_norm_backward(dh, dn, t["branch"], h, t["weight"], t["bias"],
                                                post_weight=t["post_weight"], post_bias=t["post_bias"],
                                                gate=t["gate"])]
    want = call()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(call())
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(call())
        graphs.append(g)
    for _ in range(2):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for out in got:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_captured_forward_and_backward(N):
    """(No eager graph of the same leaves may live then: the autograd engine would wait for
    the stream that it was made on.)"""
    t, dh, dn = make((4, 30, 72), F, F, "rms", True, (4, 1, 72), bias=False, post_bias=False)
    leaves = [t[k].requires_grad_() for k in ("branch", "x", "weight", "post_weight", "gate")]

    def run():
        h, n = N.residual_norm(leaves[0], leaves[1], leaves[2], post_weight=leaves[3], gate=leaves[4],
                               kind="rms")
        return torch.autograd.grad((h, n), leaves, (dh, dn))
    want = run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dn.copy_(dh)                          # a replay reads its inputs anew
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, run()))


def test_result_over_an_input(N):
    """The C call may write h over the residual or the branch."""
    from paper_2608_13578_gb300 import bcmt as C
    for over in ("x", "branch"):
        for D in (96, 101, 5000):
            t, _, _ = make((7, D), BF, BF, "layer", True, None)
            h, n = forward(N, t, 0.5, "layer")
            p = C.bcmt_norm_params(7, D, C.BCMT_BF16, C.BCMT_BF16, 0, 0, 0, 0.5, 1e-5)
            m = torch.empty_like(n)
            C.bcmt_residual_norm_forward(p, t["branch"], t["x"], t["weight"], t["bias"], t["post_weight"],
                                         t["post_bias"], None, t[over], m,
                                         torch.cuda.current_stream().cuda_stream)
            assert torch.equal(t[over], h) and torch.equal(m, n)


def test_gradients_that_are_not_wanted(N):
    """The C call computes only what it is given a place for."""
    from paper_2608_13578_gb300 import bcmt as C
    for D in (64, 1001, 8000):
        t, dh, dn = make((2, 12, D), F, F, "rms", True, (2, 1, D))
        h, _ = forward(N, t, 1.0, "rms")
        want = N.residual_norm_backward(dh, dn, t["branch"], h, t["weight"], t["bias"],
                                        post_weight=t["post_weight"], post_bias=t["post_bias"],
                                        gate=t["gate"], kind="rms")
        p = C.bcmt_norm_params(24, D, C.BCMT_F32, C.BCMT_F32, 1, 2, 0, 1.0, 1e-5)
        ws = torch.empty(C.bcmt_residual_norm_workspace_size(p, True), dtype=torch.uint8, device="cuda")
        out = [torch.empty_like(want[0])] + [None] * 6
        s = torch.cuda.current_stream().cuda_stream
        names = ["weight", "bias", "post_weight", "post_bias"]
        for only in (None, 0, 1, 2, 3):
            got = [None if i != only else torch.empty_like(t[k]) for i, k in enumerate(names)]
            C.bcmt_residual_norm_backward(p, dh, dn, t["branch"], h, t["weight"], t["post_weight"],
                                          t["post_bias"], t["gate"], out[0], None, *got, None, ws, s)
            assert torch.equal(out[0], want[0])
            if only is not None:
                assert torch.equal(got[only], want[2 + only])
