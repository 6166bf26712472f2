"""The language-model operators on the GPU against plain float64 forms.

Tolerances, fixed from the arithmetic before any run:
 * linear attention, relative to the largest entry of the reference:
   fp32 (2 T + dh + 8) 2^-24: each of a sum's terms is decayed and added at
   most T times (two roundings each), then dh products are summed;
   bf16 outputs 4 * 2^-9: half an ulp (2^-9) each for the decayed score, the
   state's copy and the result, and one more for their alignment;
   states of bf16 inputs: the decayed key is carried in 16 bits of mantissa,
   2^-16 a term, with the fp32 figure on top.
 * embedding gradient, entry by entry: (count + 1) 2^-24 times the sum of
   magnitudes, plus 2^-8 (bf16) or 2^-23 (fp32) of the entry for its rounding.
 * lookup and dropout: two fp32 roundings and the result's.
"""

import numpy as np
import pytest
import torch

from tests import lm_reference as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def F(cuda_ok):
    from paper_2608_13578_gb300 import lm_ops
    return lm_ops


@pytest.fixture(autouse=True)
def no_wait_ran_out(F):
    """A bounded wait that expires leaves a result that may be wrong and a status."""
    from paper_2608_13578_gb300 import bcmt as C
    C.bcmt_device_status()
    yield
    C.bcmt_device_status()


def np64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def check_rel(name, got, ref, tol):
    got = np64(got)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert np.isfinite(got).all(), f"{name}: non-finite"
    scale = np.abs(ref).max()
    err = np.abs(got - ref).max()
    assert err <= tol * scale + 1e-30, f"{name}: error {err:.3e} of {scale:.3e}, tolerance {tol:.2e}"


def tolerances(dtype, T, dh):
    f32 = (2 * T + dh + 8) * 2.0 ** -24
    return (f32, f32) if dtype == "fp32" else (4 * 2.0 ** -9, 2.0 ** -16 + f32)


def make(B, T, H, dh, dtype, seed=0, state=False, lengths=None, decay=None, poison=True):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(B, T, 3, H, dh, generator=g).to(DT[dtype])
    do = torch.randn(B, T, H, dh, generator=g).to(DT[dtype])
    if decay is None:
        decay = torch.linspace(0.8, 0.998, H) if H > 1 else torch.tensor([0.97])
    s0 = torch.randn(B, H, dh, dh, generator=g) if state else None
    ds = torch.randn(B, H, dh, dh, generator=g) if state else None
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    ref = dict(q=qkv[:, :, 0].double().numpy(), k=qkv[:, :, 1].double().numpy(),
               v=qkv[:, :, 2].double().numpy(), do=do.double().numpy(),
               decay=decay.double().numpy(), s0=np64(s0), ds=np64(ds),
               n=None if n is None else n.numpy())
    qkv, do = qkv.cuda(), do.cuda()
    if n is not None and poison:   # what lies past a sequence's end must not matter
        for b in range(B):
            qkv[b, max(0, int(n[b])):] = float("nan")
            do[b, max(0, int(n[b])):] = float("inf")
    dev = dict(q=qkv[:, :, 0], k=qkv[:, :, 1], v=qkv[:, :, 2], do=do, decay=decay.cuda(),
               s0=None if s0 is None else s0.cuda(), ds=None if ds is None else ds.cuda(),
               n=None if n is None else n.cuda())
    return dev, ref


SHAPES = [
    # B, T, H, dh
    (1, 1, 1, 64), (2, 2, 2, 8), (3, 63, 2, 64), (2, 64, 1, 16), (1, 65, 3, 40), (2, 127, 2, 64),
    (1, 128, 2, 128), (2, 129, 1, 128), (1, 300, 2, 96), (2, 700, 2, 64), (1, 1500, 1, 32),
    (5, 257, 3, 24), (1, 1100, 1, 128),
]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,T,H,dh", SHAPES)
@pytest.mark.parametrize("state", [False, True], ids=["zero", "state"])
def test_linear_attention_forward(F, B, T, H, dh, dtype, state):
    d, r = make(B, T, H, dh, dtype, 1, state)
    o, S = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], state=d["s0"])
    ro, rS = R.linear_attention(r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, None, r["s0"])
    to, ts = tolerances(dtype, T, dh)
    check_rel("o", o, ro, to)
    check_rel("state", S, rS, ts)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,T,H,dh", SHAPES)
@pytest.mark.parametrize("state", [False, True], ids=["zero", "state"])
def test_linear_attention_backward(F, B, T, H, dh, dtype, state):
    d, r = make(B, T, H, dh, dtype, 2, state)
    got = F.linear_attention_backward(d["do"], d["q"], d["k"], d["v"], d["decay"], state=d["s0"],
                                      dstate=d["ds"])
    ref = R.linear_attention_grads(r["do"], r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, None,
                                   r["s0"], r["ds"])
    to, ts = tolerances(dtype, T, dh)
    for name, a, b in zip(("dq", "dk", "dv"), got, ref):
        check_rel(name, a, b, to)
    if state:
        check_rel("d_state", got[3], ref[3], ts)
    else:
        assert got[3] is None


# enough heads that one CTA walks several chunks of a head (no segments)
WALKS = [(40, 4, 128, 300), (32, 10, 64, 385), (80, 1, 96, 512), (160, 2, 40, 260)]


@pytest.mark.parametrize("B,H,dh,T", WALKS)
@pytest.mark.parametrize("ragged", [False, True], ids=["full", "ragged"])
def test_linear_attention_long_walks(F, B, H, dh, T, ragged):
    lengths = [(37 * b + 101) % (T + 1) for b in range(B)] if ragged else None
    d, r = make(B, T, H, dh, "bf16", 14, True, lengths)
    o, S = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], None, d["n"], d["s0"])
    got = F.linear_attention_backward(d["do"], d["q"], d["k"], d["v"], d["decay"], None, d["n"],
                                      d["s0"], d["ds"])
    some = [0, 1, B // 2, B - 1]
    r = {k: v if k == "decay" or v is None else v[some] for k, v in r.items()}
    ro, rS = R.linear_attention(r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, r["n"], r["s0"])
    ref = R.linear_attention_grads(r["do"], r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, r["n"],
                                   r["s0"], r["ds"])
    to, ts = tolerances("bf16", T, dh)
    for name, a, b, t in zip(("o", "state", "dq", "dk", "dv", "d_state"), (o, S, *got),
                             (ro, rS, *ref), (to, ts, to, to, to, ts)):
        check_rel(name, a[some], b, t)
        assert torch.isfinite(a).all(), name


LENGTHS = [(200, [0, 1, 200, 64]), (300, [300, 129, 128, 127]), (150, [0, 0, 0, 0]),
           (130, [129, -3, 400, 2]), (1, [1, 0, 1, 1]), (1030, [1030, 513, 0, 1024])]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128, 40])
@pytest.mark.parametrize("T,lengths", LENGTHS)
def test_linear_attention_ragged(F, T, lengths, dh, dtype):
    """Lengths of zero, of one, past the end (clamped); NaN and infinities past each end."""
    d, r = make(4, T, 2, dh, dtype, 3, True, lengths)
    o, S = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], 0.2, d["n"], d["s0"])
    ro, rS = R.linear_attention(r["q"], r["k"], r["v"], r["decay"], 0.2, r["n"], r["s0"])
    to, ts = tolerances(dtype, T, dh)
    check_rel("o", o, ro, to)
    check_rel("state", S, rS, ts)
    got = F.linear_attention_backward(d["do"], d["q"], d["k"], d["v"], d["decay"], 0.2, d["n"],
                                      d["s0"], d["ds"])
    ref = R.linear_attention_grads(r["do"], r["q"], r["k"], r["v"], r["decay"], 0.2, r["n"],
                                   r["s0"], r["ds"])
    for name, a, b, t in zip(("dq", "dk", "dv", "d_state"), got, ref, (to, to, to, ts)):
        check_rel(name, a, b, t)
    for b, n in enumerate(lengths):
        n = min(max(n, 0), T)
        for x in (o, *got[:3]):
            assert not x[b, n:].any()
        if n == 0:
            assert torch.equal(S[b], d["s0"][b]) and torch.equal(got[3][b], d["ds"][b])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dh,T", [(64, 400), (128, 260), (32, 130)])
def test_linear_attention_extreme_decays(F, dh, T, dtype):
    """No memory (0), a vanishing one (1e-30: its powers underflow), a short one and no decay (1)."""
    decay = torch.tensor([0.0, 1e-30, 0.5, 1.0])
    d, r = make(2, T, 4, dh, dtype, 4, True, decay=decay)
    to, ts = tolerances(dtype, T, dh)
    o, S = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], state=d["s0"])
    ro, rS = R.linear_attention(r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, None, r["s0"])
    got = F.linear_attention_backward(d["do"], d["q"], d["k"], d["v"], d["decay"], state=d["s0"],
                                      dstate=d["ds"])
    ref = R.linear_attention_grads(r["do"], r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, None,
                                   r["s0"], r["ds"])
    for h in range(4):
        check_rel(f"o[{h}]", o[:, :, h], ro[:, :, h], to)
        check_rel(f"state[{h}]", S[:, h], rS[:, h], ts)
        for name, a, b in zip(("dq", "dk", "dv"), got, ref):
            check_rel(f"{name}[{h}]", a[:, :, h], b[:, :, h], to)
        if r["decay"][h] > 1e-20:
            check_rel(f"d_state[{h}]", got[3][:, h], ref[3][:, h], ts)


def test_linear_attention_gradient_against_differences(F):
    """Each output is linear in q, in k, in v and in the first state, so central
    differences of the forward with any step are exact up to rounding."""
    B, T, H, dh = 2, 150, 2, 64
    d, _ = make(B, T, H, dh, "fp32", 5, True)
    q, k, v, s0 = (d[x].contiguous() for x in ("q", "k", "v", "s0"))

    def f(q, k, v, s0):
        o, S = F.linear_attention_forward(q, k, v, d["decay"], state=s0)
        return (o.double() * d["do"]).sum() + (S.double() * d["ds"]).sum()
    grads = F.linear_attention_backward(d["do"], q, k, v, d["decay"], state=s0, dstate=d["ds"])
    g = torch.Generator(device="cuda").manual_seed(9)
    args = [q, k, v, s0]
    for i, gr in enumerate(grads):
        e = torch.randn(args[i].shape, generator=g, device="cuda")
        hi, lo = list(args), list(args)
        hi[i], lo[i] = args[i] + e, args[i] - e
        diff = (f(*hi) - f(*lo)) / 2
        want = (gr.double() * e).sum()
        # rounding of each of the two sums' terms, (2 T + dh) 2^-24 of magnitudes sqrt(count)
        mag = (gr.double() * e).norm() + (d["do"].double().norm() * 64)
        assert abs(diff - want) <= (2 * T + dh) * 2.0 ** -24 * mag, (i, float(diff), float(want))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,H,dh", [(1, 8, 64), (3, 2, 128), (7, 1, 40), (2, 3, 8)])
def test_linear_attention_steps_continue_a_prompt(F, B, H, dh, dtype):
    """Prompt, then single tokens from its state: the rows of the whole sequence."""
    T, P = 90, 70
    d, r = make(B, T, H, dh, dtype, 6)
    ro, rS = R.linear_attention(r["q"], r["k"], r["v"], r["decay"], dh ** -0.5)
    o, S = F.linear_attention_forward(d["q"][:, :P], d["k"][:, :P], d["v"][:, :P], d["decay"])
    rows = [o] + [F.linear_attention_step(d["q"][:, t:t + 1], d["k"][:, t:t + 1],
                                          d["v"][:, t:t + 1], d["decay"], S) for t in range(P, T)]
    to, ts = tolerances(dtype, T, dh)
    check_rel("o", torch.cat(rows, 1), ro, to)
    check_rel("state", S, rS, ts)


def test_linear_attention_step_skips_inactive_sequences(F):
    d, r = make(4, 1, 2, 64, "bf16", 7, True)
    active = torch.tensor([1, 0, 1, 0], dtype=torch.int32, device="cuda")
    d["q"][1] = float("nan")
    S = d["s0"].clone()
    out = torch.full_like(S, float("nan"))
    o = F.linear_attention_step(d["q"], d["k"], d["v"], d["decay"], S, active=active, state_out=out)
    assert torch.equal(S, d["s0"])            # another buffer was given: the old state stays
    o2 = F.linear_attention_step(d["q"], d["k"], d["v"], d["decay"], S, active=active)
    assert torch.equal(S, out) and torch.equal(o, o2)
    assert torch.equal(S[1], d["s0"][1]) and not o[1].any() and not torch.equal(S[0], d["s0"][0])


def test_linear_attention_layouts_and_repeats(F):
    """Slices of one projection, dense tensors and transposed heads give the same
    bits, and so does every repeat, on a stream of its own too."""
    d, _ = make(2, 333, 4, 64, "bf16", 8, True)
    q, k, v = d["q"], d["k"], d["v"]
    a = F.linear_attention_forward(q, k, v, d["decay"], state=d["s0"])
    ga = F.linear_attention_backward(d["do"], q, k, v, d["decay"], state=d["s0"], dstate=d["ds"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ht = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v)]
        b = F.linear_attention_forward(*ht, d["decay"], state=d["s0"])
        gb = F.linear_attention_backward(d["do"].transpose(1, 2).contiguous().transpose(1, 2), *ht,
                                         d["decay"], state=d["s0"], dstate=d["ds"])
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip((*a, *ga), (*b, *gb)):
        assert torch.equal(x, y)


def test_linear_attention_state_in_place(F):
    for T in (1, 50, 1000):
        d, _ = make(2, T, 2, 64, "bf16", 10, True)
        o, S = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], state=d["s0"])
        s = d["s0"].clone()
        o2, s2 = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], state=s,
                                            state_out=s)
        assert s2 is s and torch.equal(o, o2) and torch.equal(S, s)


def test_linear_attention_autograd(F):
    d, r = make(2, 140, 2, 64, "bf16", 11, True)
    leaves = [d[x].clone().requires_grad_() for x in ("q", "k", "v", "s0")]
    o, S = F.linear_attention(leaves[0], leaves[1], leaves[2], d["decay"], state=leaves[3])
    torch.autograd.backward([o, S], [d["do"], d["ds"]])
    ref = R.linear_attention_grads(r["do"], r["q"], r["k"], r["v"], r["decay"], 64 ** -0.5, None,
                                   r["s0"], r["ds"])
    to, ts = tolerances("bf16", 140, 64)
    for name, x, b, t in zip(("dq", "dk", "dv", "d_state"), leaves, ref, (to, to, to, ts)):
        check_rel(name, x.grad, b, t)
    # the last state alone
    q = d["q"].clone().requires_grad_()
    k = d["k"].clone().requires_grad_()
    _, S = F.linear_attention(q, k, d["v"], d["decay"])
    S.backward(d["ds"])
    ref = R.linear_attention_grads(0 * r["do"], r["q"], r["k"], r["v"], r["decay"], 64 ** -0.5,
                                   None, None, r["ds"])
    assert not q.grad.any()
    check_rel("dk", k.grad, ref[1], to)
    with pytest.raises(ValueError):
        F.linear_attention(q, k, d["v"], d["decay"].clone().requires_grad_())


@pytest.mark.parametrize("bad", ["shape", "dtype", "decay", "lengths", "state", "half", "device"])
def test_linear_attention_refusals(F, bad):
    d, _ = make(2, 5, 2, 16, "bf16", 12, True, [3, 5], poison=False)
    a = dict(q=d["q"], k=d["k"], v=d["v"], decay=d["decay"], lengths=d["n"], state=d["s0"])
    if bad == "shape":
        a["k"] = a["k"][:, :4]
    elif bad == "dtype":
        a["v"] = a["v"].float()
    elif bad == "decay":
        a["decay"] = a["decay"].double()
    elif bad == "lengths":
        a["lengths"] = a["lengths"].long()
    elif bad == "state":
        a["state"] = a["state"][:1]
    elif bad == "half":
        a.update({x: a[x].half() for x in "qkv"})
    else:
        a["decay"] = a["decay"].cpu()
    with pytest.raises(ValueError):
        F.linear_attention_forward(**a)


# ------------------------------------------------------------------- embedding
def ids_like(kind, N, V, g):
    if kind == "same":
        return torch.full((N,), V - 1)
    if kind == "zipf":
        return (V * torch.rand(N, generator=g) ** 6).long().clamp(max=V - 1)
    return torch.randint(0, V, (N,), generator=g)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,V,D,kind,ints", [
    (1, 1, 8, "uniform", torch.int64), (31, 255, 64, "uniform", torch.int32),
    (33, 256, 72, "zipf", torch.int64), (2048, 257, 264, "zipf", torch.int64),
    (2049, 40000, 64, "uniform", torch.int32), (5000, 70000, 16, "uniform", torch.int64),
    (9000, 300, 768, "zipf", torch.int64), (20000, 512, 128, "same", torch.int64),
    (4097, 65536, 8, "zipf", torch.int64), (150001, 3000, 16, "zipf", torch.int32),
    (140000, 20, 8, "same", torch.int64), (0, 100, 16, "uniform", torch.int64),
])
def test_embedding_and_its_gradient(F, N, V, D, kind, ints, dtype):
    g = torch.Generator().manual_seed(N + V)
    ids = ids_like(kind, N, V, g).to(ints)
    w = torch.randn(V, D, generator=g).to(DT[dtype])
    dy = torch.randn(N, D, generator=g).to(DT[dtype])
    ulp = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    out = np64(F.embedding_forward(ids.cuda(), w.cuda(), 1.7))
    ref = np.float32(1.7).astype(np.float64) * w.double().numpy()[ids.numpy()]
    assert (np.abs(out - ref) <= (ulp + 2.0 ** -23) * np.abs(ref)).all()
    dw = F.embedding_backward(ids.cuda(), dy.cuda(), V, 1.7)
    ref, mag, cnt = R.embedding_grad(ids.long().numpy(), dy.double().numpy(), V,
                                     float(np.float32(1.7)))
    got = np64(dw)
    bound = (cnt[:, None] + 1) * 2.0 ** -24 * mag + ulp * np.abs(ref)
    assert got.shape == ref.shape and (np.abs(got - ref) <= bound).all()
    assert not got[cnt == 0].any()
    for _ in range(3):   # the same bits at every run
        assert torch.equal(dw, F.embedding_backward(ids.cuda(), dy.cuda(), V, 1.7))


def test_embedding_autograd_and_shapes(F):
    g = torch.Generator().manual_seed(3)
    ids = torch.randint(0, 50, (4, 37), generator=g).cuda()
    w = torch.randn(50, 24, generator=g).cuda().requires_grad_()
    dy = torch.randn(4, 37, 24, generator=g).cuda()
    out = F.embedding(ids, w, 2.0)
    assert out.shape == (4, 37, 24)
    out.backward(dy)
    ref, mag, cnt = R.embedding_grad(np64(ids).astype(int).reshape(-1), np64(dy).reshape(-1, 24),
                                     50, 2.0)
    assert (np.abs(np64(w.grad) - ref) <= (cnt[:, None] + 3) * 2.0 ** -24 * mag).all()
    # differences: the lookup is linear in the table
    e = torch.randn(50, 24, generator=g).cuda()
    d = ((F.embedding_forward(ids, w.detach() + e, 2.0).double()
          - F.embedding_forward(ids, w.detach() - e, 2.0).double()) * dy).sum() / 2
    want = (w.grad.double() * e).sum()
    assert abs(d - want) <= 8 * 2.0 ** -24 * float((2 * w.detach().abs().max() + e.abs().max())
                                                 * 2 * dy.abs().sum())


def test_embedding_ids_outside_the_table(F):
    from paper_2608_13578_gb300 import bcmt as C
    C.bcmt_device_status()
    ids = torch.tensor([3, -1, 7, 8, 3, 1 << 40], device="cuda")
    w = torch.randn(8, 16, device="cuda")
    out = F.embedding_forward(ids, w)
    with pytest.raises(C.BCMTError) as e:
        C.bcmt_device_status()
    assert e.value.code == C.BCMT_ERR_ARG
    assert torch.equal(out[[0, 2, 4]], w[[3, 7, 3]]) and not out[[1, 3, 5]].any()
    dy = torch.randn(6, 16, device="cuda")
    dw = F.embedding_backward(ids, dy, 8)
    with pytest.raises(C.BCMTError):
        C.bcmt_device_status()
    assert torch.equal(dw[3], dy[0] + dy[4]) and torch.equal(dw[7], dy[2])
    assert not dw[[0, 1, 2, 4, 5, 6]].any()
    C.bcmt_device_status()     # read and cleared
    with pytest.raises(ValueError):
        F.embedding_forward(ids.float(), w)
    with pytest.raises(ValueError):
        F.embedding_backward(ids, dy[:5], 8)


# --------------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 1001, 300007])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(F, n, p, dtype):
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, generator=g).to(DT[dtype])
    res = torch.randn(n, generator=g).to(DT[dtype])
    seed, off = 0xDEADBEEFCAFE1234, 0x1_0000_0007
    keep = R.dropout_keep(n, p, seed, off)
    ref = np.where(keep, x.double().numpy() / (1.0 - p if p < 1 else 1.0), 0.0)
    ulp = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    y = np64(F.dropout_forward(x.cuda(), p, seed, off))
    assert (np.abs(y - ref) <= (ulp + 2.0 ** -22) * np.abs(ref)).all()
    assert (y[~keep] == 0).all()
    full = ref + res.double().numpy()
    y = np64(F.dropout_forward(x.cuda(), p, seed, off, residual=res.cuda()))
    assert (np.abs(y - full) <= ulp * np.abs(full) + 2.0 ** -22 * np.abs(ref)).all()
    # the gradient is the same mask
    dx = F.dropout_backward(res.cuda(), p, seed, off)
    assert ((np64(dx) != 0) == (keep & (res.double().numpy() != 0))).all()


def test_dropout_masked_values_do_not_matter(F):
    n, p = 4099, 0.4
    keep = torch.from_numpy(R.dropout_keep(n, p, 5, 6)).cuda()
    x = torch.randn(n, device="cuda")
    y = F.dropout_forward(x, p, 5, 6)
    x[~keep] = torch.tensor([float("nan"), float("inf"), -3.4e38], device="cuda")[
        torch.arange(int((~keep).sum()), device="cuda") % 3]
    assert torch.equal(y, F.dropout_forward(x, p, 5, 6))


def test_dropout_masks_differ_and_count(F):
    n, p = 1 << 20, 0.3
    x = torch.ones(n, device="cuda")
    masks = [F.dropout_forward(x, p, s, o) != 0 for s, o in ((1, 0), (1, 1), (2, 0), (1 << 40, 0))]
    sd = (p * (1 - p) / n) ** 0.5
    for m in masks:
        assert abs(float(m.double().mean()) - (1 - p)) < 6 * sd + 2.0 ** -17
    for i in range(4):
        for j in range(i):
            both = float((masks[i] & masks[j]).double().mean())
            assert abs(both - (1 - p) ** 2) < 6 / n ** 0.5


def test_dropout_autograd_step_and_layout(F):
    x = torch.randn(33, 65, device="cuda").t().requires_grad_()      # not dense
    res = torch.randn(65, 33, device="cuda", requires_grad=True)
    step = torch.tensor([4], dtype=torch.int64, device="cuda")
    y = F.dropout(x, 0.25, 9, 10, residual=res, step=step)
    step += 1                                                          # the next step's counter
    assert torch.equal(y, F.dropout_forward(x.detach(), 0.25, 9, 14, residual=res.detach()))
    dy = torch.randn_like(y)
    y.backward(dy)
    assert torch.equal(x.grad, F.dropout_backward(dy, 0.25, 9, 14))
    assert torch.equal(res.grad, dy)
    odd = torch.randn(1001, device="cuda").bfloat16()[1:]              # not 16-byte aligned
    assert torch.equal(F.dropout_forward(odd, 0.5, 1, 2), F.dropout_forward(odd.clone(), 0.5, 1, 2))
    assert F.dropout_forward(torch.empty(0, 5, device="cuda"), 0.5, 1, 2).shape == (0, 5)
    with pytest.raises(ValueError):
        F.dropout_forward(x.detach(), 0.5, 1, 2, residual=res.detach()[:3])
    with pytest.raises(ValueError):
        F.dropout_forward(x.detach().half(), 0.5, 1, 2)


def test_operators_in_a_graph(F):
    """Capture of the three operators; a device counter draws a new mask at each replay."""
    d, _ = make(2, 200, 2, 64, "bf16", 13)
    ids = torch.randint(0, 100, (2, 200), device="cuda")
    w = torch.randn(100, 128, device="cuda").bfloat16()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def body():
        x = F.embedding_forward(ids, w, 3.0)
        y = F.dropout_forward(x, 0.2, 7, 1, step=step)
        o, S = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"])
        dw = F.embedding_backward(ids, y, 100, 3.0)
        g = F.linear_attention_backward(d["do"], d["q"], d["k"], d["v"], d["decay"])[:3]
        return [x, y, o, S, dw, *g]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        body()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = body()
    for i in range(2):
        step.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, b in zip(got, body()):
            assert torch.equal(a, b)
