"""The AdamW step over many tensors: moments and 8-bit codes bit for bit, weights against
float64, many and odd tensors, device-side steps and rates, graphs, copies and files.

Tolerance of a weight, in units of 2^-23 of its update: 7.5 for the factors after the moments
(two approximate functions of one unit in the last place, a quotient of two, six operations of
half a one), 2 for m (its constants, the gradient's scale, products and sum: four roundings of
its terms, which may cancel, so that they count by their magnitudes), 1.5 for the root of v (six
roundings, halved): 11.  Keeping and adding round the weight twice; one rounding to the
stored type."""

import copy

import numpy as np
import pytest
import torch

from tests import block_reference as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
HOW = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def O(cuda_ok):
    from paper_2608_13578_gb300 import optim
    return optim


SIZES = [(1,), (3,), (255,), (256,), (257,), (16, 16), (1000,), (0,), (64, 65), (4096,), (4097,), (3, 5, 7),
         (100, 100), (8192,)]


def make(sizes, dtype, bits, master, seed=0):
    g = torch.Generator().manual_seed(seed)
    d = dict(p=[], g=[], m=[], v=[], w=[], ms=[], vs=[])
    for s in sizes:
        p = torch.randn(*s, generator=g) * 0.1
        d["g"].append((torch.randn(*s, generator=g) * 1e-2).to(dtype).cuda())
        d["p"].append(p.to(dtype).cuda())
        d["w"].append(p.cuda())
        m, v = torch.randn(*s, generator=g) * 1e-2, torch.rand(*s, generator=g) ** 4 * 1e-3
        if bits == 8:
            mc, ms = R.encode_m(m.numpy().reshape(-1)) if m.numel() else (np.zeros(0, np.int8),) + (np.zeros(0, np.float32),)
            vc, vs = R.encode_v(v.numpy().reshape(-1)) if v.numel() else (np.zeros(0, np.uint8),) + (np.zeros(0, np.float32),)
            d["m"].append(torch.from_numpy(mc).view(s).cuda())
            d["v"].append(torch.from_numpy(vc).view(s).cuda())
            d["ms"].append(torch.from_numpy(ms).cuda())
            d["vs"].append(torch.from_numpy(vs).cuda())
        else:
            d["m"].append(m.cuda())
            d["v"].append(v.cuda())
    return d


def plan(O, d, bits, master):
    return O.AdamWPlan(d["p"], d["m"], d["v"], masters=d["w"] if master else None,
                       m_scales=d["ms"] if bits == 8 else None, v_scales=d["vs"] if bits == 8 else None)


def check(d, after, bits, master, step, scale=1.0, how=HOW):
    for i, p in enumerate(d["p"]):
        if p.numel() == 0:
            continue
        m, v = (d[k][i].cpu().numpy().reshape(-1) for k in "mv")
        if bits == 8:
            m, v = R.decode_m(m, d["ms"][i].cpu().numpy()), R.decode_v(v, d["vs"][i].cpu().numpy())
        g = d["g"][i].reshape(-1)
        nm, nv = R.moments(g, m, v, how["betas"], scale)
        if bits == 8:
            for x, s, (c, r) in ((after["m"][i], after["ms"][i], R.encode_m(nm)),
                                 (after["v"][i], after["vs"][i], R.encode_v(nv))):
                assert np.array_equal(s.cpu().numpy(), r), i
                assert np.array_equal(x.cpu().numpy().reshape(-1), c), i
        else:
            assert np.array_equal(after["m"][i].cpu().numpy().reshape(-1), nm), i
            assert np.array_equal(after["v"][i].cpu().numpy().reshape(-1), nv), i
        old = (d["w"] if master else d["p"])[i].double().cpu().numpy().reshape(-1)
        ref, up = R.adamw(old, g.double().cpu().numpy(), m, v, how["lr"], how["betas"], how["eps"],
                          how["weight_decay"], step, float(np.float32(scale)))
        tol = 11 * 2.0 ** -23 * up + 2 * R.U * np.abs(old)
        for t in ([after["w"][i]] if master else []) + [after["p"][i]]:
            got = t.double().cpu().numpy().reshape(-1)
            assert (np.abs(got - ref) <= tol + R.half_step(t.dtype) * np.abs(ref)).all(), (i, t.dtype)
        if master:
            assert torch.equal(after["p"][i], after["w"][i].to(p.dtype))


def clone(d):
    return {k: [t.clone() for t in v] for k, v in d.items()}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,master", [(F, False), (BF, False), (BF, True)])
@pytest.mark.parametrize("step,scale", [(1, None), (1234567, 0.3)])
def test_step(O, dtype, master, bits, step, scale):
    d = make(SIZES, dtype, bits, master)
    a = clone(d)
    gs = None if scale is None else torch.full((1,), scale, device="cuda")
    plan(O, a, bits, master).step(a["g"], step=step, grad_scale=gs, **HOW)
    check(d, a, bits, master, step, 1.0 if scale is None else scale)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 32, 33, 129, 385, 800])
def test_many_tensors(O, count, bits):
    """Every table of tensors, and more than one launch."""
    d = make([(1 + 37 * i % 300,) for i in range(count)], F, bits, False)
    a = clone(d)
    plan(O, a, bits, False).step(a["g"], step=7, **HOW)
    check(d, a, bits, False, 7)


@pytest.mark.parametrize("bits", [32, 8])
def test_buffers_off_the_grid(O, bits):
    """Views one element into their buffers, with what lies around them left as it was."""
    d = make([(1, 4098), (1, 300)], BF, bits, True)
    a = clone(d)
    inner = {k: [t[..., 1:-1] if t.dim() == 2 else t for t in v] for k, v in a.items()}
    ref = {k: [t[..., 1:-1].contiguous() if t.dim() == 2 else t for t in v] for k, v in d.items()}
    if bits == 8:      # scales of the shorter tensors
        for i in range(2):
            n = inner["p"][i].numel()
            for k in ("ms", "vs"):
                inner[k][i], ref[k][i] = inner[k][i][:-(-n // 256)], ref[k][i][:-(-n // 256)]
    plan(O, inner, bits, True).step(inner["g"], step=3, **HOW)
    check(ref, inner, bits, True, 3)
    for k in "pmvw":
        for x, y in zip(a[k], d[k]):
            assert torch.equal(x[..., 0], y[..., 0]) and torch.equal(x[..., -1], y[..., -1])


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_missing_and_strided(O, bits):
    d = make([(20, 30), (500,), (40,)], F, bits, False)
    d["g"][0] = d["g"][0].t().contiguous().t()       # the same values, other strides
    a = clone(d)
    a["g"][0] = d["g"][0]
    plan(O, a, bits, False).step([a["g"][0], None, a["g"][2]], step=2, **HOW)
    for k in ("p", "m", "v"):
        assert torch.equal(a[k][1], d[k][1])
    keep = [0, 2]
    check({k: [v[i] for i in keep] if v else v for k, v in d.items()},
          {k: [v[i] for i in keep] if v else v for k, v in a.items()}, bits, False, 2)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.0, 0.99), (0.9, 0.0), (0.99, 0.9999)])
def test_step_and_rate_on_the_device(O, betas, bits):
    for step in (1, 2, 1000, 10 ** 6):
        how = dict(HOW, betas=betas)
        d = make([(300,), (5000,)], F, bits, False)
        a = clone(d)
        plan(O, a, bits, False).step(a["g"], step=torch.tensor(step, device="cuda"),
                                     **dict(how, lr=torch.tensor(how["lr"], device="cuda")))
        check(d, a, bits, False, step, how=dict(how, lr=float(np.float32(how["lr"]))))


def test_codes_at_their_ends(O):
    """Blocks of zeros, of one value, of values too small for a scale, and single large
    values among small ones; codes of every size."""
    m = np.zeros(256 * 6, np.float32)
    v = np.zeros(256 * 6, np.float32)
    m[256:512], v[256:512] = 1e-3, 1e-6
    m[512:768], v[512:768] = 1e-36, 1e-37
    m[768], v[768] = 5.0, 7.0
    m[769:1024] = np.linspace(-5, 5, 255)
    v[769:1024] = np.linspace(0, 1, 255) ** 8 * 7
    m[1024:1280], v[1024:1280] = -np.geomspace(1e-8, 1, 256), np.geomspace(1e-20, 1, 256)
    m[1280:] = np.random.default_rng(0).standard_normal(256)
    mc, ms = R.encode_m(m)
    vc, vs = R.encode_v(v)
    got = O.adamw8_values(torch.from_numpy(mc).cuda(), torch.from_numpy(ms).cuda(),
                          torch.from_numpy(vc).cuda(), torch.from_numpy(vs).cuda())
    assert np.array_equal(got[0].cpu().numpy(), R.decode_m(mc, ms))
    assert np.array_equal(got[1].cpu().numpy(), R.decode_v(vc, vs))
    # a step without a gradient decays the states and encodes them again
    d = dict(p=[torch.zeros(m.size, device="cuda")], g=[torch.zeros(m.size, device="cuda")],
             m=[torch.from_numpy(mc).cuda()], v=[torch.from_numpy(vc).cuda()], w=[],
             ms=[torch.from_numpy(ms).cuda()], vs=[torch.from_numpy(vs).cuda()])
    a = clone(d)
    plan(O, a, 8, False).step(a["g"], step=5, **HOW)
    check(d, a, 8, False, 5)
    assert int(a["v"][0][1024:1280].min()) >= 1          # a small v is never taken for none


@pytest.mark.parametrize("n", [0, 1, 255, 1000, 70001])
def test_values_of_any_length(O, n):
    g = torch.Generator().manual_seed(n)
    m = torch.randint(-127, 128, (n,), generator=g, dtype=torch.int8)
    v = torch.randint(0, 256, (n,), generator=g, dtype=torch.uint8)
    ms, vs = (torch.rand(-(-n // 256), generator=g) for _ in range(2))
    got = O.adamw8_values(m.cuda(), ms.cuda(), v.cuda(), vs.cuda())
    if n:
        assert np.array_equal(got[0].cpu().numpy(), R.decode_m(m.numpy(), ms.numpy()))
        assert np.array_equal(got[1].cpu().numpy(), R.decode_v(v.numpy(), vs.numpy()))


def test_a_gradient_that_is_not_finite_shows(O):
    for bits in (32, 8):
        d = make([(600,), (300,)], F, bits, False)
        a = clone(d)
        a["g"][0][300] = float("nan")
        plan(O, a, bits, False).step(a["g"], step=1, **HOW)
        assert torch.isnan(a["p"][0][300]) and torch.isfinite(a["p"][0][:256]).all()
        assert torch.isfinite(a["p"][1]).all()
        if bits == 8:
            assert torch.isnan(a["ms"][0]).tolist() == [False, True, False]
            assert torch.isfinite(a["ms"][1]).all()
        else:
            assert int(torch.isnan(a["m"][0]).sum()) == 1


# ------------------------------------------------------------------ the optimizer
def model():
    torch.manual_seed(0)
    return torch.nn.Sequential(torch.nn.Linear(40, 70), torch.nn.GELU(), torch.nn.Linear(70, 9)).cuda()


def run(net, opt, steps, seed=1, skip=()):
    g = torch.Generator().manual_seed(seed)
    for i in range(steps):
        x = torch.randn(16, 40, generator=g).cuda()
        opt.zero_grad(set_to_none=True)
        net(x).square().sum().backward()
        if i in skip:
            net[0].bias.grad = None
        opt.step()


@pytest.mark.parametrize("skip", [(), (1, 3)])
def test_optimizer_follows_torch(O, skip):
    """Twelve steps beside torch.optim.AdamW: weights differ by the roundings of twelve
    updates of at most lr each (2^-20 of them, as above) and of the weights, which the
    gradients of a smooth loss carry on by a factor that stays near 1 at this rate."""
    a, b = model(), model()
    how = dict(lr=1e-3, betas=(0.9, 0.99), weight_decay=0.05)
    run(a, O.AdamW(a.parameters(), **how), 12, skip=skip)
    run(b, torch.optim.AdamW(b.parameters(), **how), 12, skip=skip)
    for p, q in zip(a.parameters(), b.parameters()):
        assert float((p - q).detach().abs().max()) <= 12 * 16 * (1e-3 * 2.0 ** -20 + 2 * R.U * float(q.detach().abs().max()))


def test_optimizer_groups_schedules_and_versions(O):
    net = model()
    opt = O.AdamW([dict(params=[net[0].weight, net[2].weight], weight_decay=0.1),
                   dict(params=[net[0].bias, net[2].bias], weight_decay=0.0, bits=8)], lr=1e-2)
    sched = torch.optim.lr_scheduler.StepLR(opt, 2, 0.5)
    before = [p._version for p in net.parameters()]
    for _ in range(4):
        run(net, opt, 1)
        sched.step()
    assert opt.param_groups[0]["lr"] == 1e-2 / 4
    assert all(p._version > b for p, b in zip(net.parameters(), before))
    assert opt.state[net[0].bias]["exp_avg"].dtype == torch.int8
    assert opt.state[net[0].weight]["exp_avg"].dtype == F
    assert opt.state[net[0].weight]["step"] == 4


@pytest.mark.parametrize("bits,dtype,masters", [(32, F, False), (8, F, False), (8, BF, True), (32, BF, True)])
@pytest.mark.parametrize("capturable", [False, True])
def test_resumed_and_copied_runs_are_the_same(O, bits, dtype, masters, capturable):
    how = dict(lr=1e-2, bits=bits, masters=masters, capturable=capturable)

    def start():
        net = model().to(dtype)
        return net, O.AdamW(net.parameters(), **how)

    def go(net, opt, steps, seed):
        g = torch.Generator().manual_seed(seed)
        for _ in range(steps):
            opt.zero_grad(set_to_none=True)
            net(torch.randn(16, 40, generator=g).cuda().to(dtype)).square().sum().backward()
            opt.step()
    a, oa = start()
    go(a, oa, 3, 1)
    saved, weights = copy.deepcopy(oa.state_dict()), copy.deepcopy(a.state_dict())
    pair = copy.deepcopy((a, oa))
    go(a, oa, 3, 2)
    b, ob = start()
    b.load_state_dict(weights)
    ob.load_state_dict(saved)
    go(b, ob, 3, 2)
    go(*pair, 3, 2)
    for p, q, r in zip(a.parameters(), b.parameters(), pair[0].parameters()):
        assert torch.equal(p, q) and torch.equal(p, r)
    for k, s in oa.state[next(a.parameters())].items():
        t = ob.state[next(b.parameters())][k]
        assert torch.equal(s, t) if isinstance(s, torch.Tensor) else s == t


def test_a_file_of_torch_loads(O):
    """States of torch.optim.AdamW go on here as they do there."""
    a, b = model(), model()
    how = dict(lr=1e-3, weight_decay=0.05)
    oa = torch.optim.AdamW(a.parameters(), **how)
    run(a, oa, 4)
    b.load_state_dict(a.state_dict())
    ob = O.AdamW(b.parameters(), **how)
    ob.load_state_dict(copy.deepcopy(oa.state_dict()))
    run(a, oa, 3, seed=2)
    run(b, ob, 3, seed=2)
    for p, q in zip(a.parameters(), b.parameters()):
        assert float((p - q).detach().abs().max()) <= 3 * 16 * (1e-3 * 2.0 ** -20 + 2 * R.U * float(q.detach().abs().max()))
    assert ob.state[b[0].bias]["step"] == 7


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_count_on(O, bits):
    """Replays of one captured step are the steps that follow, with a rate that changes
    between them."""
    a, b = model(), model()
    oa = O.AdamW(a.parameters(), lr=1e-2, bits=bits)
    lr = torch.tensor(1e-2, device="cuda")
    ob = O.AdamW(b.parameters(), lr=lr, bits=bits, capturable=True)
    g = torch.Generator().manual_seed(0)
    for p, q in zip(a.parameters(), b.parameters()):
        p.grad = torch.randn(p.shape, generator=g).cuda()
        q.grad = p.grad.clone()
    oa.step()
    ob.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ob.step()
    for i in range(5):
        for p, q in zip(a.parameters(), b.parameters()):
            p.grad.copy_(torch.randn(p.shape, generator=g).cuda())
            q.grad.copy_(p.grad)
        rate = 1e-2 / (1 + i)
        oa.param_groups[0]["lr"] = float(np.float32(rate))
        lr.fill_(rate)
        oa.step()
        graph.replay()
    torch.cuda.synchronize()
    assert int(ob.state[b[0].weight]["step"]) == 6
    for p, q in zip(a.parameters(), b.parameters()):
        # the rate and the corrections are taken in another order: as the tolerance of a weight
        assert float((p - q).abs().max()) <= 6 * (4e-2 * 2.0 ** -20 + 2 * R.U * float(p.abs().max()))
        for k in ("exp_avg", "exp_avg_sq"):
            assert torch.equal(oa.state[p][k], ob.state[q][k])


def test_two_steps_at_once(O):
    """Plans over different tensors on two streams."""
    d = [make([(4097,), (300,)], F, 8, False, seed=s) for s in range(2)]
    a = [clone(x) for x in d]
    plans = [plan(O, x, 8, False) for x in a]
    torch.cuda.synchronize()
    for i, x in enumerate(a):
        with torch.cuda.stream(torch.cuda.Stream()):
            plans[i].step(x["g"], step=3, **HOW)
    torch.cuda.synchronize()
    for x, y in zip(d, a):
        check(x, y, 8, False, 3)
