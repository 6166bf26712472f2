"""Refusals of the norms around a block, the AdamW step and beam search's step (CPU only:
every check comes before any kernel)."""

import copy
import ctypes
import pickle

import pytest
import torch

A = 1 << 20          # an address that no check reads


@pytest.fixture(scope="module")
def C():
    from paper_2608_13578_gb300 import build
    build.build()
    from paper_2608_13578_gb300 import bcmt
    return bcmt


@pytest.fixture
def host(C, monkeypatch):
    """The torch-facing modules with tensors in host memory taken for the device's."""
    from paper_2608_13578_gb300 import beam, norms, optim
    for m in (beam, norms, optim):
        monkeypatch.setattr(m, "_device", lambda t: t.device)
        monkeypatch.setattr(m, "_raw_stream", lambda index: 0)
        if hasattr(m, "_current_device"):
            monkeypatch.setattr(m, "_current_device", lambda: None)
    return beam, norms, optim


def code(C, call, *args):
    with pytest.raises(C.BCMTError) as e:
        call(*args)
    return e.value.code


# ------------------------------------------------------------------------- norms
def norm_params(C, **kw):
    base = dict(rows=6, D=8, dtype=C.BCMT_F32, wtype=C.BCMT_F32, rms=0, gates=0, flags=0, alpha=1.0, eps=1e-5)
    return C.bcmt_norm_params(**{**base, **kw})


def norm_forward(C, p, **kw):
    names = ("branch", "x", "weight", "bias", "post_weight", "post_bias", "gate", "h", "n")
    base = dict(zip(names, (A, A, A, None, None, None, None, A, A)))
    C.bcmt_residual_norm_forward(p, *{**base, **kw}.values(), 0)


def norm_backward(C, p, **kw):
    names = ("dh", "dn", "branch", "h", "weight", "post_weight", "post_bias", "gate", "dbranch", "dx",
             "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate", "workspace")
    base = dict.fromkeys(names, None)
    base.update(dn=A, branch=A, h=A, weight=A, dbranch=A, dweight=A, workspace=A)
    C.bcmt_residual_norm_backward(p, *{**base, **kw}.values(), 0)


@pytest.mark.parametrize("kw,name", [
    (dict(dtype=7), "ARG"), (dict(wtype=-1), "ARG"), (dict(rms=2), "ARG"), (dict(rows=-1), "SHAPE"),
    (dict(rows=(1 << 30) + 1), "SHAPE"), (dict(D=0), "SHAPE"), (dict(D=8193), "UNSUPPORTED"),
    (dict(gates=4), "SHAPE"), (dict(gates=-1), "SHAPE"), (dict(gates=2), "ARG"), (dict(flags=1 << 30), "ARG"),
    (dict(alpha=float("nan")), "ARG"), (dict(alpha=float("inf")), "ARG"), (dict(eps=-1.0), "ARG"),
    (dict(eps=float("nan")), "ARG")])
def test_norm_parameters(C, kw, name):
    p = norm_params(C, **kw)
    for call in (norm_forward, norm_backward):
        assert code(C, call, C, p) == getattr(C, "BCMT_ERR_" + name)
    if kw != dict(gates=2):      # right with a gate
        assert C.bcmt_residual_norm_workspace_size(p, True) == 0


@pytest.mark.parametrize("kw,name", [
    (dict(branch=None), "ARG"), (dict(x=None), "ARG"), (dict(weight=None), "ARG"), (dict(h=None), "ARG"),
    (dict(n=None), "ARG"), (dict(branch=A + 8), "ALIGN"), (dict(x=A + 4), "ALIGN"), (dict(weight=A + 2), "ALIGN"),
    (dict(bias=A + 2), "ALIGN"), (dict(post_weight=A + 8), "ALIGN"), (dict(h=A + 8), "ALIGN"),
    (dict(post_bias=A), "ARG"), (dict(gate=A), "ARG")])
def test_norm_pointers(C, kw, name):
    assert code(C, lambda: norm_forward(C, norm_params(C), **kw)) == getattr(C, "BCMT_ERR_" + name)


@pytest.mark.parametrize("kw,name", [
    (dict(dn=None), "ARG"), (dict(branch=None), "ARG"), (dict(h=None), "ARG"), (dict(weight=None), "ARG"),
    (dict(dbranch=None), "ARG"), (dict(workspace=None), "ARG"), (dict(dh=A + 8), "ALIGN"),
    (dict(dx=A + 8), "ALIGN"), (dict(dweight=A + 8), "ALIGN"), (dict(workspace=A + 8), "ALIGN"),
    (dict(dpost_weight=A), "ARG"), (dict(dgate=A), "ARG"), (dict(gate=A), "ARG")])
def test_norm_gradient_pointers(C, kw, name):
    assert code(C, lambda: norm_backward(C, norm_params(C), **kw)) == getattr(C, "BCMT_ERR_" + name)


@pytest.mark.parametrize("change", [
    dict(x=torch.zeros(2, 3, 7)), dict(x=torch.zeros(2, 3, 8, dtype=torch.bfloat16)),
    dict(weight=torch.ones(7)), dict(weight=torch.ones(8, dtype=torch.float16)), dict(bias=torch.ones(8).bfloat16()),
    dict(post_weight=torch.ones(8).bfloat16()), dict(post_bias=torch.ones(8)),
    dict(gate=torch.ones(2, 1, 8).bfloat16()), dict(gate=torch.ones(3, 8)), dict(gate=torch.ones(2, 3, 1)),
    dict(gate=torch.ones(1, 3, 8)), dict(gate=torch.ones(1, 2, 3, 8)), dict(gate=torch.ones(())),
    dict(kind="batch"), dict(branch=torch.zeros(2, 3, 8, dtype=torch.float64)), dict(branch=torch.zeros(())),
    dict(residual_scale=torch.ones((), requires_grad=True))])
def test_norm_arguments(host, change):
    args = dict(branch=torch.zeros(2, 3, 8), x=torch.zeros(2, 3, 8), weight=torch.ones(8))
    args.update(change)
    for call in (host[1].residual_norm_forward, host[1].residual_norm):
        with pytest.raises(ValueError):
            call(**args)
    if "x" not in change:
        del args["x"]
        with pytest.raises(ValueError):
            host[1].residual_norm_backward(dh=None, dn=torch.zeros(2, 3, 8), h=torch.zeros(2, 3, 8), **args)


def test_norm_gates(host):
    """Which rows a gate belongs to."""
    rows = host[1]._gates
    for gate, shape, n in [((8,), (2, 3, 8), 1), ((1, 8), (2, 3, 8), 1), ((1, 1, 8), (2, 3, 8), 1),
                           ((2, 1, 8), (2, 3, 8), 2), ((2, 3, 8), (2, 3, 8), 6), ((8,), (8,), 1),
                           ((3, 8), (3, 8), 3), ((2, 3, 1, 8), (2, 3, 4, 8), 6), ((1, 1, 8), (1, 5, 8), 1),
                           ((2, 1, 8), (2, 0, 8), 2)]:
        assert rows(torch.empty(gate), torch.Size(shape)) == n, (gate, shape)


def test_tensors_on_the_host_are_refused(C):
    from paper_2608_13578_gb300 import beam, norms, optim
    x, w = torch.zeros(2, 8), torch.ones(8)
    for call in (lambda: norms.residual_norm(x, x, w), lambda: norms.residual_norm_backward(x, x, x, x, w),
                 lambda: beam.beam_select(torch.zeros(1, 2, 8), torch.zeros(1, 2)),
                 lambda: beam.beam_reorder([x], torch.zeros(1, 2, dtype=torch.int64)),
                 lambda: optim.AdamWPlan([x], [x], [x]),
                 lambda: optim.adamw8_values(x.to(torch.int8), w, x.to(torch.uint8), w)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


# ------------------------------------------------------------------------- AdamW
def adamw_params(C, **kw):
    base = dict(count=1, dtype=C.BCMT_BF16, bits=32, flags=0, step=1, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8,
                weight_decay=0.1)
    return C.bcmt_adamw_params(**{**base, **kw})


def adamw_tensor(C, **kw):
    t = (C.bcmt_adamw_tensor * 1)(C.bcmt_adamw_tensor(**{**dict(p=A, g=A, m=A, v=A, n=100), **kw}))
    return ctypes.addressof(t), t


@pytest.mark.parametrize("kw,name", [
    (dict(dtype=9), "ARG"), (dict(bits=16), "ARG"), (dict(count=-1), "ARG"), (dict(step=0), "ARG"),
    (dict(beta1=1.0), "ARG"), (dict(beta1=-0.1), "ARG"), (dict(beta2=1.0), "ARG"), (dict(beta2=float("nan")), "ARG"),
    (dict(lr=-1.0), "ARG"), (dict(lr=float("inf")), "ARG"), (dict(eps=-1.0), "ARG"),
    (dict(weight_decay=float("nan")), "ARG"), (dict(flags=1 << 20), "ARG"), (dict(step_ptr=A + 4), "ALIGN"),
    (dict(lr_ptr=A + 2), "ALIGN"), (dict(grad_scale=A + 1), "ALIGN")])
def test_adamw_parameters(C, kw, name):
    assert code(C, C.bcmt_adamw_step, adamw_params(C, **kw), adamw_tensor(C)[0], 0) == getattr(C, "BCMT_ERR_" + name)


@pytest.mark.parametrize("kw,name", [
    (dict(n=-1), "SHAPE"), (dict(n=(1 << 40) + 1), "SHAPE"), (dict(p=None), "ARG"), (dict(g=None), "ARG"),
    (dict(m=None), "ARG"), (dict(v=None), "ARG"), (dict(p=A + 1), "ALIGN"), (dict(g=A + 1), "ALIGN"),
    (dict(m=A + 2), "ALIGN"), (dict(v=A + 2), "ALIGN"), (dict(master=A + 2), "ALIGN")])
def test_adamw_tensors(C, kw, name):
    at, keep = adamw_tensor(C, **kw)
    assert code(C, C.bcmt_adamw_step, adamw_params(C), at, 0) == getattr(C, "BCMT_ERR_" + name)


def test_adamw_tables(C):
    assert code(C, C.bcmt_adamw_step, adamw_params(C), None, 0) == C.BCMT_ERR_ARG
    at, keep = adamw_tensor(C, master=A)
    assert code(C, C.bcmt_adamw_step, adamw_params(C, dtype=C.BCMT_F32), at, 0) == C.BCMT_ERR_ARG
    at, keep = adamw_tensor(C)          # no scales
    assert code(C, C.bcmt_adamw_step, adamw_params(C, bits=8), at, 0) == C.BCMT_ERR_ARG
    two = (C.bcmt_adamw_tensor * 2)(*[C.bcmt_adamw_tensor(p=A, g=A, m=A, v=A, n=4, master=w) for w in (None, A)])
    assert code(C, C.bcmt_adamw_step, adamw_params(C, count=2), ctypes.addressof(two), 0) == C.BCMT_ERR_ARG
    # an empty tensor has no say in whether there are masters
    two = (C.bcmt_adamw_tensor * 2)(C.bcmt_adamw_tensor(n=0), C.bcmt_adamw_tensor(p=A, g=A, m=A, v=A, n=4, master=A + 2))
    assert code(C, C.bcmt_adamw_step, adamw_params(C, count=2), ctypes.addressof(two), 0) == C.BCMT_ERR_ALIGN
    assert code(C, C.bcmt_adamw_values, A, A, A, A, A, A, -1, 0) == C.BCMT_ERR_SHAPE
    assert code(C, C.bcmt_adamw_values, A, A, A, A, A, None, 5, 0) == C.BCMT_ERR_ARG


def test_adamw_plan_arguments(host):
    f, i8, u8 = (lambda *s: torch.zeros(*s)), torch.int8, torch.uint8
    good = dict(params=[f(300), f(4)], m=[f(300), f(4)], v=[f(300), f(4)])
    plan = host[2].AdamWPlan
    plan(**good)
    for change in (dict(params=[f(300), f(4).bfloat16()]), dict(params=[]), dict(m=[f(300)]),
                   dict(m=[f(300), f(5)]), dict(v=[f(300), f(4).bfloat16()]), dict(masters=[f(300), f(4)]),
                   dict(m_scales=[f(2), f(1)]), dict(params=[f(300), None]),
                   dict(params=[f(20, 30).t(), f(4)], m=[f(30, 20), f(4)], v=[f(30, 20), f(4)])):
        with pytest.raises(ValueError):
            plan(**{**good, **change})
    x = f(600)
    with pytest.raises(ValueError, match="share"):
        plan(params=[x[:300], x[299:303]], m=good["m"], v=good["v"])
    with pytest.raises(ValueError, match="share"):
        plan(params=good["params"], m=good["m"], v=[good["m"][0], f(4)])
    eight = dict(params=good["params"], m=[torch.zeros(300, dtype=i8), torch.zeros(4, dtype=i8)],
                 v=[torch.zeros(300, dtype=u8), torch.zeros(4, dtype=u8)],
                 m_scales=[f(2), f(1)], v_scales=[f(2), f(1)])
    plan(**eight)
    for change in (dict(m=eight["v"]), dict(v=[f(300), f(4)]), dict(m_scales=[f(1), f(1)]),
                   dict(v_scales=[f(2), f(2)]), dict(m=[torch.zeros(301, dtype=i8), eight["m"][1]])):
        with pytest.raises(ValueError):
            plan(**{**eight, **change})


def test_adamw_step_arguments(host):
    f = torch.zeros
    p = host[2].AdamWPlan([f(30), f(4)], [f(30), f(4)], [f(30), f(4)])
    good = dict(grads=[f(30), f(4)], lr=1e-3, step=1)
    for change in (dict(grads=[f(30)]), dict(grads=[f(31), f(4)]), dict(grads=[f(30), f(4).bfloat16()]),
                   dict(grads=[f(30), f(4).to_sparse()]), dict(grad_scale=torch.zeros(2)),
                   dict(grad_scale=torch.zeros(1, dtype=torch.float64)), dict(grad_scale=0.5)):
        with pytest.raises(ValueError):
            p.step(**{**good, **change})
    with pytest.raises(ValueError):
        host[2].adamw8_values(f(4, dtype=torch.int8), f(1), f(5, dtype=torch.uint8), f(1))
    with pytest.raises(ValueError):
        host[2].adamw8_values(f(300, dtype=torch.int8), f(1), f(300, dtype=torch.uint8), f(2))


def test_optimizer_arguments(C):
    from paper_2608_13578_gb300 import optim
    w = torch.nn.Parameter(torch.zeros(3))
    with pytest.raises(ValueError, match="bits"):
        optim.AdamW([w], bits=4)
    opt = optim.AdamW([w], lr=0.1)
    opt.step()                          # no gradients: nothing to do
    for other in (copy.deepcopy(opt), pickle.loads(pickle.dumps(opt))):
        other.step()
        assert other.param_groups[0]["lr"] == 0.1
    old = torch.optim.AdamW([w], lr=0.2)
    opt.load_state_dict(old.state_dict())
    assert opt.param_groups[0]["lr"] == 0.2 and opt.param_groups[0]["bits"] == 32


# ------------------------------------------------------------------------- beams
def beam_params(C, **kw):
    base = dict(N=2, K=3, V=50, dtype=C.BCMT_F32, eos=4, flags=0, ld=50)
    return C.bcmt_beam_params(**{**base, **kw})


def beam_select(C, p, **kw):
    base = dict(logits=A, scores=A, finished=None, scores_out=A, parents=A, tokens=A, finished_out=A, workspace=A)
    C.bcmt_beam_select(p, *{**base, **kw}.values(), 0)


@pytest.mark.parametrize("kw,name", [
    (dict(dtype=3), "ARG"), (dict(N=-1), "SHAPE"), (dict(K=0), "SHAPE"), (dict(K=33), "SHAPE"), (dict(V=0), "SHAPE"),
    (dict(V=1 << 24, ld=1 << 24), "SHAPE"), (dict(N=1 << 22), "SHAPE"), (dict(eos=50), "ARG"), (dict(ld=49), "ARG"),
    (dict(N=1 << 20, K=4, V=1 << 21, ld=1 << 21), "SHAPE"), (dict(flags=1 << 9), "ARG")])
def test_beam_parameters(C, kw, name):
    p = beam_params(C, **kw)
    assert code(C, beam_select, C, p) == getattr(C, "BCMT_ERR_" + name)
    assert C.bcmt_beam_workspace_size(p) == 0


@pytest.mark.parametrize("kw,name", [
    (dict(logits=None), "ARG"), (dict(scores=None), "ARG"), (dict(scores_out=None), "ARG"), (dict(parents=None), "ARG"),
    (dict(tokens=None), "ARG"), (dict(finished_out=None), "ARG"), (dict(workspace=None), "ARG"),
    (dict(logits=A + 2), "ALIGN"), (dict(scores=A + 1), "ALIGN"), (dict(parents=A + 4), "ALIGN"),
    (dict(tokens=A + 4), "ALIGN"), (dict(workspace=A + 8), "ALIGN")])
def test_beam_pointers(C, kw, name):
    assert code(C, lambda: beam_select(C, beam_params(C), **kw)) == getattr(C, "BCMT_ERR_" + name)


def test_beam_without_an_end(C):
    assert code(C, lambda: beam_select(C, beam_params(C, eos=-1), finished=A)) == C.BCMT_ERR_ARG


def test_beam_reorder_tables(C):
    def table(*rows):
        t = (C.bcmt_beam_tensor * len(rows))(*[C.bcmt_beam_tensor(*r) for r in rows])
        return lambda N=2, K=3, parents=A: C.bcmt_beam_reorder(parents, N, K, ctypes.addressof(t), len(rows), 0, 0)
    far = A + (1 << 16)
    ok = table((A, far, 16))
    for kw in (dict(N=-1), dict(K=0), dict(K=33), dict(N=1 << 22)):
        assert code(C, lambda: ok(**kw)) == C.BCMT_ERR_SHAPE
    assert code(C, lambda: ok(parents=None)) == C.BCMT_ERR_ARG
    assert code(C, lambda: ok(parents=A + 4)) == C.BCMT_ERR_ALIGN
    for rows in ([(None, far, 16)], [(A, None, 16)], [(A, A, 16)], [(A, A + 95, 16)], [(A + 95, A, 16)],
                 # what one copy writes, another may neither read nor write
                 [(A, far, 16), (far + 1000, A + 90, 16)], [(A, far, 16), (A + 1000, far + 95, 16)],
                 [(far + 50, A, 16), (A + 1000, far + 20, 16)]):
        assert code(C, table(*rows)) == C.BCMT_ERR_ARG, rows
    assert code(C, lambda: ok(parents=far + 40)) == C.BCMT_ERR_ARG      # written by a copy
    assert code(C, table((A, far, -1))) == C.BCMT_ERR_SHAPE
    assert code(C, lambda: C.bcmt_beam_reorder(A, 2, 3, None, 1, 0, 0)) == C.BCMT_ERR_ARG
    assert code(C, lambda: C.bcmt_beam_reorder(A, 2, 3, None, -1, 0, 0)) == C.BCMT_ERR_ARG


def test_beam_arguments(host):
    b = host[0]
    x, s, f = torch.zeros(2, 3, 10), torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.bool)
    for args in ((x[0], s), (x.double(), s), (x, s.double()), (x, s[:1]), (x, s, f), (x, s, f.long(), 1), (x, s, f[:1], 1),
                 (x, s, f, 10), (x, s, f, -1), (x, s, None, 10), (x.clone().requires_grad_(), s),
                 (x, s.clone().requires_grad_())):
        with pytest.raises(ValueError):
            b.beam_select(*args)


def test_reorder_arguments(host):
    b, p = host[0], torch.zeros(2, 3, dtype=torch.int64)
    t = torch.zeros(2, 3, 4)
    for args in (([t], p.int()), ([t], p[0]), ([t], [[0, 1, 2]] * 2), ([torch.zeros(3, 2, 4)], p), ([torch.zeros(5)], p),
                 ([torch.zeros(())], p), ([t.clone().requires_grad_()], p), ([t], p, []),
                 ([t], p, [torch.zeros(2, 3, 5)]), ([t], p, [torch.zeros(2, 3, 4).bfloat16()]),
                 ([t], p, [torch.zeros(3, 2, 4).transpose(0, 1)])):
        with pytest.raises(ValueError):
            b.beam_reorder(*args)
    o = torch.zeros(4, 3, 4)
    for tensors, out in (([t], [t]), ([t, t.clone()], [t.clone(), t]), ([t, t], [o[:2], o[1:3]])):
        assert code(b.C, b.beam_reorder, tensors, p, out) == b.C.BCMT_ERR_ARG
    assert b.beam_reorder([], p) == []


def test_versions_of_what_is_written(host, monkeypatch):
    """A step moves the version counters of the tensors that it writes, not of those whose
    gradient is None."""
    optim = host[2]
    monkeypatch.setattr(optim.C.LIB, "bcmt_adamw_step", lambda *a: 0)
    f, i8, u8 = torch.zeros, torch.int8, torch.uint8
    sets = [dict(params=[f(300), f(4), f(5)], m=[f(300), f(4), f(5)], v=[f(300), f(4), f(5)]),
            dict(params=[f(n).bfloat16() for n in (300, 4)], m=[f(300, dtype=i8), f(4, dtype=i8)],
                 v=[f(300, dtype=u8), f(4, dtype=u8)], m_scales=[f(2), f(1)], v_scales=[f(2), f(1)],
                 masters=[f(300), f(4)])]
    for lists in sets:
        plan = optim.AdamWPlan(**lists)
        grads = [torch.ones_like(p) for p in lists["params"]]
        for missing in (None, 1, 0):
            given = [None if i == missing else g for i, g in enumerate(grads)]
            before = {k: [t._version for t in ts] for k, ts in lists.items()}
            plan.step(given, lr=1e-3, step=1)
            for k, ts in lists.items():
                assert [t._version - b for t, b in zip(ts, before[k])] == [int(g is not None) for g in given], k


@pytest.mark.parametrize("frozen", [(), ("x",), ("branch", "x"), ("weight", "bias", "post_weight", "post_bias"),
                                    ("gate",), ("branch", "weight", "post_bias", "gate"),
                                    ("x", "weight", "bias", "post_weight", "post_bias", "gate")], ids=str)
@pytest.mark.parametrize("plain", [False, True])
def test_gradients_that_nobody_wants(host, monkeypatch, frozen, plain):
    """A backward pass asks the library for the gradients of what requires them, and for dbranch,
    which it always gives."""
    norms = host[1]
    seen = []
    monkeypatch.setattr(norms.C.LIB, "bcmt_residual_norm_forward", lambda *a: 0)
    monkeypatch.setattr(norms.C.LIB, "bcmt_residual_norm_backward", lambda *a: seen.append(a) or 0)
    monkeypatch.setattr(norms, "_plan", lambda *a: (None, 0))
    names = ["branch", "x", "weight", "bias", "post_weight", "post_bias", "gate"]
    given = names[:4] if plain else names       # plain: dbranch and dx are one tensor
    t = {k: torch.ones(*((2, 3, 8) if k in ("branch", "x") else (8,))) for k in given}
    for k in set(given) - set(frozen):
        t[k].requires_grad_()
    h, n = norms.residual_norm(t["branch"], t["x"], t["weight"], t["bias"],
                               **{k: t[k] for k in given[4:]})
    (h.sum() + n.sum()).backward()
    (a,) = seen
    outputs = dict(zip(["branch", "x", "weight", "bias", "post_weight", "post_bias", "gate"], a[9:16]))
    for k in names:
        wanted = k in given and k not in frozen
        assert k not in given or (t[k].grad is not None) == wanted, k
        if k == "branch":
            assert outputs[k]
        elif k == "x" and plain:
            assert outputs[k] is None
        else:
            assert bool(outputs[k]) == wanted, k
