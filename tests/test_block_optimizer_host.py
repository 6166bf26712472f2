"""Host side of the library's AdamW (CPU only): the options of its groups, files of other
optimizers, counts of steps.  Plans are replaced by ones that record their calls."""

import copy

import pytest
import torch

from paper_2608_13578_gb300 import optim

BF, F = torch.bfloat16, torch.float32


@pytest.fixture
def calls(monkeypatch):
    """(params, their lists of states by name, what a step was called with) of every step."""
    got = []

    class Plan:
        def __init__(self, params, m, v, **lists):
            self.params, self.lists = params, dict(m=m, v=v, **lists)

        def step(self, grads, **how):
            got.append((self.params, self.lists, {**how, "grads": grads, "step": how["step"]}))
    monkeypatch.setattr(optim, "AdamWPlan", Plan)
    return got


def params(*shapes, dtype=F, seed=0):
    g = torch.Generator().manual_seed(seed)
    ps = [torch.nn.Parameter(torch.randn(s, generator=g).to(dtype)) for s in shapes]
    for p in ps:
        p.grad = torch.randn(p.shape, generator=g).to(dtype)
    return ps


# ------------------------------------------------------------- options of a group
IGNORED = [dict(maximize=True), dict(amsgrad=True), dict(differentiable=True),
           dict(decoupled_weight_decay=False, weight_decay=0.1), dict(bits=16)]


@pytest.mark.parametrize("option", IGNORED, ids=lambda o: next(iter(o)))
def test_options_that_would_be_ignored(calls, option):
    """A group with an option of torch's that changes the step, and that this one has not,
    is refused wherever it comes from, and nothing is changed by it."""
    name = next(iter(option))
    p, q = params(3, 4)
    with pytest.raises(ValueError, match=name):
        optim.AdamW([dict(params=[p], **option)])
    opt = optim.AdamW([p], lr=0.5)
    with pytest.raises(ValueError, match=name):
        opt.add_param_group(dict(params=[q], **option))
    assert len(opt.param_groups) == 1
    file = opt.state_dict()
    file["param_groups"][0].update(option, lr=0.1)
    with pytest.raises(ValueError, match=name):
        opt.load_state_dict(file)
    assert opt.param_groups[0]["lr"] == 0.5
    opt.param_groups[0].update(option)
    with pytest.raises(ValueError, match=name):
        opt.step()
    assert not calls


@pytest.mark.parametrize("option", [dict(maximize=True), dict(amsgrad=True)], ids=lambda o: next(iter(o)))
def test_a_file_of_torch_with_such_an_option(calls, option):
    (p,) = params(3)
    old = torch.optim.AdamW([p], **option)
    old.step()
    opt = optim.AdamW([p])
    with pytest.raises(ValueError, match=next(iter(option))):
        opt.load_state_dict(old.state_dict())
    assert not opt.state


def test_options_that_are_only_hints(calls):
    """foreach, fused and the switches that are off are taken as they are."""
    (p,) = params(3)
    old = torch.optim.AdamW([p], foreach=True)
    old.step()
    opt = optim.AdamW([dict(params=[p], maximize=False, amsgrad=False, fused=True)])
    opt.load_state_dict(old.state_dict())
    opt.step()
    assert len(calls) == 1 and calls[0][2]["step"] == 2


# ------------------------------------------------------ files of torch's optimizer
def torch_file(ps, steps=3, **kw):
    """The states of torch's AdamW after some steps over ps, which it moves."""
    old = torch.optim.AdamW(ps, **kw)
    for _ in range(steps):
        old.step()
    return copy.deepcopy(old.state_dict())


def test_a_file_of_torch_leaves_what_it_does_not_know(calls):
    """bits, masters and capturable of each group stay as they were made: torch's files do not
    have the first two, and their capturable=False would freeze the count of a captured step."""
    p, q = params((4, 5), 7)
    opt = optim.AdamW([dict(params=[p], capturable=True), dict(params=[q], masters=True)], lr=0.5)
    opt.load_state_dict(torch_file([dict(params=[p]), dict(params=[q])], lr=0.25))
    first, second = opt.param_groups
    assert (first["bits"], first["masters"], first["capturable"], first["lr"]) == (32, False, True, 0.25)
    assert (second["bits"], second["masters"], second["capturable"]) == (32, True, False)
    assert isinstance(opt.state[p]["step"], torch.Tensor) and opt.state[q]["step"] == 3
    opt.step()
    assert [int(c[2]["step"]) for c in calls] == [4, 4]
    # a file of this class says what its groups are
    other = optim.AdamW([dict(params=[p]), dict(params=[q])])
    other.load_state_dict(opt.state_dict())
    assert [g["capturable"] for g in other.param_groups] == [True, False]
    assert [g["masters"] for g in other.param_groups] == [False, True]


def test_files_of_another_length(calls):
    p, q = params(3, 4)
    opt = optim.AdamW([p])
    with pytest.raises(ValueError, match="group"):
        opt.load_state_dict(torch_file([dict(params=[p]), dict(params=[q])]))


def test_files_without_the_states_are_refused(calls):
    """States of another kind than the group's are refused by name, before anything changes."""
    p, q = params((4, 5), 7)
    file = torch_file([p, q], lr=0.25)
    opt = optim.AdamW([p, q], lr=0.5, bits=8)
    with pytest.raises(ValueError, match="exp_avg_scale.*8 bits"):
        opt.load_state_dict(file)
    with pytest.raises(ValueError, match="exp_avg"):
        optim.AdamW([p, q]).load_state_dict(copy.deepcopy(torch.optim.SGD([p, q], lr=1.0, momentum=0.9).state_dict())
                                            | {"state": {0: dict(momentum_buffer=torch.zeros(4, 5))}})
    assert not opt.state and opt.param_groups[0]["lr"] == 0.5
    # one parameter of several, and codes where the group wants floats
    opt = optim.AdamW([p, q])
    opt.step()
    for name in ("exp_avg", "exp_avg_sq", "step"):
        file = opt.state_dict()
        file["state"][1] = {k: x for k, x in file["state"][1].items() if k != name}
        with pytest.raises(ValueError, match=name):
            optim.AdamW([p, q]).load_state_dict(file)
    eight = optim.AdamW([p, q], bits=8)
    eight.step()
    file = eight.state_dict()
    file["param_groups"][0]["bits"] = 32
    with pytest.raises(ValueError, match="32 bits"):
        optim.AdamW([p, q]).load_state_dict(file)
    file = opt.state_dict()
    file["param_groups"][0]["bits"] = 8
    for s in file["state"].values():
        s["exp_avg_scale"] = s["exp_avg_sq_scale"] = torch.zeros(1)
    with pytest.raises(ValueError, match="8 bits"):
        optim.AdamW([p, q]).load_state_dict(file)


def test_a_parameter_that_the_file_has_no_states_of(calls):
    p, q = params(3, 4)
    grad, q.grad = q.grad, None
    file = torch_file([p, q])
    opt = optim.AdamW([p, q])
    opt.load_state_dict(file)
    q.grad = grad
    opt.step()
    assert [c[2]["step"] for c in calls] == [1, 4]


def test_masters_of_a_file_that_has_none(calls):
    """Every bf16 parameter of a group with masters gets one, whether the file has its states
    or not and whichever comes first."""
    for without in (0, 1, None):
        p, q = params((4, 5), 7, dtype=BF)
        if without is not None:
            kept = (p, q)[without].grad
            (p, q)[without].grad = None
        file = torch_file([p, q])
        if without is not None:
            (p, q)[without].grad = kept
        calls.clear()
        opt = optim.AdamW([p, q], masters=True)
        opt.load_state_dict(file)
        opt.step()
        seen = {id(x) for c in calls for x in c[1]["masters"]}
        assert seen == {id(opt.state[x]["master"]) for x in (p, q)}
        for x in (p, q):
            assert torch.equal(opt.state[x]["master"], x.detach().float()) and opt.state[x]["master"].dtype == F
        # they are kept from then on
        for x in (p, q):
            opt.state[x]["master"].add_(1.0)
        before = [opt.state[x]["master"] for x in (p, q)]
        opt.step()
        assert all(opt.state[x]["master"] is m for x, m in zip((p, q), before))
        again = optim.AdamW([p, q], masters=True)
        again.load_state_dict(opt.state_dict())
        again.step()
        assert all(torch.equal(again.state[x]["master"], m) for x, m in zip((p, q), before))


def test_no_masters_where_none_are_kept(calls):
    p, q = params(3, 4)
    r, s = params(3, 4, dtype=BF)
    opt = optim.AdamW([dict(params=[p, q], masters=True), dict(params=[r, s])])
    opt.step()
    assert [c[1].get("masters") for c in calls] == [None, None]


@pytest.mark.parametrize("masters", [False, True])
def test_moments_of_another_width(calls, masters):
    """Torch keeps the moments of bf16 parameters in bf16; here they go on in float32."""
    p, q = params((4, 5), 7, dtype=BF)
    file = torch_file([p, q])
    opt = optim.AdamW([p, q], masters=masters)
    opt.load_state_dict(file)
    for i, x in enumerate((p, q)):
        for name in ("exp_avg", "exp_avg_sq"):
            assert file["state"][i][name].dtype == BF and opt.state[x][name].dtype == F
            assert torch.equal(opt.state[x][name], file["state"][i][name].float())
    opt.step()
    assert calls[-1][2]["step"] == 4
    eight = optim.AdamW([p, q], bits=8)
    eight.step()
    again = optim.AdamW([p, q], bits=8)
    again.load_state_dict(eight.state_dict())
    assert {k: x.dtype for k, x in again.state[p].items() if k != "step"} == optim._states(8)


# --------------------------------------------------------- counts on the device
def two_devices():
    """Parameters on two devices (the second without memory, which is enough for a count)."""
    p, q = params(3, 4)
    r = torch.nn.Parameter(torch.zeros(5, device="meta"))
    r.grad = torch.zeros(5, device="meta")
    return [p, r, q]


def raised(count, before):
    return count._version - before


def test_a_count_for_each_device(calls):
    """A capturable group over two devices has a count on each, and every step raises both,
    from the start and after loading."""
    ps = two_devices()
    opt = optim.AdamW(ps, capturable=True)
    opt.step()
    for which in range(2):
        counts = [opt.state[p]["step"] for p in ps]
        assert [c.device.type for c in counts] == ["cpu", "meta", "cpu"]
        assert counts[0] is counts[2]
        for c in calls:
            assert c[2]["step"].device == c[0][0].device
        before = [c._version for c in counts]
        opt.step()
        assert [raised(c, b) for c, b in zip(counts, before)] == [1, 1, 1]
        assert int(counts[0]) == 2 + 3 * which
        if which == 0:
            opt.step()
            file = {"state": {i: {k: (x.new_zeros(x.shape, device="cpu") if k != "step" else 3)
                                  for k, x in opt.state[p].items()} for i, p in enumerate(ps)},
                    "param_groups": opt.state_dict()["param_groups"]}
            opt = optim.AdamW(ps, capturable=True)
            opt.load_state_dict(file)
            opt.step()
            calls.clear()


def test_counts_of_a_file_that_differ(calls):
    """Parameters that are behind in a file stay behind on the device."""
    p, q, r = params(3, 4, 5)
    late, q.grad = q.grad, None
    old = torch.optim.AdamW([p, q, r])
    old.step()
    old.step()
    q.grad = late
    old.step()
    opt = optim.AdamW([p, q, r], capturable=True)
    opt.load_state_dict(old.state_dict())
    assert [int(opt.state[x]["step"]) for x in (p, q, r)] == [3, 1, 3]
    opt.step()
    opt.step()
    assert [int(opt.state[x]["step"]) for x in (p, q, r)] == [5, 3, 5]
    assert opt.state[p]["step"] is opt.state[r]["step"]
    assert sorted((len(c[0]), int(c[2]["step"])) for c in calls[-2:]) == [(1, 3), (2, 5)]


def test_one_count_for_types(calls):
    """Types of one group share the count, which a step raises once."""
    ps = params(3, 4) + params(5, dtype=BF)
    opt = optim.AdamW(ps, capturable=True)
    for n in (1, 2):
        opt.step()
        assert len({id(opt.state[p]["step"]) for p in ps}) == 1 and int(opt.state[ps[0]]["step"]) == n
    assert len(calls) == 4


# ------------------------------------------------------------- what a capture holds
def test_steps_that_a_capture_would_freeze(calls, monkeypatch):
    """Under capture a count on the host, and states or masters that begin there (and would
    begin anew at each replay), are refused; a capturable step after a first one is not."""
    capturing = [False]
    monkeypatch.setattr(optim, "_capturing", lambda p: capturing[0])
    p, q = params(3, 4, dtype=BF)
    opt = optim.AdamW([p])
    opt.step()
    capturing[0] = True
    with pytest.raises(RuntimeError, match="capturable"):
        opt.step()
    assert opt.state[p]["step"] == 1
    opt = optim.AdamW([p, q], capturable=True, masters=True)
    with pytest.raises(RuntimeError, match="before the capture"):
        opt.step()
    late, q.grad = q.grad, None
    capturing[0] = False
    opt.step()
    capturing[0] = True
    opt.step()
    assert int(opt.state[p]["step"]) == 2
    q.grad = late
    with pytest.raises(RuntimeError, match="before the capture"):
        opt.step()
    assert int(opt.state[p]["step"]) == 2 and not opt.state.get(q)
    del opt.state[p]["master"]
    q.grad = None
    with pytest.raises(RuntimeError, match="before the capture"):
        opt.step()


# ----------------------------------------------------------------- refused steps
@pytest.mark.parametrize("capturable", [False, True])
def test_a_refused_step_does_not_count(calls, monkeypatch, capturable):
    p, q, r = params(3, 4) + params(5, dtype=BF)
    late, q.grad = q.grad, None
    opt = optim.AdamW([p, q, r], capturable=capturable)
    opt.step()
    q.grad = late
    opt.step()          # q is a step behind where the count is on the host

    def counts():
        return [int(opt.state[x]["step"]) for x in (p, q, r)]
    before = counts()
    assert before == ([2, 2, 2] if capturable else [2, 1, 2])
    plan = type(next(iter(opt._plans.values()))[1])

    def refuse(self, grads, **how):
        raise ValueError("refused")
    with monkeypatch.context() as m:
        m.setattr(plan, "step", refuse)
        with pytest.raises(ValueError, match="refused"):
            opt.step()
    assert counts() == before
    opt.step()
    assert counts() == [n + 1 for n in before]
    # what was stepped before the refusal counts: p and q, but not r, where counts are apart
    with monkeypatch.context() as m:
        step = plan.step
        m.setattr(plan, "step", lambda self, grads, **how: (
            refuse if self.params[0].dtype == BF else step)(self, grads, **how))
        with pytest.raises(ValueError, match="refused"):
            opt.step()
    assert counts() == ([4, 4, 4] if capturable else [4, 3, 3])


def test_a_group_that_becomes_capturable(calls, monkeypatch):
    """capturable set in a group that has been stepped: the counts move to the device, or back, and
    go on; not within a capture."""
    p, q, r = params(3, 4) + params(5, dtype=BF)
    late, q.grad = q.grad, None
    opt = optim.AdamW([p, q, r])
    opt.step()
    q.grad = late
    opt.step()
    opt.param_groups[0]["capturable"] = True
    with monkeypatch.context() as m:
        m.setattr(optim, "_capturing", lambda p: True)
        with pytest.raises(RuntimeError, match="before the capture"):
            opt.step()
    for n in (3, 4):
        opt.step()
        assert [int(opt.state[x]["step"]) for x in (p, q, r)] == [n, n - 1, n]
        assert opt.state[p]["step"] is opt.state[r]["step"] is not opt.state[q]["step"]
        assert all(isinstance(c[2]["step"], torch.Tensor) for c in calls[-3:])
    opt.param_groups[0]["capturable"] = False
    for n in (5, 6):
        opt.step()
        assert [opt.state[x]["step"] for x in (p, q, r)] == [n, n - 1, n]
        assert sorted(c[2]["step"] for c in calls[-3:]) == [n - 1, n, n]
