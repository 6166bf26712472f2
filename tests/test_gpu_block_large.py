"""The norms around a block, AdamW and beam search over more elements than 32 bits count: rows and
elements at the start, around 2^31 and at the end against small calls or the float64 forms."""

import pytest
import torch

from tests import block_reference as R
from tests import test_gpu_norms as T

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
FAR = 1 << 31


@pytest.fixture(autouse=True)
def memory(cuda_ok):
    if torch.cuda.get_device_properties(0).total_memory < 100 << 30:
        pytest.skip("needs 60 GB of device memory")
    yield
    torch.cuda.empty_cache()


def filled(*shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=BF, device="cuda").normal_(generator=g)


def places(rows, D):
    at = FAR // D
    return [slice(0, 3), slice(at - 2, at + 3), slice(rows - 3, rows)]


@pytest.mark.parametrize("every", [False, True], ids=["gate", "gate-a-row"])
@pytest.mark.parametrize("D", [1032, 1025])
def test_norms(D, every):
    from paper_2608_13578_gb300 import norms
    rows = FAR // D + 1003
    t, _, _ = T.make((3, D), BF, F, "layer", True, (D,))
    t["branch"], t["x"] = filled(rows, D, seed=1), filled(rows, D, seed=2)
    if every:
        t["gate"] = filled(rows, D, seed=3)
    h, n = T.forward(norms, t, 0.9, "layer")
    dh, dn = t["x"], filled(rows, D, seed=4)     # (any values do for a gradient)
    got = norms.residual_norm_backward(dh, dn, t["branch"], h, t["weight"], t["bias"], post_weight=t["post_weight"],
                                       post_bias=t["post_bias"], gate=t["gate"], residual_scale=0.9)
    got = dict(zip(R.NAMES, got))
    for s in places(rows, D):
        gate = t["gate"][s] if every else t["gate"]
        kw = dict(post_weight=t["post_weight"], post_bias=t["post_bias"], gate=gate, kind="layer", alpha=0.9)
        (rh, rn), (bh, bn) = R.norm_forward(t["branch"][s], t["x"][s], t["weight"], t["bias"], **kw)
        T.close(h[s], rh, bh, T.ROUNDINGS, "h")
        T.close(n[s], rn, bn, T.ROUNDINGS, "n")
        ref, bound = R.norm_backward(dh[s], dn[s], t["branch"][s], h[s], t["weight"], t["bias"], **kw)
        for k in ("dbranch", "dx") + (("dgate",) if every else ()):
            T.close(got[k][s], ref[k], bound[k], T.ROUNDINGS + T.COLUMNS, k)
    for k in ("dweight", "dbias", "dpost_weight", "dpost_bias"):
        assert bool(torch.isfinite(got[k]).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    from paper_2608_13578_gb300 import optim
    n, cut = FAR + 8192 + 1000, FAR - 8192      # cut: a multiple of what a CTA takes
    lists = dict(params=[filled(n, seed=1)])
    if bits == 8:
        g = torch.Generator(device="cuda").manual_seed(2)
        blocks = -(-n // 256)
        lists.update(m=[torch.randint(-127, 128, (n,), dtype=torch.int8, device="cuda", generator=g)],
                     v=[torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda", generator=g)],
                     m_scales=[torch.rand(blocks, device="cuda", generator=g) * 1e-6],
                     v_scales=[torch.rand(blocks, device="cuda", generator=g) * 1e-7])
    else:
        lists.update(m=[filled(n, seed=2).float()], v=[filled(n, seed=3).float().square_()])

    def part(x, s):
        return x[s // 256:] if x.numel() < n else x[s:]
    ends = {k: [part(ts[0], cut).clone()] for k, ts in lists.items()}
    starts = {k: [(ts[0][:32] if ts[0].numel() < n else ts[0][:8192]).clone()] for k, ts in lists.items()}
    g = filled(n, seed=4)
    how = dict(lr=1e-2, betas=(0.9, 0.99), weight_decay=0.1, step=3)
    optim.AdamWPlan(**lists).step([g], **how)
    optim.AdamWPlan(**ends).step([g[cut:].clone()], **how)
    optim.AdamWPlan(**starts).step([g[:8192].clone()], **how)
    for k in lists:
        assert torch.equal(part(lists[k][0], cut), ends[k][0]), k
        assert torch.equal(lists[k][0][:starts[k][0].numel()], starts[k][0]), k
    if bits == 8:
        del g
        a = [lists[k][0] for k in ("m", "m_scales", "v", "v_scales")]
        far = optim.adamw8_values(*a)
        near = optim.adamw8_values(*[part(x, cut).clone() for x in a])
        assert all(torch.equal(x[cut:], y) for x, y in zip(far, near))


@pytest.mark.parametrize("vocab", [5003, 4096])
def test_beam_selection(vocab):
    """Rows 2^23 elements apart."""
    from paper_2608_13578_gb300 import beam
    N, K, ld = 35, 8, 1 << 23
    x = torch.empty(N * K * ld, dtype=BF, device="cuda").view(N, K, ld)[:, :, :vocab]
    x.copy_(filled(N, K, vocab, seed=1) * 3)
    s = -torch.rand(N, K, device="cuda")
    for a, b in zip(beam.beam_select(x, s), beam.beam_select(x.contiguous(), s)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("size", [FAR + 48, FAR + 5])
def test_reordering(size):
    from paper_2608_13578_gb300 import beam
    t = torch.empty(1, 3, size, dtype=torch.uint8, device="cuda").random_(0, 256)
    parents = torch.tensor([[2, 0, 2]], device="cuda")
    (o,) = beam.beam_reorder([t], parents)
    assert all(torch.equal(o[0, k], t[0, p]) for k, p in enumerate((2, 0, 2)))
