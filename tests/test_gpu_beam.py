"""A step of beam search against its float64 form: the same beams and tokens, ties and
masks, ended beams, strides, streams and graphs; reordering byte for byte.

Scores: the terms of a row's sum that are not among the selected are fp32 exponentials (off
by 2^-22, and 2 * 2^-24 by their arguments) and 21 additions, so that the logarithm is off by
at most 27 * 2^-24; the rest is held in 64 bits, and the score is rounded once.  Beams are
compared where candidates that differ do so by more than two such errors."""

import pytest
import torch

from tests import block_reference as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
ERROR = 27 * 2.0 ** -24


@pytest.fixture(scope="module")
def B(cuda_ok):
    from paper_2608_13578_gb300 import beam
    return beam


def make(N, K, V, dtype=F, seed=0, masked=0.0, std=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(N, K, V, generator=g) * std).to(dtype)
    if masked:
        x[torch.rand(N, K, V, generator=g) < masked] = -float("inf")
    s = -torch.rand(N, K, generator=g) * 5
    return x.cuda(), s.cuda(), (torch.rand(N, K, generator=g) < 0.3).cuda()


def check(B, logits, scores, finished=None, eos=None, **kw):
    got = B.beam_select(logits, scores, finished, eos, **kw)
    ref, parents, tokens, ended, gap = R.beam_select(logits, scores, finished, eos)
    assert gap > 2 * ERROR, "candidates too near to one another for a test"
    assert torch.equal(got[1].cpu(), torch.from_numpy(parents))
    assert torch.equal(got[2].cpu(), torch.from_numpy(tokens))
    assert torch.equal(got[3].cpu(), torch.from_numpy(ended))
    ref = torch.from_numpy(ref)
    s = got[0].double().cpu()
    inf = torch.isinf(ref)
    assert torch.equal(torch.isinf(s) & (s < 0), inf)
    tol = 2.0 ** -24 * ref.abs() + ERROR
    assert bool(((s - ref).abs()[~inf] <= tol[~inf]).all())
    return got


SIZES = [(1, 1, 1), (1, 1, 7), (2, 3, 1), (1, 4, 8), (3, 5, 97), (2, 32, 40), (1, 2, 2047), (1, 3, 2048),
         (2, 2, 2049), (1, 4, 4097), (5, 8, 1000), (1, 32, 9000), (2, 4, 32000), (3, 5, 50257), (40, 8, 8200),
         (1, 1, 131072), (300, 2, 300)]


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(B, size, dtype):
    x, s, done = make(*size, dtype, seed=SIZES.index(size))
    if dtype == BF:      # equal logits are equal candidates of a beam
        x = x + 0
    check(B, x, s)
    check(B, x, s, done, size[2] // 2)


@pytest.mark.parametrize("masked", [0.5, 0.97, 0.9999, 1.0])
@pytest.mark.parametrize("size", [(4, 3, 50), (2, 8, 3000), (2, 32, 5001)], ids=str)
def test_masks(B, size, masked):
    """Few or no tokens left: places of -inf fill the beams in order."""
    x, s, done = make(*size, seed=3, masked=masked)
    check(B, x, s)
    check(B, x, s, done, 1)
    x[0] = -float("inf")
    check(B, x, s)
    s[0] = -float("inf")
    s[1, 1:] = -float("inf")
    check(B, x, s, done, 1)


@pytest.mark.parametrize("K", [1, 3, 8, 32])
@pytest.mark.parametrize("V", [5, 300, 2048, 20000])
def test_ties(B, K, V):
    """Rows of one value, of two, and equal beams: the lowest places win."""
    x = torch.zeros(2, K, V, device="cuda")
    s = torch.zeros(2, K, device="cuda")
    check(B, x, s)
    x[:, :, V // 2:] = 1.0
    check(B, x, s)
    x[1, :, V // 3] = 2.0
    check(B, x, s)
    x[:, :, V - 1] = 1.5
    x[:, :, 0] = 1.5
    check(B, x, s)
    x[0] = torch.tensor([0.0, -0.0], device="cuda").repeat(V)[:V]
    check(B, x, s)


def test_sums_of_every_size(B):
    """Logits far apart, nearly one token, and offsets that fp32 holds exactly."""
    x, s, _ = make(6, 4, 5000, seed=9)
    x[0] *= 20
    x[1] *= 0.01
    x[2, :, 17] += 200
    x[3] += 4096
    x[4] -= 30000
    x[5, :, :2500] -= 1e30
    check(B, x, s)


def test_scores_that_fp32_could_not_tell_apart(B):
    """Two beams whose best candidates differ by 2^-26 of their size: the better wins."""
    x = torch.full((1, 2, 64), -30.0, device="cuda")
    x[0, 0, 5] = x[0, 1, 9] = 10.0
    x[0, 1, 20] = -8.5        # takes exp(-18.5) = 9.2e-9 from its row's best
    s = torch.full((1, 2), -1.0, device="cuda")
    got = B.beam_select(x, s)
    assert got[1].tolist() == [[0, 1]] and got[2].tolist() == [[5, 9]]
    assert float(got[0][0, 0]) == float(got[0][0, 1])
    got = B.beam_select(x.flip(1).contiguous(), s)
    assert got[1].tolist() == [[1, 0]] and got[2].tolist() == [[5, 9]]


def test_strides_and_offsets(B):
    """The last token of each sequence's logits is read in place; other layouts are copied."""
    x, s, done = make(6, 4, 1000, seed=2)
    big = torch.full((6, 4, 3, 1000), float("nan"), device="cuda")
    big[:, :, 1] = x
    want = B.beam_select(x, s, done, 3)
    for view in (big[:, :, 1], x.transpose(0, 1).contiguous().transpose(0, 1),
                 torch.cat([x, x], 2)[:, :, :1000], x[:, :1].expand(6, 4, 1000)):
        ref = want if view.stride(1) else B.beam_select(view.contiguous(), s, done, 3)
        assert all(torch.equal(a, b) for a, b in zip(B.beam_select(view, s, done, 3), ref))
    odd = torch.empty(6 * 4 * 1000 + 1, device="cuda")[1:].view(6, 4, 1000).copy_(x)
    assert all(torch.equal(a, b) for a, b in zip(B.beam_select(odd, s.t().contiguous().t(), done, 3), want))


def test_results_over_the_inputs(B):
    """The C call may write the scores and the flags over those that it reads."""
    from paper_2608_13578_gb300 import bcmt as C
    for K in (1, 7, 32):
        x, s, done = make(9, K, 700, seed=K)
        want = B.beam_select(x, s, done, 11)
        p = C.bcmt_beam_params(9, K, 700, C.BCMT_F32, 11, 0, 700)
        ws = torch.empty(C.bcmt_beam_workspace_size(p), dtype=torch.uint8, device="cuda")
        parents, tokens = (torch.empty(9, K, dtype=torch.int64, device="cuda") for _ in range(2))
        C.bcmt_beam_select(p, x, s, done, s, parents, tokens, done, ws,
                           torch.cuda.current_stream().cuda_stream)
        assert all(torch.equal(a, b) for a, b in zip((s, parents, tokens, done), want))


@pytest.mark.parametrize("what", ["logit_nan", "logit_inf", "score_nan", "score_inf"])
def test_what_is_not_a_number_is_reported(B, what):
    from paper_2608_13578_gb300 import bcmt as C
    C.bcmt_device_status()
    x, s, _ = make(2, 3, 3000, seed=4)
    good = x.clone(), s.clone()
    where, value = what.split("_")
    (x[1, 1] if where == "logit" else s[1])[1 if where == "score" else 2500] = float(value)
    got = B.beam_select(x, s)
    with pytest.raises(C.BCMTError):
        C.bcmt_device_status()
    # that beam is not there; the other searches are as they were
    good[1][1, 1] = -float("inf")
    want = B.beam_select(*good)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    C.bcmt_device_status()
    # what is not read is not reported: rows of ended beams
    done = torch.zeros(2, 3, dtype=torch.bool, device="cuda")
    done[1, 1] = True
    if where == "logit":
        B.beam_select(x, s, done, 0)
        C.bcmt_device_status()


def test_repeatable_on_streams_and_in_graphs(B):
    x, s, done = make(8, 8, 20000, BF, seed=5)
    states = [torch.randn(8, 8, 3, 50, device="cuda") for _ in range(3)]

    def call():
        out = B.beam_select(x, s, done, 5)
        return [*out, *B.beam_reorder(states, out[1])]
    want, got, graphs = call(), [], []
    torch.cuda.synchronize()
    for _ in range(4):
        with torch.cuda.stream(torch.cuda.Stream()):
            got.append(call())
    torch.cuda.synchronize()
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


# ---------------------------------------------------------------------- reordering
@pytest.mark.parametrize("N,K", [(1, 1), (1, 4), (3, 5), (17, 32), (700, 2)])
def test_reorder(B, N, K):
    g = torch.Generator().manual_seed(N)
    parents = torch.randint(0, K, (N, K), generator=g).cuda()
    shapes = [((N, K), torch.int64), ((N * K, 3), torch.uint8), ((N, K, 5), BF), ((N * K, 2, 4100), F),
              ((N, K, 4096), torch.int8), ((N, K, 0), F), ((N, K, 7), torch.bool), ((N * K, 16), torch.float64)]
    tensors = [torch.randint(0, 2 if dt == torch.bool else 100, sh, generator=g).to(dt).cuda()
               for sh, dt in shapes]
    want = [t.view(N, K, -1)[torch.arange(N, device="cuda")[:, None], parents].view(t.shape)
            if t.numel() else t for t in tensors]
    got = B.beam_reorder(tensors, parents)
    out = [torch.empty_like(t) for t in tensors]
    v = [t._version for t in out]
    assert all(a is b for a, b in zip(B.beam_reorder(tensors, parents, out=out), out))
    for a, b, c in zip(got, out, want):
        assert torch.equal(a, c) and torch.equal(b, c) and a.dtype == c.dtype
    assert all(t._version > x for t, x in zip(out, v))
    # views off the 16-byte grid, and strided ones
    if N * K > 1:
        flat = torch.arange(N * K * 9 + 1, device="cuda", dtype=torch.int16)[1:].view(N, K, 9)
        a, b = B.beam_reorder([flat, flat.transpose(0, 1).contiguous().transpose(0, 1)], parents)
        want = flat[torch.arange(N, device="cuda")[:, None], parents]
        assert torch.equal(a, want) and torch.equal(b, want)


def test_no_searches(B):
    out = B.beam_select(torch.zeros(0, 3, 10, device="cuda"), torch.zeros(0, 3, device="cuda"))
    assert all(t.shape == (0, 3) for t in out)
    a, = B.beam_reorder([torch.zeros(0, 3, 4, device="cuda")], out[1])
    assert a.shape == (0, 3, 4)


def test_reorder_many(B):
    parents = torch.tensor([[1, 1, 0]], device="cuda")
    tensors = [torch.arange(3 * (1 + i % 5), device="cuda").view(1, 3, -1) + i for i in range(300)]
    for t, o in zip(tensors, B.beam_reorder(tensors, parents)):
        assert torch.equal(o, t[:, [1, 1, 0]])


def test_reorder_reports_bad_parents(B):
    from paper_2608_13578_gb300 import bcmt as C
    C.bcmt_device_status()
    t = torch.ones(2, 3, 10, device="cuda")
    o, = B.beam_reorder([t], torch.tensor([[0, 1, 3], [-1, 2, 2 ** 40]], device="cuda"))
    assert o.sum(-1).tolist() == [[10, 10, 0], [0, 10, 0]]
    with pytest.raises(C.BCMTError):
        C.bcmt_device_status()
    C.bcmt_device_status()
