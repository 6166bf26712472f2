"""The states that linear attention returns, and its walks in segments, on the GPU.

Tolerances, fixed from the arithmetic before any run:
 * outputs and states entry by entry, relative to the largest: as in
   test_gpu_lm_ops (states of bf16 inputs take the fp32 figure alone here, since
   the keys that make them are carried in 24 bits);
 * returned states in the root mean square, relative: a chunk's sum takes about 24
   additions in the tensor cores (8 steps of 16 tokens, 3 terms), each cut at 2^-23
   at the worst and independent of the others, which is 5 * 2^-23 in all, and a
   decay weight is good to 2 * 2^-23: 2^-20 covers both.  Keys in 16 bits would
   leave 2^-18.5.
"""

import numpy as np
import pytest
import torch

from tests import lm_reference as R
from tests.test_gpu_lm_ops import F, check_rel, make, no_wait_ran_out, np64  # noqa: F401

pytestmark = pytest.mark.gpu


def figures(T, dh):
    return 4 * 2.0 ** -9, (2 * T + dh + 8) * 2.0 ** -24


# B, H, dh, T, ragged: one segment, a few that the walks join, many joined apart
CUTS = [
    (1, 2, 64, 100, False), (40, 8, 64, 300, True), (32, 5, 128, 300, False),
    (4, 8, 128, 900, False), (4, 16, 64, 1000, True), (5, 12, 128, 1700, True),
    (20, 6, 64, 2300, True), (2, 8, 64, 1600, False), (1, 1, 128, 1500, False),
]


def case(B, H, dh, T, ragged, seed):
    lengths = [(611 * b + T) % (T + 1) if b % 5 else T for b in range(B)] if ragged else None
    d, r = make(B, T, H, dh, "bf16", seed, True, lengths)
    some = sorted({0, 1 % B, B // 2, B - 1})
    return d, {k: v if k == "decay" or v is None else v[some] for k, v in r.items()}, some


@pytest.mark.parametrize("in_place", [False, True], ids=["apart", "in_place"])
@pytest.mark.parametrize("B,H,dh,T,ragged", CUTS)
def test_forward_and_its_state(F, B, H, dh, T, ragged, in_place):
    d, r, some = case(B, H, dh, T, ragged, 21)
    s0 = d["s0"].clone()
    o, S = F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], None, d["n"], s0,
                                      s0 if in_place else None)
    assert (S.data_ptr() == s0.data_ptr()) == in_place
    ro, rS = R.linear_attention(r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, r["n"], r["s0"])
    to, ts = figures(T, dh)
    check_rel("o", o[some], ro, to)
    check_rel("state", S[some], rS, ts)
    assert torch.isfinite(o).all() and torch.isfinite(S).all()
    rms = np.sqrt(((np64(S[some]) - rS) ** 2).mean() / (rS ** 2).mean())
    assert rms <= 2.0 ** -20, rms


@pytest.mark.parametrize("B,H,dh,T,ragged", CUTS)
def test_backward_and_its_state(F, B, H, dh, T, ragged):
    d, r, some = case(B, H, dh, T, ragged, 22)
    got = F.linear_attention_backward(d["do"], d["q"], d["k"], d["v"], d["decay"], None, d["n"],
                                      d["s0"], d["ds"])
    ref = R.linear_attention_grads(r["do"], r["q"], r["k"], r["v"], r["decay"], dh ** -0.5, r["n"],
                                   r["s0"], r["ds"])
    to, ts = figures(T, dh)
    for name, a, b, t in zip(("dq", "dk", "dv", "d_state"), got, ref, (to, to, to, ts)):
        check_rel(name, a[some], b, t)
        assert torch.isfinite(a).all(), name
    rms = np.sqrt(((np64(got[3][some]) - ref[3]) ** 2).mean() / (ref[3] ** 2).mean())
    assert rms <= 2.0 ** -20, rms


@pytest.mark.parametrize("B,H,dh,T,ragged", CUTS)
def test_repeats_are_the_same(F, B, H, dh, T, ragged):
    d, _, _ = case(B, H, dh, T, ragged, 23)
    def call():
        return (*F.linear_attention_forward(d["q"], d["k"], d["v"], d["decay"], None, d["n"], d["s0"]),
                *F.linear_attention_backward(d["do"], d["q"], d["k"], d["v"], d["decay"], None,
                                             d["n"], d["s0"], d["ds"]))
    first = call()
    for _ in range(3):
        for a, b in zip(first, call()):
            assert torch.equal(a, b)
