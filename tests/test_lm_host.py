"""Host side of the language-model operators (CPU only, no kernel runs): the
reference's generator against its published vectors, the gradient formulas of
linear attention against differences, and the refusals of the C entry points
and of the torch-facing functions."""

import numpy as np
import pytest
import torch

from tests import lm_reference as R

A = 1 << 20   # an aligned address that is never dereferenced: validation fails first


@pytest.fixture(scope="module")
def C():
    from paper_2608_13578_gb300 import build
    build.build()
    from paper_2608_13578_gb300 import bcmt
    return bcmt


def test_philox_known_answers():
    # the vectors published with the generator (Random123, kat_vectors)
    ones = 0xFFFFFFFF
    got = R.philox4x32(np.zeros((1, 4), dtype=np.uint64), (0, 0))[0]
    assert [hex(int(x)) for x in got] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    got = R.philox4x32(np.full((1, 4), ones, dtype=np.uint64), (ones, ones))[0]
    assert [hex(int(x)) for x in got] == ["0x408f276d", "0x41c83b0e", "0xa20bc7c6", "0x6d5451fd"]


@pytest.mark.parametrize("lengths", [None, [5, 0]])
def test_reference_gradients_against_differences(lengths):
    # o is linear in each input on its own, so central differences are exact
    rng = np.random.default_rng(1)
    B, T, H, d = 2, 7, 2, 8
    q, k, v, do = (rng.standard_normal((B, T, H, d)) for _ in range(4))
    s, ds = (rng.standard_normal((B, H, d, d)) for _ in range(2))
    decay = np.array([0.9, 0.0])
    n = None if lengths is None else np.array(lengths)

    def f(q, k, v, s):
        o, S = R.linear_attention(q, k, v, decay, 0.3, n, s)
        return (o * do).sum() + (S * ds).sum()
    grads = R.linear_attention_grads(do, q, k, v, decay, 0.3, n, s, ds)
    args = [q, k, v, s]
    for i, g in enumerate(grads):
        e = rng.standard_normal(args[i].shape)
        hi, lo = list(args), list(args)
        hi[i], lo[i] = args[i] + e, args[i] - e
        assert (f(*hi) - f(*lo)) / 2 == pytest.approx((g * e).sum(), rel=1e-10, abs=1e-10)


@pytest.mark.parametrize("field,value,code", [
    ("B", 0, "BCMT_ERR_SHAPE"), ("T", 0, "BCMT_ERR_SHAPE"), ("H", 0, "BCMT_ERR_SHAPE"),
    ("dh", 0, "BCMT_ERR_SHAPE"), ("dh", 12, "BCMT_ERR_SHAPE"), ("dh", 136, "BCMT_ERR_SHAPE"),
    ("T", 1 << 30, "BCMT_ERR_SHAPE"), ("H", 1 << 24, "BCMT_ERR_SHAPE"),
    ("dtype", 5, "BCMT_ERR_ARG"), ("flags", 1, "BCMT_ERR_ARG"),
    ("scale", 0.0, "BCMT_ERR_ARG"), ("scale", float("nan"), "BCMT_ERR_ARG"),
    ("scale", float("inf"), "BCMT_ERR_ARG"),
])
def test_linattn_refuses_bad_params(C, field, value, code):
    p = C.bcmt_linattn_params(2, 5, 2, 16, C.BCMT_BF16, 0, 0.25)
    assert C.bcmt_linattn_workspace_size(p, False) >= 256
    setattr(p, field, value)
    assert C.bcmt_linattn_workspace_size(p, True) == 0
    with pytest.raises(C.BCMTError) as e:
        C.bcmt_linattn_forward(p, A, 32, A, 32, A, 32, A, None, None, A, 32, A, A, 0)
    assert e.value.code == getattr(C, code), C.bcmt_last_error()
    with pytest.raises(C.BCMTError) as e:
        C.bcmt_linattn_backward(p, A, 32, A, 32, A, 32, A, 32, A, None, None, None, A, 32, A, 32,
                                A, 32, None, A, 0)
    assert e.value.code == getattr(C, code), C.bcmt_last_error()


def test_linattn_workspace_is_needed_for_long_sequences_only(C):
    short = C.bcmt_linattn_params(2, 5, 2, 16, C.BCMT_BF16, 0, 0.25)
    assert C.bcmt_linattn_workspace_size(short, False) == 256
    for dt in (C.BCMT_BF16, C.BCMT_F32):
        long = C.bcmt_linattn_params(1, 5000, 2, 16, dt, 0, 0.25)
        assert C.bcmt_linattn_workspace_size(long, False) > 256
        for ws, code in ((None, C.BCMT_ERR_ARG), (A + 8, C.BCMT_ERR_ALIGN)):
            with pytest.raises(C.BCMTError) as e:
                C.bcmt_linattn_forward(long, A, 32, A, 32, A, 32, A, None, None, A, 32, A, ws, 0)
            assert e.value.code == code


def test_linattn_refuses_bad_pointers_and_strides(C):
    p = C.bcmt_linattn_params(2, 5, 2, 16, C.BCMT_BF16, 0, 0.25)

    def forward(**kw):
        a = dict(q=A, lq=32, k=A, lk=32, v=A, lv=32, decay=A, lengths=None, s0=None, o=A, lo=32,
                 s1=None, ws=A)
        a.update(kw)
        with pytest.raises(C.BCMTError) as e:
            C.bcmt_linattn_forward(p, a["q"], a["lq"], a["k"], a["lk"], a["v"], a["lv"],
                                   a["decay"], a["lengths"], a["s0"], a["o"], a["lo"], a["s1"],
                                   a["ws"], 0)
        return e.value.code
    assert forward(q=None) == C.BCMT_ERR_ARG
    assert forward(o=None) == C.BCMT_ERR_ARG
    assert forward(decay=None) == C.BCMT_ERR_ARG
    assert forward(k=A + 8) == C.BCMT_ERR_ALIGN
    assert forward(s0=A + 4) == C.BCMT_ERR_ALIGN
    assert forward(lv=24) == C.BCMT_ERR_ARG      # shorter than a row
    assert forward(lo=36) == C.BCMT_ERR_ARG      # not a multiple of 8
    with pytest.raises(C.BCMTError) as e:        # a gradient written over what it is read from
        C.bcmt_linattn_backward(p, A, 32, A, 32, A, 32, A, 32, A, None, None, A, A, 32, A, 32,
                                A, 32, A, A, 0)
    assert e.value.code == C.BCMT_ERR_ARG and "buffer" in C.bcmt_last_error()


@pytest.mark.parametrize("field,value,code", [
    ("N", -1, "BCMT_ERR_SHAPE"), ("N", 1 << 31, "BCMT_ERR_SHAPE"), ("V", 0, "BCMT_ERR_SHAPE"),
    ("V", 1 << 24, "BCMT_ERR_SHAPE"), ("D", 0, "BCMT_ERR_SHAPE"), ("D", 12, "BCMT_ERR_SHAPE"),
    ("dtype", 2, "BCMT_ERR_ARG"), ("id_bytes", 2, "BCMT_ERR_ARG"), ("flags", 4, "BCMT_ERR_ARG"),
    ("scale", float("nan"), "BCMT_ERR_ARG"),
])
def test_embedding_refuses_bad_params(C, field, value, code):
    p = C.bcmt_embedding_params(10, 100, 16, C.BCMT_F32, 8, 0, 1.0)
    assert C.bcmt_embedding_workspace_size(p) >= 256
    setattr(p, field, value)
    assert C.bcmt_embedding_workspace_size(p) == 0
    for call in (lambda: C.bcmt_embedding_forward(p, A, A, A, 0),
                 lambda: C.bcmt_embedding_backward(p, A, A, A, A, 0)):
        with pytest.raises(C.BCMTError) as e:
            call()
        assert e.value.code == getattr(C, code), C.bcmt_last_error()


def test_embedding_refuses_bad_pointers(C):
    p = C.bcmt_embedding_params(10, 100, 16, C.BCMT_F32, 8, 0, 1.0)
    for args, code in (((None, A, A), C.BCMT_ERR_ARG), ((A + 4, A, A), C.BCMT_ERR_ALIGN),
                       ((A, A + 8, A), C.BCMT_ERR_ALIGN), ((A, A, None), C.BCMT_ERR_ARG)):
        with pytest.raises(C.BCMTError) as e:
            C.bcmt_embedding_forward(p, *args, 0)
        assert e.value.code == code
    with pytest.raises(C.BCMTError) as e:
        C.bcmt_embedding_backward(p, A, A, A, None, 0)
    assert e.value.code == C.BCMT_ERR_ARG


@pytest.mark.parametrize("field,value,code", [
    ("n", -1, "BCMT_ERR_SHAPE"), ("p", -0.1, "BCMT_ERR_ARG"), ("p", 1.01, "BCMT_ERR_ARG"),
    ("p", float("nan"), "BCMT_ERR_ARG"), ("dtype", 9, "BCMT_ERR_ARG"), ("flags", 8, "BCMT_ERR_ARG"),
    ("step", A + 4, "BCMT_ERR_ALIGN"),
])
def test_dropout_refuses_bad_params(C, field, value, code):
    p = C.bcmt_dropout_params(100, C.BCMT_BF16, 0, 0.1, 1, 2, None)
    setattr(p, field, value)
    with pytest.raises(C.BCMTError) as e:
        C.bcmt_dropout(p, A, None, A, 0)
    assert e.value.code == getattr(C, code), C.bcmt_last_error()


def test_dropout_refuses_bad_pointers(C):
    p = C.bcmt_dropout_params(100, C.BCMT_BF16, 0, 0.1, 1, 2, None)
    for x, r, y, code in ((None, None, A, C.BCMT_ERR_ARG), (A, None, None, C.BCMT_ERR_ARG),
                          (A + 2, None, A, C.BCMT_ERR_ALIGN), (A, A + 2, A, C.BCMT_ERR_ALIGN)):
        with pytest.raises(C.BCMTError) as e:
            C.bcmt_dropout(p, x, r, y, 0)
        assert e.value.code == code


def test_torch_functions_refuse_what_the_library_would_misread(C):
    from paper_2608_13578_gb300 import lm_ops as F
    q = torch.zeros(2, 3, 2, 16, device="meta")
    a = torch.zeros(2, device="meta")
    for call in (
        lambda: F.linear_attention_forward(torch.zeros(2, 3, 2, 16), torch.zeros(2, 3, 2, 16),
                                           torch.zeros(2, 3, 2, 16), torch.zeros(2)),
        lambda: F.embedding_forward(torch.zeros(3, dtype=torch.int64), torch.zeros(5, 8)),
        lambda: F.dropout_forward(torch.zeros(8), 0.1, 1, 2),
        lambda: F.linear_attention_step(q, q, q, a, None),
    ):
        with pytest.raises(ValueError):
            call()
