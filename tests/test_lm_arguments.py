"""Arguments of the torch-facing language-model operators in every form that Python
takes (CPU only: the checks of the arguments come before any kernel)."""

import pytest
import torch


@pytest.fixture(scope="module")
def F():
    from paper_2608_13578_gb300 import build
    build.build()
    from paper_2608_13578_gb300 import lm_ops
    return lm_ops


def test_keywords_in_any_order(F):
    """The device is that of the first tensor, whichever argument comes first."""
    q, a = torch.zeros(1, 2, 2, 8), torch.zeros(2)
    ids, w = torch.zeros(3, dtype=torch.int64), torch.zeros(5, 8)
    for call in (lambda: F.linear_attention_forward(scale=0.2, q=q, k=q, v=q, decay=a),
                 lambda: F.linear_attention_forward(lengths=None, state=None, q=q, k=q, v=q, decay=a),
                 lambda: F.linear_attention_backward(need_dstate=False, do=q, q=q, k=q, v=q, decay=a),
                 lambda: F.embedding_forward(scale=2.0, ids=ids, weight=w),
                 lambda: F.embedding_backward(V=5, ids=ids, dout=torch.zeros(3, 8))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_what_is_no_tensor(F):
    for call in (lambda: F.embedding_forward([1, 2], torch.zeros(5, 8)),
                 lambda: F.dropout_forward(1.0, 0.1, 1, 2),
                 lambda: F.linear_attention_forward(None, None, None, None)):
        with pytest.raises(ValueError, match="tensor"):
            call()


@pytest.mark.parametrize("scale,refused", [(1e-39, True), (-1e-40, True), (2e-38, False), (0.1, False)])
def test_backward_refuses_a_scale_without_a_reciprocal(F, scale, refused):
    """With a gradient of the last state: the reverse states start at its ratio to the
    scale, which would be infinite."""
    from paper_2608_13578_gb300 import bcmt as C
    A, p = 1 << 20, C.bcmt_linattn_params(1, 2, 1, 8, C.BCMT_F32, 0, scale)

    def code(dstate):   # the last argument but one is checked after the scale
        with pytest.raises(C.BCMTError) as e:
            C.bcmt_linattn_backward(p, A, 8, A, 8, A, 8, A, 8, A, None, None, dstate, A, 8, A, 8,
                                    A, 8, None, A + 8, 0)
        return e.value.code
    assert code(A) == (C.BCMT_ERR_ARG if refused else C.BCMT_ERR_ALIGN)
    assert code(None) == C.BCMT_ERR_ALIGN
