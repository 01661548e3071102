"""What the C entries of the decoding operators refuse, without a device: arguments are checked before anything of CUDA is
called.  Only calls that are refused belong here: the pointers lead nowhere."""
import ctypes

import pytest

import paper_2608_12573_b200 as profk
from paper_2608_12573_b200 import _build

EINVAL = -1
P = ctypes.c_void_p(1 << 20)            # some aligned address
Q = ctypes.c_void_p(1 << 21)
NULL = ctypes.c_void_p(None)
I = ctypes.c_int64


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return profk.lib()


def _backward(lib, logits=P, grad=Q, rows=4, vocab=100, stride=100, grad_stride=100, temperature=1.0, tokens=P, g_logprob=NULL, g_lse=P, k=0, top=NULL, g_top=NULL,
              dtype="f32"):
    return getattr(lib, "profk_logprobs_backward_" + dtype)(logits, I(rows), I(vocab), I(stride), ctypes.c_double(temperature), P, NULL, tokens, g_logprob, NULL, NULL,
                                                            g_lse, I(k), top, g_top, NULL, grad, I(grad_stride))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_gradient_in_place_is_refused_where_it_cannot_be_right(lib, dtype):
    """An entry that is picked out is computed from its logit after the row has been written; rows at another stride would be
    written before they are read."""
    assert _backward(lib, grad=P, g_logprob=P, dtype=dtype) == EINVAL
    assert _backward(lib, grad=P, k=2, top=P, g_top=P, dtype=dtype) == EINVAL
    assert _backward(lib, grad=P, stride=104, dtype=dtype) == EINVAL
