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


# --- factors of the exponents, which the kernels hold in fp32 ---------------------------------------------------------

BEYOND_FP32 = [2e38, 1e60, 1e-39, 1e-46, 1e-300]          # their reciprocals or they themselves are no normal fp32 numbers (or overflow times log2 e)


def _forward(lib, temperature, dtype="f32"):
    return getattr(lib, "profk_logprobs_" + dtype)(P, I(4), I(100), I(100), NULL, I(0), ctypes.c_double(temperature), NULL, NULL, P, NULL, NULL, NULL, NULL)


@pytest.mark.parametrize("temperature", [0.0, -1.0, float("nan"), float("inf")] + BEYOND_FP32)
def test_temperatures_that_fp32_cannot_hold_are_refused(lib, temperature):
    assert _forward(lib, temperature) == EINVAL and _forward(lib, temperature, "bf16") == EINVAL
    assert _backward(lib, temperature=temperature) == EINVAL


def _attention(lib, scale=0.125, dtype="bf16", width=8, page_size=16, workspace=P):
    strides = (I * 3)(2048, 1024, 64)
    return getattr(lib, "profk_paged_attention_" + dtype)(P, I(256), I(64), P, P, strides, strides, P, I(width), P, I(2), I(4), I(2), I(64), I(page_size), I(10), I(width),
                                                          ctypes.c_double(scale), workspace, ctypes.c_size_t(1 << 40), NULL, P, P)


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf"), 3e38, 1e39, 1e-39, 1e-46, 1e-300])
def test_scales_that_fp32_cannot_hold_are_refused(lib, scale):
    assert _attention(lib, scale) == EINVAL and _attention(lib, scale, "f16") == EINVAL


# --- sizes whose products pass 64 bits -------------------------------------------------------------------------------

class _Pool(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in "layers kv_heads page_size row_bytes layer kv page head token".split()]


def _pool(kv_heads=2, page_size=16, row_bytes=128):
    return ctypes.byref(_Pool(1 << 20, 1, kv_heads, page_size, row_bytes, 1 << 24, 1 << 23, 1 << 12, 1 << 11, 128))


def _fork(lib, width=8, page_size=16, grow=1, pool=None):
    return lib.profk_pages_fork(pool, P, I(2), I(width), I(width), P, P, I(64), P, I(2), I(page_size), I(grow), Q, ctypes.c_size_t(1 << 40), NULL, P, Q, Q, Q)


def _append(lib, width=8, page_size=16, tokens=1, kv_heads=2):
    three = (I * 3)(1024, 512, 128)
    return lib.profk_pages_append(P, P, three, three, P, P, three, three, P, I(width), P, I(2), I(tokens), I(kv_heads), I(128), I(page_size), I(64), I(width), NULL)


def test_products_of_sizes_do_not_wrap(lib):
    third = (2 ** 64 + 2) // 3                                   # times 3: 2 behind 2^64
    assert 3 * third % 2 ** 64 == 2
    signed = third if third < 2 ** 63 else third - 2 ** 64
    for width, page in ((signed, 3), (2 ** 62, 4), (2 ** 60, 16), (2 ** 40, 2 ** 24), (1, 2 ** 32 + 1), (2 ** 32, 2 ** 32)):
        assert _attention(lib, width=width, page_size=page) == EINVAL, (width, page)
        assert _fork(lib, width, page) == EINVAL, (width, page)
        assert _append(lib, width, page) == EINVAL, (width, page)
        assert _append(lib, width, page, tokens=2) == EINVAL, (width, page)
    for page in (2 ** 60, 2 ** 59 + 1, 2 ** 32):                 # heads times tokens times vectors of a page
        pool = _pool(kv_heads=16, page_size=page, row_bytes=16)
        assert lib.profk_pages_copy(pool, I(10), P, P, I(1), NULL) == EINVAL
        assert lib.profk_pages_compact(pool, P, I(2), I(8), I(8), P, I(64), Q, ctypes.c_size_t(1 << 40), NULL, Q, Q, Q, Q) == EINVAL
