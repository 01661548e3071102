"""What the C entries of the operators for prompts and drafts refuse, without a device: arguments are checked before anything of
CUDA is called.  Only calls that are refused belong here: the pointers lead nowhere."""
import ctypes

import pytest

import paper_2608_12573_b200 as profk
from paper_2608_12573_b200 import _build

EINVAL = -1
P, Q, ODD = ctypes.c_void_p(1 << 20), ctypes.c_void_p(1 << 21), ctypes.c_void_p((1 << 20) + 1)
NULL = ctypes.c_void_p(None)
I = ctypes.c_int64
TYPES = ["f32", "bf16", "f16"]


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return profk.lib()


class _Rotary(ctypes.Structure):
    _fields_ = [("frequencies", ctypes.c_void_p), ("pairs", I), ("interleaved", ctypes.c_int), ("inverse", ctypes.c_int), ("magnitude", ctypes.c_double)]


class _Adjust(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_void_p), ("history", I), ("token_stride", I), ("lengths", ctypes.c_void_p), ("prompts", ctypes.c_void_p),
                ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p), ("repetition_value", ctypes.c_double),
                ("frequency_value", ctypes.c_double), ("presence_value", ctypes.c_double), ("bias_tokens", ctypes.c_void_p), ("bias_values", ctypes.c_void_p),
                ("biases", I), ("bias_token_stride", I), ("bias_value_stride", I), ("mask", ctypes.c_void_p), ("mask_stride", I)]


def _how(frequencies=1 << 20, pairs=32, magnitude=1.0):
    return ctypes.byref(_Rotary(frequencies, pairs, 0, 0, magnitude))


def _rotary(lib, x=P, outer=2, inner=3, heads=4, dim=64, positions=P, how=None, out=Q, dtype="bf16"):
    three = (I * 3)(1024, 256, 64)
    return getattr(lib, "profk_rotary_" + dtype)(x, I(outer), I(inner), I(heads), I(dim), three, positions, (I * 2)(3, 1), how or _how(), NULL, out)


@pytest.mark.parametrize("dtype", TYPES)
def test_rotary(lib, dtype):
    bad = [dict(x=NULL), dict(out=NULL), dict(positions=NULL), dict(outer=0), dict(inner=0), dict(heads=0), dict(heads=1 << 17), dict(dim=1026), dict(x=ODD), dict(out=ODD),
           dict(how=_how(pairs=0)), dict(how=_how(pairs=33)), dict(how=_how(pairs=513), dim=1026), dict(how=_how(frequencies=None)), dict(how=_how(magnitude=float("nan"))),
           dict(how=_how(magnitude=1e39)), dict(outer=2 ** 62, inner=4), dict(outer=2 ** 40, inner=2 ** 40), dict(outer=2 ** 38, inner=1, heads=8)]
    for how in bad:
        assert _rotary(lib, dtype=dtype, **how) == EINVAL, how


def _append(lib, q=P, k=P, v=P, heads=4, kv_heads=2, seqs=2, rows=6, dim=64, page_size=16, pages=8, width=4, table_stride=4, lengths=P, starts=NULL, tables=P, how=None,
            out=Q, k_pages=P, positions=NULL, dtype="bf16"):
    three = (I * 3)(1024, 256, 64)
    return getattr(lib, "profk_pages_append_rotary_" + dtype)(q, three, k, three, v, three, k_pages, P, three, three, tables, I(table_stride), lengths, starts, I(seqs), I(rows),
                                                              I(heads), I(kv_heads), I(dim), I(page_size), I(pages), I(width), positions, None, how or _how(), NULL, out)


THIRD = (2 ** 64 + 2) // 3 - 2 ** 64                              # times 3: 2 behind 2^64


@pytest.mark.parametrize("dtype", TYPES)
def test_append(lib, dtype):
    bad = [dict(k=NULL), dict(v=NULL), dict(k_pages=NULL), dict(lengths=NULL), dict(tables=NULL), dict(q=NULL), dict(out=NULL), dict(heads=0), dict(heads=-1), dict(kv_heads=0),
           dict(seqs=0), dict(rows=0), dict(rows=5), dict(rows=1 << 31), dict(seqs=1 << 25, rows=1 << 25), dict(pages=0), dict(pages=1 << 31), dict(table_stride=-1),
           dict(how=_how(pairs=40)), dict(k=ODD), dict(q=ODD), dict(positions=P)]
    bad += [dict(width=w, page_size=s) for w, s in ((0, 16), (4, 0), (THIRD, 3), (2 ** 62, 4), (2 ** 40, 2 ** 24), (1, 2 ** 32 + 1), (2 ** 32, 2 ** 32))]
    for how in bad:
        assert _append(lib, dtype=dtype, **how) == EINVAL, how


def _chunk(lib, q=P, k=P, lengths=P, starts=NULL, seqs=2, rows=6, heads=4, kv_heads=2, dim=64, page_size=16, pages=8, width=4, scale=0.125, strides=(2048, 1024, 64),
           out=Q, lse=Q, dtype="bf16"):
    three, s = (I * 3)(1024, 256, 64), (I * 3)(*strides)
    return getattr(lib, "profk_paged_attention_chunk_" + dtype)(q, three, k, P, s, s, P, I(width), lengths, starts, I(seqs), I(rows), I(heads), I(kv_heads), I(dim), I(page_size),
                                                                I(pages), I(width), ctypes.c_double(scale), P, ctypes.c_size_t(1 << 40), NULL, out, lse)


@pytest.mark.parametrize("dtype", TYPES[1:])
def test_chunk_attention(lib, dtype):
    bad = [dict(q=NULL), dict(k=NULL), dict(lengths=NULL), dict(out=NULL), dict(lse=NULL), dict(seqs=0), dict(rows=0), dict(rows=7), dict(heads=5), dict(kv_heads=0), dict(dim=4),
           dict(dim=60), dict(dim=264), dict(pages=0), dict(strides=(2044, 1024, 64)), dict(strides=(2048, 1024, 4)), dict(q=ODD), dict(k=ctypes.c_void_p((1 << 20) + 8)),
           dict(out=ctypes.c_void_p((1 << 20) + 8)), dict(rows=2 ** 30, heads=4), dict(rows=2 ** 62), dict(seqs=1 << 25, rows=1 << 25, heads=2, kv_heads=1)]
    bad += [dict(width=w, page_size=s) for w, s in ((0, 16), (THIRD, 3), (2 ** 62, 4), (1, 2 ** 32 + 1), (2 ** 32, 2 ** 32))]
    bad += [dict(scale=s) for s in (0.0, -1.0, float("nan"), float("inf"), 3e38, 1e39, 1e-39, 1e-300)]
    for how in bad:
        assert _chunk(lib, dtype=dtype, **how) == EINVAL, how
    size = ctypes.c_size_t(0)
    for dim in (0, 4, 12, 264, -8):
        assert lib.profk_paged_attention_chunk_workspace_bytes(I(dim), ctypes.byref(size)) == EINVAL
    assert lib.profk_paged_attention_chunk_workspace_bytes(I(64), None) == EINVAL


def _adjust(lib, logits=P, rows=3, vocab=100, stride=100, out=Q, out_stride=100, dtype="f32", **how):
    fields = dict(tokens=1 << 20, history=10, token_stride=10, repetition_value=1.5)
    fields.update(how)
    return getattr(lib, "profk_adjust_logits_" + dtype)(logits, I(rows), I(vocab), I(stride), ctypes.byref(_Adjust(**fields)), NULL, out, I(out_stride))


@pytest.mark.parametrize("dtype", TYPES)
def test_adjust(lib, dtype):
    bad = [dict(logits=NULL), dict(out=NULL), dict(rows=0), dict(vocab=0), dict(stride=99), dict(out_stride=99), dict(logits=ODD), dict(out=ODD), dict(out=P, out_stride=104),
           dict(tokens=None), dict(history=-1), dict(history=1 << 30), dict(biases=-1), dict(biases=8193, bias_tokens=1 << 20, bias_values=1 << 20), dict(biases=3),
           dict(biases=3, bias_tokens=1 << 20), dict(rows=2 ** 40, vocab=2 ** 10), dict(rows=1 << 28), dict(vocab=2 ** 31)]
    bad += [dict(repetition_value=r) for r in (0.0, -1.0, float("nan"), float("inf"), 1e39, 1e-60)]
    bad += [dict(frequency_value=float("inf")), dict(frequency_value=1e39), dict(presence_value=float("nan"))]
    for how in bad:
        assert _adjust(lib, dtype=dtype, **how) == EINVAL, how
    assert getattr(lib, "profk_adjust_logits_" + dtype)(P, I(3), I(100), I(100), None, NULL, Q, I(100)) == EINVAL
