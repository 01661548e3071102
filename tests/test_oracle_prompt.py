"""The 64-bit oracle of the operators for prompts and drafts, pinned by hand examples and by what must hold whatever the input."""
import numpy as np
import pytest

from oracle import decode, prompt as oracle


def test_rotary_of_hand_examples():
    x = np.array([[[1.0, 0.0, 7.0]]])
    for turn, want in ((0.0, (1, 0)), (np.pi / 2, (0, 1)), (np.pi, (-1, 0))):
        out, _, _ = oracle.rotary(x, [1], [turn])
        assert out[0, 0] == pytest.approx([*want, 7.0], abs=1e-15)
        back, _, _ = oracle.rotary(out, [1], [turn], inverse=True)
        assert back == pytest.approx(x, abs=1e-15)
    x = np.arange(8.0).reshape(1, 1, 8)
    halves, _, _ = oracle.rotary(x, [3], [0.1, 0.2, 0.3, 0.4])
    order = [0, 4, 1, 5, 2, 6, 3, 7]                     # pairs beside one another
    pairs, _, _ = oracle.rotary(x[..., order], [3], [0.1, 0.2, 0.3, 0.4], interleaved=True)
    assert pairs == pytest.approx(halves[..., order])


def test_rotary_depends_on_differences_of_positions():
    rng = np.random.default_rng(0)
    q, k, f = rng.normal(size=(1, 1, 16)), rng.normal(size=(1, 1, 16)), 10000.0 ** (-np.arange(8) / 8)
    dots = [float((oracle.rotary(q, [a], f)[0] * oracle.rotary(k, [a - 5], f)[0]).sum()) for a in (5, 100, 10 ** 6, 2 ** 31)]
    assert dots == pytest.approx([dots[0]] * 4, abs=1e-9)
    assert np.linalg.norm(oracle.rotary(q, [77], f, magnitude=2.0)[0]) == pytest.approx(2 * np.linalg.norm(q))


def test_places():
    seq, place = oracle.places([10, 3, 7], 9, starts=[1, 4, 4, 8])
    assert seq.tolist() == [-1, 0, 0, 0, 2, 2, 2, 2, -1] and place.tolist() == [0, 7, 8, 9, 3, 4, 5, 6, 0]
    seq, place = oracle.places([10, 1], 4)
    assert seq.tolist() == [0, 0, 1, 1] and place.tolist() == [8, 9, -1, 0]


def test_chunks_are_the_single_tokens_one_after_the_other():
    rng = np.random.default_rng(1)
    k, v, tables = rng.normal(size=(6, 2, 4, 8)), rng.normal(size=(6, 2, 4, 8)), np.array([[3, 0, 5], [1, 2, -1]])
    q, lengths, starts = rng.normal(size=(7, 4, 8)), [11, 6], [0, 5, 7]
    out, lse, size, reach = oracle.paged_attention_chunk(q, k, v, tables, lengths, 0.3, starts)
    for s, (a, z) in enumerate(((0, 5), (5, 7))):
        for i, r in enumerate(range(a, z)):
            one, one_lse = decode.paged_attention(q[r:r + 1], k, v, tables[s:s + 1], [lengths[s] - (z - a) + i + 1], 0.3)
            assert out[r] == pytest.approx(one[0]) and lse[r] == pytest.approx(one_lse[0])
    assert (size >= np.abs(out) - 1e-12).all() and (reach > 0).all()


def test_chunks_that_see_nothing():
    rng = np.random.default_rng(2)
    k, v = rng.normal(size=(2, 1, 4, 8)), rng.normal(size=(2, 1, 4, 8))
    q = rng.normal(size=(4, 1, 8))
    out, lse, _, _ = oracle.paged_attention_chunk(q, k, v, np.array([[0]]), [2], 0.3)       # two of four tokens lie before the beginning
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.isfinite(lse[2:]).all()
    out, lse, _, _ = oracle.paged_attention_chunk(q, k, v, np.array([[-1]]), [4], 0.3)
    assert (out == 0).all() and np.isneginf(lse).all()
    v[0, 0, 3] = np.nan                                  # seen by the last token only
    out, _, _, _ = oracle.paged_attention_chunk(q, k, v, np.array([[0]]), [4], 0.3)
    assert np.isfinite(out[:3]).all() and np.isnan(out[3]).all()


def test_adjusted_rows():
    x = [2.0, -2.0, 0.0, 4.0, 1.0, 5.0]
    y, size, changed = oracle.adjust_row(x, tokens=[0, 1, 3, 3, 0, -1, 9], prompt=2, repetition=2.0, frequency=0.5, presence=1.0)
    # 0: in the prompt and once in the answer; 1: prompt; 3: twice in the answer
    assert y.tolist() == [1.0 - 1.5, -4.0, 0.0, 2.0 - 2.0, 1.0, 5.0] and changed.tolist() == [True, True, False, True, False, False]
    y, _, _ = oracle.adjust_row(x, bias_tokens=[2, 5, 2, 99], bias_values=[1.0, -1.0, 0.25, 7.0])
    assert y.tolist() == [2.0, -2.0, 1.25, 4.0, 1.0, 4.0]
    y, _, changed = oracle.adjust_row(x, mask=[0b101001])
    assert np.isneginf(y).tolist() == [False, True, True, False, True, False] and changed.sum() == 3
