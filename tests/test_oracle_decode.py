"""The 64-bit oracle of the decoding operators, pinned by hand examples and by what must hold whatever the input."""
import numpy as np
import pytest

from oracle import decode as oracle


def test_logprobs_of_a_hand_example():
    r = oracle.logprobs_row([0.0, np.log(2.0), np.log(5.0)], token=1, k=2)
    assert r["lse"] == pytest.approx(np.log(8.0))
    assert r["logprob"] == pytest.approx(np.log(2 / 8))
    p = np.array([1, 2, 5]) / 8
    assert r["entropy"] == pytest.approx(-(p * np.log(p)).sum())
    assert r["top_tokens"].tolist() == [2, 1] and r["top_logprobs"] == pytest.approx(np.log(p[[2, 1]]))


def test_logprobs_of_masked_empty_and_special_rows():
    inf = np.inf
    r = oracle.logprobs_row([-inf, 3.0, -inf], token=0, k=3)
    assert r["lse"] == 3.0 and r["entropy"] == 0.0 and r["logprob"] == -inf and r["top_tokens"].tolist() == [1, 0, 2]
    r = oracle.logprobs_row([-inf, -inf], token=1)
    assert r["lse"] == -inf and r["logprob"] == -inf and r["entropy"] == 0.0
    assert np.isnan(oracle.logprobs_row([0.0, np.nan], token=0)["logprob"]) and np.isnan(oracle.logprobs_row([0.0, inf])["lse"])
    assert oracle.logprobs_row([0.0, np.nan, 1.0], k=3)["top_tokens"].tolist() == [2, 0, -1]
    assert oracle.logprobs_row([1.0, 2.0], token=-1)["logprob"] == 0.0 and np.isnan(oracle.logprobs_row([1.0, 2.0], token=2)["logprob"])
    assert oracle.logprobs_row([-0.0, 0.0, -0.0, 0.0], k=4)["top_tokens"].tolist() == [1, 3, 0, 2]


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_gradient_against_differences(temperature):
    rng = np.random.default_rng(0)
    x, h = rng.normal(size=9) * 2, 1e-6
    x[4] = -np.inf
    args = (temperature, 3, 0.7, -0.4, 1.3, np.array([2, 3]), np.array([0.5, -1.1]))
    grad, size = oracle.logprobs_gradient_row(x, *args)
    assert (size >= 0).all()
    for v in range(9):
        if v == 4:
            assert grad[v] == 0
            continue
        a, b = x.copy(), x.copy()
        a[v] += h
        b[v] -= h
        assert grad[v] == pytest.approx((oracle.logprobs_loss(a, *args) - oracle.logprobs_loss(b, *args)) / (2 * h), abs=1e-6)


def test_attention_weighs_the_tokens_of_a_sequence_only():
    rng = np.random.default_rng(1)
    k, v = rng.normal(size=(5, 2, 4, 8)), rng.normal(size=(5, 2, 4, 8))
    q = rng.normal(size=(3, 4, 8))
    tables = np.array([[3, 1], [0, 0], [2, 9]])
    out, lse = oracle.paged_attention(q, k, v, tables, [6, 0, 7], 0.5)
    assert (out[1] == 0).all() and (lse[1] == -np.inf).all()
    ks = np.concatenate([k[3, 1], k[1, 1, :2]])
    vs = np.concatenate([v[3, 1], v[1, 1, :2]])
    z = ks @ q[0, 2] * 0.5
    p = np.exp(z) / np.exp(z).sum()
    np.testing.assert_allclose(out[0, 2], p @ vs)
    assert lse[0, 2] == pytest.approx(np.log(np.exp(z).sum()))
    only, _ = oracle.paged_attention(q, k, v, tables, [6, 0, 4], 0.5)          # page 9 is not there
    np.testing.assert_allclose(out[2], only[2])


def test_fork_of_a_hand_example():
    pool = np.arange(1 * 2 * 6 * 1 * 4 * 1, dtype=np.float64).reshape(1, 2, 6, 1, 4, 1)
    before = pool.copy()
    tables = np.array([[4, 2, -1], [4, 5, -1]], dtype=np.int32)                # page 4 is shared, pages 2 and 5 are partly filled
    refs = np.array([0, 0, 1, 0, 2, 1], dtype=np.int32)
    new, lengths, counts, missing = oracle.fork(pool, tables, np.array([6, 7]), refs, np.array([0, 0, -1, 0]), 2)
    assert lengths.tolist() == [8, 8, 2, 8] and missing == 0
    assert new.tolist() == [[4, 2, -1], [4, 0, -1], [1, -1, -1], [4, 3, -1]]
    assert counts.tolist() == [1, 1, 1, 1, 3, 0]
    np.testing.assert_array_equal(pool[:, :, 0, :, :2], before[:, :, 2, :, :2])
    np.testing.assert_array_equal(pool[:, :, 0, :, 2:], before[:, :, 0, :, 2:])
    np.testing.assert_array_equal(pool[:, :, 3, :, :2], before[:, :, 2, :, :2])
    # one page is left for two that are needed, and a table of three entries for a sequence that wants four
    new, lengths, counts, missing = oracle.fork(pool, tables, np.array([6, 7]), np.array([0, 1, 1, 1, 2, 1]), np.array([0, 0, 1]), 6)
    assert lengths.tolist() == [12, 12, 12] and missing == 4
    assert new.tolist() == [[4, 2, 0], [4, -1, -1], [4, 5, -1]] and counts.tolist() == [1, 1, 1, 1, 3, 1]


def test_compaction_keeps_what_sequences_hold():
    rng = np.random.default_rng(2)
    pool = rng.normal(size=(2, 2, 9, 1, 2, 3))
    refs = np.array([0, 1, 0, 0, 2, 0, 1, 0, 1], dtype=np.int32)
    tables = np.array([[4, 1, -1], [4, 8, 6]], dtype=np.int32)
    held = [[pool[:, :, t].copy() for t in row if t >= 0] for row in tables]
    new, counts, page_map, live = oracle.compact(pool, tables, refs)
    assert live == 4 and page_map.tolist() == [-1, 1, -1, -1, 0, -1, 2, -1, 3] and counts.tolist() == [2, 1, 1, 1, 0, 0, 0, 0, 0]
    for row, want in zip(new, held):
        for t, w in zip([t for t in row if t >= 0], want):
            np.testing.assert_array_equal(pool[:, :, t], w)
