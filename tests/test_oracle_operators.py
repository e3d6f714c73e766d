"""Pins of the oracles of the serving calls: small cases worked out by hand, and properties."""
import numpy as np
import pytest

import oracle


def test_reserve_by_hand():
    # pages of 32 rows; request 0 grows from 1 to 3 pages, 1 ends, 2 stays, 3 grows by one
    table = np.array([[9, 0, 0, 0], [4, 5, 6, 0], [7, 0, 0, 0], [8, 0, 0, 0]], np.int32)
    free = np.array([1, 2] + [0] * 8, np.int32)
    t, held, fr, nf, short, slots = oracle.kv_reserve_paged(
        table, [1, 3, 1, 1], [31, 0, 10, 32], [40, 0, 2, 1], free, 2, 32, 40)
    # stack after the pushes: 1 2 4 5 6; request 0 takes 6, 5, request 3 takes 4
    assert t[0].tolist() == [9, 6, 5, 0] and t[3].tolist() == [8, 4, 0, 0]
    assert held.tolist() == [3, 0, 1, 2] and nf == 2 and short == 0
    assert fr[:5].tolist() == [1, 2, 4, 5, 6]
    assert slots[0, :3].tolist() == [9 * 32 + 31, 6 * 32, 6 * 32 + 1]
    assert slots[2, :3].tolist() == [7 * 32 + 10, 7 * 32 + 11, -1]
    assert slots[3, :2].tolist() == [4 * 32, -1] and (slots[1] == -1).all()


def test_reserve_short_pool():
    # two free pages: request 0 takes one, 1 needs two (short), 2 needs one but comes later
    table = np.zeros((4, 2), np.int32)
    _, held, _, nf, short, slots = oracle.kv_reserve_paged(
        table, [0, 0, 0, 0], [0, 0, 0, 0], [32, 33, 1, 65], np.array([3, 5, 0, 0]), 2, 32, 70)
    assert held.tolist() == [1, 0, 0, 0] and nf == 1 and short == 3
    assert slots[0, 0] == 5 * 32 and (slots[1:] == -1).all()


def test_decode_uniform_scores():
    # equal scores: the mean of the values; no rows: zeros
    rng = np.random.default_rng(0)
    K, V = np.ones((3, 32, 1, 64)), rng.standard_normal((3, 32, 1, 64))
    Q = rng.standard_normal((2, 2, 64))
    O, _, _ = oracle.decode_attention_paged(Q, K, V, np.array([[2, 0], [1, 0]]), [40, 0], 0.125)
    want = np.concatenate([V[2, :, 0], V[0, :8, 0]]).mean(0)
    np.testing.assert_allclose(O[0], np.stack([want, want]), rtol=1e-12)
    assert (O[1] == 0).all()


def test_sample_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    at = [0.05, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91]
    assert [oracle.sample_row(x, u)[0] for u in at] == [1, 1, 3, 3, 2, 2, 0]
    assert oracle.sample_row(x, 0.5)[1] == pytest.approx(0.3, abs=1e-12)
    assert [oracle.sample_row(x, u, top_k=2)[0] for u in (0.5, 0.6, 0.999)] == [1, 3, 3]
    assert oracle.sample_row(x, 0.999, top_p=0.65)[0] == 3         # 0.4 + 0.3 reaches 0.65
    assert oracle.sample_row(x, 0.999, top_p=0.75)[0] == 2
    assert oracle.sample_row(x, 0.999, min_p=0.6)[0] == 3          # 0.3 >= 0.6 * 0.4
    assert oracle.sample_row(x, 0.999, temperature=0.0) == (1, 1.0)


def test_sample_edges():
    inf = np.inf
    assert oracle.sample_row([np.nan, np.nan], 0.5) == (0, 0.0)
    assert oracle.sample_row([1.0, inf, np.nan, inf], 0.6) == (3, 0.5)
    assert oracle.sample_row([np.nan, -inf, -inf], 0.6) == (2, 0.5)
    assert oracle.sample_row([0.0, -0.0, 0.0, 0.0], 0.5) == (2, 0.25)   # ties by index
    assert oracle.sample_row([0.0, -0.0, 0.0, 0.0], 0.999, top_k=2) == (1, 0.5)
    assert oracle.sample_row([0.0, 0.0, 0.0, 0.0], 0.999, top_p=0.5) == (1, 0.5)
    assert oracle.sample_row([1.0, 2.0, 2.0], 0.999, min_p=1.0) == (2, 0.5)
    assert oracle.sample_row([1.0, 2.0], 0.999, top_p=0.0) == (1, 1.0)


def test_sample_frequencies():
    rng = np.random.default_rng(5)
    x = rng.standard_normal(50) * 2
    u = (np.arange(4000) + 0.5) / 4000
    tok = np.array([oracle.sample_row(x, t, temperature=0.7)[0] for t in u])
    p = np.exp(x / 0.7) / np.exp(x / 0.7).sum()
    # an even grid of 4000 numbers leaves each token's share off by less than one step
    assert np.abs(np.bincount(tok, minlength=50) / 4000 - p).max() <= 1 / 4000 + 1e-9
