"""Pins of the oracle's prompt operators."""
import math

import numpy as np
import torch

import oracle
from oracle.rope import rms_norm, rotate


def test_rotation_keeps_lengths_and_composes():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 3, 16))
    f, _ = oracle.rope_frequencies(16, 1e4)
    for il in (False, True):
        y = rotate(x, np.array([3, 0, 7, 100, 5]), f, 1.0, il)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        assert np.array_equal(y[1], x[1])
        z = rotate(y, np.array([4, 0, -7, 1, -5]), f, 1.0, il)
        assert np.allclose(z, rotate(x, np.array([7, 0, 0, 101, 0]), f, 1.0, il))
    # dot products depend on the distance alone
    q, k = rng.standard_normal((2, 1, 1, 16))
    dots = [float((rotate(q, np.array([p + 9]), f, 1.0, False) *
                   rotate(k, np.array([p]), f, 1.0, False)).sum()) for p in (0, 5, 900)]
    assert np.allclose(dots, dots[0])


def test_layouts_are_permutations_of_each_other():
    x = np.random.default_rng(1).standard_normal((4, 2, 16))
    f, _ = oracle.rope_frequencies(8, 1e4)
    pos = np.array([0, 1, 50, 7])
    p = np.r_[0, 2, 4, 6, 1, 3, 5, 7, 8:16]                # interleaved order -> halves
    a, b = rotate(x, pos, f, 1.3, True), rotate(x[..., p], pos, f, 1.3, False)
    assert np.allclose(a[..., p], b) and np.array_equal(a[..., 8:], x[..., 8:])


def test_frequencies():
    f, m = oracle.rope_frequencies(8, 1e4)
    assert np.allclose(f, [1, 0.1, 0.01, 0.001]) and m == 1
    assert np.allclose(oracle.rope_frequencies(8, 1e4, "linear", 4.0)[0], f / 4)
    ntk, _ = oracle.rope_frequencies(8, 1e4, "ntk", 4.0)
    assert math.isclose(ntk[0], 1.0) and math.isclose(ntk[-1], f[-1] / 4)
    L = 2 * math.pi * 1000                                 # turns: 1000, 100, 10, 1
    y, m = oracle.rope_frequencies(8, 1e4, "yarn", 4.0, L)
    g = 9 / 31
    assert np.allclose(y, [1, 0.1, 0.01 * (g + (1 - g) / 4), 0.001 / 4])
    assert math.isclose(m, 0.1 * math.log(4) + 1)


def test_norm():
    x = np.random.default_rng(2).standard_normal((3, 2, 8))
    y = rms_norm(x, np.ones(8), 0.0)
    assert np.allclose((y ** 2).mean(-1), 1) and np.allclose(rms_norm(5 * x, np.ones(8), 0.0), y)


def test_chunk_attention_is_causal_attention():
    rng = np.random.default_rng(3)
    K, V = rng.standard_normal((2, 6, 32, 2, 8))
    table = np.array([[4, 1, 0], [2, 5, 3]])
    Q = rng.standard_normal((47, 4, 8))
    O, _, _, N = oracle.chunk_attention_paged(Q, K, V, table, [0, 40, 47], [40, 70], 0.3)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a))  # noqa: E731
    for b, (a, e, kv) in enumerate(((0, 40, 40), (40, 47, 70))):
        k, v = (np.concatenate([x[p] for p in table[b]])[:kv].repeat(2, axis=1) for x in (K, V))
        n = e - a
        mask = torch.tril(torch.ones(kv, kv, dtype=torch.bool))[kv - n:]
        ref = torch.nn.functional.scaled_dot_product_attention(
            t(Q[a:e]).transpose(0, 1), t(k).transpose(0, 1), t(v).transpose(0, 1), attn_mask=mask,
            scale=0.3)
        assert np.allclose(O[a:e], ref.transpose(0, 1).numpy())
    assert list(N[40:]) == list(range(64, 71))
    one = oracle.chunk_attention_paged(Q[:2], K, V, table, [0, 1, 2], [33, 70], 0.3)[0]
    assert np.allclose(one, oracle.decode_attention_paged(Q[:2], K, V, table, [33, 70], 0.3)[0])


def test_chunk_windows_and_tokens_without_rows():
    rng = np.random.default_rng(4)
    K, V = rng.standard_normal((2, 2, 32, 1, 8))
    Q, table = rng.standard_normal((6, 1, 8)), np.array([[1, 0]])
    O = oracle.chunk_attention_paged(Q, K, V, table, [0, 6], [50], 0.3, window=1)[0]
    assert np.allclose(O[:, 0], np.concatenate([V[1], V[0]])[44:50, 0])   # each sees itself
    O = oracle.chunk_attention_paged(Q, K, V, table, [0, 6], [2], 0.3)[0]
    assert (O[:4] == 0).all() and np.allclose(O[4, 0], V[1, 0, 0])
    O = oracle.chunk_attention_paged(Q, K, V, table, [1, 5], [4], 0.3)[0]
    assert np.isnan(O[[0, 5]]).all() and np.isfinite(O[1:5]).all()


def test_logprobs_closed_forms():
    lp, ent, rank, idx, tlp, _ = oracle.logprobs_row(np.zeros(8), 5, 3)
    assert math.isclose(lp, -math.log(8)) and math.isclose(ent, math.log(8)) and rank == 5
    assert list(idx) == [0, 1, 2] and np.allclose(tlp, -math.log(8))
    x = np.random.default_rng(5).standard_normal(100) * 4
    lp, ent, rank, idx, tlp, _ = oracle.logprobs_row(x, 17, 100)
    ref = torch.log_softmax(torch.from_numpy(x), 0)
    assert math.isclose(lp, float(ref[17])) and math.isclose(ent, float(-(ref.exp() * ref).sum()))
    assert rank == int((x > x[17]).sum()) and np.allclose(tlp, np.sort(ref.numpy())[::-1])


def test_logprobs_special_values():
    inf, nan = math.inf, math.nan
    row = oracle.logprobs_row
    assert row(np.array([nan, nan]), 1, 2)[:3] == (-inf, 0.0, 1)
    lp, ent, rank, idx, tlp, _ = row(np.array([-inf, nan, -inf]), 2, 3)
    assert math.isclose(lp, -math.log(2)) and rank == 1 and list(idx) == [0, 2, 1]
    lp, ent, rank, idx, tlp, _ = row(np.array([1.0, inf, -inf, nan, inf]), 0, 5)
    assert lp == -inf and rank == 2 and list(idx) == [1, 4, 0, 2, 3] and math.isclose(ent, math.log(2))
    assert row(np.array([0.0, -0.0]), 1, 1)[2] == 1        # equal: by index
    assert row(np.array([1.0]), -1, 0)[0] == -inf and row(np.array([1.0]), 1, 0)[2] == -1
