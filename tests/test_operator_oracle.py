"""Pins of the oracle's part for the 4-bit cache and the scores of all prompt queries: hand examples, closed forms, brute force and
the oracle's own older functions.  (No GPU needed.)"""
import numpy as np
import pytest

from oracle import madakv_oracle as O


def block(*head):
    x = np.zeros(32)
    x[:len(head)] = head
    return x


def codes(x):
    c, s = O.quantize_mx4(x)
    return np.stack([c & 15, c >> 4], -1).reshape(-1), s.reshape(-1)


@pytest.mark.parametrize("x,byte,want", [
    (block(6.0, 4.0, -3.0, 2.0, 1.5, -1.0, 0.5), 127, [7, 6, 13, 4, 3, 10, 1]),             # the format's own values
    (block(7.0, 6.99, 5.0, 5.01, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, 0.26), 127, [7, 7, 6, 7, 6, 4, 4, 2, 2, 0, 1]),   # ties to the even code
    (block(7.0625, 3.5), 128, [6, 4]),                                                        # 7.0625 / 2 = 3.53 rounds to 4; 1.75 to 2
    (block(1.0), 125, [6]),                                                                   # 1 / 2^-2 = 4
    (block(), 7, [0]), (block(-0.0), 7, [8]), (block(1e-39), 7, [0]),
    (block(3.3e38, 1.0), 252, [7, 0]), (block(np.inf, 1.0), 252, [7, 0]), (block(-np.nan, 1.0), 252, [15, 0]),
])
def test_mx4_by_hand(x, byte, want):
    got, scale = codes(x)
    assert scale.tolist() == [byte] and got[:len(want)].tolist() == want and not (got[len(want):] & 7).any()


def test_mx4_against_search():
    """The scale is the least power that leaves the largest magnitude at most 7, and every element goes to a nearest value."""
    r = np.random.default_rng(1)
    x = (r.standard_normal((200, 64)) * 2.0 ** r.integers(-60, 60, (200, 1))).astype(np.float32).astype(np.float64)
    c, s = O.quantize_mx4(x)
    y = O.dequantize_mx4(c, s).reshape(-1, 32)
    for row, got, byte in zip(x.reshape(-1, 32), y, s.reshape(-1).astype(int)):
        unit = 2.0 ** (byte - 127)
        assert np.abs(row).max() <= 7 * unit and np.abs(row).max() > 7 * unit / 2
        grid = np.concatenate([O.MX_VALUES, -O.MX_VALUES]) * unit
        assert (np.abs(got - row) <= np.abs(row[:, None] - grid).min(1) * (1 + 1e-12)).all()


def test_mx4_twice_is_once():
    r = np.random.default_rng(2)
    x = r.standard_normal((50, 128)) * 2.0 ** r.integers(-8, 8, (50, 1))
    c, s = O.quantize_mx4(x)
    c2, s2 = O.quantize_mx4(O.dequantize_mx4(c, s))
    np.testing.assert_array_equal(O.dequantize_mx4(c, s), O.dequantize_mx4(c2, s2))


@pytest.mark.parametrize("L,W", [(40, 7), (33, 32), (5, 1)])
def test_prompt_scores_contain_the_window_scores(L, W):
    """All queries = those of the window (the older function) and the prompt without it."""
    r = np.random.default_rng(L)
    Hq, H, d = 4, 2, 8
    q, k = r.standard_normal((Hq, L, d)), r.standard_normal((H, L, d))
    late = O.window_scores(q[:, L - W:], k, 0.3)
    early = np.zeros((H, L))
    early[:, :L - W] = O.prompt_scores(q[:, :L - W], k[:, :L - W], 0.3)
    np.testing.assert_allclose(O.prompt_scores(q, k, 0.3), late + early, rtol=1e-12)


def test_prompt_scores_closed_forms():
    """Equal logits: key i gets sum over r >= i of 1 / (r + 1); whatever the logits, a head's scores add up to G L."""
    L = 50
    psi = O.prompt_scores(np.zeros((3, L, 4)), np.ones((1, L, 4)), 1.0)
    np.testing.assert_allclose(psi[0], 3 * np.cumsum((1.0 / np.arange(1, L + 1))[::-1])[::-1], rtol=1e-12)
    r = np.random.default_rng(5)
    psi = O.prompt_scores(r.standard_normal((6, L, 4)) * 3, r.standard_normal((2, L, 4)), 1.0)
    np.testing.assert_allclose(psi.sum(1), [3 * L, 3 * L], rtol=1e-12)
