"""The bound of test_gpu_decode_precision.py tells kernels apart that take the weights as they are from ones that lose parts of them: checked
on the arithmetic itself.  No GPU."""
import numpy as np
import pytest

from tests import decode_precision as DP


def through_parts(t, G, keep=3, mix=None):
    """The outputs of a decode step whose weights enter as `keep` bf16 parts, the third of them taken from other keys where `mix` says so."""
    p = np.exp(DP.logits(t, G) - DP.logits(t, G).max(1, keepdims=True)).astype(np.float32).astype(np.float64)
    x = DP.parts(p, 3)
    if mix is not None:
        x[2] = x[2][:, mix]
    return x[:keep].sum(0) / p.sum(1, keepdims=True)


def off(got, t, G):
    w = DP.weights(t, G)
    return np.abs(got - w) / w


@pytest.mark.parametrize("rows", [64, 128])
@pytest.mark.parametrize("G", [1, 7])
def test_the_bound_tells(rows, G):
    t = DP.counts(rows, rows + G)
    assert off(through_parts(t, G), t, G).max() < 0.1 * DP.BOUND
    # without the third part, and with the third part of a neighbour, of the other 16 keys of a tile, of another lane group or query column:
    # beyond the bound among any 16 keys, and by more than the other errors could make up for in every query
    r = np.arange(rows)
    for kw in (dict(keep=2), *(dict(mix=m) for m in (r ^ 1, r ^ 16, r ^ 4, r // 16 * 16 + (r + 8) % 16))):
        lost = off(through_parts(t, G, **kw), t, G).reshape(G, -1, 16).max(-1)
        assert (lost.max(1) > 2 * DP.BOUND).all() and (lost > DP.BOUND).all(), (kw, lost.min())
