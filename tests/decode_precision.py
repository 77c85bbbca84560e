"""Decode steps whose outputs are the softmax weights themselves: row r of V is 1 at dim r and 0 elsewhere, so that out[q, r] is the weight
of row r, with nothing to average errors away.

Logits are small whole numbers t times a power of two, exact in every kind of cache (K has t ones, the queries 1 + g / 8).  What is left
is, relative to a weight, with |x| < 1.4 the exponents in log2 units:
  the exponents: log2(e) as a float, the product with it, the difference to the maximum, half a step (2^-24) of |x| each: 3 * 1.4 * ln 2 * 2^-24 = 1.8e-7
  exp2: 2^-23 = 1.2e-7
    (both once in the weight and once, averaged, in the sum they are divided by)
  the sum of a head: at most four additions in a lane, five among lanes and waves, four among pieces: 13 * 2^-24 = 7.8e-7
  the weight's parts put together, rescaled to a wave's and a piece's maximum, divided: 5 * 2^-24 = 3.0e-7
1.7e-6 in all.  The matrix instructions take weights in bf16 parts: two of them leave up to 2^-17 = 7.6e-6 of a weight, three 2^-25."""
import numpy as np
import torch

BOUND = 1.7e-6
SCALE = 2.0 ** -7


def counts(rows, seed):
    """t of every row: 0 .. 64, and 64, the largest, among every 16 rows (so that all tiles have the same maximum)."""
    t = np.random.default_rng(seed).integers(0, 64, rows)
    t[7::16] = 64
    return t


def rows_of(t, d):
    """(K, V) [rows, d]"""
    k, v = torch.zeros(len(t), d), torch.zeros(len(t), d)
    for r, n in enumerate(t):
        k[r, (np.arange(n) * 5 + r) % d] = 1.0
        v[r, r % d] = 1.0
    return k, v


def queries(G, d):
    return (1 + torch.arange(G) / 8)[:, None].expand(G, d).contiguous()


def logits(t, G):
    """[G, rows] in 64 bits"""
    return SCALE * (1 + np.arange(G) / 8)[:, None] * t[None, :]


def weights(t, G):
    w = np.exp(logits(t, G) - logits(t, G).max(1, keepdims=True))
    return w / w.sum(1, keepdims=True)


def bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).to(torch.float64).numpy()


def parts(p, n):
    """p (floats, in 64 bits) as n bf16 parts: [n, ...]"""
    out, left = [], p
    for _ in range(n):
        out.append(bf16(left))
        left = left - out[-1]
    return np.stack(out)
