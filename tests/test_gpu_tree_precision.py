"""GPU: 16-bit outputs of trees of up to 64 nodes x query heads per KV head: weights as two bf16 numbers each, as decode's are."""
import math

import pytest
import torch

from tests.test_gpu_operators import KINDS, make, row_numbers, stored, values
from tests.test_gpu_tree import DEV, attend, kind_of, nodes, some_tree

pytestmark = pytest.mark.gpu


def reference(eng, args, l, b, h, q, k_new, v_new, sees):
    """(out, weighted |v|, largest sum of |q k|) of the rows of one KV head in 64 bits."""
    c = eng.cfg
    G, i = c.n_q_heads // c.n_kv_heads, (l * c.batch + b) * c.n_kv_heads + h
    at = row_numbers(eng, args, i)
    k, v = (torch.cat([values(eng, args, w)[at].double(), stored(x[l, b, h], kind_of(args)).double()]) for w, x in (("k_c", k_new), ("v_c", v_new)))
    may = torch.cat([torch.ones(len(sees), len(at), dtype=torch.bool), sees], 1)
    qq = q[l, b, h * G:(h + 1) * G].cpu().double()
    w = torch.softmax((qq @ k.T / math.sqrt(c.head_dim)).masked_fill(~may, -math.inf), -1)
    return w @ v, w @ v.abs(), float((qq.abs() @ k.abs().T).max()) / math.sqrt(c.head_dim), len(at)


def bound(d, n, size, spent):
    """Off before the output is rounded: a weight of two bf16 numbers has 2^-8 of what 2^-8 of it left; logits and sums as in attention with 32-bit
    outputs (d + 2 roundings of 2^-24 of a logit, twice; a rounding per row and merge)."""
    return (2.0 ** -16 + 2 * (d + 2) * 2.0 ** -24 * size + 2 * (n + 96) * 2.0 ** -24) * spent


CASES = [(1, [9, 64, 171], 128, 3, 0), (5, [200, 8, 300], 64, 6, 0), (16, [100, 64], 64, 8, 64), (8, [700, 513], 128, 16, 0), (32, [40, 500], 128, 4, 16), (64, [63, 1100], 64, 2, 0)]


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("T,lens,d,Hq,P", CASES)
def test_outputs_of_16_bits(T, lens, d, Hq, P, kind):
    """Off by their own rounding, half a step of 2^-8, and by little of what the weights add up to."""
    print(f"[tree_precision] T={T} lens={lens} d={d} Hq={Hq} P={P} {kind}", flush=True)
    eng, args, *_ = make(lens, n_q_heads=Hq, n_kv_heads=len(lens), head_dim=d, ctx_len=max(lens) + 100, page_rows=P, out_fp32=0, **KINDS[kind])
    q, k, v = nodes(eng, T, T)
    tree = some_tree(1, T, T)
    out = attend(eng, q, k, v, tree)
    sees = torch.tensor([[bool(int(m) >> j & 1) for j in range(T)] for m in tree[0].tolist()])
    G = Hq // len(lens)
    for h in range(len(lens)):
        ref, spent, size, n = reference(eng, args, 0, 0, h, q, k, v, sees)
        off = bound(d, n + T, size, spent)
        err = (out[0, 0, h * G:(h + 1) * G].cpu().double() - ref).abs()
        tol = off + 2.0 ** -8 * (ref.abs() + off) + 1e-30
        assert bool((err <= tol).all()), (h, float((err / tol).max()))


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("Hq", [2, 4, 12])
@pytest.mark.parametrize("P", [0, 16])
def test_token_by_token(kind, Hq, P):
    """What decode steps along a branch give, up to the two outputs' own roundings."""
    print(f"[tree_precision] token by token {kind} Hq={Hq} P={P}", flush=True)
    kw = dict(n_q_heads=Hq, n_kv_heads=2, head_dim=64, ctx_len=400, page_rows=P, max_new_tokens=40, out_fp32=0, **KINDS[kind])
    (eng, args, *_), (one, *_) = make([300, 147], **kw), make([300, 147], **kw)
    T = 10
    q, k, v = nodes(eng, T, 3)
    parents = [-1, 0, 0, 1, 3, 2, 4, 5, 6, 8]
    masks = []
    for t, p in enumerate(parents):
        masks.append((masks[p] if p >= 0 else 0) | 1 << t)
    out = attend(eng, q, k, v, torch.tensor([masks], dtype=torch.int64, device=DEV))
    sees = torch.tensor([[bool(m >> j & 1) for j in range(T)] for m in masks])
    refs = [reference(eng, args, 0, 0, h, q, k, v, sees) for h in range(2)]
    for t in (0, 1, 3, 4, 6, 8, 9):
        step = torch.empty(1, 1, Hq, 64, dtype=torch.bfloat16, device=DEV)
        one.decode_attn(0, 1, *(x[:, :, :, t].contiguous() for x in (q, k, v)), step)
        torch.cuda.synchronize()
        for h in range(2):
            ref, spent, size, n = (x[:, t] if torch.is_tensor(x) else x for x in refs[h])
            a, b = (x.cpu().double() for x in (out[0, 0, h * Hq // 2:(h + 1) * Hq // 2, t], step[0, 0, h * Hq // 2:(h + 1) * Hq // 2]))
            off = bound(64, n + T, size, spent)                  # (decode's weights have no fewer bits)
            tol = 2 * (off + 2.0 ** -8 * (ref.abs() + off)) + 1e-30
            assert bool(((a - b).abs() <= tol).all()), (t, h, float(((a - b).abs() / tol).max()))
