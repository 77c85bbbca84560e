"""GPU: decode over a 4-bit cache, and decode that leaves its weights, to the precision that three bf16 parts of a weight give
(decode_precision.py derives the bound and test_decode_precision.py shows what it tells apart)."""
import numpy as np
import pytest
import torch

from paper_2506_15724_amd import binding as MB
from tests import decode_precision as DP
from tests.test_gpu_operators import DEV, KINDS, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["fp4", "bf16", "fp8"])
@pytest.mark.parametrize("G,d,rows", [(1, 64, 64), (1, 128, 128), (7, 64, 64), (7, 128, 128), (3, 128, 64), (8, 64, 33)])
def test_weights_one_by_one(kind, G, d, rows):
    """Every output is a weight and within the bound of it, and so are the accumulated sums; of the calls without weights those over
    a 4-bit cache (the others take two parts)."""
    H = 3
    t = [DP.counts(rows, 10 * h + G) for h in range(H)]
    k, v = (torch.stack(x)[None, None].to(DEV, torch.bfloat16) for x in zip(*(DP.rows_of(x, d) for x in t)))
    eng = MB.MadaKV(n_layers=1, batch=1, n_q_heads=G * H, n_kv_heads=H, head_dim=d, ctx_len=rows, window=1, budget=rows, softmax_scale=DP.SCALE, max_new_tokens=1, device=DEV, **KINDS[kind])
    eng.select_gather(0, 1, k, v, torch.zeros(1, rows, dtype=torch.uint8, device=DEV))
    q = DP.queries(G, d).repeat(H, 1)[None, None].to(DEV, torch.bfloat16)
    acc = torch.zeros(eng.capacity, device=DEV)
    outs = {}
    for name in ("plain", "weights"):
        out = torch.full((1, 1, G * H, d), float("nan"), device=DEV)
        say(f"weights one by one, {kind} G={G} d={d} rows={rows}, {name}")
        if name == "plain":
            eng.decode_attn(0, 1, q, None, None, out)
        else:
            eng.decode_attn_weights(0, 1, q, None, None, out, acc, acc)
        torch.cuda.synchronize()
        outs[name] = out.cpu().double().numpy().reshape(H, G, d)
    for h in range(H):
        w = DP.weights(t[h], G)
        for name, out in outs.items():
            err = (np.abs(out[h][:, :rows] - w) / w).max()
            say(f"head {h} {name}: {err:.2e}")
            assert not out[h][:, rows:].any()
            if kind == "fp4" or name == "weights":
                assert err <= DP.BOUND, (h, name, err)
        at = int(eng.kv_off[0, 0, h])
        paid = acc[at:at + rows].cpu().double().numpy()
        # (a weight from its logit: the reciprocal of the sum 2^-23 instead of the parts put together; G - 1 additions)
        assert (np.abs(paid - w.sum(0)) <= (DP.BOUND + (G - 1) * 2.0 ** -24) * w.sum(0)).all()
    eng.close()
