"""GPU: decode that accumulates its weights, in the variants that calls of many heads and of long ones take (tiles of 32 rows, pieces of
256 to 1024 rows, several tiles per wave, eight rows in flight); every step against 64 bits."""
import pytest
import torch

from tests.test_gpu_operators import DEV, KINDS, make, say, weights_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,Hq,H,d,B,L,P", [
    ("bf16", 128, 64, 64, 3, 45, 0), ("fp8", 128, 64, 64, 3, 45, 0), ("fp4", 128, 64, 64, 3, 45, 0), ("bf16", 64, 32, 128, 5, 60, 16), ("bf16", 160, 40, 64, 4, 70, 16), ("fp32", 64, 64, 64, 3, 45, 0),
    ("bf16", 8, 4, 64, 1, 20011, 0), ("fp8", 8, 4, 64, 1, 20011, 0), ("fp8", 6, 3, 128, 1, 30007, 64), ("bf16", 15, 3, 128, 1, 30007, 0), ("fp4", 8, 4, 64, 1, 20011, 0),
    ("bf16", 2, 2, 128, 1, 70001, 0), ("fp8", 2, 2, 64, 1, 70001, 0), ("fp32", 2, 2, 64, 1, 40003, 0), ("fp32", 6, 2, 128, 1, 9001, 0), ("fp4", 2, 2, 128, 1, 70001, 64)])
def test_weights_of_many_and_of_long_heads(kind, Hq, H, d, B, L, P):
    """Heads that keep the whole prompt: a row appended, rows replaced at the front, inside and at the end, the row chosen by the step before."""
    eng, args, *_ = make(None, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=4, max_new_tokens=1, page_rows=P, **KINDS[kind])
    g = torch.Generator().manual_seed(L)
    acc = torch.rand(eng.capacity, generator=g).to(DEV)
    pos = torch.arange(L, L + B, dtype=torch.int32, device=DEV)
    heads = B * H
    draw = lambda: [torch.randn(1, B, h, d, generator=g).to(DEV, eng.tdtype) for h in (Hq, H, H)]      # noqa: E731
    say(f"{kind} {Hq}/{H} d={d} B={B} L={L} P={P}: append")
    acc, slot = weights_step(eng, args, *draw(), acc, 1.0, None, pos, 8)
    for slots in ([(0, L, L // 2, L - 1, -1, L + 1)[i % 6] for i in range(heads)], slot.tolist()):
        say(f"replace {slots[:6]}")
        pos += 1
        acc, slot = weights_step(eng, args, *draw(), acc, 0.9, slots, pos, 8)
    eng.close()
