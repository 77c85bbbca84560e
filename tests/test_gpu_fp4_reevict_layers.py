"""GPU: re-eviction of some layers of a 4-bit cache, whose workspace holds K as bf16 for the rows of those layers alone."""
import pytest
import torch

from paper_2506_15724_amd import binding as MB
from tests.test_gpu_operators import DEV, row_numbers, say, stored, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,H,d,W,budget", [(4, 4, 128, 16, 150), (14, 2, 64, 8, 60), (8, 1, 64, 32, 300)])
def test_fp4_reeviction_of_some_layers(Hq, H, d, W, budget):
    """Layer by layer, two at a time and all at once, with other numbers of appended rows in every layer and an empty head: as a bf16
    cache of the same values, position by position, and nothing written behind the workspace of so many layers."""
    NL, B, L, T = 4, 3, 700, 20
    kw = dict(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=W, budget=budget, max_new_tokens=T, hcc_rho=4, device=DEV)
    args = dict(n_layers=NL, batch=B, n_kv_heads=H, n_q_heads=Hq, head_dim=d, page_rows=0)
    g = torch.Generator(device=DEV).manual_seed(d)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)        # noqa: E731
    exact = lambda x: stored(x, 4).to(DEV, torch.bfloat16)                                # noqa: E731  (what 4 bits hold of it)
    q, k, v = randn(NL, B, Hq, W, d), exact(randn(NL, B, H, L, d)), exact(randn(NL, B, H, L, d))
    mask = torch.randint(0, 2, (B, L), generator=g, device=DEV).to(torch.uint8)
    engs = [MB.MadaKV(cache_fp8=kind, **kw) for kind in (4, 0)]
    for e in engs:
        e.evict(0, NL, q, k, v, mask)
        e.kv_len[2, 1, H - 1] = 0
    out = torch.zeros(1, B, Hq, d, device=DEV)
    for calls in (((0, 1), (1, 1), (2, 1), (3, 1)), ((1, 2), (0, 1), (3, 1)), ((2, 2), (0, 2)), ((0, 4),)):
        for l in range(NL):
            for step in range(3 + 4 * l if l != 2 else 7):            # (layers 1 and 2: the same number)
                x = randn(1, B, Hq, d), exact(randn(1, B, H, d)), exact(randn(1, B, H, d))
                for e in engs:
                    e.decode_attn(l, 1, *x, out)
        for l0, n in calls:
            recent = randn(n, B, Hq, W, d)
            say(f"fp4 reevict {Hq}/{H} d={d} layers {l0} .. {l0 + n - 1}")
            torch.cuda.synchronize()
            for e in engs:
                need = MB.madakv_reevict_workspace_bytes(e.h, n)
                room = torch.full((need + (1 << 20),), 0xA5, dtype=torch.uint8, device=DEV)
                e.reevict_ws = room[:need]
                e.reevict(l0, n, recent, mask)
                torch.cuda.synchronize()
                assert (room[need:] == 0xA5).all()
        for n in ("kv_len", "budgets"):
            a, b = (getattr(e, n).clone() for e in engs)
            a[2, 1, H - 1], b[2, 1, H - 1] = 0, 0                       # (of an empty head nothing is written)
            assert torch.equal(a, b)
        held = [torch.cat([row_numbers(e, args, i) for i in range(NL * B * H)]) for e in engs]
        assert torch.equal(engs[0].kept_idx.cpu()[held[0]], engs[1].kept_idx.cpu()[held[1]])
        for n in ("k_c", "v_c"):
            assert torch.equal(values(engs[0], dict(args, cache_fp8=4), n)[held[0]], values(engs[1], args, n)[held[1]])
    for e in engs:
        e.close()
