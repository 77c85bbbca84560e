"""GPU: the binding's functions of the C calls' names, on buffers of their own, against the holder's methods, which call the library
with argument lists of their own: the same bits from both."""
import pytest
import torch

from paper_2506_15724_amd import binding as MB
from tests.test_gpu_operators import DEV, KINDS, make, prompt_case, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["fp4", "fp8", "bf16"])
def test_step_and_rows(kind):
    """A replacing step over the second of two layers, with everything that can be given, and the rows behind it."""
    kw = dict(n_layers=2, batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, ctx_len=300, **KINDS[kind])
    a, b = (make([70, 110, 40, 140] * 2, **kw)[0] for _ in range(2))
    g = torch.Generator().manual_seed(4)
    q, kn, vn = (torch.randn(1, 2, h, 64, generator=g).to(DEV, torch.bfloat16) for h in (4, 2, 2))
    acc = torch.rand(a.capacity, generator=g).to(DEV)
    slot, pos = torch.tensor([3, 109, -1, 139], dtype=torch.int32, device=DEV), torch.tensor([300, 310], dtype=torch.int32, device=DEV)
    got = []
    for eng, method in ((a, True), (b, False)):
        out, acc_out, slot_out = torch.zeros(1, 2, 4, 64, device=DEV), torch.full_like(acc, -5.0), torch.full_like(slot, -9)
        rows = [torch.full((eng.capacity, 64), 77.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        say(f"{kind}: {'methods' if method else 'functions'}")
        if method:
            eng.decode_attn_weights(1, 1, q, kn, vn, out, acc, acc_out, decay=0.5, slot_in=slot, slot_out=slot_out, pos=pos, recent=5)
            if kind != "bf16":
                eng.cache_rows(1, 1, *rows)
        else:
            ws = torch.empty(MB.madakv_decode_attn_weights_workspace_bytes(eng.h, 1), dtype=torch.uint8, device=DEV)
            off, ln = eng.kv_off[1:], eng.kv_len[1:]
            MB.madakv_decode_attn_weights(eng.h, 1, 1, q, kn, vn, eng.k_c, eng.v_c, off, ln, out, acc, acc_out, 0.5, slot, slot_out, eng.kept_idx, pos, 5, ws)
            if kind != "bf16":
                MB.madakv_cache_rows(eng.h, 1, 1, eng.k_c, eng.v_c, off, ln, *rows)
            else:
                with pytest.raises(MB.MadaKVError) as e:
                    MB.madakv_cache_rows(eng.h, 1, 1, eng.k_c, eng.v_c, off, ln, *rows)
                assert e.value.status == -7
        torch.cuda.synchronize()
        got.append([out, acc_out, slot_out, *rows])
    assert all(torch.equal(x, y) for x, y in zip(*got))
    held = torch.cat([torch.arange(o, o + n) for o, n in zip(a.kv_off.view(-1).tolist(), a.kv_len.view(-1).tolist())]).to(DEV)
    assert torch.equal(a.kept_idx[held], b.kept_idx[held]) and torch.equal(a.kv_len, b.kv_len)
    assert (got[0][1] != -5.0).sum() == int(a.kv_len[1].sum()) and not (got[0][2] == -9).any()
    a.close(), b.close()


@pytest.mark.parametrize("L", [200, 700])
@pytest.mark.parametrize("stats,given", [(False, False), (True, True)])
def test_prompt_scores(L, stats, given):
    eng, q, k = prompt_case(2, 2, 4, 2, 64, L, W=8)
    mask = torch.randint(0, 2, (2, L), generator=torch.Generator().manual_seed(1)).to(DEV, torch.uint8) if stats else None
    lse = torch.rand(1, 2, 4, L, generator=torch.Generator().manual_seed(2)).to(DEV) + 8.0 if given else None
    q, k = q[1:].contiguous(), k[1:].contiguous()
    say(f"prompt scores L={L} stats={stats} lse={given}")
    eng.score_prompt(1, 1, q, k, mask=mask, row_lse=lse)
    ws = torch.empty(MB.madakv_score_prompt_workspace_bytes(eng.h, 1), dtype=torch.uint8, device=DEV)
    names = ["psi"] + (["psi_pool", "stats", "n_mod"] if stats else [])
    mine = [torch.zeros_like(getattr(eng, n) if n == "n_mod" else getattr(eng, n)[1:]) for n in names]
    MB.madakv_score_prompt(eng.h, 1, 1, q, k, mask, lse, *(mine + [None] * 3)[:4], ws)
    torch.cuda.synchronize()
    for n, x in zip(names, mine):
        y = getattr(eng, n) if n == "n_mod" else getattr(eng, n)[1:]
        assert x.any() and torch.equal(x, y), n
    eng.close()
