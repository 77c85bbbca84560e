"""GPU: a captured step that appends a row, replayed; what the calls behind the replays make of rows that the host has not counted."""
import pytest
import torch

from paper_2506_15724_amd import binding as MB
from tests.test_gpu_operators import DEV, make, row_numbers, say, values

pytestmark = pytest.mark.gpu


def captured_append(eng, args, weights=False):
    """(graph, static inputs, step): one appending step over all layers, captured and not yet run."""
    NL, B, Hq, H, d = (args[x] for x in ("n_layers", "batch", "n_q_heads", "n_kv_heads", "head_dim"))
    x = [torch.zeros(NL, B, h, d, dtype=torch.bfloat16, device=DEV) for h in (Hq, H, H)]
    out, acc = torch.zeros(NL, B, Hq, d, device=DEV), torch.zeros(eng.capacity, device=DEV)
    step = (lambda: eng.decode_attn_weights(0, NL, *x, out, acc, acc)) if weights else (lambda: eng.decode_attn(0, NL, *x, out))
    if weights:
        eng.decode_attn_weights(0, NL, x[0], None, None, out, acc, acc)            # (the holder makes its workspace)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()

    def replay(times, g):
        for _ in range(times):
            for t in x:
                t.copy_(torch.randn(t.shape, generator=g).to(DEV, torch.bfloat16))
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                graph.replay()
            torch.cuda.synchronize()
    return graph, x, out, replay


@pytest.mark.parametrize("kind,P,weights", [(4, 0, False), (4, 16, True), (1, 0, True), (1, 64, False)])
def test_rows_read_back_after_replayed_appends(kind, P, weights):
    """Every row that the heads hold, past the 64-row blocks that the rows counted on the host would fill; nothing else is written."""
    lens = [61, 40, 62]
    eng, args, *_ = make(lens, n_q_heads=6, n_kv_heads=3, head_dim=64, ctx_len=300, max_new_tokens=80, cache_fp8=kind, page_rows=P)
    graph, x, out, replay = captured_append(eng, args, weights)
    say(f"rows back, kind {kind} P={P} weights={weights}")
    replay(70, torch.Generator().manual_seed(P + kind))
    assert eng.kv_len.view(-1).tolist() == [n + 70 for n in lens]
    back = [torch.full((eng.capacity, 64), 77.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    eng.cache_rows(0, 1, *back)
    torch.cuda.synchronize()
    held = torch.cat([row_numbers(eng, args, i) for i in range(3)])
    rest = torch.ones(eng.capacity, dtype=torch.bool)
    rest[held] = False
    for name, rows in (("k_c", back[0]), ("v_c", back[1])):
        assert torch.equal(rows.cpu().double()[held], values(eng, args, name)[held])
        assert (rows.cpu()[rest] == 77.0).all()
    del graph
    eng.close()


@pytest.mark.parametrize("kw,weights", [(dict(), False), (dict(cache_fp8=4), True), (dict(cache_fp8=1, page_rows=16), False), (dict(cache_fp8=4, page_rows=16), False),
                                        (dict(page_rows=64), True)])
def test_reeviction_after_replayed_appends(kw, weights):
    """Twice, 30 and 17 replays of a captured step in front of it: lengths, budgets, positions and rows as after the same steps taken
    by calls, and the eager steps behind it give the same outputs."""
    NL, B, Hq, H, d, L, W, T = 2, 2, 4, 2, 64, 500, 8, 40
    args = dict(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, page_rows=kw.get("page_rows", 0), cache_fp8=kw.get("cache_fp8", 0))
    g = torch.Generator(device=DEV).manual_seed(L)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)        # noqa: E731
    q, k, v = randn(NL, B, Hq, W, d), randn(NL, B, H, L, d), randn(NL, B, H, L, d)
    mask = torch.randint(0, 2, (B, L), generator=g, device=DEV).to(torch.uint8)
    eager, graphed = (MB.MadaKV(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=W, budget=100, max_new_tokens=T, device=DEV, **kw) for _ in range(2))
    for e in (eager, graphed):
        e.kept_idx.zero_()                              # (a position nobody has written reads as one)
        e.evict(0, NL, q, k, v, mask)
    len0 = eager.kv_len.clone()
    graph, x, out, replay = captured_append(graphed, args, weights)
    out_e = torch.zeros_like(out)
    for round_, times in enumerate((30, 17)):
        for i in range(times):
            replay(1, torch.Generator().manual_seed(100 * round_ + i))
            eager.decode_attn(0, NL, *x, out_e)
        torch.cuda.synchronize()
        recent = randn(NL, B, Hq, W, d)
        say(f"re-eviction after {times} replays {kw} weights={weights}")
        assert torch.equal(graphed.kv_len, len0 + times)
        for e in (eager, graphed):
            e.reevict(0, NL, recent, mask)
        torch.cuda.synchronize()
        for e in (eager, graphed):
            assert torch.equal(e.kv_len, len0)
        assert torch.equal(eager.budgets, graphed.budgets)
        for i in range(NL * B * H):
            a, b = row_numbers(eager, args, i), row_numbers(graphed, args, i)
            pos = eager.kept_idx.cpu()[a]
            assert torch.equal(pos, graphed.kept_idx.cpu()[b])
            assert (pos[1:] > pos[:-1]).all() and int(pos[-1]) == L + (30, 47)[round_] - 1         # (the newest token is always kept)
            for name in ("k_c", "v_c"):
                assert torch.equal(values(eager, args, name)[a], values(graphed, args, name)[b])
        for step in range(2):
            y = randn(NL, B, Hq, d), randn(NL, B, H, d), randn(NL, B, H, d)
            outs = [torch.zeros(NL, B, Hq, d, device=DEV) for _ in range(2)]
            for e, o in zip((eager, graphed), outs):
                e.decode_attn(0, NL, y[0], None, None, o)
            torch.cuda.synchronize()
            assert torch.isfinite(outs[0]).all() and torch.equal(*outs)
    del graph
    eager.close(), graphed.close()
