"""GPU: a captured step that appends a row, replayed; what the calls behind the replays make of rows that the host has not counted."""
import pytest
import torch

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
