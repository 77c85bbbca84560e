"""GPU: attention of a drafted tree gives the same bits whatever the host knows of the lengths, in ordinary and in captured calls."""
import pytest
import torch

from paper_2506_15724_amd import binding as MB
from tests.test_gpu_operators import KINDS
from tests.test_gpu_tree import DEV, nodes, some_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("B,H,Hq,d,L,budget,T,P", [(4, 32, 32, 128, 4096, 2048, 8, 0), (2, 2, 8, 64, 6000, 3000, 13, 16), (1, 2, 8, 128, 9000, 9000, 50, 0), (1, 8, 8, 64, 300, 256, 5, 0)])
def test_same_bits_with_lengths_unknown_known_and_captured(B, H, Hq, d, L, budget, T, P, kind):
    """Even heads of a cache that has been cut: the first call comes while the eviction may still be running, a captured one does not ask."""
    print(f"[tree_bits] B={B} {Hq}/{H} d={d} L={L} budget={budget} T={T} P={P} {kind}", flush=True)
    eng = MB.MadaKV(n_layers=1, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=8, budget=budget, max_new_tokens=200, page_rows=P, device=DEV, **KINDS[kind])
    g = torch.Generator(device=DEV).manual_seed(5)
    k, v = (torch.randn(1, B, H, L, d, generator=g, device=DEV).to(eng.tdtype) for _ in range(2))
    mask, pool = torch.zeros(B, L, dtype=torch.uint8, device=DEV), torch.rand(1, B, H, L - 8, generator=g, device=DEV)
    bud = torch.zeros(1, B, H, 2, dtype=torch.int32, device=DEV)
    bud[..., 0] = budget - 8
    x, tree = nodes(eng, T, 3), some_tree(B, T, 4)
    out = [torch.full(x[0].shape, -77.0, dtype=eng._out_dtype, device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    eng.select_gather(0, 1, k, v, mask, psi_pool=pool, budgets=bud)
    eng.tree_attn(0, 1, *x, tree, out[0])
    torch.cuda.synchronize()
    assert eng.kv_len.view(-1).tolist() == [budget] * (B * H)
    eng.tree_attn(0, 1, *x, tree, out[1])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        eng.tree_attn(0, 1, *x, tree, out[2])
    for _ in range(3):
        out[2].fill_(-77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eng.tree_attn(0, 1, *x, tree, out[3])
        torch.cuda.synchronize()
        assert torch.isfinite(out[1]).all()
        for o in (out[0], out[2], out[3]):
            assert torch.equal(o, out[1])
    del graph
    eng.close()
