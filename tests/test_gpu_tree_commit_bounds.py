"""GPU: tree commits whose rows begin beyond the bound of the call."""
import pytest
import torch

from tests.test_gpu_operators import KINDS, make
from tests.test_gpu_tree import DEV, nodes

pytestmark = pytest.mark.gpu


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("P", [0, 16])
def test_start_beyond_the_bound(kind, P):
    """Segments are cut to `most` rows behind those of the eviction also where `start` names a row past it (of which the host does not count
    more than `most`); rows of a paged cache stay, and none is stored."""
    print(f"[tree_commit_bounds] {kind} P={P}", flush=True)
    eng, args, *_ = make(None, batch=4, n_q_heads=2, n_kv_heads=2, head_dim=64, ctx_len=40, max_new_tokens=30, page_rows=P, **KINDS[kind])
    _, k, v = nodes(eng, 9, 1)
    path = torch.arange(9, dtype=torch.int32, device=DEV).expand(4, 9).contiguous()
    for x in (eng.k_c, eng.v_c):
        x.zero_()
    eng.tree_commit(0, 1, k, v, path, i32(9, 9, 9, 9), i32(0, 0, 0, 0), 9)
    before = [x.view(torch.uint8).clone() for x in (eng.k_c, eng.v_c)]
    #           at the bound, past it, past it and at the end, behind the end
    eng.tree_commit(0, 1, k, v, path, i32(9, 9, 0, 9), i32(4, 5, 9, 12), 4)
    torch.cuda.synchronize()
    have = 9 if P else 4
    assert (eng.kv_len == 40 + have).all(), eng.kv_len
    assert all(torch.equal(x.view(torch.uint8), y) for x, y in zip((eng.k_c, eng.v_c), before))
    # and the room behind them is the room that the host counts
    q, kn, vn = (x[:, :, :, 0].contiguous() for x in nodes(eng, 1, 2))
    for _ in range(30 - have):
        eng.decode_attn(0, 1, q, kn, vn, torch.empty(1, 4, 2, 64, device=DEV))
    torch.cuda.synchronize()
    assert (eng.kv_len == 70).all(), eng.kv_len
