"""What the holder refuses of the arrays of prompt attention and of drafted trees before the library is called: arrays kept for more rows
per head than the call has.  No GPU: a holder without a handle, on host tensors, whose library only counts its calls."""
import pytest
import torch

from paper_2506_15724_amd import binding as MB
from tests.test_abi import good

N, B, HQ, H, D, L, T = 2, 3, 4, 2, 64, 20, 5
BF = torch.bfloat16


@pytest.fixture
def holder(monkeypatch):
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append((name, args)) or 0

    class Device:
        index = -1                                      # (what a host tensor's get_device() says)

        def __eq__(self, other): return other == torch.device("cpu")
        def __ne__(self, other): return not self == other

    def make(batch=B):
        eng = MB.MadaKV.__new__(MB.MadaKV)
        eng.cfg = good(n_layers=N, batch=batch, n_q_heads=HQ, n_kv_heads=H, head_dim=D, ctx_len=L)
        eng.h, eng.tdtype, eng._out_dtype, eng._device, eng.device, eng.n_call = None, BF, torch.float32, Device(), torch.device("cpu"), N
        eng._out_row, eng._heads, eng._kv_row, eng._ctx, eng._batch, eng._tree_ws = batch * HQ * D, batch * H, batch * H * D, L, batch, {}
        eng.k_c = eng.v_c = torch.zeros(16, dtype=torch.uint8)
        eng.kv_off, eng.kv_len = torch.zeros(N, batch, H, dtype=torch.int64), torch.zeros(N, batch, H, dtype=torch.int32)
        return eng
    monkeypatch.setattr(MB, "lib", lambda one=Library(): one)
    monkeypatch.setattr(MB, "madakv_tree_attn_workspace_bytes", lambda h, n, t: 16)
    monkeypatch.setattr(MB.MadaKV, "_own_stream", lambda self: 0)
    return make, calls


def arrays(batch, rows, names, n=N):
    heads = dict(q=HQ, out=HQ, k=H, v=H, k_new=H, v_new=H)
    return {x: torch.zeros(n, batch, heads[x], rows, D, dtype=torch.float32 if x == "out" else BF) for x in names}


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def calls_of(eng, batch):
    """name -> (arrays per row, the call)"""
    tree = torch.zeros(batch, T, dtype=torch.int64)
    return {"tree_attn": (T, ("q", "k_new", "v_new", "out"), lambda x, tree=tree: eng.tree_attn(0, N, **{"tree": tree, **x})),
            "tree_commit": (T, ("k_new", "v_new"), lambda x: eng.tree_commit(0, N, path=i32(batch, 3), n_path=i32(batch), start=i32(batch), most=3, **x)),
            "prompt_attn": (L, ("q", "k", "v", "out"), lambda x: eng.prompt_attn(0, N, **x))}


@pytest.mark.parametrize("batch", [1, B])
@pytest.mark.parametrize("call", ["tree_attn", "tree_commit", "prompt_attn"])
def test_rows_per_head_that_differ(holder, call, batch):
    """Each array in turn with more and with twice as many rows; all in step, more layers and flat arrays are taken."""
    make, calls = holder
    eng = make(batch)
    rows, names, run = calls_of(eng, batch)[call]
    good_ = arrays(batch, rows, names)
    run(good_)
    run(arrays(batch, rows, names, N + 1))
    run({x: y if x in ("q", "k_new") else y.view(-1) for x, y in good_.items()} if call != "prompt_attn" else {x: y.view(-1) for x, y in good_.items()})
    assert len(calls) == 3
    for x in names:
        if call != "prompt_attn" and x == names[0]:
            continue                                     # (the nodes are counted in it)
        for more in (rows + 1, 2 * rows):
            with pytest.raises(ValueError, match=str(rows)):
                run({**good_, **arrays(batch, more, (x,))})
    if call != "prompt_attn":
        with pytest.raises(ValueError):
            run({**good_, **arrays(batch, T - 1, names[:1])})
    assert len(calls) == 3


def test_masks_of_more_nodes(holder):
    """[B, 64] masks for fewer nodes: item 1's are not behind item 0's; of one item they are in place."""
    make, calls = holder
    for batch in (1, 2, B):
        eng = make(batch)
        _, names, run = calls_of(eng, batch)["tree_attn"]
        x = arrays(batch, T, names)
        for bad in (torch.zeros(batch, 64, dtype=torch.int64), torch.zeros(batch, T + 1, dtype=torch.int64)):
            if batch == 1:
                run({**x, "tree": bad})
                continue
            n = len(calls)
            with pytest.raises(ValueError, match="tree"):
                run({**x, "tree": bad})
            assert len(calls) == n
        run({**x, "tree": torch.zeros(batch * T, dtype=torch.int64)})
        run({**x, "tree": torch.zeros(batch + 1, T, dtype=torch.int64)})
