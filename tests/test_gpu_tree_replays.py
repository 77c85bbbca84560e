"""GPU: ordinary decode steps behind replays of a captured tree commit, whose rows the host has not counted."""
import pytest
import torch

from paper_2506_15724_amd import binding as MB
from tests.test_gpu_operators import KINDS, row_numbers, values
from tests.test_gpu_tree import DEV, nodes

pytestmark = pytest.mark.gpu


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def evict(eng, args, seed, lens):
    """Heads of these lengths, by hand-made budgets."""
    c = eng.cfg
    g = torch.Generator(device=DEV).manual_seed(seed)
    k, v = (torch.randn(1, c.batch, c.n_kv_heads, c.ctx_len, c.head_dim, generator=g, device=DEV).to(eng.tdtype) for _ in range(2))
    bud = torch.zeros(1, c.batch, c.n_kv_heads, 2, dtype=torch.int32, device=DEV)
    bud[..., 0] = i32(*lens).view(1, c.batch, c.n_kv_heads) - c.window
    eng.select_gather(0, 1, k, v, torch.zeros(c.batch, c.ctx_len, dtype=torch.uint8, device=DEV),
                      psi_pool=torch.rand(1, c.batch, c.n_kv_heads, c.ctx_len - c.window, generator=g, device=DEV), budgets=bud)
    torch.cuda.synchronize()
    assert eng.kv_len.view(-1).tolist() == list(lens)


def pair(Hq, H, d, P, lens, max_new, kind):
    args = dict(n_layers=1, batch=1, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=1500, window=8, budget=-(-sum(lens) // H), max_new_tokens=max_new, page_rows=P, **KINDS[kind])
    return [MB.MadaKV(device=DEV, **args) for _ in range(2)], args


def captured_commit(eng, T, max_new):
    """(graph, k, v, path, n, start): one commit of up to T nodes behind the rows so far, captured and not yet run."""
    _, k, v = nodes(eng, T, 0)
    path, n, start = torch.zeros(1, T, dtype=torch.int32, device=DEV), i32(0), i32(0)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        eng.tree_commit(0, 1, k, v, path, n, start, max_new)
        start.add_(n)
    return graph, k, v, path, n, start


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("Hq,H,d,P", [(2, 2, 64, 0), (8, 2, 128, 0), (6, 2, 64, 16)])
def test_decode_behind_replayed_commits(Hq, H, d, P, kind):
    """A new eviction since the capture, its lengths known to the host, then 500 rows by replays: outputs, lengths and rows as where ordinary
    commits have stored them."""
    print(f"[tree_replays] {Hq}/{H} d={d} P={P} {kind}", flush=True)
    lens, max_new, T = [190, 120], 600, 50
    (eng, ref), args = pair(Hq, H, d, P, lens, max_new, kind)
    for e in (eng, ref):
        evict(e, args, 1, lens)
    graph, k, v, path, n, start = captured_commit(eng, T, max_new)
    for e in (eng, ref):
        evict(e, args, 2, lens[::-1])
    have = 0
    for i in range(10):
        for x, y in zip((k, v), nodes(eng, T, 30 + i)[1:]):
            x.copy_(y)
        path.copy_(torch.randperm(T, generator=torch.Generator().manual_seed(i)))
        n.fill_(T)
        torch.cuda.synchronize()
        graph.replay()
        ref.tree_commit(0, 1, k, v, path, n, i32(have), have + T)
        have += T
        torch.cuda.synchronize()
    assert torch.equal(eng.kv_len, ref.kv_len) and eng.kv_len.view(-1).tolist() == [x + have for x in lens[::-1]]
    for i in range(3):
        x = [y[:, :, :, 0].contiguous() for y in nodes(eng, 1, 90 + i)]
        got, want = (torch.full(x[0].shape, -77.0, device=DEV) for _ in range(2))
        eng.decode_attn(0, 1, *x, got)
        ref.decode_attn(0, 1, *x, want)
        torch.cuda.synchronize()
        assert torch.isfinite(want).all() and torch.equal(got, want)
    assert torch.equal(eng.kv_len, ref.kv_len) and eng.kv_len.view(-1).tolist() == [x + have + 3 for x in lens[::-1]]
    for h in range(H):
        a, b = row_numbers(eng, args, h), row_numbers(ref, args, h)
        for w in ("k_c", "v_c"):
            assert torch.equal(values(eng, args, w)[a], values(ref, args, w)[b])
    del graph
    for e in (eng, ref):
        e.close()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("kind,Hq,H,d,P", [("bf16", 2, 2, 128, 0), ("bf16", 8, 2, 64, 16), ("fp32", 2, 2, 64, 0), ("fp8", 2, 2, 128, 16), ("fp8", 6, 2, 128, 0), ("fp4", 2, 2, 64, 0), ("fp4", 8, 2, 128, 32)])
def test_steps_behind_replays_end_where_the_segments_do(kind, Hq, H, d, P, weights):
    """Replays of a captured commit fill the room but for two rows, of which the host knows nothing: it goes on accepting steps, which store what
    there is room for and attend over the rows there are; nothing else in the cache changes."""
    print(f"[tree_replays] room {kind} {Hq}/{H} d={d} P={P} weights={weights}", flush=True)
    lens, max_new, T = [100, 61], 34, 32
    (eng, ref), args = pair(Hq, H, d, P, lens, max_new, kind)
    for e in (eng, ref):
        for x in (e.k_c, e.v_c):
            x.zero_()
        evict(e, args, 1, lens)
    graph, k, v, path, n, start = captured_commit(eng, T, max_new)
    for e in (eng, ref):
        evict(e, args, 2, lens)
    path.copy_(torch.arange(T))
    n.fill_(T)
    torch.cuda.synchronize()
    graph.replay()
    ref.tree_commit(0, 1, k, v, path, n, i32(0), T)
    torch.cuda.synchronize()
    acc = torch.zeros(eng.capacity, device=DEV)

    def step(e, x, new=True):
        out = torch.full(x[0].shape, -77.0, device=DEV)
        if weights:
            e.decode_attn_weights(0, 1, x[0], *(x[1:] if new else (None, None)), out, acc, acc)
        else:
            e.decode_attn(0, 1, x[0], *(x[1:] if new else (None, None)), out)
        torch.cuda.synchronize()
        return out
    for i in range(12):
        x = [y[:, :, :, 0].contiguous() for y in nodes(eng, 1, 90 + i)]
        got, want = step(eng, x), step(ref, x, i < 2)
        assert torch.isfinite(want).all() and torch.equal(got, want), i
        assert torch.equal(eng.kv_len, ref.kv_len) and eng.kv_len.view(-1).tolist() == [x + min(T + i + 1, max_new) for x in lens]
    for h in range(H):
        a, b = row_numbers(eng, args, h), row_numbers(ref, args, h)
        for w in ("k_c", "v_c"):
            assert torch.equal(values(eng, args, w)[a], values(ref, args, w)[b])
    if not P:                                            # (pages are taken in the order in which heads come)
        assert torch.equal(eng.k_c, ref.k_c) and torch.equal(eng.v_c, ref.v_c)
    del graph
    for e in (eng, ref):
        e.close()
