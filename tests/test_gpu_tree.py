"""GPU: attention of drafted trees over the reduced cache, and their accepted nodes in it, against plain arithmetic in 64 bits and against
decoding token by token: every kind of cache, one to 64 nodes, heads of all lengths, masks that name nothing, rows taken back, graphs."""
import math

import numpy as np
import pytest
import torch

from paper_2506_15724_amd import binding as MB
from tests.test_gpu_operators import KINDS, make, row_numbers, stored, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(msg):
    print(f"[tree] {msg}", flush=True)


def nodes(eng, T, seed=0):
    c = eng.cfg
    g = torch.Generator().manual_seed(seed)
    q, k, v = ((1.5 if h == c.n_q_heads and i == 0 else 1.0) * torch.randn(c.n_layers, c.batch, h, T, c.head_dim, generator=g)
               for i, h in enumerate((c.n_q_heads, c.n_kv_heads, c.n_kv_heads)))
    return [x.to(DEV, eng.tdtype) for x in (q, k, v)]


def some_tree(B, T, seed, how="tree"):
    """int64 [B, T] masks"""
    r = np.random.default_rng(seed)
    m = np.zeros((B, T), np.uint64)
    for b in range(B):
        for t in range(T):
            if how == "chain":
                m[b, t] = (2 << t) - 1 if t < 63 else 0xffffffffffffffff
            elif how == "any":                                    # whatever bits, those past the last node too; some none
                m[b, t] = 0 if r.random() < 0.3 else r.integers(0, 1 << 63, dtype=np.uint64) * np.uint64(2) + np.uint64(1)
            else:
                p = int(r.integers(-1, t)) if t else -1
                m[b, t] = (m[b, p] if p >= 0 else np.uint64(0)) | np.uint64(1 << t)
    return torch.from_numpy(m.view(np.int64)).to(DEV)


def kind_of(args):
    return args.get("cache_fp8", 0)


def check(eng, args, q, k_new, v_new, tree, out):
    c = eng.cfg
    G, T, d, u = c.n_q_heads // c.n_kv_heads, q.shape[3], c.head_dim, 2.0 ** -24
    kc, vc = values(eng, args, "k_c"), values(eng, args, "v_c")
    masks = tree.cpu().numpy().view(np.uint64)
    heads = [(l, b, h) for l in range(c.n_layers) for b in range(c.batch) for h in range(c.n_kv_heads)]
    lens = eng.kv_len.view(-1).tolist()
    for i, (l, b, h) in enumerate(heads):
        got = out[l, b, h * G:(h + 1) * G].cpu().double()
        if lens[i] == 0:
            assert not torch.isfinite(got).any()
            continue
        at = row_numbers(eng, args, i)
        new = [stored(x[l, b, h], kind_of(args)).double() for x in (k_new, v_new)]
        k, v = torch.cat([kc[at].double(), new[0]]), torch.cat([vc[at].double(), new[1]])
        sees = torch.tensor([[bool(int(m) >> j & 1) for j in range(T)] for m in masks[b]])
        may = torch.cat([torch.ones(T, len(at), dtype=torch.bool), sees], 1)
        qq = q[l, b, h * G:(h + 1) * G].cpu().double()
        s = (qq @ k.T / math.sqrt(d)).masked_fill(~may, -math.inf)
        size = float((qq.abs() @ k.abs().T).max()) / math.sqrt(d)
        w = torch.softmax(s, -1)
        ref, spent = w @ v, w @ v.abs()
        # as in prompt attention: d + 2 roundings of a logit, twice; sums over the rows, the merges of pieces and halves
        rel = 2 * (d + 2) * u * size + 2 * (len(at) + T + 32) * u
        tol = rel * spent + 1e-30
        if out.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * (1 + rel) * spent + 2.0 ** -8 * (ref.abs() + tol)
        err = (got - ref).abs()
        assert bool((err <= tol).all()), (l, b, h, float((err / tol).max()), (err > tol).nonzero()[:5].tolist())


def attend(eng, q, k_new, v_new, tree, l0=0):
    out = torch.full(q.shape, -77.0, dtype=eng._out_dtype, device=DEV)
    eng.tree_attn(l0, q.shape[0], q, k_new, v_new, tree, out)
    torch.cuda.synchronize()
    return out


CASES = [(1, [9, 64, 171], 128, 3, 0), (2, [65, 63], 64, 4, 0), (5, [200, 8, 9, 16, 300], 64, 5, 0), (7, [33, 31], 128, 2, 16), (16, [100, 64], 64, 14, 64), (17, [121, 128, 250], 128, 6, 0),
         (33, [40, 500], 128, 2, 0), (64, [63, 65], 64, 16, 0), (64, [1000, 100], 128, 14, 0), (31, [300, 17], 128, 16, 32), (3, [48, 16], 64, 2, 16), (64, [129], 128, 8, 0), (40, [77, 50, 9], 64, 9, 0)]


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("T,lens,d,Hq,P", CASES)
def test_attention(T, lens, d, Hq, P, kind):
    for out_fp32 in (1,) if kind == "fp32" else (1, 0):
        say(f"T={T} lens={lens} d={d} Hq={Hq} P={P} {kind} out_fp32={out_fp32}")
        if kind == "fp32" and Hq // len(lens) * 8 * d > 12288:
            pytest.skip("the configuration is refused")
        eng, args, *_ = make(lens, n_q_heads=Hq, n_kv_heads=len(lens), head_dim=d, ctx_len=max(lens) + 100, page_rows=P, out_fp32=out_fp32, **KINDS[kind])
        q, k, v = nodes(eng, T, T)
        for how in ("tree", "any", "chain"):
            tree = some_tree(1, T, T, how)
            bits = lambda: [x.view(torch.uint8).clone() for x in (eng.k_c, eng.v_c, eng.kv_len)]      # noqa: E731  (free rows may hold anything)
            before = bits()
            out = attend(eng, q, k, v, tree)
            check(eng, args, q, k, v, tree, out)
            assert all(torch.equal(x, y) for x, y in zip(before, bits()))
            assert torch.equal(out, attend(eng, q, k, v, tree)), "the same twice"


WIDE = [(33, [40, 500], 128, 4, 0), (64, [63, 65], 64, 16, 0), (64, [1000, 100], 128, 14, 0), (31, [300, 17], 128, 16, 32), (13, [700], 128, 7, 16), (40, [77, 50, 9], 64, 9, 0),
        (25, [8, 64, 128, 640], 128, 12, 0), (43, [900, 33], 64, 6, 64), (64, [31, 2000], 128, 16, 0)]


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4", "fp32"])
@pytest.mark.parametrize("T,lens,d,Hq,P", WIDE)
def test_attention_of_many_columns(T, lens, d, Hq, P, kind):
    """Caches with room for so many rows that launches take the kernel for many columns."""
    for out_fp32 in (1,) if kind == "fp32" else (1, 0):
        say(f"many columns T={T} lens={lens} d={d} Hq={Hq} P={P} {kind} out_fp32={out_fp32}")
        L = (1 << 23) // (Hq * T) + 1016
        eng, args, *_ = make(lens, n_q_heads=Hq, n_kv_heads=len(lens), head_dim=d, ctx_len=L, budget=L - 16, page_rows=P, out_fp32=out_fp32, **KINDS[kind])
        q, k, v = nodes(eng, T, T)
        for how in ("tree", "any", "chain"):
            tree = some_tree(1, T, T, how)
            out = attend(eng, q, k, v, tree)
            check(eng, args, q, k, v, tree, out)
            assert torch.equal(out, attend(eng, q, k, v, tree)), "the same twice"


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("B,NL,H,Hq,d,L,T", [(2, 3, 4, 8, 64, 300, 9), (4, 2, 32, 32, 128, 257, 6), (1, 1, 2, 14, 128, 5000, 20), (3, 1, 1, 8, 64, 2500, 64)])
def test_whole_caches(B, NL, H, Hq, d, L, T, kind):
    """Caches that keep everything: launches of few and of many pieces."""
    say(f"whole B={B} n={NL} {Hq}/{H} d={d} L={L} T={T} {kind}")
    if kind == "fp32" and Hq // H * 8 * d > 12288:
        pytest.skip("the configuration is refused")
    eng, args, *_ = make(None, n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, **KINDS[kind])
    q, k, v = nodes(eng, T, 5)
    tree = some_tree(B, T, 6)
    out = attend(eng, q, k, v, tree)
    check(eng, args, q, k, v, tree, out)
    for l in range(NL):
        one = attend(eng, q[l:l + 1], k[l:l + 1], v[l:l + 1], tree, l0=l)
        assert bool(((one[0] - out[l]).abs() <= 1e-4).all())          # (a launch over fewer layers cuts heads into more pieces)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4", "fp32"])
@pytest.mark.parametrize("P", [0, 16])
def test_token_by_token(kind, P):
    """A tree's outputs are those of decode steps along its branches; its accepted rows are those that the steps append."""
    say(f"token by token {kind} P={P}")
    kw = dict(n_q_heads=4, n_kv_heads=2, head_dim=64, ctx_len=200, page_rows=P, max_new_tokens=40, **KINDS[kind])
    (eng, args, *_), (one, *_) = make([60, 47], **kw), make([60, 47], **kw)
    T = 12
    q, k, v = nodes(eng, T, 3)
    parents = [-1, 0, 0, 1, 3, 2, 4, 5, 6, 6, 8, 10]
    masks = []
    for t, p in enumerate(parents):
        masks.append((masks[p] if p >= 0 else 0) | 1 << t)
    tree = torch.tensor([masks], dtype=torch.int64, device=DEV)
    out = attend(eng, q, k, v, tree)
    path = [0, 1, 3, 4, 6, 8, 10, 11]
    for t in path:
        step = torch.empty(1, 1, 4, 64, device=DEV)
        one.decode_attn(0, 1, *(x[:, :, :, t].contiguous() for x in (q, k, v)), step)
        assert bool(((out[:, :, :, t] - step).abs() <= 2e-5).all())        # (decode of 16-bit and 8-bit rows: weights as two bf16 parts, 2^-17 of each)
    # the same rows, committed in two calls
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)      # noqa: E731
    eng.tree_commit(0, 1, k, v, i32(path[:3]), i32(3), i32(0), 3)
    eng.tree_commit(0, 1, k, v, i32(path[3:]), i32(5), i32(3), 8)
    torch.cuda.synchronize()
    assert torch.equal(eng.kv_len, one.kv_len)
    for h in range(2):
        a, b = row_numbers(eng, args, h), row_numbers(one, args, h)
        for which in ("k_c", "v_c"):
            assert torch.equal(values(eng, args, which)[a], values(one, args, which)[b])
    # and decode goes on from there
    for t in (2, 5):
        got, want = torch.empty(1, 1, 4, 64, device=DEV), torch.empty(1, 1, 4, 64, device=DEV)
        for e, o in ((eng, got), (one, want)):
            e.decode_attn(0, 1, *(x[:, :, :, t].contiguous() for x in (q, k, v)), o)
        assert torch.equal(got, want)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("d", [64, 128])
def test_commit(kind, d):
    """Each batch item its own number of rows, encoded as the cache is; nothing else is written; repeated, taken back, cut, refused."""
    say(f"commit {kind} d={d}")
    B, NL, H, T, most = 4, 2, 3, 9, 20
    eng, args, *_ = make(None, n_layers=NL, batch=B, n_q_heads=H, n_kv_heads=H, head_dim=d, ctx_len=70, max_new_tokens=most, **KINDS[kind])
    for x in (eng.k_c, eng.v_c):
        if x.dtype == torch.uint8:
            x.copy_(torch.randint(0, 120, x.shape, dtype=torch.uint8, device=DEV))          # (any byte is a number)
        else:
            x.copy_(torch.randn(x.shape, device=DEV))
    q, k, v = nodes(eng, T, 4)
    k[0, 0, 0, 0, :8] = torch.tensor([1e6, -1e6, 448, 449, 464, 3e-5, 0.0, -2.5]).to(k)
    r = np.random.default_rng(1)
    have = np.zeros((B,), int)
    free = eng.kv_len[0, 0, 0].item()

    def commit(n, start, bound, bad=()):
        path = r.integers(0, T, (B, T)).astype(np.int32)
        for b, i, x in bad:
            path[b, i] = x
        before = {w: values(eng, args, w).clone() for w in ("k_c", "v_c")}
        eng.tree_commit(0, NL, k, v, torch.from_numpy(path).to(DEV), torch.tensor(n, dtype=torch.int32, device=DEV), torch.tensor(start, dtype=torch.int32, device=DEV), bound)
        torch.cuda.synchronize()
        lens = eng.kv_len.cpu()
        for b in range(B):
            m = max(0, min(n[b], T, bound - start[b]))
            m = min([m] + [i for bb, i, _ in bad if bb == b])
            left = start[b] < 0 or start[b] > have[b]
            have[b] = min(have[b], bound) if left else start[b] + m
            assert (lens[:, b] == free + have[b]).all(), (b, lens[:, b], have[b])
            for l in range(NL):
                for h in range(H):
                    off = int(eng.kv_off[l, b, h]) + free
                    for w, x in (("k_c", k), ("v_c", v)):
                        if not left and m:
                            want = stored(x[l, b, h][torch.from_numpy(path[b, :m]).long().to(DEV)], kind_of(args)).double()
                            before[w][off + start[b]:off + start[b] + m] = want
        for w in before:
            assert torch.equal(values(eng, args, w).double(), before[w].double())

    commit([3, 0, 9, 1], [0, 0, 0, 0], 9)
    commit([3, 0, 9, 1], [0, 0, 0, 0], 9)                      # the same again
    commit([2, 5, 1, 0], [3, 0, 9, 1], 10)
    commit([1, 1, 1, 1], [2, 5, 4, 2], 12)                     # rows taken back; more than there are: left alone
    commit([9, 9, 9, 9], [0, -1, 5, 7], 11)                    # beyond the bound, no such start
    commit([4, 40, -3, 9], [0, 0, 5, 1], 20, bad=[(0, 2, T), (1, 5, -1), (3, 0, 1 << 30)])
    commit([0, 0, 0, 0], [1, 1, 1, 30], 2)                     # cut to the bound
    commit([9, 9, 9, 9], [0, 0, 0, 0], 20)
    commit([9, 9, 9, 9], [9, 9, 9, 9], 20)
    commit([9, 9, 9, 9], [18, 18, 18, 18], 20)


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_commit_encodes_every_value(kind):
    """All 65536 16-bit patterns, infinities and NaN among them: the bytes that decode steps would append."""
    say(f"every value {kind}")
    kw = dict(n_q_heads=8, n_kv_heads=8, head_dim=128, ctx_len=70, max_new_tokens=64, **KINDS[kind])
    (eng, *_), (one, *_) = make(None, **kw), make(None, **kw)
    x = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(torch.bfloat16).view(1, 1, 8, 64, 128).to(DEV)
    y = x.flip(-1).contiguous()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)      # noqa: E731
    eng.tree_commit(0, 1, x, y, i32(list(range(64))), i32(64), i32(0), 64)
    q, out = torch.zeros(1, 1, 8, 1, 128, device=DEV, dtype=torch.bfloat16), torch.zeros(1, 1, 8, 128, device=DEV)
    for t in range(64):
        one.decode_attn(0, 1, q, x[:, :, :, t].contiguous(), y[:, :, :, t].contiguous(), out)
    torch.cuda.synchronize()
    assert torch.equal(eng.kv_len, one.kv_len)
    rows = torch.cat([int(eng.kv_off[0, 0, h]) + torch.arange(134) for h in range(8)])
    size = 64 if kind == "fp4" else 128
    for w in ("k_c", "v_c"):
        a, b = (getattr(e, w).view(torch.uint8).cpu() for e in (eng, one))
        assert torch.equal(a[:eng.capacity * size].view(-1, size)[rows], b[:eng.capacity * size].view(-1, size)[rows])
        if kind == "fp4":
            assert torch.equal(a[eng.capacity * size:].view(-1, 4)[rows], b[eng.capacity * size:].view(-1, 4)[rows])


def test_commit_into_pages():
    say("commit into pages")
    eng, args, *_ = make([33, 40], n_q_heads=2, n_kv_heads=2, head_dim=64, ctx_len=100, page_rows=16, max_new_tokens=60)
    T = 30
    q, k, v = nodes(eng, T, 4)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)      # noqa: E731
    want = [[values(eng, args, w)[row_numbers(eng, args, h)] for h in range(2)] for w in ("k_c", "v_c")]
    have = 0
    r = np.random.default_rng(3)
    for n, start in ((1, 0), (30, 1), (5, 7), (14, 31), (0, 45), (15, 45), (3, 60), (1, 10)):
        path = r.integers(0, T, 30)
        eng.tree_commit(0, 1, k, v, i32(list(path)), i32(n), i32(start), 60)
        torch.cuda.synchronize()
        if start == have:
            m = min(n, 60 - have)
            have += m
            for i, x in enumerate((k, v)):
                want[i] = [torch.cat([want[i][h], x[0, 0, h].cpu()[path[:m]]]) for h in range(2)]
        assert eng.kv_len.view(-1).tolist() == [33 + have, 40 + have]
        for i, w in enumerate(("k_c", "v_c")):
            for h in range(2):
                assert torch.equal(values(eng, args, w)[row_numbers(eng, args, h)], want[i][h])
    tree = some_tree(1, T, 2)
    check(eng, args, q, k, v, tree, attend(eng, q, k, v, tree))
    with pytest.raises(MB.MadaKVError):
        eng.decode_attn(0, 1, q[:, :, :, 0].contiguous(), k[:, :, :, 0].contiguous(), v[:, :, :, 0].contiguous(), torch.empty(1, 1, 2, 64, device=DEV))


@pytest.mark.parametrize("N,L,T,first", [(60, 200, 5, 100), (900, 2500, 20, 1500), (59984, 60000, 40, 59980)])
def test_empty_segments(N, L, T, first):
    """Heads that did not fit the cache stay empty, and their outputs are no numbers."""
    say(f"empty segments {N}")
    eng, args, k0, v0, mask = make([N, N], n_q_heads=8, n_kv_heads=2, head_dim=64, ctx_len=L)
    bud = torch.zeros(1, 1, 2, 2, dtype=torch.int32)
    bud[..., 0] = torch.tensor([first, N])
    eng.select_gather(0, 1, k0, v0, mask, psi_pool=torch.rand(1, 1, 2, L - 8, device=DEV), budgets=bud.to(DEV))
    torch.cuda.synchronize()
    assert eng.kv_len.view(-1).tolist() == [first + 8, 0]
    q, k, v = nodes(eng, T, 1)
    tree = some_tree(1, T, 1)
    check(eng, args, q, k, v, tree, attend(eng, q, k, v, tree))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)      # noqa: E731
    eng.tree_commit(0, 1, k, v, i32([0, 1]), i32(2), i32(0), 4)
    torch.cuda.synchronize()
    assert eng.kv_len.view(-1).tolist() == [first + 10, 0]


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("out_fp32", [0, 1])
@pytest.mark.parametrize("T", [20, 30, 50])
def test_undefined_nodes(kind, out_fp32, T):
    """Nodes that a query does not see may hold anything.  (30, 50: room for so many rows that launches take the kernel for many columns.)"""
    if kind == "fp32" and not out_fp32:
        pytest.skip("32-bit outputs")
    say(f"undefined nodes {kind} {out_fp32} T={T}")
    L = 400 if T == 20 else (1 << 23) // (6 * T) + 1016
    eng, args, *_ = make([60, 300], n_q_heads=6, n_kv_heads=2, head_dim=128, ctx_len=L, budget=180 if T == 20 else L - 16, out_fp32=out_fp32, **KINDS[kind])
    q, k, v = nodes(eng, T, 1)
    tree = some_tree(1, T, 8)
    masks = tree.cpu().numpy().view(np.uint64)[0]
    plain = attend(eng, q, k, v, tree)
    for t, what, which in ((0, math.nan, v), (7, math.inf, v), (13, math.nan, k), (19, math.nan, v)):
        y = which.clone()
        y[:, :, :, t] = what
        out = attend(eng, q, y if which is k else k, y if which is v else v, tree)
        sees = torch.tensor([bool(int(m) >> t & 1) for m in masks], device=DEV)
        a, b = out[:, :, :, ~sees].double(), plain[:, :, :, ~sees].double()
        assert bool(((a - b).abs() <= 2.0 ** (-17 if out_fp32 else -7) * (1 + b.abs())).all()), (t, what)
        assert not torch.isfinite(out[:, :, :, sees]).any()
        if what == math.inf:
            assert (out[:, :, :, sees] == math.inf).all()
    # an infinite row of the cache, the last of its segment: everybody sees it
    eng.v_c[int(eng.kv_off[0, 0, 1]) + 299] = -math.inf
    out = attend(eng, q, k, v, tree)
    assert (out[:, :, 3:] == -math.inf).all() and torch.isfinite(out[:, :, :3]).all()


@pytest.mark.parametrize("P", [0, 32])
def test_captured_speculation(P):
    """A captured step (attention of the tree, then its accepted nodes) replayed while the heads grow by as many rows as the device says."""
    say(f"captured P={P}")
    kw = dict(n_layers=2, batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, ctx_len=100, page_rows=P, max_new_tokens=60)
    (eng, args, *_), (ref, *_) = make(None, **kw), make(None, **kw)
    T = 8
    q, k, v = nodes(eng, T, 0)
    tree = some_tree(2, T, 0)
    path, n_path, start = torch.zeros(2, T, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    out = torch.empty(q.shape, device=DEV)
    eng.tree_attn(0, 2, q, k, v, tree, out)                     # (the workspace)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eng.tree_attn(0, 2, q, k, v, tree, out)
        eng.tree_commit(0, 2, k, v, path, n_path, start, 60)
        start.add_(n_path)
    r = np.random.default_rng(2)
    begun = torch.zeros(2, dtype=torch.int32, device=DEV)
    for i in range(9):
        for x, y in zip((q, k, v), nodes(eng, T, 20 + i)):
            x.copy_(y)
        tree.copy_(some_tree(2, T, 20 + i))
        path.copy_(torch.from_numpy(r.integers(0, T, (2, T))))
        n_path.copy_(torch.from_numpy(r.integers(0, 7, 2)))
        torch.cuda.synchronize()
        want = attend(ref, q, k, v, tree)
        ref.tree_commit(0, 2, k, v, path, n_path, begun, 60)
        begun += n_path
        g.replay()
        torch.cuda.synchronize()
        assert bool(((out - want).abs() <= 1e-5).all()) and torch.equal(eng.kv_len, ref.kv_len), i
        for h in range(8):
            for w in ("k_c", "v_c"):
                assert torch.equal(values(eng, args, w)[row_numbers(eng, args, h)], values(ref, args, w)[row_numbers(ref, args, h)])
    # calls that go by what the heads hold now
    a, b = attend(eng, q, k, v, tree), attend(ref, q, k, v, tree)
    assert bool(((a - b).abs() <= 1e-5).all())


def test_captured_call_keeps_its_workspace():
    say("captured, then larger trees")
    eng, args, *_ = make([1500, 900], n_q_heads=8, n_kv_heads=2, head_dim=128, ctx_len=1600)
    small, large = nodes(eng, 4, 1), nodes(eng, 40, 2)
    tree, wide = some_tree(1, 4, 1), some_tree(1, 40, 2)
    want = attend(eng, *small, tree)
    out = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eng.tree_attn(0, 1, *small, tree, out)
    for _ in range(3):
        check(eng, args, *large, wide, attend(eng, *large, wide))
        taken = [torch.full((1 << 20,), math.nan, device=DEV) for _ in range(32)]          # (freed memory would be these)
        out.fill_(-1)
        g.replay()
        torch.cuda.synchronize()
        assert bool(((out - want).abs() <= 1e-5).all())
        del taken


def test_a_generation():
    """A prompt's attention, its scores by the normalisers, eviction, drafted steps of which each item accepts its own number, re-eviction, decode."""
    say("a generation")
    c = dict(n_layers=2, batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, ctx_len=600, window=16, budget=120, max_new_tokens=30, out_fp32=1)
    eng = MB.MadaKV(device=DEV, **c)
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k, v = (torch.randn(2, 2, h, 600, 64, generator=g, device=DEV).to(torch.bfloat16) for h in (8, 2, 2))
    mask = (torch.arange(600, device=DEV) % 5 < 2).to(torch.uint8).expand(2, 600).contiguous()
    out, lse = torch.empty(q.shape, device=DEV), torch.empty(2, 2, 8, 600, device=DEV)
    eng.prompt_attn(0, 2, q, k, v, out, row_lse=lse)
    eng.score_prompt(0, 2, q, k, mask, row_lse=lse)
    eng.allocate(0, 2)
    eng.select_gather(0, 2, k, v, mask)
    torch.cuda.synchronize()
    kept = eng.kv_len.clone()
    assert int(kept.sum()) == 2 * 2 * 2 * 120
    have = torch.zeros(2, dtype=torch.int32, device=DEV)
    for step in range(4):
        qn, kn, vn = nodes(eng, 7, step)
        tree = some_tree(2, 7, step)
        check(eng, c, qn, kn, vn, tree, attend(eng, qn, kn, vn, tree))
        n = torch.tensor([step + 3, 5 - step], dtype=torch.int32, device=DEV)
        path = torch.stack([torch.randperm(7)[:7].sort().values for _ in range(2)]).int().to(DEV)
        eng.tree_commit(0, 2, kn, vn, path, n, have, 30)
        have += n
        torch.cuda.synchronize()
        assert torch.equal(eng.kv_len, kept + have.view(1, 2, 1))
    recent = torch.randn(2, 2, 8, 16, 64, generator=g, device=DEV).to(torch.bfloat16)
    eng.reevict(0, 2, recent, mask)
    torch.cuda.synchronize()
    assert torch.equal(eng.kv_len, kept)
    off, idx = eng.kv_off.view(-1).tolist(), eng.kept_idx.cpu()
    for i in range(8):                                           # the newest rows are the generated ones, in order, each item its own number
        n = int(have[i // 2 % 2])
        rows = idx[off[i]:off[i] + int(kept.view(-1)[i])]
        assert rows[-16:].tolist() == list(range(600 + n - 16, 600 + n)) and (rows[1:] > rows[:-1]).all()
    qn, kn, vn = nodes(eng, 1, 9)
    step = torch.empty(2, 2, 8, 64, device=DEV)
    tree = some_tree(2, 1, 0)
    want = attend(eng, qn, kn, vn, tree)
    eng.decode_attn(0, 2, qn[:, :, :, 0].contiguous(), kn[:, :, :, 0].contiguous(), vn[:, :, :, 0].contiguous(), step)
    torch.cuda.synchronize()
    assert bool(((step - want[:, :, :, 0]).abs() <= 2e-5).all())


def test_large_cache_rows_beyond_4_gib():
    """Heads whose rows lie past 2^32 bytes of the cache."""
    say("beyond 4 GiB")
    L, H, T = 400000, 48, 3
    eng = MB.MadaKV(n_layers=1, batch=1, n_q_heads=H, n_kv_heads=H, head_dim=128, ctx_len=L, window=8, budget=L, max_new_tokens=8, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    kp, vp = (torch.randn(1, 1, H, L, 128, generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    eng.select_gather(0, 1, kp, vp, torch.zeros(1, L, dtype=torch.uint8, device=DEV))
    q, k, v = nodes(eng, T, 2)
    tree = some_tree(1, T, 1)
    out = attend(eng, q, k, v, tree)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)      # noqa: E731
    eng.tree_commit(0, 1, k, v, i32([2, 0]), i32(2), i32(0), 2)
    torch.cuda.synchronize()
    sees = torch.tensor([[bool(int(m) >> j & 1) for j in range(T)] for m in tree[0].tolist()], device=DEV)
    for h in (0, 20, H - 1):
        off = int(eng.kv_off[0, 0, h])
        assert off * 256 > (1 << 32) or h < H - 1
        kk, vv = (torch.cat([p[0, 0, h], x[0, 0, h]]).double() for p, x in ((kp, k), (vp, v)))
        s = q[0, 0, h].double() @ kk.t().contiguous() / math.sqrt(128)
        s[:, L:].masked_fill_(~sees, -math.inf)
        ref = torch.softmax(s, -1) @ vv
        # logits within 130 roundings of 2^-24 of sums of |q k| of at most 30 (1.5 * 1.1 * 128 / 11.3 * 1.3), twice; sums of 400000 weights and weighted rows in
        # chains of at most 6250 tiles, 32 a tile; |out| and the sums of |w v| below 1
        assert bool(((out[0, 0, h].double() - ref).abs() <= 2 * 130 * 2.0 ** -24 * 30 + 2 * 6282 * 2.0 ** -24).all())
        for c, x in ((eng.k_c, k), (eng.v_c, v)):
            assert torch.equal(c[off + L:off + L + 2], x[0, 0, h][[2, 0]]) and torch.equal(c[off + L - 1], (kp if x is k else vp)[0, 0, h, L - 1])


def test_holder_refuses():
    say("refusals")
    eng, *_ = make([60, 47], n_q_heads=4, n_kv_heads=2, head_dim=64, ctx_len=200)
    q, k, v = nodes(eng, 6, 3)
    out = torch.zeros(q.shape, device=DEV)
    tree = some_tree(1, 6, 1)
    good = dict(q=q, k_new=k, v_new=v, tree=tree, out=out)
    for bad in (dict(q=q.float()), dict(q=q[0]), dict(k_new=k[:, :, :, :5]), dict(v_new=v.cpu()), dict(tree=tree.int()), dict(tree=tree[:, :4]), dict(out=out.to(torch.bfloat16)), dict(out=out[..., :8])):
        with pytest.raises((ValueError, AssertionError)):
            eng.tree_attn(0, 1, **{**good, **bad})
    big = nodes(eng, 65, 0)
    with pytest.raises(MB.MadaKVError):
        eng.tree_attn(0, 1, *big, torch.zeros(1, 65, dtype=torch.int64, device=DEV), torch.zeros(big[0].shape, device=DEV))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)      # noqa: E731
    good = dict(k_new=k, v_new=v, path=i32([0, 1]), n_path=i32(2), start=i32(0), most=4)
    for bad in (dict(k_new=k.float()), dict(v_new=v[..., :32]), dict(path=i32(0, 1)), dict(path=i32([0], [1])), dict(path=good["path"].long()), dict(n_path=i32(2).cpu()), dict(start=i32(0).long()),
                dict(most=5), dict(most=-1), dict(path=i32([0] * 65))):
        with pytest.raises((ValueError, AssertionError, MB.MadaKVError)):
            eng.tree_commit(0, 1, **{**good, **bad})
    torch.cuda.synchronize()
    assert eng.kv_len.view(-1).tolist() == [60, 47] and not out.any()
