"""GPU: the 4-bit reduced cache, decode that accumulates its weights and replaces rows, the scores of all prompt queries; each
against plain arithmetic in 64 bits, at the sizes and values where it can go wrong, and in a run together."""
import math

import numpy as np
import pytest
import torch

from oracle import madakv_oracle as O
from paper_2506_15724_amd import binding as MB

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(msg):
    print(f"[operators] {msg}", flush=True)


def make(lens=None, device_mask=None, **kw):
    """(engine, args, q, k, v, mask).  lens: rows every head of every layer holds after a selection with hand-made budgets (one
    batch item); None: a cache that keeps everything."""
    args = dict(n_layers=1, batch=1, window=8, dtype="bf16", pool_k=1, max_new_tokens=4, out_fp32=1)
    args.update(kw)
    NL, B, H, Hq, L, W, d = (args[x] for x in ("n_layers", "batch", "n_kv_heads", "n_q_heads", "ctx_len", "window", "head_dim"))
    args.setdefault("budget", L if lens is None else -(-sum(lens) // len(lens)))
    eng = MB.MadaKV(device=DEV, **args)
    g = torch.Generator().manual_seed(11)
    k, v = (torch.randn(NL, B, H, L, d, generator=g).to(DEV, eng.tdtype) for _ in range(2))
    mask = torch.zeros(B, L, dtype=torch.uint8, device=DEV)
    if lens is None:
        eng.select_gather(0, NL, k, v, mask)
    else:
        bud = torch.zeros(NL, B, H, 2, dtype=torch.int32)
        bud[..., 0] = torch.tensor(lens).view(NL, B, H) - W
        eng.select_gather(0, NL, k, v, mask, psi_pool=torch.rand(NL, B, H, L - W, generator=g).to(DEV), budgets=bud.to(DEV))
    torch.cuda.synchronize()
    if lens is not None:
        assert eng.kv_len.view(-1).tolist() == list(lens)
    return eng, args, k, v, mask


def row_numbers(eng, args, head):
    """Places in the cache of the rows of head number `head` (over layers, batch items, heads), in order."""
    off, n = int(eng.kv_off.view(-1)[head]), int(eng.kv_len.view(-1)[head])
    P = args.get("page_rows", 0)
    if not P:
        return torch.arange(off, off + n)
    tbl = eng.page_table_host().reshape(-1, eng.page_table_host().shape[-1])[head]
    r = np.arange(n)
    later = r - int(tbl[0]) * P
    page = np.where(later < 0, 0, tbl[1 + np.maximum(later, 0) // P])
    return torch.from_numpy(np.where(later < 0, off + r, page * P + np.maximum(later, 0) % P))


def values(eng, args, which):
    """The cache's rows in 64 bits, on the host."""
    c = getattr(eng, which).cpu()
    d, cap = args["head_dim"], eng.capacity
    kind = args.get("cache_fp8", 0)
    if kind == 4:
        b = c.numpy()
        return torch.from_numpy(O.dequantize_mx4(b[:cap * (d // 2)].reshape(cap, d // 2), b[cap * (d // 2):].reshape(cap, d // 32)))
    return (c.view(torch.float8_e4m3fn) if kind == 1 else c).double()


def stored(x, kind):
    """bf16 / fp32 rows as the cache holds them, in 64 bits."""
    x = x.cpu()
    if kind == 4:
        return torch.from_numpy(O.dequantize_mx4(*O.quantize_mx4(x.double().numpy())))
    return (x.float().clamp(-448, 448).to(torch.float8_e4m3fn) if kind == 1 else x).double()


def attention(q, k, v, d):
    """(out, weights) of one head's queries [G, d] in 64 bits"""
    w = torch.softmax(q.cpu().double() @ k.T / math.sqrt(d), -1)
    return w @ v, w


KINDS = {"bf16": {}, "fp8": dict(cache_fp8=1), "fp4": dict(cache_fp8=4), "fp32": dict(dtype="fp32")}


# ---- the 4-bit cache ----------------------------------------------------------------------------------
def awkward_rows(n, d, g):
    """bf16 rows whose blocks have every kind of trouble: all zero, one element, ties at every step, largest magnitudes on
    either side of where the scale changes, the smallest and largest magnitudes, infinities, NaN."""
    x = torch.randn(n, d, generator=g) * torch.exp2(torch.randint(-20, 21, (n, 1), generator=g).float())
    steps = torch.tensor([0.25, 0.5, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, 7.0])
    special = [torch.zeros(32), torch.eye(32)[5], -torch.eye(32)[31] * 3, torch.full((32,), -7.0), torch.full((32,), 7.0625),
               torch.cat([steps, -steps, torch.tensor([4.0] * 10)]), torch.full((32,), 1e-39), torch.full((32,), 3e-36), torch.full((32,), 3.3e38),
               torch.cat([torch.tensor([float("inf"), -1.0]), torch.ones(30)]), torch.cat([torch.tensor([float("nan"), 2.0]), torch.ones(30)]),
               torch.cat([torch.tensor([1e-30]), torch.zeros(31)]), torch.cat([torch.tensor([-0.0, 1e-3]), torch.ones(30)])]
    for i, s in enumerate(special):
        at = (i * 3) % n
        x[at, (i % (d // 32)) * 32:][:32] = s
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("d,H,L,lens,P", [(128, 3, 300, [9, 64, 171], 0), (64, 2, 300, [65, 63], 0), (128, 1, 70, None, 0), (64, 5, 513, [200, 8, 9, 16, 300], 0),
                                          (128, 2, 200, [33, 31], 16), (64, 2, 200, [100, 64], 64)])
def test_fp4_rows_in_and_out(d, H, L, lens, P):
    """Codes and scales bit for bit those of the format's definition, the values read back exact, and nothing written behind the
    heads' rows."""
    eng, args, k, v, mask = make(lens, n_q_heads=H, n_kv_heads=H, head_dim=d, ctx_len=L, cache_fp8=4, page_rows=P)
    g = torch.Generator().manual_seed(L)
    k, v = (torch.stack([awkward_rows(L, d, g) for _ in range(H)]).view(1, 1, H, L, d).to(DEV) for _ in range(2))
    eng.k_c.fill_(0xA5), eng.v_c.fill_(0xA5)
    say(f"fp4 rows d={d} H={H} L={L} P={P}")
    bud = torch.zeros(1, 1, H, 2, dtype=torch.int32)
    bud[..., 0] = torch.tensor(lens or [L] * H).view(1, 1, H) - 8
    eng.select_gather(0, 1, k, v, mask, psi_pool=torch.rand(1, 1, H, L - 8, generator=g).to(DEV), budgets=bud.to(DEV))
    rows = [torch.full((eng.capacity, d), -77.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    eng.cache_rows(0, 1, *rows)
    torch.cuda.synchronize()
    used = torch.zeros(eng.capacity, dtype=torch.bool)
    for h in range(H):
        at = row_numbers(eng, args, h)
        used[at] = True
        kept = eng.kept_idx.cpu()[at].long()
        for src, cache, back in ((k, eng.k_c, rows[0]), (v, eng.v_c, rows[1])):
            code, scale = O.quantize_mx4(src[0, 0, h].cpu()[kept].double().numpy())
            c = cache.cpu().numpy()
            assert np.array_equal(c[:eng.capacity * (d // 2)].reshape(-1, d // 2)[at], code)
            assert np.array_equal(c[eng.capacity * (d // 2):].reshape(-1, d // 32)[at], scale)
            assert np.array_equal(back.cpu().double().numpy()[at], O.dequantize_mx4(code, scale))
    for cache, back in ((eng.k_c, rows[0]), (eng.v_c, rows[1])):
        c = cache.cpu()
        assert (c[:eng.capacity * (d // 2)].view(-1, d // 2)[~used] == 0xA5).all() and (c[eng.capacity * (d // 2):].view(-1, d // 32)[~used] == 0xA5).all()
        assert (back.cpu()[~used] == -77.0).all()
    eng.close()


@pytest.mark.parametrize("d", [64, 128])
def test_fp8_rows_out(d):
    """cache_rows on the 8-bit cache: what the E4M3 bytes stand for, every code among them."""
    eng, args, *_ = make([100, 300], n_q_heads=2, n_kv_heads=2, head_dim=d, ctx_len=400, cache_fp8=1)
    codes = torch.arange(256, dtype=torch.uint8).repeat(eng.capacity * d // 256 + 1)[:eng.capacity * d].view(-1, d).to(DEV)
    eng.k_c.copy_(codes), eng.v_c.copy_(codes.flip(0))
    rows = [torch.zeros(eng.capacity, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    eng.cache_rows(0, 1, *rows)
    torch.cuda.synchronize()
    for h in range(2):
        at = row_numbers(eng, args, h)
        for cache, back in zip((eng.k_c, eng.v_c), rows):
            assert torch.equal(back.cpu()[at].double().nan_to_num(nan=9e9), cache.view(torch.float8_e4m3fn).cpu()[at].double().nan_to_num(nan=9e9))
    eng.close()


@pytest.mark.parametrize("Hq,H,d,L,lens", [
    (1, 1, 128, 40, [9]), (8, 1, 64, 300, [250]), (4, 4, 128, 1500, [31, 32, 33, 127]), (14, 2, 128, 1500, [128, 129]), (5, 5, 64, 700, [15, 16, 17, 255, 256]),
    (28, 4, 128, 5000, [2100, 1000, 40, 500]), (6, 3, 64, 9000, [6000, 8, 2000]), (32, 32, 128, 700, [300] * 31 + [640]), (16, 8, 64, 3000, [1023, 1024, 1025, 600, 601, 9, 8, 512])])
@pytest.mark.parametrize("out_fp32", [1, 0])
def test_fp4_decode(Hq, H, d, L, lens, out_fp32):
    """Attention over the rows as they are stored, appended ones among them.  Outputs are means of rows of N(0, 1) values in 4 bits;
    products of codes and bf16 are exact, sums of <= 128 of them in fp32 leave 1e-5 on a logit (|logit| < 8), P as three bf16
    parts next to nothing: 1e-4 covers both; a bf16 output is rounded to 8 significant bits, half a unit of the last being at most 2^-8 of the value."""
    eng, args, *_ = make(lens, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, cache_fp8=4, out_fp32=out_fp32)
    g = torch.Generator().manual_seed(3)
    G, worst = Hq // H, 0.0
    out = torch.empty(1, 1, Hq, d, dtype=torch.float32 if out_fp32 else torch.bfloat16, device=DEV)
    for step in range(5):
        q, kn, vn = (torch.randn(1, 1, h, d, generator=g).to(DEV, torch.bfloat16) for h in (Hq, H, H))
        say(f"fp4 decode {Hq}/{H} d={d} {lens[:4]} step {step}")
        eng.decode_attn(0, 1, q, *((kn, vn) if step < 4 else (None, None)), out)
        torch.cuda.synchronize()
        assert eng.kv_len.view(-1).tolist() == [n + min(step + 1, 4) for n in lens]
        k, v = values(eng, args, "k_c"), values(eng, args, "v_c")
        for h in range(H):
            at = row_numbers(eng, args, h)
            if step < 4:
                assert torch.equal(k[at[-1]], stored(kn[0, 0, h], 4)) and torch.equal(v[at[-1]], stored(vn[0, 0, h], 4))
            ref, _ = attention(q[0, 0, h * G:(h + 1) * G], k[at], v[at], d)
            err = (out[0, 0, h * G:(h + 1) * G].cpu().double() - ref).abs() - (0 if out_fp32 else ref.abs() * 2.0 ** -8)
            worst = max(worst, float(err.max()))
    say(f"worst {worst:.2e}")
    assert worst < 1e-4
    eng.close()


@pytest.mark.parametrize("Hq,H,d,P", [(4, 4, 128, 16), (8, 2, 64, 64), (7, 1, 128, 256)])
def test_fp4_paged_and_static(Hq, H, d, P):
    """Pages and the handle's own scratch give the bits of contiguous segments, across the ends of pages."""
    lens = [P - 1, P, P + 1, 300][:H]
    flat, args, *_ = make(lens, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=700, budget=310, cache_fp8=4, max_new_tokens=40)
    paged, pargs, *_ = make(lens, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=700, budget=310, cache_fp8=4, max_new_tokens=40, page_rows=P)
    g = torch.Generator().manual_seed(2)
    for step in range(36):
        q, kn, vn = (torch.randn(1, 1, h, d, generator=g).to(DEV, torch.bfloat16) for h in (Hq, H, H))
        outs = [torch.full((1, 1, Hq, d), float("nan"), device=DEV) for _ in range(3)]
        flat.decode_attn(0, 1, q, kn, vn, outs[0])
        paged.decode_attn(0, 1, q, kn, vn, outs[1])
        flat.decode_attn_static(0, 1, q, None, None, outs[2])
        torch.cuda.synchronize()
        assert torch.isfinite(outs[0]).all() and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    rows = [[torch.zeros(e.capacity, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)] for e in (flat, paged)]
    for e, r in zip((flat, paged), rows):
        e.cache_rows(0, 1, *r)
    torch.cuda.synchronize()
    for h in range(H):
        for i in range(2):
            assert torch.equal(rows[0][i].cpu()[row_numbers(flat, args, h)], rows[1][i].cpu()[row_numbers(paged, pargs, h)])
    flat.close(), paged.close()


def test_fp4_empty_heads_and_nan_queries():
    """A head without rows gives no finite output and takes no row; a query that is no number gives one that is none, and the
    other heads are as ever."""
    eng, args, *_ = make([64, 64], n_q_heads=4, n_kv_heads=2, head_dim=128, ctx_len=300, cache_fp8=4)
    eng.kv_len[0, 0, 1] = 0
    q, kn, vn = (torch.randn(1, 1, h, 128, device=DEV).to(torch.bfloat16) for h in (4, 2, 2))
    q[0, 0, 0, 5] = float("nan")
    out = torch.zeros(1, 1, 4, 128, device=DEV)
    before = eng.k_c.clone()
    eng.decode_attn(0, 1, q, kn, vn, out)
    torch.cuda.synchronize()
    assert eng.kv_len.view(-1).tolist() == [65, 0]
    assert torch.isnan(out[0, 0, 0]).all() and torch.isfinite(out[0, 0, 1]).all() and not torch.isfinite(out[0, 0, 2:]).any()
    changed = (eng.k_c != before).nonzero().view(-1).cpu()
    row = int(eng.kv_off[0, 0, 0]) + 64
    assert all(row * 64 <= c < (row + 1) * 64 or eng.capacity * 64 + row * 4 <= c < eng.capacity * 64 + (row + 1) * 4 for c in changed.tolist())
    eng.close()


@pytest.mark.parametrize("P", [0, 16, 64])
@pytest.mark.parametrize("Hq,H,d,W", [(4, 4, 128, 16), (8, 2, 64, 8)])
def test_fp4_reeviction(Hq, H, d, W, P):
    """Re-eviction of a 4-bit cache: what a bf16 cache that holds the same values does, position by position, and the survivors' codes
    and scales as they were; twice, with appended rows in between."""
    NL, B, L, T = 2, 2, 700, 20
    kw = dict(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=W, budget=150, max_new_tokens=T, page_rows=P, device=DEV)
    args = dict(n_layers=NL, batch=B, n_kv_heads=H, n_q_heads=Hq, head_dim=d, page_rows=P)
    g = torch.Generator(device=DEV).manual_seed(d + P)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)        # noqa: E731
    exact = lambda x: stored(x, 4).to(DEV, torch.bfloat16)                                # noqa: E731  (what 4 bits hold of it)
    q, k, v = randn(NL, B, Hq, W, d), randn(NL, B, H, L, d), randn(NL, B, H, L, d)
    k, v = exact(k), exact(v)
    mask = torch.randint(0, 2, (B, L), generator=g, device=DEV).to(torch.uint8)
    engs = [MB.MadaKV(cache_fp8=kind, **kw) for kind in (4, 0)]
    for e in engs:
        e.evict(0, NL, q, k, v, mask)
    out = [torch.zeros(NL, B, Hq, d, device=DEV) for _ in engs]
    for round_ in range(2):
        for step in range(T - 3 * round_):
            x = randn(NL, B, Hq, d), exact(randn(NL, B, H, d)), exact(randn(NL, B, H, d))
            for e, o in zip(engs, out):
                e.decode_attn(0, NL, *x, o)
        recent = randn(NL, B, Hq, W, d)
        say(f"fp4 reevict {Hq}/{H} d={d} P={P} round {round_}")
        for e in engs:
            e.reevict(0, NL, recent, mask)
        torch.cuda.synchronize()
        for n in ("kv_len", "budgets"):
            assert torch.equal(getattr(engs[0], n), getattr(engs[1], n))
        held = [torch.cat([row_numbers(e, args, i) for i in range(NL * B * H)]) for e in engs]
        assert torch.equal(engs[0].kept_idx.cpu()[held[0]], engs[1].kept_idx.cpu()[held[1]])
        for n in ("k_c", "v_c"):
            assert torch.equal(values(engs[0], dict(args, cache_fp8=4), n)[held[0]], values(engs[1], args, n)[held[1]])
    for e, o in zip(engs, out):
        e.decode_attn(0, NL, randn(NL, B, Hq, d) * 0 + 1, None, None, o)
    torch.cuda.synchronize()
    assert float((out[0] - out[1]).abs().max()) < 1e-4              # (the bound of test_fp4_decode)
    for e in engs:
        e.close()


# ---- decode with accumulated weights ------------------------------------------------------------------------
def weights_step(eng, args, q, kn, vn, acc, decay, slots, pos, recent, in_place=False, l0=0, n=None):
    """One call checked against 64 bits: outputs, sums, stored rows, positions, the row to go.  slots: None (append, or attend
    only), or a list with a row per head.  Returns the new sums and slot_out."""
    NL = n or args["n_layers"]
    H, Hq, d, B, kind = args["n_kv_heads"], args["n_q_heads"], args["head_dim"], args["batch"], args.get("cache_fp8", 0)
    G, heads = Hq // H, NL * args["batch"] * H
    first = l0 * B * H
    len0 = eng.kv_len.view(-1).tolist()
    kept0, k0, v0 = eng.kept_idx.clone(), values(eng, args, "k_c"), values(eng, args, "v_c")
    out = torch.full((NL, B, Hq, d), float("nan"), dtype=eng._out_dtype, device=DEV)
    acc_in = acc.clone()
    acc_out = acc_in if in_place else torch.full_like(acc, -5.0)
    slot_in = None if slots is None else torch.tensor(slots, dtype=torch.int32, device=DEV)
    slot_out = torch.full((heads,), -9, dtype=torch.int32, device=DEV)
    eng.decode_attn_weights(l0, NL, q, kn, vn, out, acc_in, acc_out, decay=decay, slot_in=slot_in, slot_out=slot_out, pos=pos, recent=recent)
    torch.cuda.synchronize()
    k, v, got, kept = values(eng, args, "k_c"), values(eng, args, "v_c"), acc_out.cpu().double(), eng.kept_idx.cpu()
    want = (acc if in_place else torch.full_like(acc, -5.0)).cpu().double()
    tol = torch.zeros_like(want)
    kept_want, k_want, v_want = kept0.cpu().clone(), k0.clone(), v0.clone()
    for i in range(heads):
        h = first + i
        at = row_numbers(eng, args, h)
        new = None
        if kn is not None and slots is None:
            assert len(at) == len0[h] + (1 if len0[h] else 0)
            new = len(at) - 1 if len0[h] else None
        else:
            assert len(at) == len0[h]
            if slots is not None and 0 <= slots[i] < len0[h]:
                new = slots[i]
        if len(at) == 0:
            assert int(slot_out[i]) == -1 and not torch.isfinite(out.view(heads, G, d)[i].float()).any()
            continue
        if new is not None:
            k_want[at[new]], v_want[at[new]] = stored(kn.reshape(heads, d)[i], kind), stored(vn.reshape(heads, d)[i], kind)
            kept_want[at[new]] = pos[i // H % B].cpu()
        ref, w = attention(q.reshape(heads, G, d)[i], k_want[at], v_want[at], d)
        paid = w.sum(0)
        old = decay * acc.cpu().double()[at]
        if new is not None:
            old[new] = 0.0
        want[at] = old + paid
        tol[at] = 5e-5 * paid + 3e-7 * old.abs() + 1e-9         # logits within 1e-5, twice (numerator and sum), exp2 and sums of fp32
        err = (out.view(heads, G, d)[i].cpu().double() - ref).abs() - (0 if out.dtype == torch.float32 else ref.abs() * 2.0 ** -8)
        assert float(err.max()) < 1e-4, (h, float(err.max()))
        # the row to go, from the library's own sums
        may = (kept_want[at].long() <= int(pos[i // H % B]) - recent).nonzero().view(-1)
        least = int(may[torch.argmin(got[at][may])]) if len(may) else -1
        assert int(slot_out[i]) == least, (h, int(slot_out[i]), least)
    assert ((got - want).abs() <= tol).all(), float(((got - want).abs() - tol).max())
    assert torch.equal(kept, kept_want)
    same = lambda x, y: torch.equal(x.nan_to_num(nan=1e300), y.nan_to_num(nan=1e300))      # noqa: E731  (rows nobody has written may hold NaN)
    assert same(k, k_want) and same(v, v_want)
    return acc_out, slot_out


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("Hq,H,d,lens", [(4, 4, 128, [9, 33, 127, 255]), (8, 1, 64, [1300]), (14, 2, 128, [2049, 16]), (3, 3, 64, [1024, 1025, 8]), (6, 2, 64, [128, 129])])
def test_weights_append_replace_attend(kind, Hq, H, d, lens):
    """Appending, replacing at the edges of tiles and pieces (the first row, the last, rows that are none), attending only; the
    sums, the rows stored, the positions and the row to go."""
    eng, args, *_ = make(lens, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=4000, max_new_tokens=3, **KINDS[kind])
    g = torch.Generator().manual_seed(5)
    acc = torch.rand(eng.capacity, generator=g).to(DEV)
    pos = torch.tensor([4000], dtype=torch.int32, device=DEV)
    draw = lambda: [torch.randn(1, 1, h, d, generator=g).to(DEV, eng.tdtype) for h in (Hq, H, H)]      # noqa: E731
    for step in range(2):
        say(f"weights {kind} {Hq}/{H} d={d} append {step}")
        acc, slot = weights_step(eng, args, *draw(), acc, 1.0, None, pos, 8)
        pos += 1
    say("attend only")
    q = draw()[0]
    acc, slot = weights_step(eng, args, q, None, None, acc, 0.5, None, pos, 40)
    ends = [n + 2 for n in lens]
    for slots in ([0] * H, [n - 1 for n in ends], [-1] * H, ends, [min(n - 1, 16) for n in ends], [min(n - 1, 128) for n in ends], [n // 2 for n in ends]):
        say(f"replace {slots}")
        acc, slot = weights_step(eng, args, *draw(), acc, 0.9, slots, pos, 3, in_place=slots[0] == 0)
        pos += 1
    for step in range(3):
        say("replace what the step before chose")
        acc, slot = weights_step(eng, args, *draw(), acc, 1.0, slot.tolist(), pos, 8)
        pos += 1
    with pytest.raises(MB.MadaKVError) as e:                # no longer in order of position
        eng.reevict(0, 1, torch.zeros(1, 1, Hq, 8, d, dtype=eng.tdtype, device=DEV), torch.zeros(1, 4000, dtype=torch.uint8, device=DEV))
    assert e.value.status == -1
    eng.close()


@pytest.mark.parametrize("kind,P", [("bf16", 16), ("fp8", 64), ("fp4", 16), ("fp32", 32)])
@pytest.mark.parametrize("Hq,H,d", [(4, 2, 128), (3, 3, 64)])
def test_weights_paged(kind, P, Hq, H, d):
    """Sums, positions and replaced rows in pages taken later."""
    lens = [P, 2 * P - 1, 200][:H]
    eng, args, *_ = make(lens, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=900, budget=210, max_new_tokens=2 * P + 2, page_rows=P, **KINDS[kind])
    g = torch.Generator().manual_seed(6)
    acc = torch.rand(eng.capacity, generator=g).to(DEV)
    eng.kept_idx.fill_(0)
    pos = torch.tensor([900], dtype=torch.int32, device=DEV)
    draw = lambda: [torch.randn(1, 1, h, d, generator=g).to(DEV, eng.tdtype) for h in (Hq, H, H)]      # noqa: E731
    out = torch.empty(1, 1, Hq, d, device=DEV)
    for step in range(P + 1):
        say(f"weights paged {kind} step {step}")
        if step % 5 == 0:
            acc, slot = weights_step(eng, args, *draw(), acc, 1.0, None, pos, 0)
        else:
            eng.decode_attn(0, 1, *draw(), out)
        pos += 1
    for slots in ([0] * H, [n + P for n in lens], [P] * H):
        acc, slot = weights_step(eng, args, *draw(), acc, 1.0, slots, pos, 0)
        pos += 1
    eng.close()


def test_weights_choice_at_ties_nan_and_none():
    """Equal sums: the lower row.  Sums that are no numbers: last.  No row old enough: -1.  A head without rows: -1, nothing written."""
    eng, args, *_ = make([40, 2000, 40], n_q_heads=3, n_kv_heads=3, head_dim=64, ctx_len=2100, max_new_tokens=1)
    off = eng.kv_off.view(-1).tolist()
    q = torch.zeros(1, 1, 3, 64, dtype=torch.bfloat16, device=DEV)              # equal weights everywhere
    out, acc_out = torch.empty(1, 1, 3, 64, device=DEV), torch.empty(eng.capacity, device=DEV)
    acc = torch.full((eng.capacity,), 2.0, device=DEV)
    acc[off[0] + 7:off[0] + 20] = 1.0
    acc[off[1]:off[1] + 2000] = float("nan")
    acc[off[1] + 1500] = 9.0
    slot, pos = torch.empty(3, dtype=torch.int32, device=DEV), torch.tensor([10 ** 6], dtype=torch.int32, device=DEV)
    eng.kv_len[0, 0, 2] = 0
    eng.decode_attn_weights(0, 1, q, None, None, out, acc, acc_out, slot_out=slot, pos=pos)
    torch.cuda.synchronize()
    assert slot.tolist() == [7, 1500, -1]
    acc[off[1] + 1500] = float("nan")
    eng.decode_attn_weights(0, 1, q, None, None, out, acc, acc_out, slot_out=slot, pos=pos)
    torch.cuda.synchronize()
    assert slot.tolist() == [7, 0, -1]
    pos.fill_(-5)
    eng.decode_attn_weights(0, 1, q, None, None, out, acc, acc_out, slot_out=slot, pos=pos, recent=2 ** 31 - 1)
    torch.cuda.synchronize()
    assert slot.tolist() == [-1, -1, -1]
    eng.close()


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
def test_weights_in_a_replayed_graph(kind):
    """A replacing step captured once and replayed, the position advanced on the device and the chosen row fed back: every replay
    as the eager steps of another handle, with that handle's work between the replays."""
    lens, Hq, H, d, B, NL = [70, 300] * 4, 4, 2, 128, 2, 2
    pair = []
    for _ in range(2):
        eng, args, *_ = make(lens, n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=600, max_new_tokens=0, **KINDS[kind])
        s = dict(eng=eng, acc=torch.rand(eng.capacity, generator=torch.Generator().manual_seed(1)).to(DEV), slot=torch.zeros(NL * B * H, dtype=torch.int32, device=DEV),
                 pos=torch.tensor([600, 640], dtype=torch.int32, device=DEV), out=torch.zeros(NL, B, Hq, d, device=DEV),
                 x=[torch.zeros(NL, B, h, d, dtype=torch.bfloat16, device=DEV) for h in (Hq, H, H)])
        pair.append(s)

    def step(s):
        for l in range(NL):
            x = [t[l:l + 1] for t in s["x"]]
            slot = s["slot"][l * B * H:(l + 1) * B * H]
            s["eng"].decode_attn_weights(l, 1, *x, s["out"][l:l + 1], s["acc"], s["acc"], slot_in=slot, slot_out=slot, pos=s["pos"], recent=16)
        s["pos"] += 1

    eager, graphed = pair
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(graphed)
    torch.cuda.synchronize()
    g = torch.Generator().manual_seed(9)
    for i in range(6):
        for t in range(3):
            new = torch.randn(eager["x"][t].shape, generator=g).to(DEV, torch.bfloat16)
            for s in pair:
                s["x"][t].copy_(new)
        step(eager)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        say(f"replay {i}")
        for name in ("acc", "slot", "pos", "out"):
            assert torch.equal(eager[name], graphed[name]), name
        for name in ("k_c", "v_c", "kept_idx", "kv_len"):
            assert torch.equal(getattr(eager["eng"], name), getattr(graphed["eng"], name)), name
    del graph
    for s in pair:
        s["eng"].close()


# ---- scores of all prompt queries -----------------------------------------------------------------------------
def prompt_reference(q, k, G):
    """(psi [H, L], lse [Hq, L]) of q [Hq, L, d], k [H, L, d] in 64 bits, on the GPU"""
    Hq, L, d = q.shape
    psi = torch.zeros(Hq // G, L, dtype=torch.float64, device=DEV)
    lse = torch.zeros(Hq, L, dtype=torch.float64, device=DEV)
    seen = torch.ones(L, L, dtype=torch.bool, device=DEV).tril_()
    for j in range(Hq):
        s = (q[j].double() @ k[j // G].double().t().contiguous() / math.sqrt(d)).masked_fill_(~seen, -math.inf)
        lse[j] = torch.logsumexp(s, -1)
        psi[j // G] += torch.exp(s - lse[j][:, None]).sum(0)
    return psi, lse


def prompt_case(NL, B, Hq, H, d, L, W=1, M=2, **kw):
    eng = MB.MadaKV(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=W, budget=min(L, W + max(1, L // 4)), n_modalities=M, device=DEV, **kw)
    g = torch.Generator(device=DEV).manual_seed(L * 7 + d)
    q, k = (torch.randn(NL, B, h, L, d, generator=g, device=DEV).to(torch.bfloat16) for h in (Hq, H))
    return eng, q, k


def check_prompt(eng, q, k, given, bound=2e-4):
    """Every score within `bound` of itself: sums of <= 128 products in fp32 leave 1e-5 .. 8e-5 on a logit in log2 units (|logit| < 8), in
    the weight and in the normaliser; 1e-12 for what underflows."""
    NL, B, Hq, L, d = q.shape
    G = Hq // k.shape[2]
    ref = [prompt_reference(q[l, b], k[l, b], G) for l in range(NL) for b in range(B)]
    psi = torch.stack([r[0] for r in ref]).view(NL, B, -1, L)
    lse = torch.stack([r[1] for r in ref]).view(NL, B, Hq, L).float().contiguous() if given else None
    eng.psi.fill_(float("nan"))
    got = []
    for _ in range(2):
        eng.score_prompt(0, NL, q, k, row_lse=lse)
        torch.cuda.synchronize()
        got.append(eng.psi.clone())
    assert torch.equal(*got)                                    # the same bits every time
    err = ((got[0].double() - psi).abs() / (psi.abs() + 1e-8)).max()
    say(f"worst relative error {float(err):.2e}")
    assert float(err) < bound
    return psi


@pytest.mark.parametrize("L", [2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 512, 513, 700])
@pytest.mark.parametrize("Hq,H,d", [(2, 2, 128), (7, 1, 64)])
@pytest.mark.parametrize("given", [False, True])
def test_prompt_scores_at_edges(L, Hq, H, d, given):
    """Lengths around tiles of 32 and 64 rows and blocks of 128 and 512 columns."""
    eng, q, k = prompt_case(1, 1, Hq, H, d, L)
    say(f"prompt {Hq}/{H} d={d} L={L} lse={given}")
    check_prompt(eng, q, k, given)
    eng.close()


@pytest.mark.parametrize("NL,B,Hq,H,d,L", [(1, 1, 28, 4, 128, 4100), (1, 2, 32, 32, 128, 1025), (2, 2, 16, 8, 64, 1500), (1, 1, 8, 8, 64, 5000), (1, 4, 32, 32, 64, 2047), (3, 1, 32, 32, 128, 640),
                                            (1, 1, 32, 8, 128, 2048), (1, 1, 12, 2, 64, 3500), (2, 1, 16, 4, 64, 1790), (4, 2, 32, 32, 64, 513), (1, 1, 20, 20, 128, 1537), (1, 2, 28, 4, 128, 1025)])
@pytest.mark.parametrize("given", [False, True])
def test_prompt_scores_of_large_calls(NL, B, Hq, H, d, L, given):
    """Calls that take blocks of 256 and 512 columns, several chunks per head, several layers and batch items."""
    eng, q, k = prompt_case(NL, B, Hq, H, d, L)
    say(f"prompt {NL} x {B} x {Hq}/{H} d={d} L={L} lse={given}")
    check_prompt(eng, q, k, given)
    eng.close()


@pytest.mark.parametrize("NL,B,Hq,H,d", [(2, 3, 4, 4, 128), (1, 2, 28, 4, 128), (3, 1, 6, 2, 64), (4, 16, 16, 8, 64)])
@pytest.mark.parametrize("L", [17, 96, 160, 192, 203, 224, 256])
@pytest.mark.parametrize("given", [False, True])
def test_prompt_scores_of_short_prompts(NL, B, Hq, H, d, L, given):
    """Prompts whose logits stay in registers: every number of blocks of 32 queries, full and ragged, layers and batch items."""
    eng, q, k = prompt_case(NL, B, Hq, H, d, L)
    say(f"prompt {NL} x {B} x {Hq}/{H} d={d} L={L} lse={given}")
    check_prompt(eng, q, k, given)
    eng.close()


@pytest.mark.parametrize("top", [90.0, 400.0, -400.0])
@pytest.mark.parametrize("Hq,L,at", [(2, 700, 300), (64, 1100, 520), (2, 130, 96)])
def test_prompt_scores_far_from_the_first_keys(Hq, L, at, top):
    """Logits that leave the reference of a row's first keys far behind, at a key in the middle of the prompt and step by step: the first
    element of Q is 8, of K top / 8 * sqrt(d) * (0 before `at`, then rising).  The logit's products are of one element, so that
    its error is that of one product and one addition: the bound of check_prompt holds up to |logit| * 2^-23 = 5e-5, twice."""
    eng, q, k = prompt_case(1, 1, Hq, Hq, 64, L)
    q[..., 0], k[..., 0] = 8.0, 0.0
    ramp = torch.linspace(0.5, 1.0, L - at, device=DEV) * top
    k[..., at:, 0] = ramp.to(torch.bfloat16)
    say(f"prompt far Hq={Hq} L={L} top={top}")
    check_prompt(eng, q, k, False, bound=4e-4)
    eng.close()


@pytest.mark.parametrize("Hq,H,d,L", [(2, 2, 128, 300), (64, 64, 64, 1100)])
def test_prompt_scores_of_tiny_and_huge_logits(Hq, H, d, L):
    """A scale under which no logit is anything: a query pays 1 / (r + 1) to each key it sees and nothing to the others.  And q . k down to
    -2e32 under a scale that makes -16 .. -176 of it (one element each, powers of two times 1 .. 11): 176 log2(e) * 2^-24 in
    the weight, in the normaliser and in the scale itself make 3 * 1.1e-5; sums of 1100 terms 1100 * 2^-24 / 2 = 3.3e-5."""
    say(f"prompt tiny and huge {Hq}/{H} d={d} L={L}")
    eng, q, k = prompt_case(1, 1, Hq, H, d, L, softmax_scale=1e-33)
    eng.score_prompt(0, 1, q, k)
    want = (1.0 / torch.arange(1, L + 1, device=DEV, dtype=torch.float64)).flip(0).cumsum(0).flip(0)
    assert float((eng.psi[0, 0].double() / want - 1).abs().max()) < 7e-5
    eng.close()
    eng, q, k = prompt_case(1, 1, Hq, H, d, L, softmax_scale=2.0 ** -100)
    level = 1 + torch.arange(L - 1, -1, -1, device=DEV) // 100
    q.zero_(), k.zero_()
    q[..., 0], k[..., 0] = 2.0 ** 52, (-level * 2.0 ** 52).to(torch.bfloat16)
    eng.score_prompt(0, 1, q, k)
    s = (-16.0 * level.double()).expand(L, L).masked_fill(~torch.ones(L, L, dtype=torch.bool, device=DEV).tril_(), -math.inf)
    want = torch.softmax(s, -1).sum(0)
    assert float(((eng.psi[0, 0].double() - want).abs() / (want + 1e-8)).max()) < 7e-5
    eng.close()


def test_prompt_scores_with_statistics():
    """The pooled scores, masses, counts and candidates that go with them, and what allocation and selection make of those: the same
    as the statistics of the scores times the power of two, by the oracle."""
    NL, B, Hq, H, d, L, W = 2, 2, 8, 4, 64, 900, 16
    eng, q, k = prompt_case(NL, B, Hq, H, d, L, W=W, pool_k=5)
    mask = torch.randint(0, 2, (B, L), generator=torch.Generator().manual_seed(4)).to(torch.uint8)
    eng.score_prompt(0, NL, q, k, mask=mask.to(DEV))
    torch.cuda.synchronize()
    psi = eng.psi.cpu().double().numpy() * 2.0 ** -6                    # the least s with 16 * 2^s >= 900
    w, cnt = eng.stats_host()
    for l in range(NL):
        for b in range(B):
            m = mask[b].numpy()
            assert eng.n_mod[b].tolist() == [int((m[:L - W] == i).sum()) for i in (0, 1)]
            for h in range(H):
                np.testing.assert_array_equal(eng.psi_pool[l, b, h].cpu().double().numpy(), O.pool_scores(psi[l, b, h][None], W, 5)[0])
                for i in (0, 1):
                    x = psi[l, b, h][:L - W][m[:L - W] == i]
                    assert abs(w[l, b, h, i] - x.sum()) <= 2e-6 * x.sum() + len(x) * 2.0 ** -45
                    c = np.cumsum(np.sort(x)[::-1])
                    n = int(cnt[l, b, h, i])
                    assert c[n - 1] >= 0.9 * x.sum() * (1 - 1e-4) and (n == 1 or c[n - 2] <= 0.9 * x.sum() * (1 + 1e-4))
    v = torch.randn(NL, B, H, L, d, device=DEV).to(torch.bfloat16)
    eng.allocate(0, NL)
    eng.select_gather(0, NL, k, v, mask.to(DEV))
    torch.cuda.synchronize()
    assert int(eng.budgets.sum()) == NL * B * H * (eng.cfg.budget - W)
    pool, off, ln, bud = eng.psi_pool.cpu().double().numpy(), eng.kv_off.cpu(), eng.kv_len.cpu(), eng.budgets.cpu().numpy()
    for l, b, h in ((0, 0, 0), (1, 1, 3), (0, 1, 2)):
        kept = eng.kept_idx.cpu()[off[l, b, h]:off[l, b, h] + ln[l, b, h]].numpy()
        np.testing.assert_array_equal(kept, O.select(pool[l, b, h], mask[b].numpy(), int(bud[l, b, h, 0]), int(bud[l, b, h, 1]), L, W))
    eng.close()


def test_statistics_of_short_prompts():
    """One query head per KV head (the kernel of short prompts writes the scaled scores itself) and four: psi with statistics is psi
    without, the pooled scores are those of psi times the power of two."""
    for NL, B, Hq, H, d, L, W, s in ((2, 3, 2, 2, 64, 200, 16, 4), (1, 2, 8, 2, 128, 256, 32, 3), (2, 1, 3, 3, 128, 40, 32, 1)):
        eng, q, k = prompt_case(NL, B, Hq, H, d, L, W=W, pool_k=3)
        mask = torch.randint(0, 2, (B, L), generator=torch.Generator().manual_seed(4)).to(DEV, torch.uint8)
        eng.score_prompt(0, NL, q, k)
        torch.cuda.synchronize()
        psi = eng.psi.clone()
        eng.psi.fill_(-1.0)
        eng.score_prompt(0, NL, q, k, mask=mask)
        torch.cuda.synchronize()
        assert torch.equal(eng.psi, psi)
        for l in range(NL):
            for b in range(B):
                want = O.pool_scores(psi[l, b].cpu().double().numpy() * 2.0 ** -s, W, 3)
                np.testing.assert_array_equal(eng.psi_pool[l, b].cpu().double().numpy(), want)
        eng.close()


@pytest.mark.parametrize("Hq,H,d,L", [(4, 4, 64, 200), (7, 1, 128, 256), (8, 2, 64, 700), (32, 8, 128, 2048)])
@pytest.mark.parametrize("given", [False, True])
def test_prompt_scores_in_a_replayed_graph(Hq, H, d, L, given):
    """Scores with statistics, captured once and replayed on other inputs, with eager calls of the same holder between the replays."""
    eng, q, k = prompt_case(1, 1, Hq, H, d, L, W=8)
    lse = torch.zeros(1, 1, Hq, L, device=DEV) if given else None
    mask = torch.randint(0, 2, (1, L), generator=torch.Generator().manual_seed(2)).to(DEV, torch.uint8)
    call = lambda: eng.score_prompt(0, 1, q, k, mask=mask, row_lse=lse)      # noqa: E731
    outs = lambda: [t.clone() for t in (eng.psi, eng.psi_pool, eng.stats, eng.n_mod)]      # noqa: E731
    call()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        call()
    g = torch.Generator(device=DEV).manual_seed(8)
    for step in range(4):
        say(f"prompt graph {Hq}/{H} d={d} L={L} lse={given} replay {step}")
        q.copy_(torch.randn(q.shape, generator=g, device=DEV)), k.copy_(torch.randn(k.shape, generator=g, device=DEV))
        if given:
            lse.copy_(5.0 + torch.rand(lse.shape, generator=g, device=DEV))
        call()
        torch.cuda.synchronize()
        want = outs()
        for t in (eng.psi, eng.psi_pool):
            t.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs(), want))
    eng.close()


def test_arrays_and_devices_that_do_not_fit(monkeypatch):
    """What the holder refuses before the library is called: arrays of another type, size or device, and a current device that is
    not the handle's."""
    eng, q, k = prompt_case(1, 2, 4, 2, 64, 64, W=8, cache_fp8=4)
    cap, f32, i32 = eng.capacity, torch.float32, torch.int32
    out = torch.empty(1, 2, 4, 64, device=DEV)
    acc = torch.zeros(cap, device=DEV)
    rows = torch.empty(cap, 64, dtype=torch.bfloat16, device=DEV)
    short, host = acc[:-1], acc.cpu()
    step = lambda **kw: eng.decode_attn_weights(0, 1, *[kw.pop(x, y) for x, y in (("q", out[..., :64].bfloat16()), ("kn", None), ("vn", None), ("out", out), ("a", acc), ("b", acc))], **kw)      # noqa: E731
    bad = [lambda: step(a=short), lambda: step(b=short), lambda: step(a=host), lambda: step(b=acc.double()), lambda: step(out=out.bfloat16()), lambda: step(out=out[:, :1].contiguous()),
           lambda: step(slot_in=torch.zeros(3, dtype=i32, device=DEV)), lambda: step(slot_out=torch.zeros(4, dtype=f32, device=DEV)), lambda: step(pos=torch.zeros(1, dtype=i32, device=DEV)),
           lambda: eng.cache_rows(0, 1, rows[:-1], rows), lambda: eng.cache_rows(0, 1, rows, rows.float()),
           lambda: eng.score_prompt(0, 1, q.float(), k), lambda: eng.score_prompt(0, 1, q, k[:, :1].contiguous()), lambda: eng.score_prompt(0, 1, q, k, row_lse=torch.zeros(4, device=DEV)),
           lambda: eng.score_prompt(0, 1, q, k, mask=torch.zeros(2, 63, dtype=torch.uint8, device=DEV)), lambda: eng.score_prompt(0, 1, q.cpu(), k)]
    for i, call in enumerate(bad):
        say(f"refused {i}")
        with pytest.raises(ValueError):
            call()
    with pytest.raises(AssertionError):                     # not contiguous
        eng.score_prompt(0, 1, q.transpose(2, 3), k)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: step(), lambda: eng.cache_rows(0, 1, rows, rows), lambda: eng.score_prompt(0, 1, q, k)):
        with pytest.raises(ValueError):
            call()
    monkeypatch.undo()
    torch.cuda.synchronize()
    eng.close()


@pytest.mark.parametrize("kind,L,NL,H", [("bf16", 2048, 32, 32), ("fp4", 4096, 6, 32)])
def test_workspaces_of_the_holder_serve_every_number_of_layers(kind, L, NL, H):
    """The pieces of a head get longer with the heads of a call, so that calls over fewer layers can need more workspace than one over all."""
    eng = MB.MadaKV(n_layers=NL, batch=1, n_q_heads=H, n_kv_heads=H, head_dim=64, ctx_len=L, window=8, budget=L // 2, max_new_tokens=0, device=DEV, **KINDS[kind])
    plain = [MB.madakv_workspace_bytes(eng.h, m)[2] for m in range(1, NL + 1)]
    more = [MB.madakv_decode_attn_weights_workspace_bytes(eng.h, m) for m in range(1, NL + 1)]
    n = 1 + int(np.argmax(plain))
    say(f"{kind}: most workspace for {n} of {NL} layers")
    assert 1 < n < NL and eng.decode_ws.numel() == plain[n - 1]
    eng.kv_off.copy_(9 * torch.arange(NL * H).view(NL, 1, H)), eng.kv_len.fill_(9)
    eng.k_c.zero_(), eng.v_c.zero_()
    q = torch.randn(n, 1, H, 64, device=DEV).to(eng.tdtype)
    out = torch.full((n, 1, H, 64), float("nan"), device=DEV)
    eng.decode_attn(0, n, q, None, None, out)
    acc = torch.zeros(eng.capacity, device=DEV)
    eng.decode_attn_weights(0, n, q, None, None, out, acc, torch.zeros_like(acc))
    torch.cuda.synchronize()
    assert not out.any() and eng.weights_ws.numel() == max(more)
    eng.close()


# ---- together ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["fp4", "bf16"])
def test_heavy_hitter_generation(kind):
    """As a program uses them: the prompt's scores, eviction by them into the reduced cache, generation that appends while there is
    room and replaces the least-weighted row afterwards, on a stream of its own; the attention and the cache against a
    simulation in 64 bits that follows the library's choices, and the rows read back at the end."""
    Hq, H, d, L, W, NL, B, room = 8, 2, 128, 700, 16, 2, 2, 3
    eng = MB.MadaKV(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=W, budget=120, max_new_tokens=room, device=DEV, **KINDS[kind])
    args = dict(n_layers=NL, batch=B, n_kv_heads=H, n_q_heads=Hq, head_dim=d, **KINDS[kind])
    g = torch.Generator().manual_seed(8)
    q, k, v = (torch.randn(NL, B, h, L, d, generator=g).to(DEV, torch.bfloat16) for h in (Hq, H, H))
    mask = torch.randint(0, 2, (B, L), generator=g).to(DEV, torch.uint8)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        eng.score_prompt(0, NL, q, k, mask=mask)
        eng.allocate(0, NL)
        eng.select_gather(0, NL, k, v, mask)
        stream.synchronize()
        # the sums start as the kept positions' scores
        acc = torch.zeros(eng.capacity, device=DEV)
        for i in range(NL * B * H):
            at = row_numbers(eng, args, i).to(DEV)
            acc[at] = eng.psi.view(-1, L)[i][eng.kept_idx[at].long()]
        pos, slot = torch.full((B,), L, dtype=torch.int32, device=DEV), None
        for step in range(8):
            say(f"heavy hitters {kind} step {step}")
            x = [torch.randn(NL, B, h, d, generator=g).to(DEV, torch.bfloat16) for h in (Hq, H, H)]
            acc, slot = weights_step(eng, args, *x, acc, 1.0, None if step < room else slot.tolist(), pos, 4)
            pos += 1
        if kind == "fp4":
            rows = [torch.zeros(eng.capacity, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            eng.cache_rows(0, NL, *rows)
            stream.synchronize()
            for i in range(NL * B * H):
                at = row_numbers(eng, args, i)
                assert torch.equal(rows[0].cpu()[at].double(), values(eng, args, "k_c")[at])
    eng.close()


def test_two_caches_on_two_streams():
    """Two handles with work in flight at once: the bits of each alone."""
    Hq, H, d, L = 4, 2, 128, 2500
    alone, both = [], []
    for where in (alone, both):
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        engs = [make([2000, 900], n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, **KINDS[kind])[0] for kind in ("fp4", "bf16")]
        g = torch.Generator(device=DEV).manual_seed(3)
        x = [torch.randn(1, 1, h, d, generator=g, device=DEV).to(torch.bfloat16) for h in (Hq, H, H)]
        res = [[torch.zeros(1, 1, Hq, d, device=DEV), torch.ones(e.capacity, device=DEV), torch.zeros(H, dtype=torch.int32, device=DEV)] for e in engs]
        pos = torch.tensor([L], dtype=torch.int32, device=DEV)
        torch.cuda.synchronize()
        for _ in range(10):
            for e, s, (out, acc, slot) in zip(engs, streams, res):
                with torch.cuda.stream(s):
                    e.decode_attn_weights(0, 1, *x, out, acc, acc, slot_in=slot, slot_out=slot, pos=pos, recent=1)
                if where is alone:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        for e, r, kind in zip(engs, res, ("fp4", "bf16")):
            held = torch.cat([row_numbers(e, {}, h) for h in range(H)])               # (what free rows hold is nobody's)
            where += [(kind + n, t.cpu()) for n, t in zip((" out", " acc", " slot"), r)]
            where += [(f"{kind} {n}", values(e, dict(head_dim=d, **KINDS[kind]), n)[held]) for n in ("k_c", "v_c")]
            e.close()
    for (name, a), (_, b) in zip(alone, both):
        assert torch.equal(a, b), name


def test_fp4_eviction_of_many_layers(monkeypatch):
    """madakv_evict over layer groups (gathers beside per-head kernels) fills the 4-bit cache with the bytes of the three calls."""
    NL, B, H, L, W, d = 8, 2, 4, 900, 16, 64
    monkeypatch.setenv("MADAKV_LAYER_GROUPS", "4")
    g = torch.Generator(device=DEV).manual_seed(12)
    q, k, v = (torch.randn(NL, B, H, n, d, generator=g, device=DEV).to(torch.bfloat16) for n in (W, L, L))
    mask = torch.randint(0, 2, (B, L), generator=g, device=DEV).to(torch.uint8)
    got = []
    for fused in (True, False):
        eng = MB.MadaKV(n_layers=NL, batch=B, n_q_heads=H, n_kv_heads=H, head_dim=d, ctx_len=L, window=W, budget=200, max_new_tokens=0, cache_fp8=4, device=DEV)
        if fused:
            eng.evict(0, NL, q, k, v, mask)
        else:
            for l in range(NL):
                eng.score(l, 1, q[l:l + 1], k[l:l + 1], mask)
                eng.allocate(l, 1)
                eng.select_gather(l, 1, k[l:l + 1], v[l:l + 1], mask)
        torch.cuda.synchronize()
        got.append([t.clone() for t in (eng.kept_idx, eng.kv_off, eng.kv_len, eng.k_c, eng.v_c)])
        eng.close()
    assert all(torch.equal(a, b) for a, b in zip(*got))             # (no free rows: every byte belongs to a head)


@pytest.mark.parametrize("d", [128, 64])
def test_rows_far_into_a_large_cache(d):
    """Segments behind the first 4 GiB of codes and the first 2^31 / d rows of values: the last layer's heads of a cache of 71 M
    (142 M) rows, set up by hand."""
    NL, B, H, Hq, L = (64 if d == 128 else 128), 16, 64, 64, 1080
    eng = MB.MadaKV(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=4, budget=L, max_new_tokens=2, cache_fp8=4, layers_per_call=1, device=DEV)
    args = dict(n_layers=1, batch=B, n_kv_heads=H, n_q_heads=Hq, head_dim=d, cache_fp8=4)
    assert eng.capacity * (d // 2) > 1 << 32
    per = eng.capacity // B                                       # a batch item's region; the layer's heads are at its end
    off = torch.zeros(1, B, H, dtype=torch.int64)
    for b in range(B):
        for h in range(H):
            off[0, b, h] = (b + 1) * per - (H - h) * (L + 2)
    lens = torch.randint(200, 600, (1, B, H), generator=torch.Generator().manual_seed(1)).int()
    eng.kv_off[NL - 1:].copy_(off), eng.kv_len[NL - 1:].copy_(lens)
    g = torch.Generator(device=DEV).manual_seed(2)
    heads = [(0, 0), (B - 1, H - 1), (B - 1, 0), (B // 2, 7)]
    src = {}
    for b, h in heads:
        o, n = int(off[0, b, h]), int(lens[0, b, h])
        for name, cache in (("k", eng.k_c), ("v", eng.v_c)):
            x = torch.randn(n, d, generator=g, device=DEV).to(torch.bfloat16)
            code, scale = O.quantize_mx4(x.cpu().double().numpy())
            cache[o * (d // 2):(o + n) * (d // 2)] = torch.from_numpy(code).view(-1).to(DEV)
            at = eng.capacity * (d // 2) + o * (d // 32)
            cache[at:at + n * (d // 32)] = torch.from_numpy(scale).view(-1).to(DEV)
            src[b, h, name] = stored(x, 4)
    q, kn, vn = (torch.randn(1, B, x, d, generator=g, device=DEV).to(torch.bfloat16) for x in (Hq, H, H))
    out = torch.zeros(1, B, Hq, d, device=DEV)
    acc = torch.zeros(eng.capacity, device=DEV)
    slot, pos = torch.zeros(B * H, dtype=torch.int32, device=DEV), torch.full((B,), 5000, dtype=torch.int32, device=DEV)
    say(f"large cache d={d}: append")
    eng.decode_attn_weights(NL - 1, 1, q, kn, vn, out, acc, acc, slot_out=slot, pos=pos)
    torch.cuda.synchronize()
    for b, h in heads:
        o, n = int(off[0, b, h]), int(lens[0, b, h])
        k, v = (torch.cat([src[b, h, x], stored(t[0, b, h][None], 4)]) for x, t in (("k", kn), ("v", vn)))
        ref, w = attention(q[0, b, h:h + 1], k, v, d)
        assert float((out[0, b, h].cpu().double() - ref[0]).abs().max()) < 1e-4
        assert float((acc[o:o + n + 1].cpu().double() - w[0]).abs().max()) < 5e-5
        assert int(eng.kept_idx[o + n]) == 5000
        src[b, h, "k"], src[b, h, "v"] = k, v
    rows = [torch.zeros(eng.capacity, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    eng.cache_rows(NL - 1, 1, *rows)
    torch.cuda.synchronize()
    for b, h in heads:
        o, n = int(off[0, b, h]), int(lens[0, b, h]) + 1
        for x, t in zip("kv", rows):
            assert torch.equal(t[o:o + n].cpu().double(), src[b, h, x])
    eng.close()
