"""GPU: attention of whole prompts against plain arithmetic in 64 bits: around every block and tile size, one, padded and packed
sequences, logits that leave their references behind, undefined numbers where nobody looks, in graphs, and with the calls that follow."""
import math

import numpy as np
import pytest
import torch

from paper_2506_15724_amd import binding as MB

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(msg):
    print(f"[prompt_attn] {msg}", flush=True)


def engine(L, Hq, H, d, B=1, NL=1, dtype="bf16", out_fp32=1, **kw):
    return MB.MadaKV(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=1, budget=L, dtype=dtype, out_fp32=out_fp32, device=DEV, **kw)


def inputs(eng, seed=0, spread=1.5):
    c = eng.cfg
    g = torch.Generator(device=DEV).manual_seed(seed)
    shape = lambda h: (c.n_layers, c.batch, h, c.ctx_len, c.head_dim)      # noqa: E731
    q, k, v = (torch.randn(*shape(h), generator=g, device=DEV) for h in (c.n_q_heads, c.n_kv_heads, c.n_kv_heads))
    return (spread * q).to(eng.tdtype), k.to(eng.tdtype), v.to(eng.tdtype)


def reference(q, k, v, lo, hi, scale):
    """(out, lse, weighted |v|, largest sum of |q_i k_i|) of the rows [lo, hi) of one head, in 64 bits."""
    q, k, v = (x[lo:hi].double() for x in (q, k, v))
    s = q @ k.t().contiguous() * scale
    size = float((q.abs() @ k.abs().t().contiguous()).max()) * scale
    s = s + torch.full_like(s, -math.inf).triu_(1)
    w = torch.softmax(s, -1)
    return w @ v, torch.logsumexp(s, -1), w @ v.abs(), size


def bounds(eng, n, size, ref, spent, lse):
    """How far a row's output and its normaliser may be off.  A logit is a sum of d exact products in 32 bits and a product with the
    scale: d + 2 roundings of 2^-24 of the sum of their magnitudes.  A weight has that, twice (its own logit, the reference's), and
    a few roundings of exp2 and of the parts it enters the product in; sums of n weights, and of n weighted rows, n roundings each.  bf16 outputs:
    weights rounded to bf16 (2^-8 of each), and the output."""
    u = 2.0 ** -24
    rel = 2 * (eng.cfg.head_dim + 2) * u * size + 2 * (n + 16) * u
    tol = rel * spent
    if eng._out_dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (1 + rel) * spent + 2.0 ** -8 * (ref.abs() + tol)
    return tol + 1e-30, (eng.cfg.head_dim + 2) * u * size + (n + 16) * u + 2 * u * lse.abs()


def check(eng, q, k, v, out, lse, off=None, heads=None):
    """Every row of a sequence by the reference, the others as they were (-77)."""
    c = eng.cfg
    G, scale = c.n_q_heads // c.n_kv_heads, c.softmax_scale or 1 / math.sqrt(c.head_dim)
    for l in range(c.n_layers):
        for b in range(c.batch):
            ends = [0, c.ctx_len] if off is None else off[b].tolist()
            inside = torch.zeros(c.ctx_len, dtype=torch.bool, device=DEV)
            inside[ends[0]:ends[-1]] = True
            assert (out[l, b][:, ~inside] == -77).all() and (lse[l, b][:, ~inside] == -77).all()
            for j in (range(c.n_q_heads) if heads is None else heads):
                for lo, hi in zip(ends[:-1], ends[1:]):
                    if lo == hi:
                        continue
                    ref, n, spent, size = reference(q[l, b, j], k[l, b, j // G], v[l, b, j // G], lo, hi, scale)
                    tol, ltol = bounds(eng, hi - lo, size, ref, spent, n)
                    err, lerr = (out[l, b, j, lo:hi].double() - ref).abs(), (lse[l, b, j, lo:hi].double() - n).abs()
                    assert bool((err <= tol).all()), (l, b, j, lo, hi, float((err / tol).max()), (err > tol).nonzero()[:4].tolist())
                    assert bool((lerr <= ltol).all()), (l, b, j, lo, hi, float((lerr / ltol).max()))


def run(eng, q, k, v, off=None, **kw):
    c = eng.cfg
    out = torch.full((c.n_layers, c.batch, c.n_q_heads, c.ctx_len, c.head_dim), -77.0, dtype=eng._out_dtype, device=DEV)
    lse = torch.full((c.n_layers, c.batch, c.n_q_heads, c.ctx_len), -77.0, device=DEV)
    eng.prompt_attn(0, c.n_layers, q, k, v, out, row_lse=lse, seq_off=off, **kw)
    torch.cuda.synchronize()
    return out, lse


SHAPES = [(2, 1, 1, 64), (31, 2, 1, 128), (33, 3, 3, 64), (64, 2, 2, 128), (65, 4, 2, 64), (127, 7, 1, 128), (128, 2, 2, 64), (129, 3, 1, 128), (193, 2, 1, 64), (255, 2, 2, 128),
          (257, 8, 1, 64), (300, 6, 3, 128), (513, 4, 4, 64), (700, 2, 1, 128), (1301, 7, 1, 64)]


@pytest.mark.parametrize("kind", ["bf16", "fp32 out", "fp32"])
@pytest.mark.parametrize("L,Hq,H,d", SHAPES)
def test_one_sequence(L, Hq, H, d, kind):
    say(f"one L={L} {Hq}/{H} d={d} {kind}")
    eng = engine(L, Hq, H, d, dtype="fp32" if kind == "fp32" else "bf16", out_fp32=int(kind != "bf16"))
    q, k, v = inputs(eng, L)
    check(eng, q, k, v, *run(eng, q, k, v))


@pytest.mark.parametrize("out_fp32", [0, 1])
@pytest.mark.parametrize("L,Hq,H,d,B,NL", [(517, 32, 8, 128, 4, 1), (1030, 32, 32, 64, 1, 2), (700, 28, 4, 128, 2, 2), (257, 32, 8, 64, 4, 2), (2111, 32, 4, 128, 1, 1)])
def test_many_rows(L, Hq, H, d, B, NL, out_fp32):
    """Launches that fill the chip take larger blocks of rows."""
    say(f"many L={L} {Hq}/{H} d={d} B={B} n={NL} out_fp32={out_fp32}")
    eng = engine(L, Hq, H, d, B, NL, out_fp32=out_fp32)
    q, k, v = inputs(eng, L)
    check(eng, q, k, v, *run(eng, q, k, v), heads=[0, Hq // 2 + 1, Hq - 1])


OFFSETS = [(300, [[0, 300], [37, 300], [300, 300]]), (300, [[0, 1, 2, 2, 130, 131, 299], [5, 5, 69, 70, 70, 200, 300], [0, 0, 0, 0, 0, 0, 0]]), (700, [[0, 64, 128, 192, 640, 700], [3, 31, 33, 95, 97, 650], [0, 256, 257, 511, 512, 700]]),
           (513, [[0, 513, 513], [512, 513, 513], [0, 1, 513]])]


@pytest.mark.parametrize("kind", ["bf16", "fp32 out", "fp32"])
@pytest.mark.parametrize("L,ends", OFFSETS)
@pytest.mark.parametrize("Hq,H,d", [(4, 2, 128), (48, 48, 64), (96, 32, 128)])
def test_several_sequences(L, ends, Hq, H, d, kind):
    """Packed and padded; what no row may look at is no number: positions of no sequence, and behind the first half of a sequence's rows its last row of V."""
    if kind == "fp32" and Hq > 48:
        pytest.skip("one block size for 32-bit rows")
    say(f"several L={L} {Hq}/{H} d={d} {kind}")
    eng = engine(L, Hq, H, d, B=3, dtype="fp32" if kind == "fp32" else "bf16", out_fp32=int(kind != "bf16"))
    q, k, v = inputs(eng, L)
    off = torch.tensor(ends, dtype=torch.int32, device=DEV)
    for b in range(3):
        for x in (q, k, v):
            x[:, b, :, :ends[b][0]], x[:, b, :, ends[b][-1]:] = math.nan, math.nan
    check(eng, q, k, v, *run(eng, q, k, v, off), off=off, heads=[0, Hq - 1] if Hq > 4 else None)


@pytest.mark.parametrize("NL,B,Hq,H,L,d", [(1, 3, 16, 8, 150, 64), (2, 1, 5, 5, 70, 128), (1, 2, 28, 4, 200, 64), (1, 1, 20, 20, 2600, 64), (3, 1, 12, 2, 130, 128), (1, 4, 32, 8, 600, 64),
                                           (1, 1, 1, 1, 1100, 64), (2, 2, 7, 1, 1000, 64), (1, 2, 24, 24, 1290, 128), (1, 1, 3, 1, 17000, 64)])
def test_every_head(NL, B, Hq, H, L, d):
    """All heads and blocks of rows have their workgroup, whichever way they are dealt to the XCDs; items of different lengths."""
    say(f"every head n={NL} B={B} {Hq}/{H} L={L} d={d}")
    eng = engine(L, Hq, H, d, B, NL, out_fp32=0)
    q, k, v = inputs(eng, L)
    out, lse = run(eng, q, k, v)
    assert bool((lse != -77).all())
    if L < 5000:
        check(eng, q, k, v, out, lse)
    off = torch.tensor([[L * b // (B + 1), L - b] for b in range(B)], dtype=torch.int32, device=DEV)
    out, lse = run(eng, q, k, v, off)
    if L < 5000:
        check(eng, q, k, v, out, lse, off=off)
    assert bool(((lse != -77) == torch.stack([(torch.arange(L, device=DEV) >= o[0]) & (torch.arange(L, device=DEV) < o[1]) for o in off])[None, :, None]).all())


def test_many_short_sequences():
    L = 1500
    say("many short sequences")
    eng = engine(L, 48, 8, 128, out_fp32=0)
    q, k, v = inputs(eng, 3)
    r = np.random.default_rng(5)
    off = torch.from_numpy(np.concatenate([[0], np.sort(r.integers(0, L - 20, 700)), [L - 20]]).astype(np.int32))[None].to(DEV)
    check(eng, q, k, v, *run(eng, q, k, v, off), off=off, heads=[0, 47])


@pytest.mark.parametrize("Hq", [2, 128])
@pytest.mark.parametrize("kind", ["bf16", "fp32 out", "fp32"])
def test_undefined_rows_behind_a_query(Hq, kind):
    """K and V of one position are no numbers: rows in front of it, and of other sequences, have what they had without."""
    if kind == "fp32" and Hq > 2:
        pytest.skip("one block size for 32-bit rows")
    say(f"undefined {Hq} {kind}")
    eng = engine(520, Hq, 1 if Hq == 2 else 16, 128, dtype="fp32" if kind == "fp32" else "bf16", out_fp32=int(kind != "bf16"))
    off = torch.tensor([[0, 200, 520]], dtype=torch.int32, device=DEV)
    q, k, v = inputs(eng, 9)
    plain, plain_lse = run(eng, q, k, v, off)
    for at, what, x in ((150, math.nan, v), (333, math.inf, v), (70, -math.inf, v), (401, math.nan, k), (199, math.inf, k)):
        y = x.clone()
        y[:, :, :, at] = what
        out, lse = run(eng, q, y if x is k else k, y if x is v else v, off)
        end = 200 if at < 200 else 520
        same = torch.ones(520, dtype=torch.bool, device=DEV)
        same[at:end] = False
        # (the masked part of a tile is added one by one then: 32 additions in another order)
        a, b = out[:, :, :, same].double(), plain[:, :, :, same].double()
        assert bool(((a - b).abs() <= 2.0 ** (-7 if kind == "bf16" else -17) * (1 + b.abs())).all()), (at, what)
        assert torch.equal(lse[:, :, :, same], plain_lse[:, :, :, same])
        got = out[:, :, :, at:end]
        if x is v:
            assert bool((~torch.isfinite(got)).all()) and (bool(torch.isnan(got).all()) or not math.isnan(what))
            if math.isinf(what):
                assert bool((got == what).all()), (at, what)
            assert torch.equal(lse, plain_lse)
        elif math.isnan(what):
            assert bool(torch.isnan(got).all()) and bool(torch.isnan(lse[:, :, :, at:end]).all())


@pytest.mark.parametrize("Hq", [2, 128])
@pytest.mark.parametrize("how", ["rising", "steps", "falling", "huge", "equal", "zero"])
def test_logits_that_move(Hq, how):
    """References that are left behind in every tile, far ones, logits of thousands, all the same."""
    L, d = 700, 64
    say(f"moving {how} {Hq}")
    eng = engine(L, Hq, 1 if Hq == 2 else 16, d)
    q, k, v = inputs(eng, 4, spread=0.3)
    at = torch.arange(L, device=DEV).view(1, 1, 1, L)
    ramp = {"rising": at * 0.5, "steps": (at // 100) * 40.0, "falling": -at * 1.0, "huge": torch.where(at % 97 == 5, 3000.0, 0.0), "equal": at * 0 + 1.0, "zero": at * 0.0}[how]
    q[..., 0], k[..., 0] = 8.0, ramp.to(k.dtype)
    if how == "equal":
        k[..., 1:] = 0
    if how == "zero":
        q.zero_()
    check(eng, q, k, v, *run(eng, q, k, v), heads=[0, Hq - 1])


def test_normalisers_go_into_prompt_scores():
    """row_lse is what madakv_score_prompt asks for; of a padded batch, +infinity counts nothing."""
    say("normalisers")
    eng = engine(900, 12, 4, 128, B=2, out_fp32=0)
    q, k, v = inputs(eng, 6)
    out, lse = run(eng, q, k, v)
    eng.score_prompt(0, 1, q, k)
    want = eng.psi.clone()
    eng.score_prompt(0, 1, q, k, row_lse=lse)
    assert bool(((eng.psi - want).abs() <= 4e-4 * want).all())        # (2e-4 for each, as those of the plain sum)
    off = torch.tensor([[0, 900], [0, 555]], dtype=torch.int32, device=DEV)
    lse.fill_(math.inf)
    eng.prompt_attn(0, 1, q, k, v, out, row_lse=lse, seq_off=off)
    eng.score_prompt(0, 1, q, k, row_lse=lse)
    torch.cuda.synchronize()
    assert bool(((eng.psi[:, 0] - want[:, 0]).abs() <= 4e-4 * want[:, 0]).all()) and bool((eng.psi[:, 1, :, 555:] == 0).all())
    few = engine(555, 12, 4, 128, out_fp32=0)
    few.score_prompt(0, 1, q[:, 1:, :, :555].contiguous(), k[:, 1:, :, :555].contiguous())
    assert bool(((eng.psi[:, 1, :, :555] - few.psi[:, 0]).abs() <= 4e-4 * few.psi[:, 0]).all())


@pytest.mark.parametrize("Hq", [4, 128])
def test_captured_and_replayed(Hq):
    say(f"captured {Hq}")
    eng = engine(600, Hq, 2 if Hq == 4 else 16, 64, out_fp32=0)
    q, k, v = inputs(eng, 1)
    off = torch.tensor([[0, 100, 600]], dtype=torch.int32, device=DEV)
    out, lse = run(eng, q, k, v, off)
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        eng.prompt_attn(0, 1, q, k, v, out, row_lse=lse, seq_off=off)
    for i in range(4):
        for x, y in zip((q, k, v), inputs(eng, 10 + i)):
            x.copy_(y)
        off.copy_(torch.tensor([[i, 100 + 77 * i, 600 - i]]))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        again, again_lse = run(eng, q, k, v, off)
        assert torch.equal(out[:, :, :, i:600 - i], again[:, :, :, i:600 - i]) and torch.equal(lse[..., i:600 - i], again_lse[..., i:600 - i])


def test_layers_alone_and_together():
    """One call over all layers is the calls over each, without the normalisers too, on another stream."""
    say("layers")
    eng = engine(333, 8, 2, 128, B=2, NL=3, out_fp32=0)
    q, k, v = inputs(eng, 2)
    out, lse = run(eng, q, k, v)
    for l in range(3):
        one = torch.empty_like(out[l:l + 1])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eng.prompt_attn(l, 1, q[l:l + 1], k[l:l + 1], v[l:l + 1], one)
        side.synchronize()
        assert torch.equal(one[0], out[l])


def test_holder_refuses():
    say("refusals")
    eng = engine(100, 4, 2, 64, B=2, out_fp32=0)
    q, k, v = inputs(eng)
    out, lse = torch.zeros_like(q), torch.zeros(1, 2, 4, 100, device=DEV)
    good = dict(q=q, k=k, v=v, out=out, row_lse=lse, seq_off=torch.tensor([[0, 9], [0, 100]], dtype=torch.int32, device=DEV))
    for bad in (dict(q=q.float()), dict(k=k[:, :, :1]), dict(v=v.cpu()), dict(out=out.float()), dict(out=out[..., :32]), dict(row_lse=lse.double()), dict(row_lse=lse[..., :9]),
                dict(seq_off=good["seq_off"].long()), dict(seq_off=good["seq_off"][:1]), dict(seq_off=good["seq_off"][:, :1]), dict(seq_off=good["seq_off"].cpu()),
                dict(seq_off=good["seq_off"].view(-1))):
        with pytest.raises((ValueError, AssertionError)):
            eng.prompt_attn(0, 1, **{**good, **bad})
    for l0, n in ((1, 1), (0, 2), (-1, 1), (0, 0)):
        with pytest.raises((MB.MadaKVError, ValueError)):
            eng.prompt_attn(l0, n, **good)
    assert not out.any() and not lse.any()
