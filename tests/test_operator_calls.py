"""The calls around the 4-bit cache, accumulated weights and prompt scores on the host: what they refuse before anything is
enqueued, and what they enqueue.  No GPU: the library runs on a runtime that only keeps a log."""
import ctypes as C

import pytest

from paper_2506_15724_amd import binding as MB
from tests.test_abi import good
from tests.test_host_calls import runtime, scenario  # noqa: F401  (a fixture)

ARGS = """
def addr(x): return 0 if x is None else x.p if isinstance(x, Room) else x
ptr = lambda x: P(addr(x))
def weights(h, l0=0, n=1, q=1, kn=1, vn=1, kc=1, vc=1, off=1, ln=1, out=1, a0=1, a1=1, decay=1.0, s0=None, s1=None, kept=None, pos=None, recent=0, ws=1, size=1 << 40, st=None):
    t = [T() if x == 1 else x for x in (q, kn, vn, kc, vc, off, ln, out, a0, a1)]
    u = [T() if x == 1 else x for x in (s0, s1, kept, pos)]
    return lib.madakv_decode_attn_weights(h, I(l0), I(n), *map(ptr, t), C.c_float(decay), *map(ptr, u), I(recent), ptr(T() if ws == 1 else ws), Z(size), ptr(st))
def prompt(h, l0=0, n=1, q=1, k=1, mask=None, lse=None, psi=1, pool=None, stats=None, nmod=None, ws=1, size=1 << 40):
    t = [T() if x == 1 else x for x in (q, k, mask, lse, psi, pool, stats, nmod)]
    return lib.madakv_score_prompt(h, I(l0), I(n), *map(ptr, t), ptr(T() if ws == 1 else ws), Z(size), P(0))
def rows(h, l0=0, n=1, **kw):
    t = [T() if kw.get(x, 1) == 1 else kw[x] for x in ("kc", "vc", "off", "ln", "kr", "vr")]
    return lib.madakv_cache_rows(h, I(l0), I(n), *map(ptr, t), P(0))
kinds = lambda: [x.rest[3] if x.kind == "launch" else x.kind for x in log()]
"""


def test_decode_with_weights_refuses(runtime):  # noqa: F811
    out = scenario(runtime, ARGS + """
h = create(sys.argv[3])
log()
at = lambda d: Room.at + (1 << 30) + d            # an address with an offset
bad = [dict(l0=2), dict(n=3), dict(n=0), dict(q=None), dict(kc=None), dict(vc=at(8)), dict(off=at(4)), dict(ln=at(2)), dict(out=None), dict(a0=None), dict(a1=None), dict(a1=at(2)),
       dict(kn=None), dict(vn=None), dict(kn=at(4)), dict(decay=-0.1), dict(decay=1.5), dict(decay=float("nan")), dict(recent=-1), dict(s0=1, kn=None, vn=None), dict(s1=1), dict(kept=1),
       dict(pos=1), dict(s0=at(2)), dict(s1=at(1), kept=1, pos=1), dict(kept=at(2), pos=1), dict(kept=1, pos=at(2)), dict(ws=None), dict(ws=at(8)), dict(size=(1 << 64) - 1)]
for kw in bad:
    assert weights(h, **kw) == -1, kw
b = Z()
assert lib.madakv_decode_attn_weights_workspace_bytes(h, I(1), C.byref(b)) == 0
assert weights(h, size=b.value - 1) == -4
for n, out in ((0, C.byref(b)), (3, C.byref(b)), (1, None)):
    assert lib.madakv_decode_attn_weights_workspace_bytes(h, I(n), out) == -1
assert lib.madakv_decode_attn_weights_workspace_bytes(None, I(1), C.byref(b)) == -1 and weights(None) == -1
assert not log(), "nothing is enqueued"
# four rows can be appended, as with madakv_decode_attn; replacing takes none of them
for i in range(4): assert weights(h) == 0 and weights(h, s0=1) == 0 and weights(h, kn=None, vn=None) == 0
assert weights(h) == -1 and lib.madakv_decode_attn(h, I(0), I(1), *[P(T().p) for _ in range(8)], P(T().p), Z(1 << 40), P(0)) == -1
assert weights(h, s0=1) == 0
k = kinds()
assert len(k) == 26 and all("decode" in x for x in k[::2]) and all("row_weights" in x for x in k[1::2]), k
print("ok")
""", good())
    assert out.strip() == "ok"


def test_replaced_rows_are_not_reevicted(runtime):  # noqa: F811
    """Until an eviction has laid the rows out anew: by layer, by either eviction call."""
    out = scenario(runtime, ARGS + """
h = create(sys.argv[3])
re = lambda l, n: lib.madakv_reevict(h, I(l), I(n), *[P(T().p) for _ in range(8)], P(T().p), Z(1 << 40), P(0))
assert re(0, 2) == 0
assert weights(h, l0=1, s0=1) == 0
assert re(0, 2) == -1 and re(1, 1) == -1 and re(0, 1) == 0
assert lib.madakv_select_gather(h, I(1), I(1), *[P(T().p) for _ in range(10)], P(T().p), Z(1 << 40), P(0)) == 0
assert re(0, 2) == 0
assert weights(h, l0=0, n=2, s0=1) == 0 and re(1, 1) == -1
assert lib.madakv_evict(h, I(0), I(2), *[P(T().p) for _ in range(14)], P(T().p), Z(1 << 40), P(T().p), Z(1 << 40), P(0)) == 0
assert re(0, 2) == 0
print("ok")
""", good())
    assert out.strip() == "ok"


def test_prompt_scores_refuse(runtime):  # noqa: F811
    out = scenario(runtime, ARGS + """
h, f = create(sys.argv[3]), create(sys.argv[4])
log()
at = lambda d: Room.at + (1 << 30) + d
rest = dict(mask=1, pool=1, stats=1, nmod=1)
bad = [dict(l0=-1), dict(n=3), dict(q=None), dict(k=None), dict(q=at(8)), dict(psi=None), dict(psi=at(2)), dict(lse=at(2)), dict(ws=None), dict(ws=at(4)),
       dict(mask=1), dict(pool=1), dict(stats=1), dict(nmod=1), dict(rest, mask=None), dict(rest, pool=None), dict(rest, stats=None), dict(rest, nmod=None),
       dict(rest, pool=at(2)), dict(rest, stats=at(2)), dict(rest, nmod=at(1))]
for kw in bad:
    assert prompt(h, **kw) == -1, kw
assert prompt(None) == -1 and prompt(f) == -7                    # fp32
b = Z()
assert lib.madakv_score_prompt_workspace_bytes(h, I(2), C.byref(b)) == 0
assert prompt(h, n=2, size=100) == -4
assert lib.madakv_score_prompt_workspace_bytes(h, I(0), C.byref(b)) == -1 and lib.madakv_score_prompt_workspace_bytes(None, I(1), C.byref(b)) == -1
assert lib.madakv_score_prompt_workspace_bytes(h, I(1), None) == -1
assert not log(), "nothing is enqueued"
for kw in (dict(), dict(lse=1), rest, dict(rest, lse=1)):
    for n in (1, 2):
        assert lib.madakv_score_prompt_workspace_bytes(h, I(2), C.byref(b)) == 0 and prompt(h, n=n, size=b.value, **kw) == 0
        k = kinds()
        sweeps = sum("prompt_sweep" in x for x in k)
        assert sweeps == (1 if "lse" in kw else 2) and ("stats_kernel" in str(k)) == ("mask" in kw), k
print("ok")
""", good(), good(dtype=MB.FP32, head_dim=64, window=16))
    assert out.strip() == "ok"


@pytest.mark.parametrize("L", [2, 65, 513, 8192, 131072, 1 << 20])
@pytest.mark.parametrize("Hq,H", [(1, 1), (8, 1), (28, 4), (32, 32)])
def test_prompt_workspace_serves_calls_over_fewer_layers(runtime, L, Hq, H):  # noqa: F811
    scenario(runtime, ARGS + """
h = create(sys.argv[3])
last = 0
for n in (1, 2, 3, 5, 9):
    b = Z()
    assert lib.madakv_score_prompt_workspace_bytes(h, I(n), C.byref(b)) == 0
    assert b.value >= last
    last = b.value
    for m in range(1, n + 1):
        assert prompt(h, n=m, size=b.value) == 0
""", good(n_layers=9, n_q_heads=Hq, n_kv_heads=H, ctx_len=L, window=1, budget=L))


def test_rows_of_the_cache_refuse(runtime):  # noqa: F811
    out = scenario(runtime, ARGS + """
h16, h8, h4 = (create(x) for x in sys.argv[3:])
log()
at = lambda d: Room.at + (1 << 30) + d
assert rows(h16) == -7 and rows(None) == -1
for h in (h8, h4):
    for kw in [dict(l0=2), dict(n=3), *[{x: None} for x in ("kc", "vc", "off", "ln", "kr", "vr")], dict(kc=at(8)), dict(off=at(4)), dict(ln=at(2)), dict(vr=at(4))]:
        assert rows(h, **kw) == -1, kw
assert not log()
assert rows(h8, n=2) == 0 and rows(h4, n=2) == 0
assert ["cache_rows" in x for x in kinds()] == [True, True]
print("ok")
""", good(), good(cache_fp8=1), good(cache_fp8=4))
    assert out.strip() == "ok"


def test_four_bit_cache_on_the_host(runtime):  # noqa: F811
    """Eviction, decode and re-eviction take a 4-bit cache (the last one reads K back first); other widths and fp32 are refused."""
    out = scenario(runtime, ARGS + """
h = create(sys.argv[3])
log()
assert lib.madakv_reevict(h, I(0), I(2), *[P(T().p) for _ in range(8)], P(T().p), Z(1 << 40), P(0)) == 0
k = [x for x in kinds() if x != "query"]
assert "cache_rows" in k[0] and "score" in k[1], k
b = Z()
assert lib.madakv_reevict_workspace_bytes(h, I(2), C.byref(b)) == 0
assert lib.madakv_reevict(h, I(0), I(2), *[P(T().p) for _ in range(8)], P(T().p), Z(b.value - 1), P(0)) == -4 and "launch" not in str(log())
assert lib.madakv_evict(h, I(0), I(2), *[P(T().p) for _ in range(14)], P(T().p), Z(1 << 40), P(T().p), Z(1 << 40), P(0)) == 0
log()
assert lib.madakv_decode_attn(h, I(0), I(1), *[P(T().p) for _ in range(8)], P(T().p), Z(1 << 40), P(0)) == 0
(k,) = [x for x in kinds() if x != "query"]
assert "decode_fp4" in k
print("ok")
""", good(cache_fp8=4))
    assert out.strip() == "ok"
    for kw, status in ((dict(cache_fp8=3), -1), (dict(cache_fp8=5), -1), (dict(cache_fp8=-1), -1), (dict(cache_fp8=4, dtype=MB.FP32, head_dim=64, window=16), -5)):
        h = C.c_void_p()
        assert MB.lib().madakv_create(C.byref(good(**kw)), C.byref(h)) == status and not h.value


def test_rows_replaced_by_replays_are_not_reevicted(runtime):  # noqa: F811
    """A captured replacing step replaces rows whenever its graph is replayed, also behind a later eviction."""
    out = scenario(runtime, ARGS + """
h = create(sys.argv[3])
st = 0x7000
re = lambda l, n: lib.madakv_reevict(h, I(l), I(n), *[P(T().p) for _ in range(8)], P(T().p), Z(1 << 40), P(0))
fake.fake_capture(P(st))
assert weights(h, l0=0, st=st) == 0                     # (appends: the layer can be re-evicted)
assert weights(h, l0=1, s0=1, st=st) == 0
fake.fake_capture(P(0))
assert re(0, 1) == 0 and re(1, 1) == -1
assert lib.madakv_select_gather(h, I(0), I(2), *[P(T().p) for _ in range(10)], P(T().p), Z(1 << 40), P(0)) == 0
assert re(0, 1) == 0 and re(1, 1) == -1 and re(0, 2) == -1
print("ok")
""", good())
    assert out.strip() == "ok"
