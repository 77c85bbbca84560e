"""Prompt attention and the calls of drafted trees on the host: what they refuse before anything is enqueued, what they enqueue, and how
many appended rows a layer counts afterwards.  No GPU: the library runs on a runtime that only keeps a log."""
import pytest

from paper_2506_15724_amd import binding as MB
from tests.test_abi import good
from tests.test_host_calls import runtime, scenario  # noqa: F401  (a fixture)

ARGS = """
def addr(x): return 0 if x is None else x.p if isinstance(x, Room) else x
ptr = lambda x: P(addr(x))
at = lambda d: Room.at + (1 << 30) + d            # an address with an offset
def given(kw, *names): return [ptr(T() if kw.get(x, 1) == 1 else kw[x]) for x in names]
def attn(h, l0=0, n=1, n_seq=0, **kw):
    kw.setdefault("off", None); kw.setdefault("lse", None)
    q, k, v, off, out, lse = given(kw, "q", "k", "v", "off", "out", "lse")
    return lib.madakv_prompt_attn(h, I(l0), I(n), q, k, v, off, I(n_seq), out, lse, P(0))
def tree(h, l0=0, n=1, t=4, size=1 << 40, st=None, **kw):
    return lib.madakv_tree_attn(h, I(l0), I(n), I(t), *given(kw, "q", "kn", "vn", "tree", "kc", "vc", "off", "ln", "out", "ws"), Z(size), ptr(st))
def commit(h, l0=0, n=1, t=4, deep=4, most=4, st=None, **kw):
    kn, vn, path, count, start, kc, vc, off, ln = given(kw, "kn", "vn", "path", "count", "start", "kc", "vc", "off", "ln")
    return lib.madakv_tree_commit(h, I(l0), I(n), I(t), kn, vn, path, count, I(deep), start, I(most), kc, vc, off, ln, ptr(st))
def need(h, n, t):
    b = Z()
    assert lib.madakv_tree_attn_workspace_bytes(h, I(n), I(t), C.byref(b)) == 0
    return b.value
append = lambda h, l=0: lib.madakv_decode_attn(h, I(l), I(1), *[P(T().p) for _ in range(8)], P(T().p), Z(1 << 40), P(0))
kinds = lambda: [x.rest[3] if x.kind == "launch" else x.kind for x in log()]
"""


def test_prompt_attention_refuses(runtime):  # noqa: F811
    out = scenario(runtime, ARGS + """
for h in map(create, sys.argv[3:]):
    log()
    for kw in [dict(l0=2), dict(l0=-1), dict(n=3), dict(n=0), *[{x: None} for x in ("q", "k", "v", "out")], *[{x: at(8)} for x in ("q", "k", "v", "out")], dict(lse=at(2)),
               dict(off=1), dict(off=1, n_seq=-1), dict(n_seq=1), dict(off=at(2), n_seq=1)]:
        assert attn(h, **kw) == -1, kw
    assert attn(None) == -1 and not log()
    for kw in (dict(), dict(lse=1), dict(off=1, n_seq=1), dict(off=1, n_seq=1000, n=2, lse=1)):
        assert attn(h, **kw) == 0
        k = kinds()
        assert len(k) == 1 and "prompt_attn" in k[0], k
print("ok")
""", good(), good(dtype=MB.FP32, head_dim=64, window=16), good(out_fp32=0, head_dim=64, n_q_heads=32, batch=64))
    assert out.strip() == "ok"


def test_tree_attention_refuses(runtime):  # noqa: F811
    out = scenario(runtime, ARGS + """
for h in map(create, sys.argv[3:]):
    log()
    names = ("q", "kn", "vn", "kc", "vc", "out", "ws")
    for kw in [dict(l0=2), dict(n=3), dict(n=0), *[{x: None} for x in names + ("tree", "off", "ln")], *[{x: at(8)} for x in names], dict(tree=at(4)), dict(off=at(4)), dict(ln=at(2))]:
        assert tree(h, **kw) == -1, kw
    assert tree(None) == -1
    for t in (0, 65, -1): assert tree(h, t=t) == -2 and lib.madakv_tree_attn_workspace_bytes(h, I(1), I(t), C.byref(Z())) == -1
    for t in (1, 64):
        if need(h, 1, t) > 16: assert tree(h, t=t, size=15) == -4
    assert lib.madakv_tree_attn_workspace_bytes(h, I(1), I(1), None) == -1 and lib.madakv_tree_attn_workspace_bytes(None, I(1), I(1), C.byref(Z())) == -1
    for n in (0, 3): assert lib.madakv_tree_attn_workspace_bytes(h, I(n), I(1), C.byref(Z())) == -1
    assert not log(), "nothing is enqueued"
    for t in (1, 4, 5, 16, 64):
        for n in (1, 2):
            assert tree(h, n=n, t=t, size=need(h, 2, 64)) == 0
            k = kinds()
            k = [x for x in k if x != "query"]
            assert "tree_attn" in k[0] or "tree_narrow" in k[0], k
            assert [("tree_join" in x) for x in k[1:]] in ([], [True]), k
print("ok")
""", good(), good(dtype=MB.FP32, head_dim=64, window=16), good(cache_fp8=1, out_fp32=0), good(cache_fp8=4, n_q_heads=64, window=8, page_rows=16))
    assert out.strip() == "ok"


@pytest.mark.parametrize("L,budget", [(2, 2), (513, 100), (131072, 2048), (1 << 20, 1 << 20)])
@pytest.mark.parametrize("Hq,H,B", [(1, 1, 1), (8, 1, 1), (28, 4, 2), (32, 32, 4)])
def test_workspaces_serve_smaller_calls(runtime, L, budget, Hq, H, B):  # noqa: F811
    """Fewer layers, and smaller trees."""
    scenario(runtime, ARGS + """
h = create(sys.argv[3])
last = 0
for n in (1, 2, 5, 9):
    for t in (1, 3, 8, 33, 64):
        size = need(h, n, t)
        for m in range(1, n + 1):
            for s in range(1, t + 1):
                assert tree(h, n=m, t=s, size=size) == 0
        log()
""", good(n_layers=9, batch=B, n_q_heads=Hq, n_kv_heads=H, ctx_len=L, window=1, budget=budget))


def test_commit_refuses_and_counts(runtime):  # noqa: F811
    out = scenario(runtime, ARGS + """
h, paged = map(create, sys.argv[3:])
for x in (h, paged):
    log()
    for kw in [dict(l0=2), dict(n=3), dict(n=0), *[{y: None} for y in ("kn", "vn", "path", "count", "start", "kc", "vc", "off", "ln")], *[{y: at(8)} for y in ("kn", "vn", "kc", "vc")],
               dict(path=at(2)), dict(count=at(1)), dict(start=at(2)), dict(off=at(4)), dict(ln=at(2)), dict(most=-1), dict(most=5)]:
        assert commit(x, **kw) == -1, kw
    for kw in (dict(t=0), dict(t=65), dict(deep=0), dict(deep=65)): assert commit(x, **kw) == -2, kw
    assert commit(None) == -1 and not log(), "nothing is enqueued"
# `most` rows count as appended: of four, decode may append what is left
assert commit(h, most=3) == 0 and ["tree_commit" in y for y in kinds()] == [True]
assert append(h) == 0 and append(h) == -1 and append(h, 1) == 0
assert commit(h, most=2, n=2) == 0 and append(h) == 0 and append(h) == 0 and append(h) == -1
assert append(h, 1) == 0 and append(h, 1) == 0 and append(h, 1) == -1
# rows of a paged cache are not taken back
assert commit(paged, most=3) == 0 and commit(paged, most=1) == 0 and append(paged) == 0 and append(paged) == -1
# an eviction starts anew
assert lib.madakv_select_gather(h, I(0), I(1), *[P(T().p) for _ in range(10)], P(T().p), Z(1 << 40), P(0)) == 0
assert append(h) == 0
# one that did not reach the device counts nothing
fake.fake_fail(b"tree_commit")
assert commit(h, l0=1, most=0) == -6
fake.fake_fail(b"")
assert append(h, 1) == -1
print("ok")
""", good(), good(page_rows=16))
    assert out.strip() == "ok"


def test_captured_commit(runtime):  # noqa: F811
    """Nobody tells the host of replays: calls that look at whatever a head holds cover all the rows there is room for."""
    out = scenario(runtime, ARGS + """
h = create(sys.argv[3])
assert lib.madakv_select_gather(h, I(0), I(2), *[P(T().p) for _ in range(10)], P(T().p), Z(1 << 40), P(0)) == 0
fake.fake_events_done(1)
log()
grid = lambda: [x.rest[1] for x in log() if x.kind == "launch" and "tree_join" not in x.rest[3]][-1]
assert tree(h) == 0
short = grid()
s = 0x77000
fake.fake_capture(P(s))
assert tree(h, st=s) == 0
room = grid()
assert commit(h, st=s, most=0) == 0
fake.fake_capture(P(0))
log()
assert tree(h) == 0 and grid() == room != short
assert tree(h, l0=1) == 0 and grid() == short
print("ok")
""", good(n_q_heads=1, n_kv_heads=1, ctx_len=2048, budget=1000, max_new_tokens=1000))
    assert out.strip() == "ok"


def test_pieces_of_lopsided_caches(runtime):  # noqa: F811
    """Heads that may be far longer than the typical one: not more pieces than the chip takes at once."""
    out = scenario(runtime, ARGS + """
h = create(sys.argv[3])
for t in (1, 8, 64):
    assert need(h, 1, t) <= 8 * 512 * 8 * 64 * (128 + 2) * 4, need(h, 1, t)
    log()
    assert tree(h, t=t) == 0
print("ok")
""", good(n_q_heads=64, n_kv_heads=8, ctx_len=1 << 20, budget=2000, hcc_rho=1024))
    assert out.strip() == "ok"
