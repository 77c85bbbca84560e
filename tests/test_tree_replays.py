"""What the host knows of rows that captured tree commits leave whenever their graph is replayed, on the runtime that only keeps a log.  No GPU."""
import pytest

from tests.test_abi import good
from tests.test_host_calls import runtime, scenario  # noqa: F401  (a fixture)
from tests.test_tree_calls import ARGS

CALLS = ARGS + """
st = 0x77000
none = lambda: P(0)
evict = lambda h: lib.madakv_select_gather(h, I(0), I(2), *[P(T().p) for _ in range(10)], P(T().p), Z(1 << 40), P(0))
plain = lambda h, l=0, new=True: lib.madakv_decode_attn(h, I(l), I(1), P(T().p), *[P(T().p) if new else None for _ in range(2)], *[P(T().p) for _ in range(5)], P(T().p), Z(1 << 40), P(0))
static = lambda h, l=0: lib.madakv_decode_attn_static(h, I(l), I(1), *[P(T().p) for _ in range(8)], P(0))
weighed = lambda h, l=0: lib.madakv_decode_attn_weights(h, I(l), I(1), *[P(T().p) for _ in range(10)], C.c_float(1), None, None, None, None, I(0), P(T().p), Z(1 << 40), P(0))
def captured(f):
    fake.fake_capture(P(st))
    assert f() == 0
    fake.fake_capture(P(0))
def grid(part="decode"):
    (x,) = [x for x in log() if x.kind == "launch" and part in x.rest[3]]
    return [int(g) for g in x.rest[1].split(",")]
"""


@pytest.mark.parametrize("kw", [dict(), dict(page_rows=16), dict(cache_fp8=1), dict(cache_fp8=4), dict(n_q_heads=1)])
def test_decode_behind_replayed_commits(runtime, kw):  # noqa: F811
    """Lengths known, an eviction since the capture: a decode step has a workgroup for every piece that the rows of replays can make; the
    other layer's as before."""
    out = scenario(runtime, CALLS + """
h = create(sys.argv[3])
fake.fake_events_done(1)
assert evict(h) == 0
for f in (plain, static, weighed):
    log()
    assert f(h) == 0 and grid()[1] == 1              # (the runtime's eviction leaves heads of no rows)
captured(lambda: commit(h, most=3000, st=st))
assert evict(h) == 0
for f in (plain, static, weighed):
    log()
    assert f(h) == 0
    room = grid()[1]
    assert room * 1024 >= 3000, room
    assert f(h, 1) == 0 and grid()[1] == 1
log()
assert weighed(h) == 0 and grid("row_weights")[1] > 1
assert plain(h, new=False) == 0 and grid()[1] == room
print("ok")
""", good(**{**dict(n_q_heads=4, n_kv_heads=1, ctx_len=4000, budget=3000, max_new_tokens=3000, window=8), **kw}))
    assert out.strip() == "ok"


@pytest.mark.parametrize("kw", [dict(), dict(page_rows=16)])
def test_a_commit_that_is_only_captured_takes_no_rows_back(runtime, kw):  # noqa: F811
    """Three of four rows are there; a captured commit with a lower bound has not run yet, so one more fits.  A commit that is enqueued counts its bound
    (rows of a paged cache are not taken back)."""
    out = scenario(runtime, CALLS + """
h, paged = create(sys.argv[3]), int(sys.argv[4])
evict(h)
for _ in range(3): assert plain(h) == 0
captured(lambda: commit(h, most=1, st=st))
assert plain(h) == 0 and plain(h) == -1
captured(lambda: commit(h, most=1, st=st))
assert plain(h) == -1
assert commit(h, most=1) == 0 and plain(h) == (-1 if paged else 0)
evict(h)
captured(lambda: commit(h, most=3, st=st))
assert plain(h) == 0 and plain(h) == -1
print("ok")
""".replace("int(sys.argv[4])", str(bool(kw))), good(**kw))
    assert out.strip() == "ok"
