"""What the host knows of rows that a captured step appends whenever its graph is replayed, on the runtime that only keeps a log:
calls that look at all rows of a head cover every row that replays can have left.  No GPU."""
import pytest

from tests.test_abi import good
from tests.test_host_calls import runtime, scenario  # noqa: F401  (a fixture)
from tests.test_operator_calls import ARGS

CALLS = ARGS + """
st = 0x7000
evict = lambda h, n=2: lib.madakv_evict(h, I(0), I(n), *[P(T().p) for _ in range(14)], P(T().p), Z(1 << 40), P(T().p), Z(1 << 40), P(0))
plain = lambda h, l0=0, n=1, st=0: lib.madakv_decode_attn(h, I(l0), I(n), *[P(T().p) for _ in range(8)], P(T().p), Z(1 << 40), P(st))
def grids(part): return [[int(g) for g in x.rest[1].split(",")] for x in log() if x.kind == "launch" and part in x.rest[3]]
"""


@pytest.mark.parametrize("step", ["plain(h, 0, 1, st)", "weights(h, st=st)"])
@pytest.mark.parametrize("kw", [dict(cache_fp8=4), dict(cache_fp8=1, page_rows=16)])
def test_rows_read_back_cover_replayed_appends(runtime, step, kw):  # noqa: F811
    """madakv_cache_rows after a captured append: as many blocks of 64 rows as a head with every free row taken has, also behind a
    later eviction; the other layer's as before."""
    out = scenario(runtime, CALLS + f"""
h = create(sys.argv[3])
fake.fake_events_done(1)
assert evict(h) == 0
assert plain(h, 0, 2) == 0 and rows(h) == 0 and rows(h, l0=1) == 0
assert [g[0] for g in grids("cache_rows")] == [1, 1]             # (the runtime's eviction leaves heads of no rows)
fake.fake_capture(P(st))
assert {step} == 0
fake.fake_capture(P(0))
for _ in range(2):
    assert rows(h) == 0 and rows(h, l0=1) == 0 and rows(h, n=2) == 0
    assert [g[0] for g in grids("cache_rows")] == [4, 1, 4]
    assert evict(h) == 0
print("ok")
""", good(max_new_tokens=200, **kw))
    assert out.strip() == "ok"


@pytest.mark.parametrize("kw", [dict(), dict(page_rows=16), dict(cache_fp8=4)])
def test_reeviction_covers_replayed_appends(runtime, kw):  # noqa: F811
    """madakv_reevict after a captured append: its kernels over rows of a head cover every row that replays can have left."""
    out = scenario(runtime, CALLS + """
h = create(sys.argv[3])
fake.fake_events_done(1)
re = lambda: lib.madakv_reevict(h, I(0), I(2), *[P(T().p) for _ in range(8)], P(T().p), Z(1 << 40), P(0))
def widest():
    found = {}
    for x in log():
        if x.kind == "launch":
            for part in ("cache_rows", "linear_copy", "write_back", "score_fused"):
                if part in x.rest[3]: found.setdefault(part, int(x.rest[1].split(",")[0]))
    return found
assert evict(h) == 0 and plain(h) == 0
widest()
assert re() == 0
before = widest()
fake.fake_capture(P(st))
assert plain(h, 0, 1, st) == 0
fake.fake_capture(P(0))
widest()
for _ in range(2):
    assert re() == 0
    after = widest()
    assert before.keys() == after.keys() and "score_fused" in after
    assert all(v == 1 for v in before.values()), before
    assert all(v == (-(-5000 // 64) if x != "score_fused" else -(-5000 // 1024)) for x, v in after.items()), after
print("ok")
""", good(max_new_tokens=5000, **kw))
    assert out.strip() == "ok"
