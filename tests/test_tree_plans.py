"""How attention of a drafted tree cuts its heads, and in which order it joins the pieces: by the configuration, the call and the rows that
the heads hold, and not by what the host has heard of them.  No GPU: the library runs on a runtime that only keeps a log."""
import pytest

from tests.test_abi import good
from tests.test_host_calls import runtime, scenario  # noqa: F401  (a fixture)
from tests.test_tree_calls import ARGS

PLANS = ARGS + """
words = lambda x: [int(y, 16) for y in x.rest[4:]]
fake.fake_events_done(0)
h = create(sys.argv[3])
longest, NL, B = SIZES
log()
assert lib.madakv_select_gather(h, I(0), I(NL), *[P(T().p) for _ in range(10)], P(T().p), Z(1 << 40), P(0)) == 0
(where,) = [words(x)[7] for x in log() if x.kind == "launch" and "offsets" in x.rest[3]]
(C.c_int32 * (NL * B)).from_address(where)[:] = [longest] * (NL * B)          # what the layout kernel tells the host of the longest heads
def plan(t, st=None):
    log()
    assert tree(h, t=t, n=NL, st=st) == 0
    x = [x for x in log() if x.kind == "launch"]
    w = words(x[0])
    assert "tree_join" not in x[0].rest[3]
    join = x[1].rest[1] if len(x) > 1 else None
    return (x[0].rest[3], w[12] & 0xffffffff, w[12] >> 32, join)
def cut(p, rows):                                        # (as cut_of in tree.hip)
    _, chunk, most, _ = p
    n = min(max(1, (rows - chunk // 8 + chunk - 1) // chunk), most)
    return max(1, -(-(-(-rows // n)) // 64)) * 64
TS = (1, 5, 8, 16, 33, 64)
unknown = [plan(t) for t in TS]
s = 0x77000
fake.fake_events_done(1)
fake.fake_capture(P(s))
captured = [plan(t, s) for t in TS]
fake.fake_capture(P(0))
known = [plan(t) for t in TS]
assert lib.madakv_decode_attn(h, I(0), I(NL), *[P(T().p) for _ in range(8)], P(T().p), Z(1 << 40), P(0)) == 0
grown = [plan(t) for t in TS]
for a, b in ((unknown, known), (captured, known), (unknown, grown)):
    for p, q in zip(a, b):
        assert p[:2] == q[:2], (p, q)
        assert p[3] == q[3] or None in (p[3], q[3]), (p, q)          # the threads that share the pieces of a column
        for rows in {1, 63, 64, 200, longest // 2, longest - 1, longest}: assert cut(p, rows) == cut(q, rows), (p, q, rows)
print("ok")
"""

CASES = [dict(batch=4, n_kv_heads=32, n_q_heads=32, ctx_len=4096, budget=2048, longest=2048), dict(batch=4, n_kv_heads=32, n_q_heads=32, ctx_len=32768, budget=16384, longest=17000),
         dict(batch=2, n_kv_heads=8, n_q_heads=32, ctx_len=16384, budget=16384, longest=16384, cache_fp8=4), dict(batch=1, n_kv_heads=4, n_q_heads=28, ctx_len=4096, budget=2048, longest=5000),
         dict(batch=1, n_kv_heads=2, n_q_heads=8, ctx_len=60000, budget=20000, longest=20001, page_rows=16), dict(batch=1, n_kv_heads=8, n_q_heads=64, ctx_len=1 << 18, budget=3000, hcc_rho=256, longest=90000),
         dict(batch=3, n_kv_heads=4, n_q_heads=4, ctx_len=3000, budget=700, longest=710, dtype=0), dict(batch=1, n_kv_heads=8, n_q_heads=8, ctx_len=300, budget=256, longest=256, head_dim=64)]


@pytest.mark.parametrize("max_new", [1, 64, 3000])
@pytest.mark.parametrize("kw", CASES)
def test_pieces_do_not_follow_the_hosts_knowledge(runtime, kw, max_new):  # noqa: F811
    """Lengths unknown, known, captured, after a step."""
    kw = dict(kw, window=8, max_new_tokens=max_new, n_layers=2)
    longest = kw.pop("longest")
    out = scenario(runtime, PLANS.replace("SIZES", f"{longest}, 2, {kw['batch']}"), good(**kw))
    assert out.strip() == "ok"
