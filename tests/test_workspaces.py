"""A workspace of the size reported for n layers serves every call over n layers or fewer, on the runtime that only keeps a log.  No GPU."""
import pytest

from tests.test_abi import good
from tests.test_host_calls import runtime, scenario  # noqa: F401  (a fixture)
from tests.test_operator_calls import ARGS

CONFIGS = [dict(n_layers=32, n_q_heads=32, n_kv_heads=32, ctx_len=16384, budget=2048), dict(n_layers=40, batch=2, n_q_heads=28, n_kv_heads=4, ctx_len=9000, budget=1100, max_new_tokens=200),
           dict(n_layers=32, n_q_heads=32, n_kv_heads=32, head_dim=64, ctx_len=2048, window=8, budget=1024), dict(n_layers=24, n_q_heads=16, n_kv_heads=8, ctx_len=70000, budget=9000, cache_fp8=4),
           dict(n_layers=40, batch=4, n_q_heads=8, n_kv_heads=8, ctx_len=4096, budget=512, cache_fp8=1, page_rows=16), dict(n_layers=33, n_q_heads=32, n_kv_heads=32, ctx_len=4096, budget=2048, cache_fp8=4, page_rows=64),
           dict(n_layers=24, n_q_heads=32, n_kv_heads=32, head_dim=64, window=16, ctx_len=3000, budget=400, dtype=0)]


@pytest.mark.parametrize("cfg", CONFIGS, ids=lambda c: "-".join(str(x) for x in c.values()))
def test_workspaces_serve_calls_over_fewer_layers(runtime, cfg):  # noqa: F811
    """No call over m <= n layers says that its workspace is too small; one byte less than the size for one layer is."""
    out = scenario(runtime, ARGS + """
h = create(sys.argv[3])
NL, fp32, whole = int.from_bytes(bytes.fromhex(sys.argv[3])[:4], "little"), %r, %r
t = lambda k: [P(T().p) for _ in range(k)]
def size(call, n):
    z = Z()
    assert call(h, I(n), C.byref(z)) == 0
    return z.value
def sizes(n):
    a, b, c = Z(), Z(), Z()
    assert lib.madakv_workspace_bytes(h, I(n), C.byref(a), C.byref(b), C.byref(c)) == 0
    return dict(score=a.value, select=b.value, decode=c.value, window=size(lib.madakv_window_attn_workspace_bytes, n), reevict=size(lib.madakv_reevict_workspace_bytes, n),
                weights=size(lib.madakv_decode_attn_weights_workspace_bytes, n), prompt=size(lib.madakv_score_prompt_workspace_bytes, n))
W = lambda z: (P(T().p), Z(z))
calls = dict(
    score=lambda m, s: lib.madakv_score(h, I(0), I(m), *t(7), *W(s["score"]), P(0)),
    select=lambda m, s: lib.madakv_select_gather(h, I(0), I(m), *t(10), *W(s["select"]), P(0)),
    evict=lambda m, s: lib.madakv_evict(h, I(0), I(m), *t(14), *W(s["score"]), *W(s["select"]), P(0)),
    decode=lambda m, s: lib.madakv_decode_attn(h, I(0), I(m), P(T().p), P(0), P(0), *t(5), *W(s["decode"]), P(0)),
    weights=lambda m, s: weights(h, n=m, kn=None, vn=None, size=s["weights"]))
if not fp32:
    calls.update(window=lambda m, s: lib.madakv_window_attn_score(h, I(0), I(m), *t(10), *W(s["window"]), P(0)),
                 prompt=lambda m, s: prompt(h, n=m, size=s["prompt"]),
                 reevict=lambda m, s: lib.madakv_reevict(h, I(0), I(m), *t(8), *W(s["reevict"]), P(0)))
for n in range(1, NL + 1):
    s = sizes(n)
    for name, call in calls.items():
        for m in range(1, n + 1):
            if name == "reevict" and whole and m < NL: continue         # (a paged cache is re-evicted as a whole)
            rc = call(m, s)
            assert rc in (0, -7), (name, n, m, rc)
    log()
less = {x: y - 1 for x, y in sizes(1).items()}
for name in calls:
    if name in ("reevict",) and whole: continue
    assert calls[name](1, less) in (-4, -7) or name == "select", name   # (the selection makes do with less than a slice per layer group)
print("ok")
""" % (cfg.get("dtype") == 0, bool(cfg.get("page_rows"))), good(**cfg))
    assert out.strip() == "ok"


@pytest.mark.parametrize("kw", [dict(), dict(n_q_heads=28, n_kv_heads=4, window=16)])
def test_reeviction_of_one_layer_in_4_bits_holds_one_layer_of_k(runtime, kw):  # noqa: F811
    """The workspace has K as bf16 for the rows that the call's layers can hold, not for all layers of the model."""
    cfg = dict(n_layers=32, n_q_heads=128, n_kv_heads=64, batch=2, ctx_len=16384, budget=4096, max_new_tokens=100, cache_fp8=4)
    cfg.update(kw)
    capacity = cfg["n_layers"] * cfg["batch"] * cfg["n_kv_heads"] * (cfg["budget"] + 100)
    layer = cfg["batch"] * cfg["n_kv_heads"] * (cfg["ctx_len"] + 100)
    out = scenario(runtime, f"""
h = create(sys.argv[3])
z, cap = Z(), C.c_int64()
assert lib.madakv_compact_capacity_tokens(h, C.byref(cap)) == 0 and cap.value == {capacity}
def size(n): assert lib.madakv_reevict_workspace_bytes(h, I(n), C.byref(z)) == 0; return z.value
for n in (1, 2, 32):
    held = min({capacity}, n * {layer})
    # per row of the cache 13 bytes of scores, choices and modalities; per row of the call K, and a score for every 64 proxy rows
    least = 13 * {capacity} + 2 * 128 * held
    assert least <= size(n) <= least + (4 * 4 * held) + n * (64 << 20), (n, size(n), least)
print("ok")
""", good(**cfg))
    assert out.strip() == "ok"
