"""Timed cases of attention over whole prompts, and of decoding several drafted tokens per step over a reduced cache.

A case names one of three operators and a shape (layers, batch, heads, head_dim, context, window, budget):

  op "prompt"   causal attention of all positions of a prompt, grouped heads, with the softmax normalisers of the rows
                (madakv_prompt_attn).  The L positions of a batch item hold one prompt, one padded prompt, or several that
                follow each other and do not see each other; positions of none are left as they are
  op "tree"     attention of a tree of drafted tokens: every node attends over the rows of the reduced cache and over the nodes
                that its mask names, its ancestors and itself, whose rows count with the values the cache would give them
                (madakv_tree_attn)
  op "commit"   the nodes of the accepted path become rows of the cache, each batch item its own number of them
                (madakv_tree_commit)

With `own` false the operators are computed in elementary torch operations in 32 bits; with `own` true by the library.
Every pass can be repeated on the same state: an accepted path is stored at the same place again.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"

# what a case has unless it says otherwise
BASE = dict(n_layers=1, batch=1, n_q_heads=32, n_kv_heads=32, head_dim=128, ctx_len=16384, window=32, budget=2048, out="bf16")
# (queries x keys) of all query heads of a drawn "prompt" case; bytes of a drawn case's K of the prompt
MOST_PAIRS = 28 * 16384 ** 2
MOST_PROMPT = 4 * 32 * 16384 * 128 * 2
FREE = 64                    # rows that the segments of a tree's cache have room for


def _case(name, op, **kw):
    return dict(BASE, name=name, op=op, **kw)


def listed():
    gqa = dict(n_q_heads=28, n_kv_heads=4)
    return [
        # a layer of a small model over a short prompt of odd length: latency
        _case("prompt_203", "prompt", n_q_heads=8, n_kv_heads=8, head_dim=64, ctx_len=203, window=16, budget=64, seqs=0, padding=0, dtype="bf16"),
        # four prompts of different lengths, padded on the left so that they end together
        _case("prompt_padded_2k", "prompt", batch=4, n_kv_heads=8, ctx_len=2048, seqs=1, padding=700, dtype="bf16"),
        # requests of very different lengths behind each other in one row, some of it unused
        _case("prompt_packed_6k", "prompt", **gqa, ctx_len=6001, seqs=11, padding=130, dtype="bf16"),
        # one layer of an 8K prompt, every head with its own keys
        _case("prompt_8k", "prompt", ctx_len=8192, seqs=0, padding=0, dtype="bf16"),
        # grouped queries over 16K tokens: the benchmark's shape of a grouped-query layer at half its context
        _case("prompt_gqa_16k", "prompt", **gqa, seqs=0, padding=0, dtype="bf16"),
        # a few drafted tokens of one short sequence
        _case("tree_small", "tree", n_q_heads=8, n_kv_heads=8, head_dim=64, ctx_len=300, window=16, budget=256, nodes=5, ragged=True, cache="bf16", pages=0),
        # a tree of 16 nodes, grouped queries, heads of very different lengths
        _case("tree_gqa_2k", "tree", **gqa, ctx_len=4096, nodes=16, ragged=True, cache="bf16", pages=0),
        # four sequences of 32 heads each, 8-bit rows, a chain of eight tokens
        _case("tree_2k_fp8", "tree", batch=4, ctx_len=4096, nodes=8, ragged=True, cache="fp8", pages=0),
        # a large tree over a cache that is kept whole in 4 bits
        _case("tree_gqa_16k_fp4", "tree", batch=2, n_kv_heads=8, budget=16384, nodes=60, ragged=False, cache="fp4", pages=0),
        # a cache kept whole: four sequences of 16K rows, 32 nodes, outputs as they come
        _case("tree_16k", "tree", batch=4, budget=16384, nodes=32, ragged=False, cache="bf16", pages=0, out="fp32"),
        # the accepted tokens of one layer of one sequence
        _case("commit_gqa", "commit", **gqa, ctx_len=4096, nodes=16, accept=4, cache="bf16"),
        # those of all layers of a model at once, 8-bit rows
        _case("commit_model_fp8", "commit", n_layers=32, batch=4, ctx_len=512, window=16, budget=64, nodes=16, accept=6, cache="fp8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed kinds: sizes over the whole range, odd ones among them."""
    c = dict(BASE)
    c["op"] = op = rng.choice(["prompt", "prompt", "tree", "tree", "commit"])
    c["n_q_heads"], c["n_kv_heads"] = rng.choice([(32, 32), (28, 4), (8, 8), (32, 8), (12, 2), (20, 20), (8, 1)])
    c["head_dim"] = rng.choice([128, 128, 64])
    c["window"] = rng.choice([8, 16, 32])
    c["batch"], c["n_layers"] = rng.choice([1, 1, 2, 4]), rng.choice([1, 1, 2])
    c["ctx_len"] = L = _log_int(rng, 70, 16384)
    c["out"] = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op == "prompt":
        c["dtype"] = "fp32" if rng.random() < 0.1 else "bf16"
        if c["dtype"] == "fp32":                                 # (a row of the group's proxy queries has to fit)
            c["out"], c["window"] = "fp32", 8
        c["budget"] = max(c["window"] + 1, L // 8)
        c["seqs"] = rng.choice([0, 1, _log_int(rng, 2, max(3, L // 40))])
        c["padding"] = rng.choice([0, rng.randrange(L // 2)]) if c["seqs"] else 0
        while c["n_layers"] * c["batch"] * c["n_q_heads"] * L * L * (16 if c["dtype"] == "fp32" or c["out"] == "fp32" else 1) > MOST_PAIRS:
            if c["batch"] * c["n_layers"] == 1:
                if c["dtype"] == "bf16" and c["out"] == "fp32":
                    c["out"] = "bf16"
                    continue
                c["ctx_len"] = L = L // 2
                c["padding"] = c["padding"] // 2
                c["budget"] = max(c["window"] + 1, L // 8)
            c["batch"], c["n_layers"] = max(1, c["batch"] // 2), 1
        return c
    c["nodes"] = _log_int(rng, 1, 64)
    c["cache"] = rng.choice(["bf16", "bf16", "fp8", "fp4"] if op == "tree" else ["bf16", "bf16", "fp8"])
    if rng.random() < 0.1:
        c["cache"], c["out"], c["window"] = "fp32", "fp32", 8
    if op == "commit":
        c["accept"] = rng.randint(1, c["nodes"])
        c["ctx_len"], c["n_layers"] = L, _ = min(L, 1024), rng.choice([1, 1, 2, 8, 32])
        c["budget"] = max(c["window"] + 8, L // 8)
    else:
        c["pages"] = rng.choice([0, 0, 0, 16, 64])
        c["ragged"] = rng.choice([True, True, False])
        c["budget"] = max(c["window"] + 8, int(L * math.exp(rng.uniform(math.log(1 / 8), math.log(0.7))))) if c["ragged"] else L
    while c["n_layers"] * c["batch"] * c["n_kv_heads"] * L * c["head_dim"] * (4 if c["cache"] == "fp32" else 2) > MOST_PROMPT // (2 if c["out"] == "fp32" else 1):
        c["batch"], c["n_layers"] = max(1, c["batch"] // 2), max(1, c["n_layers"] // 2)
    return c


# ---- inputs ---------------------------------------------------------------------------------------
def _sizes(case):
    return tuple(case[k] for k in ("n_layers", "batch", "n_q_heads", "n_kv_heads", "head_dim", "ctx_len", "window", "budget"))


def _dtype(case):
    return torch.float32 if "fp32" in (case.get("cache"), case.get("dtype")) else torch.bfloat16


def _bounds(case):
    """int [B, seqs + 1]: where the sequences of a "prompt" case start and the last one ends; None: one of all positions.  One
    sequence: padded in front, every item differently.  Several: behind each other, unused positions at the end."""
    B, L, S = case["batch"], case["ctx_len"], case["seqs"]
    if not S:
        return None
    r = np.random.default_rng(L * 31 + S)
    out = np.zeros((B, S + 1), np.int32)
    for b in range(B):
        pad = case["padding"] * (b + 1) // B
        out[b, -1] = L - (pad if S > 1 else 0)
        out[b, 0] = pad if S == 1 else 0
        out[b, 1:-1] = np.sort((out[b, -1] * r.random(S - 1) ** 1.5).astype(np.int32))
    return out


def _budgets(case, seed):
    """int32 [n, B, H, 2]: candidates to keep per head; a batch item's add up to n * H * (budget - W)."""
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    r = np.random.default_rng(seed)
    heads, nc = NL * H, L - W
    out = np.zeros((NL, B, H, 2), np.int32)
    for b in range(B):
        t = np.full(heads, min(keep, L) - W)
        if case.get("ragged"):                                   # rows change hands between two heads
            for i, j in r.permutation(heads)[:heads // 2 * 2].reshape(-1, 2):
                x = int(r.integers(0, min(t[i] // 2, nc - t[j]) + 1))
                t[i], t[j] = t[i] - x, t[j] + x
        out[:, b, :, 0] = t.reshape(NL, H)
    return torch.from_numpy(out)


def _counts(case):
    """Accepted nodes per batch item: `accept` on average."""
    B, a = case["batch"], case["accept"]
    n = np.full(B, a)
    for b in range(0, B - 1, 2):
        x = min(a, case["nodes"] - a) * (b + 2) // (B + 2)
        n[b], n[b + 1] = a - x, a + x
    return n


def _tree(case, seed):
    """int64 [B, T]: bit i of entry t: node t sees node i, an ancestor or itself.  The parents are earlier nodes, the newer the
    likelier; the first node follows the last token of the sequence, some others do too."""
    B, T = case["batch"], case["nodes"]
    r = np.random.default_rng(seed + 1)
    out = np.zeros((B, T), np.uint64)
    for b in range(B):
        for t in range(T):
            parent = t - 1 - int(min(r.geometric(0.4) - 1, t - 1)) if t and r.random() < 0.9 else -1
            out[b, t] = (out[b, parent] if parent >= 0 else np.uint64(0)) | np.uint64(1 << t)
    return torch.from_numpy(out.view(np.int64))


def _inputs(case, seed):
    """What a layer of a model hands over, on the GPU."""
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 29)
    dt = _dtype(case)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)      # noqa: E731
    # some dims of K are much larger than others, as rotary keys have them; the queries' match, so that logits have a spread of about 2
    spread = (0.7 * randn(NL, B, H, 1, d)).exp_()
    per_q = (2.0 / spread).repeat_interleave(Hq // H, dim=2)
    x = {"k": randn(NL, B, H, L, d).mul_(spread).to(dt), "v": randn(NL, B, H, L, d).to(dt)}
    if case["op"] == "prompt":
        x["q"] = (randn(NL, B, Hq, L, d) * per_q).to(dt)
        off = _bounds(case)
        x["seq_off"] = None if off is None else torch.from_numpy(off).to(DEV)
        return x
    T = case["nodes"]
    x["score"] = torch.rand(NL, B, H, L - W, generator=g, device=DEV)
    x["budgets"] = _budgets(case, seed).to(DEV)
    x["k_new"], x["v_new"] = (randn(NL, B, H, T, d) * spread).to(dt), randn(NL, B, H, T, d).to(dt)
    if case["op"] == "tree":
        x["q"] = (randn(NL, B, Hq, T, d) * per_q).to(dt)
        x["tree"] = _tree(case, seed).to(DEV)
        return x
    n = _counts(case)
    r = np.random.default_rng(seed + 2)
    path = np.zeros((B, int(n.max())), np.int32)
    for b in range(B):
        path[b, :n[b]] = np.sort(r.choice(T, n[b], replace=False))
    x["path"], x["n_path"], x["start"] = torch.from_numpy(path).to(DEV), torch.from_numpy(n.astype(np.int32)).to(DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    return x


# ---- the plain forms ---------------------------------------------------------------------------------
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _power(e):
    """2^e of whole numbers in -126 .. 127, in 32 bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _encode4(x):
    """(codes, scales) of rows [..., d]: per block of 32 a scale of 2^e, the least that takes the largest magnitude below 7 (it
    rounds to 6 at most), e in -120 .. 125; elements to the nearest of E2M1, ties to the even code."""
    y = x.float().unflatten(-1, (-1, 32))
    m, e = torch.frexp(y.abs().amax(-1))                         # largest = m 2^e, m in [0.5, 1)
    e = torch.where(m == 0, -120, e - 3 + (m > 0.875).int()).clamp(-120, 125)
    a = y.abs() * _power(-e).unsqueeze(-1)
    code = sum((a > t).int() for t in (0.25, 1.25, 2.5, 5.0)) + sum((a >= t).int() for t in (0.75, 1.75, 3.5))
    code = code + 8 * torch.signbit(y).int()
    code = code.flatten(-2).unflatten(-1, (-1, 2))
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), (e + 127).to(torch.uint8)


def _decode4(codes, scales):
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    return (table[code].unflatten(-1, (-1, 32)) * _power(scales.int() - 127).unsqueeze(-1)).flatten(-2)


def _choose(x, case):
    """(kept positions, lengths [n, B, H], first rows): per head the best-scored candidates, equal scores the lower position, in
    ascending position, then the window; heads of a batch item follow each other, layer by layer, each with FREE rows behind it."""
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    take = torch.ones(NL, B, H, L, dtype=torch.bool, device=DEV)
    if min(keep, L) < L:
        order = torch.sort(x["score"], dim=-1, descending=True, stable=True).indices
        rank = torch.arange(L - W, device=DEV).expand_as(order)
        take[..., :L - W].scatter_(-1, order, rank < x["budgets"][..., :1])
    lens = take.sum(-1)
    by_item = (lens + FREE).permute(1, 0, 2).reshape(-1)
    off = (by_item.cumsum(0) - by_item).view(B, NL, H).permute(1, 0, 2).contiguous()
    return take, lens.int(), off


def _prompt(state):
    case, x = state["case"], state["x"]
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    row = torch.arange(L, device=DEV)
    if x["seq_off"] is None:
        first, inside = torch.zeros(B, L, dtype=torch.int64, device=DEV), None
    else:                                                        # the start of the row's sequence; rows of none
        behind = row.view(1, L, 1) >= x["seq_off"].unsqueeze(1)
        nth = behind.sum(-1)
        first = torch.gather(x["seq_off"].long(), 1, (nth - 1).clamp_min(0))
        inside = ((nth > 0) & ~behind[..., -1]).view(1, B, 1, L, 1)
    s = torch.bmm(x["q"].float().view(NL * B * H, -1, d), x["k"].float().view(NL * B * H, L, d).transpose(1, 2).contiguous())
    s = s.mul_(1 / math.sqrt(d)).view(NL, B, Hq, L, L)
    hidden = (row > row.view(L, 1)) | (row < first.unsqueeze(-1))
    s.masked_fill_(hidden.view(1, B, 1, L, L), -math.inf)
    top = s.amax(-1, keepdim=True)
    w = s.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    out = torch.bmm(w.view(NL * B * H, -1, L), x["v"].float().view(NL * B * H, L, d)).view(NL, B, Hq, L, d) / total
    lse = top + total.log()
    if inside is not None:
        out, lse = torch.where(inside, out, state["out"].float()), torch.where(inside, lse, state["lse"].unsqueeze(-1))
    state["out"].copy_(out)
    state["lse"].copy_(lse.squeeze(-1))
    return {"out": state["out"], "lse": state["lse"]}


def _tree_attn(state):
    case, x = state["case"], state["x"]
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    T, rows, there = case["nodes"], state["rows"], state["there"]
    k, v = (_decode4(*c) if case["cache"] == "fp4" else c.float() for c in (state["k"], state["v"]))
    new = [x[n].view(NL * B * H, T, d) for n in ("k_new", "v_new")]
    new = [_decode4(*_encode4(c)) if case["cache"] == "fp4" else c.clamp(-448, 448).to(torch.float8_e4m3fn).float() if case["cache"] == "fp8" else c.float() for c in new]
    k, v = (torch.cat([c[rows], n], 1) for c, n in zip((k, v), new))
    sees = (x["tree"].unsqueeze(-1) >> torch.arange(T, device=DEV)) & 1
    sees = sees.bool().view(1, B, 1, 1, T, T).expand(NL, B, H, Hq // H, T, T).reshape(NL * B * H, -1, T)
    may = torch.cat([there.unsqueeze(1).expand(-1, sees.shape[1], -1), sees], -1)
    s = torch.bmm(x["q"].float().view(NL * B * H, -1, d), k.transpose(1, 2).contiguous()) / math.sqrt(d)
    s = s.masked_fill_(~may, -math.inf)
    w = s.sub_(s.amax(-1, keepdim=True)).exp_()
    out = torch.bmm(w, v) / w.sum(-1, keepdim=True)
    state["out"].copy_(out.view(NL, B, Hq, T, d))
    return {"out": state["out"]}


def _commit(state):
    case, x = state["case"], state["x"]
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    i = torch.arange(x["path"].shape[1], device=DEV)
    layer, item, head, step = (i < x["n_path"].unsqueeze(1)).view(1, B, 1, -1).expand(NL, B, H, -1).nonzero(as_tuple=True)
    at = state["off"][layer, item, head] + state["lens"][layer, item, head] + x["start"][item] + step
    node = x["path"][item, step].long()
    for c, n in (("k", "k_new"), ("v", "v_new")):
        new = x[n][layer, item, head, node]
        state[c][at] = new.clamp(-448, 448).to(torch.float8_e4m3fn) if case["cache"] == "fp8" else new
    state["kv_len"].copy_(state["lens"] + (x["start"] + x["n_path"]).view(1, B, 1))
    return {"k": state["k"], "v": state["v"], "len": state["kv_len"]}


# ---- a pass ------------------------------------------------------------------------------------------
def _handle(case):
    from paper_2506_15724_amd import binding as MB
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    return MB.MadaKV(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=W, budget=keep,
                     dtype="fp32" if _dtype(case) == torch.float32 else "bf16", max_new_tokens=FREE, out_fp32=int(case["out"] == "fp32"),
                     cache_fp8={"fp8": 1, "fp4": 4}.get(case.get("cache"), 0), page_rows=case.get("pages", 0), device=DEV)


def prepare(case, seed):
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    x = _inputs(case, seed)
    state = {"case": case, "x": x}
    if own:
        state["eng"] = eng = _handle(case)
    if case["op"] != "commit":
        rows = L if case["op"] == "prompt" else case["nodes"]
        state["out"] = torch.zeros(NL, B, Hq, rows, d, dtype=torch.float32 if case["out"] == "fp32" else torch.bfloat16, device=DEV)
    if case["op"] == "prompt":
        state["lse"] = torch.zeros(NL, B, Hq, L, device=DEV)
        return state
    if own:                                                      # the cache as the prompt's eviction leaves it
        eng.k_c.zero_(), eng.v_c.zero_()
        eng.select_gather(0, NL, x["k"], x["v"], torch.zeros(B, L, dtype=torch.uint8, device=DEV), x["score"], x["budgets"])
    else:
        take, state["lens"], state["off"] = _choose(x, case)
        state["kv_len"] = state["lens"].clone()
        r = torch.arange(int(state["lens"].max()), device=DEV)
        state["there"] = r < state["lens"].reshape(-1, 1)
        state["rows"] = torch.where(state["there"], state["off"].reshape(-1, 1) + r, 0)
        for n in ("k", "v"):
            c = torch.zeros(NL * B * H * (min(keep, L) + FREE), d, dtype=_dtype(case), device=DEV)
            c[state["rows"][state["there"]]] = x[n][take]
            state[n] = _encode4(c) if case["cache"] == "fp4" else c.clamp(-448, 448).to(torch.float8_e4m3fn) if case["cache"] == "fp8" else c
    for n in ("k", "v", "score", "budgets"):
        del x[n]
    return state


def run(state):
    case = state["case"]
    if not own:
        return {"prompt": _prompt, "tree": _tree_attn, "commit": _commit}[case["op"]](state)
    eng, x, NL = state["eng"], state["x"], case["n_layers"]
    if case["op"] == "prompt":
        eng.prompt_attn(0, NL, x["q"], x["k"], x["v"], state["out"], row_lse=state["lse"], seq_off=x["seq_off"])
        return {"out": state["out"], "lse": state["lse"]}
    if case["op"] == "tree":
        eng.tree_attn(0, NL, x["q"], x["k_new"], x["v_new"], x["tree"], state["out"])
        return {"out": state["out"]}
    eng.tree_commit(0, NL, x["k_new"], x["v_new"], x["path"], x["n_path"], x["start"], x["path"].shape[1])
    k, v = (t.view(torch.float8_e4m3fn) if case["cache"] == "fp8" else t for t in (eng.k_c, eng.v_c))
    return {"k": k, "v": v, "len": eng.kv_len}


def _pairs(case):
    """(query, key) pairs that see each other, over the batch, and positions in some sequence."""
    B, L = case["batch"], case["ctx_len"]
    off = _bounds(case)
    if off is None:
        return B * L * (L + 1) // 2, B * L
    n = np.diff(off.astype(np.int64), axis=1)
    return int((n * (n + 1) // 2).sum()), int(n.sum())


def work(case):
    """Bytes: every input read once, every output written once.  "prompt": q, k, v, out and normalisers of the positions in some
    sequence.  "tree": the rows of the cache (codes and scales), the nodes' q, k, v, out.  "commit": the accepted nodes' rows read,
    and written as the cache has them.  Flops: the two products of attention over the pairs that see each other (of a tree: over
    the cache's rows, and each node itself)."""
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    es = 4 if _dtype(case) == torch.float32 else 2
    os = 4 if case["out"] == "fp32" else 2
    if case["op"] == "prompt":
        pairs, rows = _pairs(case)
        return {"bytes": NL * rows * (Hq * (d * (es + os) + 4) + 2 * H * d * es), "flops": 4 * NL * Hq * d * pairs}
    T = case["nodes"]
    row = {"bf16": 2 * d, "fp8": d, "fp4": d // 2 + d // 32, "fp32": 4 * d}[case["cache"]]
    if case["op"] == "commit":
        n = NL * H * B * case["accept"]
        return {"bytes": n * 2 * (es * d + row) + NL * B * H * 12, "flops": 0}
    rows = NL * B * H * min(keep, L)
    return {"bytes": rows * 2 * row + NL * B * T * (Hq * d * (es + os) + 2 * H * d * es), "flops": 4 * d * Hq // H * T * (rows + NL * B * H)}


# ---- in 64 bits, from the definitions -------------------------------------------------------------------
def _value4(x):
    """The values that rows x [n, d] have in the 4-bit cache, in 64 bits: every element to the nearest multiple of its own step."""
    y = x.double().reshape(-1, 32)
    bits = y.abs().max(1).values.view(torch.int64)               # exponent and fraction of the largest magnitude
    e = (bits >> 52) - 1023 - 2 + ((bits & ((1 << 52) - 1)) > (3 << 50)).long()
    unit = ((e.clamp(-120, 125) + 1023) << 52).view(torch.float64)[:, None]
    z = y / unit
    step = torch.where(z.abs() < 2, 0.5, torch.where(z.abs() < 4, 1.0, 2.0))
    return ((z / step).round() * step).clamp(-6, 6).mul(unit).reshape(x.shape)


def _exact_prompt(case, x):
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    out = torch.zeros(NL, B, Hq, L, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(NL, B, Hq, L, dtype=torch.float64, device=DEV)
    off = _bounds(case)
    for b in range(B):
        ends = [0, L] if off is None else off[b].tolist()
        for lo, hi in zip(ends[:-1], ends[1:]):
            step = max(1, (1 << 27) // max(1, hi - lo))          # query rows at a time: 1 GB of logits
            for r0 in range(lo, hi, step):
                r1 = min(hi, r0 + step)
                for l in range(NL):
                    for j in range(Hq):
                        k, v = x["k"][l, b, j * H // Hq, lo:r1].double(), x["v"][l, b, j * H // Hq, lo:r1].double()
                        s = x["q"][l, b, j, r0:r1].double() @ k.t().contiguous() / math.sqrt(d)
                        s += torch.full_like(s, -math.inf).triu_(r0 - lo + 1)
                        n = torch.logsumexp(s, 1)
                        lse[l, b, j, r0:r1] = n
                        out[l, b, j, r0:r1] = torch.exp(s - n[:, None]) @ v
    return {"out": out, "lse": lse}


def exact(case, seed):
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    if case["op"] == "commit":
        return None
    if case["op"] == "prompt" and case["seqs"] * NL * B * Hq > 20000:
        return None
    x = _inputs(case, seed)
    if case["op"] == "prompt":
        return _exact_prompt(case, x)
    G, T = Hq // H, case["nodes"]
    score, budgets = x["score"].cpu().numpy(), x["budgets"].cpu().numpy()
    tree = x["tree"].cpu().numpy().view(np.uint64)
    out = torch.zeros(NL, B, Hq, T, d, dtype=torch.float64, device=DEV)
    for l in range(NL):
        for b in range(B):
            sees = torch.tensor([[float((int(m) >> i) & 1) for i in range(T)] for m in tree[b]], dtype=torch.float64, device=DEV)
            for h in range(H):
                p = np.arange(L)
                if keep < L:
                    c = np.lexsort((np.arange(L - W), -score[l, b, h]))[:budgets[l, b, h, 0]]
                    p = np.concatenate([np.sort(c), np.arange(L - W, L)])
                k, v = (torch.cat([x[n][l, b, h][torch.from_numpy(p).to(DEV)], x[n + "_new"][l, b, h]]) for n in ("k", "v"))
                if case["cache"] == "fp4":
                    k, v = _value4(k), _value4(v)
                elif case["cache"] == "fp8":
                    k, v = (t.clamp(-448, 448).to(torch.float8_e4m3fn) for t in (k, v))
                k, v = k.double(), v.double()
                may = torch.cat([torch.ones(T, len(p), dtype=torch.float64, device=DEV), sees], 1)
                for j in range(h * G, (h + 1) * G):
                    s = x["q"][l, b, j].double() @ k.t().contiguous() / math.sqrt(d)
                    w = torch.exp(s - s.max(1, keepdim=True).values) * may
                    out[l, b, j] = (w / w.sum(1, keepdim=True)) @ v
    return {"out": out}
