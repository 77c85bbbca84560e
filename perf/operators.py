"""Timed cases of the operators around a reduced cache that is held in 4 bits or evicted by accumulated attention weight.

A case names one of four operators and a shape (layers, batch, heads, head_dim, context, window, budget):

  op "store"    rows into the 4-bit cache and out of it: the kept rows of the prompt's K and V are chosen, encoded (blocks of 32
                dims share a power of two, elements are E2M1 floats) and read back in the type of the model
                (madakv_select_gather with a 4-bit cache, madakv_cache_rows)
  op "attend"   one decode step's attention over a 4-bit cache (madakv_decode_attn)
  op "prompt"   the weight that all queries of a prompt pay to each of its keys, summed over the queries and the query heads
                of a KV head (madakv_score_prompt), with the softmax normalisers of the rows at hand or without
  op "weights"  one decode step that adds the weights it pays to a running sum per row, stores the new token in the place of
                the row chosen by the step before and chooses the row that the next token takes, the one of the least
                accumulated weight (madakv_decode_attn_weights)

With `own` false the operators are computed in elementary torch operations in 32 bits; with `own` true by the library.
Every pass can be repeated on the same state: attention is without an appended row, a replaced row gets the same token again.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"

# what a case has unless it says otherwise
BASE = dict(n_layers=1, batch=1, n_q_heads=32, n_kv_heads=32, head_dim=128, ctx_len=16384, window=32, budget=2048, ragged=True)
# (queries x keys) of all query heads of a drawn "prompt" case, bytes of a drawn case's prompt K
MOST_PAIRS = 32 * 16384 ** 2
MOST_PROMPT = 32 * 4 * 16384 * 128 * 2


def _case(name, op, **kw):
    return dict(BASE, name=name, op=op, **kw)


def listed():
    gqa = dict(n_q_heads=28, n_kv_heads=4)
    return [
        # a layer of a small model right after a short prompt: launches and latency
        _case("store_small", "store", n_q_heads=8, n_kv_heads=8, head_dim=64, ctx_len=1024, window=16, budget=256),
        # a layer of grouped queries after a 32K prompt
        _case("store_gqa_32k", "store", **gqa, ctx_len=32768, budget=2048),
        # four 16K prompts, a layer of 32 heads, an eighth of the rows kept
        _case("store_16k", "store", batch=4, budget=2048),
        # a token of one short sequence
        _case("attend_small", "attend", n_q_heads=8, n_kv_heads=8, head_dim=64, ctx_len=300, window=16, budget=256),
        # grouped queries, heads of very different lengths
        _case("attend_gqa_2k", "attend", **gqa, ctx_len=4096, budget=2048),
        # a cache that is kept whole because it is in 4 bits: four sequences of 16K
        _case("attend_16k", "attend", batch=4, budget=16384, ragged=False),
        # a short prompt of odd length, normalisers not at hand
        _case("prompt_203", "prompt", n_q_heads=8, n_kv_heads=8, head_dim=64, ctx_len=203, window=16, budget=64, given_lse=False),
        # one layer of an 8K prompt whose prefill attention handed the normalisers over
        _case("prompt_8k_lse", "prompt", ctx_len=8192, given_lse=True),
        # grouped queries over 16K tokens, normalisers not at hand
        _case("prompt_gqa_16k", "prompt", **gqa, given_lse=False),
        # a token of one sequence of grouped queries, whose cache has its final size
        _case("weights_gqa_2k", "weights", **gqa, ctx_len=4096, budget=2048, cache="bf16", replace=True),
        # four sequences with 32 heads each, 8-bit rows
        _case("weights_2k_fp8", "weights", batch=4, ctx_len=4096, budget=2048, cache="fp8", replace=True),
        # the same with long heads in bf16, whose weights are accumulated without storing a token
        _case("weights_16k", "weights", batch=2, budget=16384, ragged=False, cache="bf16", replace=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed kinds: sizes over the whole range, odd ones among them."""
    c = dict(BASE)
    c["op"] = op = rng.choice(["store", "attend", "prompt", "weights"])
    c["n_q_heads"], c["n_kv_heads"] = rng.choice([(32, 32), (28, 4), (8, 8), (32, 8), (12, 2), (20, 20), (8, 1)])
    c["head_dim"] = rng.choice([128, 128, 64])
    c["window"] = rng.choice([8, 16, 32])
    c["batch"], c["n_layers"] = rng.choice([1, 1, 2, 4]), rng.choice([1, 1, 2])
    c["ctx_len"] = L = _log_int(rng, 70, 16384)
    if op == "prompt":
        c["given_lse"] = rng.choice([False, True])
        c["budget"] = max(c["window"] + 1, L // 8)
        while c["n_layers"] * c["batch"] * c["n_q_heads"] * L * L > MOST_PAIRS:
            c["batch"], c["n_layers"] = max(1, c["batch"] // 2), 1
        return c
    c["ragged"] = rng.choice([True, True, False])
    c["budget"] = max(c["window"] + 8, int(L * math.exp(rng.uniform(math.log(1 / 8), math.log(0.7))))) if c["ragged"] else L
    while c["n_layers"] * c["batch"] * c["n_kv_heads"] * L * c["head_dim"] * 2 > MOST_PROMPT:
        c["batch"], c["n_layers"] = max(1, c["batch"] // 2), 1
    if op == "weights":
        c["cache"] = rng.choice(["bf16", "bf16", "fp8", "fp4"])
        c["replace"] = c["cache"] != "fp4" and rng.choice([True, True, False])
        if rng.random() < 0.15 and c["cache"] == "bf16" and c["n_q_heads"] == c["n_kv_heads"]:
            c["cache"] = "fp32"
    return c


# ---- inputs ---------------------------------------------------------------------------------------
def _sizes(case):
    return tuple(case[k] for k in ("n_layers", "batch", "n_q_heads", "n_kv_heads", "head_dim", "ctx_len", "window", "budget"))


def _dtype(case):
    return torch.float32 if case.get("cache") == "fp32" else torch.bfloat16


def _budgets(case, seed, n_mod):
    """int32 [n, B, H, 2]: candidates to keep per head and modality; a batch item's add up to n * H * (budget - W)."""
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    r = np.random.default_rng(seed)
    heads, nc = NL * H, L - W
    out = np.zeros((NL, B, H, 2), np.int32)
    for b in range(B):
        t = np.full(heads, min(keep, L) - W)
        if case["ragged"]:
            # rows change hands between two heads, within half and twice the average
            for i, j in r.permutation(heads)[:heads // 2 * 2].reshape(-1, 2):
                x = int(r.integers(0, min(t[i] // 2, nc - t[j]) + 1))
                t[i], t[j] = t[i] - x, t[j] + x
        text = np.clip(np.round(t * r.random(heads)), t - n_mod[b][1], n_mod[b][0]).astype(np.int32)
        out[:, b, :, 0], out[:, b, :, 1] = text.reshape(NL, H), (t - text).reshape(NL, H)
    return torch.from_numpy(out)


def _inputs(case, seed):
    """What a layer of a model hands over, on the GPU: K and V of the prompt, queries, the scores and budgets of an eviction."""
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 17)
    dt = _dtype(case)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)      # noqa: E731
    # some dims of K are much larger than others, as rotary keys have them; the queries' match, so that logits have a spread of about 2
    spread = (0.7 * randn(NL, B, H, 1, d)).exp_()
    k = randn(NL, B, H, L, d).mul_(spread).to(dt)
    per_q = (2.0 / spread).repeat_interleave(Hq // H, dim=2)
    x = {"k": k}
    if case["op"] == "prompt":
        x["q"] = (randn(NL, B, Hq, L, d) * per_q).to(dt)
        return x
    x["v"] = randn(NL, B, H, L, d).to(dt)
    mask = torch.rand(B, L, generator=g, device=DEV) < 0.5
    mask = mask.to(torch.uint8)
    mask[:, 0], mask[:, 1], mask[:, L - W:] = 0, 1, 0
    x["mask"] = mask
    # scores of an observation window: a heavy tail, and a tenth of the candidates that nothing looks at
    s = torch.rand(NL, B, H, L - W, generator=g, device=DEV)
    x["score"] = torch.where(s < 0.1, 0.0, -(1.0 - s).clamp_min(1e-7).log()).contiguous()
    image = mask[:, :L - W].sum(1).tolist()
    x["budgets"] = _budgets(case, seed, [(L - W - i, i) for i in image]).to(DEV)
    if case["op"] == "store":
        return x
    x["q"] = (randn(NL, B, Hq, 1, d) * per_q).squeeze(3).to(dt)
    if case["op"] == "weights":
        rows = NL * B * H * min(keep, L)
        x["acc"] = -torch.rand(rows, generator=g, device=DEV).clamp_min(1e-7).log() * (0.01 * Hq / H)
        x["k_new"], x["v_new"] = (randn(NL, B, H, 1, d) * spread).squeeze(3).to(dt), randn(NL, B, H, d).to(dt)
        x["slot"] = (torch.rand(NL, B, H, generator=g, device=DEV) * (x["budgets"].sum(-1) + W)).int()
        x["pos"] = torch.full((B,), L, dtype=torch.int32, device=DEV)
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
    """(kept positions, offsets, lengths): per head and modality the best-scored candidates, equal scores the lower position,
    in ascending position, then the window; heads of a batch item follow each other, layer by layer."""
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    take = torch.ones(NL, B, H, L, dtype=torch.bool, device=DEV)
    if min(keep, L) < L:
        best = torch.zeros(NL, B, H, L - W, dtype=torch.bool, device=DEV)
        for m in (0, 1):
            s = torch.where((x["mask"][:, :L - W] == m)[None, :, None], x["score"], -1.0)
            order = torch.sort(s, dim=-1, descending=True, stable=True).indices
            rank = torch.arange(L - W, device=DEV).expand_as(order)
            best |= torch.zeros_like(best).scatter_(-1, order, rank < x["budgets"][..., m:m + 1])
        take[..., :L - W] = best
    lens = take.sum(-1)
    by_item = lens.permute(1, 0, 2).reshape(-1)
    off = (by_item.cumsum(0) - by_item).view(B, NL, H).permute(1, 0, 2).contiguous()
    item, layer, head, at = take.permute(1, 0, 2, 3).nonzero(as_tuple=True)
    return (layer, item, head, at), off, lens.int()


def _padded(off, lens):
    """Rows of every head side by side: their places in the cache, and which of them are there."""
    r = torch.arange(int(lens.max()), device=DEV)
    there = r < lens.reshape(-1, 1)
    return torch.where(there, off.reshape(-1, 1) + r, 0), there


def _attend(case, q, k, v, there):
    """(out, weights) of q [heads, G, d] over k, v [heads, rows, d], in 32 bits."""
    s = torch.bmm(q.float(), k.float().transpose(1, 2).contiguous()) / math.sqrt(case["head_dim"])
    w = torch.softmax(s.masked_fill(~there.unsqueeze(1), -math.inf), -1)
    return torch.bmm(w, v.float()), w


def _store(state):
    case, x = state["case"], state["x"]
    at, off, lens = _choose(x, case)
    state["k_rows"].copy_(_decode4(*_encode4(x["k"][at])))
    state["v_rows"].copy_(_decode4(*_encode4(x["v"][at])))
    return {"k": state["k_rows"], "v": state["v_rows"], "kept": at[3].int(), "off": off, "len": lens}


def _attend4(state):
    case, x = state["case"], state["x"]
    k, v = _decode4(*state["k4"]), _decode4(*state["v4"])
    out, _ = _attend(case, x["q"].reshape(-1, case["n_q_heads"] // case["n_kv_heads"], case["head_dim"]), k[state["rows"]], v[state["rows"]], state["there"])
    return {"out": out.view_as(x["q"])}


def _prompt(state):
    case, x = state["case"], state["x"]
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    q, k = x["q"].float().view(NL * B * H, -1, d), x["k"].float().view(NL * B * H, L, d)
    s = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1 / math.sqrt(d)).view(NL, B, Hq, L, L)
    s.masked_fill_(torch.ones(L, L, dtype=torch.bool, device=DEV).triu_(1), -math.inf)
    if case["given_lse"]:
        w = s.sub_(x["lse"].unsqueeze(-1)).exp_()
    else:
        w = s.sub_(s.amax(-1, keepdim=True)).exp_()
        w /= w.sum(-1, keepdim=True)
    return {"psi": w.sum(-2).view(NL, B, H, Hq // H, L).sum(-2)}


def _weights(state):
    case, x = state["case"], state["x"]
    G, d, W = case["n_q_heads"] // case["n_kv_heads"], case["head_dim"], case["window"]
    k, v, off, rows, there = state["k"], state["v"], state["off"], state["rows"], state["there"]
    acc_in = x["acc"]
    if case["replace"]:
        at = (off + x["slot"]).view(-1)
        new = [x[n].reshape(-1, d) for n in ("k_new", "v_new")]
        k[at], v[at] = [t.clamp(-448, 448).to(k.dtype) if case["cache"] == "fp8" else t for t in new]
        state["kept"][at] = x["pos"].view(1, -1, 1).expand_as(off).reshape(-1)
        acc_in = acc_in.index_fill(0, at, 0.0)
    kk, vv = (_decode4(*state["k4"]), _decode4(*state["v4"])) if case["cache"] == "fp4" else (k.float(), v.float())
    out, w = _attend(case, x["q"].reshape(-1, G, d), kk[rows], vv[rows], there)
    acc = acc_in[rows] + w.sum(1)
    state["acc"][rows[there]] = acc[there]
    may = there & (state["kept"][rows] <= x["pos"].view(1, -1, 1).expand_as(off).reshape(-1, 1) - W)
    least, slot = torch.where(may, acc, math.inf).min(-1)
    slot = torch.where(least < math.inf, slot, -1).int().view_as(off)
    r = {"out": out.view_as(x["q"]), "acc": state["acc"], "slot": slot, "kept": state["kept"]}
    return dict(r, k=k, v=v) if case["replace"] else r


# ---- a pass ------------------------------------------------------------------------------------------
def _handle(case):
    from paper_2506_15724_amd import binding as MB
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    bits = {"store": 4, "attend": 4, "prompt": 0}.get(case["op"], {"fp8": 1, "fp4": 4}.get(case.get("cache"), 0))
    return MB.MadaKV(n_layers=NL, batch=B, n_q_heads=Hq, n_kv_heads=H, head_dim=d, ctx_len=L, window=W, budget=keep,
                     dtype="fp32" if case.get("cache") == "fp32" else "bf16", max_new_tokens=0, out_fp32=1, cache_fp8=bits, device=DEV)


def prepare(case, seed):
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    x = _inputs(case, seed)
    state = {"case": case, "x": x}
    if case["op"] == "prompt" and case["given_lse"]:             # as the prefill attention leaves them
        q, k = x["q"].float().view(NL * B * H, -1, d), x["k"].float().view(NL * B * H, L, d)
        s = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1 / math.sqrt(d)).view(NL, B, Hq, L, L)
        x["lse"] = s.masked_fill_(torch.ones(L, L, dtype=torch.bool, device=DEV).triu_(1), -math.inf).logsumexp(-1)
    rows = NL * B * H * min(keep, L)
    if case["op"] == "store":
        state["k_rows"], state["v_rows"] = (torch.zeros(rows, d, dtype=_dtype(case), device=DEV) for _ in range(2))
    if case["op"] == "attend" or case["op"] == "weights":
        state["out"] = torch.empty(NL, B, Hq, d, dtype=torch.float32, device=DEV)
    if case["op"] == "weights":
        state["acc"], state["slot"] = torch.zeros(rows, device=DEV), torch.zeros(NL, B, H, dtype=torch.int32, device=DEV)
    if own:
        state["eng"] = eng = _handle(case)
        if case["op"] == "attend" or case["op"] == "weights":    # the cache as the prompt's eviction leaves it
            eng.select_gather(0, NL, x["k"], x["v"], x["mask"], x["score"], x["budgets"])
    elif case["op"] == "attend" or case["op"] == "weights":
        at, state["off"], lens = _choose(x, case)
        state["rows"], state["there"] = _padded(state["off"], lens)
        state["kept"] = at[3].int()
        for n in ("k", "v"):
            c = x[n][at]
            if case["op"] == "attend" or case["cache"] == "fp4":
                state[n + "4"], state[n] = _encode4(c), None
            else:
                state[n] = c.clamp(-448, 448).to(torch.float8_e4m3fn) if case["cache"] == "fp8" else c
    if case["op"] == "attend" or case["op"] == "weights":
        for n in ("k", "v", "score", "mask", "budgets"):
            del x[n]
    return state


def run(state):
    case = state["case"]
    if not own:
        return {"store": _store, "attend": _attend4, "prompt": _prompt, "weights": _weights}[case["op"]](state)
    eng, x, NL = state["eng"], state["x"], case["n_layers"]
    if case["op"] == "store":
        eng.select_gather(0, NL, x["k"], x["v"], x["mask"], x["score"], x["budgets"])
        eng.cache_rows(0, NL, state["k_rows"], state["v_rows"])
        return {"k": state["k_rows"], "v": state["v_rows"], "kept": eng.kept_idx, "off": eng.kv_off, "len": eng.kv_len}
    if case["op"] == "attend":
        eng.decode_attn(0, NL, x["q"], None, None, state["out"])
        return {"out": state["out"]}
    if case["op"] == "prompt":
        eng.score_prompt(0, NL, x["q"], x["k"], row_lse=x.get("lse"))
        return {"psi": eng.psi}
    r = {"out": state["out"], "acc": state["acc"], "slot": state["slot"], "kept": eng.kept_idx}
    if not case["replace"]:
        eng.decode_attn_weights(0, NL, x["q"], None, None, state["out"], x["acc"], state["acc"],
                                slot_out=state["slot"], pos=x["pos"], recent=case["window"])
        return r
    eng.decode_attn_weights(0, NL, x["q"], x["k_new"], x["v_new"], state["out"], x["acc"], state["acc"], slot_in=x["slot"],
                            slot_out=state["slot"], pos=x["pos"], recent=case["window"])
    k, v = (t.view(torch.float8_e4m3fn) if case["cache"] == "fp8" else t for t in (eng.k_c, eng.v_c))
    return dict(r, k=k, v=v)


def work(case):
    """Bytes: every input read once, every output written once.  "store": the kept rows of the prompt, their codes, the rows
    read back; candidates' scores and modalities, kept positions.  "attend": the codes and scales, queries, outputs.
    "prompt": queries, keys, the scores (and normalisers).  "weights": the cache's rows, the sums read and written, the
    positions.  Flops: the two products of attention; of "prompt" one over the (query, key) pairs that the causal mask
    leaves, although the normalisers, where they are not given, cost a second one."""
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    rows, code = NL * B * H * min(keep, L), d // 2 + d // 32
    if case["op"] == "store":
        picked = 0 if keep >= L else NL * B * H * (L - W) * 4 + B * L
        return {"bytes": rows * (2 * (2 * d + code + 2 * d) + 4) + picked, "flops": 0}
    if case["op"] == "prompt":
        nbytes = NL * B * ((Hq + H) * L * d * 2 + H * L * 4 + (Hq * L * 4 if case["given_lse"] else 0))
        return {"bytes": nbytes, "flops": 2 * NL * B * Hq * d * (L * (L + 1) // 2)}
    row = code if case["op"] == "attend" else {"bf16": 2 * d, "fp8": d, "fp4": code, "fp32": 4 * d}[case["cache"]]
    nbytes = rows * 2 * row + NL * B * Hq * d * (2 + 4)
    if case["op"] == "weights":
        nbytes += rows * 12 + (NL * B * H * (4 * d + 2 * row) if case["replace"] else 0)
    return {"bytes": nbytes, "flops": 4 * d * rows * (Hq // H)}


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


def _kept(case, x):
    """Kept positions of every head, in the order of the cache's segments: {(layer, item, head): positions}."""
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    mask, score, budgets = x["mask"].cpu().numpy(), x["score"].cpu().numpy(), x["budgets"].cpu().numpy()
    kept = {}
    for b in range(B):
        for l in range(NL):
            for h in range(H):
                if keep >= L:
                    kept[l, b, h] = np.arange(L)
                    continue
                some = []
                for m in (0, 1):
                    of = np.nonzero(mask[b, :L - W] == m)[0]
                    some.append(of[np.lexsort((of, -score[l, b, h][of]))][:budgets[l, b, h, m]])
                kept[l, b, h] = np.sort(np.concatenate(some + [np.arange(L - W, L)]))
    return kept


def exact(case, seed):
    NL, B, Hq, H, d, L, W, keep = _sizes(case)
    x = _inputs(case, seed)
    G, scale = Hq // H, 1 / math.sqrt(d)
    if case["op"] == "prompt":
        if NL * B * Hq * L * L > MOST_PAIRS:
            return None
        psi = torch.zeros(NL, B, H, L, dtype=torch.float64, device=DEV)
        step = max(1, (1 << 27) // L)                            # query rows at a time: 1 GB of logits
        for l in range(NL):
            for b in range(B):
                for j in range(Hq):
                    k = x["k"][l, b, j // G].double().t().contiguous()
                    for r0 in range(0, L, step):
                        q = x["q"][l, b, j, r0:r0 + step].double()
                        n = r0 + q.shape[0]
                        w = torch.exp((q @ k[:, :n]) * scale).tril_(r0)
                        psi[l, b, j // G, :n] += (1 / w.sum(1)) @ w
        return {"psi": psi}
    kept = _kept(case, x)
    if case["op"] == "store":
        rows = {n: torch.cat([_value4(x[n][i][torch.from_numpy(p).to(DEV)]) for i, p in kept.items()]) for n in ("k", "v")}
        return {"k": rows["k"], "v": rows["v"], "kept": None, "off": None, "len": None}
    out = torch.zeros(NL, B, Hq, d, dtype=torch.float64, device=DEV)
    acc = []
    at = 0
    for i, p in kept.items():
        l, b, h = i
        k, v = (x[n][i][torch.from_numpy(p).to(DEV)] for n in ("k", "v"))
        before = x["acc"][at:at + len(p)].double() if case["op"] == "weights" else None
        at += len(p)
        if case.get("replace"):
            s = int(x["slot"][i])
            k[s], v[s], before[s] = x["k_new"][i], x["v_new"][i], 0.0
        if case["op"] == "attend" or case["cache"] == "fp4":
            k, v = _value4(k), _value4(v)
        elif case["cache"] == "fp8":
            k, v = k.clamp(-448, 448).to(torch.float8_e4m3fn), v.clamp(-448, 448).to(torch.float8_e4m3fn)
        s = x["q"][l, b, h * G:(h + 1) * G].double() @ k.double().t().contiguous() * scale
        w = torch.exp(s - s.max(1, keepdim=True).values)
        w /= w.sum(1, keepdim=True)
        out[l, b, h * G:(h + 1) * G] = w @ v.double()
        if before is not None:
            acc.append(before + w.sum(0))
    if case["op"] == "attend":
        return {"out": out}
    r = {"out": out, "acc": torch.cat(acc), "slot": None, "kept": None}
    return dict(r, k=None, v=None) if case["replace"] else r
