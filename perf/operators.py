"""The attention side of an engine step: the calls that the key/value pages and attention operators answer for.

A step works on the flattened batch of the apply calls (segments of prompt rows and decode rows).  Four operators
belong to it: ``plan`` extends the block tables and makes the slot map of the batch's rows, ``store`` writes their keys
and values into the pages, ``prompt`` is causal attention over whole packed prompts, and ``cached`` is attention of
decode rows (and of further chunks of a prompt) over the pages, where requests may share a long prefix.

``listed`` names usual calls from the smallest to the largest and ``draw`` makes more of the same kinds.  Lengths are the
quantiles of a length law, so that the work of a case does not depend on the seed; order, pages and all values do.
With ``own`` false ``run`` computes the operators from their formulas with elementary torch operations in 32 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"

# op      plan, store, prompt or cached
# prompts requests with lo..hi new rows ("uniform", or "lognormal" with median lo, sigma 0.8, clipped to [32, hi])
# decode  requests with `rows` new rows each (1; more: tokens proposed ahead that are checked together)
# ctx_lo..ctx_hi  tokens that are in the pages before the step, of every request (prompt: none)
# groups  requests are split evenly into groups that share their first `prefix` tokens; ctx is what follows them
BASE = dict(op="cached", dtype="bf16", heads=32, kv_heads=8, dim=128, prompts=0, lo=0, hi=0, law="uniform",
            decode=0, rows=1, ctx_lo=0, ctx_hi=0, groups=0, prefix=0, page=16)


def _case(name, **kw):
    c = dict(BASE, **kw)
    c["name"] = name
    return c


def listed():
    return [
        # host-bound bookkeeping of a decode step: 32 requests in flight, one new token each
        _case("plan_decode_32", op="plan", decode=32, ctx_lo=500, ctx_hi=4000),
        # the largest mixed batch: 512 prompts (median 512 rows) and 3584 decode rows
        _case("plan_mixed_4096", op="plan", prompts=512, lo=512, hi=8192, law="lognormal", decode=3584, ctx_lo=32, ctx_hi=2048,
              page=64),
        # new keys and values of a decode step of a small batch, stored in 32 bits
        _case("store_decode_f32", op="store", dtype="f32", decode=33, ctx_lo=100, ctx_hi=2000),
        # ... and of the ordinary mixed step of an 8B layer: 32 prompts of 256..2048 rows and 224 decode rows
        _case("store_mixed_8b", op="store", prompts=32, lo=256, hi=2048, decode=224, ctx_lo=100, ctx_hi=2000, page=64),
        # exactness checks in 32 bits: eight prompts of 64 rows, eight decode rows beside them, heads of their own
        _case("prompt_tiny_f32", op="prompt", dtype="f32", heads=8, kv_heads=8, dim=64, prompts=8, lo=64, hi=64, decode=8),
        # chat-length prompts of a small model: seven query heads to a key head, lengths of a few rows to ninety
        _case("prompt_chat_ragged", op="prompt", heads=14, kv_heads=2, dim=64, prompts=40, lo=3, hi=90),
        # prompts of the ordinary mixed step of an 8B layer
        _case("prompt_mixed_8b", op="prompt", prompts=32, lo=256, hi=2048, decode=224),
        # one long prompt at 70B width
        _case("prompt_long_70b", op="prompt", heads=64, prompts=1, lo=16001, hi=16001),
        # a single request, one token: latency
        _case("decode_one_8b", decode=1, ctx_lo=1500, ctx_hi=1500),
        # proposed tokens checked in 32 bits on a small model
        _case("check_ahead_f32", dtype="f32", heads=14, kv_heads=2, dim=64, decode=9, rows=5, ctx_lo=30, ctx_hi=1111),
        # decode rows of the ordinary step of an 8B layer, each with a context of its own
        _case("decode_8b", decode=224, ctx_lo=256, ctx_hi=4096, page=64),
        # 256 requests of 8 adapters with a long system prompt each, at 70B width: prompts are shared, answers are short
        _case("decode_prefix_70b", heads=64, decode=256, ctx_lo=16, ctx_hi=700, groups=8, prefix=8192, page=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = dict(BASE)
        c["op"] = rng.choice(["plan", "store", "prompt", "prompt", "prompt", "cached", "cached", "cached"])
        c["dtype"] = "f32" if rng.random() < 0.2 else "bf16"
        c["heads"], c["kv_heads"], c["dim"] = rng.choice([(32, 8, 128), (32, 8, 128), (64, 8, 128), (14, 2, 64), (8, 8, 64),
                                                          (16, 16, 128), (12, 4, 64), (16, 1, 128)])
        c["page"] = rng.choice([8, 16, 16, 32, 64, 64, 128])
        c["law"] = rng.choice(["uniform", "lognormal"])
        if c["op"] != "cached" or rng.random() < 0.25:
            c["prompts"] = _log_int(rng, 1, 512 if c["op"] in ("plan", "store") else 48 if c["op"] == "prompt" else 4)
            c["lo"] = _log_int(rng, 1, 2048)
            c["hi"] = max(c["lo"], 32, _log_int(rng, 32, 16000 if c["prompts"] < 4 else 4096))
        if c["op"] in ("plan", "store", "cached") or rng.random() < 0.5:
            c["decode"] = _log_int(rng, 1, 4000 if c["op"] == "plan" else 400)
            c["rows"] = rng.choice([1, 1, 1, 1, 2, 3, 5, 8])
        if c["op"] != "prompt":
            c["ctx_lo"] = _log_int(rng, 1, 3000)
            c["ctx_hi"] = c["ctx_lo"] + _log_int(rng, 1, 8000)
        if c["op"] == "cached" and c["prompts"] == 0 and c["decode"] > 1 and rng.random() < 0.5:
            c["groups"] = _log_int(rng, 1, min(c["decode"], 24))
            c["prefix"] = c["page"] * max(1, _log_int(rng, 128, 16384) // c["page"])
            c["ctx_hi"] = c["ctx_lo"] + _log_int(rng, 1, 1000)
        n, ctx, _ = _lengths(c)
        w = work(c)
        if w["flops"] > 4.0e12 or w["bytes"] > 4.0e9 or 3072 in (c["lo"], c["hi"], c["prefix"], c["ctx_lo"], c["ctx_hi"]):
            continue
        # what the plain form lays out whole: padded scores, or padded keys and values
        if c["op"] == "prompt" and c["prompts"] * c["heads"] * int(n.max()) ** 2 > 1.2e10:
            continue
        if c["op"] == "cached":
            most = int((n + ctx).max()) + c["prefix"]
            if len(n) * most * max(c["kv_heads"] * c["dim"], int(n.max()) * c["heads"]) > 4.0e9:
                continue
        return c


def _lengths(c):
    """New rows of each request, tokens of its own before them, and whether it is a prompt: by the case alone."""
    u = (np.arange(c["prompts"]) + 0.5) / max(c["prompts"], 1)
    if c["law"] == "lognormal":
        z = np.sqrt(2.0) * np.array([_inverse_erf(2 * x - 1) for x in u])
        n = np.clip(np.rint(c["lo"] * np.exp(0.8 * z)), min(32, c["hi"]), c["hi"])
    else:
        n = np.rint(c["lo"] + u * (c["hi"] - c["lo"]))
    n = np.concatenate([np.maximum(n, 1), np.full(c["decode"], c["rows"])]).astype(np.int64)
    v = (np.arange(len(n)) * 0.6180339887498949 + 0.5) % 1.0
    ctx = np.rint(c["ctx_lo"] + v * (c["ctx_hi"] - c["ctx_lo"])).astype(np.int64)
    return n, ctx, np.arange(len(n)) < c["prompts"]


def _inverse_erf(x):
    """Rational form of the normal quantile (Winitzki): close enough for a length law."""
    a, t = 0.147, math.log(max(1e-12, 1 - x * x))
    b = 2 / (math.pi * a) + t / 2
    return math.copysign(math.sqrt(math.sqrt(b * b - t / a) - b), x)


def work(case):
    c = case
    n, ctx, prompt = _lengths(c)
    e = 4 if c["dtype"] == "f32" else 2
    S, T, kv_row = len(n), int(n.sum()), c["kv_heads"] * c["dim"]
    if c["op"] == "plan":
        # read: offsets, lengths, the block-table entry of a page that is begun already, the pages handed out
        new = int((-(-(ctx + n) // c["page"]) - -(-ctx // c["page"])).sum())
        begun = int((ctx % c["page"] != 0).sum())
        return {"bytes": 4 * (2 * S + 1 + begun + new) + 12 * T + 4 * (S + new + 2), "flops": 0}
    if c["op"] == "store":
        return {"bytes": T * (4 * kv_row * e + 8), "flops": 0}
    if c["op"] == "prompt":
        n = n[prompt]
        pairs = float((n * (n + 1.0) / 2).sum())
        return {"bytes": int(n.sum()) * e * (2 * c["heads"] * c["dim"] + 2 * kv_row) + 8 * S, "flops": 4.0 * c["dim"] * c["heads"] * pairs}
    pairs = float((n * (c["prefix"] + ctx + (n + 1) / 2.0)).sum())
    keys = float((ctx + n).sum()) + c["prefix"] * max(c["groups"], 0)
    tables = 4.0 * (2 * S + 1 + keys / c["page"])
    return {"bytes": keys * 2 * kv_row * e + T * e * 2 * c["heads"] * c["dim"] + tables, "flops": 4.0 * c["dim"] * c["heads"] * pairs}


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def prepare(case, seed):
    c = dict(case)
    rng = np.random.Generator(np.random.PCG64(seed))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device=DEV, dtype=dtype)

    n, ctx, prompt = _lengths(c)
    order = rng.permutation(len(n))                       # requests stand in the batch in any order
    n, ctx, prompt = n[order], ctx[order], prompt[order]
    S, T, page, kv_row = len(n), int(n.sum()), c["page"], c["kv_heads"] * c["dim"]
    start = np.concatenate([[0], np.cumsum(n)])
    s = {"case": c, "S": S, "T": T, "most_new": int(n.max()), "seg_start": _i32(start), "host": (n, ctx, prompt, start)}
    s["scale"] = 1.0 / math.sqrt(c["dim"])

    if c["op"] in ("plan", "store", "cached"):
        shared = c["prefix"] // page                      # pages of a shared prefix: whole ones
        have = -(-ctx // page) if c["op"] == "plan" else -(-(ctx + n) // page)
        want = -(-(ctx + n) // page)
        pages = rng.permutation(int(want.sum()) + shared * c["groups"] + 7).astype(np.int64)   # the pool has some to spare
        own_pages = shared * c["groups"]
        max_pages = shared + int(want.max()) + 3
        table = np.full((S, max_pages), -1, dtype=np.int64)
        first = own_pages + np.concatenate([[0], np.cumsum(have)])[:-1]
        k = np.arange(max_pages)
        mine = k[None, :] < have[:, None]
        np.copyto(table[:, shared:], np.where(mine, pages[np.where(mine, first[:, None] + k, 0)], -1)[:, : max_pages - shared])
        if c["groups"]:
            cut = np.round(np.linspace(0, S, c["groups"] + 1)).astype(np.int64)
            group = np.repeat(np.arange(c["groups"]), np.diff(cut))
            table[:, :shared] = pages[group[:, None] * shared + np.arange(shared)[None, :]]
            s["group_start"], s["group_prefix_len"] = _i32(cut), _i32(np.full(c["groups"], shared * page))
        s["n_pages"], s["max_pages"] = len(pages), max_pages

    if c["op"] == "plan":
        s["ctx_len"], s["block_table"] = _i32(ctx), _i32(table)
        s["free_pages"] = _i32(pages[own_pages + int(have.sum()):])
        s["slot_map"] = torch.empty(T, dtype=torch.int64, device=DEV)
        s["positions"] = torch.empty(T, dtype=torch.int32, device=DEV)
        s["kv_len"] = torch.empty(S, dtype=torch.int32, device=DEV)
        s["counts"] = torch.empty(2, dtype=torch.int32, device=DEV)
        return s

    if c["op"] == "store":
        # keys and values are columns of the fused projection's output; now and then a row is padding without a slot
        qkv = randn(T, (c["heads"] + 2 * c["kv_heads"]) * c["dim"])
        s["k"], s["v"] = qkv[:, c["heads"] * c["dim"]:][:, :kv_row], qkv[:, c["heads"] * c["dim"] + kv_row:]
        request = np.repeat(np.arange(S), n)
        at = ctx[request] + np.arange(T) - start[request]
        slot = table[request, at // page] * page + at % page
        slot[rng.random(T) < 0.01] = -1
        s["slot_map"] = torch.from_numpy(slot).to(DEV)
        # one page more than the slots name: the plain form puts rows without a slot there
        s["pool"] = [torch.zeros(len(pages) + 1, c["kv_heads"], page, c["dim"], dtype=dtype, device=DEV) for _ in "kv"]
        s["k_cache"], s["v_cache"] = (p[:-1] for p in s["pool"])
        return s

    heads = c["heads"] * c["dim"]
    if c["op"] == "prompt":
        qkv = randn(T, heads + 2 * kv_row)
        s["q"], s["k"], s["v"] = qkv[:, :heads], qkv[:, heads:heads + kv_row], qkv[:, heads + kv_row:]
        s["seg_prefill_len"] = _i32(np.where(prompt, n, 0))
        s["prompts"] = torch.from_numpy(np.flatnonzero(prompt)).to(DEV)
        s["most_new"] = int(n[prompt].max())
    else:
        s["q"] = randn(T, heads)
        s["k_cache"] = randn(len(pages), c["kv_heads"], page, c["dim"])
        s["v_cache"] = randn(len(pages), c["kv_heads"], page, c["dim"])
        s["block_table"], s["kv_len"] = _i32(table), _i32(c["prefix"] + ctx + n)
        s["most_pages"] = shared + int(want.max())
    s["out"] = torch.zeros(T, heads, dtype=dtype, device=DEV)
    if own:                                               # the scratch memory that a serving program keeps for its steps
        import paper_2605_14217_amd as preft
        s["workspace"] = preft.new_attention_workspace(T, S, c["heads"], c["kv_heads"], c["dim"], c["groups"], device=DEV)
    return s


def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        return _OWN[op](s)
    return _PLAIN[op](s)


# ---- the framework's calls --------------------------------------------------------------------------------------

def _own_plan(s):
    import paper_2605_14217_amd as preft
    preft.preft_kv_plan(s["slot_map"], s["positions"], s["kv_len"], s["block_table"], s["counts"], s["seg_start"], s["ctx_len"],
                        s["free_pages"], s["case"]["page"])
    return {"slot_map": s["slot_map"], "positions": s["positions"], "kv_len": s["kv_len"], "block_table": s["block_table"],
            "counts": s["counts"]}


def _own_store(s):
    import paper_2605_14217_amd as preft
    preft.preft_kv_store(s["k_cache"], s["v_cache"], s["k"], s["v"], s["slot_map"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_prompt(s):
    import paper_2605_14217_amd as preft
    c = s["case"]
    preft.preft_prompt_attention(s["out"], s["q"], s["k"], s["v"], s["seg_start"], s["seg_prefill_len"], c["heads"], c["kv_heads"],
                                 s["scale"], 0, s["workspace"])
    return s["out"]


def _own_cached(s):
    import paper_2605_14217_amd as preft
    preft.preft_cached_attention(s["out"], s["q"], s["seg_start"], None, s["kv_len"], s["k_cache"], s["v_cache"], s["block_table"],
                                 s.get("group_start"), s.get("group_prefix_len"), s["case"]["heads"], s["scale"], 0, s["workspace"])
    return s["out"]


# ---- the plain forms --------------------------------------------------------------------------------------------

def _plain_plan(s):
    page, S, T = s["case"]["page"], s["S"], s["T"]
    start, ctx, table, free = s["seg_start"].long(), s["ctx_len"].long(), s["block_table"].long(), s["free_pages"].long()
    n = start[1:] - start[:-1]
    have, want = (ctx + page - 1) // page, (ctx + n + page - 1) // page
    end = torch.cumsum(want - have, 0)
    k = torch.arange(s["max_pages"], device=DEV)
    fresh = (k >= have[:, None]) & (k < want[:, None])
    pick = (end - (want - have))[:, None] + k - have[:, None]
    table = torch.where(fresh, free[pick.clamp(0, len(free) - 1)], table)
    row = torch.arange(T, device=DEV)
    seg = torch.searchsorted(start, row, right=True) - 1
    at = ctx[seg] + row - start[seg]
    slot = table[seg, at // page] * page + at % page
    counts = torch.stack([end[-1], torch.zeros_like(end[-1])])
    return {"slot_map": slot, "positions": at.int(), "kv_len": (ctx + n).int(), "block_table": table.int(), "counts": counts.int()}


def _plain_store(s):
    c = s["case"]
    slot = torch.where(s["slot_map"] >= 0, s["slot_map"], s["n_pages"] * c["page"])
    at, off = slot // c["page"], slot % c["page"]
    s["pool"][0][at, :, off] = s["k"].reshape(-1, c["kv_heads"], c["dim"])
    s["pool"][1][at, :, off] = s["v"].reshape(-1, c["kv_heads"], c["dim"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attend(s, q, k, v, row, seen):
    """softmax(q k^T scale) v in 32 bits, written to the rows `row` [S, R] (T: to none).  q [S, R, heads * dim], k and v
    [S, kv_heads, K, dim], seen [S, R, K]: which keys a row sees.  A row that sees none is zero."""
    c = s["case"]
    S, R, K = seen.shape
    G = c["heads"] // c["kv_heads"]
    q = q.float().view(S, R, c["kv_heads"], G, c["dim"]).permute(0, 2, 3, 1, 4).reshape(S, c["kv_heads"], G * R, c["dim"])
    p = torch.matmul(q, k.float().transpose(2, 3).contiguous())
    p = p.mul_(s["scale"]).view(S, c["kv_heads"], G, R, K).masked_fill_(~seen[:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True).clamp_(min=-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(S, c["kv_heads"], G * R, K), v.float().contiguous()).view(S, c["kv_heads"], G, R, c["dim"])
    o = (o / total.clamp(min=1e-37)).permute(0, 3, 1, 2, 4).reshape(S, R, c["heads"] * c["dim"])
    out = torch.zeros(s["T"] + 1, c["heads"] * c["dim"], dtype=s["q"].dtype, device=DEV)
    out[row] = o.to(s["q"].dtype)
    return out[:-1]


def _plain_prompt(s):
    c = s["case"]
    start = s["seg_start"].long()[s["prompts"]]
    n = s["seg_prefill_len"].long()[s["prompts"]]
    i = torch.arange(s["most_new"], device=DEV)
    there = i < n[:, None]
    row = torch.where(there, start[:, None] + i, 0)
    k = s["k"][row].view(*row.shape, c["kv_heads"], c["dim"]).transpose(1, 2)
    v = s["v"][row].view(*row.shape, c["kv_heads"], c["dim"]).transpose(1, 2)
    seen = (i[None, :] <= i[:, None]) & there[:, None, :]
    return _attend(s, s["q"][row], k, v, torch.where(there, row, s["T"]), seen)


def _plain_cached(s):
    c = s["case"]
    start = s["seg_start"].long()
    n = start[1:] - start[:-1]
    i = torch.arange(s["most_new"], device=DEV)
    there = i < n[:, None]
    row = torch.where(there, start[:-1, None] + i, 0)
    pages = s["block_table"][:, : s["most_pages"]].long().clamp(min=0)
    k = s["k_cache"][pages].transpose(1, 2).reshape(s["S"], c["kv_heads"], -1, c["dim"])
    v = s["v_cache"][pages].transpose(1, 2).reshape(s["S"], c["kv_heads"], -1, c["dim"])
    j = torch.arange(k.shape[2], device=DEV)
    sees = s["kv_len"].long()[:, None] - n[:, None] + 1 + i          # keys that row i of a request sees
    seen = (j < sees[:, :, None]) & there[:, :, None]
    return _attend(s, s["q"][row], k, v, torch.where(there, row, s["T"]), seen)


_OWN = {"plan": _own_plan, "store": _own_store, "prompt": _own_prompt, "cached": _own_cached}
_PLAIN = {"plan": _plain_plan, "store": _plain_store, "prompt": _plain_prompt, "cached": _plain_cached}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    """Request by request and head by head, from the same inputs: every value in 64 bits."""
    c = case
    s = prepare(case, seed)
    n, ctx, prompt, start = s["host"]
    if c["op"] == "plan":
        return None                                       # whole numbers
    if c["op"] == "store":
        k, v = (torch.zeros_like(s["k_cache"], dtype=torch.float64) for _ in "kv")
        slot = s["slot_map"]
        rows = torch.nonzero(slot >= 0).squeeze(1)
        for h in range(c["kv_heads"]):
            cols = slice(h * c["dim"], (h + 1) * c["dim"])
            k[slot[rows] // c["page"], h, slot[rows] % c["page"]] = s["k"][rows, cols].double()
            v[slot[rows] // c["page"], h, slot[rows] % c["page"]] = s["v"][rows, cols].double()
        return {"k_cache": k, "v_cache": v}
    out = torch.zeros(s["T"], c["heads"], c["dim"], dtype=torch.float64, device=DEV)
    q = s["q"].view(s["T"], c["heads"], c["dim"])
    G = c["heads"] // c["kv_heads"]
    for r in range(s["S"]):
        if c["op"] == "prompt" and not prompt[r]:
            continue
        at, rows = int(start[r]), int(n[r])
        if c["op"] == "prompt":
            K = s["k"][at:at + rows].reshape(rows, c["kv_heads"], c["dim"]).transpose(0, 1)
            V = s["v"][at:at + rows].reshape(rows, c["kv_heads"], c["dim"]).transpose(0, 1)
        else:
            keys = c["prefix"] + int(ctx[r]) + rows
            pages = s["block_table"][r, : -(-keys // c["page"])].long()
            K = s["k_cache"][pages].transpose(0, 1).reshape(c["kv_heads"], -1, c["dim"])[:, :keys]
            V = s["v_cache"][pages].transpose(0, 1).reshape(c["kv_heads"], -1, c["dim"])[:, :keys]
        hidden = torch.ones(rows, K.shape[1], dtype=torch.bool, device=DEV).triu(K.shape[1] - rows + 1)
        for h in range(c["heads"]):
            x = (q[at:at + rows, h].double() @ K[h // G].double().t().contiguous()) / math.sqrt(c["dim"])
            w = torch.softmax(x.masked_fill_(hidden, -math.inf), dim=1)
            out[at:at + rows, h] = w @ V[h // G].double()
    return out.view(s["T"], -1)


if __name__ == "__main__":
    for case in listed() + [draw(random.Random(k)) for k in range(6)]:
        print(case.get("name", "drawn"), case, work(case))
