"""Engine steps of a small decoder with prefill-only adapters, attention and pages included.

Requests of three adapters are served.  Every adapter has a system prompt that all its requests begin with; its keys and values, which the
adapter edits, are computed once and shared as pages.  A step is: slots for its rows (preft_kv_plan); in every layer the q, k and v projections with the
adapters' LoRA on prompt rows (preft_lora_apply_packed), the rows' keys and values to their slots (preft_kv_store), attention, and the o projection with its LoRA.
The first step prefills the system prompts (whole prompts: preft_prompt_attention); in the second every request sends the rest of its prompt, and in the others one token
(preft_cached_attention, grouped by adapter, so that a system prompt's keys are read once for all its requests).  In the fourth two requests without a system prompt
join: a mixed step, whose layers make both calls on one workspace.

    python examples/serve_step.py            runs the steps and compares every row with the same model in 64 bits

The model is random, of one width throughout and without norms or MLP: what is shown is the calls.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_14217_amd as preft  # noqa: E402

LAYERS, HEADS, KV_HEADS, DIM, RANK, PAGE = 2, 8, 2, 64, 8, 16
WIDTH, KV_WIDTH = HEADS * DIM, KV_HEADS * DIM
LORA_SCALE, ATTN_SCALE = 0.5, 1.0 / math.sqrt(DIM)
SYSTEM = [96, 160, 64]                                     # tokens of the adapters' system prompts: whole pages


def i32(values, device):
    return torch.tensor(values, dtype=torch.int32, device=device)


class Model:
    """Projections of every layer, and each adapter's LoRA of them; pointer tables for the apply calls."""

    def __init__(self, dtype, device, seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)

        def randn(*shape, scale=1.0):
            return (scale * torch.randn(*shape, generator=gen, device=device)).to(dtype)
        self.w, self.lora, self.pools = [], [], []
        for _ in range(LAYERS):
            widths = {"q": WIDTH, "k": KV_WIDTH, "v": KV_WIDTH, "o": WIDTH}
            self.w.append({n: randn(WIDTH, d, scale=WIDTH ** -0.5) for n, d in widths.items()})
            self.lora.append({n: [(randn(RANK, WIDTH, scale=WIDTH ** -0.5), randn(d, RANK, scale=RANK ** -0.5)) for _ in SYSTEM] for n, d in widths.items()})
            self.pools.append({n: (preft.pointer_table([a for a, _ in m]), preft.pointer_table([b for _, b in m])) for n, m in self.lora[-1].items()})


class Engine:
    def __init__(self, model, dtype, device, n_pages=256, max_pages=32):
        self.model, self.dtype, self.device, self.max_pages = model, dtype, device, max_pages
        self.free = list(range(n_pages))[::-1]              # any order
        self.caches = [[torch.empty(n_pages, KV_HEADS, PAGE, DIM, dtype=dtype, device=device) for _ in "kv"] for _ in range(LAYERS)]

    def step(self, x, lengths, prompt, adapters, context, tables, groups=None, prefix=None):
        """x [T, WIDTH]: rows of all requests one after the other; `prompt`: whether a request's rows are prompt rows; `context`: tokens it has in the
        pages; tables [S, max_pages]: block tables, extended in place.  Returns the rows after the last layer."""
        dev, T, S = self.device, x.shape[0], len(lengths)
        start = [0]
        for n in lengths:
            start.append(start[-1] + n)
        seg_start, seg_adapter = i32(start, dev), i32(adapters, dev)
        prefill = i32([n if p else 0 for n, p in zip(lengths, prompt)], dev)
        # slots of the rows, once for all layers
        slot_map, positions = torch.empty(T, dtype=torch.int64, device=dev), torch.empty(T, dtype=torch.int32, device=dev)
        kv_len, counts = torch.empty(S, dtype=torch.int32, device=dev), torch.empty(2, dtype=torch.int32, device=dev)
        preft.preft_kv_plan(slot_map, positions, kv_len, tables, counts, seg_start, i32(context, dev), i32(self.free, dev), PAGE)
        taken = sum(-(-(c + n) // PAGE) - -(-c // PAGE) for c, n in zip(context, lengths))      # the host knows the lengths too
        self.free = self.free[taken:]
        # the schedules of the step: the first layer's calls build them
        adapter_ws = preft.new_workspace(T, S, device=dev, z_rank=RANK, z_proj=3)
        attn_ws = preft.new_attention_workspace(T, S, HEADS, KV_HEADS, DIM, len(prefix or []), device=dev)
        group_start = None if prefix is None else i32(groups, dev)
        group_prefix = None if prefix is None else i32(prefix, dev)
        # whole prompts by their own keys and values, all other rows over the pages
        first = [n if p and c == 0 else 0 for n, p, c in zip(lengths, prompt, context)]
        whole, rest = i32(first, dev), sum(lengths) > sum(first)
        for layer, (w, pools, (k_cache, v_cache)) in enumerate(zip(self.model.w, self.model.pools, self.caches)):
            mode = preft.PREFT_PREFILL_ONLY | (preft.PREFT_SCHEDULE_READY if layer else 0)
            ready = preft.PREFT_SCHEDULE_READY if layer else 0
            qkv = torch.cat([x @ w["q"], x @ w["k"], x @ w["v"]], dim=1)
            q, k, v = qkv[:, :WIDTH], qkv[:, WIDTH:WIDTH + KV_WIDTH], qkv[:, WIDTH + KV_WIDTH:]
            preft.preft_lora_apply_packed([q, k, v], x, seg_start, seg_adapter, prefill, [pools[n][0] for n in "qkv"], [pools[n][1] for n in "qkv"],
                                          RANK, LORA_SCALE, mode, adapter_ws)
            preft.preft_kv_store(k_cache, v_cache, k, v, slot_map)
            out = torch.empty(T, WIDTH, dtype=self.dtype, device=dev)
            if any(first):
                preft.preft_prompt_attention(out, q, k, v, seg_start, whole, HEADS, KV_HEADS, ATTN_SCALE, ready, attn_ws)
            if rest:
                preft.preft_cached_attention(out, q, seg_start, whole, kv_len, k_cache, v_cache, tables, group_start, group_prefix, HEADS, ATTN_SCALE,
                                             ready, attn_ws)
            y = out @ w["o"]
            preft.preft_lora_apply(y, out, seg_start, seg_adapter, prefill, *pools["o"], RANK, LORA_SCALE, preft.PREFT_PREFILL_ONLY | preft.PREFT_SCHEDULE_READY,
                                   adapter_ws)
            x = x + y
        return x


def exact(model, x, n_prompt, adapter):
    """The same for one request, all its tokens at once, in 64 bits on the CPU."""
    x = x.double().cpu()
    n = x.shape[0]
    on = (torch.arange(n) < n_prompt).double()[:, None]
    hidden = torch.ones(n, n).triu(1).bool()
    for w, lora in zip(model.w, model.lora):
        def project(name, h):
            a, b = (m.double().cpu() for m in lora[name][adapter])
            return h @ w[name].double().cpu() + LORA_SCALE * on * (h @ a.T @ b.T)
        q, k, v = project("q", x).view(n, HEADS, DIM), project("k", x).view(n, KV_HEADS, DIM), project("v", x).view(n, KV_HEADS, DIM)
        k, v = k.repeat_interleave(HEADS // KV_HEADS, 1), v.repeat_interleave(HEADS // KV_HEADS, 1)
        s = torch.einsum("ihd,jhd->hij", q, k) * ATTN_SCALE
        p = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
        x = x + project("o", torch.einsum("hij,jhd->ihd", p, v).reshape(n, WIDTH))
    return x


def main(dtype=torch.float32, device="cuda", new_tokens=4, requests=9, seed=1):
    """Serves the requests; the largest error of a row against the model in 64 bits, over the largest value of the row."""
    gen = torch.Generator(device=device).manual_seed(seed)

    def embeddings(n):
        return torch.randn(n, WIDTH, generator=gen, device=device).to(dtype)
    model = Model(dtype, device)
    engine = Engine(model, dtype, device)
    n_adapters = len(SYSTEM)
    system = [embeddings(n) for n in SYSTEM]
    tables = torch.full((n_adapters, engine.max_pages), -1, dtype=torch.int32, device=device)
    got_system = engine.step(torch.cat(system), SYSTEM, [True] * n_adapters, list(range(n_adapters)), [0] * n_adapters, tables)
    # requests stand by adapter: the groups are runs of them, and their tables begin with the shared pages
    adapter = sorted(r % n_adapters for r in range(requests))
    groups = [adapter.index(a) for a in range(n_adapters)] + [requests]
    own = [3 + 5 * r for r in range(requests)]              # tokens of the requests' own prompts
    tokens = [embeddings(n) for n in own]
    more = [embeddings(new_tokens) for _ in range(requests)]
    tables = tables[i32(adapter, device).long()].contiguous()
    context = [SYSTEM[a] for a in adapter]
    got = [engine.step(torch.cat(tokens), own, [True] * requests, adapter, context, tables, groups, SYSTEM).split(own)]
    context = [c + n for c, n in zip(context, own)]
    late, joined = [(0, embeddings(37 + new_tokens)), (2, embeddings(70 + new_tokens))], [37, 70]       # adapter and tokens; how many are the prompt
    got_late = []
    for t in range(new_tokens):
        rows = [m[t:t + 1] for m in more]
        lengths, prompt = [1] * requests, [False] * requests
        if t == 1:                                          # they stand after the groups, in none
            tables = torch.cat([tables, torch.full((len(late), engine.max_pages), -1, dtype=torch.int32, device=device)])
            adapter, context = adapter + [a for a, _ in late], context + [0] * len(late)
        if t >= 1:
            at = context[requests:]
            lengths += [n if t == 1 else 1 for n in joined]
            prompt += [t == 1] * len(late)
            rows += [x[c:c + n] for (_, x), c, n in zip(late, at, lengths[requests:])]
        parts = engine.step(torch.cat(rows), lengths, prompt, adapter, context, tables, groups, SYSTEM).split(lengths)
        got.append(parts[:requests])
        if t >= 1:
            got_late.append(parts[requests:])
        context = [c + n for c, n in zip(context, lengths)]
    worst = 0.0

    def compare(a, b):
        return ((a.double().cpu() - b).abs().amax(1) / b.abs().amax(1)).max().item()
    for a, rows in enumerate(got_system.split(SYSTEM)):
        worst = max(worst, compare(rows, exact(model, system[a], SYSTEM[a], a)))
    for r in range(requests):
        all_ = torch.cat([system[adapter[r]], tokens[r], more[r]])
        want = exact(model, all_, SYSTEM[adapter[r]] + own[r], adapter[r])[SYSTEM[adapter[r]]:]
        worst = max(worst, compare(torch.cat([step[r] for step in got]), want))
    for r, ((a, x), n) in enumerate(zip(late, joined)):
        rows = torch.cat([step[r] for step in got_late])
        worst = max(worst, compare(rows, exact(model, x[:len(rows)], n, a)))
    return worst


if __name__ == "__main__":
    for dtype in (torch.float32, torch.bfloat16):
        print(f"{dtype}: rows off by at most {main(dtype):.1e} of their largest value")
