"""Attention of prompts and over pages against the definitions in 64 bits, through the C ABI: within bounds that follow from the arithmetic
(attention_reference), other rows untouched, and what a row does not see kept from it."""
import math

import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2605_14217_amd as preft

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HEADS = [("bf16", 8, 2, 128), ("bf16", 7, 1, 64), ("f32", 6, 3, 64), ("f32", 4, 1, 128), ("bf16", 3, 3, 128), ("bf16", 40, 1, 64)]


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def starts(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int64)


def guarded(T, width, dtype, pad):
    """An output whose neighbours are watched: 2 rows around it and `pad` columns beside it."""
    buf = torch.full((T + 4, width + pad), 7.5, dtype=dtype, device="cuda")
    return buf, buf[2:2 + T, :width]


def check_guard(buf, T, width):
    assert bool((buf[:2] == 7.5).all()) and bool((buf[2 + T:] == 7.5).all()) and bool((buf[:, width:] == 7.5).all()), "written beside the output"


# ---- prompts ----------------------------------------------------------------------------------------------------

def prompt_case(dtype, H, Hkv, D, n, prefill, seed=0, sharp=1.0, edit=None, pad=16, layout="fused"):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    start, td = starts(n), DT[dtype]
    T, wq, wk = int(start[-1]), H * D, Hkv * D
    if layout == "fused":
        qkv = normal(gen, T, wq + 2 * wk + pad).to(td)
        q, k, v = qkv[:, :wq], qkv[:, wq:wq + wk], qkv[:, wq + wk:wq + 2 * wk]
    else:
        q, k, v = normal(gen, T, wq).to(td), normal(gen, T, wk + pad).to(td)[:, :wk], normal(gen, T, wk).to(td)
    q *= sharp
    if edit:
        edit(q, k, v, start)
    buf, out = guarded(T, wq, td, pad)
    before = out.clone().cpu()
    scale = 1.0 / math.sqrt(D)
    ws = preft.new_attention_workspace(T, len(n), H, Hkv, D)
    args = (q, k, v, i32(start), i32(prefill), H, Hkv, scale)
    preft.preft_prompt_attention(out, *args, 0, ws)
    torch.cuda.synchronize()
    check_guard(buf, T, wq)
    return out, before, args, ws, ref.prompt(q.cpu(), k.cpu(), v.cpu(), start, prefill, H, Hkv, scale)


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
def test_prompts_of_every_length(dtype, H, Hkv, D):
    """One row to several tiles, empty segments, decode rows between, prompts that end inside their segment."""
    print(f"\n[case] prompts {dtype} {H}/{Hkv}x{D}", flush=True)
    n = [1, 0, 2, 31, 32, 1, 33, 63, 64, 65, 1, 127, 128, 129, 20, 200]
    prefill = [1, 0, 2, 31, 32, 0, 33, 63, 64, 65, 0, 127, 128, 129, 7, 500]       # 500: cut to the segment
    out, before, _, _, want = prompt_case(dtype, H, Hkv, D, n, prefill)
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
@pytest.mark.parametrize("sharp", [0.01, 6.0, 40.0])
def test_prompts_with_flat_and_sharp_weights(dtype, H, Hkv, D, sharp):
    """Weights that are all alike, and rows that follow one key after another as the largest changes from tile to tile."""
    print(f"\n[case] sharp {sharp} {dtype} {H}/{Hkv}x{D}", flush=True)

    def grow(q, k, v, start):                                # scores rise along the keys: the running maximum moves in every tile
        k *= torch.linspace(0.1, 2.0, k.shape[0], device=k.device)[:, None].to(k.dtype)
    out, before, _, _, want = prompt_case(dtype, H, Hkv, D, [150, 300], [150, 300], sharp=sharp, edit=grow, layout="apart")
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
def test_a_long_prompt_whose_keys_are_divided(dtype, H, Hkv, D):
    """Few tiles and many keys: the schedule cuts the keys and joins the parts.  Rows at both ends and between are compared."""
    print(f"\n[case] long prompt {dtype} {H}/{Hkv}x{D}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(5)
    T = 2111
    q, k, v = (normal(gen, T, w * D).to(DT[dtype]) for w in (H, Hkv, Hkv))
    out = torch.zeros_like(q)
    ws = preft.new_attention_workspace(T, 1, H, Hkv, D)
    preft.preft_prompt_attention(out, q, k, v, i32([0, T]), i32([T]), H, Hkv, 1 / math.sqrt(D), 0, ws)
    assert preft.preft_schedule_counts(ws)[1] > 0, "nothing was divided"
    rows = [0, 1, 63, 64, 511, 512, 513, 1023, 1300, 2047, 2048, 2109, 2110]
    qc, kc, vc = q.cpu(), k.cpu(), v.cpu()
    for t in rows:
        o, bound = ref.attend_row(qc[t].double().view(H, D), kc[:t + 1].double().view(t + 1, Hkv, D).transpose(0, 1),
                                  vc[:t + 1].double().view(t + 1, Hkv, D).transpose(0, 1), 1 / math.sqrt(D), q.dtype)
        assert ((out[t].cpu().double().view(H, D) - o).abs() <= bound).all(), t


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
def test_later_rows_do_not_reach_earlier_ones(dtype, H, Hkv, D, bad):
    """Keys and values of later rows, of other segments and of rows that are no prompt may hold anything."""
    print(f"\n[case] {bad} in later rows, {dtype} {H}/{Hkv}x{D}", flush=True)
    n, prefill = [40, 3, 90, 1, 50], [40, 0, 90, 0, 20]
    start = starts(n)

    def edit(q, k, v, start):
        for t in (start[0] + 39, start[1], start[2] + 70, start[3], start[4] + 20, start[4] + 49):   # row 70 of the third: rows 70.. see it
            k[t], v[t] = bad, bad
        v[start[2] + 75, ::2] = bad                          # only values, and only some
        k[start[2] + 85, 0] = bad
    out, before, _, _, _ = prompt_case(dtype, H, Hkv, D, n, prefill, edit=edit)
    clean, _, _, _, want = prompt_case(dtype, H, Hkv, D, n, prefill)
    want = {t: w for t, w in want.items() if t not in range(start[2] + 70, start[2] + 90) and t != start[0] + 39}
    got, ok = out.cpu(), clean.cpu()
    for t in list(range(start[2] + 70, start[2] + 90)) + [start[0] + 39]:
        assert not torch.isfinite(got[t]).any() or bad == -float("inf"), t
        got[t], before[t] = ok[t], ok[t]
    ref.check(got, want, before)


def test_a_row_that_sees_an_infinite_value():
    """v = inf at a key with a weight: inf in that dimension alone; a NaN likewise."""
    print("\n[case] infinite values that are seen", flush=True)
    H, D, T = 2, 64, 70

    def edit(q, k, v, start):
        v[10, 3], v[60, 5], v[65, 7] = float("inf"), -float("inf"), float("nan")
    out, _, _, _, _ = prompt_case("bf16", H, 1, D, [T], [T], edit=edit)
    got = out.float().view(T, H, D)
    for t in range(T):
        for d, at, ok in ((3, 10, lambda x: (x == float("inf")).all()), (5, 60, lambda x: (x == -float("inf")).all()), (7, 65, lambda x: x.isnan().all())):
            assert bool(ok(got[t, :, d])) if t >= at else bool(torch.isfinite(got[t, :, d]).all()), (t, d)
        rest = got[t][:, [d for d in range(D) if d not in (3, 5, 7)]]
        assert torch.isfinite(rest).all()


def test_prompts_on_another_stream_and_from_a_ready_schedule():
    print("\n[case] ready schedule, streams", flush=True)
    out, before, args, ws, want = prompt_case("bf16", 8, 2, 128, [70, 1, 150], [70, 0, 150])
    first = out.clone()
    out.fill_(1.0)
    before = out.clone().cpu()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    preft.preft_prompt_attention(out, *args, preft.PREFT_SCHEDULE_READY, ws, stream=side)
    side.synchronize()
    ref.check(out.cpu(), want, before)
    rows = sorted(want)
    assert torch.equal(out[rows], first[rows])                # the same bits
    # another batch does not run on that schedule
    q, k, v, ss, sp, H, Hkv, scale = args
    small = torch.zeros(100, 8 * 128, dtype=torch.bfloat16, device="cuda")
    preft.preft_prompt_attention(small, q[:100], k[:100], v[:100], i32([0, 100]), i32([100]), H, Hkv, scale, preft.PREFT_SCHEDULE_READY, ws)
    assert not small.any()
    with pytest.raises(preft.PreftError) as e:
        preft.preft_schedule_counts(ws)
    assert e.value.code == preft.PREFT_ESCHEDULE


# ---- over the pages ---------------------------------------------------------------------------------------------

def cached_case(dtype, H, Hkv, D, page, rows, kv, prefill=None, groups=None, prefix=None, seed=0, poison=float("nan"), sharp=1.0, pad=8, extra=3,
                big=False):
    """groups: [(first, past the last)] segments; prefix: their shared tokens.  Whatever no row may see is `poison`."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.Generator(np.random.PCG64(seed))
    kv = np.asarray(kv, np.int64)
    n = np.asarray(rows, np.int64) + (0 if prefill is None else np.asarray(prefill, np.int64))
    start, S, td = starts(n), len(n), DT[dtype]
    T, need = int(start[-1]), -(-np.maximum(kv, 0) // page)
    max_pages = int(max(need.max(), max(-(-p // page) for p in prefix) if prefix else 0)) + 2
    # shared pages first, each request's own after them
    shared = {s: g for g, (a, b) in enumerate(groups or []) for s in range(a, b)}
    n_pages = int(need.sum()) + sum(-(-p // page) for p in (prefix or [])) + extra
    ids, used, table = rng.permutation(n_pages), 0, np.full((S, max_pages), n_pages + 1000, np.int64)
    table[:, -1] = -5
    group_pages = []
    for p in prefix or []:
        group_pages.append(ids[used:used + -(-p // page)])
        used += -(-p // page)
    k_cache, v_cache = (torch.full((n_pages, Hkv, page, D), poison, dtype=td, device="cuda") for _ in "kv")

    def fill(pages, tokens):
        for i, p in enumerate(pages):
            m = min(page, tokens - i * page)
            k_cache[p, :, :m] = normal(gen, Hkv, m, D).to(td)
            v_cache[p, :, :m] = normal(gen, Hkv, m, D).to(td)
    for g, p in enumerate(prefix or []):
        fill(group_pages[g], p)
    for s in range(S):
        own_from = 0
        if s in shared:
            p = prefix[shared[s]]
            own_from = p // page                               # whole pages are shared, a page that the prefix ends in is a copy
            table[s, : -(-p // page)] = group_pages[shared[s]]
        count = max(0, int(need[s]) - own_from)
        pages = ids[used:used + count]
        used += count
        table[s, own_from:own_from + count] = pages
        fill(pages, int(max(kv[s], 0)) - own_from * page)
        if s in shared and prefix[shared[s]] % page and count:
            m = prefix[shared[s]] % page
            for c in (k_cache, v_cache):
                c[pages[0], :, :m] = c[group_pages[shared[s]][-1], :, :m]
    assert used <= n_pages
    q = (sharp * normal(gen, T, H * D + pad)).to(td)[:, : H * D]
    buf, out = guarded(T, H * D, td, pad)
    before = out.clone().cpu()
    scale = 1.0 / math.sqrt(D)
    dev_table = i32(table)
    G = len(prefix or [])
    gs = gp = None
    if G:                                                      # the runs as given are consecutive; in between: none
        gs, gp = i32([a for a, _ in groups] + [groups[-1][1]]), i32(prefix)
    ws = preft.new_attention_workspace(T, S, H, Hkv, D, G)
    args = (q, i32(start), None if prefill is None else i32(prefill), i32(kv), k_cache, v_cache, dev_table)
    preft.preft_cached_attention(out, *args, gs, gp, H, scale, 0, ws)
    torch.cuda.synchronize()
    check_guard(buf, T, H * D)
    want = ref.cached(q.cpu(), start, prefill, kv, k_cache.cpu(), v_cache.cpu(), table, H, scale)
    return out, before, want, args, ws, (gs, gp, H, scale)


@pytest.mark.parametrize("page", [8, 16, 64, 1024])
@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
def test_decode_rows_of_every_length(dtype, H, Hkv, D, page):
    """No key at all, one, lengths around tiles and pages; prompts between the decode rows; everything that is not a token is NaN."""
    print(f"\n[case] decode {dtype} {H}/{Hkv}x{D} page={page}", flush=True)
    kv = [0, 1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 700]
    prefill = [0] * len(kv)
    prefill[3], prefill[8] = 5, 40
    out, before, want, *_ = cached_case(dtype, H, Hkv, D, page, [1] * len(kv), kv, prefill)
    assert not out[0].any()                                    # a request without tokens
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
def test_several_rows_of_a_request(dtype, H, Hkv, D):
    """Tokens proposed ahead, chunks of prompts, and rows whose own keys are not there: the first of them see fewer tokens, or none."""
    print(f"\n[case] rows {dtype} {H}/{Hkv}x{D}", flush=True)
    rows, kv = [1, 5, 0, 8, 3, 70, 150, 4, 6], [40, 77, 33, 8, 2, 70, 400, 0, 300]
    out, before, want, *_ = cached_case(dtype, H, Hkv, D, 16, rows, kv)
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
def test_one_long_request(dtype, H, Hkv, D):
    """A row whose keys are divided among many workgroups."""
    print(f"\n[case] long decode {dtype} {H}/{Hkv}x{D}", flush=True)
    out, before, want, _, ws, _ = cached_case(dtype, H, Hkv, D, 64, [1, 1], [9001, 17], sharp=3.0)
    assert preft.preft_schedule_counts(ws)[1] > 0
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
def test_requests_that_share_a_prefix(dtype, H, Hkv, D):
    """Groups of several sizes, prefixes inside a page and at its end, members that are shorter than the prefix, end at it, or have no row; a group of
    one; requests in no group before, between (a run without prefix) and after."""
    print(f"\n[case] groups {dtype} {H}/{Hkv}x{D}", flush=True)
    rows = [1, 1, 2, 1, 0, 1, 1, 1, 1, 1, 3, 1]
    kv = [30, 300, 333, 290, 250, 100, 256, 80, 500, 90, 700, 20]
    groups, prefix = [(1, 7), (7, 8), (8, 9), (9, 11)], [256, 0, 400, 75]
    out, before, want, args, ws, rest = cached_case(dtype, H, Hkv, D, 16, rows, kv, groups=groups, prefix=prefix)
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)
    again = torch.full_like(out, 3.0)
    gs, gp, H, scale = rest
    preft.preft_cached_attention(again, *args, gs, gp, H, scale, preft.PREFT_SCHEDULE_READY, ws)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:3])
def test_many_rows_share_a_long_prefix(dtype, H, Hkv, D):
    """More columns than a unit has, a prefix that is divided, members with parts in two tiles."""
    print(f"\n[case] wide group {dtype} {H}/{Hkv}x{D}", flush=True)
    rng = np.random.Generator(np.random.PCG64(3))
    S = 45
    out, before, want, *_ = cached_case(dtype, H, Hkv, D, 64, [1] * S, 1030 + rng.integers(0, 100, size=S), groups=[(0, 30), (30, S)], prefix=[1024, 1001])
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype,H,Hkv,D", [("bf16", 8, 4, 128), ("bf16", 4, 2, 64), ("f32", 2, 2, 64)])
def test_many_short_requests(dtype, H, Hkv, D):
    """Units enough that each is one wavefront's: decode rows, some of several, with and without groups; and short prompts."""
    print(f"\n[case] many short requests {dtype} {H}/{Hkv}x{D}", flush=True)
    rng = np.random.Generator(np.random.PCG64(8))
    S = 1100 // Hkv + 40
    kv = rng.integers(0, 150, size=S)
    kv[::7] = rng.integers(300, 900, size=len(kv[::7]))
    out, before, want, *_ = cached_case(dtype, H, Hkv, D, 16, rng.integers(0, 3, size=S), kv)
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)
    cut = [0, S // 3, S - 60]
    out, before, want, *_ = cached_case(dtype, H, Hkv, D, 16, np.ones(S, int), 100 + kv, groups=[(cut[0], cut[1]), (cut[1], cut[2])], prefix=[96, 100])
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)
    n = rng.integers(0, 16, size=S)
    n[5] = 90
    out, before, _, _, want = prompt_case(dtype, H, Hkv, D, n, n)
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
def test_tokens_that_only_later_rows_see(dtype, H, Hkv, D, bad):
    print(f"\n[case] {bad} in later tokens, {dtype} {H}/{Hkv}x{D}", flush=True)
    rows, kv = [6, 80], [50, 200]
    out, before, want, args, ws, rest = cached_case(dtype, H, Hkv, D, 16, rows, kv)
    q, ss, sp, kvl, kc, vc, table = args
    for s, token in ((0, 47), (1, 170)):                       # seen by rows 3.. of the first and 50.. of the second
        p = int(table[s, token // 16])
        kc[p, :, token % 16], vc[p, :, token % 16] = bad, bad
    gs, gp, H, scale = rest
    got = torch.full_like(out, 7.5)
    preft.preft_cached_attention(got, *args, gs, gp, H, scale, 0, ws)
    hit = list(range(3, 6)) + list(range(6 + 50, 86))
    assert not torch.isfinite(got[hit]).any()
    got[hit] = out[hit]
    ref.check(got.cpu(), want, before)


def test_pages_past_32_bits():
    """Pages whose byte offset does not fit 32 bits."""
    print("\n[case] pages past 4 GiB", flush=True)
    H, Hkv, D, page = 8, 8, 128, 64
    n_pages = (5 << 30) // (Hkv * D * page * 2)
    gen = torch.Generator(device="cuda").manual_seed(1)
    kc, vc = (torch.zeros(n_pages, Hkv, page, D, device="cuda", dtype=torch.bfloat16) for _ in "kv")
    table = np.array([[n_pages - 1, (4 << 30) // (Hkv * D * page * 2), 0, n_pages // 2]])
    for p in table[0]:
        kc[p], vc[p] = normal(gen, Hkv, page, D).bfloat16(), normal(gen, Hkv, page, D).bfloat16()
    q = normal(gen, 1, H * D).bfloat16()
    out = torch.zeros_like(q)
    preft.preft_cached_attention(out, q, i32([0, 1]), None, i32([250]), kc, vc, i32(table), None, None, H, 0.1, 0,
                                 preft.new_attention_workspace(1, 1, H, Hkv, D))
    pages = torch.from_numpy(table[0]).cuda()
    small = ref.cached(q.cpu(), [0, 1], None, [250], kc[pages].cpu(), vc[pages].cpu(), np.arange(4)[None], H, 0.1)
    ref.check(out.cpu(), small, torch.zeros_like(q).cpu())


def test_malformed_tables_stay_in_bounds():
    """Offsets that decrease, lengths beyond the table, groups out of order, pages outside the pool: unspecified results, no fault, other rows of the
    guard untouched."""
    print("\n[case] malformed tables", flush=True)
    H, Hkv, D, page, T, S = 4, 2, 64, 16, 60, 5
    kc, vc = (torch.randn(7, Hkv, page, D, device="cuda") for _ in "kv")
    q = torch.randn(T, H * D, device="cuda")
    table = i32([[0, 99, -3, 2 ** 30]] * S)
    for start, kv, gs, gp in (([0, 50, 20, 90, -4, 60], [2 ** 31 - 1, 60, -9, 64, 33], [3, 0, 9], [64, 2 ** 30]),
                              ([5, 5, 5, 100, 100, 1], [64, 64, 64, 64, 64], [-2, 7, 2], [70, -1])):
        buf, out = guarded(T, H * D, torch.float32, 8)
        preft.preft_cached_attention(out, q, i32(start), None, i32(kv), kc, vc, table, i32(gs), i32(gp), H, 0.1, 0,
                                     preft.new_attention_workspace(T, S, H, Hkv, D, 2))
        torch.cuda.synchronize()
        check_guard(buf, T, H * D)
        buf, out = guarded(T, H * D, torch.float32, 8)
        preft.preft_prompt_attention(out, q, q[:, :Hkv * D], q[:, Hkv * D:2 * Hkv * D], i32(start), i32(kv), H, Hkv, 0.1, 0,
                                     preft.new_attention_workspace(T, S, H, Hkv, D))
        torch.cuda.synchronize()
        check_guard(buf, T, H * D)


def test_captured_calls_follow_the_tables():
    """A step's calls in a graph, replayed with other contents of the same tables between eager work: every replay as the eager call."""
    print("\n[case] graph", flush=True)
    H, Hkv, D, page, S = 8, 2, 128, 16, 6
    gen = torch.Generator(device="cuda").manual_seed(2)
    kc, vc = (normal(gen, 60, Hkv, page, D).bfloat16() for _ in "kv")
    qkv = normal(gen, 90, (H + 2 * Hkv) * D).bfloat16()
    q, k, v = qkv[:, :H * D], qkv[:, H * D:(H + Hkv) * D], qkv[:, (H + Hkv) * D:]
    start, prefill, kv = i32([0, 50, 51, 52, 53, 89, 90]), i32([50, 0, 0, 0, 36, 0]), i32([0, 100, 33, 128, 0, 7])
    table = i32(np.random.Generator(np.random.PCG64(0)).permutation(60).reshape(S, 10))
    gs, gp = i32([1, 4]), i32([96])
    out = torch.zeros(90, H * D, dtype=torch.bfloat16, device="cuda")
    w1, w2 = preft.new_attention_workspace(90, S, H, Hkv, D), preft.new_attention_workspace(90, S, H, Hkv, D, 1)

    def step(to):
        preft.preft_prompt_attention(to, q, k, v, start, prefill, H, Hkv, 0.09, 0, w1)
        preft.preft_cached_attention(to, q, start, prefill, kv, kc, vc, table, gs, gp, H, 0.09, 0, w2)
    step(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for i in range(4):
        kv.copy_(i32([0, 100 + i, 33 + 5 * i, 128 - 3 * i, 0, 7 + i]))
        prefill.copy_(i32([50 - i, 0, 0, 0, 36 - 2 * i, 0]))
        q += 0.01
        want = torch.full_like(out, 2.0)
        out.fill_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        step(want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
