"""Forms of the attention calls in which every row needs a second look: groups over short tables, replayed graphs.  Against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2605_14217_amd as preft
from test_gpu_attention import HEADS, cached_case, i32, normal, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("most,page,prefix", [(64, 16, 64), (96, 8, 75), (128, 64, 128), (192, 16, 100), (256, 64, 200), (272, 16, 256)])
@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
def test_groups_over_short_tables(dtype, H, Hkv, D, most, page, prefix):
    """Block tables of 64 to 272 tokens, where no keys are cut: a group's rows still have their shared keys as a part of their own.  Shared prefixes at the end of a
    page and inside one, members that end before it, a second group, prompt rows in between, and requests in no group."""
    print(f"\n[case] short groups {dtype} {H}/{Hkv}x{D} most={most} page={page} prefix={prefix}", flush=True)
    rows = [1, 2, 1, 1, 1, 3, 1]
    kv = [most, most, prefix, prefix - 3, most - 1, most, 20]
    out, before, want, args, _, (gs, gp, H, scale) = cached_case(dtype, H, Hkv, D, page, rows, kv, prefill=[0, 0, 5, 0, 0, 0, 0], groups=[(0, 4), (4, 6)],
                                                                 prefix=[prefix, 64])
    print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)
    narrow = args[6][:, : -(-most // page)]                    # a table without room for more
    again = torch.full_like(out, -3.0)
    preft.preft_cached_attention(again, *args[:6], narrow, gs, gp, H, scale, 0, preft.new_attention_workspace(out.shape[0], len(rows), H, Hkv, D, 2))
    ref.check(again.cpu(), want, torch.full_like(before, -3.0))


@pytest.mark.parametrize("pages", [6, 40])
def test_replayed_steps_against_the_definitions(pages):
    """A step's two calls in a graph, replayed with other contents of the same tables between eager work; every replay against the definitions, in an output that held something
    else before.  Tables in which nothing is cut, and longer ones."""
    print(f"\n[case] graph and definitions, {pages} pages", flush=True)
    H, Hkv, D, page, S = 8, 2, 128, 16, 6
    gen = torch.Generator(device="cuda").manual_seed(2)
    pool = S * pages
    kc, vc = (normal(gen, pool, Hkv, page, D).bfloat16() for _ in "kv")
    qkv = normal(gen, 90, (H + 2 * Hkv) * D).bfloat16()
    q, k, v = qkv[:, :H * D], qkv[:, H * D:(H + Hkv) * D], qkv[:, (H + Hkv) * D:]
    start, long = [0, 50, 51, 52, 53, 89, 90], pages * page - 20
    table = np.random.Generator(np.random.PCG64(0)).permutation(pool).reshape(S, pages)
    table[2:4, :5] = table[1, :5]                              # the group's shared pages
    dev, gs, gp = i32(table), i32([1, 4]), i32([80])
    prefill, kv = i32([50, 0, 0, 0, 36, 0]), i32([0, long, 33, long, 0, 7])
    seg = i32(start)
    out = torch.zeros(90, H * D, dtype=torch.bfloat16, device="cuda")
    w1, w2 = preft.new_attention_workspace(90, S, H, Hkv, D), preft.new_attention_workspace(90, S, H, Hkv, D, 1)

    def step():
        preft.preft_prompt_attention(out, q, k, v, seg, prefill, H, Hkv, 0.09, 0, w1)
        preft.preft_cached_attention(out, q, seg, prefill, kv, kc, vc, dev, gs, gp, H, 0.09, 0, w2)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        n, kvl = [50 - i, 0, 0, 0, 36 - 2 * i, 0], [0, long - i, 33 + 5 * i, long - 3 * i, 0, 7 + i]
        kv.copy_(i32(kvl))
        prefill.copy_(i32(n))
        q += 0.01
        out.fill_(2.0 + i)
        before = out.cpu()
        graph.replay()
        torch.cuda.synchronize()
        want = ref.cached(q.cpu(), start, n, kvl, kc.cpu(), vc.cpu(), table, H, 0.09)
        want.update(ref.prompt(q.cpu(), k.cpu(), v.cpu(), start, n, H, Hkv, 0.09))
        assert len(want) == 90
        print(f"  replay {i}: {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


def test_a_wide_chunk_over_very_many_tokens():
    """8184 rows of 16 heads over one key/value head and 600 000 tokens: more work than the search for units once summed.  Every row is
    written; rows of several tiles, and at their ends."""
    print("\n[case] 8184 rows over 600 000 tokens", flush=True)
    H, D, page, T, kv = 16, 64, 256, 8184, 600_000
    gen = torch.Generator(device="cuda").manual_seed(4)
    n_pages = -(-kv // page)
    kc, vc = (normal(gen, n_pages, 1, page, D).bfloat16() for _ in "kv")
    q = (2.0 * normal(gen, T, H * D)).bfloat16()
    table = torch.randperm(n_pages, generator=gen, device="cuda").int()[None]
    out = torch.full_like(q, 7.5)
    ws = preft.new_attention_workspace(T, 1, H, 1, D)
    preft.preft_cached_attention(out, q, i32([0, T]), None, i32([kv]), kc, vc, table, None, None, H, 0.125, 0, ws)
    assert not bool((out == 7.5).all(1).any())
    K, V = (c[table[0].long()].reshape(1, -1, D).cpu().double() for c in (kc, vc))
    for t in (0, 7, 8, 15, 2047, 4096, 8175, 8176, 8183):
        o, bound = ref.attend_row(q[t].cpu().double().view(H, D), K[:, : kv - (T - 1 - t)], V[:, : kv - (T - 1 - t)], 0.125, q.dtype)
        assert ((out[t].cpu().double().view(H, D) - o).abs() <= bound).all(), t


@pytest.mark.parametrize("groups", [0, 2])
@pytest.mark.parametrize("S,most", [(3, 320), (5, 4000), (300, 64), (300, 1000)])
def test_segments_that_overlap_leave_the_output_alone(S, most, groups):
    """Offsets that go back, over tables long enough to be cut and joined and over short ones, searched for and listed: nothing is written, and the next call on the workspace is as ever."""
    print(f"\n[case] overlapping segments S={S} most={most} groups={groups}", flush=True)
    H, Hkv, D, page, T = 4, 2, 64, 16, 1000
    gen = torch.Generator(device="cuda").manual_seed(S)
    kc, vc = (normal(gen, 40, Hkv, page, D).bfloat16() for _ in "kv")
    qkv = normal(gen, T, (H + 2 * Hkv) * D).bfloat16()
    q, k, v = qkv[:, :H * D], qkv[:, H * D:(H + Hkv) * D], qkv[:, (H + Hkv) * D:]
    start = [0, T] * (S // 2) + [0, 900][: S + 1 - 2 * (S // 2)]
    assert len(start) == S + 1
    table = torch.randint(0, 40, (S, -(-most // page)), generator=gen, device="cuda", dtype=torch.int32)
    gs, gp = (i32([0, S // 2, S]), i32([64, 64])) if groups else (None, None)
    ws = preft.new_attention_workspace(T, S, H, Hkv, D, groups)
    ws.fill_(0x9d)                                             # no sensible entry of any list
    out = torch.full((T, H * D), 7.5, dtype=torch.bfloat16, device="cuda")
    kv = i32([most] * S)
    preft.preft_cached_attention(out, q, i32(start), None, kv, kc, vc, table, gs, gp, H, 0.1, 0, ws)
    preft.preft_prompt_attention(out, q, k, v, i32(start), i32([T] * S), H, Hkv, 0.1, 0, preft.new_attention_workspace(T, S, H, Hkv, D).fill_(0x9d))
    torch.cuda.synchronize()
    assert bool((out == 7.5).all())
    good = np.linspace(0, T, S + 1).astype(int)
    preft.preft_cached_attention(out, q, i32(good), None, kv, kc, vc, table, gs, gp, H, 0.1, 0, ws)
    assert not bool((out == 7.5).all(1).any())


def mixed_step(S, seed, groups, dtype=torch.bfloat16):
    """Whole prompts and decode rows of one batch, layer after layer with other values: (tables of the step, layers of (q, k, v, caches))."""
    H, Hkv, D, page = 8, 2, 64, 16
    rng, gen = np.random.Generator(np.random.PCG64(seed)), torch.Generator(device="cuda").manual_seed(seed)
    prompt = rng.random(S) < 0.4
    prompt[:4] = False                                         # the group's
    n = np.where(prompt, rng.integers(1, 90, size=S), rng.integers(1, 3, size=S))
    kv = np.where(prompt, n, rng.integers(130, 400, size=S))
    pages = 26
    table = rng.permutation(S * pages).reshape(S, pages)
    table[1:4, :8] = table[0, :8]
    start = np.concatenate([[0], np.cumsum(n)])
    T = int(start[-1])
    layers = [tuple((normal(gen, *shape) * f).to(dtype) for shape, f in (((T, H * D), 2.0), ((T, Hkv * D), 1.0), ((T, Hkv * D), 1.0),
                                                                         ((S * pages, Hkv, page, D), 1.0), ((S * pages, Hkv, page, D), 1.0))) for _ in range(3)]
    return dict(H=H, Hkv=Hkv, D=D, S=S, T=T, start=start, prefill=np.where(prompt, n, 0), kv=kv, table=table, dev=i32(table), seg=i32(start),
                groups=(i32([0, 4]), i32([128])) if groups else (None, None), n_groups=1 if groups else 0), layers


@pytest.mark.parametrize("groups", [False, True])
@pytest.mark.parametrize("S", [9, 300])
def test_both_kinds_of_a_mixed_step_keep_their_schedules_in_one_workspace(S, groups):
    """Every layer makes both calls; the first builds both schedules, the others find them again."""
    print(f"\n[case] mixed step S={S} groups={groups}", flush=True)
    s, layers = mixed_step(S, S, groups)
    ws = preft.new_attention_workspace(s["T"], S, s["H"], s["Hkv"], s["D"], s["n_groups"])
    ws.fill_(0x9d)
    prefill, kv = i32(s["prefill"]), i32(s["kv"])
    for i, (q, k, v, kc, vc) in enumerate(layers):
        ready = preft.PREFT_SCHEDULE_READY if i else 0
        out = torch.full_like(q, 7.5)
        before = out.cpu()
        preft.preft_prompt_attention(out, q, k, v, s["seg"], prefill, s["H"], s["Hkv"], 0.125, ready, ws)
        preft.preft_cached_attention(out, q, s["seg"], prefill, kv, kc, vc, s["dev"], *s["groups"], s["H"], 0.125, ready, ws)
        preft.preft_schedule_counts(ws)                        # raises where a call was refused
        if S > 100 and i != 2:                                 # the last layer alone: 300 requests take the reference a while
            assert not bool((out == 7.5).all(1).any())
            continue
        want = ref.prompt(q.cpu(), k.cpu(), v.cpu(), s["start"], s["prefill"], s["H"], s["Hkv"], 0.125)
        want.update(ref.cached(q.cpu(), s["start"], s["prefill"], s["kv"], kc.cpu(), vc.cpu(), s["table"], s["H"], 0.125))
        assert len(want) == s["T"]
        print(f"  layer {i}: {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


def test_a_refused_call_of_either_kind_is_reported_until_its_next_schedule():
    print("\n[case] refused calls", flush=True)
    s, layers = mixed_step(9, 1, False)
    q, k, v, kc, vc = layers[0]
    T, H, Hkv = s["T"], s["H"], s["Hkv"]
    ws = preft.new_attention_workspace(T, 9, H, Hkv, s["D"])
    ws.fill_(0x9d)
    out, prefill, kv = torch.full_like(q, 7.5), i32(s["prefill"]), i32(s["kv"])

    def prompt(mode, rows=T):
        preft.preft_prompt_attention(out[:rows], q[:rows], k[:rows], v[:rows], s["seg"], prefill, H, Hkv, 0.125, mode, ws)

    def cached(mode, rows=T):
        preft.preft_cached_attention(out[:rows], q[:rows], s["seg"], prefill, kv, kc, vc, s["dev"], None, None, H, 0.125, mode, ws)

    def refused():
        try:
            preft.preft_schedule_counts(ws)
        except preft.PreftError as e:
            assert e.code == preft.PREFT_ESCHEDULE
            return True
        return False
    READY = preft.PREFT_SCHEDULE_READY
    prompt(0)
    assert not refused()
    out.fill_(7.5)
    cached(READY)                                              # no schedule of this kind was ever built
    assert refused() and bool((out == 7.5).all())
    prompt(READY)
    assert refused() and not bool((out == 7.5).all())
    prompt(0)                                                  # the other kind's mark stays
    assert refused()
    cached(0)
    assert not refused()
    out.fill_(7.5)
    prompt(READY, T - 1)
    cached(READY, T - 1)
    assert refused() and bool((out == 7.5).all())
    cached(0)
    assert refused()
    prompt(0)
    assert not refused()


@pytest.mark.parametrize("S,H,Hkv", [(300, 32, 8), (300, 4, 2), (20, 8, 2)])
@pytest.mark.parametrize("first", ["bf16", "f32"])
def test_a_schedule_serves_calls_of_its_type_and_its_tables_room(S, H, Hkv, first):
    """How keys are cut goes by the type and by how long the tables may be: a call with others is refused, not run on lists that do not fit its grid."""
    print(f"\n[case] other type, narrower table, S={S} {H}/{Hkv} {first}", flush=True)
    D, page, gen = 64, 16, torch.Generator(device="cuda").manual_seed(S)
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    other = "f32" if first == "bf16" else "bf16"
    kc, vc = (normal(gen, 500, Hkv, page, D) for _ in "kv")
    q = normal(gen, S, H * D)
    table = torch.randint(0, 500, (S, 12), generator=gen, device="cuda", dtype=torch.int32)
    start, kv = i32(np.arange(S + 1)), i32([192 - s % 90 for s in range(S)])
    ws = preft.new_attention_workspace(S, S, H, Hkv, D)
    ws.fill_(0x9d)

    def run(dtype, mode, pages=12):
        t = types[dtype]
        out = torch.full((S, H * D), 7.5, dtype=t, device="cuda")
        preft.preft_cached_attention(out, q.to(t), start, None, kv, kc.to(t), vc.to(t), table[:, :pages], None, None, H, 0.125, mode, ws)
        return out
    READY = preft.PREFT_SCHEDULE_READY
    built = run(first, 0)
    assert torch.equal(built, run(first, READY)) and not bool((built == 7.5).any(1).all())
    preft.preft_schedule_counts(ws)
    for dtype, pages in ((other, 12), (first, 11), (first, 6)):
        run(first, 0)
        preft.preft_schedule_counts(ws)
        assert bool((run(dtype, READY, pages) == 7.5).all())
        with pytest.raises(preft.PreftError) as e:
            preft.preft_schedule_counts(ws)
        assert e.value.code == preft.PREFT_ESCHEDULE
    assert torch.equal(built, run(first, READY))


def test_workspaces_that_are_no_device_memory_are_refused():
    """On the host, or fewer bytes than they seem: refused before any launch, by either way into the library."""
    print("\n[case] workspaces", flush=True)
    s, layers = mixed_step(9, 1, False)
    q, k, v, kc, vc = layers[0]
    n = preft.preft_attention_workspace_bytes(s["T"], 9, s["H"], s["Hkv"], s["D"])
    out, prefill, kv = torch.full_like(q, 7.5), i32(s["prefill"]), i32(s["kv"])
    for ws in (torch.zeros(n, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8, device="cuda").expand(n), torch.zeros(2 * n, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            preft.preft_prompt_attention(out, q, k, v, s["seg"], prefill, s["H"], s["Hkv"], 0.125, 0, ws)
        with pytest.raises(ValueError, match="workspace"):
            preft.preft_cached_attention(out, q, s["seg"], prefill, kv, kc, vc, s["dev"], None, None, s["H"], 0.125, 0, ws)
    assert bool((out == 7.5).all())


def infinite_scores(k, q, H, Hkv, D, hidden, top=None):
    """Scores of the keys `hidden` become -inf for every row, that of `top` +inf: q's first dimension is 1, theirs infinite."""
    q.view(q.shape[0], H, D)[..., 0] = 1.0
    k[hidden, ..., 0] = -float("inf")
    if top is not None:
        k[top, ..., 0] = float("inf")


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
def test_infinite_scores_in_prompts(dtype, H, Hkv, D):
    """Keys of score -inf weigh nothing, rows that see no others are zero, and rows that see a score of +inf are NaN."""
    print(f"\n[case] infinite scores, prompts {dtype} {H}/{Hkv}x{D}", flush=True)
    td = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    gen = torch.Generator(device="cuda").manual_seed(9)
    for T, none, top in ((200, 10, 150), (40, 33, 39), (2111, 700, None)):          # the last: long enough to be divided
        q, k, v = (normal(gen, T, w * D).to(td) for w in (H, Hkv, Hkv))
        infinite_scores(k.view(T, Hkv, D), q, H, Hkv, D, slice(0, none), top)
        out = torch.full_like(q, 7.5)
        preft.preft_prompt_attention(out, q, k, v, i32([0, T]), i32([T]), H, Hkv, D ** -0.5, 0, preft.new_attention_workspace(T, 1, H, Hkv, D))
        got, qc, kc, vc = out.cpu().double().view(T, H, D), q.cpu().double().view(T, H, D), *(x.cpu().double().view(T, Hkv, D).transpose(0, 1) for x in (k, v))
        assert not got[:none].any()
        if top is not None:
            assert got[top:].isnan().all()
        for t in sorted({none, none + 1, (none + T) // 2, (top or T) - 1} - {none - 1}):
            if top is not None and t >= top:
                continue
            o, bound = ref.attend_row(qc[t], kc[:, none:t + 1], vc[:, none:t + 1], D ** -0.5, td)
            assert ((got[t] - o).abs() <= bound).all(), t


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
def test_infinite_scores_over_pages(dtype, H, Hkv, D):
    """The same for decode rows: requests whose first keys, or all, have the score -inf, short and divided, and groups whose shared keys do."""
    print(f"\n[case] infinite scores, pages {dtype} {H}/{Hkv}x{D}", flush=True)
    page, rows = 16, [1] * 7
    kv, none = [300, 9001, 40, 9001, 260, 200, 128], [100, 5000, 40, 9001, 128, 200, 128]      # the last three share 128 tokens
    out, before, _, args, ws, (gs, gp, H, scale) = cached_case(dtype, H, Hkv, D, page, rows, kv, groups=[(4, 7)], prefix=[128])
    q, start, _, kvl, kc, vc, table = args
    q = q.clone()
    for s in range(7):
        for i in range(-(-none[s] // page)):
            infinite_scores(kc[int(table[s, i])].transpose(0, 1), q, H, Hkv, D, slice(0, min(page, none[s] - i * page)))
    got = torch.full_like(q, 7.5)
    preft.preft_cached_attention(got, q, start, None, kvl, kc, vc, table, gs, gp, H, scale, 0, ws)
    got = got.cpu().double().view(7, H, D)
    for s in range(7):
        if none[s] == kv[s]:
            assert not got[s].any(), s
            continue
        pages = table[s, : -(-kv[s] // page)].long()
        K, V = (c[pages].transpose(0, 1).reshape(Hkv, -1, D)[:, none[s]:kv[s]].cpu().double() for c in (kc, vc))
        o, bound = ref.attend_row(q[s].cpu().double().view(H, D), K, V, scale, q.dtype)
        assert ((got[s] - o).abs() <= bound).all(), s
    # and one score of +inf
    infinite_scores(kc[int(table[0, 7])].transpose(0, 1), q, H, Hkv, D, slice(0, 0), 3)
    infinite_scores(kc[int(table[4, 2])].transpose(0, 1), q, H, Hkv, D, slice(0, 0), 3)
    out = torch.full_like(q, 7.5)
    preft.preft_cached_attention(out, q, start, None, kvl, kc, vc, table, gs, gp, H, scale, 0, ws)
    assert out[[0, 4, 5, 6]].isnan().all() and torch.isfinite(out[1:4]).all()


def test_more_requests_than_the_schedule_keeps_in_lds():
    """4500 requests: the offsets of their tiles stand in memory; with and without groups."""
    print("\n[case] 4500 requests", flush=True)
    rng = np.random.Generator(np.random.PCG64(6))
    S = 4500
    kv = rng.integers(0, 60, size=S)
    kv[::50] = rng.integers(100, 400, size=len(kv[::50]))
    for groups, prefix, more in ((None, None, 0), ([(0, 60), (60, 2000)], [96, 72], 100)):
        out, before, want, *_ = cached_case("bf16", 7, 1, 64, 16, rng.integers(0, 3, size=S) if groups is None else np.ones(S, int), more + kv, groups=groups, prefix=prefix)
        print(f"  {ref.check(out.cpu(), want, before):.3f} of the bound", flush=True)


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
def test_rows_that_see_a_key_of_infinities_are_nan(dtype, H, Hkv, D):
    """A key that is -inf in every dimension: its score adds infinities of both signs, so that rows that see it are NaN, and the others are as by the definition."""
    print(f"\n[case] key of -inf, {dtype} {H}/{Hkv}x{D}", flush=True)
    td = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    gen = torch.Generator(device="cuda").manual_seed(10)
    T, at = 150, 70
    q, k, v = (normal(gen, T, w * D).to(td) for w in (H, Hkv, Hkv))
    kc, vc = (x.view(1, T, Hkv, D)[:, :144].reshape(9, 16, Hkv, D).transpose(1, 2).contiguous() for x in (k, v))
    table = torch.arange(9, device="cuda", dtype=torch.int32)[None]
    want = ref.prompt(q.cpu(), k.cpu(), v.cpu(), [0, at], [at], H, Hkv, D ** -0.5)
    k[at], v[at] = -float("inf"), -float("inf")
    kc[at // 16, :, at % 16], vc[at // 16, :, at % 16] = -float("inf"), -float("inf")
    out, paged = torch.full_like(q, 7.5), torch.full_like(q[:144], 7.5)
    preft.preft_prompt_attention(out, q, k, v, i32([0, T]), i32([T]), H, Hkv, D ** -0.5, 0, preft.new_attention_workspace(T, 1, H, Hkv, D))
    preft.preft_cached_attention(paged, q[:144], i32([0, 144]), None, i32([144]), kc, vc, table, None, None, H, D ** -0.5, 0,
                                 preft.new_attention_workspace(144, 1, H, Hkv, D))
    for got in (out, paged):
        print(f"  {ref.check(got[:at].cpu(), want, got[:at].cpu()):.3f} of the bound", flush=True)
        assert got[at:].isnan().all()


def test_layers_with_heads_of_two_sizes_share_their_schedules():
    """Prompts that are divided and decode rows of one step, in layers of heads of 64, 128 and 64 again, on one workspace for the larger: the first layer builds both schedules."""
    print("\n[case] heads of two sizes", flush=True)
    H, Hkv, page, n, kv = 4, 1, 16, [1600, 1, 2], [1600, 700, 3000]
    start, T, prefill = starts(n), 1603, [1600, 0, 0]
    gen = torch.Generator(device="cuda").manual_seed(21)
    table = np.arange(3 * 188).reshape(3, 188)
    ws = preft.new_attention_workspace(T, 3, H, Hkv, 128)
    ws.fill_(0x9d)
    for i, D in enumerate((64, 128, 64)):
        q, k, v = (normal(gen, T, w * D).bfloat16() for w in (H, Hkv, Hkv))
        kc, vc = (normal(gen, 3 * 188, Hkv, page, D).bfloat16() for _ in "kv")
        out, ready = torch.full_like(q, 7.5), preft.PREFT_SCHEDULE_READY if i else 0
        preft.preft_prompt_attention(out, q, k, v, i32(start), i32(prefill), H, Hkv, D ** -0.5, ready, ws)
        preft.preft_cached_attention(out, q, i32(start), i32(prefill), i32(kv), kc, vc, i32(table), None, None, H, D ** -0.5, ready, ws)
        preft.preft_schedule_counts(ws)                        # raises where a call was refused
        want = ref.cached(q.cpu(), start, prefill, kv, kc.cpu(), vc.cpu(), table, H, D ** -0.5)
        for t in (0, 63, 64, 900, 1599):
            want[t] = ref.attend_row(q[t].cpu().double().view(H, D), *(x[:t + 1].cpu().double().view(t + 1, Hkv, D).transpose(0, 1) for x in (k, v)), D ** -0.5, q.dtype)
        for t, (o, bound) in want.items():
            assert ((out[t].cpu().double().view(H, D) - o).abs() <= bound).all(), (i, t)
        assert not bool((out == 7.5).all(1).any())
