"""Attention over pages of 4-bit numbers against the definitions in 64 bits: within bounds that follow from the arithmetic, other rows untouched, and what a row does not see
kept from it.

The bounds are those of attention_reference, whose bf16 part holds as it stands (values of 4-bit pages are bf16 numbers).  In fp32, queries and weights are three numbers each,
so that a score has 3 D products to sum and a result 3 n beside the n weights: (3 D + 2) 2^-24 and 4 n 2^-24 stand where (D + 2) and 2 n did.
"""
import math

import numpy as np
import pytest
import torch

import attention_reference as base
import heads_reference as ref
import paper_2605_14217_amd as preft

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HEADS = [("bf16", 8, 2, 128), ("bf16", 7, 1, 64), ("f32", 6, 3, 64), ("f32", 4, 1, 128), ("bf16", 3, 3, 128), ("bf16", 40, 1, 64), ("f32", 48, 1, 128)]


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def starts(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int64)


def attend_row(q, k, v, scale, dtype):
    o, bound = base.attend_row(q, k, v, scale, dtype)
    if dtype == torch.float32 and k.shape[1]:
        H, D = q.shape
        G, n = H // k.shape[0], k.shape[1]
        kk, vv = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
        w = torch.softmax(torch.matmul(kk, q[:, :, None])[..., 0] * scale, 1)
        A = torch.matmul(w[:, None], vv.abs())[:, 0]
        products = (torch.matmul(kk.abs(), q.abs()[:, :, None])[..., 0] * scale).amax(1, keepdim=True)
        bound = bound + 1.05 * (2 * 2 * D * 2.0 ** -24 * products + 2 * n * 2.0 ** -24) * A
    return o, bound


def cached(q, start, prefill, kv_len, K, V, table, H, scale, rows=None):
    """{row: (o, bound)}; K, V: values [pages, heads, page, D] in 64 bits."""
    page, D, out = K.shape[2], K.shape[3], {}
    for s in range(len(kv_len)):
        lo = int(start[s]) + (0 if prefill is None else min(int(prefill[s]), int(start[s + 1] - start[s])))
        r, kv = int(start[s + 1]) - lo, max(0, int(kv_len[s]))
        pages = torch.as_tensor(np.asarray(table[s, : -(-kv // page)])).long()
        k, v = (c[pages].transpose(0, 1).reshape(c.shape[1], -1, D) for c in (K, V))
        for i in range(r):
            if rows is not None and lo + i not in rows:
                continue
            n = max(0, kv - (r - 1 - i))
            out[lo + i] = attend_row(q[lo + i].double().reshape(H, D), k[:, :n], v[:, :n], scale, q.dtype)
    return out


def random_pages(rng, n, heads, page, dim, powers=(124, 129)):
    """(bytes, values): numbers and powers of all kinds."""
    codes = rng.integers(0, 16, size=(n, heads, page, dim)).astype(np.uint8)
    p = rng.integers(*powers, size=(n, heads, page, dim // 32)).astype(np.uint8)
    return ref.join(codes, p), ref.from_four(codes, p)


class Case:
    """groups: [(first, past the last)] segments; prefix: their shared tokens.  What no row may see is NaN."""

    def __init__(self, dtype, H, Hkv, D, page, rows, kv, prefill=None, groups=None, prefix=None, seed=0, sharp=1.0, pad=8):
        rng = np.random.Generator(np.random.PCG64(seed))
        kv = np.asarray(kv, np.int64)
        n = np.asarray(rows, np.int64) + (0 if prefill is None else np.asarray(prefill, np.int64))
        self.start, S, td = starts(n), len(n), DT[dtype]
        self.H, self.Hkv, self.D, self.page, self.kv, self.prefill, self.S = H, Hkv, D, page, kv, prefill, S
        T, need = int(self.start[-1]), -(-np.maximum(kv, 0) // page)
        self.T = T
        max_pages = int(max(need.max(), max(-(-p // page) for p in prefix) if prefix else 0)) + 2
        shared = {s: g for g, (a, b) in enumerate(groups or []) for s in range(a, b)}
        n_pages = int(need.sum()) + sum(-(-p // page) for p in (prefix or [])) + 3
        ids, used, table = rng.permutation(n_pages), 0, np.full((S, max_pages), n_pages + 1000, np.int64)
        table[:, -1] = -5
        group_pages = []
        for p in prefix or []:
            group_pages.append(ids[used:used + -(-p // page)])
            used += -(-p // page)
        nan = 255
        codes = [rng.integers(0, 16, size=(n_pages, Hkv, page, D)).astype(np.uint8) for _ in "kv"]
        powers = [np.full((n_pages, Hkv, page, D // 32), nan, np.uint8) for _ in "kv"]

        def fill(pages, tokens):
            for i, p in enumerate(pages):
                m = min(page, tokens - i * page)
                for x in powers:
                    x[p, :, :m] = rng.integers(124, 129, size=(Hkv, m, D // 32))
        for g, p in enumerate(prefix or []):
            fill(group_pages[g], p)
        for s in range(S):
            own_from = 0
            if s in shared:
                p = prefix[shared[s]]
                own_from = p // page                           # whole pages are shared, a page that the prefix ends in is a copy
                table[s, : -(-p // page)] = group_pages[shared[s]]
            count = max(0, int(need[s]) - own_from)
            pages = ids[used:used + count]
            used += count
            table[s, own_from:own_from + count] = pages
            fill(pages, int(max(kv[s], 0)) - own_from * page)
            if s in shared and prefix[shared[s]] % page and count:
                m = prefix[shared[s]] % page
                for x in (*codes, *powers):
                    x[pages[0], :, :m] = x[group_pages[shared[s]][-1], :, :m]
        assert used <= n_pages
        self.codes, self.powers, self.table, self.n_pages = codes, powers, table, n_pages
        gen = torch.Generator().manual_seed(seed)
        self.q = (sharp * torch.randn(T, H * D + pad, generator=gen)).to(td).cuda()[:, : H * D]
        self.scale = 1.0 / math.sqrt(D)
        self.gs = self.gp = None
        self.n_groups = len(prefix or [])
        if self.n_groups:
            self.gs, self.gp = i32([a for a, _ in groups] + [groups[-1][1]]), i32(prefix)
        self.ws = preft.new_attention_workspace(T, S, H, Hkv, D, self.n_groups)
        self.dev_table = i32(table)
        self.pad = pad
        self.upload()

    def upload(self):
        self.caches = [torch.from_numpy(ref.join(c, p)).cuda() for c, p in zip(self.codes, self.powers)]
        with np.errstate(invalid="ignore"):
            self.values = [torch.from_numpy(ref.from_four(c, p)) for c, p in zip(self.codes, self.powers)]

    def args(self):
        return (self.q, i32(self.start), None if self.prefill is None else i32(self.prefill), i32(self.kv), *self.caches, self.dev_table, self.gs, self.gp, self.H, self.scale)

    def run(self, mode=0, fill=7.5, ws=None, **kw):
        buf = torch.full((self.T + 4, self.H * self.D + self.pad), fill, dtype=self.q.dtype, device="cuda")
        out = buf[2:2 + self.T, :self.H * self.D]
        preft.preft_cached_attention_mx(out, *self.args(), mode, self.ws if ws is None else ws, **kw)
        torch.cuda.synchronize()
        assert bool((buf[:2] == fill).all()) and bool((buf[2 + self.T:] == fill).all()) and bool((buf[:, self.H * self.D:] == fill).all()), "written beside the output"
        return out.cpu()

    def want(self, rows=None):
        return cached(self.q.cpu(), self.start, self.prefill, self.kv, *self.values, self.table, self.H, self.scale, rows)

    def check(self, rows=None):
        got = self.run()
        before = torch.full_like(got, 7.5)
        want = self.want(rows)
        if rows is not None:
            got, before = got[sorted(rows)], before[sorted(rows)]
            want = {i: want[r] for i, r in enumerate(sorted(rows))}
        print(f"  {base.check(got, want, before):.3f} of the bound", flush=True)
        return got


@pytest.mark.parametrize("page", [8, 16, 64, 1024])
@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
def test_decode_rows_of_every_length(dtype, H, Hkv, D, page):
    """No key at all, one, lengths around tiles and pages; prompts between the decode rows; everything that is not a token is NaN."""
    print(f"\n[case] 4-bit decode {dtype} {H}/{Hkv}x{D} page={page}", flush=True)
    kv = [0, 1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 700]
    prefill = [0] * len(kv)
    prefill[3], prefill[8] = 5, 40
    c = Case(dtype, H, Hkv, D, page, [1] * len(kv), kv, prefill)
    got = c.check()
    assert not got[0].any()                                    # a request without tokens


@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
def test_several_rows_of_a_request(dtype, H, Hkv, D, page):
    """Tokens proposed ahead, chunks of prompts, and rows whose own keys are not there: the first of them see fewer tokens, or none."""
    print(f"\n[case] 4-bit rows {dtype} {H}/{Hkv}x{D}", flush=True)
    Case(dtype, H, Hkv, D, page, [1, 5, 0, 8, 3, 70, 150, 4, 6], [40, 77, 33, 8, 2, 70, 400, 0, 300]).check()


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
@pytest.mark.parametrize("sharp", [0.01, 8.0])
def test_flat_and_sharp_weights(dtype, H, Hkv, D, sharp):
    print(f"\n[case] 4-bit sharp {sharp} {dtype} {H}/{Hkv}x{D}", flush=True)
    Case(dtype, H, Hkv, D, 16, [1, 40], [900, 500], sharp=sharp, seed=3).check()


@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
def test_one_long_request(dtype, H, Hkv, D):
    """A row, and a chunk, whose keys are divided among many workgroups."""
    print(f"\n[case] 4-bit long {dtype} {H}/{Hkv}x{D}", flush=True)
    c = Case(dtype, H, Hkv, D, 64, [1, 1], [9001, 17], sharp=2.0)
    c.check()
    assert preft.preft_schedule_counts(c.ws)[1] > 0
    c = Case(dtype, H, Hkv, D, 16, [130], [5003], sharp=2.0)
    c.check(rows={0, 1, 63, 64, 65, 128, 129})


@pytest.mark.parametrize("dtype,kv", [("bf16", 3000), ("f32", 1500)])
def test_tiles_cut_into_one_round_of_workgroups(dtype, kv):
    """30 tiles of 40 columns for each of 8 heads, which take two parts each, and a join that is shared by several workgroups a tile."""
    print(f"\n[case] 4-bit one round {dtype}", flush=True)
    c = Case(dtype, 32, 8, 64, 64, [10] * 30, [kv + 3 * s for s in range(30)], seed=9)
    c.check(rows={0, 4, 9, 10, 144, 150, 155, 290, 299})
    assert preft.preft_schedule_counts(c.ws)[1] == 30


@pytest.mark.parametrize("most,page,prefix", [(64, 16, 64), (96, 8, 75), (192, 16, 100), (1500, 64, 1100), (700, 16, 256)])
@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
def test_groups(dtype, H, Hkv, D, most, page, prefix):
    """Shared prefixes at the end of a page and inside one, members that end before it, a second group, prompt rows in between, and requests in no group."""
    print(f"\n[case] 4-bit groups {dtype} {H}/{Hkv}x{D} most={most} page={page} prefix={prefix}", flush=True)
    Case(dtype, H, Hkv, D, page, [1, 2, 1, 1, 1, 3, 1], [most, most, prefix, prefix - 3, most - 1, most, 20], prefill=[0, 0, 5, 0, 0, 0, 0], groups=[(0, 4), (4, 6)],
         prefix=[prefix, 64]).check()


@pytest.mark.parametrize("S,rows", [(300, 1), (270, 3), (40, 33)])
@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS[:4])
def test_many_requests(dtype, H, Hkv, D, S, rows):
    """Units that are one wavefront's, and more segments than workgroups search through."""
    print(f"\n[case] 4-bit many {dtype} {H}/{Hkv}x{D} S={S} rows={rows}", flush=True)
    rng = np.random.Generator(np.random.PCG64(S))
    kv = rng.integers(0, 500, size=S)
    c = Case(dtype, H, Hkv, D, 16, [rows] * S, kv, seed=S)
    c.check(rows=set(int(t) for t in rng.integers(0, S * rows, size=60)) | {0, S * rows - 1})


@pytest.mark.parametrize("rows,kv", [(1, 300), (5, 300), (90, 300), (90, 3000)])
@pytest.mark.parametrize("dtype,H,Hkv,D", HEADS)
def test_nan_reaches_the_rows_that_see_it(dtype, H, Hkv, D, rows, kv):
    """A NaN block of V: 32 elements of every row that sees the key; of K: all of the row's heads of it.  Rows before the key are as ever."""
    print(f"\n[case] 4-bit NaN {dtype} {H}/{Hkv}x{D} rows={rows} kv={kv}", flush=True)
    c = Case(dtype, H, Hkv, D, 16, [rows, 1], [kv, 40], seed=1)
    clean = c.run()
    at = [(kv - 1, 0), (kv - 1 - rows // 2, 1), (kv - 1 - rows // 3, D // 32 - 1), (10, 0) if rows == 5 else (kv - 2, 1)]
    seen = torch.zeros(c.T, H, D, dtype=torch.bool)
    for key, block in at:
        page, off = c.table[0, key // 16], key % 16
        head = key % Hkv
        c.powers[1][page, head, off, block] = 255
        for t in range(rows):
            if key < kv - (rows - 1 - t):
                seen[t, head * (H // Hkv):(head + 1) * (H // Hkv), 32 * block:32 * block + 32] = True
    c.upload()
    got = c.run().view(c.T, H, D)
    assert got[seen].isnan().all() and torch.equal(got[~seen], clean.view(c.T, H, D)[~seen])
    key = kv - 1 - rows // 2                                   # and a key
    c.powers[1][:] = np.where(c.powers[1] == 255, 126, c.powers[1])
    c.powers[0][c.table[0, key // 16], 0, key % 16, 0] = 255
    c.upload()
    got = c.run().view(c.T, H, D)
    G = H // Hkv
    for t in range(rows):
        assert bool(got[t, :G].isnan().all()) == (key < kv - (rows - 1 - t)) and torch.isfinite(got[t, G:]).all() and (t >= rows - 1 - rows // 2 or torch.isfinite(got[t]).all())


def test_powers_from_the_least_to_the_largest():
    """Values of 2^-126 to 1.5 * 2^127 beside each other: one key dominates, or all are alike."""
    print("\n[case] 4-bit powers", flush=True)
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 4, 2, 64, 16, [1, 1], [50, 33], seed=2)
        p = c.powers[1]
        rng = np.random.Generator(np.random.PCG64(0))
        p[:] = np.where(p == 255, 255, rng.choice([2, 60, 127, 190, 245], size=p.shape))
        c.upload()
        got, want = c.run(), c.want()
        base.check(got, {t: (o, b + 2.0 ** -126) for t, (o, b) in want.items()}, torch.full_like(got, 7.5))


def test_infinite_and_nan_queries():
    print("\n[case] 4-bit infinite queries", flush=True)
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 4, 2, 128, 16, [1, 1, 1], [50, 33, 0], seed=2)
        clean = c.run().view(3, 4, 128)
        c.q[0, 5], c.q[1, 128 + 7], c.q[2, 3] = float("nan"), float("inf"), float("nan")
        got = c.run().view(3, 4, 128)
        assert got[0, 0].isnan().all() and got[1, 1].isnan().all() and not got[2].any()
        for t, h in ((0, 0), (1, 1)):
            keep = [x for x in range(4) if x != h]
            assert torch.equal(got[t, keep], clean[t, keep])


def test_ready_schedules_and_the_other_pages():
    """A second layer takes the schedule, on another stream too; a call on pages of activations does not, and the other way round."""
    print("\n[case] 4-bit ready schedule", flush=True)
    c = Case("bf16", 8, 2, 128, 16, [1] * 300, [100] * 300, seed=4)
    first = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(c.run(mode=preft.PREFT_SCHEDULE_READY, stream=side), first)
    plain = [torch.zeros(c.n_pages, 2, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    out = torch.full((c.T, 8 * 128), 7.5, dtype=torch.bfloat16, device="cuda")
    a = c.args()
    preft.preft_cached_attention(out, *a[:4], *plain, *a[6:], preft.PREFT_SCHEDULE_READY, c.ws)
    assert bool((out == 7.5).all())
    with pytest.raises(preft.PreftError) as e:
        preft.preft_schedule_counts(c.ws)
    assert e.value.code == preft.PREFT_ESCHEDULE
    preft.preft_cached_attention(out, *a[:4], *plain, *a[6:], 0, c.ws)
    assert not out.any()
    assert bool((c.run(mode=preft.PREFT_SCHEDULE_READY) == 7.5).all())
    assert torch.equal(c.run(), first)


@pytest.mark.parametrize("S", [6, 300])
def test_replayed_steps(S):
    """A step's appends and attention in a graph, replayed with other contents of the same tables between eager work: the bits of the eager calls."""
    print(f"\n[case] 4-bit graph S={S}", flush=True)
    H, Hkv, D, page = 8, 2, 128, 16
    rng = np.random.Generator(np.random.PCG64(S))
    gen = torch.Generator(device="cuda").manual_seed(S)
    pages = 8
    caches = [torch.from_numpy(random_pages(rng, S * pages, Hkv, page, D)[0]).cuda() for _ in "kv"]
    table = i32(rng.permutation(S * pages).reshape(S, pages))
    qkv = torch.randn(S, (H + 2 * Hkv) * D, generator=gen, device="cuda").bfloat16()
    q, k, v = qkv[:, :H * D], qkv[:, H * D:(H + Hkv) * D], qkv[:, (H + Hkv) * D:]
    seg, ctx = i32(np.arange(S + 1)), i32(rng.integers(0, pages * page, size=S))
    slot, pos, kv, counts = torch.empty(S, dtype=torch.int64, device="cuda"), i32(np.zeros(S)), i32(np.zeros(S)), i32([0, 0])
    free = i32([0])
    rotation = preft.new_rotation(pages * page, 10000.0 ** (-np.arange(0, D, 2) / D))
    q_out, out = torch.zeros_like(q), torch.zeros_like(q)
    ws = preft.new_attention_workspace(S, S, H, Hkv, D)

    def step(caches, q_out, out, ws):
        preft.preft_kv_plan(slot, pos, kv, table, counts, seg, ctx, free, page)
        preft.preft_kv_append_mx(*caches, q_out, q, None, k, v, slot, pos, rotation, H)
        preft.preft_cached_attention_mx(out, q_out, seg, None, kv, *caches, table, None, None, H, 0.09, 0, ws)
    step(caches, q_out, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches, q_out, out, ws)
    for turn in range(4):
        ctx.copy_(i32(np.maximum(rng.integers(0, pages * page, size=S) // page * page + 1 + turn, 0)))
        qkv += 0.1
        twin = [x.clone() for x in caches]
        other = torch.zeros_like(q), torch.full_like(q, 3.0)
        step(twin, *other, preft.new_attention_workspace(S, S, H, Hkv, D))
        q_out.zero_()
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, other[0]) and torch.equal(out, other[1]) and all(torch.equal(x, y) for x, y in zip(caches, twin))
        assert torch.isfinite(out).all() and bool(out.any(1).all())


@pytest.mark.parametrize("seed", range(40))
def test_random_calls(seed):
    rng = np.random.Generator(np.random.PCG64(1000 + seed))
    dtype, H, Hkv, D = HEADS[rng.integers(len(HEADS))]
    page = int(rng.choice([8, 16, 32, 64, 256]))
    S = int(rng.choice([1, 2, 5, 12, 40]))
    rows = rng.choice([0, 1, 1, 1, 2, 7, 30, 100], size=S)
    kv = rng.choice([0, 1, 30, 64, 200, 800, 2500], size=S) + rng.integers(0, 40, size=S) * rng.integers(0, 2)
    prefill = rng.choice([0, 0, 3, 20], size=S) if rng.random() < 0.4 else None
    if rows.sum() == 0:
        rows[0] = 1
    groups = prefix = None
    if S >= 5 and rng.random() < 0.5:
        cut = sorted(rng.choice(np.arange(S + 1), size=3, replace=False))
        groups, prefix = [(cut[0], cut[1]), (cut[1], cut[2])], [int(rng.integers(1, 300)) for _ in range(2)]
        for g, (a, b) in enumerate(groups):
            kv[a:b] = prefix[g] + rng.integers(0, 100, size=b - a)
    print(f"\n[case] 4-bit random seed={seed} {dtype} {H}/{Hkv}x{D} page={page} rows={rows.tolist()} kv={kv.tolist()} groups={groups} {prefix}", flush=True)
    c = Case(dtype, H, Hkv, D, page, rows, kv, prefill, groups, prefix, seed=seed)
    mine = sorted(c.want(rows=set()) or [])                    # every row of the call, or forty of them
    every = [t for s in range(S) for t in range(int(c.start[s]) + (0 if prefill is None else int(prefill[s])), int(c.start[s + 1]))]
    some = set(every) if len(every) <= 40 else set(int(t) for t in rng.choice(every, size=40, replace=False))
    got = c.run()
    want = c.want(some)
    order = sorted(some)
    base.check(got[order], {i: want[t] for i, t in enumerate(order)}, torch.full((len(order), H * D), 7.5, dtype=got.dtype))
    others = [t for t in range(c.T) if t not in set(every)]
    assert not mine and bool((got[others] == 7.5).all())
    assert torch.equal(got, c.run())                           # the same bits


def test_pages_past_32_bits():
    """Pages whose byte offset in the cache does not fit 32 bits."""
    print("\n[case] 4-bit attention past 4 GiB", flush=True)
    H, Hkv, D, page = 8, 8, 128, 64
    per_page = Hkv * page * 68
    n_pages = (9 << 29) // per_page
    caches = [torch.zeros(n_pages, Hkv, page, 68, dtype=torch.uint8, device="cuda") for _ in "kv"]
    ids = [n_pages - 1, (2 << 30) // per_page + 1, 0, (4 << 30) // per_page + 1, n_pages - 7]
    rng = np.random.Generator(np.random.PCG64(0))
    values = []
    for c in caches:
        b, v = random_pages(rng, len(ids), Hkv, page, D)
        c[torch.tensor(ids, device="cuda")] = torch.from_numpy(b).cuda()
        values.append(torch.from_numpy(v))
    for rows in (1, 40):
        kv = len(ids) * page - 5
        q = torch.randn(rows, H * D, generator=torch.Generator().manual_seed(1)).bfloat16()
        out = torch.zeros_like(q).cuda()
        preft.preft_cached_attention_mx(out, q.cuda(), i32([0, rows]), None, i32([kv]), *caches, i32([ids]), None, None, H, 0.09, 0,
                                        preft.new_attention_workspace(rows, 1, H, Hkv, D))
        want = cached(q, [0, rows], None, [kv], *values, np.arange(len(ids))[None], H, 0.09)
        base.check(out.cpu(), want, torch.zeros_like(q))


@pytest.mark.parametrize("rows", [1, 70])
def test_no_pages_at_all(rows):
    """A pool or a table without pages: every row sees no key and is zero; tables and caches may be empty."""
    print(f"\n[case] 4-bit no pages rows={rows}", flush=True)
    H, Hkv, D = 4, 2, 64
    q = torch.randn(rows, H * D, device="cuda").bfloat16()
    ws = preft.new_attention_workspace(rows, 1, H, Hkv, D)
    for n_pages, columns, page in ((0, 4, 16), (3, 0, 64), (0, 0, 32), (0, 3, 64)):
        caches = [preft.new_mx_cache(n_pages, Hkv, page, D) for _ in "kv"]
        table = torch.zeros(1, columns, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 7.5)
        preft.preft_cached_attention_mx(out, q, i32([0, rows]), None, i32([50]), *caches, table, None, None, H, 0.1, 0, ws)
        assert not out.any()
