"""Norms and rotation of heads, appends to pages of activations and of 4-bit numbers, and rows out of these, against the definitions."""
import numpy as np
import pytest
import torch

import heads_reference as ref
import paper_2605_14217_amd as preft

pytestmark = pytest.mark.gpu

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


class Case:
    """Inputs of a call: q, k and v as columns of one buffer, positions with padding among them, slots anywhere and some without."""

    def __init__(self, dtype, heads, kv_heads, dim, T, rot, norm, seed=0, page=16, reach=3000, pad=True, apart=8):
        gen = torch.Generator().manual_seed(seed)
        rng = np.random.Generator(np.random.PCG64(seed))
        self.dtype, self.heads, self.kv_heads, self.dim, self.T, self.page = dtype, heads, kv_heads, dim, T, page
        wq, wk = heads * dim, kv_heads * dim
        self.qkv = torch.randn(T, wq + 2 * wk + apart, generator=gen).to(dtype).cuda()
        self.q, self.k, self.v = self.qkv[:, :wq], self.qkv[:, wq:wq + wk], self.qkv[:, wq + wk:wq + 2 * wk]
        pos = rng.integers(0, reach, size=T)
        pos[rng.random(T) < 0.1] = reach + 5                   # past the table: as its last
        if pad and T > 2:
            pos[-1] = -1
            pos[T // 3] = -7
        self.positions = torch.tensor(pos, dtype=torch.int32)
        self.rotation = preft.new_rotation(reach, 10000.0 ** (-np.arange(0, rot, 2) / rot), device="cpu") if rot else None
        self.weights = [(1 + 0.3 * torch.randn(dim, generator=gen)).to(dtype) if norm else None for _ in "qk"]
        self.n_pages = -(-2 * T // page) + 2
        slot = rng.permutation(self.n_pages * page)[:T].astype(np.int64)
        slot[rng.random(T) < 0.15] = -1
        if T > 4:
            slot[2] = self.n_pages * page
        self.slot = torch.from_numpy(slot)
        self.real = self.positions >= 0

    def dev(self):
        d = lambda t: None if t is None else t.cuda()  # noqa: E731
        return dict(positions=d(self.positions), rotation=d(self.rotation), q_weight=d(self.weights[0]), k_weight=d(self.weights[1]), eps=1e-5)

    def want(self, x, heads, weight, pairs):
        return ref.turned(x.cpu(), heads, weight, 1e-5, self.positions, self.rotation, pairs)


SHAPES = [("bf16", 32, 8, 128), ("bf16", 14, 2, 64), ("f32", 8, 8, 64), ("f32", 5, 3, 128), ("bf16", 1, 1, 128), ("bf16", 64, 9, 128), ("bf16", 17, 16, 64), ("f32", 16, 1, 64)]


@pytest.mark.parametrize("pairs", [0, 1])
@pytest.mark.parametrize("rot,norm", [("dim", True), ("dim", False), (16, True), (48, False), (0, True)])
@pytest.mark.parametrize("dtype,heads,kv_heads,dim", SHAPES)
def test_rotate(dtype, heads, kv_heads, dim, rot, norm, pairs):
    rot = dim if rot == "dim" else rot
    for T in (1, 37):
        print(f"\n[case] rotate {dtype} {heads}/{kv_heads}x{dim} T={T} rot={rot} norm={norm} pairs={pairs}", flush=True)
        c = Case(DTYPE[dtype], heads, kv_heads, dim, T, rot, norm, seed=T)
        q_out, k_out = torch.full_like(c.q, 7.0), torch.full((T, kv_heads * dim + 16), 7.0, dtype=c.dtype, device="cuda")[:, 8:8 + kv_heads * dim]
        before = q_out.clone(), k_out.clone()
        preft.preft_qk_rotate(q_out, c.q, k_out, c.k, n_heads=heads, n_kv_heads=kv_heads, pairs=pairs, **c.dev())
        for out, b, x, n, w in ((q_out, before[0], c.q, heads, c.weights[0]), (k_out, before[1], c.k, kv_heads, c.weights[1])):
            ref.check_rows(out, b, *c.want(x, n, w, pairs), c.real)
        # in place, one without the other
        whole = c.qkv.clone()
        kw = c.dev()
        preft.preft_qk_rotate(c.q, c.q, None, None, n_heads=heads, n_kv_heads=0, pairs=pairs, **kw)
        assert torch.equal(c.q[c.real.cuda()], q_out[c.real.cuda()]) and torch.equal(c.qkv[:, heads * dim:], whole[:, heads * dim:])
        preft.preft_qk_rotate(None, None, c.k, c.k, n_heads=3, n_kv_heads=kv_heads, pairs=pairs, **kw)
        assert torch.equal(c.k[c.real.cuda()], k_out[c.real.cuda()])
        assert torch.equal(c.qkv[~c.real.cuda()], whole[~c.real.cuda()]) and torch.equal(c.v, whole[:, (heads + kv_heads) * dim:(heads + 2 * kv_heads) * dim])


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("pairs,rot,norm", [(0, "dim", True), (0, "dim", False), (1, "dim", True), (0, 48, True), (1, 16, False), (0, 0, False)])
@pytest.mark.parametrize("dtype,heads,kv_heads,dim", SHAPES)
def test_append(dtype, heads, kv_heads, dim, pairs, rot, norm, mx4):
    rot = dim if rot == "dim" else rot
    for T, page in ((1, 8), (37, 16), (5, 1024)):
        print(f"\n[case] append mx4={mx4} {dtype} {heads}/{kv_heads}x{dim} T={T} page={page} rot={rot} norm={norm} pairs={pairs}", flush=True)
        c = Case(DTYPE[dtype], heads, kv_heads, dim, T, rot, norm, seed=T, page=page)
        kw = dict(c.dev(), pairs=pairs, n_heads=heads, slot_map=c.slot.cuda())
        want_k, bound_k = c.want(c.k, kv_heads, c.weights[1], pairs)
        keeps = c.real & (c.slot >= 0) & (c.slot < c.n_pages * page)
        # the rows as preft_qk_rotate gives them
        rows = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0)
        preft.preft_qk_rotate(rows[0], c.q, rows[1], c.k, kw["positions"], kw["rotation"], heads, kv_heads, kw["q_weight"], kw["k_weight"], 1e-5, pairs)
        if mx4:
            caches = [torch.randint(0, 256, (c.n_pages, kv_heads, page, dim * 17 // 32), dtype=torch.uint8, device="cuda") for _ in "kv"]
        else:
            caches = [torch.randn(c.n_pages, kv_heads, page, dim, device="cuda").to(c.dtype) for _ in "kv"]
        old = [x.clone().cpu() for x in caches]
        for keep in (True, False):
            for x, o in zip(caches, old):
                x.copy_(o)
            q_out, k_out = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0) if keep else None
            (preft.preft_kv_append_mx if mx4 else preft.preft_kv_append)(*caches, q_out, c.q, k_out, c.k, c.v, **kw)
            assert torch.equal(q_out, rows[0]) and (k_out is None or torch.equal(k_out, rows[1]))
            at, off = (c.slot // page)[keeps], (c.slot % page)[keeps]
            for x, o, new in zip(caches, old, (rows[1], c.v)):
                new = new.cpu()[keeps].reshape(-1, kv_heads, dim)
                if mx4:
                    codes, powers = ref.split(o.numpy(), dim)
                    codes, powers = codes.copy(), powers.copy()
                    codes[at, :, off], powers[at, :, off] = ref.to_four(new.double().numpy())
                    np.testing.assert_array_equal(x.cpu().numpy(), ref.join(codes, powers))
                else:
                    w = o.clone()
                    w[at, :, off] = new
                    assert torch.equal(x.cpu().view(torch.uint8), w.view(torch.uint8))
            ref.check_rows(rows[1], torch.full_like(c.k, 7.0), want_k, bound_k, c.real)
        # keys only, and in place
        for x, o in zip(caches, old):
            x.copy_(o)
        stored = [x.clone() for x in caches]
        (preft.preft_kv_append_mx if mx4 else preft.preft_kv_append)(*stored, None, None, None, c.k, c.v, **kw)
        (preft.preft_kv_append_mx if mx4 else preft.preft_kv_append)(*caches, c.q, c.q, c.k, c.k, c.v, **kw)
        for x, y in zip(caches, stored):
            assert torch.equal(x, y)
        assert torch.equal(c.q[c.real.cuda()], rows[0][c.real.cuda()]) and torch.equal(c.k[c.real.cuda()], rows[1][c.real.cuda()])
        if mx4:                                               # and back
            k_back, v_back = (torch.full((T, kv_heads * dim + 8), 7.0, dtype=c.dtype, device="cuda")[:, 8:] for _ in "kv")
            preft.preft_kv_fetch_mx(k_back, v_back, kw["slot_map"], *caches)
            inside = (c.slot >= 0) & (c.slot < c.n_pages * page)
            for back, x in zip((k_back, v_back), caches):
                want = np.full((T, kv_heads, dim), 7.0)
                v = ref.values(x.cpu().numpy(), dim)
                want[inside.numpy()] = v[(c.slot // page)[inside], :, (c.slot % page)[inside]]
                with np.errstate(over="ignore"):                      # pages of random bytes hold powers that appends do not make
                    want = torch.from_numpy(want).float().to(c.dtype).double().numpy()
                np.testing.assert_array_equal(back.cpu().double().numpy(), want.reshape(T, -1))


@pytest.mark.parametrize("dtype,heads,kv_heads,dim,rot", [("bf16", 4, 2, 128, 112), ("bf16", 3, 1, 128, 80), ("f32", 3, 2, 128, 112), ("f32", 2, 2, 64, 48), ("bf16", 1024, 1024, 64, 32)])
def test_other_shares_that_turn_and_the_most_heads(dtype, heads, kv_heads, dim, rot):
    """Shares of a head that are no power of two, whose last lanes turn nothing; and as many heads as there may be."""
    for pairs in (0, 1):
        c = Case(DTYPE[dtype], heads, kv_heads, dim, 19, rot, True, seed=rot)
        q_out, k_out = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0)
        preft.preft_qk_rotate(q_out, c.q, k_out, c.k, n_heads=heads, n_kv_heads=kv_heads, pairs=pairs, **c.dev())
        for out, x, n, w in ((q_out, c.q, heads, c.weights[0]), (k_out, c.k, kv_heads, c.weights[1])):
            ref.check_rows(out, torch.full_like(out, 7.0), *c.want(x, n, w, pairs), c.real)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_rows_with_one_slot(dtype, mx4):
    """Every 16 bytes of pages of activations, every number and every power of 4-bit pages, are one row's or the other's; nothing else is touched."""
    heads, dim, page, T = 3, 64, 8, 40
    c = Case(DTYPE[dtype], 2, heads, dim, T, 0, False, seed=5, pad=False)
    slot = torch.arange(T) // 2 * 3                            # rows 2 i and 2 i + 1 to slot 3 i
    n_pages = 3 * T // 2 // page + 1
    append = preft.preft_kv_append_mx if mx4 else preft.preft_kv_append
    results = []
    for rows in (slice(0, T), slice(0, T, 2), slice(1, T, 2)):
        caches = [torch.full((n_pages, heads, page, dim * 17 // 32), 0x5a, dtype=torch.uint8, device="cuda") if mx4 else
                  torch.full((n_pages, heads, page, dim), 9.0, dtype=c.dtype, device="cuda") for _ in "kv"]
        append(*caches, None, None, None, c.k[rows], c.v[rows], slot[rows].contiguous().cuda(), None, None, 0)
        results.append([x.cpu() for x in caches])
    for both, first, second in zip(*results):
        if mx4:
            parts = [ref.split(x.numpy(), dim) for x in (both, first, second)]
            for x, a, b in zip(*parts):
                assert ((x == a) | (x == b)).all()
        else:
            x, a, b = (t.reshape(-1).view(torch.int32).reshape(-1, 4) for t in (both, first, second))
            assert bool(((x == a).all(1) | (x == b).all(1)).all())


@pytest.mark.parametrize("T", [1000, 4500])
def test_many_rows(T):
    """A row's heads are one wavefront's or several's, by the rows."""
    print(f"\n[case] many rows T={T}", flush=True)
    c = Case(torch.bfloat16, 9, 2, 128, T, 128, True, seed=T)
    kw = dict(c.dev(), pairs=0, n_heads=9, slot_map=c.slot.cuda())
    caches = [preft.new_mx_cache(c.n_pages, 2, c.page, 128) for _ in "kv"]
    q_out, k_out = torch.zeros_like(c.q), torch.zeros_like(c.k)
    preft.preft_kv_append_mx(*caches, q_out, c.q, k_out, c.k, c.v, **kw)
    ref.check_rows(q_out, torch.zeros_like(c.q), *c.want(c.q, 9, c.weights[0], 0), c.real)
    ref.check_rows(k_out, torch.zeros_like(c.k), *c.want(c.k, 2, c.weights[1], 0), c.real)
    inside = c.real & (c.slot >= 0) & (c.slot < c.n_pages * c.page)
    for x, rows in zip(caches, (k_out, c.v)):
        codes, powers = ref.split(x.cpu().numpy(), 128)
        a, b = ref.to_four(rows.cpu()[inside].double().numpy().reshape(-1, 2, 128))
        at, off = (c.slot // c.page)[inside], (c.slot % c.page)[inside]
        np.testing.assert_array_equal(codes[at, :, off], a)
        np.testing.assert_array_equal(powers[at, :, off], b)
        assert codes.astype(np.int64).sum() == a.astype(np.int64).sum()          # and nothing else


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_numbers_on_borders(dtype):
    """Every border between two numbers and its neighbours, at powers from the least to the largest; zeros, subnormal numbers, infinities and NaN."""
    print(f"\n[case] borders {dtype}", flush=True)
    td = DTYPE[dtype]
    tops = np.array([0.0, 0.5, 1, 3.49, 3.5, 4, 6, 6.98, 6.99, 7, 7.01, 7.9, 8, 13.9, 14])
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    rows = []
    for e in (-149, -133, -128, -127, -126, -125, -124, -60, -1, 0, 1, 77, 123, 124, 125):
        for top in tops:
            x = np.concatenate([borders, -borders, np.nextafter(borders, 0), np.nextafter(borders, 9), [0.0, -0.0]]) * 2.0 ** e
            x = np.clip(x, -top * 2.0 ** e, top * 2.0 ** e)
            x = np.concatenate([x, [top * 2.0 ** e, -top * 2.0 ** e]])
            rows.append(x)
    big = torch.finfo(td).max
    for odd in ([big], [-big, 1.0], [np.inf], [-np.inf, 2.0], [np.nan], [big / 1.75, 3.0], [0.0]):
        rows.append(np.array(odd + [1.0] * (32 - len(odd))))
    rows = [np.concatenate([r, np.zeros(32 - len(r))]) for r in rows]
    while len(rows) % 4:
        rows.append(np.zeros(32))
    with np.errstate(over="ignore"):
        x = torch.from_numpy(np.stack(rows).reshape(-1, 128)).float().to(td)
    T = x.shape[0]
    caches = [preft.new_mx_cache(T // 8 + 1, 1, 8, 128) for _ in "kv"]
    slot = torch.arange(T, device="cuda")
    preft.preft_kv_append_mx(*caches, None, None, None, x.cuda(), x.cuda().flip(0).contiguous(), slot, None, None, 0)
    for cache, rows in zip(caches, (x, x.flip(0))):
        a, b = ref.to_four(rows.double().numpy()[:, None])
        codes, powers = ref.split(cache.cpu().numpy(), 128)
        np.testing.assert_array_equal(powers.transpose(0, 2, 1, 3).reshape(-1, 4)[:T], b.reshape(T, 4))
        finite = np.repeat(b.reshape(T, 4) != 255, 32, 1)
        np.testing.assert_array_equal(codes.transpose(0, 2, 1, 3).reshape(-1, 128)[:T][finite], a.reshape(T, 128)[finite])
    back = [torch.zeros(T, 128, dtype=td, device="cuda") for _ in "kv"]
    preft.preft_kv_fetch_mx(*back, slot, *caches)
    v = ref.from_four(*ref.to_four(x.double().numpy()))
    np.testing.assert_array_equal(back[0].cpu().double().numpy(), v)
    assert np.isfinite(v).sum() > 0.95 * v.size and np.isnan(v).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_how_far_a_number_is_off(dtype):
    """At most a fifth of itself or a quarter of its power; from 7 * 2^125 on, where no power puts the largest of the 32 below 7, what is above 6 * 2^125 becomes that: up to a quarter of itself."""
    print(f"\n[case] how far {dtype}", flush=True)
    td = DTYPE[dtype]
    top, gen = 2.0 ** 125, torch.Generator().manual_seed(1)
    x = torch.randn(64, 128, generator=gen).double() * torch.logspace(-120, 120, 64, 2.0, dtype=torch.float64)[:, None]
    edge = torch.tensor([top, 6 * top, 6.5 * top, 6.9375 * top, 7 * top, 7.5 * top, torch.finfo(td).max], dtype=torch.float64)
    x = torch.cat([x, edge[:, None] * (2 * torch.rand(7, 128, generator=gen).double() - 1)])
    x[64:, ::32] = edge[:, None]
    x = x.to(td)
    T = x.shape[0]
    caches = [preft.new_mx_cache(T // 8 + 1, 1, 8, 128) for _ in "kv"]
    slot = torch.arange(T, device="cuda")
    preft.preft_kv_append_mx(*caches, None, None, None, x.cuda(), x.cuda(), slot, None, None, 0)
    back = [torch.zeros(T, 128, dtype=td, device="cuda") for _ in "kv"]
    preft.preft_kv_fetch_mx(*back, slot, *caches)
    x = x.double().view(T, 4, 32)
    powers = torch.from_numpy(ref.split(caches[0].cpu().numpy(), 128)[1].transpose(0, 2, 1, 3).reshape(-1, 4)[:T].astype(np.float64)) - 127
    unit, most = 2.0 ** powers[..., None], x.abs().amax(-1, keepdim=True)
    assert bool((powers <= 125).all()) and bool(((most < 7 * unit) | (most >= 7 * top)).all()) and bool((most >= 7 * top).any())
    for b in back:
        off = (b.cpu().double().view(T, 4, 32) - x).abs()
        usual = (off <= x.abs() / 5) | (off <= unit / 4)
        cut = (most >= 7 * top) & (x.abs() > 6 * top)
        assert bool((usual | (cut & (off == x.abs() - 6 * top) & (off < x.abs() / 4 * (1 + 2.0 ** -20)))).all())
        assert bool(usual.all(2)[:64].all()) and not bool(usual[-1].all())


@pytest.mark.parametrize("what", [float("inf"), float("nan")])
def test_what_is_not_finite_stays_in_its_head(what):
    print(f"\n[case] not finite {what}", flush=True)
    c = Case(torch.bfloat16, 4, 2, 128, 6, 64, True, pad=False)
    c.q[1, 128 + 5] = what                                    # of the turned elements
    c.q[2, 256 + 100] = what                                  # of the others
    c.k[3, 7] = -what
    for pairs in (0, 1):
        for norm in (True, False):
            if not norm:
                c.weights = [None, None]
            q_out, k_out = torch.zeros_like(c.q), torch.zeros_like(c.k)
            preft.preft_qk_rotate(q_out, c.q, k_out, c.k, n_heads=4, n_kv_heads=2, pairs=pairs, **c.dev())
            for out, x, n, w in ((q_out, c.q, 4, c.weights[0]), (k_out, c.k, 2, c.weights[1])):
                ref.check_rows(out, torch.zeros_like(out), *c.want(x, n, w, pairs), c.real)
            assert torch.isfinite(q_out.view(6, 4, 128)[:, [0, 3]]).all() and torch.isfinite(k_out[[0, 1, 2, 4, 5]]).all()
        c = Case(torch.bfloat16, 4, 2, 128, 6, 64, True, pad=False)
        c.q[1, 128 + 5] = what
        c.k[3, 7] = -what


def test_zero_heads():
    """A head of zeros: zeros under a norm with eps, NaN (0 / 0) without."""
    x = torch.zeros(3, 128, device="cuda")
    w = torch.ones(128, device="cuda")
    out = torch.ones_like(x)
    preft.preft_qk_rotate(out, x, None, None, None, None, 1, 0, w, None, 1e-6)
    assert not out.any()
    preft.preft_qk_rotate(out, x, None, None, None, None, 1, 0, w, None, 0.0)
    assert torch.isnan(out).all()


def test_nothing_to_do_is_no_error():
    z = torch.zeros(0, 256, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    table = preft.new_rotation(4, [1.0] * 8)
    preft.preft_qk_rotate(z, z, None, None, none, table, 2, 0)
    caches = [preft.new_mx_cache(2, 2, 16, 128) for _ in "kv"]
    preft.preft_kv_append_mx(*caches, None, None, None, z, z, none.long(), none, table, 0)
    preft.preft_kv_fetch_mx(z, z, none.long(), *caches)
    some = torch.randn(3, 256, device="cuda")
    empty = [preft.new_mx_cache(0, 2, 16, 128) for _ in "kv"]              # no page: nothing is stored, rows are written
    out = torch.zeros_like(some)
    preft.preft_kv_append_mx(*empty, None, None, out, some, some, torch.zeros(3, dtype=torch.int64, device="cuda"), None, None, 0)
    assert torch.equal(out, some)
    back = out.clone()
    preft.preft_kv_fetch_mx(out, back, torch.zeros(3, dtype=torch.int64, device="cuda"), *empty)
    assert torch.equal(out, some) and torch.equal(back, some)


def test_pages_past_32_bits():
    """Slots whose byte offset in a cache of 4-bit numbers does not fit 32 bits, signed or unsigned."""
    print("\n[case] 4-bit pages past 4 GiB", flush=True)
    heads, dim, page = 8, 128, 64
    per_page = heads * page * 68
    n_pages = (5 << 30) // per_page
    caches = [torch.zeros(n_pages, heads, page, 68, device="cuda", dtype=torch.uint8) for _ in "kv"]
    k, v = (torch.randn(6, heads * dim, device="cuda").bfloat16() for _ in "kv")
    pages = [0, n_pages // 2, (2 << 30) // per_page, (4 << 30) // per_page, n_pages - 1, n_pages - 1]
    slot = torch.tensor([p * page + o for p, o in zip(pages, (0, 3, 0, 0, 62, 63))], device="cuda")
    preft.preft_kv_append_mx(*caches, None, None, None, k, v, slot, None, None, 0)
    back = [torch.zeros_like(k) for _ in "kv"]
    preft.preft_kv_fetch_mx(*back, slot, *caches)
    for b, x, cache in zip(back, (k, v), caches):
        np.testing.assert_array_equal(b.cpu().double().numpy(), ref.from_four(*ref.to_four(x.cpu().double().numpy().reshape(6, heads, dim))).reshape(6, -1))
        for i, p in enumerate(pages):
            page_bytes = cache[p].cpu().numpy()[None]
            codes, powers = ref.split(page_bytes, dim)
            assert (powers[0, :, slot[i].item() % page] != 0).all()
        mine = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
        mine[torch.tensor(pages, device="cuda")] = True
        assert not any(cache[i:i + 4096][~mine[i:i + 4096]].any().item() for i in range(0, n_pages, 4096))


def test_on_another_stream_and_in_a_graph():
    print("\n[case] stream and graph", flush=True)
    c = Case(torch.bfloat16, 8, 2, 64, 40, 64, True)
    caches = [preft.new_mx_cache(c.n_pages, 2, c.page, 64) for _ in "kv"]
    q_out, back = torch.zeros_like(c.q), [torch.zeros_like(c.k), torch.zeros_like(c.v)]
    kw = dict(c.dev(), n_heads=8, slot_map=c.slot.cuda())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    preft.preft_kv_append_mx(*caches, q_out, c.q, None, c.k, c.v, stream=side, **kw)
    with torch.cuda.stream(side):
        preft.preft_kv_fetch_mx(*back, kw["slot_map"], *caches)
    side.synchronize()
    first = q_out.clone(), back[0].clone(), back[1].clone()
    assert all(x.any() for x in first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        preft.preft_kv_append_mx(*caches, q_out, c.q, None, c.k, c.v, **kw)
        preft.preft_kv_fetch_mx(*back, kw["slot_map"], *caches)
    for turn in range(3):
        c.qkv.mul_(2.0)                                       # a power of two: values double, and so do the pages'
        for x in (q_out, *back, *caches):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(back[1], first[2] * 2.0 ** (turn + 1))
        fresh = [torch.zeros_like(x) for x in (q_out, *back)]
        other = [torch.zeros_like(x) for x in caches]
        preft.preft_kv_append_mx(*other, fresh[0], c.q, None, c.k, c.v, **kw)
        preft.preft_kv_fetch_mx(*fresh[1:], kw["slot_map"], *other)
        assert all(torch.equal(x, y) for x, y in zip((q_out, *back, *caches), (*fresh, *other)))
