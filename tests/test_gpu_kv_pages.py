"""Block tables, slot maps and page stores against the definitions, through the C ABI."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2605_14217_amd as preft

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def run_plan(n, ctx, page, max_pages, n_free, pad=0, seed=0):
    rng = np.random.Generator(np.random.PCG64(seed))
    n, ctx = np.asarray(n, np.int64), np.asarray(ctx, np.int64)
    S, start = len(n), np.concatenate([[0], np.cumsum(n)])
    table = rng.integers(0, 10 ** 6, size=(S, max_pages + pad)).astype(np.int32)       # entries that the call must not touch, too
    free = rng.permutation(10 ** 6)[:n_free].astype(np.int32)
    T = int(start[-1])
    dev = i32(table)
    out = dict(slot_map=torch.full((T,), -7, dtype=torch.int64, device="cuda"), positions=torch.full((T,), -7, dtype=torch.int32, device="cuda"),
               kv_len=torch.full((S,), -7, dtype=torch.int32, device="cuda"), block_table=dev[:, :max_pages],
               counts=torch.full((2,), -7, dtype=torch.int32, device="cuda"))
    want = ref.plan(start, ctx, table[:, :max_pages], free, page)
    for _ in range(2):                                      # nothing is consumed: the second call writes the same
        preft.preft_kv_plan(seg_start=i32(start), ctx_len=i32(ctx), free_pages=i32(free), page_size=page, **out)
        for key, w in zip(("slot_map", "positions", "kv_len", "block_table", "counts"), want):
            np.testing.assert_array_equal(out[key].cpu().numpy(), w, err_msg=key)
    np.testing.assert_array_equal(dev[:, max_pages:].cpu().numpy(), table[:, max_pages:])
    return want


@pytest.mark.parametrize("page", [8, 16, 64, 1024])
def test_plan_of_ragged_requests(page):
    print(f"\n[case] plan page={page}", flush=True)
    n = [1, 0, 17, 1, 1, 300, 8, 0, 0, 1, 64, 1025, 2]
    ctx = [0, 5, 0, 7, 8, 9, 1023, 0, 16, 2047, 1, 15, 4096]
    run_plan(n, ctx, page, max_pages=-(-5000 // page), n_free=400, pad=3)


@pytest.mark.parametrize("n,ctx", [([1], [0]), ([1], [16]), ([0, 0, 1], [3, 0, 15]), ([2500], [13]), ([1] * 70, list(range(70))), ([0, 5, 0], [7, 8, 9])])
def test_plan_of_small_and_single_requests(n, ctx):
    print(f"\n[case] plan n={n[:4]}", flush=True)
    run_plan(n, ctx, 16, max_pages=200, n_free=300)


def test_plan_without_new_rows():
    run_plan([0, 0], [5, 0], 16, max_pages=4, n_free=3)


@pytest.mark.parametrize("n_free,max_pages", [(0, 50), (5, 50), (400, 2), (3, 1), (0, 0)])
def test_plan_that_runs_out_of_pages(n_free, max_pages):
    print(f"\n[case] plan n_free={n_free} max_pages={max_pages}", flush=True)
    want = run_plan([40, 1, 33, 1, 100], [0, 16, 5, 31, 20], 16, max_pages=max_pages, n_free=n_free)
    assert want[4][1] > 0


@pytest.mark.parametrize("S,most", [(3000, 3), (1500, 120), (1024, 1), (1025, 2)])
def test_plan_of_more_requests_than_a_workgroup_has_threads(S, most):
    print(f"\n[case] plan S={S}", flush=True)
    rng = np.random.Generator(np.random.PCG64(S))
    n = rng.integers(0, most + 1, size=S)
    run_plan(n, rng.integers(0, 200, size=S), 32, max_pages=12, n_free=int(S * (most / 32 + 1)))


@pytest.mark.parametrize("dtype,heads,dim,page", [("bf16", 8, 128, 16), ("bf16", 2, 64, 64), ("f32", 1, 128, 8), ("f32", 3, 64, 128), ("bf16", 16, 128, 1024)])
@pytest.mark.parametrize("T", [1, 5, 131])
def test_store(dtype, heads, dim, page, T):
    print(f"\n[case] store {dtype} heads={heads} dim={dim} page={page} T={T}", flush=True)
    rng = np.random.Generator(np.random.PCG64(T))
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    n_pages, width = max(3, -(-2 * T // page)), heads * dim
    qkv = torch.randn(T, 5 * width, device="cuda").to(td)          # keys and values are columns of a wider buffer
    qkv[T // 2, 2 * width] = float("nan")                          # values are copied as they are
    k, v = qkv[:, width:2 * width], qkv[:, 2 * width:3 * width]
    slot = rng.permutation(n_pages * page)[:T].astype(np.int64)
    slot[rng.random(T) < 0.2] = -1
    if T > 4:
        slot[2] = n_pages * page                                   # just past the cache
    caches = [torch.randn(n_pages, heads, page, dim, device="cuda").to(td) for _ in "kv"]
    want = [c.clone().cpu() for c in caches]
    for w, x in zip(want, (k.cpu(), v.cpu())):
        for t in range(T):
            if 0 <= slot[t] < n_pages * page:
                w[slot[t] // page, :, slot[t] % page] = x[t].reshape(heads, dim)
    preft.preft_kv_store(*caches, k, v, torch.from_numpy(slot).cuda())
    for c, w in zip(caches, want):
        assert torch.equal(c.cpu().view(torch.uint8), w.view(torch.uint8))


def test_store_past_32_bits():
    """Slots whose byte offset in the cache does not fit 32 bits, signed or unsigned."""
    print("\n[case] store past 4 GiB", flush=True)
    heads, dim, page = 8, 128, 64
    n_pages = (5 << 30) // (heads * dim * page * 2)
    caches = [torch.zeros(n_pages, heads, page, dim, device="cuda", dtype=torch.bfloat16) for _ in "kv"]
    k, v = (torch.randn(6, heads * dim, device="cuda").bfloat16() for _ in "kv")
    pages = [0, n_pages // 2, (2 << 30) // (heads * dim * page * 2), (4 << 30) // (heads * dim * page * 2), n_pages - 1, n_pages - 1]
    slot = torch.tensor([p * page + o for p, o in zip(pages, (0, 3, 0, 0, 62, 63))], device="cuda")
    preft.preft_kv_store(*caches, k, v, slot)
    for c, x in zip(caches, (k, v)):
        assert torch.equal(c[slot // page, :, slot % page], x.view(6, heads, dim))
        c[slot // page, :, slot % page] = 0
        assert not c.any()


def test_plan_and_store_on_another_stream():
    print("\n[case] another stream", flush=True)
    side = torch.cuda.Stream()
    heads, dim, page = 2, 64, 16
    k, v = (torch.randn(40, heads * dim, device="cuda") for _ in "kv")
    caches = [torch.zeros(9, heads, page, dim, device="cuda") for _ in "kv"]
    slot, pos = torch.empty(40, dtype=torch.int64, device="cuda"), torch.empty(40, dtype=torch.int32, device="cuda")
    kv, counts, table = i32([0, 0]), i32([0, 0]), torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    args = (i32([0, 33, 40]), i32([0, 0]), i32([5, 2, 8, 1]))
    side.wait_stream(torch.cuda.current_stream())
    preft.preft_kv_plan(slot, pos, kv, table, counts, *args, page, stream=side)
    with torch.cuda.stream(side):                                  # the current stream is taken where none is named
        preft.preft_kv_store(*caches, k, v, slot)
    side.synchronize()
    assert counts.tolist() == [4, 0] and table[0].tolist() == [5, 2, 8, -1] and table[1].tolist() == [1, -1, -1, -1]
    for c, x in zip(caches, (k, v)):
        assert torch.equal(c[slot // page, :, slot % page], x.view(40, heads, dim))
