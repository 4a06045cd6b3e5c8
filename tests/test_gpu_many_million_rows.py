"""Calls of more rows than a launch may have threads for along one dimension (64 a row, fewer than 2^32): every row is done."""
import numpy as np
import pytest
import torch

import heads_reference as ref
import paper_2605_14217_amd as preft

pytestmark = pytest.mark.gpu

T, DIM, PAGE, PAGES, POSITIONS = (1 << 26) + 7, 64, 8, 5, 100
# the first and last row, and around every multiple of 2^24
ROWS = sorted({r for b in range(0, T + 1, 1 << 24) for r in (b - 1, b, b + 3) if 0 <= r < T} | {T - 2, T - 1})


@pytest.fixture(autouse=True)
def free_memory():
    yield
    torch.cuda.empty_cache()


def rotation():
    return preft.new_rotation(POSITIONS, 10000.0 ** (-np.arange(0, DIM, 2) / DIM), device="cpu")


def positions():
    at = torch.arange(T, dtype=torch.int32, device="cuda") % POSITIONS
    at[5::1000] = -1
    return at


def slots(gen):
    """Few rows have one: those of ROWS, anywhere in the cache."""
    at = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    at[torch.tensor(ROWS, device="cuda")] = torch.randperm(PAGES * PAGE, generator=gen)[:len(ROWS)].cuda()
    return at


def test_rotate():
    print(f"\n[case] rotate {T} rows", flush=True)
    x, at, table = torch.randn(T, DIM, device="cuda", dtype=torch.bfloat16), positions(), rotation()
    weight, on_card = (1 + 0.3 * torch.randn(DIM)).bfloat16(), table.cuda()
    got = x.clone()
    preft.preft_qk_rotate(None, None, got, got, at, on_card, 0, 1, None, weight.cuda(), 1e-5)
    rows = torch.tensor(ROWS)
    want = ref.turned(x[rows.cuda()].cpu(), 1, weight, 1e-5, at[rows.cuda()].cpu(), table, 0)
    ref.check_rows(got[rows.cuda()], x[rows.cuda()], *want, at[rows.cuda()].cpu() >= 0)
    for a in range(0, T, 10_000_019):                          # and all of them as calls of fewer rows give them
        part, p = x[a:a + 10_000_019].clone(), at[a:a + 10_000_019].clone()
        preft.preft_qk_rotate(None, None, part, part, p, on_card, 0, 1, None, weight.cuda(), 1e-5)
        assert torch.equal(part, got[a:a + 10_000_019])


@pytest.mark.parametrize("mx4", [False, True])
def test_append_and_fetch(mx4):
    print(f"\n[case] append mx4={mx4} {T} rows", flush=True)
    gen = torch.Generator().manual_seed(3)
    k, v = (torch.randn(T, DIM, device="cuda", dtype=torch.bfloat16) for _ in "kv")
    at, table, slot = positions(), rotation().cuda(), slots(gen)
    rows = torch.tensor(ROWS, device="cuda")
    at[rows] = at[rows].abs()                                  # none of them is padding
    shape = (PAGES, 1, PAGE, DIM * 17 // 32) if mx4 else (PAGES, 1, PAGE, DIM)
    caches = [torch.zeros(shape, dtype=torch.uint8 if mx4 else torch.bfloat16, device="cuda") for _ in "kv"]
    few = [torch.zeros_like(c) for c in caches]
    append = preft.preft_kv_append_mx if mx4 else preft.preft_kv_append
    k_out = torch.full_like(k, 7.0)
    append(*caches, None, None, k_out, k, v, slot, at, table, 0)
    some = torch.empty(len(ROWS), DIM, dtype=torch.bfloat16, device="cuda")
    append(*few, None, None, some, k[rows], v[rows], slot[rows], at[rows], table, 0)
    assert all(torch.equal(a, b) and bool(a.any()) for a, b in zip(caches, few)) and torch.equal(k_out[rows], some)
    pad = at < 0
    assert bool((k_out[pad] == 7.0).all()) and not bool((k_out == 7.0).all(1)[~pad].any())
    if mx4:
        back = k.fill_(7.0), v.fill_(7.0)
        preft.preft_kv_fetch_mx(*back, slot, *caches)
        want = [torch.zeros(len(ROWS), DIM, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        preft.preft_kv_fetch_mx(*want, slot[rows], *caches)
        for b, w in zip(back, want):
            assert torch.equal(b[rows], w) and bool(w.any())
            b[rows] = 7.0
            assert bool((b == 7.0).all())


def test_store():
    print(f"\n[case] store {T} rows", flush=True)
    gen = torch.Generator().manual_seed(4)
    k, v = (torch.randn(T, DIM, device="cuda", dtype=torch.bfloat16) for _ in "kv")
    slot, rows = slots(gen), torch.tensor(ROWS, device="cuda")
    caches = [torch.zeros(PAGES, 1, PAGE, DIM, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    preft.preft_kv_store(*caches, k, v, slot)
    for cache, x in zip(caches, (k, v)):
        want = torch.zeros(PAGES * PAGE, DIM, dtype=torch.bfloat16, device="cuda")
        want[slot[rows]] = x[rows]
        assert torch.equal(cache.view(-1, DIM), want)
