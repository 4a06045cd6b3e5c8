"""Attention of so many short requests that their units are more workgroups than one launch may have (2^24 of 256 threads): every row has its result."""
import math

import numpy as np
import pytest
import torch

import attention_reference as base
import heads_reference as ref
import paper_2605_14217_amd as preft

pytestmark = pytest.mark.gpu

H, D, PAGE, PAGES = 16, 64, 16, 40


@pytest.fixture(autouse=True)
def free_memory():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("mx4", [False, True])
def test_decode_rows(mx4):
    """With keys that may be cut there are up to three units a row and key/value head, 352 000 x 16 x 3 workgroups; all of those that a launch of 2^32 threads fewer would have do less than a fifth of the rows."""
    T, table_pages = 352_000, 40
    print(f"\n[case] {T} decode rows, 4-bit pages {mx4}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(7)
    q = torch.randn(T, H * D, generator=gen, device="cuda", dtype=torch.bfloat16)
    rows = [torch.randn(PAGES * PAGE, H * D, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in "kv"]
    every = torch.arange(PAGES * PAGE, device="cuda")
    if mx4:
        caches = [preft.new_mx_cache(PAGES, H, PAGE, D) for _ in "kv"]
        preft.preft_kv_append_mx(*caches, None, None, None, *rows, every, None, None, 0)
        K, V = (torch.from_numpy(ref.values(c.cpu().numpy(), D)) for c in caches)
        attend = preft.preft_cached_attention_mx
    else:
        caches = [torch.empty(PAGES, H, PAGE, D, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        preft.preft_kv_store(*caches, *rows, every)
        K, V = (c.double().cpu() for c in caches)
        attend = preft.preft_cached_attention
    table = torch.randint(0, PAGES, (T, table_pages), generator=gen, device="cuda", dtype=torch.int32)
    kv_len = torch.randint(1, 60, (T,), generator=gen, device="cuda", dtype=torch.int32)
    start = torch.arange(T + 1, dtype=torch.int32, device="cuda")
    out, scale = torch.full_like(q, math.nan), 1 / math.sqrt(D)
    attend(out, q, start, None, kv_len, *caches, table, None, None, H, scale, 0, preft.new_attention_workspace(T, T, H, H, D))
    assert not bool(torch.isnan(out).any())
    for r in sorted({0, 1, T - 1} | set(range(7, T, T // 24))):
        n = int(kv_len[r])
        pages = table[r].cpu().long()
        k, v = (x[pages].permute(1, 0, 2, 3).reshape(H, -1, D)[:, :n] for x in (K, V))
        o, bound = base.attend_row(q[r].cpu().double().view(H, D), k, v, scale, torch.bfloat16)
        assert bool(((out[r].cpu().double().view(H, D) - o).abs() <= bound).all()), r
    # and all of them beside calls of fewer rows.  Either is a weighted mean of V, off by at most 2^-8 of the largest value for the weights, 2^-8 for itself and 2^-10 for scores and sums
    far = 2 * 1.05 * (2 * 2.0 ** -8 + 2.0 ** -10) * float(V.abs().max())
    ws = preft.new_attention_workspace(50_000, 50_000, H, H, D)
    for a in range(0, T, 50_000):
        b = min(a + 50_000, T)
        part = torch.empty_like(q[a:b])
        attend(part, q[a:b], start[:b - a + 1], None, kv_len[a:b].clone(), *caches, table[a:b], None, None, H, scale, 0, ws)
        assert float((part.float() - out[a:b].float()).abs().max()) <= far


def test_prompts_of_one_row():
    """Every row is its only key: its value, whatever the score."""
    T = 1_045_000
    print(f"\n[case] {T} prompts of one row", flush=True)
    q, k, v = (torch.randn(T, H * D, device="cuda", dtype=torch.bfloat16) for _ in "qkv")
    out = torch.full_like(q, math.nan)
    start, one = torch.arange(T + 1, dtype=torch.int32, device="cuda"), torch.ones(T, dtype=torch.int32, device="cuda")
    preft.preft_prompt_attention(out, q, k, v, start, one, H, H, 0.125, 0, preft.new_attention_workspace(T, T, H, H, D))
    assert torch.equal(out, v)
