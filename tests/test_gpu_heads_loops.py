"""Batches of so many rows that a wavefront goes over several shares of a row's heads: every type, head size and pairing, as rows, into pages of activations and into pages of 4-bit numbers."""
import numpy as np
import pytest
import torch

import heads_reference as ref
import paper_2605_14217_amd as preft
from test_gpu_heads import DTYPE, Case

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS = 21, 5                                    # shares of 4, 8 or 16 heads, the last of them not full


@pytest.mark.parametrize("T", [1500, 4300])                # two wavefronts a row, and one
@pytest.mark.parametrize("pages", ["none", "activations", "4-bit"])
@pytest.mark.parametrize("pairs", [0, 1])
@pytest.mark.parametrize("dim,rot", [(128, 96), (64, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_several_shares(dtype, dim, rot, pairs, pages, T):
    print(f"\n[case] shares {dtype} {dim} rot={rot} pairs={pairs} {pages} T={T}", flush=True)
    c = Case(DTYPE[dtype], HEADS, KV_HEADS, dim, T, rot, True, seed=T + dim)
    q_out, k_out = torch.full_like(c.q, 7.0), torch.full_like(c.k, 7.0)
    before = q_out.clone(), k_out.clone()
    four = pages == "4-bit"
    if pages == "none":
        preft.preft_qk_rotate(q_out, c.q, k_out, c.k, n_heads=HEADS, n_kv_heads=KV_HEADS, pairs=pairs, **c.dev())
    else:
        caches = [preft.new_mx_cache(c.n_pages, KV_HEADS, c.page, dim) if four else torch.zeros(c.n_pages, KV_HEADS, c.page, dim, dtype=c.dtype, device="cuda") for _ in "kv"]
        append = preft.preft_kv_append_mx if four else preft.preft_kv_append
        append(*caches, q_out, c.q, k_out, c.k, c.v, slot_map=c.slot.cuda(), n_heads=HEADS, pairs=pairs, **c.dev())
    for out, b, x, n, w in ((q_out, before[0], c.q, HEADS, c.weights[0]), (k_out, before[1], c.k, KV_HEADS, c.weights[1])):
        ref.check_rows(out, b, *c.want(x, n, w, pairs), c.real)
    if pages == "none":
        return
    keeps = c.real & (c.slot >= 0) & (c.slot < c.n_pages * c.page)
    at, off = (c.slot // c.page)[keeps], (c.slot % c.page)[keeps]
    for cache, rows in zip(caches, (k_out, c.v)):
        new = rows.cpu()[keeps].reshape(-1, KV_HEADS, dim)
        if four:
            codes, powers = (np.zeros_like(x) for x in ref.split(cache.cpu().numpy(), dim))
            codes[at, :, off], powers[at, :, off] = ref.to_four(new.double().numpy())
            np.testing.assert_array_equal(cache.cpu().numpy(), ref.join(codes, powers))
        else:
            want = torch.zeros(cache.shape, dtype=c.dtype)
            want[at, :, off] = new
            assert torch.equal(cache.cpu(), want)
    # keys without queries or rows of their own: the same pages
    other = [torch.zeros_like(x) for x in caches]
    append(*other, None, None, None, c.k, c.v, slot_map=c.slot.cuda(), n_heads=0, pairs=pairs, **c.dev())
    assert all(torch.equal(a, b) for a, b in zip(caches, other))
