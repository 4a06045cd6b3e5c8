"""Pages and attention from their definitions, in 64 bits on the CPU, request by request and row by row; and the bounds that the
kernels' results are held to.

Bound of one output o = sum_j w_j v_j (w_j = p_j / sum p), A = sum_j w_j |v_j|:
  scores   q.k is summed in fp32: off by at most (D + 2) 2^-24 sum_d |q_d k_d| scale =: ds (natural exponent), plus the exponent's own
           rounding, 3 * 2^-24 times the largest exponent; a weight is then off by ds relative, and so is the normalisation: 2 ds A;
  weights  exp2 in hardware and the running rescale: below 2^-20 relative each way: 2^-19 A;
  bf16     eight bits of precision: the numbers from 1 to 2 are 2^-7 apart, so rounding to nearest is off by up to 2^-8 relative.  A weight is
           rounded for the product with v: 2^-8 A, and the result once more: 2^-8 |o|;
  sums     n terms in fp32, numerator and denominator: 2 n 2^-24 A (the matrix cores add in blocks, which is less); f32 results: 2^-24 |o|.
The bound is the sum, with 5 % for products of these terms.
"""
import numpy as np
import torch


def plan(seg_start, ctx_len, table, free_pages, page):
    """(slot_map, positions, kv_len, table, counts) by walking over the requests."""
    table = table.copy()
    S, T, max_pages = len(ctx_len), int(seg_start[-1]), table.shape[1]
    slot, at_, kv, taken, missing = np.full(T, -1, np.int64), np.zeros(T, np.int32), np.zeros(S, np.int32), 0, 0
    for s in range(S):
        n, ctx = int(seg_start[s + 1] - seg_start[s]), max(0, int(ctx_len[s]))
        kv[s] = ctx + n
        for k in range(-(-ctx // page), -(-(ctx + n) // page)):
            if k >= max_pages:
                missing += 1
                continue
            if taken < len(free_pages):
                table[s, k] = free_pages[taken]
            else:
                table[s, k] = -1
                missing += 1
            taken += 1
        for i in range(n):
            at = ctx + i
            at_[seg_start[s] + i] = at
            if at // page < max_pages and table[s, at // page] >= 0:
                slot[seg_start[s] + i] = int(table[s, at // page]) * page + at % page
    return slot, at_, kv, table, np.array([min(taken, len(free_pages)), missing], np.int32)


def attend_row(q, k, v, scale, dtype):
    """q [H, D], k and v [Hkv, n, D] (64-bit): (o, bound), each [H, D]; zeros where n is 0."""
    H, D = q.shape
    G, n = H // k.shape[0], k.shape[1]
    if n == 0:
        return torch.zeros_like(q), torch.full_like(q, 1e-30)
    kk, vv = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
    s = torch.einsum("hd,hnd->hn", q, kk) * scale
    w = torch.softmax(s, 1)
    o = torch.einsum("hn,hnd->hd", w, vv)
    A = torch.einsum("hn,hnd->hd", w, vv.abs())
    ds = (D + 2) * 2.0 ** -24 * (torch.einsum("hd,hnd->hn", q.abs(), kk.abs()) * scale).amax(1, keepdim=True)
    ds = ds + 3 * 2.0 ** -24 * s.abs().amax(1, keepdim=True)
    eps = 2 * ds + 2.0 ** -19 + 2 * n * 2.0 ** -24 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    bound = 1.05 * (eps * A + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * o.abs())
    return o, bound + 1e-30


def prompt(q, k, v, seg_start, prefill, H, Hkv, scale):
    """{row: (o, bound)} of the prompt rows; q, k, v CPU tensors [T, heads * D]."""
    D, out = q.shape[1] // H, {}
    for s in range(len(prefill)):
        lo = int(seg_start[s])
        for i in range(min(int(prefill[s]), int(seg_start[s + 1]) - lo)):
            kk = k[lo:lo + i + 1].double().reshape(-1, Hkv, D).transpose(0, 1)
            vv = v[lo:lo + i + 1].double().reshape(-1, Hkv, D).transpose(0, 1)
            out[lo + i] = attend_row(q[lo + i].double().reshape(H, D), kk, vv, scale, q.dtype)
    return out


def cached(q, seg_start, prefill, kv_len, k_cache, v_cache, table, H, scale):
    """{row: (o, bound)} of the other rows; CPU tensors."""
    page, out = k_cache.shape[2], {}
    D = k_cache.shape[3]
    for s in range(len(kv_len)):
        lo = int(seg_start[s]) + (0 if prefill is None else min(int(prefill[s]), int(seg_start[s + 1] - seg_start[s])))
        r, kv = int(seg_start[s + 1]) - lo, max(0, int(kv_len[s]))
        pages = torch.as_tensor(table[s, : -(-kv // page)]).long()
        K = k_cache[pages].transpose(0, 1).reshape(k_cache.shape[1], -1, D)
        V = v_cache[pages].transpose(0, 1).reshape(k_cache.shape[1], -1, D)
        for i in range(r):
            n = max(0, kv - (r - 1 - i))
            out[lo + i] = attend_row(q[lo + i].double().reshape(H, D), K[:, :n].double(), V[:, :n].double(), scale, q.dtype)
    return out


def check(got, want, before):
    """got, before: CPU tensors [T, H * D].  Rows of `want` within their bounds, all others bit for bit as before; the largest error over its bound."""
    worst = 0.0
    for t in range(got.shape[0]):
        if t not in want:
            assert torch.equal(got[t].view(torch.uint8), before[t].view(torch.uint8)), f"row {t} is not the call's and was written"
            continue
        o, bound = want[t]
        g = got[t].double().reshape(o.shape)
        assert torch.isfinite(g).all(), f"row {t} is not finite"
        over = ((g - o).abs() / bound).amax().item()
        worst = max(worst, over)
        assert over <= 1.0, f"row {t}: {over:.3f} times the bound"
    return worst
