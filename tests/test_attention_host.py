"""What the page and attention entry points refuse, before any launch; and the 64-bit reference of their GPU tests against hand-worked values and
against another way to compute the same."""
import ctypes
import math

import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2605_14217_amd as preft

A, B, C, D_, E, W = (0x7f0000000000 + i * 0x100000000 for i in range(6))     # never dereferenced: every call must fail first


@pytest.fixture(scope="module")
def lib():
    return preft.load_library()


def plan(lib, slot=A, pos=B, kv=C, table=D_, ld=10, max_pages=10, counts=E, start=A, ctx=A, S=3, T=5, free=B, n_free=4, page=16):
    return lib.preft_kv_plan(slot, pos, kv, table, ld, max_pages, counts, start, ctx, S, T, free, n_free, page, None)


def test_plan_refusals(lib):
    for bad in (dict(S=-1), dict(T=-1), dict(n_free=-1), dict(max_pages=-1), dict(ld=9), dict(slot=None), dict(pos=None), dict(kv=None),
                dict(table=None), dict(counts=None), dict(start=None), dict(ctx=None), dict(free=None), dict(S=0)):
        assert plan(lib, **bad) == -1, bad
    for page in (0, -16, 1, 4, 12, 48, 2048):
        assert plan(lib, page=page) == -2, page
    assert plan(lib, S=0, T=0) == 0


def store(lib, kc=A, vc=B, n_pages=100, page=16, k=C, ldk=1024, v=D_, ldv=1024, T=7, heads=8, dim=128, slot=E, dtype=1):
    return lib.preft_kv_store(kc, vc, n_pages, page, k, ldk, v, ldv, T, heads, dim, slot, dtype, None)


def test_store_refusals(lib):
    for bad in (dict(T=-1), dict(n_pages=-1), dict(heads=0), dict(heads=1025), dict(dtype=2), dict(slot=None), dict(k=None), dict(v=None),
                dict(kc=None), dict(vc=None), dict(ldk=1016), dict(ldv=(1 << 20) + 8), dict(vc=A), dict(k=A + 64), dict(v=B)):
        assert store(lib, **bad) == -1, bad
    assert store(lib, dim=96) == -2 and store(lib, page=24) == -2
    for bad in (dict(k=C + 8), dict(ldv=1028), dict(kc=A + 4)):
        assert store(lib, **bad) == -3, bad
    assert store(lib, T=0) == 0 and store(lib, n_pages=0) == 0


def prompt(lib, out=A, ldo=1024, q=B, ldq=1024, k=C, ldk=256, v=D_, ldv=256, T=100, H=8, Hkv=2, D=128, start=E, prefill=E, S=4, scale=0.1, dtype=1,
           mode=0, ws=W, wsb=None):
    if wsb is None:
        wsb = preft.preft_attention_workspace_bytes(max(T, 1), max(S, 1), 8, 2, 128)
    return lib.preft_prompt_attention(out, ldo, q, ldq, k, ldk, v, ldv, T, H, Hkv, D, start, prefill, S, scale, dtype, mode, ws, wsb, None)


def test_prompt_refusals(lib):
    for bad in (dict(T=-1), dict(S=-1), dict(H=0), dict(Hkv=0), dict(H=7), dict(dtype=3), dict(mode=1), dict(mode=0x200), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(out=None), dict(q=None), dict(k=None), dict(v=None), dict(start=None),
                dict(prefill=None), dict(ldo=1016), dict(ldk=248), dict(ldq=(1 << 20) + 8), dict(q=A), dict(k=A + 512), dict(v=A), dict(H=2048, Hkv=2)):
        assert prompt(lib, **bad) == -1, bad
    for bad in (dict(D=32), dict(D=96), dict(D=256)):
        assert prompt(lib, **bad) == -2, bad
    for bad in (dict(out=A + 8), dict(ldq=1028), dict(v=D_ + 2)):
        assert prompt(lib, **bad) == -3, bad
    good = preft.preft_attention_workspace_bytes(100, 4, 8, 2, 128)
    assert good > 0 and prompt(lib, ws=None) == -4 and prompt(lib, wsb=good - 1) == -4 and prompt(lib, ws=W + 8) == -4
    assert prompt(lib, T=1 << 28, wsb=1 << 40) == -8
    assert prompt(lib, T=0) == 0 and prompt(lib, S=0) == 0
    # an output beside its inputs in one buffer is no overlap (the call gets as far as the workspace)
    assert prompt(lib, out=B + 2048, ldo=2048, ldq=2048, ws=None) == -4 and prompt(lib, out=B + 2046, ldo=2048, ldq=2048, ws=None) == -3
    assert prompt(lib, out=B + 2032, ldo=2048, ldq=2048, ws=None) == -1


def cached(lib, out=A, ldo=1024, q=B, ldq=1024, T=100, H=8, Hkv=2, D=128, start=E, prefill=None, kv=E, S=4, kc=C, vc=D_, n_pages=50, page=16, table=E,
           ld=20, max_pages=20, gs=None, gp=None, groups=0, scale=0.1, dtype=1, mode=0, ws=W, wsb=1 << 40):
    return lib.preft_cached_attention(out, ldo, q, ldq, T, H, Hkv, D, start, prefill, kv, S, kc, vc, n_pages, page, table, ld, max_pages, gs, gp, groups,
                                      scale, dtype, mode, ws, wsb, None)


def test_cached_refusals(lib):
    for bad in (dict(T=-1), dict(S=-1), dict(groups=-1), dict(H=9), dict(dtype=-1), dict(mode=2), dict(scale=0.0), dict(n_pages=-1), dict(max_pages=-1),
                dict(ld=19), dict(start=None), dict(kv=None), dict(groups=1), dict(groups=1, gs=E), dict(out=None), dict(q=None), dict(kc=None),
                dict(vc=None), dict(table=None), dict(q=A), dict(out=C), dict(vc=A - 64)):
        assert cached(lib, **bad) == -1, bad
    for bad in (dict(D=80), dict(page=0), dict(page=100)):
        assert cached(lib, **bad) == -2, bad
    for bad in (dict(kc=C + 8), dict(q=B + 8), dict(ldo=1025)):
        assert cached(lib, **bad) == -3, bad
    assert cached(lib, ws=None) == -4 and cached(lib, wsb=100) == -4
    with_groups, without = (preft.preft_attention_workspace_bytes(100, 4, 8, 2, 128, g) for g in (2, 0))
    assert with_groups > without and cached(lib, gs=E, gp=E, groups=2, wsb=without) == -4
    assert cached(lib, T=0) == 0 and cached(lib, S=0) == 0


def test_workspace_sizes(lib):
    size = preft.preft_attention_workspace_bytes
    for bad in ((-1, 1, 8, 2, 128, 0), (1, -1, 8, 2, 128, 0), (1, 1, 8, 3, 128, 0), (1, 1, 0, 1, 128, 0), (1, 1, 8, 2, 96, 0), (1, 1, 8, 2, 128, -1),
                (1 << 27, 1, 8, 2, 128, 0)):
        assert size(*bad) == 0, bad
    assert size(0, 0, 1, 1, 64) > 0
    assert size(1, 1, 32, 8, 128) < 8 << 20                    # a single decode row does not ask for much
    with pytest.raises(ValueError):
        preft.new_attention_workspace(1, 1, 8, 3, 128, device="cpu")


def test_binding_refuses_what_is_no_device_tensor():
    t, i = torch.zeros(4, 128), torch.zeros(3, dtype=torch.int32)
    cache, ws = torch.zeros(2, 2, 16, 64), torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="slot_map"):
        preft.preft_kv_plan(i.long(), i, i, i[None], i[:2], i, i[:2], i, 16, stream=0)
    with pytest.raises(ValueError, match="k_cache"):
        preft.preft_kv_store(cache, cache, t, t, i.long(), stream=0)
    with pytest.raises(ValueError, match="out: need a 2-D device tensor"):
        preft.preft_prompt_attention(t, t, t, t, i, i[:2], 2, 2, 0.1, 0, ws, stream=0)
    with pytest.raises(ValueError, match="out: need a 2-D device tensor"):
        preft.preft_cached_attention(t, t, i, None, i[:2], cache, cache, i[None], None, None, 2, 0.1, 0, ws, stream=0)


def test_marshalling_declines_what_is_no_ordinary_call():
    from paper_2605_14217_amd import binding
    preft.load_library()
    native = binding._native
    assert native is not None
    t, i, cache, ws = torch.zeros(4, 128), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 2, 16, 64), torch.zeros(64, dtype=torch.uint8)
    assert native.kv_plan(i.long(), i, i, i[None], i, i, i, i, 16, 0) is None and native.kv_plan() is None
    assert native.kv_store(cache, cache, t, t, i.long(), 0) is None and native.kv_store(None, cache, t, t, i, 0) is None
    assert native.prompt_attention(t, t, t, t, i, i, 2, 2, 0.1, 0, ws, 0) is None and native.prompt_attention(t) is None
    assert native.cached_attention(t, t, i, None, i, cache, cache, i[None], None, None, 2, 0.1, 0, ws, 0) is None
    with pytest.raises(TypeError):
        native.bind_attention(1)


# ---- the reference itself ---------------------------------------------------------------------------------------

def test_reference_plan_by_hand():
    table = np.array([[4, -9, -9], [6, 7, -9], [-9, -9, -9]], np.int32)
    slot, at, kv, table, counts = ref.plan(np.array([0, 3, 4, 13]), np.array([6, 16, 0]), table, np.array([30, 31, 32, 33]), 8)
    assert slot.tolist() == [38, 39, 240, 248] + [256 + i for i in range(8)] + [264]
    assert at.tolist() == [6, 7, 8, 16] + list(range(9)) and kv.tolist() == [9, 17, 9] and counts.tolist() == [4, 0]
    assert table.tolist() == [[4, 30, -9], [6, 7, 31], [32, 33, -9]]


def test_reference_attention_is_torchs_softmax():
    gen = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(6, w, generator=gen) for w in (4 * 8, 2 * 8, 2 * 8))
    got = ref.prompt(q, k, v, [0, 6], [6], 4, 2, 0.3)
    for h in range(4):
        s = (q[:, 8 * h:8 * h + 8].double() @ k[:, 8 * (h // 2):8 * (h // 2) + 8].double().T * 0.3).masked_fill(torch.ones(6, 6).triu(1).bool(), -math.inf)
        o = torch.softmax(s, 1) @ v[:, 8 * (h // 2):8 * (h // 2) + 8].double()
        for t in range(6):
            assert torch.allclose(got[t][0][h], o[t], rtol=1e-12, atol=1e-14)
    # the same through pages
    table = np.array([[2, 0, 1]])
    kc, vc = torch.zeros(3, 2, 2, 8), torch.zeros(3, 2, 2, 8)
    for t in range(6):
        kc[table[0, t // 2], :, t % 2], vc[table[0, t // 2], :, t % 2] = k[t].view(2, 8), v[t].view(2, 8)
    paged = ref.cached(q, [0, 6], None, [6], kc, vc, table, 4, 0.3)
    assert all(torch.allclose(paged[t][0], got[t][0]) for t in range(6))
    bound = got[5][1]
    assert (bound > 0).all() and (bound < 1e-3).all()
