"""What the calls on heads and the pages of 4-bit numbers refuse, before any launch; and the 64-bit reference of their GPU tests against hand-worked values."""
import math

import numpy as np
import pytest
import torch

import heads_reference as ref
import paper_2605_14217_amd as preft

A, B, C, D_, E, F, G, W = (0x7f0000000000 + i * 0x100000000 for i in range(8))     # never dereferenced: every call must fail first


@pytest.fixture(scope="module")
def lib():
    return preft.load_library()


def rotate(lib, qo=A, ldqo=1024, q=B, ldq=2048, ko=C, ldko=256, k=B + 2048, ldk=2048, T=7, H=8, Hkv=2, dim=128, qw=D_, kw=D_, eps=1e-6, pos=E, rot=F, n=100,
           rdim=128, pairs=0, dtype=1):
    return lib.preft_qk_rotate(qo, ldqo, q, ldq, ko, ldko, k, ldk, T, H, Hkv, dim, qw, kw, eps, pos, rot, n, rdim, pairs, dtype, None)


def test_rotate_refusals(lib):
    for bad in (dict(T=-1), dict(H=-1), dict(Hkv=-1), dict(H=1025), dict(Hkv=2000), dict(dtype=2), dict(pairs=2), dict(pairs=-1), dict(eps=-1e-9), dict(eps=math.nan),
                dict(eps=math.inf), dict(rdim=144), dict(rdim=-16), dict(pos=None), dict(rot=None), dict(n=0), dict(qo=None), dict(q=None), dict(ko=None), dict(k=None),
                dict(ldqo=1016), dict(ldq=1000), dict(ldko=248), dict(ldk=(1 << 20) + 8), dict(qo=B + 64), dict(qo=B, ldqo=1024), dict(ko=A), dict(ko=B + 2048 + 256, ldko=2048),
                dict(ko=B + 1024, ldko=2048), dict(qo=B + 1024, ldqo=2048)):
        assert rotate(lib, **bad) == -1, bad
    for bad in (dict(dim=32), dict(dim=256), dict(rdim=8), dict(rdim=40)):
        assert rotate(lib, **bad) == -2, bad
    for bad in (dict(qo=A + 8), dict(ldq=2052), dict(qw=D_ + 2), dict(kw=D_ + 8), dict(rot=F + 4)):
        assert rotate(lib, **bad) == -3, bad
    # the rows' own place, or beside them, is no overlap: the call gets as far as the weights
    for good in (dict(qo=B, ldqo=2048), dict(ko=B + 2048, ldko=2048), dict(qo=B, ldqo=2048, ko=B + 2048, ldko=2048), dict(qo=B + 2560, ldqo=2048, H=2, q=B)):
        assert rotate(lib, qw=D_ + 2, **good) == -3, good
    assert rotate(lib, T=0) == 0 and rotate(lib, H=0, Hkv=0) == 0
    assert rotate(lib, H=0, Hkv=0, qo=None, q=None, ko=None, k=None, pos=None, rot=None, n=0, rdim=0) == 0


def append(lib, mx4=False, kc=A, vc=B, n_pages=100, page=16, qo=C, ldqo=1024, q=D_, ldq=2048, ko=E, ldko=256, k=D_ + 2048, ldk=2048, v=D_ + 2560, ldv=2048, T=7, H=8, Hkv=2,
           dim=128, slot=F, qw=None, kw=None, eps=1e-6, pos=G, rot=W, n=100, rdim=64, pairs=1, dtype=1):
    f = lib.preft_kv_append_mx if mx4 else lib.preft_kv_append
    return f(kc, vc, n_pages, page, qo, ldqo, q, ldq, ko, ldko, k, ldk, v, ldv, T, H, Hkv, dim, slot, qw, kw, eps, pos, rot, n, rdim, pairs, dtype, None)


@pytest.mark.parametrize("mx4", [False, True])
def test_append_refusals(lib, mx4):
    size = 100 * 16 * 2 * (68 if mx4 else 256)                        # bytes of a cache
    for bad in (dict(T=-1), dict(n_pages=-1), dict(H=-1), dict(Hkv=0), dict(dtype=7), dict(pairs=5), dict(eps=-1.0), dict(rdim=256), dict(kc=None), dict(vc=None), dict(q=None),
                dict(qo=None), dict(k=None), dict(v=None), dict(slot=None), dict(pos=None), dict(rot=None), dict(n=-1), dict(ldv=248), dict(ldk=100), dict(ldko=8), dict(vc=A),
                dict(vc=A + size - 16), dict(kc=B - size + 16), dict(qo=A + 1024), dict(q=B), dict(ko=A), dict(k=A), dict(v=B), dict(ko=D_ + 2560, ldko=2048),
                dict(qo=D_ + 1536, ldqo=2048)):
        assert append(lib, mx4, **bad) == -1, bad
    for bad in (dict(dim=96), dict(page=24), dict(page=4), dict(rdim=24)):
        assert append(lib, mx4, **bad) == -2, bad
    for bad in (dict(kc=A + 8), dict(vc=B + 4), dict(k=D_ + 2050), dict(qw=D_ + 6), dict(ldv=2049)):
        assert append(lib, mx4, **bad) == -3, bad
    # caches side by side, new keys in place or not wanted: as far as the cache's alignment
    for good in (dict(kc=B - size + 8), dict(kc=A + 8, ko=None, ldko=0), dict(kc=A + 8, ko=D_ + 2048, ldko=2048), dict(kc=A + 8, H=0, q=None, qo=None)):
        assert append(lib, mx4, **good) == -3, good
    assert append(lib, mx4, T=0) == 0


def fetch(lib, k=A, ldk=256, v=B, ldv=256, T=5, Hkv=2, dim=128, slot=C, kc=D_, vc=E, n_pages=9, page=16, dtype=1):
    return lib.preft_kv_fetch_mx(k, ldk, v, ldv, T, Hkv, dim, slot, kc, vc, n_pages, page, dtype, None)


def test_fetch_refusals(lib):
    for bad in (dict(T=-1), dict(n_pages=-1), dict(Hkv=0), dict(dtype=3), dict(slot=None), dict(k=None), dict(v=None), dict(kc=None), dict(vc=None), dict(ldk=248), dict(v=A),
                dict(k=D_), dict(v=E + 128)):
        assert fetch(lib, **bad) == -1, bad
    assert fetch(lib, dim=80) == -2 and fetch(lib, page=12) == -2
    for bad in (dict(k=A + 2), dict(ldv=260), dict(kc=D_ + 8)):
        assert fetch(lib, **bad) == -3, bad
    assert fetch(lib, T=0) == 0 and fetch(lib, n_pages=0) == 0


def cached(lib, out=A, ldo=1024, q=B, ldq=1024, T=100, H=8, Hkv=2, D=128, start=E, prefill=None, kv=E, S=4, kc=C, vc=D_, n_pages=50, page=16, table=E,
           ld=20, max_pages=20, gs=None, gp=None, groups=0, scale=0.1, dtype=1, mode=0, ws=W, wsb=1 << 40):
    return lib.preft_cached_attention_mx(out, ldo, q, ldq, T, H, Hkv, D, start, prefill, kv, S, kc, vc, n_pages, page, table, ld, max_pages, gs, gp, groups,
                                         scale, dtype, mode, ws, wsb, None)


def test_attention_refusals(lib):
    size = 50 * 16 * 2 * 68
    for bad in (dict(T=-1), dict(S=-1), dict(groups=-1), dict(H=9), dict(dtype=-1), dict(dtype=0x11), dict(mode=2), dict(scale=0.0), dict(n_pages=-1), dict(max_pages=-1),
                dict(ld=19), dict(start=None), dict(kv=None), dict(groups=1), dict(groups=1, gs=E), dict(out=None), dict(q=None), dict(kc=None),
                dict(vc=None), dict(table=None), dict(q=A), dict(out=C), dict(out=C + size - 16), dict(out=D_ + 64)):
        assert cached(lib, **bad) == -1, bad
    assert cached(lib, out=C + size, ws=None) == -4            # right behind the cache
    for bad in (dict(D=80), dict(page=0), dict(page=100)):
        assert cached(lib, **bad) == -2, bad
    for bad in (dict(kc=C + 8), dict(q=B + 8), dict(ldo=1025)):
        assert cached(lib, **bad) == -3, bad
    assert cached(lib, ws=None) == -4 and cached(lib, wsb=100) == -4 and cached(lib, ws=W + 4) == -4
    assert cached(lib, T=1 << 28) == -8
    assert cached(lib, T=0) == 0 and cached(lib, S=0) == 0


def test_binding_refuses_what_is_no_device_tensor():
    t, i = torch.zeros(4, 128), torch.zeros(4, dtype=torch.int32)
    cache, four = torch.zeros(2, 2, 16, 64), preft.new_mx_cache(2, 2, 16, 64, device="cpu")
    assert four.shape == (2, 2, 16, 34) and preft.new_mx_cache(1, 3, 8, 128, device="cpu").numel() == 3 * 8 * 68
    with pytest.raises(ValueError, match="head_dim"):
        preft.new_mx_cache(1, 1, 8, 96, device="cpu")
    with pytest.raises(ValueError, match="q: need a 2-D device tensor"):
        preft.preft_qk_rotate(t, t, None, None, i, t, 2, 2, stream=0)
    with pytest.raises(ValueError, match="need one of them"):
        preft.preft_qk_rotate(None, None, None, None, i, t, 2, 2, stream=0)
    with pytest.raises(ValueError, match="k_cache"):
        preft.preft_kv_append(cache, cache, None, None, None, t, t, i.long(), i, t, 2, stream=0)
    for c in (cache, four):
        with pytest.raises(ValueError, match="k_cache: need a contiguous uint8 device tensor"):
            preft.preft_kv_append_mx(c, c, None, None, None, t, t, i.long(), i, t, 2, stream=0)
        with pytest.raises(ValueError, match="k_cache: need a contiguous uint8 device tensor"):
            preft.preft_kv_fetch_mx(t, t, i.long(), c, c, stream=0)
    with pytest.raises(ValueError, match="out: need a 2-D device tensor"):
        preft.preft_cached_attention_mx(t, t, i, None, i[:2], four, four, i[None], None, None, 2, 0.1, 0, four, stream=0)


def test_marshalling_declines_what_is_no_ordinary_call():
    from paper_2605_14217_amd import binding
    preft.load_library()
    native = binding._native
    assert native is not None
    t, i, cache, four = torch.zeros(4, 128), torch.zeros(4, dtype=torch.int32), torch.zeros(2, 2, 16, 64), preft.new_mx_cache(2, 2, 16, 64, device="cpu")
    assert native.qk_rotate(t, t, None, None, i, t, 2, 2, None, None, 1e-6, 0, 0) is None and native.qk_rotate() is None
    assert native.qk_rotate(None, None, None, None, i, t, 2, 2, None, None, 1e-6, 0, 0) is None
    for mx4, c in ((False, cache), (True, four), (True, cache), (False, None)):
        assert native.kv_append(mx4, c, c, None, None, None, t, t, i.long(), i, t, 2, None, None, 1e-6, 0, 0) is None
    assert native.cached_attention_mx(t, t, i, None, i, four, four, i[None], None, None, 2, 0.1, 0, four, 0) is None and native.cached_attention_mx(t) is None
    assert native.kv_append() is None and native.kv_fetch(t, t, i.long(), four, four, 0) is None and native.kv_fetch(1) is None
    with pytest.raises(TypeError):
        native.bind_heads(1)


# ---- the reference itself ---------------------------------------------------------------------------------------

def test_rotation_table():
    t = preft.new_rotation(100001, [1.0, 0.01], scale=0.5, device="cpu")
    assert t.shape == (100001, 4) and t.dtype == torch.float32
    for p in (0, 1, 77, 100000):
        want = [0.5 * math.cos(p), 0.5 * math.cos(0.01 * p), 0.5 * math.sin(p), 0.5 * math.sin(0.01 * p)]
        assert t[p].tolist() == pytest.approx(want, abs=2.0 ** -25 + 1e-12)


def test_reference_rotation_by_hand():
    x = torch.arange(1.0, 65.0)[None].repeat(2, 1)
    table = torch.zeros(3, 16)
    table[2, :8], table[2, 8:] = 0.0, 1.0                    # a quarter turn at position 2
    table[0, :8] = 1.0
    got, _ = ref.turned(x, 1, None, 0.0, torch.tensor([0, 9]), table, 0)
    assert torch.equal(got[0], x[0].double())
    assert got[1, :8].tolist() == [-v for v in range(9, 17)] and got[1, 8:16].tolist() == list(range(1, 9)) and torch.equal(got[1, 16:], x[1, 16:].double())
    got, _ = ref.turned(x, 1, None, 0.0, torch.tensor([-1, 2]), table, 1)
    assert torch.isnan(got[0]).all() and got[1, :4].tolist() == [-2, 1, -4, 3]
    got, _ = ref.turned(x, 1, torch.full((64,), 2.0), 0.0, None, None, 0)
    assert torch.allclose((got[0] ** 2).mean(), torch.tensor(4.0, dtype=torch.float64))


def test_reference_four_bits_by_hand():
    x = np.zeros((1, 32))
    x[0, :10] = [6.9, -6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.25, -0.26, 0.75]
    codes, powers = ref.to_four(x)
    assert powers.tolist() == [[127]] and codes[0, :10].tolist() == [7, 15, 6, 6, 4, 4, 2, 0, 9, 2]
    assert ref.from_four(codes, powers)[0, :10].tolist() == [6, -6, 4, 4, 2, 2, 1, 0, -0.5, 1]
    x[0, 0] = 7.0                                             # the next power: 3.5 is between 3 and 4, whose code is even
    codes, powers = ref.to_four(x)
    assert powers.tolist() == [[128]] and codes[0, :4].tolist() == [6, 13, 4, 4]          # 3.5 -> 4, -3, 2.5 -> 2, 1.75 -> 2
    x[0, 0] = np.inf
    assert ref.to_four(x)[1].tolist() == [[255]]
    assert ref.to_four(np.zeros((1, 32)))[1].tolist() == [[2]]
    page = ref.join(np.arange(64, dtype=np.uint8).reshape(1, 1, 1, 64) % 16, np.array([[[[9, 8]]]], np.uint8))
    assert page.reshape(-1)[:3].tolist() == [0x10, 0x32, 0x54] and page.reshape(-1)[-2:].tolist() == [9, 8] and page.shape == (1, 1, 1, 34)
    codes, powers = ref.split(page, 64)
    assert codes.reshape(-1).tolist() == [i % 16 for i in range(64)] and powers.reshape(-1).tolist() == [9, 8]
