"""Calls over pages of 4-bit numbers whose keys are cut into one full round of workgroups, run on the CPU by the schedule's own code: every row from its keys once, no index outside its list."""
import shutil

import numpy as np
import pytest

from test_attention_schedule import BF16, CACHED, F32, answers, call, driver  # noqa: F401

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
MX = 0x10                                                     # as attention_plan.hpp marks the type of such a call


@pytest.mark.parametrize("rows,kv,units,units_f32", [([10] * 30, [3000] * 30, 60, 60),        # 30 tiles of 47 key tiles, 8 heads: two parts each, 480 workgroups
                                                     ([512], [30512], 64, 64),                # 16 tiles of 477: four parts each, 512 workgroups
                                                     ([40] * 16, [2000] * 16, 32, 64)])       # 32 of 32: bf16 makes no parts below 24 key tiles here, f32 two, 512 workgroups
def test_one_full_round(driver, rows, kv, units, units_f32):  # noqa: F811
    for dtype, want in ((MX | BF16, units), (MX | F32, units_f32)):
        (direct, split, merge, got, grid, _), = answers(driver, [call(CACHED, dtype, 32, 8, rows, kv=kv, max_keys=32768)])
        assert direct and split and merge and got == want <= grid


def test_a_little_more_than_one_round(driver):  # noqa: F811
    """40 tiles of 16 to 140 key tiles, 8 heads: by 1/384 of the work they make more than 512 workgroups and fewer than 768, a part and an even share of the work are shorter than the longest tile."""
    kv = [1000 + 200 * s for s in range(40)]
    (direct, split, merge, got, grid, _), = answers(driver, [call(CACHED, MX | BF16, 32, 8, [10] * 40, kv=kv, max_keys=16384)])
    tiles = [-(-k // 64) for k in kv]
    to = -(-sum(tiles) * 8 // 384)
    assert direct and split and merge and got == sum(-(-n // to) for n in tiles) <= grid and 64 < got <= 96


@pytest.mark.parametrize("seed", range(3))
def test_random_calls_of_wide_tiles(driver, seed):  # noqa: F811
    """Around the sizes that it is for: tiles of all key/value heads between 64 and 512, lengths alike and not, tables short and long; and the lists that groups need."""
    rng = np.random.Generator(np.random.PCG64(seed + 40))
    calls = []
    for _ in range(60):
        kv_heads = int(rng.choice([1, 2, 3, 8, 16]))
        group = int(rng.choice([1, 3, 4, 8, 16]))
        S = int(rng.choice([1, 2, 7, 30, 100, 250]))
        most = int(rng.choice([512, 5000, 40000, 1 << 20]))
        tiles = int(rng.integers(1, 700)) // kv_heads + 1
        rows = np.maximum(1, rng.integers(0, 2 * max(1, tiles * 128 // (group * S)) + 1, size=S))
        kv = rng.integers(0, most + 1, size=S) if rng.random() < 0.5 else np.full(S, most - int(rng.integers(0, 500)))
        g = int(rng.integers(1, 4)) if rng.random() < 0.2 else 0
        start = np.sort(rng.integers(0, S + 1, size=g + 1))
        calls.append(call(CACHED, MX | int(rng.integers(0, 2)), kv_heads * group, kv_heads, rows, rng.integers(0, 3, size=S) if rng.random() < 0.2 else None, kv, most,
                          start if g else None, rng.integers(0, most + 1, size=g) if g else None))
    got = answers(driver, calls)
    assert all(units <= grid for _, _, _, units, grid, _ in got) and {g[0] for g in got} == {0, 1}


def test_very_long_tables(driver):  # noqa: F811
    calls = [call(CACHED, MX | BF16, 16, 1, [3000], kv=[600_000], max_keys=600_000), call(CACHED, MX | F32, 8, 8, [400, 3, 40], kv=[2_000_000, 17, 1 << 20], max_keys=1 << 21),
             call(CACHED, MX | BF16, 4, 4, [40] * 60, kv=[(1 << 30) >> (s % 31) for s in range(60)], max_keys=1 << 30),
             call(CACHED, MX | BF16, 32, 8, [100] * 2, kv=[1 << 30] * 2, max_keys=1 << 30)]
    got = answers(driver, calls)
    assert all(units <= grid for _, _, _, units, grid, _ in got)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_decode_rows_beside_a_prompt_are_cut_as_without_it(driver, dtype):  # noqa: F811
    """A prompt's rows are in the batch, but not in the call: its tiles are all narrow, for which one full round is not looked for.  40 rows, 8 heads: ranges of 1/256 of all their key tiles."""
    kv = [1000 + 200 * s for s in range(40)] + [350]
    (direct, split, merge, got, grid, _), = answers(driver, [call(CACHED, MX | dtype, 32, 8, [1] * 40 + [350], [0] * 40 + [350], kv, 16384)])
    tiles = [-(-k // 64) for k in kv[:40]]
    to = -(-sum(tiles) * 8 // 256)
    assert direct and split and merge and got == sum(-(-n // to) for n in tiles) <= grid
    # a chunk of ten rows among them is a wide tile
    kv[39] = 9000
    (direct, _, _, got, _, _), = answers(driver, [call(CACHED, MX | dtype, 32, 8, [1] * 39 + [10, 350], [0] * 40 + [350], kv, 16384)])
    tiles[39] = -(-9000 // 64)
    to = -(-sum(tiles) * 8 // 384)
    assert direct and got == sum(-(-n // to) for n in tiles)
