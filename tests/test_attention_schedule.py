"""The schedule of attention calls, run on the CPU by the kernels' own code (tests/attention_schedule_driver.hip): every row of a call gets its result once, from its keys, whatever the
batch looks like, and no index leaves its list."""
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
F32, BF16 = 0, 1
PROMPT, CACHED, MALFORMED = 1, 2, 10


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = tmp_path_factory.mktemp("attention_schedule") / "driver"
    build = subprocess.run(["hipcc", "--cuda-host-only", "-std=c++17", "-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                            "-Xarch_host", "-fno-sanitize-recover=all", os.path.join(ROOT, "tests", "attention_schedule_driver.hip"), "-o", str(exe)],
                           capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    return exe


def call(kind, dtype, heads, kv_heads, rows, prefill=None, kv=None, max_keys=0, group_start=None, prefix=None, start=None, T=None):
    """One call of the driver's input; rows of the segments, or their offsets."""
    if start is None:
        start = np.concatenate([[0], np.cumsum(rows)])
    S, prefix = len(start) - 1, [] if prefix is None else prefix
    words = [kind, dtype, int(start[-1]) if T is None else T, S, heads, kv_heads, len(prefix) if kind % MALFORMED == CACHED else 0, max_keys, *start, *([0] * S if prefill is None else prefill)]
    if kind % MALFORMED == CACHED:
        words += [*kv, *(group_start if len(prefix) else []), *prefix]
    return " ".join(str(int(w)) for w in words)


def answers(driver, calls):
    """direct, split, merge, units, grid, entries of every call, after a look at the verdicts."""
    run = subprocess.run([str(driver)], input="\n".join(calls) + "\n", capture_output=True, text=True, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"), timeout=600)
    assert run.returncode == 0, run.stdout[-500:] + run.stderr[-3000:]
    lines = [line.split(" ", 6) for line in run.stdout.splitlines()]
    assert len(lines) == len(calls)
    for asked, line in zip(calls, lines):
        assert line[6] == "ok", (line, asked[:400])
    return [[int(x) for x in line[:6]] for line in lines]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_groups_over_short_tables_are_joined(driver, dtype):
    """Tables so short that no keys are cut: the rows of a group are parts all the same."""
    calls, lengths = [], [64, 96, 128, 160, 192, 256, 272, 320]
    for most in lengths:
        calls.append(call(CACHED, dtype, 8, 2, [1, 1, 1, 40, 1, 1], kv=[most, most - 1, 64, 60, most, 9], max_keys=most, group_start=[0, 3, 5], prefix=[64, 64 if most > 64 else 3]))
    got = answers(driver, calls)
    assert {g[1] for g in got} == {0, 1}, "tables on both sides of the line are meant"
    for most, (direct, _, merge, _, _, joins) in zip(lengths, got):
        assert not direct and merge and joins >= 3


def random_call(rng):
    kv_heads = int(rng.choice([1, 2, 3, 8]))
    heads = kv_heads * int(rng.choice([1, 1, 4, 7, 8, 40]))
    S = int(rng.choice([1, 2, 5, 17, 60, 300]))
    dtype = int(rng.integers(0, 2))
    most_rows = int(rng.choice([1, 2, 8, 40, 300 if S < 20 else 8]))
    rows = rng.integers(0, most_rows + 1, size=S)
    if rng.random() < 0.4:
        rows[:] = np.minimum(rows, 1)
    if rows.sum() == 0:
        rows[0] = 1
    if rng.random() < 0.35:
        prefill = rng.integers(0, rows.max() + 2, size=S)
        if rng.random() < 0.3:
            rows[0] = 2500 // max(1, heads // kv_heads // 8)
            prefill[0] = rows[0]
        return call(PROMPT, dtype, heads, kv_heads, rows, prefill)
    max_keys = 16 * int(rng.choice([2, 8, 10, 16, 17, 40, 300, 3000]))
    kv = np.maximum(rng.integers(0, max_keys + 1, size=S) - rng.integers(0, 2) * rng.integers(0, max_keys, size=S), 0)
    prefill = rng.integers(0, 3, size=S) if rng.random() < 0.3 else None
    if rng.random() < 0.5:
        return call(CACHED, dtype, heads, kv_heads, rows, prefill, kv, max_keys)
    g = int(rng.integers(1, 6))
    start = np.sort(rng.integers(0, S + 1, size=g + 1))
    if rng.random() < 0.5:
        start[0], start[-1] = 0, S
    return call(CACHED, dtype, heads, kv_heads, rows, prefill, kv, max_keys, start, rng.integers(0, max_keys + 1, size=g))


@pytest.mark.parametrize("seed", range(3))
def test_every_row_of_random_batches_is_written_once_from_its_keys(driver, seed):
    rng = np.random.Generator(np.random.PCG64(seed))
    got = answers(driver, [random_call(rng) for _ in range(60)])
    assert {(g[0], g[2]) for g in got} == {(0, 0), (0, 1), (1, 0), (1, 1)}
    assert all(units <= grid for _, _, _, units, grid, _ in got)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_requests_than_the_schedule_keeps_in_lds(driver, dtype):
    rng = np.random.Generator(np.random.PCG64(7))
    S = 4500
    rows, kv = rng.integers(0, 3, size=S), rng.integers(0, 700, size=S)
    answers(driver, [call(CACHED, dtype, 4, 1, rows, rng.integers(0, 2, size=S), kv, 704),
                     call(CACHED, dtype, 8, 2, rows, None, kv, 704, [0, 100, 300, S - 900], [300, 64, 500]),
                     call(PROMPT, dtype, 8, 2, rows, rows)])


def test_batches_over_very_long_tables(driver):
    """Workgroups and parts are enough whatever the keys come to: many tiles over millions of tokens, and tables so long that the work of all tiles does not fit 31 bits, on both sides of
    that line."""
    calls = [call(CACHED, BF16, 16, 1, [8184], kv=[600_000], max_keys=600_000),              # 1023 tiles of 9375 key tiles
             call(CACHED, F32, 16, 1, [4000], kv=[3_000_000], max_keys=3_000_000),
             call(CACHED, BF16, 8, 8, [1500, 3, 40], kv=[2_000_000, 17, 1 << 20], max_keys=1 << 21),
             call(CACHED, F32, 2, 1, [8000, 6000, 9000], kv=[9_000_000, 9_000_000, 100], max_keys=10_000_000),
             call(PROMPT, BF16, 8, 2, [8000], prefill=[8000])]
    for S in (1, 8, 126, 127, 128, 200, 300):
        calls.append(call(CACHED, BF16, 4, 1, [1] * S, kv=[(1 << 30) - 7 * s for s in range(S)], max_keys=1 << 30))
        calls.append(call(CACHED, F32, 4, 4, [1] * S, kv=[(1 << 30) >> (s % 31) for s in range(S)], max_keys=1 << 30))
    got = answers(driver, calls)
    assert {g[0] for g in got[5:]} == {0, 1}
    assert all(units <= grid for _, _, _, units, grid, _ in got)


def goes_back(start, T):
    at = np.clip(start, 0, T)
    return bool((np.diff(at) < 0).any())


def test_offsets_that_go_back_leave_nothing_to_run(driver):
    """Segments that overlap, in both forms of the schedule, with keys to cut and without: no unit, no entry of the join, whatever the sums over them would be.  Offsets outside the batch
    that do not go back within it are ordinary."""
    T, big = 1000, 1 << 24
    tables = [[0, 1000, 0, 1000], [0, 500, 200, 900, -4, 1000], [5, 5, 4, 1000, 1000], [0, 1000] * 2000 + [0], [0, 2 ** 31 - 1, -2 ** 31, 1000]]
    calls = []
    for start in tables:
        S = len(start) - 1
        for dtype in (BF16, F32):
            calls.append(call(MALFORMED + PROMPT, dtype, 4, 2, None, [1000] * S, start=start, T=T))
            for most in (64, 320, 100_000):
                calls.append(call(MALFORMED + CACHED, dtype, 4, 2, None, None, [most] * S, most, start=start, T=T))
                calls.append(call(MALFORMED + CACHED, dtype, 4, 2, None, None, [most] * S, most, [0, S // 2, S], [most, 64], start=start, T=T))
    # rows and tiles of all segments together past 31 bits
    calls.append(call(MALFORMED + CACHED, BF16, 8, 8, None, None, [64] * 400, 64, [0, 400], [64], start=[0, big] * 200 + [0], T=big))
    # groups that overlap
    for gstart in ([0, 3, 1, 4], [2, 1], [4, 0, 4]):
        calls.append(call(MALFORMED + CACHED, BF16, 4, 2, [1, 2, 3, 1], None, [300] * 4, 320, gstart, [100] * (len(gstart) - 1)))
    for _, _, _, units, _, joins in answers(driver, calls):
        assert units == 0 and joins == 0
    outside = [-7, 0, 10, 900, 900, 5000]
    got = answers(driver, [call(MALFORMED + PROMPT, BF16, 4, 2, None, [100] * 5, start=outside, T=T),
                           call(MALFORMED + CACHED, BF16, 4, 2, None, None, [100] * 5, 320, [-3, 2, 9], [100, 64], start=outside, T=T)])
    assert all(g[3] > 0 for g in got)


@pytest.mark.parametrize("seed", range(2))
def test_random_tables_stay_within_the_lists(driver, seed):
    """Anything in any table: no index leaves its list, and the join takes no entry that nobody wrote."""
    rng = np.random.Generator(np.random.PCG64(100 + seed))
    calls, back = [], []

    def wild(n, most):
        v = rng.integers(-3, most + 4, size=n)
        odd = rng.random(n) < 0.1
        v[odd] = rng.choice([-2 ** 31, -1, 0, 2 ** 30, 2 ** 31 - 1], size=int(odd.sum()))
        return v
    for _ in range(60):
        kv_heads = int(rng.choice([1, 2, 8]))
        S, T = int(rng.choice([1, 3, 20, 270])), int(rng.choice([1, 60, 500, 4000]))
        start = wild(S + 1, T)
        if rng.random() < 0.5:
            start = np.sort(start)
        max_keys = 16 * int(rng.choice([1, 9, 20, 400]))
        g = int(rng.choice([0, 0, 1, 4]))
        gstart = wild(g + 1, S) if rng.random() < 0.4 else np.sort(wild(g + 1, S))
        kind = PROMPT if rng.random() < 0.3 else CACHED
        calls.append(call(MALFORMED + kind, int(rng.integers(0, 2)), 4 * kv_heads, kv_heads, None, wild(S, 40), wild(S, max_keys), max_keys,
                          gstart, wild(g, max_keys) if kind == CACHED else None, start=start, T=T))
        back.append(goes_back(start, T) or (kind == CACHED and g > 0 and goes_back(gstart, S)))
    for got, b in zip(answers(driver, calls), back):
        assert got[3] <= got[4] and got[5] >= 0
        assert not b or got[3] == 0


def test_sizes_that_are_taken_keep_grids_and_lists_in_32_bits(driver):
    """The largest calls by every size that counts, many more groups than rows among them: workgroups and capacities stay countable."""
    sizes = [(T, S, heads, kv_heads, groups) for T, heads in ((1, 1), (10, 1024), (1 << 17, 1024), ((1 << 18) - 1, 1024), ((1 << 28) - 1, 1), (1 << 20, 128)) for kv_heads in {1, heads}
             for S, groups in ((1, 0), (1, (1 << 28) - 2), (T, min(T, (1 << 28) - T - 1) // 2), (min(T, (1 << 28) - 1), 0), (5, 10_000_000))]
    lines = [f"22 {dtype} {T} {S} {heads} {kv_heads} {groups} {most}" for T, S, heads, kv_heads, groups in sizes for dtype in (BF16, F32) for most in (64, 1 << 30)]
    taken = [g for g in answers(driver, lines) if g[0]]
    assert len(taken) > len(lines) // 2
    for _, workgroups, *caps in taken:
        assert 0 < workgroups < 2 ** 32 and all(0 < c < 2 ** 31 for c in caps)


def test_schedules_stand_in_one_place_whatever_the_head_size(driver):
    """Layers whose heads differ in size take one schedule: nothing before the lists depends on head_dim, prompts that are cut included."""
    answers(driver, [f"22 {BF16} {T} {S} {heads} {kv_heads} {groups} 4096" for T, S in ((1, 1), (600, 1), (1200, 2), (4000, 1), (20_000, 3)) for heads, kv_heads in ((4, 1), (8, 2), (32, 8))
                     for groups in (0, 3)])


def test_prompts_that_are_cut_have_room_for_their_parts(driver):
    """Few long prompts, of every number of tiles that is cut, even and uneven."""
    rng, calls = np.random.Generator(np.random.PCG64(12)), []
    while len(calls) < 40:
        kv_heads, G, S = int(rng.choice([1, 2, 4, 8])), int(rng.choice([1, 2, 4, 7])), int(rng.choice([1, 1, 2, 3]))
        most = min(2500, (256 // kv_heads - S) * 128 // G)                # tiles that fill no more than half the chip
        if most <= 512 * S:
            continue
        T = int(rng.integers(512 * S, most))
        cut = np.sort(rng.integers(0, T + 1, size=S - 1)) if rng.random() < 0.7 else np.linspace(0, T, S + 1).astype(int)[1:-1]
        start = np.concatenate([[0], cut, [T]])
        calls.append(call(PROMPT, int(rng.integers(0, 2)), kv_heads * G, kv_heads, None, np.diff(start) - rng.integers(0, 3, size=S), start=start, T=T))
    got = answers(driver, calls)
    assert sum(g[2] for g in got) >= 20 and all(units <= grid for _, _, _, units, grid, _ in got)
