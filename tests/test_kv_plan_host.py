"""preft_kv_plan's kernel run on the CPU (tests/kv_plan_driver.hip): tables that no device should be handed stay within their bounds."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import attention_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
ALL = -1000000


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = tmp_path_factory.mktemp("kv_plan") / "driver"
    build = subprocess.run(["hipcc", "--cuda-host-only", "-std=c++17", "-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                            "-Xarch_host", "-fno-sanitize-recover=all", os.path.join(ROOT, "tests", "kv_plan_driver.hip"), "-o", str(exe)],
                           capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    return exe


def ask(driver, lines, *args):
    run = subprocess.run([str(driver), *args], input="\n".join(lines) + "\n", capture_output=True, text=True, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"), timeout=300)
    assert run.returncode == 0, run.stdout[-500:] + run.stderr[-3000:]
    return [[int(x) for x in line.split()] for line in run.stdout.splitlines()]


def test_ordinary_tables_by_the_driver(driver):
    """The driver itself: what it runs is the plan."""
    start = [0, 17, 17, 18, 60, 700, 1300]
    got, = ask(driver, [f"6 1300 100 90 16 {ALL} 0 0 0 {' '.join(map(str, start))} 13"])
    slot, at, _, _, counts = ref.plan(np.array(start), np.full(6, 13), np.zeros((6, 100), int), np.arange(90), 16)      # pages that hold earlier tokens: 0
    assert got == [0, 2, *counts, 1300, at.sum(), slot.sum()]


def test_pages_of_overlapping_requests_past_31_bits(driver):
    """16 500 requests that all claim the same million rows need more than 2^31 pages before the last one's: no page is picked from outside the list."""
    T = 1 << 20
    overlapping = f"33000 {T} 140000 50 8 -1 16500 0 {T - 2048} {T} 0"
    short = f"4 3000 400 50 8 {ALL} 2 0 2900 3000 0"
    for line, rows in ((overlapping, 1024), (short, 3000)):
        got, = ask(driver, [line])
        assert got[0] == 0 and got[4] == rows


def test_store_of_as_many_rows_as_32_bits_count(driver):
    rows = [1, 4, 5, 2 ** 31 - 4, 2 ** 31 - 3, 2 ** 31 - 1]
    assert ask(driver, [str(t) for t in rows], "store") == [[0, -(-t // 4)] for t in rows]
