"""How attention over a 4-bit cache is laid out, on the CPU: csrc/attention4_plan.cpp is host
code from sizes alone, compiled here by itself.  Every layout has room for the columns of any
row ends, and fits the card; the GPU tests' shapes meet every kind of it."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
CSRC = f"{ROOT}/paper_2608_01653_amd/csrc"
pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(f"{ROCM}/include/hip/hip_runtime.h"),
                                reason="needs g++ and the HIP headers")

DRIVER = r"""
#include <cstdio>
#include "cache4.h"
int main() {
    int batch, rows, heads, share, dim, ragged, window;
    long long max_len;
    while (std::scanf("%d %d %d %d %d %lld %d %d", &batch, &rows, &heads, &share, &dim, &max_len, &ragged, &window) == 8) {
        const hatq::AttentionPlan p = hatq::plan_attention(batch, rows, heads, share, dim, max_len, ragged != 0, window);
        std::printf("%d %d %d %lld %d\n", p.cols, p.waves, p.splits, (long long)p.tiles, hatq::wide_cols(dim));
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "driver.cpp").write_text(DRIVER)
    exe = str(d / "plan")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{CSRC}", str(d / "driver.cpp"),
                    f"{CSRC}/attention4_plan.cpp", "-o", exe], check=True, capture_output=True, timeout=300)

    def ask(cases):
        text = "\n".join(" ".join(str(int(v)) for v in c) for c in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return ask


def draw(rng):
    batch = int(2 ** rng.uniform(0, 12))
    ragged = rng.random() < 0.5
    per = int(2 ** rng.uniform(0, 11))
    rows = batch * per if not ragged else max(1, int(batch * per * rng.uniform(0.1, 1.0)))
    return (batch, rows, rng.choice([1, 2, 3, 8, 40]), rng.choice([1, 2, 5, 8, 64]), rng.choice([1, 32, 64, 65, 128, 129, 192, 200, 256]),
            int(2 ** rng.uniform(4, 30)), ragged, rng.choice([0, 0, 1, 500, 2 ** 30]))


def test_room_for_any_rows_and_inside_the_card(plan):
    rng = random.Random(1)
    cases = [draw(rng) for _ in range(4000)]
    for c, (cols, waves, splits, tiles, wide) in zip(cases, plan(cases)):
        batch, rows, heads, share, dim, max_len, ragged, window = c
        blocks = -(-dim // 64)
        assert cols in (16, wide) and waves in (1, 2, 4, 8, 16), c
        assert splits >= 1 and (splits == 1 or cols == 16), c
        assert waves * (blocks * 4096 + 128) <= 160 * 1024 and (waves <= 8 or blocks <= 2), c
        # (a block of many columns has at most 256 threads, the others 1024 and 512)
        assert cols == 16 or waves <= 4, c
        assert splits == 1 or tiles * heads * splits <= 512, c
        if ragged:
            for _ in range(3):
                ends = sorted(rng.randint(0, rows) for _ in range(batch))
                met = sum(-(-(e - b) * share // cols) for b, e in zip([0] + ends, ends))
                assert met <= tiles, c
        else:
            assert tiles == batch * -(-(rows // batch) * share // cols), c


def test_the_gpu_tests_shapes(plan):
    """(test_gpu_attention4.py: one token, long sequences, splits, blocks of many columns)"""
    got = plan([(14, 14, 2, 4, 128, 320, 0, 0), (1, 1, 2, 4, 128, 1024, 0, 0), (2, 2, 1, 4, 128, 9008, 0, 0), (2, 2, 1, 4, 128, 9008, 0, 40),
                (2, 2, 1, 4, 128, 2 ** 17, 0, 0), (1, 1, 1, 4, 64, 20, 0, 0)])
    assert [g[:3] for g in got] == [(16, 8, 1), (16, 8, 2), (16, 8, 17), (16, 2, 1), (16, 8, 128), (16, 1, 1)]
    for dim, wide in ((64, 64), (40, 64), (128, 48), (80, 48), (192, 32), (136, 32)):
        assert plan([(5, 508, 8, 8, dim, 400, 1, 0)])[0][0] == wide
    assert plan([(5, 508, 8, 8, 256, 400, 1, 0)])[0][0] == 16
    # one token a sequence is never wide
    assert plan([(64, 64, 8, 8, 128, 16384, 0, 0)])[0][:3] == (16, 8, 1)


def test_the_widest_window(plan):
    """A window of any size is at most all positions."""
    for batch, rows, max_len in ((1, 1, 65536), (2, 64, 4096), (1, 2 ** 24, 2 ** 30)):
        whole = plan([(batch, rows, 8, 4, 128, max_len, 0, 0)])
        assert plan([(batch, rows, 8, 4, 128, max_len, 0, 2 ** 31 - 1)]) == whole
