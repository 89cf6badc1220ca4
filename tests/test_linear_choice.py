"""Which kernel the linear layers over tokens take, on the CPU: csrc/linear_choice.cpp is
host code from sizes alone, compiled here by itself.  The shapes of the GPU tests have to
meet every kernel in every form, so that a new rule cannot leave one without a test."""
import os
import shutil
import subprocess

import pytest

import test_gpu_expert_block as blocks
import test_gpu_linear_paths as paths

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
CSRC = f"{ROOT}/paper_2608_01653_amd/csrc"
pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(f"{ROCM}/include/hip/hip_runtime.h"),
                                reason="needs g++ and the HIP headers")

DRIVER = r"""
#include <cstdio>
#include "hatq.h"
#include "linear.h"
int main() {
    int rows, cin, cout, experts, gated;
    while (std::scanf("%d %d %d %d %d", &rows, &cin, &cout, &experts, &gated) == 5) {
        static const int32_t ends = 0;
        hatq::LinearArgs a{};
        a.rows = a.x_rows = rows;
        a.experts = experts > 0 ? experts : 1;
        a.ends = experts > 0 ? &ends : nullptr;
        a.cout = cout;
        a.cout_pad = (cout + 31) / 32 * 32 * (gated ? 2 : 1);
        a.k_stride = (cin + 63) / 64 * 64;
        a.gated = gated;
        const hatq::LinearChoice c = hatq::choose_linear(a);
        const hatq::TokenChoice t = hatq::choose_tokens(a);
        std::printf("%d %d %d %d %d\n", c.kernel, c.waves, (int)hatq::linear_takes_tokens(a), (int)t.small, t.ch);
    }
}
"""
TILES = ["32x64", "64x64", "64x128", "128x128", "128x256", "256x256"]


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    """choose(shapes) of (rows, cin, cout, experts (0: one layer), gated): for each the
    kernel of codes, and that of floats or None where the tokens are quantized first."""
    d = tmp_path_factory.mktemp("choice")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{ROOT}/include", f"-I{CSRC}",
                    "-fsanitize=undefined", "-fno-sanitize-recover=all", "-O1", f"{CSRC}/linear_choice.cpp", str(d / "driver.cpp"), "-o", str(d / "choose")],
                   check=True, capture_output=True, timeout=300)

    def run(shapes):
        text = "".join(f"{r} {i} {o} {e} {int(g)}\n" for r, i, o, e, g in shapes)
        out = subprocess.run([str(d / "choose")], input=text, capture_output=True, text=True, timeout=60, check=True).stdout
        names = []
        for (_, _, _, e, g), line in zip(shapes, out.splitlines()):
            kernel, waves, takes, small, ch = map(int, line.split())
            form = (bool(e), bool(g))
            codes = ("tile " + TILES[kernel] if kernel < 6 else f"stream {16 << (kernel - 6)} rows, {waves} waves", *form)
            names.append((codes, (("small" if small else "token") + f" {ch}", *form) if takes else None))
        assert len(names) == len(shapes)
        return names
    return run


FORMS = [(e, g) for e in (False, True) for g in (False, True)]


def test_codes_meet_every_kernel(choose):
    met = {c for c, _ in choose(paths.PRODUCTS)}
    want = {("tile " + t, *f) for t in TILES for f in FORMS}
    want |= {(f"stream 16 rows, {w} waves", *f) for w in (2, 4, 8) for f in FORMS}
    want |= {("stream 32 rows, 8 waves", *f) for f in FORMS}
    assert want <= met, sorted(want - met)


def test_floats_meet_every_kernel(choose):
    met = {t for _, t in choose(paths.FORWARDS)}
    want = {(f"small {ch}", *f) for ch in (1, 2, 4) for f in FORMS} | {(f"token {ch}", False, g) for ch in (1, 2, 4) for g in (False, True)}
    assert want <= met, sorted(want - met)
    assert None in met


def test_blocks_meet_every_path(choose):
    """Of the expert block: the first launch's instances (waves a row and chunks of a lane),
    its two fallbacks, and both layouts of the hidden and output rows."""
    first, layout = set(), set()
    shapes = [(tokens * topk, hidden, width, e, False) for tokens, topk, e, width, hidden, _ in blocks.BLOCKS]
    for (tokens, topk, e, width, hidden, _), (_, floats) in zip(blocks.BLOCKS, choose(shapes)):
        chunks = (width + 63) // 64 * 8
        first.add("pairs" if tokens * topk > 32768 else next((n for n in (64, 128, 256, 512, 1024) if chunks <= n), "width"))
        layout.add("beside" if floats else "in place, " + ("wider" if hidden < width else "narrower" if hidden > width else "as wide"))
    assert first == {64, 128, 256, 512, 1024, "pairs", "width"}
    assert layout == {"beside", "in place, wider", "in place, narrower", "in place, as wide"}


def test_rows_that_may_meet_in_one_expert(choose):
    """Floats by expert: the small kernel reads an expert's weights again for every 16 of its
    rows, so past 8 rows an expert it takes only small products; the ends are not known."""
    wide = [(12 * e, 2048, cout, e, g) for e, cout, g in ((1024, 8192, 0), (256, 8192, 0), (64, 8192, 0), (64, 4096, 1), (256, 2048, 0))]
    assert [t for _, t in choose(wide)] == [None] * len(wide)
    small = [(8 * 256, 2048, 8192, 256, 0), (12 * 64, 2048, 1024, 64, 0), (12 * 1024, 512, 512, 1024, 0), (300, 320, 320, 8, 0)]
    assert all(t for _, t in choose(small))
