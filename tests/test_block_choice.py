"""Which kernel kq_block_linear takes of a size, on the host (no GPU): row by row of W for few rows and small products, in tiles
otherwise.  tests/test_gpu_block_linear_tiles.py multiplies the sizes."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2003_05148_amd")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
F32, BF16, F16, E4M3 = 0, 1, 2, 3   # KQ_T_*

PROGRAM = r"""
#include <cstdio>
#include "kq_block.h"
using namespace kq;
int main() {
    int xt, yt;
    long long m, n, k;
    while (scanf("%d %d %lld %lld %lld", &xt, &yt, &m, &n, &k) == 5) {
        const BlockLinearPlan z = block_linear_plan(xt, yt, m, n, k);
        printf("%d %d %d %d %lld %d %d %d\n", z.few, z.plan.bi, z.plan.bj, z.plan.splits, (long long)z.plan.rest_from, z.few_plan.row_tiles, z.few_plan.waves, z.few_plan.splits);
    }
}
"""

# (m, n, k) of kq_block_linear
TILES = [(1025, 1, 1), (1030, 260, 300), (1100, 130, 700), (1537, 129, 127), (2049, 300, 257), (1040, 200, 5000), (2100, 1030, 520),
         (1200, 2050, 1300), (1030, 700, 9000)]
LARGE_TILES = [(3900, 4090, 700), (4000, 4100, 2100), (4097, 4500, 1000), (4353, 4500, 2200)]
FEW = [(1, 1, 1), (5, 100, 300), (16, 129, 1000), (17, 129, 130), (33, 5, 300), (17, 1000, 512), (64, 1000, 4000), (100, 130, 2100),
       (130, 1000, 300), (257, 300, 385), (300, 17, 5000), (1000, 60, 900), (1024, 1, 1)]


@pytest.fixture(scope="module")
def choices(tmp_path_factory):
    if not os.path.exists(HIPCC) and shutil.which("hipcc") is None:
        pytest.skip("hipcc not installed")
    pytest.importorskip("paper_2003_05148_amd")   # (the library is built)
    d = tmp_path_factory.mktemp("choice")
    (d / "choice.hip").write_text(PROGRAM)
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), str(d / "choice.hip"),
           f"-L{PKG}", "-l:libkq.so", f"-Wl,-rpath,{PKG}", "-o", str(d / "choice")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def of(cases):
        r = subprocess.run([str(d / "choice")], input="\n".join(" ".join(map(str, c)) for c in cases) + "\n", capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        out = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
        assert len(out) == len(cases)
        return out
    return of


@pytest.mark.parametrize("x", [F32, BF16, F16, E4M3])
@pytest.mark.parametrize("y", [F32, BF16, F16])
def test_the_multiplied_sizes_take_tiles_or_rows(choices, x, y):
    got = choices([(x, y, *s) for s in TILES + LARGE_TILES])
    assert not any(g[0] for g in got), got
    assert {(g[1], g[2]) for g in got} == {(128, 64), (128, 128), (256, 256)}
    small = got[:len(TILES)]
    assert any(g[3] > 1 for g in small) and any(g[3] == 1 for g in small)      # split contractions and whole ones
    assert any(g[4] > 0 for g in got)                                          # the last columns in a tile of their own
    got = choices([(x, y, *s) for s in FEW])
    assert all(g[0] for g in got), got
    assert {g[5] for g in got} >= {1, 2} and any(g[7] > 1 for g in got)


def test_many_rows_and_large_products_take_tiles(choices):
    cases = [(x, y, m, n, k) for x in (F32, BF16, E4M3) for y in (F32, BF16) for m, n, k in
             [(1025, 1, 1), (1 << 22, 100, 100), (1025, 1 << 20, 128), (512, 4096, 4096), (1024, 4096, 25088), (256, 8192, 8192)]]
    assert not any(g[0] for g in choices(cases))
    cases = [(x, y, m, n, k) for x in (F32, BF16, E4M3) for y in (F32, BF16) for m in (1, 16) for n, k in [(1, 1), (1 << 24, 128), (128, 1 << 24)]]
    assert all(g[0] for g in choices(cases))
