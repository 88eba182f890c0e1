"""The plans of the 4-bit products on the host (no GPU): a workgroup's rows of the operand that goes to LDS directly
are addressed by 32-bit byte offsets from its first row, so a plan may not pair a tall tile with a long pitch."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2003_05148_amd")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

PROGRAM = r"""
#include <cstdio>
#include "kq_group.h"
using namespace kq;
int main() {
    long long product, ldb, i, j, c, aligned;
    while (scanf("%lld %lld %lld %lld %lld %lld", &product, &aligned, &ldb, &i, &j, &c) == 6) {
        const GemmPlan g = gemm_plan((Product)product, (const void*)(aligned ? 0x10000 : 0x10002), ldb, i, j, c, 1);
        printf("%d %d %d %d %d %lld\n", g.bi, g.bj, g.splits, g.steps_per_split, (int)g.stage_b, (long long)g.pitch);
    }
}
"""
LINEAR, GRAD_INPUT, GRAD_WEIGHT, GRAD_SCALES = range(4)
MAX_FEATURES, MAX_ROWS, MAX_VALUES = 1 << 24, 1 << 22, 1 << 34


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """A function from lists of (product, aligned, ldb, I, J, C) to their plans."""
    if not os.path.exists(HIPCC) and shutil.which("hipcc") is None:
        pytest.skip("hipcc not installed")
    pytest.importorskip("paper_2003_05148_amd")   # (the library is built)
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.hip").write_text(PROGRAM)
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"), str(d / "plan.hip"),
           f"-L{PKG}", "-l:libkq.so", f"-Wl,-rpath,{PKG}", "-o", str(d / "plan")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def of(cases):
        r = subprocess.run([str(d / "plan")], input="\n".join(" ".join(map(str, c)) for c in cases) + "\n", capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        out = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
        assert len(out) == len(cases)
        return out
    return of


def last_offset(case, plan):
    """The largest byte offset of a workgroup's rows and chunks."""
    _, _, ldb, _, J, _ = case
    _, bj, _, _, stage, pitch = plan
    return (min(bj, J) - 1) * 2 * (pitch if stage else ldb) + 16 * 7


def test_row_offsets_stay_in_32_bits(plans):
    """The whole range of accepted sizes, around the pitch at which 255 rows pass 2^32 bytes and at the largest."""
    cases = []
    long = [MAX_FEATURES, MAX_FEATURES - 1, 9_000_000, 8_421_503, 8_421_504, 8_421_568, 1 << 23, (1 << 22) + 8, 1 << 22, 1 << 20, 100_003]
    for c in long:
        for j in (17, 128, 129, 255, 256, 257, 512, 1000, 1024, 4096):
            for i in (1, 100, 128, 256, 1000, 1024, 2048):
                if i * c > MAX_VALUES or j * c > MAX_VALUES:
                    continue
                for product in (LINEAR, GRAD_INPUT):
                    for aligned, ldb in ((1, c), (0, c), (1, c + 8), (1, 1 << 30)):
                        cases.append((product, aligned, ldb, i, j, c))
    for c in (MAX_ROWS, MAX_ROWS - 1, 100_000):
        for j in (1, 255, 256, 1000, 4096):
            for i in (1, 256, 4096):
                for product in (GRAD_WEIGHT, GRAD_SCALES):
                    cases.append((product, 1, j, i, j, c))
    assert len(cases) > 500
    for case, plan in zip(cases, plans(cases)):
        assert last_offset(case, plan) < 1 << 32, (case, plan)


def test_ordinary_sizes_take_the_tall_tile(plans):
    """The bound is one on the pitch alone: ordinary products take 256 rows a tile, and so does the longest pitch below it."""
    (a, b, c) = plans([(GRAD_INPUT, 1, 4096, 4096, 4096, 4096), (LINEAR, 1, 25088, 4096, 4096, 25088), (LINEAR, 1, 8_388_608, 2048, 2048, 8_388_608)])
    assert a[1] == 256 and b[1] == 256 and c[1] == 256
