"""The plans of the 8-bit products on the host (no GPU): which tiles and splits sizes take, and that what a kernel addresses
with 32 bits stays inside them over the whole range of accepted sizes."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2003_05148_amd")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

PROGRAM = r"""
#include <cstdio>
#include "kq_block.h"
using namespace kq;
int main() {
    char what;
    long long exact, i, j, c;
    while (scanf(" %c %lld %lld %lld %lld", &what, &exact, &i, &j, &c) == 5) {
        if (what == 'g') {
            const BlockGemmPlan g = block_gemm_plan(exact != 0, i, j, c);
            printf("%d %d %d %d %lld %d %d %lld\n", g.bi, g.bj, g.splits, g.steps_per_split, (long long)g.rest_from, g.rest_bi, g.rest_bj, (long long)g.part_bytes);
        } else {
            const BlockMatvecPlan v = what == 'v' ? block_matvec_plan((int)j, i, c) : block_matvec_plan((int)exact, (int)j, i, c);
            printf("%d %d %d %d %lld 0 0 0\n", v.row_tiles, v.waves, v.splits, v.blocks_per_split, (long long)v.ws_bytes);
        }
    }
}
"""
MAX_FEATURES, MAX_ROWS, MAX_VALUES = 1 << 24, 1 << 22, 1 << 34

# (i, j, c) of products: columns and rows of the output, contraction.  tests/test_gpu_block_linear.py multiplies them.
SIZES = [(300, 20, 5000), (1000, 40, 1100), (2100, 130, 4100), (2050, 1030, 400), (1500, 2300, 520), (3000, 2990, 130),
         (4090, 3900, 700), (4100, 4000, 2100), (4500, 4097, 3000)]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
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


def pitch(c):
    return -(-c // 128) * 128


def accepted():
    long = [MAX_FEATURES, MAX_FEATURES - 1, 1 << 20, 100_003, 25088, 4096, 1000, 129, 128, 127, 1]
    for c in long:
        for i in (1, 100, 128, 129, 1000, 4096, 25088, MAX_FEATURES):
            for j in (1, 16, 17, 64, 65, 129, 1000, 4096, MAX_ROWS):
                if i * c <= MAX_VALUES and j * c <= MAX_VALUES and i * j <= MAX_VALUES:
                    yield i, j, c


def test_products_over_the_whole_range(plans):
    cases = [("g", e, i, j, c) for e in (0, 1) for i, j, c in accepted()]
    assert len(cases) > 500
    for (_, _, i, j, c), (bi, bj, splits, per, rest, rbi, rbj, part) in zip(cases, plans(cases)):
        steps = pitch(c) // 128
        assert (bi, bj) in ((128, 64), (128, 128), (256, 256))
        # a tile's rows are addressed by 32-bit byte offsets from its first one, their exponents too
        assert (min(bi, i) - 1) * pitch(c) + 127 < 1 << 32 and (min(bj, j) - 1) * pitch(c) + 127 < 1 << 32
        assert 1 <= splits <= 65535 and per >= 1 and (splits - 1) * per < steps <= splits * per
        assert -(-i // bi) * -(-j // bj) * splits < 1 << 31
        assert part == (0 if splits == 1 else (splits * i * j * 4 + 255) // 256 * 256)
        if rest:
            assert splits == 1 and rest % 256 == 0 and 0 < rest < i and (rbi, rbj) in ((128, 64), (128, 128), (256, 256))
        if splits > 1:
            assert per % 2 == 0 or per == 1     # the kernel takes two blocks at a time


def test_few_rows_over_the_whole_range(plans):
    cases = [("v", 0, n, m, k) for n, m, k in accepted() if m <= 16] + [("v", 0, n, m, k) for n in (1, 15, 16, 17, 2048, 8192, 10000) for m in (1, 4, 5, 16) for k in (1, 128, 2048, 12288, 25088, 100000)]
    for (_, _, n, m, k), (rt, waves, splits, per, ws, *_rest) in zip(cases, plans(cases)):
        blocks = pitch(k) // 128
        assert (rt, waves) in ((4, 4), (2, 4), (2, 8), (1, 4), (1, 8), (1, 16))
        assert 1 <= splits <= 65535 and (splits - 1) * per < blocks <= splits * per
        assert ws == (0 if splits == 1 else splits * m * n * 4)


def test_more_rows_over_the_whole_range(plans):
    cases = [("w", t, n, m, k) for t in (0, 1, 2, 3) for n, m, k in accepted() if 16 < m <= 1024] + \
            [("w", 1, n, m, k) for n in (1, 100, 1000, 4096) for m in (17, 33, 100, 1024) for k in (1, 129, 640, 1025, 25088)]
    got = plans(cases)
    for (_, _, n, m, k), (rt, waves, splits, per, ws, *_rest) in zip(cases, got):
        blocks = pitch(k) // 128
        assert rt in (1, 2, 4) and waves == 4
        assert 1 <= splits <= 8 and (splits - 1) * per < blocks <= splits * per
        assert ws == (0 if splits == 1 else splits * m * n * 4)
    assert {g[0] for g in got} == {1, 2, 4} and any(g[2] > 1 for g in got)


def test_the_multiplied_sizes_take_every_tile(plans):
    """What the GPU tests multiply: every tile, in both forms, whole and split contractions, and a tile of their own for the last
    columns."""
    cases = [("g", e, *s) for e in (0, 1) for s in SIZES]
    got = plans(cases)
    for e in (0, 1):
        mine = [g for c, g in zip(cases, got) if c[1] == e]
        assert {(g[0], g[1]) for g in mine} == {(128, 64), (128, 128), (256, 256)}
        assert any(g[2] > 1 for g in mine) and any(g[2] == 1 for g in mine)
        assert any(g[4] > 0 for g in mine), e
