"""Which rows distillation cuts into segments, on the host (no GPU): those that need a workspace, for each segment's sums (12 bytes)
and the logits at the entries and the label.  tests/test_gpu_distill_segments.py computes CUT and WHOLE."""
import pytest

kq = pytest.importorskip("paper_2003_05148_amd")
F32, BF16, F16 = 0, 1, 2   # KQ_T_*
N = {F32: 4, BF16: 8, F16: 8}                    # logits of a chunk
LONG = {F32: 7500, BF16: 4096, F16: 4096}        # rows of more chunks are cut, if there are fewer than 128

# (m, v, type)
CUT = [(6, 40000, BF16), (5, 32777, F16), (1, 70001, BF16), (127, 32776, BF16), (6, 33001, F32), (3, 131071, F32), (100, 30004, F32)]
WHOLE = [(6, 32768, BF16), (5, 32767, F16), (128, 33000, BF16), (6, 29999, F32), (130, 40001, F32)]


def up(n, to):
    return -(-n // to) * to


def segments(m, v, kind):
    chunks = -(-v // N[kind])
    if m >= 128 or chunks <= LONG[kind]:
        return 1
    per = -(-chunks // min(-(-512 // m), -(-chunks // 512)))
    return -(-chunks // per)


def workspace(m, v, kind, top):
    s = segments(m, v, kind)
    return 0 if s == 1 else up(m * s * 12, 256) + up(m * (top + 1) * 4, 256)


def test_the_computed_sizes():
    for sizes, cut in ((CUT, True), (WHOLE, False)):
        for m, v, kind in sizes:
            assert (segments(m, v, kind) > 1) == cut, (m, v, kind)
            assert (kq.lib.kq_distill_workspace_bytes(kind, m, v, 20) > 0) == cut, (m, v, kind)
    assert {segments(*c) for c in CUT} >= {5, 18}     # as many as have 512 chunks each, and as many as make up 512 in all


@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_over_the_whole_range(kind):
    edge = LONG[kind] * N[kind]
    for v in (1, 1000, edge - 1, edge, edge + 1, edge + N[kind], 50001, 131072, 1 << 20, (1 << 24) - 1, 1 << 24):
        for m in (1, 2, 3, 16, 100, 126, 127, 128, 129, 2048):
            for top in (1, 256):
                assert kq.lib.kq_distill_workspace_bytes(kind, m, v, top) == workspace(m, v, kind, top), (m, v, top)
            s = segments(m, v, kind)
            assert m * s < 1 << 12 if s > 1 else True     # (about 512 workgroups of segments, at most one more a row)
