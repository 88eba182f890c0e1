"""kq_block_linear in tiles (more than 1024 rows, or products too large to go row by row of W), in every tile and kind of plan:
whole and split contractions, the last columns in a tile of their own; and that few rows and small products are exact.  The
sizes are those that tests/test_block_choice.py holds to their kernel.  Tolerances: those of tests/test_gpu_block_linear.py's
head.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from test_block_choice import FEW, LARGE_TILES, TILES
from test_gpu_block_linear import BF, DEV, F32, HF, TINY, U, acts, check, gen, hat, layer

kq = pytest.importorskip("paper_2003_05148_amd")
SPLIT = (1040, 200, 5000)


def strided(m, n, dtype):
    """A [m, n] view of odd strides in a larger matrix, and that matrix."""
    whole = torch.full((m + 1, n + 5), 7.0, dtype=dtype, device=DEV)
    return whole[:m, 3:3 + n], whole


def untouched(whole, m, n):
    return bool(torch.all(whole[:, :3] == 7) and torch.all(whole[:, 3 + n:] == 7) and torch.all(whole[m] == 7))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("m,n,k", TILES)
def test_linear(m, n, k, dtype):
    """Every output type, with and without a bias, from X and from its 8-bit values, into rows of their own and strided ones."""
    (values, exps), W = layer(n, k, m + n + k)
    X, bias = acts(m, k, dtype, m + k), torch.randn(n, generator=gen(5))
    wide = torch.full((m, k + 13), math.nan, dtype=dtype, device=DEV)
    wide[:, 5:5 + k] = X.to(DEV)
    x = kq.kq_quantize_blocks(X.to(DEV))
    Xh = hat(X, 1)
    for out in (BF, HF, F32):
        for b in (None, bias):
            on = None if b is None else b.to(DEV)
            y, whole = strided(m, n, out)
            kq.kq_block_linear(wide[:, 5:5 + k], values, exps, on, Y=y)
            check(y, Xh, W, k, out == F32, None if b is None else b.double())
            assert untouched(whole, m, n)
            assert torch.equal(kq.kq_block_linear(X.to(DEV), values, exps, on, dtype=out), y)
            assert torch.equal(kq.kq_block_linear(x[0], values, exps, on, x[1], dtype=out), y)
            y8, whole = strided(m, n, out)
            kq.kq_block_linear(x[0], values, exps, on, x[1], Y=y8)
            assert torch.equal(y8, y) and untouched(whole, m, n)


@pytest.mark.parametrize("out", [BF, HF, F32])
@pytest.mark.parametrize("m,n,k", LARGE_TILES)
def test_large_linear(m, n, k, out):
    """Tiles of 256 x 256, their last columns apart from them: the bias of those columns, 8-bit X, strided rows."""
    g = torch.Generator(device=DEV).manual_seed(m + n)
    W = torch.randn(n, k, device=DEV, generator=g) / math.sqrt(k) * torch.exp(0.5 * torch.randn(n, 1, device=DEV, generator=g))
    X = (torch.randn(m, k, device=DEV, generator=g) * torch.exp(0.5 * torch.randn(m, 1, device=DEV, generator=g))).to(BF)
    bias = torch.randn(n, device=DEV, generator=g)
    values, exps = kq.kq_quantize_blocks(W, rows=128)
    x = kq.kq_quantize_blocks(X)
    y, whole = strided(m, n, out)
    kq.kq_block_linear(x[0], values, exps, bias, x[1], Y=y)
    assert untouched(whole, m, n)
    a, b = kq.kq_reconstruct_blocks(*x, k).double(), kq.kq_reconstruct_blocks(values, exps, k, rows=128).double()
    y64, S = a @ b.t() + bias.double(), a.abs() @ b.abs().t() + bias.double().abs()
    exact = out == F32
    tol = U[out] * y64.abs() + ((k + 16) * 2.0 ** -24 + (0 if exact else 7 * 2.0 ** -13)) * S + TINY[out]
    err = (y.double() - y64).abs()
    assert torch.all(err <= tol), float((err - tol).max())
    rel = float(err.norm() / y64.norm())
    assert rel <= U[out] + 2.0 ** -18 + (0 if exact else 2.0 ** -14), rel
    assert torch.equal(kq.kq_block_linear(X, values, exps, bias, dtype=out), y)


@pytest.mark.parametrize("m,n,k", [(1030, 260, 300), SPLIT, (1200, 2050, 1300), (4353, 4500, 2200)])
def test_rows_do_not_touch_each_other(m, n, k):
    """A row of infinities, NaN or huge values leaves the others alone, the last row among those."""
    g = torch.Generator(device=DEV).manual_seed(m)
    values, exps = kq.kq_quantize_blocks(torch.randn(n, k, device=DEV, generator=g) / math.sqrt(k), rows=128)
    for dtype, row in ((BF, 1), (F32, 1), (BF, m - 1), (HF, m - 1)):
        X = torch.randn(m, k, device=DEV, generator=g).to(dtype)
        want = kq.kq_block_linear(X, values, exps)
        assert torch.all(torch.isfinite(want))
        for bad in (math.inf, math.nan, 3e38 if dtype != HF else 6e4):
            B = X.clone()
            B[row, k - 1] = bad
            got = kq.kq_block_linear(B, values, exps)
            keep = torch.arange(m, device=DEV) != row
            assert torch.equal(got[keep], want[keep])
            if not math.isfinite(bad):
                assert torch.all(torch.isnan(got[row]))
                x = kq.kq_quantize_blocks(B)
                assert torch.equal(kq.kq_block_linear(x[0], values, exps, x_exps=x[1], dtype=dtype)[keep], want[keep])


@pytest.mark.parametrize("m,n,k", [(1030, 300, 260), (1040, 300, 5000), (4353, 4500, 2200)])
def test_weight_blocks_of_nan(m, n, k):
    """A block of the weight with an infinity makes its 128 outputs NaN and no other: in the middle, and the last one."""
    for row in (140, n - 1):
        W = torch.randn(n, k, generator=gen(2))
        W[row, k - 2] = math.inf
        values, exps = kq.kq_quantize_blocks(W.to(DEV), rows=128)
        first, end = row // 128 * 128, min(row // 128 * 128 + 128, n)
        for dtype in (BF, HF, F32):
            Y = kq.kq_block_linear(acts(m, k, dtype, 1, 0.1).to(DEV), values, exps, torch.ones(n, device=DEV))
            nan = torch.isnan(Y)
            assert torch.all(nan[:, first:end]) and not torch.any(nan[:, :first]) and not torch.any(nan[:, end:])


@pytest.mark.parametrize("m,n,k", [(1030, 200, 256), (1040, 200, 5120), (1200, 2050, 1300)])
def test_exponent_255_is_nan_whatever_the_values(m, n, k):
    (values, exps), _ = layer(n, k, 1)
    x, xe = kq.kq_quantize_blocks(acts(m, k, BF, 1).to(DEV))
    for dtype in (BF, HF, F32):
        for block in (0, exps.shape[1] - 1):
            e = exps.clone()
            e[1, block] = 255
            Y = kq.kq_block_linear(x, values, e, x_exps=xe, dtype=dtype)
            assert torch.all(torch.isnan(Y[:, 128:256])) and not torch.any(torch.isnan(Y[:, :128])) and not torch.any(torch.isnan(Y[:, 256:]))
            e = xe.clone()
            e[m - 1, block] = 255
            Y = kq.kq_block_linear(x, values, exps, x_exps=e, dtype=dtype)
            assert torch.all(torch.isnan(Y[m - 1])) and not torch.any(torch.isnan(Y[:m - 1]))


@pytest.mark.parametrize("m,n,k", [(1030, 130, 256), SPLIT])
def test_extreme_scales(m, n, k):
    """Blocks near both ends of fp32's range whose products are ordinary."""
    for dtype in (F32, BF):
        W, X = torch.randn(n, k, generator=gen(1)), torch.randn(m, k, generator=gen(2)).to(dtype).float()
        for a, b in ((2.0 ** 120, 2.0 ** -110), (2.0 ** -100, 2.0 ** 105), (2.0 ** -60, 2.0 ** -55)):
            values, exps = kq.kq_quantize_blocks((W * a).to(DEV), rows=128)
            Xb = (X * b).to(dtype)
            check(kq.kq_block_linear(Xb.to(DEV), values, exps), hat(Xb, 1), hat(W * a, 128), k, dtype == F32)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_values_below_the_smallest_normal_number(dtype):
    """They may count as zero: no more than their terms are missing."""
    m, n, k = 1030, 130, 256
    for a, b in ((2.0 ** 100, 2.0 ** -130), (2.0 ** -132, 2.0 ** 110)):
        W, X = torch.randn(n, k, generator=gen(1)) * a, (torch.randn(m, k, generator=gen(2)) * b).to(dtype)
        q = kq.kq_quantize_blocks(W.to(DEV), rows=128)
        Wh, Xh = hat(W, 128), hat(X, 1)
        small = lambda x: torch.where(x.abs() < 2.0 ** -126, x.abs(), 0.0)
        lost = small(Xh) @ Wh.abs().t() + Xh.abs() @ small(Wh).t()
        S, y64 = Xh.abs() @ Wh.abs().t(), Xh @ Wh.t()
        tol = U[dtype] * (y64.abs() + lost) + ((k + 16) * 2.0 ** -24 + (0 if dtype == F32 else 7 * 2.0 ** -13)) * S + TINY[dtype] + lost
        for x, xe in ((X.to(DEV), None), kq.kq_quantize_blocks(X.to(DEV))):
            y = kq.kq_block_linear(x, *q, x_exps=xe, dtype=dtype).double().cpu()
            assert torch.all((y - y64).abs() <= tol)


def test_every_length_of_the_contraction():
    """One to ten blocks, whole and not, in tiles of 128 x 64 and of 128 x 128: where the products' loops begin and end."""
    for m, n in ((1030, 130), (1100, 1500)):
        g = torch.Generator(device=DEV).manual_seed(m)
        for k in [128 * s - 5 for s in range(1, 11)] + [256, 512, 1024]:
            values, exps = kq.kq_quantize_blocks(torch.randn(n, k, device=DEV, generator=g) / math.sqrt(k), rows=128)
            x = kq.kq_quantize_blocks(torch.randn(m, k, device=DEV, generator=g))
            a, b = kq.kq_reconstruct_blocks(*x, k).double(), kq.kq_reconstruct_blocks(values, exps, k, rows=128).double()
            y64, S = a @ b.t(), a.abs() @ b.abs().t()
            for out in (BF, HF, F32):
                y = kq.kq_block_linear(x[0], values, exps, x_exps=x[1], dtype=out).double()
                tol = U[out] * y64.abs() + ((k + 16) * 2.0 ** -24 + (0 if out == F32 else 7 * 2.0 ** -13)) * S + TINY[out]
                assert torch.all((y - y64).abs() <= tol), (m, n, k, out)


@pytest.mark.parametrize("m,n,k", [(1030, 260, 300), SPLIT, (4353, 4500, 2200)])
def test_streams_and_graphs(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m)
    values, exps = kq.kq_quantize_blocks(torch.randn(n, k, device=DEV, generator=g) / math.sqrt(k), rows=128)
    X, bias = torch.randn(m, k, device=DEV, generator=g).to(BF), torch.randn(n, device=DEV, generator=g)

    def step():
        x = kq.kq_quantize_blocks(X)
        return [kq.kq_block_linear(X, values, exps, bias), kq.kq_block_linear(x[0], values, exps, x_exps=x[1], dtype=F32)]
    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step()
    other = step()     # at the same time: each stream has its own scratch
    s.synchronize()
    for a, b, c in zip(want, got, other):
        assert torch.equal(a, b) and torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(4):
        X.copy_(torch.randn(m, k, device=DEV, generator=g))
        want = [t.clone() for t in step()]
        graph.replay()
        step()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_leading_sizes_layer_and_no_host_helper(monkeypatch):
    (values, exps), _ = layer(140, 300, 4)
    W, b = torch.randn(140, 300, generator=gen(1)) / 17, torch.randn(140, generator=gen(2))
    fc = kq.BlockLinear(W.to(DEV), b.to(DEV))
    X = acts(1200, 300, BF, 3).to(DEV)

    def calls():
        x = kq.kq_quantize_blocks(X)
        return [kq.kq_block_linear(X, values, exps), kq.kq_block_linear(X, values, exps, bias=b.to(DEV), dtype=HF),
                kq.kq_block_linear(x[0], values, exps, x_exps=x[1]), fc(X), fc.forward(X)[0]]
    want = calls()
    check(want[3], hat(X.cpu(), 1), hat(W, 128), 300, False, b.double())
    assert torch.equal(want[3], want[4])
    lead = X.view(3, 4, 100, 300)
    assert torch.equal(kq.kq_block_linear(lead, values, exps).view(1200, 140), want[0])
    assert torch.equal(fc(lead).view(1200, 140), want[3]) and torch.equal(fc.forward(lead)[0].view(1200, 140), want[3])
    monkeypatch.setattr(kq, "_fast", None)
    for a, c in zip(want, calls()):
        assert a.dtype == c.dtype and torch.equal(a, c)


# ---- few rows and small products ---------------------------------------------------------------------

@pytest.mark.parametrize("m,n,k", FEW)
def test_few_rows_and_small_products_are_exact(m, n, k):
    """Whatever X's and the output's type: the tolerance without the 8-bit matrix instruction's."""
    (values, exps), W = layer(n, k, m + n)
    bias = torch.randn(n, generator=gen(n))
    for dtype in (BF, HF, F32):
        X = acts(m, k, dtype, m)
        x, Xh = kq.kq_quantize_blocks(X.to(DEV)), hat(X, 1)
        for out in (BF, HF, F32):
            y = kq.kq_block_linear(X.to(DEV), values, exps, bias.to(DEV), dtype=out)
            check(y, Xh, W, k, True, bias.double())
            check(kq.kq_block_linear(x[0], values, exps, bias.to(DEV), x[1], dtype=out), Xh, W, k, True, bias.double())
