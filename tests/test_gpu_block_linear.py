"""Fully-connected layers in 8-bit floats with a power of two for each block of 128, on the GPU against plain forms in
64 bits.

Tolerances (set from the arithmetic).  u = torch.finfo(type).eps / 2, half a step of the output's type relative to the
value (bf16 has 8 significant bits: its steps in [1, 2) are 2^-7, and half of one is 2^-8; fp16 2^-11, fp32 2^-24), S = sum |a| |b| of a product's terms in 64 bits:
  * values, exponents and what they stand for: equal, bit for bit;
  * products that are summed exactly (fp32 outputs, up to 16 rows): |y - y64| <= u |y64| + (c + 16) 2^-24 S over c terms;
  * products on the 8-bit matrix instruction (other 16-bit outputs): it adds eight products at a time and cuts each off
    13 bits below the largest one's exponent, so the seven others are off by less than 2^-13 of it, and it is at most
    the eight's sum of magnitudes: 7 2^-13 S more;
  * for random operands in the 2-norm: ||y - y64|| <= (u + 2^-18) ||y64||, and 2^-14 ||y64|| more for the latter (errors
    of 2^-13 of the largest of eight products, independent: below 2^-15 of a typical result).
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_block_plan import SIZES

kq = pytest.importorskip("paper_2003_05148_amd")
DEV = torch.device("cuda:0")
BF, HF, F32, E4 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
U = {BF: 2.0 ** -8, HF: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF: 2.0 ** -134, HF: 2.0 ** -25, F32: 2.0 ** -126}   # half the smallest subnormal; fp32 sums may flush


def gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


# ---- the definition, block by block in 64 bits ---------------------------------------------------------

def quantize64(x, rows):
    """x (CPU, any type) -> (values in 64 bits [m, kp], exponent bytes, x_hat [m, k])."""
    x = x.double().numpy()
    m, k = x.shape
    kb, mb = -(-k // 128), -(-m // rows)
    v = np.zeros((m, kb * 128))
    exps = np.zeros((mb, kb), np.uint8)
    hat = np.zeros((m, k))
    for i in range(mb):
        for j in range(kb):
            r, c = slice(i * rows, min((i + 1) * rows, m)), slice(j * 128, min((j + 1) * 128, k))
            b = x[r, c]
            a = np.abs(b).max()
            if not np.isfinite(a):
                v[r, c], exps[i, j], hat[r, c] = np.nan, 255, np.nan
                continue
            e = -126
            if a > 0:
                E = math.frexp(a)[1] - 1
                e = max(E - 8 if a <= 1.75 * 2.0 ** E else E - 7, -126)
            s = np.ldexp(b, -e)
            step = np.ldexp(1.0, np.maximum(np.frexp(s)[1] - 4, -9))
            q = np.rint(s / step) * step
            v[r, c], exps[i, j], hat[r, c] = q, e + 127, np.ldexp(q, e)
    return torch.from_numpy(v), torch.from_numpy(exps), torch.from_numpy(hat)


def hat(x, rows):
    return quantize64(x, rows)[2]


def acts(m, k, dtype, seed, spread=1.0):
    x = torch.randn(m, k, generator=gen(seed)) * torch.exp(spread * torch.randn(m, 1, generator=gen(seed + 1)))
    return x.to(dtype)


def layer(n, k, seed):
    """A weight on the GPU and its exact values."""
    W = torch.randn(n, k, generator=gen(seed)) / math.sqrt(k) * torch.exp(torch.randn(n, 1, generator=gen(seed + 7)))
    return kq.kq_quantize_blocks(W.to(DEV), rows=128), hat(W, 128)


def check(y, a, b, terms, exact, bias=None):
    """y against a @ b.T (+ bias) in 64 bits within the tolerances of this file's head."""
    dtype = y.dtype
    y = y.double().cpu()
    y64 = a @ b.t()
    S = a.abs() @ b.abs().t()
    if bias is not None:
        y64, S = y64 + bias, S + bias.abs()
    u = U[dtype]
    tol = u * y64.abs() + (terms + 16) * 2.0 ** -24 * S + TINY[dtype]
    if not exact:
        tol = tol + 7 * 2.0 ** -13 * S
    err = (y - y64).abs()
    assert torch.all(err <= tol), float((err - tol).max())
    if y64.numel() >= 64:
        rel = float(err.norm() / y64.norm())
        assert rel <= u + 2.0 ** -18 + (0 if exact else 2.0 ** -14), rel


# ---- quantizer ---------------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("m,k", [(1, 1), (3, 7), (2, 127), (129, 128), (5, 129), (128, 300), (257, 1000)])
def test_quantizer(rows, dtype, m, k):
    X = acts(m, k, dtype, 10 * m + k, 2.0)
    values, exps = kq.kq_quantize_blocks(X.to(DEV), rows=rows)
    v, e, h = quantize64(X, rows)
    assert values.dtype == E4 and tuple(values.shape) == tuple(v.shape)
    assert torch.equal(exps.cpu(), e)
    assert torch.equal(values.float().double().cpu(), v)
    for out in (F32, BF, HF):
        r = kq.kq_reconstruct_blocks(values, exps, k, rows=rows, dtype=out)
        assert torch.equal(r.cpu(), h.to(F32).to(out))


@pytest.mark.parametrize("rows", [1, 128])
def test_quantizer_every_rounding(rows):
    """All magnitudes an e4m3 number can be rounded from: numbers, midpoints and their fp32 neighbours, both signs."""
    grid = torch.arange(0, 127, dtype=torch.uint8).view(E4).float()
    mid = (grid[1:] + grid[:-1]) / 2
    inf = torch.full((), math.inf)
    pts = torch.cat([grid, mid, torch.nextafter(mid, inf), torch.nextafter(mid, -inf), torch.nextafter(grid[1:], -inf)])
    pts = torch.cat([pts, -pts])
    pts = torch.nn.functional.pad(pts, (0, -len(pts) % 127)).view(-1, 127)
    pts = torch.cat([torch.full((len(pts), 1), 448.0), pts], 1)   # every block's largest is 448
    for shift in (-100, -20, 0, 1, 90):
        X = torch.ldexp(pts, torch.tensor(shift))
        values, exps = kq.kq_quantize_blocks(X.to(DEV), rows=rows)
        v, e, _ = quantize64(X, rows)
        assert torch.equal(exps.cpu(), e) and torch.equal(values.float().double().cpu(), v)


@pytest.mark.parametrize("rows", [1, 128])
def test_quantizer_borders(rows):
    """The exponent at 1.75 of a power of two, at the smallest and largest magnitudes, blocks of zeros, infinities and NaN."""
    f = np.float32
    cases = [f(1.75), np.nextafter(f(1.75), f(2)), f(2), np.nextafter(f(2), f(0)), f(1), f(3.4028235e38), f(2.0 ** -126),
             f(2.0 ** -149), f(2.0 ** -118), np.nextafter(f(2.0 ** -118), f(1)), f(1.75 * 2.0 ** -118), f(0), f(-0.0),
             f(np.inf), f(-np.inf), f(np.nan), f(2.0 ** -130)]
    X = torch.randn(128, 128 * len(cases), generator=gen(1))
    for i, a in enumerate(cases):
        b = X[:, 128 * i:128 * i + 128]
        top = b.abs().max(1, keepdim=True).values if rows == 1 else b.abs().max()
        b *= 0 if not np.isfinite(a) else (torch.tensor(float(a), dtype=torch.float64) / top / 1.0001).float()
        b[:, 17 + i % 3] = float(a)
    values, exps = kq.kq_quantize_blocks(X.to(DEV), rows=rows)
    v, e, h = quantize64(X, rows)
    assert torch.equal(exps.cpu(), e)
    assert np.array_equal(values.float().double().cpu().numpy(), v.numpy(), equal_nan=True)
    r = kq.kq_reconstruct_blocks(values, exps, X.shape[1], rows=rows)
    assert np.array_equal(r.cpu().numpy(), h.float().numpy(), equal_nan=True)


def test_quantizer_strides_shapes_and_given_outputs():
    big = acts(40, 700, BF, 3).to(DEV)
    for view in (big[:, 5:305], big[::3, 1:301], big.view(4, 10, 700)[1], big[3]):
        values, exps = kq.kq_quantize_blocks(view)
        x = view.cpu().reshape(-1, view.shape[-1])
        v, e, h = quantize64(x, 1)
        assert torch.equal(exps.cpu(), e) and torch.equal(values.float().double().cpu(), v)
        out = torch.full((x.shape[0], x.shape[1] + 9), 7.0, device=DEV)
        kq.kq_reconstruct_blocks(values, exps, x.shape[1], X_hat=out[:, 4:4 + x.shape[1]])
        assert torch.equal(out[:, 4:4 + x.shape[1]].cpu().double(), h)
        assert torch.all(out[:, :4] == 7) and torch.all(out[:, 4 + x.shape[1]:] == 7)
        values.view(torch.uint8).fill_(9)
        exps.fill_(9)
        r = kq.kq_quantize_blocks(view, values=values, exps=exps)
        assert r[0] is values and torch.equal(exps.cpu(), e) and torch.equal(values.float().double().cpu(), v)
    values, exps = kq.kq_quantize_blocks(big[:0])
    assert values.shape == (0, 768) and exps.shape == (0, 6)


# ---- the product ---------------------------------------------------------------------------------

LINEAR = [(1, 1, 1), (1, 16, 128), (1, 1000, 512), (2, 5, 7), (3, 130, 127), (7, 100, 129), (15, 300, 300), (16, 129, 1000),
          (16, 33, 9000), (17, 1, 1), (17, 129, 130), (32, 100, 128), (33, 5, 300), (64, 256, 1000), (100, 130, 2100),
          (128, 128, 256), (129, 257, 127), (257, 300, 385), (300, 700, 640), (520, 1030, 129)]


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("m,n,k", LINEAR)
def test_linear(m, n, k, dtype):
    (values, exps), W = layer(n, k, m + n + k)
    X = acts(m, k, dtype, m * k)
    bias = torch.randn(n, generator=gen(5)) if (m + n) % 2 else None
    Y = kq.kq_block_linear(X.to(DEV), values, exps, bias=None if bias is None else bias.to(DEV))
    assert Y.dtype == dtype and Y.shape == (m, n)
    check(Y, hat(X, 1), W, k, dtype == F32 or m <= 16, None if bias is None else bias.double())


@pytest.mark.parametrize("m,n,k", [(17, 1000, 512), (64, 1000, 4000), (100, 200, 1000), (130, 1000, 300), (1000, 60, 900), (1024, 1, 1), (300, 17, 5000)])
def test_small_products_of_many_rows(m, n, k):
    """Sixteens of rows without a launch for the quantizer: exact products whatever the output's type, with strided rows, a
    bias and quantized rows too."""
    (values, exps), W = layer(n, k, m + n)
    X, bias = acts(m, k, BF, m), torch.randn(n, generator=gen(n))
    wide = torch.full((m, k + 13), math.nan, dtype=BF, device=DEV)
    wide[:, 5:5 + k] = X.to(DEV)
    for dtype in (BF, HF, F32):
        Y = torch.full((m + 1, n + 3), 7.0, dtype=dtype, device=DEV)
        kq.kq_block_linear(wide[:, 5:5 + k], values, exps, bias.to(DEV), Y=Y[:m, 2:2 + n])
        check(Y[:m, 2:2 + n], hat(X, 1), W, k, dtype == F32, bias.double())
        assert torch.all(Y[:, :2] == 7) and torch.all(Y[:, 2 + n:] == 7) and torch.all(Y[m] == 7)
    q = kq.kq_quantize_blocks(X.to(DEV))
    Y = kq.kq_block_linear(q[0], values, exps, bias.to(DEV), q[1])
    check(Y, hat(X, 1), W, k, False, bias.double())


@pytest.mark.parametrize("out", [BF, HF, F32])
@pytest.mark.parametrize("m,n,k", [(1, 100, 300), (13, 129, 512), (40, 130, 130), (300, 260, 700)])
def test_linear_of_quantized_rows(m, n, k, out):
    """8-bit values give what X gives that they were made from, bit for bit where the output's type is the same."""
    (values, exps), W = layer(n, k, m)
    X = acts(m, k, BF, m + 1)
    x = kq.kq_quantize_blocks(X.to(DEV))
    Y = kq.kq_block_linear(x[0], values, exps, x_exps=x[1], dtype=out)
    check(Y, hat(X, 1), W, k, out == F32 or m <= 16)
    assert torch.equal(Y, kq.kq_block_linear(X.to(DEV), values, exps, dtype=out))


def test_linear_rows_do_not_touch_each_other():
    """A row of infinities, NaN or huge values leaves the others alone, in every kernel."""
    for m in (2, 16, 40, 300):
        for dtype in (BF, F32):
            (values, exps), _ = layer(200, 300, m)
            X = acts(m, 300, dtype, m).to(DEV)
            want = kq.kq_block_linear(X, values, exps)
            for bad in (math.inf, math.nan, 3e38):
                B = X.clone()
                B[1, 77] = bad
                got = kq.kq_block_linear(B, values, exps)
                keep = torch.arange(m, device=DEV) != 1
                assert torch.equal(got[keep], want[keep])
                if bad != 3e38:
                    assert torch.all(torch.isnan(got[1]))


def test_linear_weight_blocks_of_nan():
    """A block of the weight with an infinity makes its 128 outputs NaN and no other."""
    W = torch.randn(300, 260, generator=gen(2))
    W[140, 200] = math.inf
    values, exps = kq.kq_quantize_blocks(W.to(DEV), rows=128)
    for m in (3, 50):
        Y = kq.kq_block_linear(acts(m, 260, BF, 1).to(DEV), values, exps)
        nan = torch.isnan(Y)
        assert torch.all(nan[:, 128:256]) and not torch.any(nan[:, :128]) and not torch.any(nan[:, 256:])


def test_exponent_255_is_nan_whatever_the_values():
    for m, dtype in ((3, BF), (50, BF), (50, F32)):
        (values, exps), _ = layer(200, 256, 1)
        e = exps.clone()
        e[1, 1] = 255
        Y = kq.kq_block_linear(acts(m, 256, dtype, 1).to(DEV), values, e)
        assert torch.all(torch.isnan(Y[:, 128:])) and not torch.any(torch.isnan(Y[:, :128]))
        x, xe = kq.kq_quantize_blocks(acts(m, 256, dtype, 1).to(DEV))
        xe[1, 0] = 255
        Y = kq.kq_block_linear(x, values, exps, x_exps=xe, dtype=dtype)
        assert torch.all(torch.isnan(Y[1])) and not torch.any(torch.isnan(Y[0]))


def test_linear_extreme_scales():
    """Blocks near both ends of fp32's range whose products are ordinary."""
    for m, dtype in ((5, F32), (40, F32), (5, BF), (40, BF)):
        W, X = torch.randn(130, 256, generator=gen(1)), torch.randn(m, 256, generator=gen(2)).to(dtype).float()
        for a, b in ((2.0 ** 120, 2.0 ** -110), (2.0 ** -100, 2.0 ** 105), (2.0 ** -60, 2.0 ** -55)):
            values, exps = kq.kq_quantize_blocks((W * a).to(DEV), rows=128)
            Y = kq.kq_block_linear((X * b).to(dtype).to(DEV), values, exps)
            check(Y, hat((X * b).to(dtype), 1), hat(W * a, 128), 256, dtype == F32 or m <= 16)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_values_below_the_smallest_normal_number(dtype):
    """Blocks whose values are around and below 2^-126 meet large ones.  Values below it may count as zero: no more than
    their terms are missing."""
    n, k = 130, 256

    def near(y, a, b, terms, exact):
        small = lambda x: torch.where(x.abs() < 2.0 ** -126, x.abs(), 0.0)
        lost = small(a) @ b.abs().t() + a.abs() @ small(b).t()
        S, y64, y = a.abs() @ b.abs().t(), a @ b.t(), y.double().cpu()
        tol = U[dtype] * (y64.abs() + lost) + ((terms + 16) * 2.0 ** -24 + (0 if exact else 7 * 2.0 ** -13)) * S + TINY[dtype]
        assert torch.all((y - y64).abs() <= tol + lost)

    for m in (5, 40):
        for a, b in ((2.0 ** 100, 2.0 ** -130), (2.0 ** -132, 2.0 ** 110)):
            W, X = torch.randn(n, k, generator=gen(1)) * a, (torch.randn(m, k, generator=gen(2)) * b).to(dtype)
            q = kq.kq_quantize_blocks(W.to(DEV), rows=128)
            Wh, Xh = hat(W, 128), hat(X, 1)
            for x, xe in ((X.to(DEV), None), kq.kq_quantize_blocks(X.to(DEV))):
                near(kq.kq_block_linear(x, *q, x_exps=xe, dtype=dtype), Xh, Wh, k, dtype == F32 or m <= 16)
            dY = (torch.randn(m, n, generator=gen(3)) * (2.0 ** -30 / b)).to(dtype)   # (1 / b alone is past fp32)
            x = kq.kq_quantize_blocks(X.to(DEV))
            dW, _ = kq.kq_block_linear_grad_weight(dY.to(DEV), *x, k, dtype=dtype)
            near(dW, hat(dY.double().t().contiguous(), 1), hat(Xh.t().contiguous(), 1), m, dtype == F32)


def test_linear_strides_leading_sizes_and_outputs():
    (values, exps), W = layer(100, 300, 4)
    big = acts(60, 700, BF, 3).to(DEV)
    for m in (9, 30):
        X = big[:m, 3:303]
        want = kq.kq_block_linear(X.contiguous(), values, exps)
        out = torch.full((m + 2, 140), 7.0, dtype=BF, device=DEV)
        got = kq.kq_block_linear(X, values, exps, Y=out[1:m + 1, 3:103])
        assert torch.equal(got, want) and got.data_ptr() == out[1:, 3:].data_ptr()
        assert torch.all(out[0] == 7) and torch.all(out[m + 1] == 7) and torch.all(out[:, :3] == 7) and torch.all(out[:, 103:] == 7)
        lead = X.contiguous().view(3, m // 3, 300)
        assert torch.equal(kq.kq_block_linear(lead, values, exps).view(m, 100), want)
    assert torch.equal(kq.kq_block_linear(big[0, :300], values, exps), kq.kq_block_linear(big[:1, :300], values, exps)[0])
    assert kq.kq_block_linear(big[:0, :300], values, exps).shape == (0, 100)


# ---- the gradients ---------------------------------------------------------------------------------

GRADS = [(1, 1, 1), (1, 300, 200), (5, 7, 129), (17, 128, 128), (37, 100, 300), (128, 129, 127), (130, 257, 300), (300, 520, 640)]


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("m,n,k", GRADS)
def test_grad_input(m, n, k, dtype):
    (values, exps), W = layer(n, k, m + n + k)
    dY = (0.01 * acts(m, n, F32, m * n)).to(dtype)
    dX = kq.kq_block_linear_grad_input(dY.to(DEV), values, exps, k)
    assert dX.dtype == dtype
    check(dX, hat(dY, 1), W.t(), n, dtype == F32)


@pytest.mark.parametrize("n,k", [(130, 300), (257, 130), (300, 700), (1, 1)])
def test_input_gradient_of_weight_blocks_of_nan(n, k):
    """A block of the last, partial rows of W that is NaN: its columns of dX, and no other."""
    for m, dtype in ((3, BF), (300, HF), (40, F32)):
        W = torch.randn(n, k, generator=gen(n)) / math.sqrt(k)
        W[n - 1, 0] = math.nan
        values, exps = kq.kq_quantize_blocks(W.to(DEV), rows=128)
        dY = (0.01 * acts(m, n, F32, k)).to(dtype)
        dX = kq.kq_block_linear_grad_input(dY.to(DEV), values, exps, k)
        assert torch.all(torch.isnan(dX[:, :128]))
        if k > 128:
            W[n - 1, 0] = 0.0
            check(dX[:, 128:], hat(dY, 1), hat(W, 128).t().contiguous()[128:], n, dtype == F32)


@pytest.mark.parametrize("m", [64 * 128, 64 * 128 + 1, 70 * 128, 95 * 128 + 5, 128 * 128])
def test_bias_gradient_of_many_rows(m):
    """Sums over 128 rows are added in groups above 64 of them, and the rest of them alone: within the tolerance of m terms."""
    n, k = 5, 130
    dY, x = acts(m, n, BF, m), kq.kq_quantize_blocks(acts(m, k, BF, 1).to(DEV))
    _, db = kq.kq_block_linear_grad_weight(dY.to(DEV), *x, k, True)
    d = dY.double()
    assert torch.all((db.double().cpu() - d.sum(0)).abs() <= (m + 16) * 2.0 ** -24 * d.abs().sum(0))
    ones = torch.ones(m, n, dtype=BF, device=DEV)
    assert torch.all(kq.kq_block_linear_grad_weight(ones, *x, k, True)[1] == m)     # (each sum of integers is exact)


@pytest.mark.parametrize("out", [F32, BF, HF])
@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("m,n,k", GRADS)
def test_grad_weight(m, n, k, dtype, out):
    X = acts(m, k, BF, m * k)
    dY = (0.01 * acts(m, n, F32, m * n)).to(dtype)
    x = kq.kq_quantize_blocks(X.to(DEV))
    dW, db = kq.kq_block_linear_grad_weight(dY.to(DEV), *x, k, bias=True, dtype=out)
    assert dW.dtype == out
    check(dW, hat(dY.t().contiguous(), 1), hat(hat(X, 1).t().contiguous(), 1), m, out == F32)
    d = dY.double()
    assert torch.all((db.double().cpu() - d.sum(0)).abs() <= (m + 1) * 2.0 ** -24 * d.abs().sum(0))
    again, none = kq.kq_block_linear_grad_weight(dY.to(DEV), *x, k, dtype=out)
    assert none is None and torch.equal(again, dW)


def test_gradients_against_differences():
    """The layer's loss sum(Y * R) in 64 bits with the operands as they are after quantization: its differences along
    random directions are the gradients' products with them."""
    m, n, k = 130, 140, 150
    (values, exps), W = layer(n, k, 1)
    X, R = acts(m, k, BF, 2), (0.01 * acts(m, n, F32, 3)).to(BF)
    x = kq.kq_quantize_blocks(X.to(DEV))
    dX = kq.kq_block_linear_grad_input(R.to(F32).to(DEV), values, exps, k).double().cpu()
    dW = kq.kq_block_linear_grad_weight(R.to(DEV), *x, k)[0].double().cpu()

    def loss(x64, w64, r64):
        return float((r64 * (x64 @ w64.t())).sum())
    Xh, Rr, Rc = hat(X, 1), hat(R, 1), hat(R.t().contiguous(), 1).t()
    Xc = hat(Xh.t().contiguous(), 1).t()
    for seed in range(3):
        D, E = torch.randn(m, k, generator=gen(seed)).double(), torch.randn(n, k, generator=gen(seed + 9)).double()
        h = 2.0 ** -10
        num = (loss(Xh + h * D, W, Rr) - loss(Xh - h * D, W, Rr)) / (2 * h)
        assert abs(num - float((dX * D).sum())) <= 2.0 ** -18 * float((Rr.abs() @ W.abs() * D.abs()).sum())
        num = (loss(Xc, W + h * E, Rc) - loss(Xc, W - h * E, Rc)) / (2 * h)
        assert abs(num - float((dW * E).sum())) <= 2.0 ** -18 * float((Rc.abs().t() @ Xc.abs() * E.abs()).sum())


def test_gradients_of_no_rows_and_bad_rows():
    (values, exps), _ = layer(100, 200, 1)
    dY, X = torch.zeros(0, 100, dtype=BF, device=DEV), torch.zeros(0, 200, dtype=BF, device=DEV)
    assert kq.kq_block_linear_grad_input(dY, values, exps, 200).shape == (0, 200)
    dW, db = kq.kq_block_linear_grad_weight(dY, *kq.kq_quantize_blocks(X), 200, bias=True)
    assert dW.shape == (100, 200) and torch.all(dW == 0) and torch.all(db == 0)
    for out in (F32, BF):
        dY, X = (0.01 * acts(150, 100, BF, 1)).to(DEV), acts(150, 200, BF, 2).to(DEV)
        dY[3, 7], X[140, 9] = math.inf, math.nan     # a NaN in a row of X makes its whole block of 128 columns NaN
        dW, db = kq.kq_block_linear_grad_weight(dY, *kq.kq_quantize_blocks(X), 200, bias=True, dtype=out)
        nan = torch.isnan(dW)
        want = torch.zeros_like(nan)
        want[7], want[:, :128] = True, True
        assert torch.equal(nan, want)
        assert not torch.isfinite(db[7]) and torch.all(torch.isfinite(db[:7]))
    dX = kq.kq_block_linear_grad_input(dY, values, exps, 200)
    assert torch.all(torch.isnan(dX[3])) and torch.all(torch.isfinite(dX[4:]))


def test_gradients_strides_and_outputs():
    m, n, k = 70, 90, 200
    (values, exps), _ = layer(n, k, 1)
    big = (0.01 * acts(m, 300, BF, 1)).to(DEV)
    dY = big[:, 7:7 + n]
    out = torch.full((m, k + 20), 3.0, dtype=BF, device=DEV)
    got = kq.kq_block_linear_grad_input(dY, values, exps, k, dX=out[:, 11:11 + k])
    assert torch.equal(got, kq.kq_block_linear_grad_input(dY.contiguous(), values, exps, k))
    assert torch.all(out[:, :11] == 3) and torch.all(out[:, 11 + k:] == 3)
    x = kq.kq_quantize_blocks(acts(m, k, HF, 2).to(DEV))
    for dtype in (F32, HF):
        out = torch.full((n + 1, k + 20), 3.0, dtype=dtype, device=DEV)
        db = torch.empty(n, device=DEV)
        got, db2 = kq.kq_block_linear_grad_weight(dY, *x, k, dW=out[:n, 11:11 + k], dbias=db)
        want, db3 = kq.kq_block_linear_grad_weight(dY.contiguous(), *x, k, bias=True, dtype=dtype)
        assert torch.equal(got, want) and torch.equal(db2, db3) and db2 is db
        assert torch.all(out[:, :11] == 3) and torch.all(out[:, 11 + k:] == 3) and torch.all(out[n] == 3)


def again(x):
    """x (GPU) as it is after quantization in blocks of one row, in 64 bits (the quantizer itself is tested above)."""
    return kq.kq_reconstruct_blocks(*kq.kq_quantize_blocks(x.contiguous()), x.shape[1]).double()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i,j,c", SIZES)
def test_every_tile(i, j, c, dtype):
    """Sizes of every tile and kind of plan, odd at every edge: the product and both gradients against 64 bits on the GPU."""
    g = torch.Generator(device=DEV).manual_seed(i + j + c)

    def randn(a, b, spread=0.5):
        return torch.randn(a, b, device=DEV, generator=g) * torch.exp(spread * torch.randn(a, 1, device=DEV, generator=g))

    def check_gpu(y, a, b):
        y64, S = a @ b.t(), a.abs() @ b.abs().t()
        u, exact = U[y.dtype], y.dtype == F32
        tol = u * y64.abs() + (c + 16) * 2.0 ** -24 * S + TINY[y.dtype] + (0 if exact else 7 * 2.0 ** -13) * S
        err = (y.double() - y64).abs()
        assert torch.all(err <= tol), float((err - tol).max())
        rel = float(err.norm() / y64.norm())
        assert rel <= u + 2.0 ** -18 + (0 if exact else 2.0 ** -14), rel

    W, X = randn(i, c) / math.sqrt(c), randn(j, c).to(dtype)
    values, exps = kq.kq_quantize_blocks(W, rows=128)
    check_gpu(kq.kq_block_linear(X, values, exps), again(X), kq.kq_reconstruct_blocks(values, exps, c, rows=128).double())
    W, dY = randn(c, i) / math.sqrt(c), (0.01 * randn(j, c)).to(dtype)
    values, exps = kq.kq_quantize_blocks(W, rows=128)
    check_gpu(kq.kq_block_linear_grad_input(dY, values, exps, i), again(dY),
              kq.kq_reconstruct_blocks(values, exps, i, rows=128).double().t())
    x, dY = kq.kq_quantize_blocks(randn(c, i).to(BF)), (0.01 * randn(c, j)).to(BF)
    dW, db = kq.kq_block_linear_grad_weight(dY, *x, i, bias=True, dtype=dtype)
    check_gpu(dW, again(dY.t()), again(kq.kq_reconstruct_blocks(*x, i).t()))
    d = dY.double()
    assert torch.all((db.double() - d.sum(0)).abs() <= (c + 1) * 2.0 ** -24 * d.abs().sum(0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i,j", [(130, 70), (1500, 1000), (2050, 1030)])
def test_every_length_of_the_contraction(i, j, dtype):
    """One to ten blocks, whole and not: where the products' loops begin and end."""
    g = torch.Generator(device=DEV).manual_seed(i)
    for c in [128 * s - 5 for s in range(1, 11)] + [256, 512, 1024]:
        W = torch.randn(c, i, device=DEV, generator=g) / math.sqrt(c)
        dY = (0.01 * torch.randn(j, c, device=DEV, generator=g)).to(dtype)
        values, exps = kq.kq_quantize_blocks(W, rows=128)
        a, b = again(dY), kq.kq_reconstruct_blocks(values, exps, i, rows=128).double().t()
        dX = kq.kq_block_linear_grad_input(dY, values, exps, i)
        y64, S = a @ b.t(), a.abs() @ b.abs().t()
        tol = U[dtype] * y64.abs() + ((c + 16) * 2.0 ** -24 + (0 if dtype == F32 else 7 * 2.0 ** -13)) * S + TINY[dtype]
        assert torch.all((dX.double() - y64).abs() <= tol), c
        x = kq.kq_quantize_blocks(torch.randn(c, i, device=DEV, generator=g).to(BF))
        dW, _ = kq.kq_block_linear_grad_weight(dY.t().contiguous(), *x, i, dtype=dtype)
        a, b = again(dY), again(kq.kq_reconstruct_blocks(*x, i).t())
        y64, S = a @ b.t(), a.abs() @ b.abs().t()
        tol = U[dtype] * y64.abs() + ((c + 16) * 2.0 ** -24 + (0 if dtype == F32 else 7 * 2.0 ** -13)) * S + TINY[dtype]
        assert torch.all((dW.double() - y64).abs() <= tol), c


# ---- how the calls run ---------------------------------------------------------------------------------

def test_same_bits_every_time_and_on_another_stream():
    (values, exps), _ = layer(1000, 4000, 1)
    W2 = torch.randn(64, 64, device=DEV)
    for m in (1, 16, 40, 400):
        X = acts(m, 4000, BF, m).to(DEV)
        x = kq.kq_quantize_blocks(X)
        dY = (0.01 * acts(m, 1000, BF, m)).to(DEV)

        def all_calls():
            return [kq.kq_block_linear(X, values, exps), kq.kq_block_linear_grad_input(dY, values, exps, 4000),
                    kq.kq_block_linear_grad_weight(dY, *x, 4000, bias=True)[0],
                    kq.kq_block_linear_grad_weight(dY, *x, 4000, dtype=BF)[0]]
        want = all_calls()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got = all_calls()
            W2 @ W2
        other = all_calls()     # at the same time: each stream has its own scratch
        s.synchronize()
        for a, b, c in zip(want, got, other):
            assert torch.equal(a, b) and torch.equal(a, c)


def test_captured_and_replayed():
    n, k = 300, 520
    (values, exps), _ = layer(n, k, 1)
    for m in (3, 50):
        X = acts(m, k, BF, 1).to(DEV)
        dY = (0.01 * acts(m, n, BF, 2)).to(DEV)

        def step():
            x = kq.kq_quantize_blocks(X)
            Y = kq.kq_block_linear(x[0], values, exps, x_exps=x[1])
            return [Y, kq.kq_block_linear(X, values, exps), kq.kq_block_linear_grad_input(dY, values, exps, k),
                    *kq.kq_block_linear_grad_weight(dY, *x, k, bias=True)]
        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        for seed in range(4):
            X.copy_(acts(m, k, BF, seed))
            dY.copy_(0.01 * acts(m, n, BF, seed + 50))
            want = [t.clone() for t in step()]
            g.replay()
            step()          # eager work beside the replay
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b)


def test_without_the_host_helper(monkeypatch):
    """The binding's own checks and calls give what the C++ helper's plain case gives."""
    (values, exps), _ = layer(300, 600, 1)
    X, dY = acts(40, 600, BF, 1).to(DEV), (0.01 * acts(40, 300, BF, 2)).to(DEV)
    bias = torch.randn(300, device=DEV)

    def calls():
        x = kq.kq_quantize_blocks(X)
        return [x[0].view(torch.uint8), x[1], kq.kq_reconstruct_blocks(*x, 600, dtype=HF), kq.kq_block_linear(X, values, exps, bias=bias),
                kq.kq_block_linear(X[:3], values, exps, dtype=F32), kq.kq_block_linear(x[0], values, exps, x_exps=x[1], dtype=HF),
                kq.kq_block_linear_grad_input(dY, values, exps, 600), *kq.kq_block_linear_grad_weight(dY, *x, 600, bias=True, dtype=BF)]
    want = calls()
    monkeypatch.setattr(kq, "_fast", None)
    for a, b in zip(want, calls()):
        assert a.dtype == b.dtype and torch.equal(a, b)


def test_given_workspace():
    (values, exps), _ = layer(300, 600, 1)
    X = acts(1100, 600, BF, 1).to(DEV)
    nb = kq.lib.kq_block_linear_workspace_bytes(kq.KQ_T_BF16, kq.KQ_T_BF16, 1100, 300, 600)
    ws = torch.full((nb + 256,), 255, dtype=torch.uint8, device=DEV)
    assert torch.equal(kq.kq_block_linear(X, values, exps, workspace=ws), kq.kq_block_linear(X, values, exps))
    assert torch.all(ws[nb:] == 255)
    with pytest.raises(kq.KqError):
        kq.kq_block_linear(X, values, exps, workspace=ws[:nb - 1])


def test_offsets_past_32_bits():
    """A weight of more than 2^32 values and rows of X far apart: the last rows against 64 bits."""
    n, k = 33000, 131200
    values = torch.randint(0, 256, (n * (k // 64),), device=DEV, dtype=torch.uint8).repeat_interleave(64).view(n, k)
    values &= 0xb7          # no NaN, magnitudes up to 15
    values = values.view(E4)
    exps = torch.randint(120, 130, (-(-n // 128), k // 128), device=DEV, dtype=torch.uint8)
    W = values[-3:].float().double() * torch.exp2(exps[-1].double() - 127).repeat_interleave(128)
    for m in (2, 20):
        far = torch.empty(m, 1 << 26, dtype=BF, device=DEV)    # 2^27 bytes a row
        X = far[:, 5:5 + k]
        X.copy_(acts(m, k, BF, m))
        Y = kq.kq_block_linear(X, values, exps)
        check(Y[:, -3:], hat(X.cpu(), 1), W.cpu(), k, m <= 16)
        del far
    dY = torch.zeros(20, n, dtype=F32, device=DEV)
    dY[:, -3:] = acts(20, 3, F32, 1).to(DEV)
    dX = kq.kq_block_linear_grad_input(dY, values, exps, k)
    h = hat(dY[:, 32896:].cpu(), 1)
    check(dX, h[:, -3:], W.cpu().t().contiguous()[:k], 3, True)


# ---- the layer ---------------------------------------------------------------------------------

def test_layer_trains():
    """forward, backward and step against the same arithmetic from the single calls."""
    W, b = torch.randn(140, 300, generator=gen(1)) / 17, torch.randn(140, generator=gen(2))
    fc = kq.BlockLinear(W.to(DEV), b.to(DEV), master=True)
    assert torch.equal(fc.weight().cpu().double(), hat(W, 128))
    X = acts(60, 300, BF, 3).to(DEV).view(6, 10, 300)
    Y, kept = fc.forward(X)
    assert Y.shape == (6, 10, 140) and torch.equal(Y, fc(X))
    dY = (0.01 * acts(60, 140, BF, 4)).to(DEV).view(6, 10, 140)
    dX, dW, db = fc.backward(dY, kept)
    assert dX.shape == X.shape and dW.dtype == F32
    fc.step(dW, db, 0.5)
    want = W - 0.5 * dW.cpu()
    assert torch.equal(fc.master.cpu(), want) and torch.equal(fc.weight().cpu().double(), hat(want, 128))
    assert torch.equal(fc.bias.cpu(), b - 0.5 * db.cpu())
    assert fc.backward(dY, kept, input_grad=False)[0] is None
    with pytest.raises(ValueError):
        kq.BlockLinear(W.to(DEV)).step(dW, None, 0.5)


# ---- refusals ---------------------------------------------------------------------------------

def test_layer_of_parameters():
    """A layer made from a network's parameters keeps no graph, and its steps build none."""
    W = torch.nn.Parameter(torch.randn(130, 200, device=DEV))
    b = torch.nn.Parameter(torch.randn(130, device=DEV))
    fc = kq.BlockLinear(W, b, master=True)
    X = torch.randn(9, 200, device=DEV, dtype=BF, requires_grad=True)
    Y, kept = fc.forward(X)
    fc.step(*fc.backward(torch.ones_like(Y), kept)[1:], 0.1)
    assert not any(t.requires_grad for t in (fc.master, fc.bias, Y, fc.weight(), fc(X), *kept))
    assert fc.master.data_ptr() != W.data_ptr() and fc.bias.data_ptr() != b.data_ptr()


def test_refusals():
    (values, exps), _ = layer(100, 200, 1)
    X = acts(5, 200, BF, 1).to(DEV)
    x = kq.kq_quantize_blocks(X)
    bad = [lambda: kq.kq_quantize_blocks(X, rows=2), lambda: kq.kq_quantize_blocks(X.t()), lambda: kq.kq_quantize_blocks(X.int()),
           lambda: kq.kq_quantize_blocks(X, values=x[0][:4], exps=x[1]), lambda: kq.kq_quantize_blocks(X, values=x[0].view(torch.uint8)),
           lambda: kq.kq_reconstruct_blocks(x[0], x[1], 300), lambda: kq.kq_reconstruct_blocks(x[0], x[1], 200, rows=128),
           lambda: kq.kq_reconstruct_blocks(x[0], x[1], 200, dtype=torch.float64),
           lambda: kq.kq_block_linear(X[:, :100], values, exps), lambda: kq.kq_block_linear(X, values, exps[:, :1]),
           lambda: kq.kq_block_linear(X, values.view(torch.uint8), exps), lambda: kq.kq_block_linear(x[0], values, exps),
           lambda: kq.kq_block_linear(X, values, exps, x_exps=x[1]), lambda: kq.kq_block_linear(X, values, exps, bias=torch.zeros(99, device=DEV)),
           lambda: kq.kq_block_linear(X, values, exps, Y=torch.empty(5, 99, dtype=BF, device=DEV)),
           lambda: kq.kq_block_linear(X, values, exps, dtype=F32, Y=torch.empty(5, 100, dtype=BF, device=DEV)),
           lambda: kq.kq_block_linear(X, values, exps, dtype=torch.float64), lambda: kq.kq_block_linear(X.cpu(), values, exps),
           lambda: kq.kq_block_linear_grad_input(X, values, exps, 200), lambda: kq.kq_block_linear_grad_input(X[:, :100], values, exps, 300),
           lambda: kq.kq_block_linear_grad_weight(X[:4], *x, 200), lambda: kq.kq_block_linear_grad_weight(X, x[0], x[1], 100),
           lambda: kq.kq_block_linear_grad_weight(X, *x, 200, dbias=torch.zeros(3, device=DEV)),
           lambda: kq.kq_block_linear_grad_weight(X, *x, 200, dtype=torch.int32)]
    for i, f in enumerate(bad):
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            f()
            print("accepted", i)
