"""The 4-bit fully-connected layer and the 8-bit checkpoints at the edges of their matrices and of their numbers, on
the GPU against plain forms in 64 bits.  Tolerances and helpers are those of test_gpu_group_linear.py."""
import pytest
import torch

from test_gpu_group_linear import BF, DEV, F32, HF, Layer, acts, check, grad_inputs, pack, table, values

pytestmark = pytest.mark.gpu

kq = pytest.importorskip("paper_2003_05148_amd")


def group_sums(v, group):
    """Sums over groups of columns."""
    n, k = v.shape
    G = -(-k // group)
    return torch.zeros(n, G, dtype=torch.float64, device=v.device).index_add_(1, torch.arange(k, device=v.device) // group, v)


# ---- groups that the matrix ends in ------------------------------------------------------------------

@pytest.mark.parametrize("k", [32, 64, 93, 95, 96, 160, 192, 576, 960, 2208])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype,lut", [(BF, False), (BF, True), (HF, False), (HF, True)])
@pytest.mark.parametrize("m", [1, 200])
def test_scale_gradient_of_a_partial_last_group(m, k, group, dtype, lut):
    """Widths whose last group is not whole: what lies past the matrix adds nothing to it."""
    n = 37
    L = Layer(n, k, group, table(k) if lut else None, seed=k + group)
    dY, q, exps, xh = grad_inputs(m, n, k, dtype)
    ds, _ = kq.kq_checkpoint_grad_scales(dY.to(DEV), q, exps, L.packed, k, **L.kw())
    lv = values(L.levels)[L.codes.long()]
    d = dY.double()
    check(ds, group_sums((d.T @ xh) * lv, group), group_sums((d.abs().T @ xh.abs()) * lv.abs(), group), F32, m + group, False, False,
          norm=False)


@pytest.mark.parametrize("m,n,k,group,lut", [(130, 3500, 4128, 128, True), (130, 3500, 4128, 64, False), (1111, 2100, 2144, 128, False),
                                             (5000, 300, 544, 128, True), (5000, 300, 544, 64, False)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_partial_last_group_in_larger_tiles_and_splits(m, n, k, group, lut, dtype):
    """The same through the larger tile and through split contractions (the reference in 64 bits on the GPU)."""
    L = Layer(n, k, group, table(k) if lut else None, seed=n + k)
    dY = acts(m, n, dtype, seed=m + 1, scale=0.05).to(DEV)
    q, exps = kq.kq_checkpoint_pack(acts(m, k, dtype, seed=m + 2).to(DEV))
    ds, _ = kq.kq_checkpoint_grad_scales(dY, q, exps, L.packed, k, **L.kw())
    xh, d = kq.kq_checkpoint_restore(q, exps, k).double(), dY.double()
    lv = values(L.levels).to(DEV)[L.codes.long().to(DEV)]
    want, S = (d.T.contiguous() @ xh) * lv, (d.abs().T.contiguous() @ xh.abs()) * lv.abs()
    check(ds, group_sums(want, group).cpu(), group_sums(S, group).cpu(), F32, m + group, False, False, norm=False)


@pytest.mark.parametrize("k,group", [(96, 64), (160, 128), (95, 128)])
def test_partial_last_group_against_differences(k, group):
    """The loss is linear in the scales: its central difference is the last group's gradient."""
    m, n = 40, 9
    L = Layer(n, k, group, table(k), seed=k)
    dY, q, exps, xh = grad_inputs(m, n, k, BF)
    ds, _ = kq.kq_checkpoint_grad_scales(dY.to(DEV), q, exps, L.packed, k, **L.kw())
    lv = values(L.levels)[L.codes.long()]
    which = torch.arange(k) // group

    def loss(s):
        return float((dY.double() * (xh @ (lv * s[:, which]).T)).sum())

    s0 = L.scales.double()
    S = group_sums((dY.double().abs().T @ xh.abs()) * lv.abs(), group)
    for r in range(n):
        h = torch.zeros_like(s0)
        h[r, -1] = 2.0 ** -6
        num = (loss(s0 + h) - loss(s0 - h)) / 2.0 ** -5
        assert abs(num - float(ds[r, -1])) <= (m + group + 16) * 2.0 ** -24 * float(S[r, -1]) + 1e-7


@pytest.mark.parametrize("k", [40, 64, 70])
@pytest.mark.parametrize("lut", [False, True])
def test_infinite_gradient_of_a_partial_last_group(k, lut):
    """Every term of the last group is positive, one infinite: so is its sum, whatever lies past the matrix."""
    m, n, group = 3, 20, 128
    L = Layer(n, k, group, torch.arange(-8, 8).to(BF) if lut else None, seed=k)
    L.packed = pack(torch.full((n, k), 12, dtype=torch.uint8)).to(DEV)      # level 4
    q, exps = kq.kq_checkpoint_pack(torch.ones(m, k, dtype=BF, device=DEV))
    dY = torch.ones(m, n, dtype=BF, device=DEV)
    dY[1, 7] = float("inf")
    ds, _ = kq.kq_checkpoint_grad_scales(dY, q, exps, L.packed, k, **L.kw())
    want = torch.full((n, 1), 4.0 * m * k, device=DEV)
    want[7] = float("inf")
    assert torch.equal(ds, want)


# ---- the largest numbers -----------------------------------------------------------------------------------

@pytest.mark.parametrize("m,n,k", [(3, 20, 40), (130, 40, 257), (1000, 2049, 1026)])
@pytest.mark.parametrize("lut", [False, True])
def test_gradients_from_the_largest_checkpoints(m, n, k, lut):
    """Values up to bf16's largest number (steps of 2^121): finite gradients of finite values."""
    X = 0.2 * acts(m, k, BF, seed=m + k).clamp(-5, 5) * 3.3e38
    X[:, ::7] = 3.3895314e38
    q, exps = kq.kq_checkpoint_pack(X.to(DEV))
    assert int(exps.max()) == 121 + 127
    dY = acts(m, n, BF, seed=m + n, scale=1e-36)
    L = Layer(n, k, 64, table(k) if lut else None, seed=n)
    xh, d = kq.kq_checkpoint_restore(q, exps, k).double(), dY.to(DEV).double()
    want, S = d.T.contiguous() @ xh, d.abs().T.contiguous() @ xh.abs()
    dW, _ = kq.kq_checkpoint_grad_weight(dY.to(DEV), q, exps, k)
    check(dW, want.cpu(), S.cpu(), F32, m, False, False)
    ds, _ = kq.kq_checkpoint_grad_scales(dY.to(DEV), q, exps, L.packed, k, **L.kw())
    lv = values(L.levels).to(DEV)[L.codes.long().to(DEV)]
    check(ds, group_sums(want * lv, 64).cpu(), group_sums(S * lv.abs(), 64).cpu(), F32, m + 64, False, False, norm=False)


def of_scale(n, k, group, levels, scale, seed):
    """A layer with one scale, whose codes are 1 .. 15: the lowest level stands past the matrix alone."""
    L = Layer(n, k, group, levels, seed=seed)
    L.codes.clamp_(min=1)
    L.packed = pack(L.codes).to(DEV)
    L.scales.fill_(scale)
    L.dscales = L.scales.to(DEV)
    return L


@pytest.mark.parametrize("m", [1, 16, 17, 64, 300])
def test_products_with_the_largest_scales(m):
    """Scales of 2^125 and more, as weights near bf16's largest number have: 7 of them is still finite."""
    n, k = 192, 256
    for scale in (2.0 ** 125, 2.0 ** 125 * (1 + 17 / 128)):
        L = of_scale(n, k, 128, None, scale, seed=m)
        X, dY = acts(m, k, BF, seed=m, scale=1e-30), acts(m, n, BF, seed=m + 1, scale=1e-30)
        W = L.W
        assert float(W.abs().max()) <= 3.3895314e38
        Y = kq.kq_group_linear(X.to(DEV), L.packed, L.dscales, **L.kw())
        check(Y, X.double() @ W.T, X.double().abs() @ W.abs().T, BF, k, m > 16, True)
        dX = kq.kq_group_linear_grad_input(dY.to(DEV), L.packed, L.dscales, k, **L.kw())
        check(dX, dY.double() @ W, dY.double().abs() @ W.abs(), BF, n, True, False)


@pytest.mark.parametrize("m,n,k", [(1, 40, 70), (17, 40, 70), (64, 33, 1000), (300, 515, 1030), (2048, 2100, 300)])
@pytest.mark.parametrize("dtype,lut", [(HF, False), (HF, True), (BF, False), (BF, True)])
def test_weights_past_the_matrix_may_overflow(m, n, k, dtype, lut):
    """Scales at which the lowest level, that of the codes past the matrix, is beyond the activations' type, and no
    level that the matrix has."""
    levels = torch.tensor([-2.0] + [-0.9 + 0.12 * i for i in range(15)]).to(BF) if lut else None
    scale = {(HF, False): 2.0 ** 13, (HF, True): 2.0 ** 15 * 1.5, (BF, False): 2.0 ** 125, (BF, True): 2.0 ** 127}[dtype, lut]
    L = of_scale(n, k, 32, levels, scale, seed=k)
    X = acts(m, k, dtype, seed=m, scale=1e-3 if dtype == HF else 1e-30)
    Y = kq.kq_group_linear(X.to(DEV), L.packed, L.dscales, **L.kw())
    W = L.W
    check(Y, X.double() @ W.T, X.double().abs() @ W.abs().T, dtype, k, m > 16, not lut, xsum=X.double().abs().sum(1, keepdim=True))


@pytest.mark.parametrize("m", [1, 4, 5, 16, 17])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("size", [2.0 ** 122, 2.0 ** 124])
def test_linear_of_large_activations(m, group, size):
    """One value in a group near bf16's largest number, the others ordinary: the level's product is taken off nothing
    that overflows."""
    n, k = 70, 300
    L = Layer(n, k, group, None, seed=m, scale=2.0 ** -100)
    X = acts(m, k, BF, seed=m)
    X[:, 5::group] = size
    X[m // 2] *= -1
    Y = kq.kq_group_linear(X.to(DEV), L.packed, L.dscales, **L.kw())
    check(Y, X.double() @ L.W.T, X.double().abs() @ L.W.abs().T, BF, k, m > 16, True)


@pytest.mark.parametrize("m", [1, 90])
def test_checkpoint_beyond_the_gradients_type_is_not_clipped(m):
    """An fp16 dY with a checkpoint of larger values: infinities or NaN, not the gradient of other values."""
    n, k = 20, 64
    X = torch.ones(m, k, dtype=BF)
    X[m // 2, 32:] = 1e5
    q, exps = kq.kq_checkpoint_pack(X.to(DEV))
    dY = torch.ones(m, n, dtype=HF, device=DEV)
    dW, _ = kq.kq_checkpoint_grad_weight(dY, q, exps, k)
    assert torch.all(dW[:, :32] == m) and not torch.isfinite(dW[:, 32:]).any()
    L = Layer(n, k, 32, None, seed=1)
    L.packed = pack(torch.full((n, k), 9, dtype=torch.uint8)).to(DEV)       # level 1
    ds, _ = kq.kq_checkpoint_grad_scales(dY, q, exps, L.packed, k, **L.kw())
    assert torch.all(ds[:, 0] == 32 * m) and not torch.isfinite(ds[:, 1]).any()


@pytest.mark.parametrize("m", [1, 4, 5, 16, 17])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** -20, 2.0 ** 20, 2.0 ** 110])
def test_level_tables_outside_of_fp16(m, group, size):
    """fp16 activations and levels that fp16 does not hold, with scales that bring the weights into its range."""
    n, k = 70, 300
    levels = (table(m).double() * size).to(BF)
    L = Layer(n, k, group, levels, seed=m, scale=0.02 / size)
    X = acts(m, k, HF, seed=m + 1)
    Y = kq.kq_group_linear(X.to(DEV), L.packed, L.dscales, **L.kw())
    check(Y, X.double() @ L.W.T, X.double().abs() @ L.W.abs().T, HF, k, m > 16, False, xsum=X.double().abs().sum(1, keepdim=True))
