"""Distillation from a teacher's top logits on the GPU, against the formulas in 64 bits.

Tolerances (set from the arithmetic, before any run), eps = 2^-24.  An exponential's argument is a difference times a
constant, two roundings and a third in the constant, so exp((z - M) / T) is off by at most (3 A + 4) eps of itself with A the largest
|z - M| / T of the row in powers of two; a sum of v of them in 256 or more parts adds (v / 64 + 16) eps.  With R = (8 A +
v / 32 + 64) eps:
  * dz: |dz - dz64| <= u |dz64| + R |d| ((1 - alpha) T (q + p) + alpha (s + [label]))  (u = torch.finfo(type of dz).eps / 2, half a step);
  * loss: sums of p (log p - log q), whose terms are differences of logits and logarithms: off by at most R of the sum of
    p (|t - t_max| / T + |z - M| / T + log S + log S_t + 1), times (1 - alpha) T^2, and the label's term likewise.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

kq = pytest.importorskip("paper_2003_05148_amd")
DEV = torch.device("cuda:0")
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF: 2.0 ** -8, HF: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF: 2.0 ** -126, HF: 2.0 ** -25, F32: 2.0 ** -126}


def gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def logits(m, v, top, dtype, seed, absent=0.2):
    g = gen(seed)
    t = 3 * torch.randn(m, v, generator=g)
    values, idx = t.topk(min(top, v), 1)
    if top > v:     # more places than classes: the rest are absent
        values = torch.nn.functional.pad(values, (0, top - v))
        idx = torch.nn.functional.pad(idx, (0, top - v), value=-1)
    idx = torch.where(torch.rand(m, top, generator=g) < absent, torch.full_like(idx, -1), idx)
    Z = (0.8 * t + torch.randn(m, v, generator=g)).to(dtype)
    labels = torch.where(torch.rand(m, generator=g) < 0.2, torch.full((m,), -100), t.argmax(1))
    return Z, values, idx, labels


def formula(Z, values, idx, labels, T, alpha, d):
    """(loss, dz, bound of the loss' error in units of R, bound of dz's), all in 64 bits, row by row."""
    Z = Z.double()
    m, v = Z.shape
    loss, dz = torch.zeros(m, dtype=torch.float64), torch.zeros_like(Z)
    lb, db = torch.zeros(m, dtype=torch.float64), torch.zeros_like(Z)
    for r in range(m):
        z = Z[r]
        M = z.max()
        if alpha < 1:
            here = [(int(idx[r, j]), float(values[r, j]) / T) for j in range(idx.shape[1])
                    if 0 <= int(idx[r, j]) < v and float(values[r, j]) != -math.inf]
            if here:
                t = torch.tensor([h[1] for h in here], dtype=torch.float64)
                p, logp, at = torch.softmax(t, 0), torch.log_softmax(t, 0), torch.tensor([h[0] for h in here])
                logq = torch.log_softmax(z / T, 0)
                live = p > 0
                w = (1 - alpha) * T * T
                loss[r] += w * (p * (logp - logq[at]))[live].sum()
                lb[r] += w * (p * ((t - t.max()).abs() + (z[at] - M).abs() / T + (M / T - logq.max()).abs() * 0 + (-logq.max()).abs()
                                   + (-logp.max()).abs() + 1))[live].sum()
                q = torch.exp(logq)
                pc = torch.zeros(v, dtype=torch.float64).index_add_(0, at, p)
                dz[r] += d[r] * (1 - alpha) * T * (q - pc)
                db[r] += abs(d[r]) * (1 - alpha) * T * (q + pc)
        y = int(labels[r]) if labels is not None else -1
        if alpha > 0 and 0 <= y < v:
            logs = torch.log_softmax(z, 0)
            loss[r] -= alpha * logs[y]
            lb[r] += alpha * ((z[y] - M).abs() + logs.max().abs() + 1)
            s = torch.exp(logs)
            one = torch.zeros(v, dtype=torch.float64)
            one[y] = 1
            dz[r] += d[r] * alpha * (s - one)
            db[r] += abs(d[r]) * alpha * (s + one)
    return loss, dz, lb, db


def check(loss, dz, Z, values, idx, labels, T, alpha, d):
    want, wdz, lb, db = formula(Z, values, idx, labels, T, alpha, d)
    v = Z.shape[1]
    z = Z.double()
    z = torch.where(torch.isinf(z), z.max(1, keepdim=True).values, z)
    A = (z.max(1).values - z.min(1).values) / min(T, 1.0 if alpha > 0 else T) * 1.4427
    R = (8 * A + v / 32 + 64) * 2.0 ** -24
    if loss is not None:
        assert torch.all((loss.double().cpu() - want).abs() <= R * lb + 2.0 ** -24 * want.abs())
    if dz is not None:
        tol = U[dz.dtype] * wdz.abs() + R[:, None] * db + TINY[dz.dtype]
        err = (dz.double().cpu() - wdz).abs()
        assert torch.all(err <= tol), float((err - tol).max())


def on(*ts):
    return [None if t is None else t.to(DEV) for t in ts]


SIZES = [(1, 1, 1), (3, 2, 1), (5, 7, 10), (9, 64, 10), (70, 1000, 10), (4, 1001, 64), (3, 2047, 256), (6, 2050, 33),
         (3, 5003, 100), (2, 16400, 20), (40, 9000, 5), (1, 70001, 100), (17, 33000, 64)]


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("m,v,top", SIZES)
def test_loss_and_gradient(m, v, top, dtype):
    T, alpha = [(1.0, 0.0), (2.0, 0.3), (1.0, 0.5), (3.5, 0.0), (0.7, 1.0)][(m + v + top) % 5]
    Z, values, idx, labels = logits(m, v, top, dtype, m + v)
    d = 0.5 + torch.rand(m, generator=gen(1))
    z, tv, ti, y, dl = on(Z, values, idx, labels, d)
    loss, dz = kq.kq_distill(z, tv, ti, temperature=T, labels=y, alpha=alpha, dloss=dl)
    check(loss, dz, Z, values, idx, labels, T, alpha, d.double())
    l2, stats = kq.kq_distill_loss(z, tv, ti, T, y, alpha)
    check(l2, kq.kq_distill_grad(z, tv, ti, stats, dl, T, y, alpha), Z, values, idx, labels, T, alpha, d.double())
    a, b = kq.kq_distill(z, tv, ti, temperature=T, labels=y, alpha=alpha, dloss=dl)
    assert torch.equal(a, loss) and torch.equal(b, dz)      # the same bits every time


@pytest.mark.parametrize("v,dtype", [(4500, F32), (9001, BF), (12000, F32), (20003, HF), (30001, F32), (50001, BF), (65530, F32), (70001, BF),
                                     (110001, BF), (130000, HF), (140001, F32)])
def test_long_rows_of_many(v, dtype):
    """As many rows as have a workgroup each, with every number of chunks a thread: single rows against the formula, by one call
    and by two (which may add a row in another order), and all of them again and in place."""
    m, rows = 193, [0, 1, 2, 96, 191, 192]
    Z, values, idx, labels = logits(m, v, 20, dtype, v)
    idx[1], labels[1] = -1, -1                    # a row without a term
    Z[2, :v // 2] = -math.inf
    Z[2, idx[2].clamp(min=0)] = 0.0
    Z[2, labels[2].clamp(min=0)] = 0.0
    z, tv, ti, y = on(Z, values, idx, labels)
    for T, alpha in ((1.0, 0.0), (1.0, 0.5), (2.5, 0.3)):
        loss, dz = kq.kq_distill(z, tv, ti, temperature=T, labels=y, alpha=alpha)
        pick = lambda x: x[rows]
        check(loss[rows], dz[rows], pick(Z), pick(values), pick(idx), pick(labels), T, alpha, torch.ones(len(rows)).double())
        l2, stats = kq.kq_distill_loss(z, tv, ti, T, y, alpha)
        g = kq.kq_distill_grad(z, tv, ti, stats, None, T, y, alpha)
        check(l2[rows], g[rows], pick(Z), pick(values), pick(idx), pick(labels), T, alpha, torch.ones(len(rows)).double())
        l3, same = kq.kq_distill(z.clone(), tv, ti, temperature=T, labels=y, alpha=alpha, dZ=None)
        inplace = z.clone()
        l4, out = kq.kq_distill(inplace, tv, ti, temperature=T, labels=y, alpha=alpha, dZ=inplace)
        assert out is inplace and torch.equal(l3, loss) and torch.equal(l4, loss) and torch.equal(same, dz) and torch.equal(inplace, dz)


@pytest.mark.parametrize("T", [1.0, 4.0, 2.0 ** -3])
@pytest.mark.parametrize("alpha", [0.0, 0.25, 1.0])
def test_weights_and_types_of_the_inputs(T, alpha):
    Z, values, idx, labels = logits(20, 300, 12, BF, 7)
    for tt in (F32, BF, HF):
        for it in (torch.int32, torch.int64):
            t = values.to(tt)
            z, tv, ti, y = on(Z, t, idx.to(it), labels.to(it))
            loss, dz = kq.kq_distill(z, tv, ti, temperature=T, labels=y, alpha=alpha, scale=0.125)
            check(loss, dz, Z, t, idx, labels, T, alpha, torch.full((20,), 0.125).double())
            l2, stats = kq.kq_distill_loss(z, tv, ti, T, y, alpha)
            check(l2, kq.kq_distill_grad(z, tv, ti, stats, None, T, y, alpha, scale=0.125), Z, t, idx, labels, T, alpha,
                  torch.full((20,), 0.125).double())


@pytest.mark.parametrize("v", [12, 900, 3001, 20000])
def test_the_same_index_twice(v):
    """Entries of one class add up, the label among them, however many there are and wherever they stand."""
    Z, values, idx, labels = logits(6, v, 200, F32, v, absent=0.0)
    idx[0] = 5
    idx[1, ::2] = 3
    idx[2, 150:] = idx[2, :50]
    idx[3] = torch.arange(200) % 7
    idx[4, 199] = idx[4, 0]
    labels = torch.tensor([5, 3, int(idx[2, 0]), 6, 11, 0])
    for alpha in (0.0, 0.4):
        z, tv, ti, y = on(Z, values, idx, labels)
        loss, dz = kq.kq_distill(z, tv, ti, temperature=2.0, labels=y, alpha=alpha)
        check(loss, dz, Z, values, idx, labels, 2.0, alpha, torch.ones(6).double())
        l2, stats = kq.kq_distill_loss(z, tv, ti, 2.0, y, alpha)
        check(l2, kq.kq_distill_grad(z, tv, ti, stats, None, 2.0, y, alpha), Z, values, idx, labels, 2.0, alpha, torch.ones(6).double())


@pytest.mark.parametrize("v", [10, 1500, 9000])
def test_rows_with_nothing(v):
    """No present entry, no label, neither, indices far outside, teacher's logits of -infinity."""
    m = 8
    Z, values, idx, labels = logits(m, v, 9, F32, v, absent=0.0)
    idx[1] = -1
    idx[2, :5], idx[2, 5:] = v, -(1 << 40)
    labels[3], labels[2], labels[4] = -100, v, 1 << 40
    values[5] = -math.inf
    values[6, 2:] = -math.inf
    for T, alpha in ((2.0, 0.5), (1.0, 0.0)):
        z, tv, ti, y = on(Z, values, idx, labels)
        loss, dz = kq.kq_distill(z, tv, ti, temperature=T, labels=y, alpha=alpha)
        check(loss, dz, Z, values, idx, labels, T, alpha, torch.ones(m).double())
        assert float(loss[2]) == 0 and torch.all(dz[2] == 0)
        l2, stats = kq.kq_distill_loss(z, tv, ti, T, y, alpha)
        g = kq.kq_distill_grad(z, tv, ti, stats, None, T, y, alpha)
        check(l2, g, Z, values, idx, labels, T, alpha, torch.ones(m).double())
        assert torch.all(g[2] == 0)


@pytest.mark.parametrize("v", [10, 1500, 9000, 70001])
def test_rows_without_a_term_are_zero_whatever_they_hold(v):
    m = 5
    for dtype in (F32, BF):
        Z, values, idx, labels = logits(m, v, 4, dtype, v, absent=0.0)
        idx[:4], labels[:4] = -1, -1
        Z[0], Z[1, v - 1], Z[2, 0] = -math.inf, math.nan, math.inf
        z, tv, ti, y = on(Z, values, idx, labels)
        for T, alpha in ((2.0, 0.5), (1.0, 0.25), (1.0, 0.0)):
            loss, dz = kq.kq_distill(z, tv, ti, temperature=T, labels=y, alpha=alpha)
            l2, stats = kq.kq_distill_loss(z, tv, ti, T, y, alpha)
            for a, g in ((loss, dz), (l2, kq.kq_distill_grad(z, tv, ti, stats, None, T, y, alpha))):
                assert torch.all(a[:4] == 0) and torch.all(g[:4] == 0)
                check(a[4:], g[4:], Z[4:], values[4:], idx[4:], labels[4:], T, alpha, torch.ones(1).double())


@pytest.mark.parametrize("v", [10, 1500, 9000, 70001])
def test_masked_classes_and_bad_rows(v):
    m = 6
    Z, values, idx, labels = logits(m, v, 5, F32, v, absent=0.0)
    labels = idx[:, 0].clone()
    keep = torch.zeros(v, dtype=torch.bool)
    keep[idx[0]] = True
    keep[0] = True
    Z[0, ~keep] = -math.inf             # all but a few masked out
    Z[1, idx[1, 1]] = -math.inf         # the teacher's second choice masked out: an infinite loss, a finite gradient
    Z[2, v // 2] = math.nan
    Z[3, v // 3] = math.inf
    Z[4] = -math.inf
    z, tv, ti, y = on(Z, values, idx, labels)
    for alpha in (0.0, 0.3):
        loss, dz = kq.kq_distill(z, tv, ti, temperature=2.0, labels=y, alpha=alpha)
        l2, stats = kq.kq_distill_loss(z, tv, ti, 2.0, y, alpha)
        for a, g in ((loss, dz), (l2, kq.kq_distill_grad(z, tv, ti, stats, None, 2.0, y, alpha))):
            for r in (0, 5):
                check(a[r:r + 1], g[r:r + 1], Z[r:r + 1], values[r:r + 1], idx[r:r + 1], labels[r:r + 1], 2.0, alpha, torch.ones(1).double())
            assert torch.all(g[0].cpu()[~keep] == 0)
            assert float(a[1]) == math.inf
            check(None, g[1:2], Z[1:2], values[1:2], idx[1:2], labels[1:2], 2.0, alpha, torch.ones(1).double())
            for r in (2, 3, 4):
                assert math.isnan(float(a[r])) and torch.all(torch.isnan(g[r]))
    values[0, 0], values[1, 0] = math.nan, math.inf
    loss, dz = kq.kq_distill(z, values.to(DEV), ti, temperature=2.0)
    assert math.isnan(float(loss[0])) and torch.all(torch.isnan(dz[0])) and math.isnan(float(loss[1]))
    check(loss[5:], dz[5:], Z[5:], values[5:], idx[5:], labels[5:], 2.0, 0.0, torch.ones(1).double())


def test_gradient_against_differences():
    m, v = 4, 50
    Z, values, idx, labels = logits(m, v, 8, F32, 3)
    T, alpha = 2.5, 0.35
    z, tv, ti, y = on(Z, values, idx, labels)
    dz = kq.kq_distill(z, tv, ti, temperature=T, labels=y, alpha=alpha)[1].double().cpu()
    h = 2.0 ** -12
    for seed in range(3):
        D = torch.randn(m, v, generator=gen(seed)).double()
        ones = torch.ones(m).double()
        up = formula(Z.double() + h * D, values, idx, labels, T, alpha, ones)[0].sum()
        down = formula(Z.double() - h * D, values, idx, labels, T, alpha, ones)[0].sum()
        # a third derivative of at most about 1 a row: h^2 |D|^3 / 6
        assert abs(float((up - down) / (2 * h)) - float((dz * D).sum())) <= h * h * float(D.abs().sum()) * 8 + 1e-5


@pytest.mark.parametrize("m,v", [(3, 100), (7, 3000), (2, 70001), (64, 1000)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_in_place_strides_and_leading_sizes(m, v, dtype):
    Z, values, idx, labels = logits(m, v, 6, dtype, v)
    z, tv, ti, y = on(Z, values, idx, labels)
    how = dict(temperature=2.0, labels=y, alpha=0.3)
    loss, dz = kq.kq_distill(z, tv, ti, **how)
    _, stats = kq.kq_distill_loss(z, tv, ti, **how)
    g = kq.kq_distill_grad(z, tv, ti, stats, **how)
    big = torch.full((m, v + 13), 5.0, dtype=dtype, device=DEV)
    view = big[:, 6:6 + v]
    view.copy_(z)
    one = torch.ones(m).double()
    l1, d1 = kq.kq_distill(view, tv, ti, **how)      # (rows that begin elsewhere: another order of the sums)
    check(l1, d1, Z, values, idx, labels, 2.0, 0.3, one)
    l2, d2 = kq.kq_distill(view, tv, ti, dZ=view, **how)
    assert torch.equal(l2, l1) and torch.equal(view, d1) and d2 is view
    view.copy_(z)
    kq.kq_distill_grad(view, tv, ti, stats, dZ=view, **how)
    assert torch.equal(view, g)     # (no sums in it)
    assert torch.all(big[:, :6] == 5) and torch.all(big[:, 6 + v:] == 5)
    if m % 2 == 0:
        l3, d3 = kq.kq_distill(z.view(2, m // 2, v), tv.view(2, m // 2, -1), ti.view(2, m // 2, -1), temperature=2.0,
                               labels=y.view(2, m // 2), alpha=0.3)
        assert torch.equal(l3, loss) and torch.equal(d3.view(m, v), dz)
    e, de = kq.kq_distill(z[:0], tv[:0], ti[:0])
    assert e.shape == (0,) and de.shape == (0, v)


@pytest.mark.parametrize("m,v", [(5, 1000), (3, 70001), (40, 9000)])
def test_streams_and_graphs(m, v):
    Z, values, idx, labels = logits(m, v, 6, BF, v)
    z, tv, ti, y = on(Z, values, idx, labels)

    def step():
        l1, d1 = kq.kq_distill(z, tv, ti, temperature=2.0, labels=y, alpha=0.3)
        l2, stats = kq.kq_distill_loss(z, tv, ti, 2.0, y, 0.3)
        return l1, d1, l2, kq.kq_distill_grad(z, tv, ti, stats, l2, 2.0, y, 0.3)
    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step()
    other = step()
    s.synchronize()
    for a, b, c in zip(want, got, other):
        assert torch.equal(a, b) and torch.equal(a, c)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for seed in range(4):
        z.copy_(logits(m, v, 6, BF, seed)[0])
        want = [t.clone() for t in step()]
        g.replay()
        step()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_without_the_host_helper(monkeypatch):
    """The binding's own checks and calls give what the C++ helper's plain case gives."""
    z, tv, ti, y = on(*logits(9, 700, 6, BF, 1))
    d = torch.rand(9, device=DEV)

    def calls():
        l2, stats = kq.kq_distill_loss(z, tv, ti, 2.0, y, 0.3)
        return [*kq.kq_distill(z, tv, ti, temperature=2.0, labels=y, alpha=0.3, dloss=d), *kq.kq_distill(z, tv, ti, scale=0.5), l2, stats,
                kq.kq_distill_grad(z, tv, ti, stats, d, 2.0, y, 0.3)]
    want = calls()
    monkeypatch.setattr(kq, "_fast", None)
    for a, b in zip(want, calls()):
        assert a.dtype == b.dtype and torch.equal(a, b)


def test_offsets_past_32_bits():
    """Rows more than 2^32 bytes apart, and a large number of classes."""
    v = 200000
    buf = torch.zeros(3, 1 << 30, dtype=BF, device=DEV)
    Z, values, idx, labels = logits(3, v, 6, BF, 1)
    z = buf[:, 3:3 + v]
    z.copy_(Z)
    tv, ti, y = on(values, idx, labels)
    loss, dz = kq.kq_distill(z, tv, ti, temperature=2.0, labels=y, alpha=0.3, dZ=z)
    check(loss, dz.contiguous(), Z, values, idx, labels, 2.0, 0.3, torch.ones(3).double())
    assert torch.all(buf[:, :3] == 0) and torch.all(buf[:, 3 + v:4 + v + 1000] == 0)


def test_refusals():
    Z, values, idx, labels = on(*logits(4, 50, 5, BF, 1))
    s = torch.empty(4, 3, device=DEV)
    bad = [lambda: kq.kq_distill(Z.cpu(), values, idx), lambda: kq.kq_distill(Z.t(), values, idx),
           lambda: kq.kq_distill(Z, values[:3], idx), lambda: kq.kq_distill(Z, values, idx[:, :4]),
           lambda: kq.kq_distill(Z, values, idx.float()), lambda: kq.kq_distill(Z, values.int(), idx),
           lambda: kq.kq_distill(Z, values[:, ::2], idx[:, ::2]), lambda: kq.kq_distill(Z, values, idx, alpha=0.5),
           lambda: kq.kq_distill(Z, values, idx, alpha=1.5, labels=labels), lambda: kq.kq_distill(Z, values, idx, alpha=math.nan, labels=labels),
           lambda: kq.kq_distill(Z, values, idx, temperature=0.0), lambda: kq.kq_distill(Z, values, idx, temperature=math.nan),
           lambda: kq.kq_distill(Z, values, idx, temperature=math.inf), lambda: kq.kq_distill(Z, values, idx, temperature=-1.0),
           lambda: kq.kq_distill(Z, values, idx, labels=labels[:3], alpha=0.1), lambda: kq.kq_distill(Z, values, idx, labels=labels.float(), alpha=0.1),
           lambda: kq.kq_distill(Z, values, idx, dloss=torch.ones(3, device=DEV)), lambda: kq.kq_distill(Z, values, idx, dZ=torch.empty(4, 50, device=DEV)),
           lambda: kq.kq_distill(Z, values, idx, loss=torch.empty(4, dtype=BF, device=DEV)),
           lambda: kq.kq_distill(Z, values[:, :0], idx[:, :0]),
           lambda: kq.kq_distill(Z, torch.zeros(4, 257, device=DEV), torch.zeros(4, 257, dtype=torch.int64, device=DEV)),
           lambda: kq.kq_distill_loss(Z, values, idx, stats=torch.empty(4, 2, device=DEV)),
           lambda: kq.kq_distill_grad(Z, values, idx, s[:3]), lambda: kq.kq_distill_grad(Z, values, idx, s.to(BF))]
    for i, f in enumerate(bad):
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            f()
            print("accepted", i)


# ---- a run of the operators together ---------------------------------------------------------------------------------

def test_a_retraining_step():
    """An 8-bit classifier against an uncompressed one: logits, loss and its gradient, and the layer's gradients, each
    against the formulas on the values that the step before gave."""
    m, n, k = 60, 300, 260
    g = gen(5)
    W = torch.randn(n, k, generator=g) / math.sqrt(k)
    b = 0.1 * torch.randn(n, generator=g)
    X = torch.randn(m, k, generator=g).relu().to(BF)
    fc = kq.BlockLinear(W.to(DEV), b.to(DEV), master=True)
    t = X.double() @ W.double().t() + b.double()
    values, idx = (4 * t).topk(10, 1)
    values = values.float()
    Z, kept = fc.forward(X.to(DEV), dtype=F32)
    w_hat = fc.weight().double().cpu()
    x_hat = kq.kq_reconstruct_blocks(*kept, k).double().cpu()
    assert torch.allclose(Z.double().cpu(), x_hat @ w_hat.t() + b.double(), rtol=1e-5, atol=1e-5)
    loss, dZ = kq.kq_distill(Z, values.to(DEV), idx.to(DEV), temperature=2.0, scale=1 / m)
    check(loss, dZ, Z.cpu(), values, idx, None, 2.0, 0.0, torch.full((m,), 1 / m).double())
    dX, dW, db = fc.backward(dZ, kept)
    d64 = dZ.double().cpu()
    # e4m3 rounds to 2^-4 of a value: of a sum's norm that is less than 2^-4
    for got, want in ((dX, d64 @ w_hat), (dW, d64.t() @ x_hat)):
        assert float((got.double().cpu() - want).norm() / want.norm()) < 2.0 ** -4
    assert torch.all((db.double().cpu() - d64.sum(0)).abs() <= 64 * 2.0 ** -24 * d64.abs().sum(0))
    fc.step(dW, db, 0.1)
    # the product with 0.1 is rounded (2^-24 of it, and 0.1 itself 2^-25) or fused, then the difference (2^-24 of it)
    want = W.double() - 0.1 * dW.double().cpu()
    assert torch.all((fc.master.double().cpu() - want).abs() <= 2.0 ** -24 * want.abs() + 2.0 ** -23 * 0.1 * dW.double().cpu().abs())


def example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "fc8_distill.py")
    spec = importlib.util.spec_from_file_location("fc8_distill", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_retraining_example_runs():
    losses, (fc1, fc2) = example().retrain(n_in=300, n_hidden=260, classes=100, batch=70, steps=4)
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses)
    assert fc2(torch.relu(fc1(torch.randn(1, 300, device=DEV, dtype=BF)))).shape == (1, 100)


def test_retraining_examples_gradients():
    """Against the formulas in 64 bits on what the 8-bit layers stand for.  The 8-bit steps of the activation, of dZ (twice) and of dA
    (twice) are at most 2^-4 of a value each, bf16's 2^-8: of a sum's norm (errors of random signs) less than 2^-4 for dZ's
    products and 2^-3 for those that come after dA."""
    m, n_in, n_hidden, classes = 70, 300, 260, 100
    g = gen(8)
    W1, W2 = torch.randn(n_hidden, n_in, generator=g) / math.sqrt(n_in), 2 * torch.randn(classes, n_hidden, generator=g) / math.sqrt(n_hidden)
    b1, b2 = 0.1 * torch.randn(n_hidden, generator=g), 0.1 * torch.randn(classes, generator=g)
    X = torch.randn(m, n_in, generator=g).relu().to(BF)
    fc1, fc2 = kq.BlockLinear(W1.to(DEV), b1.to(DEV)), kq.BlockLinear(W2.to(DEV), b2.to(DEV))
    t = torch.relu(X.float() @ W1.t() + b1) @ W2.t() + b2
    values, idx = t.topk(10, 1)
    labels = idx[:, 0].contiguous()
    loss, got = example().gradients(fc1, fc2, X.to(DEV), values.to(DEV), idx.to(DEV), labels.to(DEV))
    w2 = fc2.weight().double().cpu()
    H = fc1.forward(X.to(DEV))[0]
    Z = fc2.forward(torch.relu(H))[0].cpu()
    want, dz, _, _ = formula(Z, values, idx, labels, 2.0, 0.3, torch.full((m,), 1 / m).double())
    check(loss, None, Z, values, idx, labels, 2.0, 0.3, torch.full((m,), 1 / m).double())
    A = torch.relu(H).double().cpu()
    dH = (dz @ w2) * (A > 0)
    for a, b, bound in ((got[0], dH.t() @ X.double(), 2.0 ** -3), (got[1], dH.sum(0), 2.0 ** -3), (got[2], dz.t() @ A, 2.0 ** -4),
                        (got[3], dz.sum(0), 2.0 ** -4)):
        assert float((a.double().cpu() - b).norm() / b.norm()) < bound
