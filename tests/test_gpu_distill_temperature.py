"""Distillation where p and q are close, at temperatures above 4, with entries that are all the classes a row has (all of v, or
all that are not masked out): the loss is T^2 times a small difference there.  (Up to T = 4 the bounds of
tests/test_gpu_distill.py hold, 64 eps T^2 at least.)

Against the definition in 80 bits (numpy's longdouble: at T = 2^20 its own error is below 10^-6 of the loss).

Tolerance of the loss (set from the arithmetic, before any run), eps = 2^-24.  With x_j = (t_j - z_j) / T less its mean under p
and A the largest of |t - t_max|, |z - M| and |t - z| of a row, x_j is off by the three differences' roundings, those of 1 / T and
the product, and the mean's: at most 16 A eps / T, a part that is common to all j counting only in its square.  The
loss is T^2 sum p (e^-x - 1 + x) (its logarithm changes nothing but for large x), whose derivative is at most
1.72 |x| p T^2 for |x| <= 1: 16 A eps 1.72 T sum p |x| <= 28 A eps sqrt(2 L 1.4) with L the loss itself, since
x^2 / 2 <= 1.4 (e^-x - 1 + x).  The p_j are off by (3 A / T log2 e + 16) eps of themselves, sums of at most 256 terms by 16
eps more: 2 (16 + 16 + 5 A / T) eps L.  In all 32 eps (1.5 A sqrt(L) + (2 + A / T) L).

Tolerance of the gradient T (q - p) = T p ((e^-x - 1) - y) / (1 + y), y what the logarithm above is taken of: x's five roundings
are 5 A eps / T, the mean's as many and 32 eps A / T for those of the p; T p times that, times e^|x| / (1 + y) <= 1.4
where T is above 4 and x is small, is below 64 A eps p.  p, y and the other factors are off by at most 64 eps of the result.  Then
half a step of dz's type.  kq_distill_grad of rows of more than 512 chunks of 16 bytes takes q - p as it stands: 64 + 8 A / T +
v / 32 eps of T (q + p) (tests/test_gpu_distill.py).
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

kq = pytest.importorskip("paper_2003_05148_amd")
DEV = torch.device("cuda:0")
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
EPS = 2.0 ** -24


def gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def rows(m, v, top, dtype, seed, noise=1.0):
    """Logits with `top` classes that are not masked out, spread over the row, and the teacher's at all of them, in any order."""
    g = gen(seed)
    Z = torch.full((m, v), -float("inf"))
    idx = torch.stack([torch.randperm(v, generator=g)[:top] for _ in range(m)])
    t = 3 * torch.randn(m, top, generator=g)
    Z.scatter_(1, idx, t + noise * torch.randn(m, top, generator=g))
    return Z.to(dtype), t, idx


def exact(Z, t, idx, T):
    """(loss, p - q at the entries, p, A) of each row, from the definition in 80 bits."""
    z = Z.double().gather(1, idx).numpy().astype(np.longdouble)
    t = t.double().numpy().astype(np.longdouble)
    w, u = t / np.longdouble(T), z / np.longdouble(T)
    w, u = w - w.max(1, keepdims=True), u - u.max(1, keepdims=True)
    logp = w - np.log(np.exp(w).sum(1, keepdims=True))
    logq = u - np.log(np.exp(u).sum(1, keepdims=True))
    p = np.exp(logp)
    loss = (p * (logp - logq)).sum(1) * np.longdouble(T) ** 2
    A = np.maximum(np.maximum(np.ptp(t, 1), np.ptp(z, 1)), np.abs((t - t.max(1, keepdims=True)) - (z - z.max(1, keepdims=True))).max(1))
    return loss, p - np.exp(logq), p, A


def near(loss, want, A, T, weight=1.0):
    got = loss.double().cpu().numpy().astype(np.longdouble)
    want = want * weight
    tol = 32 * EPS * (1.5 * A * np.sqrt(np.abs(want) * weight) + (2 + A / T) * np.abs(want))
    assert np.all(np.abs(got - want) <= tol), (got, want, tol)


U = {BF: 2.0 ** -8, HF: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF: 2.0 ** -126, HF: 2.0 ** -25, F32: 2.0 ** -126}


def near_gradient(dz, Z, idx, less, p, A, T, d, plain=False):
    """less: p - q at the entries.  Masked classes have no gradient at all."""
    assert torch.all(dz.cpu()[torch.isinf(Z)] == 0)
    got = dz.double().cpu().gather(1, idx).numpy().astype(np.longdouble)
    want, A = -d * np.longdouble(T) * less, A[:, None]
    tol = EPS * (64 * A * p * d + 64 * np.abs(want)) + U[dz.dtype] * np.abs(want) + TINY[dz.dtype]
    if plain:
        tol = tol + EPS * (64 + 8 * A / T + Z.shape[1] / 32) * d * T * (2 * p - less)
    assert np.all(np.abs(got - want) <= tol), (np.abs(got - want) / tol).max()


TEMPERATURES = [4.25, 7.0, 20.0, 100.0, 1024.0, 2.0 ** 20]
SIZES = [(5, 10, 10), (5, 100, 100), (3, 256, 256), (9, 1000, 100), (5, 3000, 256), (5, 9001, 60), (4, 20000, 100), (3, 33000, 7),
         (3, 70001, 100), (130, 70001, 50), (130, 140001, 30)]


@pytest.mark.parametrize("T", TEMPERATURES)
@pytest.mark.parametrize("m,v,top", SIZES)
def test_loss_of_rows_whose_classes_are_all_entries(m, v, top, T):
    for dtype in (F32, BF) if v < 100000 else (F32,):
        # (at the lowest temperature also a network near its teacher)
        Z, t, idx = rows(m, v, top, dtype, v + top, noise=1.0 if T > 5 else 0.02)
        if dtype == BF:
            t = t.to(BF).float()      # (else half a step of bf16 is most of the difference)
        loss, _, _, A = exact(Z, t, idx, T)
        z, tv, ti = Z.to(DEV), t.to(DEV), idx.to(DEV)
        near(kq.kq_distill(z, tv, ti, temperature=T)[0], loss, A, T)
        near(kq.kq_distill_loss(z, tv, ti, T)[0], loss, A, T)
        inplace = z.clone()
        near(kq.kq_distill(inplace, tv, ti, temperature=T, dZ=inplace)[0], loss, A, T)


@pytest.mark.parametrize("T", TEMPERATURES)
@pytest.mark.parametrize("m,v,top", SIZES)
def test_gradient_of_rows_whose_classes_are_all_entries(m, v, top, T):
    for dtype in (F32, HF, BF) if v < 100000 else (F32,):
        Z, t, idx = rows(m, v, top, dtype, v + top + 1, noise=1.0 if T > 5 else 0.02)
        _, less, p, A = exact(Z, t, idx, T)
        z, tv, ti = Z.to(DEV), t.to(DEV), idx.to(DEV)
        near_gradient(kq.kq_distill(z, tv, ti, temperature=T, scale=0.5)[1], Z, idx, less, p, A, T, 0.5)
        stats = kq.kq_distill_loss(z, tv, ti, T)[1]
        plain = v // (4 if dtype == F32 else 8) > 512
        near_gradient(kq.kq_distill_grad(z, tv, ti, stats, None, T, scale=0.5), Z, idx, less, p, A, T, 0.5, plain)
        inplace = z.clone()
        kq.kq_distill(inplace, tv, ti, temperature=T, scale=0.5, dZ=inplace)
        near_gradient(inplace, Z, idx, less, p, A, T, 0.5)


@pytest.mark.parametrize("T", [20.0, 2.0 ** 20])
def test_gradient_of_classes_that_stand_twice_and_labels(T):
    """The label's term is added to a close row's, and an entry that stands twice has both its p.  The sum of the entries'
    exponentials passes S_T by one class then: the difference of two sums of at most 91 terms, each off by at most 64 eps of
    itself, is 128 eps S_T of y more, and 128 eps T p of the gradient."""
    m, v, alpha = 6, 90, 0.25
    Z, t, idx = rows(m, v, v, F32, 4)
    labels = idx[:, 7].contiguous()
    t2, idx2 = torch.cat([t, t[:, 5:6]], 1), torch.cat([idx, idx[:, 5:6]], 1)
    w = t2.double().numpy().astype(np.longdouble) / np.longdouble(T)
    p2 = np.exp(w - w.max(1, keepdims=True))
    p2 /= p2.sum(1, keepdims=True)
    u = Z.double().numpy().astype(np.longdouble)
    A = np.maximum(np.ptp(t.numpy(), 1), np.ptp(u, 1)).astype(np.longdouble)[:, None]

    def soft(x):
        e = np.exp(x - x.max(1, keepdims=True))
        return e / e.sum(1, keepdims=True)
    want = (1 - alpha) * np.longdouble(T) * soft(u / np.longdouble(T))
    s = soft(u)
    for r in range(m):
        for j in range(v + 1):
            want[r, int(idx2[r, j])] -= (1 - alpha) * np.longdouble(T) * p2[r, j]
        want[r] += alpha * s[r]
        want[r, int(labels[r])] -= alpha
    z, tv, ti, y = Z.to(DEV), t2.to(DEV), idx2.to(DEV), labels.to(DEV)
    stats = kq.kq_distill_loss(z, tv, ti, T, y, alpha)[1]
    for dz in (kq.kq_distill(z, tv, ti, temperature=T, labels=y, alpha=alpha)[1], kq.kq_distill_grad(z, tv, ti, stats, None, T, y, alpha)):
        got = dz.double().cpu().numpy().astype(np.longdouble)
        p = soft(t.double().numpy().astype(np.longdouble) / np.longdouble(T))
        byclass = np.zeros_like(p)
        np.put_along_axis(byclass, idx.numpy(), p, 1)
        tol = EPS * (64 * A * byclass + 128 * T * byclass + 64 * np.abs(want) + 64 * alpha * (s + 1))
        assert np.all(np.abs(got - want) <= tol), (np.abs(got - want) / tol).max()


@pytest.mark.parametrize("T", [20.0, 2.0 ** 20])
def test_equal_networks_have_no_loss(T):
    """Every difference is zero then, and the loss with it."""
    for v, top in ((100, 100), (3000, 64), (70001, 200)):
        Z, t, idx = rows(4, v, top, F32, v, noise=0.0)
        loss = kq.kq_distill(Z.to(DEV), t.to(DEV), idx.to(DEV), temperature=T)[0]
        assert torch.all(loss == 0)


@pytest.mark.parametrize("T", [20.0, 100.0, 2.0 ** 20])
def test_classes_outside_the_entries_count(T):
    """One more class, or as many again: the loss is T^2 times the logarithm of their share, and the sums' rounding of a few
    eps of S counts against that share."""
    for v, top, more in ((200, 100, 1), (200, 100, 100), (9001, 200, 1), (70001, 100, 3)):
        Z, t, idx = rows(4, v, top + more, F32, v + more)
        t, idx, z_idx = t[:, :top].contiguous(), idx[:, :top].contiguous(), idx
        z = Z.double().gather(1, z_idx).numpy().astype(np.longdouble) / np.longdouble(T)
        w = t.double().numpy().astype(np.longdouble) / np.longdouble(T)
        logp = w - np.log(np.exp(w).sum(1, keepdims=True))
        logq = (z - np.log(np.exp(z).sum(1, keepdims=True)))[:, :top]
        want = (np.exp(logp) * (logp - logq)).sum(1) * np.longdouble(T) ** 2
        share = np.exp(z)[:, top:].sum(1) / np.exp(z).sum(1)
        for loss in (kq.kq_distill(Z.to(DEV), t.to(DEV), idx.to(DEV), temperature=T)[0],
                     kq.kq_distill_loss(Z.to(DEV), t.to(DEV), idx.to(DEV), T)[0]):
            got = loss.double().cpu().numpy().astype(np.longdouble)
            # each of the two sums is off by at most 64 eps (as many roundings and exponentials follow each other), of S
            assert np.all(np.abs(got - want) <= (128 / share + 64) * EPS * want), (got, want, share)


def test_entries_that_underflow_and_classes_that_stand_twice():
    """Entries whose p or q is nothing in fp32, where p and q are close all the same; and classes that stand twice, whose sums of
    entries pass S: within the tolerance of a plain sum, R of tests/test_gpu_distill.py."""
    from test_gpu_distill import check
    m, v, top = 6, 300, 40
    g = gen(3)
    t = 2 * torch.randn(m, v, generator=g)
    values, idx = t.topk(top, 1)
    Z = t + 0.05 * torch.randn(m, v, generator=g)
    values[0, -3:] = values[0, 0] - 3000.0        # p of nothing, q as the others
    values[1, 5:] = values[1, 0] - 2000.0
    Z[2, idx[2, 20]] = -1500.0                    # q of nothing where p is small
    values[2, 20] = values[2, 0] - 300.0
    idx[3, 20:] = idx[3, :20]
    values[3, 20:] = values[3, :20]
    Z[4, idx[4, 0]] = 200.0                       # one class has everything in both
    values[4, 0] = 200.0
    Z[5] = -float("inf")                          # two entries of the only class
    Z[5, idx[5, 0]] = 1.0
    idx[5, 1:], idx[5, 1] = -1, idx[5, 0]
    for T in (1.0, 4.5, 10.0):
        loss, dz = kq.kq_distill(Z.to(DEV), values.to(DEV), idx.to(DEV), temperature=T)
        check(loss, dz, Z, values, idx, None, T, 0.0, torch.ones(m).double())
        check(kq.kq_distill_loss(Z.to(DEV), values.to(DEV), idx.to(DEV), T)[0], None, Z, values, idx, None, T, 0.0, torch.ones(m).double())


def test_with_labels_and_weights():
    Z, t, idx = rows(8, 120, 120, F32, 5)
    labels = idx[:, 3].contiguous()
    for T, alpha in ((100.0, 0.5), (1024.0, 2.0 ** -20)):
        loss, _, _, A = exact(Z, t, idx, T)
        ce = -torch.log_softmax(Z.double(), 1).gather(1, labels[:, None])[:, 0].numpy()
        got = kq.kq_distill(Z.to(DEV), t.to(DEV), idx.to(DEV), temperature=T, labels=labels.to(DEV), alpha=alpha)[0].double().cpu().numpy()
        tol = 32 * EPS * (1.5 * A * np.sqrt(loss) + (2 + A / T) * loss) + alpha * 64 * EPS * (ce + A + 8) + 2 * EPS * (loss + ce)
        assert np.all(np.abs(got - ((1 - alpha) * loss + alpha * ce)) <= tol)
