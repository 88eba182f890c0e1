"""Distillation of rows that are cut into segments, and of rows just short of it: the sizes that tests/test_distill_plan.py holds
to their plan.  Formulas and tolerances: those of tests/test_gpu_distill.py."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_distill_plan import CUT, N, WHOLE, segments
from test_gpu_distill import BF, DEV, F32, HF, check, gen, logits, on

kq = pytest.importorskip("paper_2003_05148_amd")
TYPES = [F32, BF, HF]


def spread(m, v, top, dtype, seed):
    """Entries all over the row, every class at least twice: at places 64 and more apart and in other segments than its
    neighbours in the list, the row's first and last classes (single values, where rows begin anywhere) among them; the label
    is an entry, no entry, or absent."""
    Z, values, idx, labels = logits(m, v, top, dtype, seed, absent=0.0)
    half = top // 2
    where = torch.randint(0, v, (m, half), generator=gen(seed + 1))
    where[:, 0], where[:, 1], where[:, 2] = 0, v - 1, v - 2
    where[:, 3] = 1
    idx[:, :half], idx[:, half:2 * half] = where, where.flip(1)
    idx[:, half // 2] = idx[:, 0]
    values = torch.randn(m, top, generator=gen(seed + 2)) + values.mean(1, keepdim=True)
    idx[m - 1, ::3] = -1
    labels = where[:, 4 % half].clone()
    labels[0] = v - 1
    if m > 2:
        labels[1], labels[2] = 0, -100
    if m > 3:
        labels[3] = (int(labels[3]) + v // 2) % v
    return Z, values, idx, labels


@pytest.mark.parametrize("T,alpha", [(1.0, 0.0), (2.0, 0.4), (1.0, 0.5), (2.5, 1.0), (9.0, 0.25)])
@pytest.mark.parametrize("m,v,kind", CUT + WHOLE)
def test_classes_that_stand_twice(m, v, kind, T, alpha):
    """In one call, in place, into other rows, and in two calls: every class has all of its entries and its label's term."""
    dtype, top = TYPES[kind], 150
    Z, values, idx, labels = spread(m, v, top, dtype, v)
    rows = sorted({0, 1 % m, 2 % m, 3 % m, m // 2, m - 1})
    pick = lambda x: x[rows]
    d = 0.5 + torch.rand(m, generator=gen(1))
    z, tv, ti, y, dl = on(Z, values, idx, labels, d)
    how = dict(temperature=T, labels=y, alpha=alpha)

    def near(loss, dz):
        check(None if loss is None else loss[rows], dz[rows], pick(Z), pick(values), pick(idx), pick(labels), T, alpha, pick(d).double())
    loss, dz = kq.kq_distill(z, tv, ti, dloss=dl, **how)
    near(loss, dz)
    inplace = z.clone()
    l2, _ = kq.kq_distill(inplace, tv, ti, dloss=dl, dZ=inplace, **how)
    assert torch.equal(l2, loss) and torch.equal(inplace, dz)
    wide = torch.full((m, v + 7), 5.0, dtype=dtype, device=DEV)
    kq.kq_distill(z, tv, ti, dloss=dl, dZ=wide[:, 3:3 + v], **how)
    assert torch.equal(wide[:, 3:3 + v], dz) and torch.all(wide[:, :3] == 5) and torch.all(wide[:, 3 + v:] == 5)
    l3, stats = kq.kq_distill_loss(z, tv, ti, **how)
    g = kq.kq_distill_grad(z, tv, ti, stats, dloss=dl, **how)
    near(l3, g)
    inplace.copy_(z)
    kq.kq_distill_grad(inplace, tv, ti, stats, dloss=dl, dZ=inplace, **how)
    assert torch.equal(inplace, g)


@pytest.mark.parametrize("m,v,kind", CUT[:1] + CUT[4:])
def test_segments_that_are_masked_out(m, v, kind):
    """All classes but those of one segment, the first or the last, masked out; and all entries in it."""
    dtype = TYPES[kind]
    Z, values, idx, labels = spread(m, v, 40, dtype, v + 1)
    per = -(-v // segments(m, v, kind))
    for first in (0, v - per + 2 * N[kind]):
        M = torch.full_like(Z, -float("inf"))
        M[:, first:first + per - 2 * N[kind]] = Z[:, first:first + per - 2 * N[kind]]
        i = first + idx % (per - 2 * N[kind])
        y = first + labels.abs() % (per - 2 * N[kind])
        z, tv, ti, yd = on(M, values, i, y)
        loss, dz = kq.kq_distill(z, tv, ti, temperature=2.0, labels=yd, alpha=0.3)
        r = [0, m - 1]
        check(loss[r], dz[r], M[r], values[r], i[r], y[r], 2.0, 0.3, torch.ones(2).double())
        assert torch.all(dz.cpu()[torch.isinf(M)] == 0)


@pytest.mark.parametrize("m,v,kind", [CUT[0], CUT[5]])
def test_streams_and_graphs(m, v, kind):
    dtype = TYPES[kind]
    Z, values, idx, labels = spread(m, v, 30, dtype, v)
    z, tv, ti, y = on(Z, values, idx, labels)

    def step():
        return kq.kq_distill(z, tv, ti, temperature=2.0, labels=y, alpha=0.3)
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
        z.copy_(logits(m, v, 6, dtype, seed)[0])
        want = [t.clone() for t in step()]
        g.replay()
        step()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
