"""The C entry points of the 8-bit fully-connected layer and of distillation check their arguments on the host before they
touch HIP (no GPU needed)."""
import ctypes
import math

import pytest

kq = pytest.importorskip("paper_2003_05148_amd")
lib = kq.lib
FAKE = 0x10000  # well aligned, never dereferenced on these paths
OK, ARG, UNS, WS = kq.KQ_OK, kq.KQ_ERR_ARG, kq.KQ_ERR_UNSUPPORTED, kq.KQ_ERR_WORKSPACE
MAXF, MAXM = 1 << 24, 1 << 22


def call(name, defaults, **kw):
    a = dict(defaults)
    assert set(kw) <= set(a), kw
    a.update(kw)
    return getattr(lib, name)(*a.values())


def test_quantize_and_reconstruct():
    q = dict(X=FAKE, type=0, ldx=100, m=20, k=100, rows=1, values=FAKE, exps=FAKE, stream=None)
    r = dict(values=FAKE, exps=FAKE, m=20, k=100, rows=128, type=0, X=FAKE, ldx=100, stream=None)
    for name, d in (("kq_quantize_blocks", q), ("kq_reconstruct_blocks", r)):
        f = lambda **kw: call(name, d, **kw)
        assert f(k=0) == ARG and f(m=-1) == ARG
        assert f(k=MAXF + 1) == UNS and f(m=MAXF + 1) == UNS and f(m=1 << 20, k=1 << 15) == UNS
        for rows in (0, 2, 64, 256, -1):
            assert f(rows=rows) == UNS
        assert f(type=3) == UNS and f(type=-1) == UNS
        assert f(X=None) == ARG and f(X=FAKE + 2) == ARG and f(X=FAKE + 1, type=1) == ARG and f(ldx=99) == ARG
        assert f(values=None) == ARG and f(values=FAKE + 8) == ARG and f(exps=None) == ARG
        assert f(m=0, X=None, values=None, exps=None) == OK


def sizes_refused(f, weights=True):
    assert f(n=0) == ARG and f(k=0) == ARG and f(n=-3) == ARG and f(m=-1) == ARG
    assert f(n=MAXF + 1) == UNS and f(k=MAXF + 1) == UNS and f(n=1 << 20, k=1 << 15) == UNS and f(m=MAXM + 1) == UNS
    assert f(m=1 << 21, n=1 << 14, k=1) == UNS
    if weights:
        assert f(values=None) == ARG and f(values=FAKE + 8) == ARG and f(exps=None) == ARG


def test_linear():
    lin = dict(X=FAKE, xt=1, ldx=100, xe=None, m=3, n=20, k=100, values=FAKE, exps=FAKE, bias=None, Y=FAKE, yt=1, ldy=20, ws=None,
               wsb=0, stream=None)
    f = lambda **kw: call("kq_block_linear", lin, **kw)
    sizes_refused(f)
    assert f(xt=4) == UNS and f(xt=-1) == UNS and f(yt=3) == UNS and f(yt=7) == UNS
    assert f(X=None) == ARG and f(X=FAKE + 1) == ARG and f(ldx=99) == ARG and f(xe=FAKE) == ARG
    assert f(xt=3, xe=None, ldx=128) == ARG and f(xt=3, xe=FAKE, ldx=100) == ARG and f(xt=3, xe=FAKE, ldx=128, X=FAKE + 8) == ARG
    assert f(Y=None) == ARG and f(Y=FAKE + 2, yt=0) == ARG and f(ldy=19) == ARG and f(bias=FAKE + 2) == ARG
    assert f(m=0, X=None, Y=None) == OK
    w = lib.kq_block_linear_workspace_bytes
    need = w(1, 1, 1100, 20, 100)
    assert need > 0 and need % 256 == 0
    assert f(m=1100) == WS and f(m=1100, ws=FAKE, wsb=need - 1) == WS and f(m=1100, ws=FAKE + 16, wsb=need) == WS
    assert w(1, 1, 0, 20, 100) == 0 and w(4, 1, 1100, 20, 100) == 0 and w(1, 3, 1100, 20, 100) == 0 and w(1, 1, 1100, 0, 100) == 0
    assert w(3, 1, 1100, 20, 100) < need


def test_gradients():
    need = lib.kq_block_linear_grad_input_workspace_bytes(1, 3, 24, 100)
    gi = dict(dY=FAKE, type=1, ldy=24, m=3, n=24, k=100, values=FAKE, exps=FAKE, dX=FAKE, ldx=100, ws=FAKE, wsb=need, stream=None)
    f = lambda **kw: call("kq_block_linear_grad_input", gi, **kw)
    sizes_refused(f)
    assert f(type=3) == UNS and f(dY=None) == ARG and f(ldy=23) == ARG and f(dX=None) == ARG and f(dX=FAKE + 1) == ARG and f(ldx=99) == ARG
    assert f(ws=None) == WS and f(wsb=need - 1) == WS and f(ws=FAKE + 64) == WS
    assert f(m=0, dY=None, dX=None, ws=None) == OK
    w = lib.kq_block_linear_grad_weight_workspace_bytes
    need = w(0, 7, 24, 100)
    assert need > 0 and need % 256 == 0 and w(0, 0, 24, 100) == 0 and w(3, 7, 24, 100) == 0
    gw = dict(dY=FAKE, type=1, ldy=24, m=7, n=24, k=100, values=FAKE, exps=FAKE, dW=FAKE, wt=0, lddw=100, db=None, ws=FAKE,
              wsb=need, stream=None)
    f = lambda **kw: call("kq_block_linear_grad_weight", gw, **kw)
    sizes_refused(f)
    assert f(type=3) == UNS and f(wt=3) == UNS and f(dY=None) == ARG and f(ldy=23) == ARG
    assert f(dW=None) == ARG and f(dW=FAKE + 2) == ARG and f(lddw=99) == ARG and f(db=FAKE + 1) == ARG
    assert f(ws=None) == WS and f(wsb=need - 1) == WS and f(ws=FAKE + 64) == WS


def test_distill():
    def args(**kw):
        a = dict(Z=FAKE, type=1, ldz=50, m=4, v=50, top_values=FAKE, top_type=0, top_idx=FAKE, idx_bytes=8, top=5, labels=FAKE,
                 label_bytes=8, temperature=2.0, alpha=0.5)
        assert set(kw) <= set(a)
        a.update(kw)
        return kq.KqDistillArgs(*a.values())

    # outputs that are refused come after the arguments' own checks
    calls = [lambda a: lib.kq_distill(a, None, 1.0, None, FAKE, 50, None, 0, None),
             lambda a: lib.kq_distill(a, None, 1.0, FAKE, None, 50, None, 0, None),
             lambda a: lib.kq_distill(a, FAKE + 1, 1.0, FAKE, FAKE, 50, None, 0, None),
             lambda a: lib.kq_distill(a, None, 1.0, FAKE + 2, FAKE, 50, None, 0, None),
             lambda a: lib.kq_distill(a, None, 1.0, FAKE, FAKE, 49, None, 0, None),
             lambda a: lib.kq_distill_loss(a, None, FAKE, None, 0, None), lambda a: lib.kq_distill_loss(a, FAKE, None, None, 0, None),
             lambda a: lib.kq_distill_loss(a, FAKE, FAKE + 2, None, 0, None),
             lambda a: lib.kq_distill_grad(a, None, None, 1.0, FAKE, 50, None),
             lambda a: lib.kq_distill_grad(a, FAKE, FAKE + 2, 1.0, FAKE, 50, None),
             lambda a: lib.kq_distill_grad(a, FAKE, None, 1.0, FAKE + 1, 50, None)]
    for f in calls:
        assert f(ctypes.byref(args())) == ARG
        assert f(None) == ARG
        for kw in (dict(m=-1), dict(v=0), dict(top=0), dict(Z=None), dict(Z=FAKE + 1), dict(ldz=49), dict(top_values=None),
                   dict(top_values=FAKE + 2), dict(top_idx=None), dict(top_idx=FAKE + 4), dict(labels=None), dict(labels=FAKE + 4),
                   dict(alpha=-0.1), dict(alpha=1.1), dict(alpha=math.nan)):
            assert f(ctypes.byref(args(**kw))) == ARG, kw
        for kw in (dict(m=MAXM + 1), dict(v=MAXF + 1), dict(m=1 << 20, v=(1 << 15) + 1, ldz=1 << 16), dict(top=257), dict(type=3), dict(top_type=3), dict(idx_bytes=2),
                   dict(label_bytes=2), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan),
                   dict(temperature=math.inf), dict(temperature=2.0 ** -11), dict(temperature=2.0 ** 21)):
            assert f(ctypes.byref(args(**kw))) == UNS, kw
    assert lib.kq_distill(ctypes.byref(args(m=0, Z=None)), None, 1.0, None, None, 50, None, 0, None) == OK


def test_python_refuses_host_tensors():
    import torch
    X = torch.zeros(4, 64, dtype=torch.bfloat16)
    for f in (lambda: kq.kq_quantize_blocks(X), lambda: kq.kq_block_linear(X, X, X), lambda: kq.kq_block_linear_grad_input(X, X, X, 64),
              lambda: kq.kq_block_linear_grad_weight(X, X, X, 64), lambda: kq.kq_distill(X, X, X), lambda: kq.kq_distill_loss(X, X, X),
              lambda: kq.kq_distill_grad(X, X, X, X)):
        with pytest.raises(TypeError):
            f()
