"""The C entry points of the 4-bit fully-connected layer and of the 8-bit checkpoints check their arguments on the
host before they touch HIP (no GPU needed)."""
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


def test_code_bytes():
    assert lib.kq_group_code_bytes(1, 1) == 1024
    assert lib.kq_group_code_bytes(16, 128) == 1024
    assert lib.kq_group_code_bytes(17, 129) == 4 * 1024
    assert lib.kq_group_code_bytes(4096, 25088) == 4096 * 25088 // 2
    assert lib.kq_group_code_bytes(0, 5) == 0 and lib.kq_group_code_bytes(MAXF + 1, 1) == 0
    assert lib.kq_group_code_bytes(1 << 20, 1 << 15) == 0          # more than 2^34 weights


def weights_refused(f):
    assert f(n=0) == ARG and f(k=0) == ARG and f(n=-3) == ARG
    assert f(n=MAXF + 1) == UNS and f(k=MAXF + 1) == UNS and f(n=1 << 20, k=1 << 15) == UNS
    for g in (0, 16, 48, 256, -32):
        assert f(group=g) == UNS
    assert f(codes=None) == ARG and f(codes=FAKE + 8) == ARG
    assert f(levels=FAKE + 1) == ARG


def test_quantize_and_reconstruct():
    q = dict(W=FAKE, type=0, ldw=100, n=20, k=100, group=32, levels=None, codes=FAKE, scales=FAKE, stream=None)
    f = lambda **kw: call("kq_quantize_groups", q, **kw)
    weights_refused(f)
    assert f(scales=None) == ARG and f(scales=FAKE + 1) == ARG
    assert f(type=3) == UNS and f(type=-1) == UNS
    assert f(W=None) == ARG and f(W=FAKE + 2) == ARG and f(type=1, W=FAKE + 1) == ARG and f(ldw=99) == ARG
    r = dict(codes=FAKE, scales=FAKE, levels=None, n=20, k=100, group=32, type=0, W=FAKE, ldw=100, stream=None)
    f = lambda **kw: call("kq_reconstruct_groups", r, **kw)
    weights_refused(f)
    assert f(type=5) == UNS and f(W=None) == ARG and f(W=FAKE + 2) == ARG and f(ldw=99) == ARG


def test_linear_and_its_gradient():
    lin = dict(X=FAKE, type=1, ldx=100, m=3, n=20, k=100, codes=FAKE, scales=FAKE, levels=None, group=32, bias=None, Y=FAKE,
               ldy=20, ws=None, wsb=0, stream=None)
    f = lambda **kw: call("kq_group_linear", lin, **kw)
    weights_refused(f)
    assert f(type=0) == UNS and f(type=4) == UNS
    assert f(m=-1) == ARG and f(m=MAXM + 1) == UNS and f(m=1 << 21, k=1 << 14, ldx=1 << 14) == UNS
    assert f(X=None) == ARG and f(X=FAKE + 1) == ARG and f(ldx=99) == ARG
    assert f(Y=None) == ARG and f(ldy=19) == ARG and f(bias=FAKE + 2) == ARG
    assert f(m=0, X=None, Y=None) == OK                            # nothing to do
    need = lib.kq_group_linear_workspace_bytes(FAKE, 100, 17, 20, 100)
    assert need > 0 and need % 256 == 0                            # 100 columns: rows of X are copied
    assert f(m=17) == WS and f(m=17, ws=FAKE, wsb=need - 1) == WS and f(m=17, ws=FAKE + 16, wsb=need) == WS
    assert lib.kq_group_linear_workspace_bytes(FAKE, 128, 17, 20, 128) == 0
    assert lib.kq_group_linear_workspace_bytes(FAKE + 8, 128, 17, 20, 128) > 0
    assert lib.kq_group_linear_workspace_bytes(FAKE, 128, 0, 20, 128) == 0
    gi = dict(dY=FAKE, type=2, ldy=24, m=3, n=24, k=100, codes=FAKE, scales=FAKE, levels=None, group=32, dX=FAKE, ldx=100,
              ws=None, wsb=0, stream=None)
    f = lambda **kw: call("kq_group_linear_grad_input", gi, **kw)
    weights_refused(f)
    assert f(type=0) == UNS and f(m=-1) == ARG and f(m=MAXM + 1) == UNS
    assert f(dY=None) == ARG and f(ldy=23) == ARG and f(dX=None) == ARG and f(ldx=99) == ARG and f(dX=FAKE + 1) == ARG
    assert f(m=0, dY=None, dX=None) == OK
    assert f(dY=FAKE + 2) == WS                                    # copied: needs the workspace


def test_checkpoints():
    pk = dict(X=FAKE, type=0, ldx=100, m=3, k=100, q=FAKE, exps=FAKE, stream=None)
    f = lambda **kw: call("kq_checkpoint_pack", pk, **kw)
    assert f(k=0) == ARG and f(m=-1) == ARG and f(k=MAXF + 1) == UNS and f(m=MAXM + 1) == UNS and f(type=3) == UNS
    assert f(X=None) == ARG and f(X=FAKE + 2) == ARG and f(ldx=99) == ARG
    assert f(q=None) == ARG and f(q=FAKE + 4) == ARG and f(exps=None) == ARG
    assert f(m=0, X=None, q=None, exps=None) == OK
    rs = dict(q=FAKE, exps=FAKE, m=3, k=100, type=1, X=FAKE, ldx=100, stream=None)
    f = lambda **kw: call("kq_checkpoint_restore", rs, **kw)
    assert f(k=0) == ARG and f(m=MAXM + 1) == UNS and f(type=3) == UNS and f(X=FAKE + 1) == ARG and f(ldx=99) == ARG
    assert f(q=FAKE + 4) == ARG and f(exps=None) == ARG and f(m=0, X=None, q=None, exps=None) == OK


def test_gradients_from_a_checkpoint():
    need = lib.kq_checkpoint_grad_workspace_bytes(7, 20, 100, 32)
    assert need > 0 and need % 256 == 0 and lib.kq_checkpoint_grad_workspace_bytes(7, 20, 100, 0) > 0
    assert lib.kq_checkpoint_grad_workspace_bytes(7, 20, 100, 33) == 0
    assert lib.kq_checkpoint_grad_workspace_bytes(0, 20, 100, 32) == 0
    gs = dict(dY=FAKE, type=1, ldy=20, m=7, n=20, k=100, q=FAKE, exps=FAKE, codes=FAKE, levels=None, group=32, ds=FAKE, db=None,
              ws=FAKE, wsb=need, stream=None)
    f = lambda **kw: call("kq_checkpoint_grad_scales", gs, **kw)
    weights_refused(f)
    assert f(type=0) == UNS and f(m=-1) == ARG and f(m=MAXM + 1) == UNS
    assert f(dY=None) == ARG and f(ldy=19) == ARG and f(q=None) == ARG and f(q=FAKE + 1) == ARG and f(exps=None) == ARG
    assert f(ds=None) == ARG and f(ds=FAKE + 2) == ARG and f(db=FAKE + 2) == ARG
    assert f(ws=None) == WS and f(wsb=need - 1) == WS and f(ws=FAKE + 64) == WS
    need = lib.kq_checkpoint_grad_workspace_bytes(7, 20, 100, 0)
    gw = dict(dY=FAKE, type=2, ldy=20, m=7, n=20, k=100, q=FAKE, exps=FAKE, dW=FAKE, lddw=100, db=None, ws=FAKE, wsb=need, stream=None)
    f = lambda **kw: call("kq_checkpoint_grad_weight", gw, **kw)
    assert f(n=0) == ARG and f(k=MAXF + 1) == UNS and f(type=0) == UNS and f(lddw=99) == ARG and f(dW=None) == ARG
    assert f(dW=FAKE + 2) == ARG and f(wsb=need - 1) == WS and f(m=MAXM + 1) == UNS


def test_python_refuses_host_tensors():
    import torch
    X = torch.zeros(4, 64, dtype=torch.bfloat16)
    for f in (lambda: kq.kq_quantize_groups(X), lambda: kq.kq_checkpoint_pack(X), lambda: kq.kq_group_linear(X, X, X)):
        with pytest.raises(TypeError):
            f()
