"""The operators of a worker's local step without a GPU: what they refuse, and what they ask for as scratch."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def P():
    import paper_1709_09393_b200 as pkg
    return pkg


INVALID, WORKSPACE = -1, -2
A = ctypes.c_void_p(0x10000)          # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x10002)
BYTE = ctypes.c_void_p(0x10001)
BIG = 1 << 40


def test_workspace_sizes(P):
    assert P.layernorm_workspace_bytes(0, 8) >= 64
    assert P.layernorm_workspace_bytes(100, 1000) >= 100 * 2 * 1000 * 4
    assert P.layernorm_workspace_bytes(1, 0) == 0 and P.layernorm_workspace_bytes(2 ** 31, 8) == 0
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        sizes = [P.linear_workspace_bytes(m, 300, 500, dtype) for m in (0, 1, 100, 10000)]
        assert all(s > 0 for s in sizes)
        assert P.linear_workspace_bytes(1, 0, 5, dtype) == 0 and P.linear_workspace_bytes(1, 5, 2 ** 31, dtype) == 0
    assert P.lib.slimdp_linear_workspace_bytes(1, 1, 1, 7) == 0
    with pytest.raises(TypeError):
        P.linear_workspace_bytes(1, 1, 1, torch.float64)


def test_layernorm_refusals(P):
    f = P.lib.slimdp_layernorm_forward
    ok = [A, 8, 4, 8, 1, A, A, 1e-5, A, 8, A, A, None]

    def with_(**kw):
        names = ["x", "ldx", "rows", "dim", "type", "gamma", "beta", "eps", "y", "ldy", "mean", "rstd", "stream"]
        return f(*[kw.get(n, v) for n, v in zip(names, ok)])

    for bad in (dict(x=None), dict(y=None), dict(ldx=7), dict(ldy=7), dict(dim=0), dict(rows=2 ** 31), dict(type=3),
                dict(type=-1), dict(eps=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(x=BYTE),
                dict(gamma=ODD), dict(beta=ODD), dict(mean=ODD), dict(rstd=BYTE), dict(type=0, x=ODD),
                dict(dim=2 ** 31, ldx=2 ** 31, ldy=2 ** 31), dict(ldx=2 ** 63)):
        assert with_(**bad) == INVALID, bad
    assert with_(rows=0, x=None, y=None) == 0             # nothing to do, nothing enqueued
    g = P.lib.slimdp_layernorm_backward
    ok_b = [A, 8, A, 8, 4, 8, 1, A, A, A, A, 8, A, A, 0, A, 1 << 20, None]
    names = ["dy", "lddy", "x", "ldx", "rows", "dim", "type", "gamma", "mean", "rstd", "dx", "lddx", "dgamma", "dbeta",
             "accumulate", "ws", "ws_bytes", "stream"]

    def back(**kw):
        return g(*[kw.get(n, v) for n, v in zip(names, ok_b)])

    for bad in (dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(lddy=1), dict(ldx=1),
                dict(lddx=1), dict(ws=None), dict(ws=ctypes.c_void_p(0x10008)), dict(dgamma=ODD), dict(type=9)):
        assert back(**bad) == INVALID, bad
    assert back(ws_bytes=16) == WORKSPACE


def test_linear_refusals(P):
    lib = P.lib
    fwd = ["x", "ldx", "w", "ldw", "bias", "residual", "ldr", "m", "n", "k", "type", "act", "y", "ldy", "z", "ldz", "ws",
           "ws_bytes", "stream"]
    ok = [A, 8, A, 8, A, A, 16, 4, 16, 8, 1, 0, A, 16, A, 16, A, BIG, None]

    def forward(**kw):
        return lib.slimdp_linear_forward(*[kw.get(n, v) for n, v in zip(fwd, ok)])

    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(ldx=7), dict(ldw=7), dict(ldr=15), dict(ldy=15),
                dict(ldz=15), dict(n=0), dict(k=0), dict(m=2 ** 31), dict(type=3), dict(act=5), dict(act=-1),
                dict(x=BYTE), dict(bias=ODD), dict(residual=BYTE), dict(z=BYTE), dict(ws=None),
                dict(ws=ctypes.c_void_p(0x10080))):
        assert forward(**bad) == INVALID, bad
    assert forward(ws_bytes=0) == WORKSPACE
    bwd = ["dy", "lddy", "w", "ldw", "z", "ldz", "add", "ldadd", "m", "n", "k", "type", "act", "dx", "lddx", "ws",
           "ws_bytes", "stream"]
    okb = [A, 16, A, 8, A, 8, A, 8, 4, 16, 8, 2, 2, A, 8, A, BIG, None]

    def backward(**kw):
        return lib.slimdp_linear_backward_input(*[kw.get(n, v) for n, v in zip(bwd, okb)])

    for bad in (dict(dy=None), dict(w=None), dict(dx=None), dict(z=None), dict(lddy=15), dict(ldw=7), dict(ldz=7),
                dict(ldadd=7), dict(lddx=7), dict(act=9), dict(ws=None)):
        assert backward(**bad) == INVALID, bad
    assert backward(ws_bytes=0) == WORKSPACE
    wgt = ["dy", "lddy", "x", "ldx", "m", "n", "k", "type", "dw", "lddw", "db", "accumulate", "ws", "ws_bytes", "stream"]
    okw = [A, 16, A, 8, 4, 16, 8, 1, A, 8, A, 0, A, BIG, None]

    def weight(**kw):
        return lib.slimdp_linear_backward_weight(*[kw.get(n, v) for n, v in zip(wgt, okw)])

    for bad in (dict(dy=None), dict(x=None), dict(dw=None), dict(dw=ODD), dict(db=ODD), dict(lddy=15), dict(ldx=7),
                dict(lddw=7), dict(ws=None), dict(n=0)):
        assert weight(**bad) == INVALID, bad
    assert weight(ws_bytes=0) == WORKSPACE
    act = lib.slimdp_activation_backward
    assert act(None, 8, A, 8, 4, 8, 1, 1, A, 8, None) == INVALID
    assert act(A, 8, None, 8, 4, 8, 1, 1, A, 8, None) == INVALID
    assert act(A, 8, A, 7, 4, 8, 1, 1, A, 8, None) == INVALID
    assert act(A, 8, A, 8, 4, 8, 1, 7, A, 8, None) == INVALID


def test_distill_refusals(P):
    names = ["logits", "ldl", "rows", "vocab", "type", "idx", "teacher", "teacher_type", "top", "label", "weight", "T",
             "kd", "ce", "loss", "dlogits", "ldd", "stream"]
    ok = [A, 100, 4, 100, 1, A, A, 0, 5, A, A, 2.0, 1.0, 0.5, A, A, 100, None]

    def f(**kw):
        return P.lib.slimdp_distill(*[kw.get(n, v) for n, v in zip(names, ok)])

    for bad in (dict(logits=None), dict(ldl=99), dict(ldd=99), dict(vocab=0), dict(rows=2 ** 31), dict(type=3),
                dict(teacher_type=3), dict(top=1025), dict(idx=None), dict(teacher=None), dict(T=0.0), dict(T=-1.0),
                dict(T=float("inf")), dict(T=float("nan")), dict(kd=float("nan")), dict(ce=float("inf")),
                dict(loss=None), dict(loss=ODD), dict(idx=ODD), dict(label=ODD), dict(weight=ODD), dict(teacher=ODD),
                dict(logits=BYTE), dict(dlogits=BYTE), dict(ldd=101)):
        assert f(**bad) == INVALID, bad
    assert f(rows=0, logits=None, dlogits=None, idx=None, teacher=None, loss=None) == 0


def test_binding_checks_tensors(P):
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        P.slimdp_layernorm_forward(x, None, None, 1e-5, x)               # not on the GPU
    with pytest.raises(TypeError):
        P.slimdp_linear_forward(x, x, None, x, x)
    with pytest.raises(TypeError):
        P.slimdp_distill(x, None, None, torch.zeros(4))
