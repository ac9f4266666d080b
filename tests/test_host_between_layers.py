"""Refusals of the calls between two aggregations and between the clipped gradient and the weight, on the host: every call here returns before anything is launched."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib(hgnn):
    return hgnn.load()


A, B, C, D, E = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000  # stand for device addresses
F16, F32 = 0, 1
NONE, RMS, LAYER = 0, 1, 2
NAN, INF = float("nan"), float("inf")


def block(hgnn, post=LAYER, post_w=A, post_b=A, gate=A, gate_rows=None, ld_gate=0, alpha=1.0, pre=RMS, pre_w=A, pre_b=A, eps=1e-5):
    return hgnn.binding._BlockStruct(post, post_w, post_b, gate, gate_rows, ld_gate, alpha, pre, pre_w, pre_b, eps)


def test_norm_refuses(lib, hgnn):
    EINVAL, EUNSUP = hgnn.HGNN_EINVAL, hgnn.HGNN_EUNSUPPORTED

    def call(n=4, F=8, kind=F16, R=B, ldr=8, Y=C, ldy=8, H=D, ldh=8, Z=E, ldz=8, none=False, **b):
        return lib.hgnn_residual_norm(n, F, None if none else block(hgnn, **b), kind, R, ldr, Y, ldy, H, ldh, Z, ldz, None)
    for bad in (dict(n=-1), dict(F=0), dict(none=True), dict(kind=2), dict(post=3), dict(pre=-1), dict(ldr=7), dict(ldy=7), dict(ldh=7), dict(ldz=7), dict(alpha=NAN), dict(alpha=INF),
                dict(eps=0.0), dict(eps=1e-39), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(post=NONE), dict(post=NONE, post_w=None), dict(pre=NONE, Z=None), dict(pre=NONE, pre_w=None, pre_b=None),
                dict(gate_rows=A, ld_gate=8), dict(gate=None, gate_rows=A, ld_gate=7), dict(Y=None), dict(Z=None), dict(R=None, Y=None, post=NONE, post_w=None, post_b=None, gate=None),
                dict(R=B + 1), dict(kind=F32, R=B + 2), dict(Y=C + 1), dict(H=D + 1), dict(Z=E + 1), dict(post_w=A + 2), dict(post_b=A + 1), dict(gate=A + 2), dict(pre_w=A + 3), dict(pre_b=A + 2),
                dict(gate=None, gate_rows=A + 1, ld_gate=8), dict(H=B, ldh=16), dict(H=None, Z=None, pre=NONE, pre_w=None, pre_b=None)):
        assert call(**bad) == EINVAL, bad
        assert b"hgnn_residual_norm" in lib.hgnn_last_error()
    assert call(F=8193, ldr=9000, ldy=9000, ldh=9000, ldz=9000) == EUNSUP and call(n=(1 << 40) + 1) == EUNSUP
    assert call(n=0, R=None, Y=None, H=None, Z=None) == 0  # nothing to do


def test_norm_gradient_refuses(lib, hgnn):
    EINVAL, EUNSUP = hgnn.HGNN_EINVAL, hgnn.HGNN_EUNSUPPORTED
    need = hgnn.hgnn_residual_norm_grad_workspace(4, 8)
    assert need > 0

    def call(n=4, F=8, kind=F16, H=B, ldh=8, Y=C, ldy=8, dH=D, lddh=8, dZ=E, lddz=8, dR=A, lddr=8, dY=A, lddy=8, dgate=A, dgate_rows=None, ldd=0, dpw=A, dpb=A, dqw=A, dqb=A, ws=B, bytes=need, no=False, **b):
        g = hgnn.binding._BlockGradStruct(dR, lddr, dY, lddy, dgate, dgate_rows, ldd, dpw, dpb, dqw, dqb)
        return lib.hgnn_residual_norm_grad(n, F, block(hgnn, **b), kind, H, ldh, Y, ldy, dH, lddh, dZ, lddz, None if no else g, ws, bytes, None)
    rows = dict(gate=None, gate_rows=A, ld_gate=8, dgate=None)
    for bad in (dict(n=-1), dict(F=0), dict(no=True), dict(kind=5), dict(post=3), dict(ldh=7), dict(ldy=7), dict(lddh=7), dict(lddz=7), dict(lddr=7), dict(lddy=7), dict(H=None), dict(dZ=None), dict(Y=None),
                dict(eps=0.0), dict(ws=None), dict(bytes=need - 1), dict(ws=B + 8), dict(gate=None), dict(rows, dgate=A), dict(dgate_rows=A, ldd=8), dict(rows, dgate_rows=A, ldd=7),
                dict(post=NONE, post_w=None, post_b=None), dict(pre=NONE, pre_w=None, pre_b=None), dict(pre=NONE, pre_w=None, pre_b=None, dqw=None, dqb=None),
                dict(pre=NONE, pre_w=None, pre_b=None, dqw=None, dqb=None, dZ=None, dH=None), dict(H=B + 1), dict(kind=F32, dH=D + 2), dict(dZ=E + 1), dict(dR=A + 1), dict(dY=A + 1), dict(dgate=A + 1),
                dict(dpw=A + 2), dict(dpb=A + 2), dict(dqw=A + 2), dict(dqb=A + 2), dict(Y=C + 1), dict(dR=D, lddr=16)):
        assert call(**bad) == EINVAL, bad
        assert b"hgnn_residual_norm_grad" in lib.hgnn_last_error()
    assert call(F=8193, ldh=9000, ldy=9000, lddh=9000, lddz=9000, lddr=9000, lddy=9000) == EUNSUP
    nothing = dict(dgate=None, dpw=None, dpb=None, dqw=None, dqb=None, ws=None, bytes=0)
    assert call(n=0, **nothing) == 0
    assert hgnn.hgnn_residual_norm_grad_workspace(0, 8) == 0 and hgnn.hgnn_residual_norm_grad_workspace(4, 8193) == 0


def test_gated_refuses(lib, hgnn):
    EINVAL, EUNSUP = hgnn.HGNN_EINVAL, hgnn.HGNN_EUNSUPPORTED
    need, need2 = hgnn.hgnn_gated_workspace(100, 4096, 64), hgnn.hgnn_gated_grad_workspace(100, 4096, 64)
    assert 0 < need <= need2

    def call(n=100, K=4096, F=64, act=0, X=A, ldx=4096, Wg=B, Wu=C, ldw=64, trans=0, Y=D, ldy=64, ws=E, bytes=need):
        return lib.hgnn_gated(n, K, F, act, X, ldx, Wg, Wu, ldw, trans, Y, ldy, ws, bytes, None)

    def grad(n=100, K=4096, F=64, act=0, X=A, ldx=4096, Wg=B, Wu=C, ldw=64, trans=0, Y=D, ldy=64, dX=A, lddx=4096, dWg=B, dWu=C, lddw=64, ws=E, bytes=need2):
        return lib.hgnn_gated_grad(n, K, F, act, X, ldx, Wg, Wu, ldw, trans, Y, ldy, dX, lddx, dWg, dWu, lddw, ws, bytes, None)
    for f, who in ((call, b"hgnn_gated"), (grad, b"hgnn_gated_grad")):
        for bad in (dict(n=-1), dict(K=0), dict(F=0), dict(act=4), dict(act=-1), dict(ldx=4088), dict(ldw=56), dict(ldy=56), dict(trans=1), dict(X=None), dict(Wg=None), dict(Wu=None), dict(Y=None), dict(ws=None),
                    dict(bytes=need - 1), dict(ws=E + 8)):
            assert f(**bad) == EINVAL, bad
            assert who in lib.hgnn_last_error()
        for no in (dict(X=A + 2), dict(Wg=B + 8), dict(Wu=C + 2), dict(Y=D + 4), dict(ldx=4100), dict(ldw=66), dict(ldy=68), dict(K=65537, ldx=65544),
                   dict(F=65537, ldw=65544, ldy=65544), dict(n=1 << 31), dict(ldx=(1 << 22) + 8), dict(ldw=1 << 23),
                   dict(ldy=1 << 40)):
            assert f(**no) == EUNSUP, no
    for bad in (dict(dWg=None), dict(dWu=None), dict(dWu=B), dict(lddx=4088), dict(lddw=56)):
        assert grad(**bad) == EINVAL, bad
    for no in (dict(dX=A + 2), dict(dWg=B + 2), dict(dWu=C + 2), dict(lddx=4100), dict(lddw=68)):
        assert grad(**no) == EUNSUP, no
    assert call(n=0, X=None, Y=None, ws=None) == 0 and grad(n=0, dWg=None, dWu=None, X=None, ws=None) == 0
    assert grad(dX=None, dWg=None, dWu=None) == 0  # nothing is wanted
    for f in (lib.hgnn_gated_workspace, lib.hgnn_gated_grad_workspace):
        assert f(0, 8, 8) == 0 and f(-1, 8, 8) == 0 and f(1 << 31, 8, 8) == 0 and f(8, 0, 8) == 0 and f(8, 8, 65537) == 0


def test_orthogonalize_refuses(lib, hgnn):
    from paper_2411_01109_amd.binding import _GradStruct
    EINVAL, EUNSUP = hgnn.HGNN_EINVAL, hgnn.HGNN_EUNSUPPORTED

    def m(grad=A, out=None, rows=4, cols=8, ld=8, ld_out=8, kind=F32, out_kind=F32):
        return _GradStruct(grad, out, rows, cols, ld, ld_out, kind, out_kind)
    need = lib.hgnn_orthogonalize_workspace(1, (_GradStruct * 1)(m()))
    assert need > 0

    def call(*mats, steps=1, coef=(1.5, -0.5, 0.0), scales=None, ws=E, bytes=need, count=None):
        a = (_GradStruct * max(len(mats), 1))(*mats)
        return lib.hgnn_orthogonalize(len(mats) if count is None else count, a, steps, None if coef is None else (ctypes.c_float * len(coef))(*coef),
                                      None if scales is None else (ctypes.c_float * len(scales))(*scales), ws, bytes, None)
    for bad in (dict(rows=-1), dict(cols=-1), dict(kind=2), dict(ld=7), dict(grad=None), dict(grad=A + 2), dict(kind=F16, grad=A + 1), dict(out=C, out_kind=2), dict(out=C, ld_out=7), dict(out=C + 2),
                dict(out=A, out_kind=F16), dict(out=A, ld_out=9)):
        assert call(m(**bad)) == EINVAL, bad
        assert b"hgnn_orthogonalize" in lib.hgnn_last_error()
    for bad in (dict(steps=-1), dict(steps=65), dict(coef=None), dict(coef=(NAN, 0, 0)), dict(coef=(1, INF, 0)), dict(coef=(8.5, 0, 0)), dict(coef=(0, 65, 0)), dict(coef=(0, 0, 65)), dict(coef=(1, 130, -200)),
                dict(steps=2, coef=(4.0, 0, 0, 4.0, 0, 0)), dict(scales=(NAN,)), dict(scales=(INF,)), dict(ws=None), dict(bytes=need - 1), dict(ws=E + 8), dict(count=-1)):
        assert call(m(), **bad) == EINVAL, bad
    assert call(m(), m()) == EINVAL and b"same output" in lib.hgnn_last_error()
    assert call(m(rows=65537)) == EUNSUP and call(m(cols=65537, ld=65537)) == EUNSUP
    assert call() == 0 and call(m(rows=0, grad=None)) == 0 and lib.hgnn_orthogonalize(0, None, 0, None, None, None, 0, None) == 0
    assert lib.hgnn_orthogonalize(1, None, 0, None, None, E, need, None) == EINVAL
    assert lib.hgnn_orthogonalize_workspace(1, (_GradStruct * 1)(m(rows=65537))) == 0 and lib.hgnn_orthogonalize_workspace(0, None) == 0


def test_binding_refuses(hgnn):
    """Tensors that are not on the GPU, by every wrapper; the structures are the header's."""
    import torch
    h = torch.zeros(8, 8).half()
    for call in (lambda: hgnn.hgnn_residual_norm(h, h, h, None), lambda: hgnn.hgnn_residual_norm_grad(h, h, h, None, h, h, None), lambda: hgnn.hgnn_gated(h, h, h, h),
                 lambda: hgnn.hgnn_gated_grad(h, h, h, h, h, h, h, None), lambda: hgnn.hgnn_orthogonalize([h], None, [(1.5, -0.5, 0.0)], None)):
        with pytest.raises(TypeError):
            call()
    assert ctypes.sizeof(hgnn.binding._BlockStruct) == 80 and ctypes.sizeof(hgnn.binding._BlockGradStruct) == 88
