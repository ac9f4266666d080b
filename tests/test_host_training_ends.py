"""Refusals of the calls at the two ends of a training step and of its guard, on the host: every call here returns before anything is launched."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib(hgnn):
    return hgnn.load()


A, B, C, D = 0x10000, 0x20000, 0x30000, 0x40000  # stand for device addresses
F16, F32 = 0, 1


def test_lookup_refuses(lib, hgnn):
    EINVAL, EUNSUP = hgnn.HGNN_EINVAL, hgnn.HGNN_EUNSUPPORTED

    def call(n=4, F=8, ids=A, V=5, kind=F16, table=B, ldt=8, out=C, ldo=8):
        return lib.hgnn_embedding(n, F, ids, V, kind, table, ldt, 1.0, out, ldo, None)
    for bad in (dict(n=-1), dict(F=0), dict(V=-1), dict(kind=2), dict(kind=-1), dict(ldt=7), dict(ldo=7), dict(ids=None), dict(table=None), dict(out=None),
                dict(ids=A + 2), dict(table=B + 1), dict(kind=F32, table=B + 2), dict(out=C + 1)):
        assert call(**bad) == EINVAL, bad
        assert b"hgnn_embedding" in lib.hgnn_last_error()
    assert call(F=65537, ldt=70000, ldo=70000) == EUNSUP
    for many in (dict(n=(1 << 40) + 1), dict(n=1 << 38), dict(n=1 << 62)):
        assert call(**many) == EUNSUP, many
    assert call(n=0, ids=None, table=None, out=None) == 0  # nothing to do


def test_table_gradient_refuses(lib, hgnn):
    EINVAL, EUNSUP = hgnn.HGNN_EINVAL, hgnn.HGNN_EUNSUPPORTED
    need = hgnn.hgnn_embedding_grad_workspace(100, 8, 5)
    assert need > 0

    def call(n=100, F=8, ids=A, V=5, dY=B, ldy=8, add=0, kind=F32, dT=C, ldt=8, ws=D, bytes=need):
        return lib.hgnn_embedding_grad(n, F, ids, V, dY, ldy, 1.0, add, kind, dT, ldt, ws, bytes, None)
    for bad in (dict(n=-1), dict(n=1 << 31), dict(F=0), dict(V=-1), dict(kind=2), dict(ldy=7), dict(ldt=7), dict(ids=None), dict(dY=None), dict(dT=None),
                dict(ws=None), dict(bytes=need - 1), dict(ws=D + 8), dict(ids=A + 1), dict(dY=B + 1), dict(dT=C + 2)):
        assert call(**bad) == EINVAL, bad
        assert b"hgnn_embedding_grad" in lib.hgnn_last_error()
    assert call(F=65537, ldy=70000, ldt=70000, bytes=1 << 40) == EUNSUP
    assert call(n=0, add=1, ids=None, dY=None, ws=None, bytes=0) == 0 and call(V=0) == 0  # nothing to do
    # the workspace: enough for the words of both sides of a sort, nothing for nothing
    assert hgnn.hgnn_embedding_grad_workspace(0, 8, 5) == 0 and hgnn.hgnn_embedding_grad_workspace(1 << 31, 8, 5) == 0
    assert hgnn.hgnn_embedding_grad_workspace(10 ** 6, 128, 10) >= 16 * 10 ** 6


def test_logprob_refuses(lib, hgnn):
    EINVAL, EUNSUP = hgnn.HGNN_EINVAL, hgnn.HGNN_EUNSUPPORTED
    need = hgnn.hgnn_logprob_workspace(2, 100000, 4)

    def call(n=2, c=100000, kind=F16, x=A, ld=100000, y=B, lp=C, st=C, en=C, k=4, tv=C, tc=C, ws=D, bytes=need):
        return lib.hgnn_logprob(n, c, kind, x, ld, y, lp, st, en, k, tv, tc, ws, bytes, None)
    cases = [dict(n=-1), dict(c=0), dict(kind=7), dict(ld=99999), dict(k=-1), dict(c=3, k=4), dict(x=None), dict(tv=None), dict(tc=None), dict(y=None), dict(lp=None),
             dict(x=A + 1), dict(kind=F32, x=A + 2), dict(y=B + 2), dict(lp=C + 1), dict(st=C + 2), dict(en=C + 3), dict(tv=C + 1), dict(tc=C + 2)]
    if need:
        cases += [dict(ws=None), dict(bytes=need - 1), dict(ws=D + 2)]
    for bad in cases:
        assert call(**bad) == EINVAL, bad
        assert b"hgnn_logprob" in lib.hgnn_last_error()
    assert call(k=33) == EUNSUP and call(c=(1 << 30) + 1, ld=1 << 31) == EUNSUP
    assert call(n=0, x=None, tv=None, tc=None) == 0
    for many in (dict(n=(1 << 40) + 1), dict(n=1 << 33, c=500, ld=500), dict(n=1 << 28, c=4000, ld=4000), dict(n=1 << 62)):
        assert call(**many) == EUNSUP, many
    assert hgnn.hgnn_logprob_workspace(0, 100, 0) == 0 and hgnn.hgnn_logprob_workspace(1000, 41, 5) == 0


def test_logprob_gradient_refuses(lib, hgnn):
    EINVAL = hgnn.HGNN_EINVAL

    def call(n=2, c=10, kind=F16, x=A, ld=10, y=B, st=C, g=C, en=None, h=None, dx=D, ldd=10):
        return lib.hgnn_logprob_grad(n, c, kind, x, ld, y, st, g, en, h, dx, ldd, None)
    for bad in (dict(n=-1), dict(c=0), dict(kind=2), dict(ld=9), dict(ldd=9), dict(y=None), dict(g=None), dict(h=C), dict(x=None), dict(st=None), dict(dx=None),
                dict(dx=A, ldd=16), dict(x=A + 1), dict(dx=D + 1), dict(st=C + 1), dict(g=C + 2), dict(en=C + 1, h=C), dict(en=C, h=C + 1), dict(y=B + 1)):
        assert call(**bad) == EINVAL, bad
        assert b"hgnn_logprob_grad" in lib.hgnn_last_error()
    assert call(n=0, x=None, st=None, dx=None) == 0
    for many in (dict(n=(1 << 40) + 1), dict(n=1 << 40, c=1 << 30, ld=1 << 30, ldd=1 << 30), dict(n=1 << 33, c=500, ld=500, ldd=500), dict(n=1 << 62)):
        assert call(**many) == hgnn.HGNN_EUNSUPPORTED, many


def test_clip_refuses(lib, hgnn):
    from paper_2411_01109_amd.binding import _GradStruct
    EINVAL, EUNSUP = hgnn.HGNN_EINVAL, hgnn.HGNN_EUNSUPPORTED
    need = hgnn.hgnn_grad_norm_workspace()

    def tensor(grad=A, out=None, rows=1, cols=8, ld=8, ld_out=8, kind=F32, out_kind=F32):
        return _GradStruct(grad, out, rows, cols, ld, ld_out, kind, out_kind)

    def clip(*tensors, inv=1.0, most=1.0, norm=C, ws=D, bytes=need, count=None):
        a = (_GradStruct * max(len(tensors), 1))(*tensors)
        return lib.hgnn_grad_clip(len(tensors) if count is None else count, a, inv, most, norm, ws, bytes, None)

    def norm_of(*tensors, inv=1.0, norm=C, ws=D, bytes=need):
        a = (_GradStruct * max(len(tensors), 1))(*tensors)
        return lib.hgnn_grad_norm(len(tensors), a, inv, norm, ws, bytes, None)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(kind=3), dict(ld=7), dict(grad=None), dict(grad=A + 2), dict(kind=F16, grad=A + 1)):
        assert clip(tensor(), tensor(**{**dict(grad=B), **bad})) == EINVAL, bad
        assert norm_of(tensor(), tensor(**{**dict(grad=B), **bad})) == EINVAL, bad
    for bad in (dict(out=C, out_kind=2), dict(out=C, ld_out=7), dict(out=C + 2), dict(out=A, out_kind=F16), dict(out=A, rows=2, ld_out=9)):
        assert clip(tensor(**bad)) == EINVAL, bad
    for bad in (dict(inv=0.0), dict(inv=-1.0), dict(inv=nan), dict(inv=inf), dict(norm=None), dict(norm=C + 2), dict(ws=None), dict(ws=D + 4), dict(bytes=need - 1)):
        assert clip(tensor(), **bad) == EINVAL and norm_of(tensor(), **bad) == EINVAL, bad
    assert clip(tensor(), most=-1.0) == EINVAL and clip(tensor(), most=nan) == EINVAL and clip(count=-1) == EINVAL
    assert clip(tensor(), tensor()) == EINVAL and b"same output" in lib.hgnn_last_error()
    assert clip(tensor(out=B), tensor(grad=B)) == EINVAL  # another's place is written
    assert clip(tensor(rows=2, cols=1 << 31, ld=1 << 31)) == EUNSUP
    assert lib.hgnn_grad_clip(1, None, 1.0, 1.0, C, D, need, None) == EINVAL and lib.hgnn_grad_norm(1, None, 1.0, C, D, need, None) == EINVAL


def test_binding_refuses(hgnn):
    """Tensors that are not on the GPU, by every wrapper."""
    import torch
    h, i, f = torch.zeros(4, 8).half(), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    calls = [lambda: hgnn.hgnn_embedding(i, h, h), lambda: hgnn.hgnn_embedding_grad(i, h, h, None), lambda: hgnn.hgnn_logprob(h, i, f),
             lambda: hgnn.hgnn_logprob_grad(h, i, torch.zeros(4, 2), f, h), lambda: hgnn.hgnn_grad_norm([h], torch.zeros(1), f),
             lambda: hgnn.hgnn_grad_clip([h], 1.0, torch.zeros(1), f)]
    for call in calls:
        with pytest.raises(TypeError):
            call()
    assert ctypes.sizeof(hgnn.binding._GradStruct) == 56
