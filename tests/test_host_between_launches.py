"""What the calls between two aggregations, and between the clipped gradient and the weight, launch and refuse, on the host: libhgnn.so on a runtime that executes
nothing and writes launches down (fake_hip.cpp)."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

from test_host_memory import A, LIB, Host, fake, i64, vp  # noqa: F401

F16, F32 = 0, 1
f32, size_t = ctypes.c_float, ctypes.c_size_t


class Grad(ctypes.Structure):
    _fields_ = [("grad", vp), ("out", vp), ("rows", i64), ("cols", i64), ("ld", i64), ("ld_out", i64), ("type", ctypes.c_int), ("out_type", ctypes.c_int)]


def launches(h, call):
    h.fake.fake_reset(h.path)
    st = call()
    return st, [re.match(r"_ZN4hgnn(\d+)(.*)", n) for n in h.fake.fake_launched().decode().split()]


def names_of(found):
    return [m.group(2)[:int(m.group(1))] for m in found]


def orthogonalize(h, sides, steps, in_place):
    mats = (Grad * len(sides))()
    for i, (r, c) in enumerate(sides):
        at = h.data + (i + 1) * (1 << 21)
        mats[i] = Grad(at, None if in_place else at + (1 << 20), r, c, c, c, F32, F32)
    h.lib.hgnn_orthogonalize_workspace.restype = size_t
    need = h.lib.hgnn_orthogonalize_workspace(len(sides), mats)
    coef = (f32 * max(1, 3 * steps))(*([1.5, -0.5, 0.0] * steps))
    st, found = launches(h, lambda: h.lib.hgnn_orthogonalize(len(sides), mats, steps, coef, None, vp(h.data), size_t(need), vp(A)))
    assert st == 0
    return names_of(found)


def norms_before_results(h):
    """No launch reads all of a gradient and writes the result, which in place is that gradient: without steps the norms are a launch of their own."""
    for in_place in (True, False):
        assert orthogonalize(h, [(64, 608)], 0, in_place) == ["narrow_norms_kernel", "narrow_scale_kernel"]
        assert orthogonalize(h, [(64, 4096)] * 30, 0, in_place) == ["narrow_norms_kernel", "narrow_scale_kernel"] * 2
        assert orthogonalize(h, [(65, 100)], 0, in_place) == ["orth_squares_kernel", "orth_begin_kernel"]
        assert orthogonalize(h, [(64, 608), (64, 64)], 2, in_place) == ["narrow_begin_kernel"] + ["narrow_step_kernel"] * 2


def sizes(h):
    """The queries, with 64-bit results."""
    for f in (h.lib.hgnn_gated_workspace, h.lib.hgnn_gated_grad_workspace, h.lib.hgnn_residual_norm_grad_workspace):
        f.restype = size_t
    return (lambda n, K, F: h.lib.hgnn_gated_workspace(i64(n), K, F), lambda n, K, F: h.lib.hgnn_gated_grad_workspace(i64(n), K, F),
            lambda n, F: h.lib.hgnn_residual_norm_grad_workspace(i64(n), F))


NUMBERS = sorted({*range(1, 2400, 7), *(64 * k + d for k in range(1, 40) for d in (-1, 0, 1)), *(1 << k for k in range(8, 21)), 3000, 4099, 70001, 99991, 233000})


def workspaces_for_fewer_rows(h):
    """What holds a call of n rows holds any of fewer: a program keeps one workspace for batches of all sizes."""
    gated, grad, norm = sizes(h)
    x = vp(h.data)
    for F in (8, 100, 333, 512, 513, 1024, 2048, 4096, 8192):
        need = [norm(n, F) for n in NUMBERS]
        assert need == sorted(need) and need[0] > 0, F
    for K, F in ((16, 8), (100, 200), (128, 256), (1024, 4096), (2048, 2048), (2048, 8192), (4096, 64), (4096, 20), (20, 4096), (8192, 333), (65536, 65536)):
        for f in (gated, grad):
            need = [f(n, K, F) for n in NUMBERS]
            assert need == sorted(need), (K, F, f is grad)
        up = lambda n: (n + 7) // 8 * 8  # noqa: E731
        most = NUMBERS[-1]
        for n in NUMBERS[::9]:
            st, _ = launches(h, lambda: h.lib.hgnn_gated(i64(n), K, F, 0, x, i64(up(K)), x, x, i64(up(F)), 0, x, i64(up(F)), x, size_t(gated(most, K, F)), vp(A)))
            assert st == 0, (n, K, F)
            st, _ = launches(h, lambda: h.lib.hgnn_gated_grad(i64(n), K, F, 0, x, i64(up(K)), x, x, i64(up(F)), 0, x, i64(up(F)), x, i64(up(K)), x, vp(h.data + 64), i64(up(F)), x,
                                                              size_t(grad(most, K, F)), vp(A)))
            assert st == 0, (n, K, F)
    # and the queries do not ask for much more than a call needs: sums of at most 256 tiles of 128 x 128, twice for pairs, and for the gradients D
    for K, F in ((2048, 2048), (4096, 64), (1024, 4096), (65536, 65536)):
        for n in (1, 100, 1000, 10000):
            tiles = 256 * 2 * 2 * 128 * 128 * 4
            assert gated(n, K, F) <= tiles and grad(n, K, F) <= tiles + n * 2 * (F + 31) * 2 + 256, (n, K, F)


def more_tiles_than_a_grid(h):
    """A result of more tiles than a grid has room for takes several launches; the grid's lanes fit 32 bits in each."""
    x, far = vp(h.data), vp(h.data + 64)
    room = size_t(1 << 50)
    for n, K, F, most in ((500000000, 300, 8, 1), (600000000, 300, 8, 2), (1100000, 300, 65536, 2), (1000000, 300, 65536, 1), (2000000000, 300, 32, 4)):
        st, found = launches(h, lambda: h.lib.hgnn_gated(i64(n), K, F, 0, x, i64(304), x, x, i64(65536), 0, x, i64(65536), None, size_t(0), vp(A)))
        names = names_of(found)
        assert st == 0 and len(names) == most and set(names) == {"product_kernel"}, (n, K, F, st, names)
        assert 0 < h.fake.fake_last_grid() * h.fake.fake_last_block() < 1 << 32
    for n, K, F, most in ((500000000, 8, 8, 1), (600000000, 8, 8, 2), (1100000000, 64, 16, 3)):
        st, found = launches(h, lambda: h.lib.hgnn_gated_grad(i64(n), K, F, 0, x, i64(64), x, x, i64(64), 0, x, i64(64), x, i64(64), None, None, i64(0), far, room, vp(A)))
        names = names_of(found)
        assert st == 0 and names == ["gated_rows_kernel"] + ["product_kernel"] * most, (n, K, F, st, names)


SCENARIOS = [norms_before_results, workspaces_for_fewer_rows, more_tiles_than_a_grid]


@pytest.mark.parametrize("name", [s.__name__ for s in SCENARIOS])
def test_launches(hgnn, fake, name):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, LIB, name], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    host = Host(sys.argv[1], sys.argv[2])
    {s.__name__: s for s in SCENARIOS}[sys.argv[3]](host)
    print("ok")
