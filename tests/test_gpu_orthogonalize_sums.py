"""Long sums of narrow matrices: what their low parts add is not lost beside the high parts' sum.

One row of 4096 elements 32 + t at the scale of the products, t near 2^-13, and a last one that makes the norm 64, so that A is 1: with x <- A x the result is the row
over its norm.  The high parts' sums are whole numbers and exact, and the low parts of 32 steps add 0.12 twice: in ONE sum that is cut to 24 bits (as the matrix
cores cut) beside partial sums of up to 2^21, whose last bit is worth 1/8, most of it is lost, some 4e-6 of A (cut_sums below); summed apart it is not.

Tolerance, relative, in units of 2^-24: the row over its norm in fp32 1 (its last element 4 more, two parts of 11 bits each), A 3 for the last element's product and
the additions of the two halves and of high and low, 2 + 2 for A and b A as two parts, the last product 2, the store 1: 20 at most."""
import numpy as np
import pytest
import torch

from parity import down

U = 2.0 ** -24
T = 0.12 / 1024  # a low part
N = 4096


def row():
    g = np.full(N, 1 + T / 32, np.float32)
    g[-1] = np.sqrt(N - (g[:-1].astype(np.float64) ** 2).sum())
    return g


def parts(x):
    hi = x.astype(np.float16)
    return hi.astype(np.float64), (x - hi.astype(np.float32)).astype(np.float16).astype(np.float64)


def cut(v):
    """to 24 bits, towards zero"""
    m, e = np.frexp(v)
    return np.ldexp(np.trunc(m * 2.0 ** 24), int(e) - 24)


def cut_sums(x):
    """The square's sum in one cut sum for each half of the 32-step blocks, the way that loses the low parts."""
    hi, lo = (p.reshape(-1, 32) for p in parts(x))
    total = 0.0
    for team in range(2):
        acc = 0.0
        for h, s in zip(hi[team::2], lo[team::2]):
            for v in ((h * s).sum(), (h * s).sum(), (h * h).sum()):
                acc = cut(acc + v)
        total += acc
    return total


def test_one_cut_sum_would_show():
    g = row()
    x = (g.astype(np.float64) / np.linalg.norm(g.astype(np.float64)) * 2048).astype(np.float32)
    assert (parts(x)[0][:-1] == 32).all() and abs(np.linalg.norm(x.astype(np.float64)) / 2048 - 1) < U
    assert 1 - cut_sums(x) / 2048 ** 2 > 3 * 20 * U


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, N), (N, 1)])
def test_low_parts_count(hgnn, dev, shape):
    g = row()
    t = torch.from_numpy(g.reshape(shape)).to(dev)
    out = torch.full_like(t, 3)
    ws = torch.empty(hgnn.hgnn_orthogonalize_workspace([t]), dtype=torch.uint8, device=dev)
    hgnn.hgnn_orthogonalize([t], [out], [(0.0, 1.0, 0.0)], ws)
    want = g.astype(np.float64) / np.linalg.norm(g.astype(np.float64))
    off = np.abs(down(out).reshape(-1).astype(np.float64) / want - 1)
    assert off.max() <= 20 * U, off.max() / U
