"""The slopes of the gated projection's activations, each relative to itself, against 64 bits on the host.

One input carries the argument, G = X[i, 0], a second the other side, U = 2^10, both exact, and dX[i, 0] = dG = dY U act'(G), where dY is the power of two that brings
it near 1.  Tolerance relative to dG, u = 2^-24: an exponent's argument of size z is off by three roundings of it (a product of a square, or of a rounded constant) and
so is the exponential by 3 z u, z = |G| or G^2 / 2; its own rounding, those of the sums and reciprocals and of the products behind are 32 u; where a slope is a
difference (1 + G (1 - p), Phi + G phi away from their zeros) its terms are at most 4 times its size.  In all 4 (32 + 6 z) u, and 2^-11 for dG in fp16, which dX only
repeats."""
import numpy as np
import pytest
import torch

from parity import down

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SILU, GELU, SIGMOID, RELU = range(4)


def slope(x, act):
    from scipy.special import expit, ndtr
    if act == GELU:
        return ndtr(x) + x * np.exp(-x * x / 2) / np.sqrt(2 * np.pi)
    p, q = expit(x), expit(-x)
    return p * q if act == SIGMOID else p * (1 + x * q)


# arguments away from the zeros of a slope, as far out as 2^25 dY can bring it near 1
RANGES = {SIGMOID: [(-24, 24)], SILU: [(-24, -3), (-0.5, 24)], GELU: [(-5, -2), (-0.25, 24)]}


@pytest.mark.parametrize("act", [SIGMOID, SILU, GELU])
@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("n", [16, 300, 2500])
def test_slopes(hgnn, dev, act, trans, n):
    print("slopes", act, trans, n, flush=True)
    K, F = 16, 8
    parts = RANGES[act]
    g = np.concatenate([np.linspace(a, b, n // len(parts)) for a, b in parts]).astype(np.float16)
    n = len(g)
    G = g.astype(np.float64)
    s = slope(G, act)
    d = np.exp2(np.clip(np.round(-np.log2(np.abs(s))) - 10, -14, 15))
    X, dY = np.zeros((n, K), np.float16), np.zeros((n, F), np.float16)
    X[:, 0], X[:, 1], dY[:, 0] = g, 1, d
    Wg, Wu = np.zeros((K, F), np.float16), np.zeros((K, F), np.float16)
    Wg[0, 0], Wu[1, 0] = 1, 2 ** 10
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
    w = lambda a: t(a.T if trans else a)  # noqa: E731
    dX = torch.full((n, K), 3, dtype=torch.float16, device=dev)
    ws = torch.empty(hgnn.hgnn_gated_grad_workspace(n, K, F), dtype=torch.uint8, device=dev)
    hgnn.hgnn_gated_grad(t(X), w(Wg), w(Wu), t(dY), dX, None, None, ws, act=act, trans_w=trans)
    want = d * 2.0 ** 10 * s
    assert (np.abs(want) >= 2.0 ** -10).all() and (np.abs(want) < 65504).all()
    z = G * G / 2 if act == GELU else np.abs(G)
    off = np.abs(down(dX)[:, 0].astype(np.float64) - want) / np.abs(want)
    room = 2.0 ** -11 + 4 * (32 + 6 * z) * U
    bad = ~(off <= room)
    assert not bad.any(), (int(bad.sum()), G[bad][:4], off[bad][:4], room[bad][:4], off.max())
