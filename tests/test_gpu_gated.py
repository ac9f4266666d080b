"""The gated projection and its gradients against 64 bits on the host.

Tolerances, u = 2^-24.  A sum of K products of fp16 numbers, which are exact in fp32, is off by at most 2 K u of the sum of their absolute values (an addition and
whatever the matrix cores round inside a step), so G by eG = 2 K u |X||Wg| and U by eU likewise.  act has a slope of at most 1.13 and its own rounding 16 u (1 + |G|)
(the exponent's argument), so act(G) U is off by 1.13 eG |U| + |act| eU + 16 u (1 + |G|) |act U|, and the store adds 2^-11 or 2^-25.  act' has a slope of at most 0.8
(but for a kink, where relu's G is near 0: those places are held to nothing less than the whole step).  dG and dU pass through fp16: 2^-11 of them or 2^-25 more.  dX
and the weights' gradients sum such values: the sums of what their terms are off by, times the other factor, and 2 (terms) u of the sum of the absolute values."""
import numpy as np
import pytest
import torch

from parity import down

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
FILL = 7.0
F16 = np.float16
SILU, GELU, SIGMOID, RELU = range(4)
NAN = float("nan")


def act_of(x, act):
    """-> (act, its derivative)"""
    from scipy.special import ndtr, expit
    if act == RELU:
        return np.maximum(x, 0), (x > 0) * 1.0
    if act == GELU:
        return x * ndtr(x), ndtr(x) + x * np.exp(-x * x / 2) / np.sqrt(2 * np.pi)
    p = expit(x)
    return (p, p * (1 - p)) if act == SIGMOID else (x * p, p * (1 + x * (1 - p)))


def up8(n):
    return (n + 7) // 8 * 8


def place(a, dev, pitch=None, offset=0, fill=NAN):
    """A device copy in rows of a pitch, `offset` elements in; everything else in the buffer is `fill` -> (view, buffer)"""
    t = torch.from_numpy(np.ascontiguousarray(a))
    n, F = t.shape
    pitch = up8(F) if pitch is None else pitch
    buf = torch.full((n * pitch + offset + 8,), fill, dtype=t.dtype, device=dev)
    v = torch.as_strided(buf, (n, F), (pitch, 1), offset)
    v.copy_(t)
    return v, buf


def untouched(view, buf):
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, view.shape, view.stride(), view.storage_offset()).fill_(False)
    assert bool((buf[mask] == FILL).all()), "something beside the tensor was written"


def near(name, got, ref, tol):
    got = got.astype(np.float64)
    bad = ~(np.abs(got - ref) <= tol + np.abs(ref) * 2.0 ** -11 + 2.0 ** -25)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], ref[bad][:3], tol[bad][:3])


class Case:
    def __init__(self, n, K, F, act=SILU, trans=False, sd=1.0, seed=0):
        print(f"gated n={n} K={K} F={F} act={act} trans={trans}", flush=True)
        rng = np.random.default_rng(seed + n * 7 + K * 3 + F)
        self.n, self.K, self.F, self.act, self.trans = n, K, F, act, trans
        self.X = (rng.standard_normal((n, K)) * sd).astype(F16)
        self.Wg, self.Wu = ((rng.standard_normal((K, F)) / np.sqrt(K)).astype(F16) for _ in range(2))
        self.dY = (rng.standard_normal((n, F)) / np.sqrt(F)).astype(F16)

    def tensors(self, dev, extra=0, offset=0):
        w = lambda a: place(a.T if self.trans else a, dev, up8(self.K if self.trans else self.F) + extra, offset)[0]  # noqa: E731
        return place(self.X, dev, up8(self.K) + extra, offset)[0], w(self.Wg), w(self.Wu)

    def sums(self):
        X, Wg, Wu = (a.astype(np.float64) for a in (self.X, self.Wg, self.Wu))
        e = 2 * self.K * U
        return X, Wg, Wu, X @ Wg, X @ Wu, e * (np.abs(X) @ np.abs(Wg)), e * (np.abs(X) @ np.abs(Wu))


def forward(hgnn, dev, c, extra=0, offset=0):
    X, Wg, Wu = c.tensors(dev, extra, offset)
    Y, Yb = place(np.full((c.n, c.F), 3, F16), dev, up8(c.F) + extra, offset, FILL)
    ws = torch.full((max(hgnn.hgnn_gated_workspace(c.n, c.K, c.F), 16),), 255, dtype=torch.uint8, device=dev)
    hgnn.hgnn_gated(X, Wg, Wu, Y, act=c.act, trans_w=c.trans, workspace=ws)
    _, _, _, G, V, eG, eU = c.sums()
    a, _ = act_of(G, c.act)
    near("Y", down(Y), a * V, 1.13 * eG * np.abs(V) + np.abs(a) * eU + 16 * U * (1 + np.abs(G)) * np.abs(a * V))
    untouched(Y, Yb)
    return Y


def backward(hgnn, dev, c, extra=0, offset=0, dx=True, dw=True):
    X, Wg, Wu = c.tensors(dev, extra, offset)
    dY = place(c.dY, dev, up8(c.F) + extra, offset)[0]
    out = lambda shape, there: place(np.full(shape, 3, F16), dev, up8(shape[1]) + extra, offset, FILL) if there else (None, None)  # noqa: E731
    shape = (c.F, c.K) if c.trans else (c.K, c.F)
    (dX, dXb), (dWg, dWgb), (dWu, dWub) = out((c.n, c.K), dx), out(shape, dw), out(shape, dw)
    ws = torch.full((max(hgnn.hgnn_gated_grad_workspace(c.n, c.K, c.F), 16),), 255, dtype=torch.uint8, device=dev)
    hgnn.hgnn_gated_grad(X, Wg, Wu, dY, dX, dWg, dWu, ws, act=c.act, trans_w=c.trans)
    X, Wg, Wu, G, V, eG, eU = c.sums()
    a, s = act_of(G, c.act)
    d = c.dY.astype(np.float64)
    dG, dU = d * V * s, d * a
    es = np.where(np.abs(G) <= eG, 1.0, 0.0) if c.act == RELU else 0.8 * eG
    tG = np.abs(d) * (np.abs(s) * eU + np.abs(V) * (es + 16 * U * (1 + np.abs(G)) ** 2)) + 2.0 ** -25
    tU = np.abs(d) * (1.13 * eG + 16 * U * (1 + np.abs(G)) * np.abs(a)) + 2.0 ** -25
    tG, tU = tG + 2.0 ** -11 * (np.abs(dG) + tG), tU + 2.0 ** -11 * (np.abs(dU) + tU)
    if dx:
        tol = tG @ np.abs(Wg).T + tU @ np.abs(Wu).T + 4 * c.F * U * (np.abs(dG) @ np.abs(Wg).T + np.abs(dU) @ np.abs(Wu).T)
        near("dX", down(dX), dG @ Wg.T + dU @ Wu.T, tol)
        untouched(dX, dXb)
    if dw:
        for name, t, buf, v, e in (("dWg", dWg, dWgb, dG, tG), ("dWu", dWu, dWub, dU, tU)):
            ref, tol = X.T @ v, np.abs(X).T @ e + 2 * c.n * U * (np.abs(X).T @ np.abs(v))
            near(name, down(t), ref.T if c.trans else ref, tol.T if c.trans else tol)
            untouched(t, buf)
    return dX, dWg, dWu


SHAPES = [(1, 1, 1), (1, 8, 8), (3, 32, 16), (2, 33, 31), (16, 64, 64), (17, 40, 72), (1, 200, 300), (5, 7, 500), (64, 128, 64), (65, 31, 65), (63, 257, 129), (128, 128, 128), (129, 100, 200), (300, 41, 9),
          (255, 96, 33), (1000, 64, 32), (513, 8, 130), (13, 1000, 77), (70, 515, 20), (4000, 16, 24), (1, 1024, 640), (16, 2050, 33), (32, 700, 100), (33, 90, 47), (49, 1500, 64), (64, 33, 300)]


@pytest.mark.parametrize("n,K,F", SHAPES)
@pytest.mark.parametrize("trans", [False, True])
def test_shapes(hgnn, dev, n, K, F, trans):
    c = Case(n, K, F, (n + K) % 4, trans)
    forward(hgnn, dev, c)
    backward(hgnn, dev, c)


@pytest.mark.parametrize("act", [SILU, GELU, SIGMOID, RELU])
@pytest.mark.parametrize("trans", [False, True])
def test_activations(hgnn, dev, act, trans):
    """Large and small arguments, wide pitches, an offset of a piece; what stands beside the rows is NaN."""
    for sd in (0.01, 1.0, 12.0):
        c = Case(90, 50, 70, act, trans, sd)
        forward(hgnn, dev, c, extra=16, offset=8)
        backward(hgnn, dev, c, extra=16, offset=8)


# (n, K, F) of each size of tile, with and without parts: few rows, a narrow side, tiles that fill the chip, and sizes around them
@pytest.mark.parametrize("n,K,F", [(1, 1024, 4096), (16, 1024, 4096), (16, 1017, 4095), (17, 1024, 4096), (1, 1025, 100), (2, 1032, 64), (5, 1024, 4097), (13, 2048, 5461), (1, 4000, 40),
                                   (64, 2000, 33), (30, 65000, 24), (16, 65, 4090), (9, 992, 1), (11, 961, 66)])
@pytest.mark.parametrize("trans", [False, True])
def test_few_rows(hgnn, dev, n, K, F, trans):
    """Up to 16 rows by up to 1024 inputs and 4096 features in one launch, and what is just beyond."""
    c = Case(n, K, F, GELU, trans)
    forward(hgnn, dev, c)
    backward(hgnn, dev, c)


@pytest.mark.parametrize("n,K,F", [(40, 700, 90), (700, 600, 500), (2100, 300, 700), (20000, 70, 20), (4099, 72, 2049), (8200, 40, 1100), (66000, 24, 40), (17000, 128, 256), (16400, 256, 130), (16500, 99, 300), (8192, 520, 4100), (16400, 30, 60), (16401, 60, 100),
                                   (16400, 200, 50), (17000, 150, 70), (16384, 256, 64), (16999, 100, 128), (16390, 190, 260), (2048, 100, 4096), (2047, 100, 4100), (2050, 250, 40), (3001, 33, 64)])
@pytest.mark.parametrize("trans", [False, True])
def test_tiles(hgnn, dev, n, K, F, trans):
    c = Case(n, K, F, SILU, trans)
    forward(hgnn, dev, c)
    backward(hgnn, dev, c)


def test_one_gradient_alone(hgnn, dev):
    c = Case(150, 60, 80)
    both = backward(hgnn, dev, c)
    assert torch.equal(backward(hgnn, dev, c, dw=False)[0], both[0])
    _, g, u = backward(hgnn, dev, c, dx=False)
    assert torch.equal(g, both[1]) and torch.equal(u, both[2])


def test_no_rows(hgnn, dev):
    x, w, y = torch.empty(0, 24, dtype=torch.float16, device=dev), torch.zeros(24, 16, dtype=torch.float16, device=dev), torch.empty(0, 16, dtype=torch.float16, device=dev)
    hgnn.hgnn_gated(x, w, w, y)
    g, u = torch.full_like(w, FILL), torch.full_like(w, FILL)
    hgnn.hgnn_gated_grad(x, w, w, y, x, g, u, torch.empty(16, dtype=torch.uint8, device=dev))
    assert bool((g == 0).all()) and bool((u == 0).all())


def test_halves_of_one_weight(hgnn, dev):
    """Wg and Wu side by side in one matrix, as programs keep them; and their gradients."""
    c = Case(100, 48, 64)
    W = torch.from_numpy(np.concatenate([c.Wg, c.Wu], 1)).to(dev)
    X, dY = torch.from_numpy(c.X).to(dev), torch.from_numpy(c.dY).to(dev)
    Y = torch.empty(100, 64, dtype=torch.float16, device=dev)
    hgnn.hgnn_gated(X, W[:, :64], W[:, 64:], Y, workspace=torch.empty(max(16, hgnn.hgnn_gated_workspace(100, 48, 64)), dtype=torch.uint8, device=dev))
    assert torch.equal(Y, forward(hgnn, dev, c))
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    ws = torch.empty(hgnn.hgnn_gated_grad_workspace(100, 48, 64), dtype=torch.uint8, device=dev)
    hgnn.hgnn_gated_grad(X, W[:, :64], W[:, 64:], dY, dX, dW[:, :64], dW[:, 64:], ws)
    x, g, u = backward(hgnn, dev, c)
    assert torch.equal(dX, x) and torch.equal(dW[:, :64], g) and torch.equal(dW[:, 64:], u)


def test_rows_that_are_not_finite(hgnn, dev):
    """A row with NaN spoils itself alone."""
    c = Case(300, 40, 56)
    want = forward(hgnn, dev, c)
    c.X[17, 3] = np.nan
    X, Wg, Wu = c.tensors(dev)
    Y = torch.empty(300, 56, dtype=torch.float16, device=dev)
    hgnn.hgnn_gated(X, Wg, Wu, Y, workspace=torch.empty(max(16, hgnn.hgnn_gated_workspace(300, 40, 56)), dtype=torch.uint8, device=dev))
    rest = torch.arange(300, device=dev) != 17
    assert bool(Y[17].isnan().all()) and torch.equal(Y[rest], want[rest])


def test_gradients_against_differences(hgnn, dev):
    """The loss sum(dY Y) of the formula in 64 bits on the host, by central differences, against the gradients of the call."""
    for act in (SILU, GELU, SIGMOID):
        c = Case(9, 20, 24, act)
        got = dict(zip(("X", "Wg", "Wu"), backward(hgnn, dev, c)))
        at = {k: getattr(c, k).astype(np.float64) for k in got}
        d = c.dY.astype(np.float64)
        loss = lambda X, Wg, Wu: (d * act_of(X @ Wg, act)[0] * (X @ Wu)).sum()  # noqa: E731
        rng = np.random.default_rng(act)
        for name, t in got.items():
            for _ in range(6):
                i = tuple(rng.integers(0, s) for s in at[name].shape)
                up, lo = dict(at), dict(at)
                up[name], lo[name] = at[name].copy(), at[name].copy()
                up[name][i] += 1e-4
                lo[name][i] -= 1e-4
                want = (loss(**up) - loss(**lo)) / 2e-4
                # roundings of at most 48 dG or dU (2^-11 of up to ~1) times factors of about 1, and the result's own
                assert abs(float(t[i]) - want) <= 48 * 2.0 ** -11 * 0.5 + 2.0 ** -11 * abs(want), (name, i)


def test_the_same_bits_again_on_a_stream_and_in_graphs(hgnn, dev):
    """Twice, by ctypes, on another stream, and captured in two graphs that share a workspace and are replayed in turn with other data."""
    for n, K, F in ((12, 300, 200), (5000, 64, 96)):
        c = Case(n, K, F)
        X, Wg, Wu = c.tensors(dev)
        dY = place(c.dY, dev)[0]
        out = [torch.zeros(n, up8(F), dtype=torch.float16, device=dev)[:, :F], torch.zeros(n, up8(K), dtype=torch.float16, device=dev)[:, :K], torch.zeros_like(Wg), torch.zeros_like(Wu)]
        ws = torch.empty(max(hgnn.hgnn_gated_grad_workspace(n, K, F), hgnn.hgnn_gated_workspace(n, K, F)), dtype=torch.uint8, device=dev)

        def first(stream=None):
            hgnn.hgnn_gated(X, Wg, Wu, out[0], workspace=ws, stream=stream)

        def second(stream=None):
            hgnn.hgnn_gated_grad(X, Wg, Wu, dY, *out[1:], ws, stream=stream)

        def taken():
            torch.cuda.synchronize()
            return [t.clone() for t in out]

        def same(a):
            return all(torch.equal(x, y) for x, y in zip(a, taken()))
        first(), second()
        want = taken()
        ws.fill_(255)
        first(), second()
        assert same(want)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        first(side), second(side)
        side.synchronize()
        assert same(want)
        native, hgnn.binding._calls = hgnn.binding._calls, None
        try:
            first(), second()
            assert native is not None and same(want)
        finally:
            hgnn.binding._calls = native
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        for g, call in zip(graphs, (first, second)):
            with torch.cuda.graph(g):
                call()
        for _ in range(3):
            X.mul_(0.75)
            for g in graphs:
                g.replay()
            replayed = taken()
            first(), second()
            assert same(replayed)


def test_refusals_of_the_binding(hgnn, dev):
    h = lambda *s: torch.zeros(*s, dtype=torch.float16, device=dev)  # noqa: E731
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
    x, w, y = h(100, 64), h(64, 32), h(100, 32)
    call = lambda x=x, g=w, u=w, y=y, ws=ws, **k: hgnn.hgnn_gated(x, g, u, y, workspace=ws, **k)  # noqa: E731
    call()
    bad = [lambda: call(x=x.float()), lambda: call(g=w.t()), lambda: call(g=h(64, 40)[:, :32]), lambda: call(y=h(99, 32)), lambda: call(act=4), lambda: call(act=-1), lambda: call(trans_w=True),
           lambda: call(x=h(100, 66)[:, :64]), lambda: call(x=h(100, 72)[:, 4:68]), lambda: call(ws=None, x=h(100, 4000), g=h(4000, 32), u=h(4000, 32), y=h(100, 32)),
           lambda: call(x=h(100, 63), g=h(63, 32), u=h(63, 32)),
           lambda: call(x=torch.as_strided(h(99 * 64 + 61), (100, 61), (64, 1)), g=h(61, 32), u=h(61, 32)),  # no room behind the last row
           lambda: hgnn.hgnn_gated_grad(x, w, w, y, h(100, 64), h(64, 32), None, ws), lambda: hgnn.hgnn_gated_grad(x, w, w, y, h(100, 64), h(64, 32), h(64, 32), None),
           lambda: hgnn.hgnn_gated_grad(x, w, w, y, h(100, 64), y[:64], y[:64], ws), lambda: hgnn.hgnn_gated_grad(x, w, w, y, h(100, 60), h(64, 32), h(64, 32), ws)]
    for b in bad:
        with pytest.raises((hgnn.HgnnError, TypeError, ValueError)):
            b()
