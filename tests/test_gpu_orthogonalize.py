"""Updates made orthogonal by Newton-Schulz products, against the definition in 64 bits on the host.

Tolerance.  What an error of a step becomes depends on the matrix (up to a^steps of it), so the measure is the same steps in fp32 on the host: a value that is two fp16
numbers has 22 bits in the place of 24, four times the rounding, and of a product the low parts' product is left out, as much again: the error (2-norm over
the result's) is at most 8 times that of fp32, or 8 roundings of 2^-22 where fp32 is exact by luck, and the output's rounding 2^-11 or 2^-24."""
import numpy as np
import pytest
import torch

from parity import down

pytestmark = pytest.mark.gpu
FILL = 7.0
F16, F32 = np.float16, np.float32
QUINTIC, CUBIC = (3.4445, -4.775, 2.0315), (1.5, -0.5, 0.0)


def steps_of(g, coef, dtype):
    x = g.astype(np.float64)
    flip = x.shape[0] > x.shape[1]
    x = x.T if flip else x
    norm = np.sqrt((x * x).sum())
    if not 0 < norm < np.inf:
        return np.zeros(g.shape)
    x = (x / norm).astype(dtype)
    for a, b, c in coef:
        a, b, c = (dtype(F32(v)) for v in (a, b, c))
        A = x @ x.T
        x = a * x + (b * A + c * (A @ A)) @ x
    return (x.T if flip else x).astype(np.float64)


def place(a, dev, pitch=None, offset=0):
    t = torch.from_numpy(np.ascontiguousarray(a))
    n, F = t.shape
    pitch = F if pitch is None else pitch
    buf = torch.full((max(n - 1, 0) * pitch + (F if n else 0) + offset + 1,), FILL, dtype=t.dtype, device=dev)
    v = torch.as_strided(buf, (n, F), (pitch, 1), offset)
    v.copy_(t)
    return v, buf


def matrix(rows, cols, dtype=F32, seed=0):
    rng = np.random.default_rng(seed + 100 * rows + cols)
    few = max(1, min(rows, cols) // 4)
    g = (rng.standard_normal((rows, few)) * np.linspace(1, 0.1, few)) @ rng.standard_normal((few, cols)) / np.sqrt(few) + 0.5 * rng.standard_normal((rows, cols))
    return g.astype(dtype)


def check(hgnn, dev, mats, coef, out_dtype=F32, scales=None, pitch=0, offset=0, in_place=False):
    print("orthogonalize", [m.shape for m in mats], len(coef), out_dtype.__name__, pitch, offset, flush=True)
    grads = [place(m, dev, m.shape[1] + pitch, offset) for m in mats]
    outs = grads if in_place else [place(np.full(m.shape, 3, out_dtype), dev, m.shape[1] + pitch, offset) for m in mats]
    ws = torch.full((max(hgnn.hgnn_orthogonalize_workspace([g[0] for g in grads]), 16),), 255, dtype=torch.uint8, device=dev)
    hgnn.hgnn_orthogonalize([g[0] for g in grads], None if in_place else [o[0] for o in outs], coef, ws, scales=scales)
    for i, m in enumerate(mats):
        scale = 1.0 if scales is None else scales[i]
        ref, single = steps_of(m, coef, np.float64), steps_of(m, coef, F32)
        got = down(outs[i][0])
        norm = np.linalg.norm(ref)
        assert np.isfinite(got).all()
        if got.dtype == F16:
            room = 2.0 ** -11 * abs(scale) * norm + 2.0 ** -25 * np.sqrt(m.size)
        else:
            room = 2.0 ** -24 * abs(scale) * norm
        off = np.linalg.norm(got.astype(np.float64) - scale * ref)
        assert off <= abs(scale) * (8 * np.linalg.norm(single - ref) + 8 * 2.0 ** -22 * norm) + room, (m.shape, off / max(norm, 1e-300), np.linalg.norm(single - ref) / max(norm, 1e-300))
        view, buf = outs[i]
        mask = torch.ones_like(buf, dtype=torch.bool)
        torch.as_strided(mask, view.shape, view.stride(), view.storage_offset()).fill_(False)
        assert bool((buf[mask] == FILL).all()), "something beside the matrix was written"
        if not in_place:
            assert np.array_equal(down(grads[i][0]), m)
    return [o[0] for o in outs]


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (8, 8), (31, 33), (32, 32), (64, 64), (65, 40), (42, 64), (64, 608), (608, 64), (100, 129), (128, 128), (130, 257), (300, 200), (256, 1000), (700, 90), (520, 519)]


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_shapes(hgnn, dev, rows, cols):
    check(hgnn, dev, [matrix(rows, cols)], [QUINTIC] * 5)
    check(hgnn, dev, [matrix(rows, cols, F16)], [CUBIC] * 7, F16, scales=[0.2 * max(1, rows / cols) ** 0.5], pitch=3, offset=1)


@pytest.mark.parametrize("rows,cols", [(4096, 4096), (4130, 4101)])
def test_tiles_left_over(hgnn, dev, rows, cols):
    """Sides whose tiles are a few more than run at once: those have their contraction cut and their sums joined."""
    check(hgnn, dev, [matrix(rows, cols)], [QUINTIC])


@pytest.mark.parametrize("rows,cols", [(1024, 1500), (1300, 1200), (100, 5000), (5000, 70), (2100, 300), (60, 4096), (4096, 33), (10, 4097), (2500, 2), (64, 4500)])
def test_large(hgnn, dev, rows, cols):
    check(hgnn, dev, [matrix(rows, cols)], [QUINTIC] * 5)


def test_result_is_orthogonal(hgnn, dev):
    """The classical steps to their end: singular values of one."""
    out = check(hgnn, dev, [matrix(48, 200)], [CUBIC] * 20)[0].double()
    s = torch.linalg.svdvals(out.cpu())
    assert float((s - 1).abs().max()) <= 1e-5


def test_lists(hgnn, dev):
    mats = [matrix(*s, dtype=t, seed=i) for i, (s, t) in enumerate([((64, 64), F32), ((608, 64), F16), ((64, 42), F32), ((300, 500), F32), ((1, 5), F16), ((42, 42), F32)])]
    check(hgnn, dev, mats, [QUINTIC] * 5, F32, scales=[1.0, -0.5, 2.0, 0.0, 1.0, 0.25])
    check(hgnn, dev, mats, [QUINTIC] * 5, F16)
    check(hgnn, dev, mats, [QUINTIC, CUBIC, (2.0, -1.5, 0.5)], in_place=True)
    assert hgnn.hgnn_orthogonalize_workspace([]) == 0
    hgnn.hgnn_orthogonalize([], None, [QUINTIC], None)
    check(hgnn, dev, mats, [], F32, scales=[3.0] * 6)  # no steps: divided by their norms


def test_nothing_and_what_has_no_norm(hgnn, dev):
    """Zeros and what is not finite give zeros; no rows or no columns nothing; very large and very small matrices what any others do."""
    m = matrix(40, 50)
    mats = [np.zeros((40, 50), F32), m.copy(), m.copy(), np.zeros((0, 5), F32), np.zeros((5, 0), F32), m * F32(1e30), m * F32(1e-30), np.full((3, 4), 65504, F16), np.full((2, 2), 2.0 ** -24, F16)]
    mats[1][3, 4], mats[2][0, 0] = np.nan, np.inf
    finite = [bool(np.isfinite(m).all()) for m in mats]
    check(hgnn, dev, [m for m, f in zip(mats, finite) if f], [QUINTIC] * 5)
    grads = [torch.from_numpy(m).to(dev) for m in mats]
    got = [torch.full(m.shape, 3.0, device=dev) for m in mats]
    ws = torch.empty(hgnn.hgnn_orthogonalize_workspace(grads), dtype=torch.uint8, device=dev)
    hgnn.hgnn_orthogonalize(grads, got, [QUINTIC] * 5, ws)
    assert finite.count(False) == 2 and all(bool((g == 0).all()) for g, f in zip(got, finite) if not f)


def test_the_same_bits_again_on_a_stream_and_in_a_graph(hgnn, dev):
    mats = [matrix(64, 64), matrix(608, 64), matrix(300, 700)]
    grads = [torch.from_numpy(m).to(dev) for m in mats]
    outs = [torch.zeros_like(g) for g in grads]
    ws = torch.empty(hgnn.hgnn_orthogonalize_workspace(grads), dtype=torch.uint8, device=dev)
    coef = [QUINTIC] * 5

    def call(stream=None):
        hgnn.hgnn_orthogonalize(grads, outs, coef, ws, stream=stream)

    def taken():
        torch.cuda.synchronize()
        return [t.clone() for t in outs]
    call()
    want = taken()
    ws.fill_(255)
    call()
    assert all(torch.equal(a, b) for a, b in zip(want, taken()))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, taken()))
    native, hgnn.binding._calls = hgnn.binding._calls, None
    try:
        call()
        assert native is not None and all(torch.equal(a, b) for a, b in zip(want, taken()))
    finally:
        hgnn.binding._calls = native
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        for g in grads:
            g.add_(0.1)
        graph.replay()
        replayed = taken()
        call()
        assert all(torch.equal(a, b) for a, b in zip(replayed, taken())), k


def test_refusals_of_the_binding(hgnn, dev):
    g, h = torch.ones(8, 16, device=dev), torch.ones(8, 16, dtype=torch.float16, device=dev)
    ws = torch.empty(hgnn.hgnn_orthogonalize_workspace([g]), dtype=torch.uint8, device=dev)
    q = [QUINTIC]
    for bad in (lambda: hgnn.hgnn_orthogonalize([g], [g[:, :8]], q, ws), lambda: hgnn.hgnn_orthogonalize([g.double()], None, q, ws), lambda: hgnn.hgnn_orthogonalize([g[0]], None, q, ws),
                lambda: hgnn.hgnn_orthogonalize([g], None, q, None), lambda: hgnn.hgnn_orthogonalize([g], None, q, ws[:64]), lambda: hgnn.hgnn_orthogonalize([g, h], [h, h], q, ws),
                lambda: hgnn.hgnn_orthogonalize([g], None, [(1.0, 2.0)], ws), lambda: hgnn.hgnn_orthogonalize([g], None, [(9.0, 0.0, 0.0)], ws), lambda: hgnn.hgnn_orthogonalize([g], None, [(float("nan"), 0, 0)], ws),
                lambda: hgnn.hgnn_orthogonalize([g], None, [(1.5, -70.0, 0.0)], ws), lambda: hgnn.hgnn_orthogonalize([g], None, [QUINTIC] * 65, ws), lambda: hgnn.hgnn_orthogonalize([g], None, q, ws, scales=[1.0, 2.0]),
                lambda: hgnn.hgnn_orthogonalize([g], None, q, ws, scales=[float("inf")]), lambda: hgnn.hgnn_orthogonalize([g.t()], None, q, ws), lambda: hgnn.hgnn_orthogonalize([g], [], q, ws)):
        with pytest.raises((hgnn.HgnnError, TypeError, ValueError)):
            bad()
