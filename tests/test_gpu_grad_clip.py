"""The norm over all gradients and the clipped gradients, against 64 bits on the host.

Tolerances, u = 2^-24.  Squares of fp16 are exact in fp32, eight of them are added there (8 u of a sum of squares, 4 u of the norm), all else in 64 bits; the stored norm is off by u more.  A
clipped value takes the factor's rounding and the product's, u each, and the norm's error; stored as fp16 2^-11 of it, or 2^-25."""
import numpy as np
import pytest
import torch

from parity import down, up

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NP = {torch.float16: np.float16, torch.float32: np.float32}
HALF, SINGLE = torch.float16, torch.float32
FILL = 7.0


def place(a, dev, pitch=None, offset=0):
    """A device copy; with a pitch a matrix in a buffer of that pitch that begins `offset` elements in -> (tensor, buffer)"""
    t = torch.from_numpy(np.ascontiguousarray(a))
    if pitch is None:
        buf = torch.full((t.numel() + offset + 1,), FILL, dtype=t.dtype, device=dev)
        v = buf[offset:offset + t.numel()].view(t.shape)
    else:
        buf = torch.full((t.shape[0] * pitch + offset + 1,), FILL, dtype=t.dtype, device=dev)
        v = torch.as_strided(buf, tuple(t.shape), (pitch, 1), offset)
    v.copy_(t)
    return v, buf


def check(hgnn, dev, arrays, outs=None, inv_scale=1.0, max_norm=1.0, pitches=None, offsets=None):
    """outs: types of the outputs, or None: in place"""
    pitches, offsets = pitches or [None] * len(arrays), offsets or [0] * len(arrays)
    ws = torch.full((hgnn.hgnn_grad_norm_workspace(),), 255, dtype=torch.uint8, device=dev)
    norm = torch.full((1,), FILL, device=dev)
    placed = [place(a, dev, p, o) for a, p, o in zip(arrays, pitches, offsets)]
    grads = [p[0] for p in placed]
    with np.errstate(invalid="ignore", over="ignore"):
        ref = inv_scale * np.sqrt(sum(float((a.astype(np.float64) ** 2).sum()) for a in arrays))
        stored = np.float64(np.float32(ref))
    hgnn.hgnn_grad_norm(grads, norm, ws, inv_scale=inv_scale)
    got = float(down(norm)[0])
    if np.isfinite(stored):
        assert abs(got - ref) <= 6 * U * ref + 2.0 ** -149, (got, ref)
    else:
        assert np.array_equal(np.float32(got), np.float32(ref), equal_nan=True)
    targets = [place(np.full(a.shape, 3, NP[o]), dev, p, f) for a, o, p, f in zip(arrays, outs, pitches, offsets)] if outs else placed
    norm.fill_(FILL)
    hgnn.hgnn_grad_clip(grads, max_norm, norm, ws, outs=[t[0] for t in targets] if outs else None, inv_scale=inv_scale)
    assert np.array_equal(np.float32(got), down(norm)[0], equal_nan=True)
    factor = np.float64(inv_scale) * (min(1.0, max_norm / ref) if ref > 0 else 1.0) if np.isfinite(stored) else 0.0
    for a, (t, buf), p, f in zip(arrays, targets, pitches, offsets):
        with np.errstate(invalid="ignore"):
            want = a.astype(np.float64) * factor if np.isfinite(stored) else np.zeros(a.shape)
        tol = 8 * U * np.abs(want) + 2.0 ** -149
        if t.dtype == HALF:
            tol += np.abs(want) * 2.0 ** -11 + 2.0 ** -25
        out = down(t).astype(np.float64)
        fits = np.abs(want) <= 65504 if t.dtype == HALF else np.ones(a.shape, bool)
        assert np.all(np.abs(out - want)[fits] <= tol[fits]) and np.all(np.isinf(out[np.abs(want) > 65520 * (1 + 8 * U)])) if t.dtype == HALF else np.all(np.abs(out - want) <= tol)
        whole, mask = down(buf), np.ones(buf.numel(), bool)
        rows = a.shape[0] if p is not None else 1
        mask[np.add.outer(np.arange(rows) * (p or 0) + f, np.arange(a.size // max(rows, 1))).ravel()] = False
        assert np.all(whole[mask] == FILL), "something beside the tensors was written"
        if outs:
            pass
    if outs:  # what was read is as it was
        for a, g in zip(arrays, grads):
            assert np.array_equal(down(g), a, equal_nan=True)


def arrays_of(shapes, rng, sd=1.0):
    return [(rng.standard_normal(s) * sd).astype(t) for s, t in shapes]


F16, F32 = np.float16, np.float32
LISTS = [
    [((1,), F32)], [((3,), F16)], [((64, 64), F16), ((64,), F32)], [((0,), F32), ((5,), F16), ((0, 4), F16)],
    [((7, 9, 11), F32), ((1001,), F16), ((2, 3), F16), ((33000,), F32)], [((200003,), F16)], [((1 << 20,), F32), ((3,), F16)], [((300, 1001), F32)] * 3,
]


@pytest.mark.parametrize("shapes", LISTS, ids=[str(i) for i in range(len(LISTS))])
@pytest.mark.parametrize("inv_scale,max_norm", [(1.0, 1.0), (2.0 ** -10, 1.0), (2.0 ** -10, 0.001), (1.0, 1e30), (3.0, float("inf")), (1.0, 0.0)])
def test_lists(hgnn, dev, shapes, inv_scale, max_norm):
    print(f"clip {shapes} inv_scale={inv_scale} max_norm={max_norm}", flush=True)
    rng = np.random.default_rng(len(shapes))
    a = arrays_of(shapes, rng, 1.0 / inv_scale if inv_scale < 1 else 1.0)
    check(hgnn, dev, a, None, inv_scale, max_norm)
    check(hgnn, dev, a, [SINGLE] * len(a), inv_scale, max_norm)
    check(hgnn, dev, a, [HALF] * len(a), inv_scale, max_norm)
    check(hgnn, dev, a, None, inv_scale, max_norm, offsets=[i % 5 + 1 for i in range(len(a))])


@pytest.mark.parametrize("count", [55, 56, 57, 95, 96, 97, 113, 192, 193, 400])
def test_many_tensors(hgnn, dev, count):
    """More than the arguments of a launch hold; a small first launch and a large last one."""
    print(f"clip of {count}", flush=True)
    rng = np.random.default_rng(count)
    shapes = [((int(rng.integers(1, 300)),), (F16, F32)[i % 2]) for i in range(count - 1)] + [((2000003,), F32)]
    check(hgnn, dev, arrays_of(shapes, rng))
    check(hgnn, dev, arrays_of(shapes[::-1], rng), [SINGLE] * count)


PITCHED = [((5, 3), 4), ((100, 42), 48), ((1, 10), 16), ((3, 40000), 40001), ((7000, 7), 8), ((333, 130), 200), ((2, 65537), 65552), ((50000, 1), 3)]


@pytest.mark.parametrize("dtype", [F16, F32])
def test_matrices_with_a_pitch(hgnn, dev, dtype):
    """What is between the rows is not counted, and not written."""
    rng = np.random.default_rng(8)
    for shape, pitch in PITCHED:
        print(f"clip {shape} pitch {pitch}", flush=True)
        a = [rng.standard_normal(shape).astype(dtype), rng.standard_normal(100).astype(F32)]
        check(hgnn, dev, a, None, pitches=[pitch, None], offsets=[1, 0])
        check(hgnn, dev, a, [HALF, SINGLE], pitches=[pitch, None])
    # rows with gaps into a tensor without, and the other way round
    m = rng.standard_normal((40, 42)).astype(dtype)
    gaps, _ = place(m, dev, 48)
    dense = torch.empty((40, 42), device=dev)
    ws = torch.empty(hgnn.hgnn_grad_norm_workspace(), dtype=torch.uint8, device=dev)
    norm = torch.empty(1, device=dev)
    hgnn.hgnn_grad_clip([gaps], float("inf"), norm, ws, outs=[dense])
    assert np.array_equal(down(dense), m.astype(F32))
    back = torch.zeros((40, 48), device=dev)[:, :42]
    hgnn.hgnn_grad_clip([dense], float("inf"), norm, ws, outs=[back])
    assert np.array_equal(down(back), m.astype(F32))


def test_far_values(hgnn, dev):
    """Squares beyond fp32, tiny values, infinities and NaN."""
    rng = np.random.default_rng(2)
    check(hgnn, dev, [np.full(1000, 1e25, F32), np.full(9, 1.0, F32)])
    check(hgnn, dev, [np.full(1000, 3e-30, F32)], max_norm=1e-29)
    check(hgnn, dev, [np.full(100000, 65504, F16)], [SINGLE], inv_scale=2.0 ** -16)
    check(hgnn, dev, [np.full(100, 3e38, F32)])  # each is finite, the norm is not
    check(hgnn, dev, [np.zeros(100, F32), np.zeros(3, F16)])
    check(hgnn, dev, [np.array([1e20, 1e-20, -1e20], F32)], [HALF], max_norm=float("inf"))
    for bad in (np.inf, -np.inf, np.nan):
        for dtype in (F16, F32):
            a = arrays_of([((5000,), dtype), ((70000,), F32)], rng)
            a[0][4321] = bad
            check(hgnn, dev, a)
            check(hgnn, dev, a, [SINGLE, HALF], max_norm=float("inf"))


def test_nothing(hgnn, dev):
    ws = torch.full((hgnn.hgnn_grad_norm_workspace(),), 255, dtype=torch.uint8, device=dev)
    norm = torch.full((1,), FILL, device=dev)
    hgnn.hgnn_grad_norm([], norm, ws)
    assert float(norm) == 0
    for grads in ([], [torch.empty(0, device=dev)]):
        norm.fill_(FILL)
        hgnn.hgnn_grad_clip(grads, 1.0, norm, ws)
        assert float(norm) == 0


def test_the_same_bits_again(hgnn, dev):
    gen = torch.Generator(device=dev).manual_seed(1)
    grads = [torch.randn(n, generator=gen, device=dev) for n in (3000000, 17, 500001)] + [torch.randn(999, generator=gen, device=dev).half()]
    ws = torch.empty(hgnn.hgnn_grad_norm_workspace(), dtype=torch.uint8, device=dev)
    norms = []
    for _ in range(3):
        norm = torch.empty(1, device=dev)
        hgnn.hgnn_grad_norm(grads, norm, ws)
        norms.append(norm)
    assert torch.equal(norms[0], norms[1]) and torch.equal(norms[0], norms[2])


def test_far_elements(hgnn, dev):
    """A tensor of more than 2^31 elements."""
    n = 2 ** 31 + 12345
    g = torch.zeros(n, dtype=HALF, device=dev)
    g[-1], g[5], g[2 ** 31 - 1] = 3.0, 4.0, 12.0
    ws = torch.empty(hgnn.hgnn_grad_norm_workspace(), dtype=torch.uint8, device=dev)
    norm = torch.empty(1, device=dev)
    hgnn.hgnn_grad_clip([g], 6.5, norm, ws)
    assert float(norm) == 13.0 and [float(g[i]) for i in (-1, 5, 2 ** 31 - 1)] == [1.5, 2.0, 6.0] and int(torch.count_nonzero(g)) == 3
