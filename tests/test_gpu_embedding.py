"""Rows of a learned table by id and the table's gradient, against their definition in 64 bits on the host.

Tolerances.  A row times the scale is rounded to fp32 and then to fp16: 2^-24 + 2^-11 of the value, half a subnormal step (2^-25) below the normal range.  A sum of m
rows in fp32, in any order, is off by at most m * 2^-24 of the sum of the magnitudes, the scale and a stored fp32 value by 2^-24 of the value each, one in fp16 by
2^-11 of it or 2^-25."""
import numpy as np
import pytest
import torch

from parity import down, up

pytestmark = pytest.mark.gpu

NP = {torch.float16: np.float16, torch.float32: np.float32}
FILL = 7.0  # of what may not be written


def view(rows, cols, pitch, dtype, dev, offset=0, data=None):
    """-> (tensor of rows x cols inside a buffer of that pitch that begins `offset` elements in, the buffer)"""
    buf = torch.full((rows * pitch + offset + 1,), FILL, dtype=dtype, device=dev)
    v = torch.as_strided(buf, (rows, cols), (pitch, 1), offset)
    if data is not None:
        v.copy_(up(data, dev))
    return v, buf


def ids_of(n, V, kind, rng):
    if kind == "uniform":
        ids = rng.integers(0, V, n)
    elif kind == "one":  # all the same
        ids = np.full(n, V // 2)
    elif kind == "hubs":  # half of them one id, the others few
        ids = np.where(rng.random(n) < 0.5, V - 1, rng.integers(0, max(V // 50, 1), n))
    elif kind == "none":  # nothing but padding
        ids = np.where(rng.random(n) < 0.5, -1, V)
    else:  # ids that are none among the others, the type's ends too
        ids = rng.choice(np.array([-1, V, -2 ** 31, 2 ** 31 - 1]), n)
        ids = np.where(rng.random(n) < 0.3, ids, rng.integers(0, V, n))
    return ids.astype(np.int32)


LOOKUPS = [  # n, V, F, pitch of the table, of the output, offset into both buffers
    (1, 1, 1, 1, 1, 0), (3, 5, 7, 7, 7, 0), (64, 4096, 64, 64, 64, 0), (1000, 300, 42, 48, 48, 0), (257, 100, 333, 333, 335, 1), (100, 50, 1000, 1001, 1008, 3),
    (5000, 20000, 128, 128, 128, 0), (4097, 33, 8, 9, 11, 5), (70, 10, 512, 520, 512, 8), (33, 9, 2500, 2500, 2500, 0), (100000, 1000, 2, 2, 2, 0),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("n,V,F,ldt,ldo,offset", LOOKUPS)
def test_lookup(hgnn, dev, n, V, F, ldt, ldo, offset, dtype):
    print(f"lookup n={n} V={V} F={F} {dtype}", flush=True)
    rng = np.random.default_rng(n + V + F)
    T = rng.standard_normal((V, F)).astype(NP[dtype])
    table, _ = view(V, F, ldt, dtype, dev, offset, T)
    for kind, scale in (("uniform", 1.0), ("padded", 3.3), ("none", 2.0)):
        ids = ids_of(n, V, kind, rng)
        out, buf = view(n, F, ldo, torch.float16, dev, offset)
        hgnn.hgnn_embedding(up(ids, dev), table, out, scale=scale)
        got, whole = down(out), down(buf)
        real = (ids >= 0) & (ids < V)
        ref = np.where(real[:, None], T[np.where(real, ids, 0)].astype(np.float64) * np.float64(np.float32(scale)), 0.0)
        if scale == 1.0:
            assert np.array_equal(got, ref.astype(np.float16))
        assert np.all(np.abs(got - ref) <= np.abs(ref) * (2.0 ** -11 + 2.0 ** -24) + 2.0 ** -25)
        mask = np.ones(whole.size, bool)
        mask[np.add.outer(np.arange(n) * ldo + offset, np.arange(F)).ravel()] = False
        assert np.all(whole[mask] == FILL), "something beside the rows was written"


def test_lookup_takes_values_as_they_are(hgnn, dev):
    """Infinities and NaN stay, values beyond fp16 become infinite, padding is zero beside them."""
    T = np.array([[np.inf, -np.inf, np.nan, 65519.0, 65521.0, 1e-9]], np.float32)
    out = torch.full((2, 6), FILL, dtype=torch.float16, device=dev)
    hgnn.hgnn_embedding(up(np.array([0, -1], np.int32), dev), up(T, dev), out)
    got = down(out)
    assert np.array_equal(got[0], np.array([np.inf, -np.inf, np.nan, 65504, np.inf, 0], np.float16), equal_nan=True) and np.all(got[1] == 0)


@pytest.mark.parametrize("scale", [float("inf"), float("nan"), 1e30])
def test_padding_is_zero_whatever_the_scale(hgnn, dev, scale):
    T = np.ones((3, 11), np.float32)
    out = torch.full((5, 11), FILL, dtype=torch.float16, device=dev)
    hgnn.hgnn_embedding(up(np.array([3, 2, -1, 0, -2 ** 31], np.int32), dev), up(T, dev), out, scale=scale)
    got = down(out)
    assert np.all(got[[0, 2, 4]] == 0) and np.array_equal(got[[1, 3]], np.full((2, 11), np.inf if scale == scale else np.nan, np.float16), equal_nan=True)


def test_lookup_far_rows(hgnn, dev):
    """Rows beyond 2^31 elements of a table, and beyond 2^31 bytes of the output."""
    V, F = 2 ** 31 // 256 + 7, 256
    table = torch.zeros((V, F), dtype=torch.float16, device=dev)
    table[V - 1] = 3.0
    table[V - 5] = 5.0
    n = 2 ** 31 // 512 + 3
    ids = torch.full((n,), V - 1, dtype=torch.int32, device=dev)
    ids[-1] = V - 5
    out = torch.zeros((n, F), dtype=torch.float16, device=dev)
    hgnn.hgnn_embedding(ids, table, out)
    torch.cuda.synchronize()
    assert bool((out[:-1] == 3).all()) and bool((out[-1] == 5).all())


def check_grad(hgnn, dev, ids, dY, V, F, dtype, scale, add, ldy, ldt, offset=0, label=""):
    n = ids.size
    print(f"table gradient {label} n={n} V={V} F={F} {dtype} scale={scale} add={add}", flush=True)
    rng = np.random.default_rng(5)
    y, _ = view(n, F, ldy, torch.float16, dev, offset, dY)
    before = rng.standard_normal((V, F)).astype(NP[dtype]) if add else None
    T, buf = view(V, F, ldt, dtype, dev, offset, before)
    need = hgnn.hgnn_embedding_grad_workspace(n, F, V)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device=dev)  # NaN in every word
    d = up(ids, dev)
    hgnn.hgnn_embedding_grad(d, y, T, ws, scale=scale, accumulate=add)
    got, whole = down(T).astype(np.float64), down(buf)
    real = (ids >= 0) & (ids < V)
    ref, mag, m = np.zeros((V, F)), np.zeros((V, F)), np.zeros(V)
    s = np.float64(np.float32(scale))
    np.add.at(ref, ids[real], dY[real].astype(np.float64) * s)
    np.add.at(mag, ids[real], np.abs(dY[real].astype(np.float64) * s))
    np.add.at(m, ids[real], 1)
    if add:
        ref += before
        mag += np.abs(before) * (m > 0)[:, None]
    tol = ((m + 1)[:, None] * mag + 2 * np.abs(ref)) * 2.0 ** -24
    if dtype == torch.float16:
        tol += np.abs(ref) * 2.0 ** -11 + 2.0 ** -25
    if add:
        assert np.array_equal(got[m == 0], before[m == 0].astype(np.float64)), "rows without an id were touched"
    else:
        assert np.all(got[m == 0] == 0)
    err = np.abs(got - ref)
    assert np.all(err[m > 0] <= tol[m > 0]), (label, err.max(), tol[np.unravel_index(err.argmax(), err.shape)])
    mask = np.ones(whole.size, bool)
    mask[np.add.outer(np.arange(V) * ldt + offset, np.arange(F)).ravel()] = False
    assert np.all(whole[mask] == FILL), "something beside the rows was written"
    if not add:  # the same bits again, whatever the workspace and the output held
        ws.fill_(1)
        T2 = torch.full((V, F), FILL, dtype=dtype, device=dev)
        hgnn.hgnn_embedding_grad(d, y, T2, ws, scale=scale)
        assert torch.equal(T2, T.contiguous())


GRADS = [  # n, V, F, pitch of dY, of dT, offset
    (1, 1, 1, 1, 1, 0), (2, 3, 5, 5, 5, 0), (16, 4, 8, 8, 8, 0), (17, 40, 64, 64, 64, 0), (1000, 4096, 64, 64, 64, 0), (1023, 7, 42, 48, 48, 0),
    (5000, 300, 100, 101, 103, 1), (8193, 20000, 16, 16, 16, 0), (20011, 97, 200, 200, 200, 0), (3000, 50, 1000, 1000, 1000, 0), (30000, 5, 2, 3, 2, 0),
    (2049, 1000, 513, 520, 515, 3), (200003, 1001, 24, 24, 24, 0),
]


@pytest.mark.parametrize("kind", ["uniform", "hubs", "one", "padded", "none"])
@pytest.mark.parametrize("n,V,F,ldy,ldt,offset", GRADS)
def test_table_gradient(hgnn, dev, n, V, F, ldy, ldt, offset, kind):
    rng = np.random.default_rng(n + V + F)
    ids = ids_of(n, V, kind, rng)
    dY = rng.standard_normal((n, F)).astype(np.float16)
    for dtype, scale, add in ((torch.float32, 1.0, False), (torch.float16, 0.1, False), (torch.float32, 3.0, True), (torch.float16, 1.0, True)):
        check_grad(hgnn, dev, ids, dY, V, F, dtype, scale, add, ldy, ldt, offset, kind)


def test_table_gradient_of_runs_that_end_at_shares(hgnn, dev):
    """Runs of every length up to some shares, one behind the other, in the order of the ids and mixed."""
    lengths = np.concatenate([np.arange(1, 70), [16, 16, 32, 48, 15, 17, 128, 256, 512, 1024, 1023, 1025, 2048, 40000]])
    ids = np.repeat(np.arange(lengths.size), lengths).astype(np.int32)
    rng = np.random.default_rng(1)
    for order in (np.arange(ids.size), rng.permutation(ids.size)):
        dY = rng.standard_normal((ids.size, 40)).astype(np.float16)
        check_grad(hgnn, dev, ids[order], dY, lengths.size, 40, torch.float32, 1.0, False, 40, 40, label="runs")


@pytest.mark.parametrize("kind", ["uniform", "hubs", "one"])
def test_table_gradient_of_many_positions(hgnn, dev, kind):
    """Longer shares, and a run over more workgroups than one has groups of lanes."""
    rng = np.random.default_rng(6)
    n, V, F = 2 ** 19 + 77, 3001, 12
    check_grad(hgnn, dev, ids_of(n, V, kind, rng), rng.standard_normal((n, F)).astype(np.float16), V, F, torch.float32, 1.0, False, 16, 12, label=kind)


def test_table_gradient_without_positions(hgnn, dev):
    T = torch.full((70, 9), FILL, device=dev)
    none = torch.empty((0,), dtype=torch.int32, device=dev)
    dY = torch.empty((0, 9), dtype=torch.float16, device=dev)
    hgnn.hgnn_embedding_grad(none, dY, T, None, accumulate=True)
    assert bool((T == FILL).all())
    hgnn.hgnn_embedding_grad(none, dY, T, None)
    assert bool((T == 0).all())


def test_table_gradient_far_rows(hgnn, dev):
    """Rows of dT beyond 2^31 elements."""
    V, F = 2 ** 31 // 128 + 5, 128
    T = torch.full((V, F), FILL, dtype=torch.float16, device=dev)
    ids = torch.tensor([V - 1, 3, V - 1, V - 4], dtype=torch.int32, device=dev)
    dY = torch.arange(1, 5, device=dev).half()[:, None].expand(4, F).contiguous()
    ws = torch.empty(hgnn.hgnn_embedding_grad_workspace(4, F, V), dtype=torch.uint8, device=dev)
    hgnn.hgnn_embedding_grad(ids, dY, T, ws)
    assert [float(T[v].float().min()) for v in (V - 1, V - 4, 3)] == [4, 4, 2] and [float(T[v].float().max()) for v in (V - 1, V - 4, 3)] == [4, 4, 2]
    T[[V - 1, V - 4, 3]] = 0
    assert int(torch.count_nonzero(T)) == 0


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("F,ldt,offset", [(100, 104, 0), (333, 333, 0), (256, 256, 0), (161, 200, 3), (1000, 1008, 0), (1300, 1301, 1)])
def test_table_gradient_of_large_tables(hgnn, dev, F, ldt, offset, dtype):
    """Tables too large for the last-level cache: rows and zeros in whole lines and in parts of lines, what lies between the rows as it was, NaN at positions without an id."""
    size = 2 if dtype == torch.float16 else 4
    V = (2 ** 28 + 2 ** 20) // (ldt * size)
    buf = torch.full((V * ldt + offset,), FILL, dtype=dtype, device=dev)
    T = torch.as_strided(buf, (V, F), (ldt, 1), offset)
    ids = torch.tensor([5, V - 1, -1, 5, V, 64, 63, 5, V // 2], dtype=torch.int32, device=dev)
    dY = torch.arange(1, 10, device=dev).half()[:, None].repeat(1, F)
    dY[2] = dY[4] = float("nan")
    ws = torch.empty(hgnn.hgnn_embedding_grad_workspace(9, F, V), dtype=torch.uint8, device=dev)
    hgnn.hgnn_embedding_grad(ids, dY, T, ws)
    for v, want in ((5, 1 + 4 + 8), (V - 1, 2), (64, 6), (63, 7), (V // 2, 9)):
        assert bool((T[v] == want).all()), v
        T[v] = 0
    assert int(torch.count_nonzero(T)) == 0
    if ldt > F:  # the rows are counted out, the rest is as it was
        T.fill_(FILL)
        assert bool((buf == FILL).all())


@pytest.mark.parametrize("F", [65535, 65536])
def test_widest_rows(hgnn, dev, F):
    rng = np.random.default_rng(F)
    n, V = 75, 6
    ids = ids_of(n, V, "hubs", rng)
    dY = rng.standard_normal((n, F)).astype(np.float16)
    for dtype, add in ((torch.float32, False), (torch.float16, True)):
        check_grad(hgnn, dev, ids, dY, V, F, dtype, 0.5, add, F + 1, F, label="widest")
    T = up(rng.standard_normal((V, F)).astype(np.float16), dev)
    out = torch.full((n, F), FILL, dtype=torch.float16, device=dev)
    hgnn.hgnn_embedding(up(ids, dev), T, out)
    real = (ids >= 0) & (ids < V)
    assert np.array_equal(down(out), np.where(real[:, None], down(T)[np.where(real, ids, 0)], np.float16(0)))


def test_gradient_is_the_lookups(hgnn, dev):
    """<lookup(T), dY> moves with T as the gradient says: the lookup is linear in T, so differences are exact up to the roundings of both sides."""
    rng = np.random.default_rng(3)
    n, V, F = 300, 40, 24
    ids = ids_of(n, V, "padded", rng)
    d = up(ids, dev)
    dY = rng.integers(-8, 9, (n, F)).astype(np.float16)
    T = torch.zeros((V, F), device=dev)
    dT = torch.empty((V, F), device=dev)
    ws = torch.empty(hgnn.hgnn_embedding_grad_workspace(n, F, V), dtype=torch.uint8, device=dev)
    hgnn.hgnn_embedding_grad(d, up(dY, dev), dT, ws, scale=0.5)
    got = down(dT)
    out = torch.empty((n, F), dtype=torch.float16, device=dev)
    for v, f in ((0, 0), (7, 23), (39, 11), (20, 3)):
        T.zero_()
        T[v, f] = 1.0
        hgnn.hgnn_embedding(d, T, out, scale=0.5)
        assert float((down(out).astype(np.float64) * dY).sum()) == got[v, f]  # small whole numbers and halves: no rounding anywhere
