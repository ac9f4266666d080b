"""Log probabilities of labels, entropies, best alternatives and their gradient, against the definitions in 64 bits on the host.

Tolerances, u = 2^-24.  With d = x - max, e = exp(d): d is off by u |d|, the argument of the power of two by 2 u |d| more and the power by 2 u, so e by (3 |d| + 2) u of itself; a
lane adds up to D classes (and joins some 16 times), 2 u each.  So S = sum e is off by (2 D + 34 + 3 sum p |d|) u of itself, and log S by as much plus 2 u |log S|; the log
probability adds u (|d| + |log p|) of its own.  sum p d is off by sum p |d| (3 |d| + 5 + 2 D + 34) u.  The gradient's p is off by what log p is plus (3 |log p| + 2) u of itself."""
import numpy as np
import pytest
import torch

from parity import down, up

pytestmark = pytest.mark.gpu

NP = {torch.float16: np.float16, torch.float32: np.float32}
U = 2.0 ** -24
FILL = 7.0


def reference(x):
    """-> dict of float64: max, L, log p, p, entropy, and what the tolerances need; rows of -inf alone as the interface has them"""
    x = x.astype(np.float64)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = x.max(1)
        empty = np.isneginf(m)
        d = x - np.where(empty, 0, m)[:, None]
        e = np.exp(d)
        S = np.where(empty, 1, e.sum(1))
        L = np.log(S)
        lp = d - L[:, None]
        p = e / S[:, None]
        far = np.where(p > 0, np.abs(d), 0)
        H = L + (p * far).sum(1)
    D = -(-x.shape[1] // 256) + 8
    first, second = (p * far).sum(1), (p * far * far).sum(1)
    dL = (2 * D + 34 + 3 * first) * U + 2 * U * np.abs(L)
    dH = dL + (3 * second + (39 + 2 * D) * first) * U + 2 * U * (np.abs(L) + first)
    return dict(m=m, L=L, lp=lp, p=p, H=H, d=d, dL=dL, dH=dH, empty=empty)


def tol_lp(r):
    with np.errstate(invalid="ignore"):
        return r["dL"][:, None] + 2 * U * (np.where(np.isfinite(r["d"]), np.abs(r["d"]), 0) + np.where(np.isfinite(r["lp"]), np.abs(r["lp"]), 0))


def near(got, ref, tol):
    """equal where the reference is not finite, within the tolerance elsewhere"""
    # what is above fp32's largest value by half of its last step or more (2^128 - 2^103: a lowest score beside a largest one, -2 * (2^128 - 2^104)) rounds to infinity
    ref = np.where(np.abs(ref) >= 2.0 ** 128 - 2.0 ** 103, np.copysign(np.inf, ref), ref)
    got, fine = got.astype(np.float64), np.isfinite(ref)
    assert np.array_equal(got[~fine], ref[~fine], equal_nan=True)
    err = np.abs(got[fine] - ref[fine])
    assert np.all(err <= tol[fine]), (err.max(), tol[fine][err.argmax()])


def alternatives(x, k):
    order = np.argsort(-x.astype(np.float64), axis=1, kind="stable")
    return order[:, :k]


def placed(a, pitch, offset, dev):
    n, C = a.shape
    buf = torch.full((n * pitch + offset + 1,), FILL, dtype=torch.float16 if a.dtype == np.float16 else torch.float32, device=dev)
    v = torch.as_strided(buf, (n, C), (pitch, 1), offset)
    v.copy_(up(a, dev))
    return v, buf


def run(hgnn, dev, x, labels, k, pitch, offset=0):
    n, C = x.shape
    t, _ = placed(x, pitch, offset, dev)
    need = hgnn.hgnn_logprob_workspace(n, C, k)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=dev) if need else None
    make = lambda *s: torch.full(s, FILL, device=dev)  # noqa: E731
    out = dict(logprob=make(n), stats=make(n, 2), entropy=make(n))
    if k:
        out.update(top_logprob=make(n, k), top_class=torch.full((n, k), -5, dtype=torch.int32, device=dev))
    y = up(labels, dev)
    hgnn.hgnn_logprob(t, y, workspace=ws, **out)
    return t, y, out


def check(hgnn, dev, x, labels, k, pitch, offset=0):
    n, C = x.shape
    t, y, out = run(hgnn, dev, x, labels, k, pitch, offset)
    r = reference(x)
    T = tol_lp(r)
    rows = np.arange(n)
    real = (labels >= 0) & (labels < C)
    at = np.where(real, labels, 0)
    near(down(out["logprob"]), np.where(real, r["lp"][rows, at], 0.0), np.where(real, T[rows, at], 0.0))
    stats = down(out["stats"]).astype(np.float64)
    assert np.array_equal(stats[:, 0], r["m"])
    near(stats[:, 1], r["L"], r["dL"])
    near(down(out["entropy"]), r["H"], r["dH"])
    if k:
        best = alternatives(x, k)
        assert np.array_equal(down(out["top_class"]), best)
        near(down(out["top_logprob"]), np.take_along_axis(r["lp"], best, 1), np.take_along_axis(T, best, 1))
    return t, y, out, r


def check_grad(hgnn, dev, x, labels, pitch, offset, t, y, out, r, with_entropy, rng):
    n, C = x.shape
    g = rng.standard_normal(n).astype(np.float32)
    h = rng.standard_normal(n).astype(np.float32) if with_entropy else np.zeros(n, np.float32)
    dx, buf = placed(np.full((n, C), 3, x.dtype), pitch, offset, dev)
    more = dict(entropy=out["entropy"], dentropy=up(h, dev)) if with_entropy else {}
    hgnn.hgnn_logprob_grad(t, y, out["stats"], up(g, dev), dx, **more)
    real = (labels >= 0) & (labels < C) & ~r["empty"]
    g64 = np.where(real, g, 0).astype(np.float64)[:, None]
    hot = np.zeros((n, C))
    hot[np.arange(n)[real], labels[real]] = 1
    p = r["p"]
    with np.errstate(invalid="ignore"):
        term = np.where(p > 0, p * (r["lp"] + r["H"][:, None]), 0)
        ref = g64 * (hot - p) - h[:, None].astype(np.float64) * term
        lp = np.where(p > 0, np.abs(r["lp"]), 0)
        size = lp + r["H"][:, None]
        rel = tol_lp(r) + (3 * lp + 4) * U
        tol = np.abs(g64) * (p * rel + U * (hot + p)) + np.abs(h[:, None]) * p * (size * (rel + 4 * U) + tol_lp(r) + r["dH"][:, None]) + 4 * U * np.abs(ref) + 2.0 ** -126
    if x.dtype == np.float16:
        tol = tol * (1 + 2.0 ** -11) + np.abs(ref) * 2.0 ** -11 + 2.0 ** -25
    near(down(dx), ref, tol)
    whole = down(buf)
    mask = np.ones(whole.size, bool)
    mask[np.add.outer(np.arange(n) * pitch + offset, np.arange(C)).ravel()] = False
    assert np.all(whole[mask] == FILL), "something beside the rows was written"
    again = t.clone() if t.is_contiguous() else t  # in its own place
    hgnn.hgnn_logprob_grad(again, y, out["stats"], up(g, dev), again, **more)
    assert np.array_equal(down(again), down(dx))


SHAPES = [  # n, C, pitch, offset, k
    (1, 1, 1, 0, 1), (5, 2, 2, 0, 2), (1000, 7, 7, 0, 3), (333, 8, 8, 0, 0), (70, 9, 11, 1, 9), (4099, 41, 48, 0, 5), (300, 47, 47, 3, 8), (129, 100, 104, 0, 1),
    (65, 255, 255, 0, 20), (64, 512, 512, 0, 32), (33, 513, 513, 1, 5), (40, 1000, 1000, 0, 8), (17, 2047, 2048, 0, 4), (9, 2049, 2051, 5, 32), (3, 8192, 8192, 0, 5),
    (1, 50021, 50021, 0, 8), (2, 100003, 100003, 0, 0), (1, 131072, 131072, 0, 20), (1100, 5003, 5003, 0, 2), (1, 300007, 300008, 0, 5),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("n,C,pitch,offset,k", SHAPES)
def test_shapes(hgnn, dev, n, C, pitch, offset, k, dtype):
    print(f"logprob n={n} C={C} pitch={pitch} k={k} {dtype}", flush=True)
    rng = np.random.default_rng(n + C + k)
    x = (rng.standard_normal((n, C)) * 2).astype(NP[dtype])
    labels = rng.integers(0, C, n).astype(np.int32)
    labels[rng.random(n) < 0.2] = -1
    if n > 3:
        labels[:4] = C, -2 ** 31, 2 ** 31 - 1, C - 1
    got = check(hgnn, dev, x, labels, k, pitch, offset)
    for with_entropy in (False, True):
        t, y, out, r = check(hgnn, dev, x, labels, k, pitch, offset) if with_entropy else got
        check_grad(hgnn, dev, x, labels, pitch, offset, t, y, out, r, with_entropy, rng)


ROWS = [(65536, 9, 9, 0, 9), (66001, 41, 48, 0, 5), (70000, 16, 17, 1, 2), (65800, 64, 64, 0, 20), (80001, 57, 59, 3, 0), (68000, 24, 24, 0, 1), (70000, 47, 47, 0, 8), (66000, 33, 40, 0, 32),
        (65536, 64, 64, 0, 3), (65600, 33, 40, 0, 5), (66000, 27, 29, 1, 4), (66000, 49, 50, 1, 5), (4100, 300, 300, 0, 20), (4097, 512, 513, 1, 9), (4096, 257, 264, 0, 32)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("n,C,pitch,offset,k", ROWS)
def test_many_rows_of_few_classes(hgnn, dev, n, C, pitch, offset, k, dtype):
    """With rows among them that the mask leaves empty or nearly so, whose scores are equal, and that hold no numbers."""
    print(f"logprob n={n} C={C} pitch={pitch} k={k} {dtype}", flush=True)
    rng = np.random.default_rng(n + C + k)
    x = (rng.standard_normal((n, C)) * 2).astype(NP[dtype])
    x[5], x[64 * 7 + 63], x[n - 1] = -np.inf, -np.inf, 1.0
    x[9], x[9, C - 1] = -np.inf, 3.0
    x[100:200] = np.round(x[100:200])
    x[300:400][rng.random((100, C)) < 0.7] = -np.inf
    x[500] = np.finfo(NP[dtype]).min
    labels = rng.integers(0, C, n).astype(np.int32)
    labels[rng.random(n) < 0.2] = -1
    labels[:4] = C, -2 ** 31, 2 ** 31 - 1, C - 1
    for with_entropy in (False, True):
        t, y, out, r = check(hgnn, dev, x, labels, k, pitch, offset)
        check_grad(hgnn, dev, x, labels, pitch, offset, t, y, out, r, with_entropy, rng)
    x[77, C // 2] = np.nan
    x[78, 0] = np.inf
    t, y, out = run(hgnn, dev, x, labels, k, pitch, offset)
    for name in ("logprob", "stats", "entropy") + (("top_logprob",) if k else ()):
        v = down(out[name]).reshape(n, -1)
        bad = np.isnan(v).any(1)
        assert bad[77] == (name != "logprob" or 0 <= labels[77] < C) and np.all(np.isnan(v[bad])) and not bad[[76, 79, 80]].any(), name
    if k:
        c = down(out["top_class"])
        assert np.all((c >= 0) & (c < C)) and all(len(set(c[i])) == k for i in (77, 78, 5, 9))


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("C", [1, 2, 7, 8, 9, 16, 17, 33, 64, 65, 128, 129, 247, 511, 512, 513, 2049, 3200, 20011])
def test_all_alternatives(hgnn, dev, C, dtype):
    """As many alternatives as there may be, of rows that lanes share, of one for a wave or more: equal scores, both zeros, few above -inf, the last rows of a wave; NaN takes places, but no two the same."""
    rng = np.random.default_rng(C)
    n, k = 75, min(C, 32)
    x = rng.standard_normal((n, C)).astype(NP[dtype])
    x[3:20] = np.round(x[3:20])
    x[20:30] = np.where(rng.random((10, C)) < 0.5, NP[dtype](-0.0), NP[dtype](0.0))
    x[30:50][rng.random((20, C)) < 0.8] = -np.inf
    x[50], x[51] = -np.inf, np.finfo(NP[dtype]).min
    x[52] = np.arange(C)
    x[53] = -np.arange(C)
    labels = rng.integers(0, C, n).astype(np.int32)
    for m in sorted({1, (k + 1) // 2, k}):
        check(hgnn, dev, x, labels, m, C)
    x[60:70][rng.random((10, C)) < 0.3] = np.nan
    x[60:70, C // 2] = np.nan
    t, y, out = run(hgnn, dev, x, labels, k, C)
    c, v = down(out["top_class"]), down(out["top_logprob"])
    assert np.all((c >= 0) & (c < C)) and all(len(set(row)) == k for row in c)
    assert np.all(np.isnan(v[60:70])) and not np.isnan(np.delete(v, range(60, 70), 0)).any()
    keep = np.delete(np.arange(n), range(60, 70))
    assert np.array_equal(c[keep], alternatives(x[keep], k))


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("C", [6, 41, 300, 700, 5000, 70001])
def test_masks_and_far_values(hgnn, dev, C, dtype):
    """Rows where the mask (-inf, or the type's lowest value) leaves little or nothing, equal scores, scores at the ends of the type, very sure ones."""
    print(f"masks C={C} {dtype}", flush=True)
    rng = np.random.default_rng(C)
    top = np.finfo(NP[dtype]).max
    x = (rng.standard_normal((14, C)) * 3).astype(NP[dtype])
    x[0] = -np.inf
    x[1], x[1, C // 2] = -np.inf, 2.5
    x[2], x[2, C - 1], x[2, 0] = -np.inf, 1.0, 1.0
    x[3] = -top
    x[4], x[4, 3] = -top, 0.0
    x[5] = 1.5  # all equal
    x[6, ::2] = -np.inf
    x[7] = top
    x[8], x[8, 1] = -top, top
    x[9, 4] = 60.0 if C > 4 else 0.0
    x[10] = np.where(rng.random(C) < 0.98, -np.inf, x[10])
    x[11] = np.round(x[11])  # many equal scores
    x[12] = x[12] * 1000
    x[13] = np.where(np.arange(C) < C - 2, -np.inf, 0.0)
    labels = rng.integers(0, C, 14).astype(np.int32)
    labels[0], labels[1], labels[6] = 2, C // 2, 1
    for k in (1, min(5, C)):
        t, y, out, r = check(hgnn, dev, x, labels, k, C)
    check_grad(hgnn, dev, x, labels, C, 0, t, y, out, r, True, rng)


@pytest.mark.parametrize("C", [5, 41, 600, 20011])
def test_infinite_and_no_numbers(hgnn, dev, C):
    """Rows with +inf or NaN are NaN everywhere, their alternatives some different classes; other rows do not notice."""
    rng = np.random.default_rng(C)
    x = rng.standard_normal((6, C)).astype(np.float32)
    x[1, 3], x[2, C - 1], x[3], x[4, 0], x[4, 1] = np.inf, np.nan, np.nan, -np.inf, np.nan
    k = min(C, 8)
    labels = np.full(6, 2, np.int32)
    t, y, out = run(hgnn, dev, x, labels, k, C)
    bad = np.array([0, 1, 1, 1, 1, 0], bool)
    for name in ("logprob", "stats", "entropy", "top_logprob"):
        v = down(out[name]).reshape(6, -1)
        assert np.all(np.isnan(v[bad])) and np.all(np.isfinite(v[~bad])), name
    c = down(out["top_class"])
    assert np.all((c >= 0) & (c < C)) and all(len(set(row)) == k for row in c) and np.array_equal(c[~bad], alternatives(x[~bad], k))
    dx = torch.empty_like(t)
    hgnn.hgnn_logprob_grad(t, y, out["stats"], torch.ones(6, device=dev), dx)
    assert np.all(np.isnan(down(dx)[bad])) and np.all(np.isfinite(down(dx)[~bad]))


def test_parts_alone(hgnn, dev):
    """Every output by itself, without labels, without anything."""
    rng = np.random.default_rng(0)
    for C in (41, 5001):
        x = up((rng.standard_normal((30, C))).astype(np.float16), dev)
        y = up(rng.integers(0, C, 30).astype(np.int32), dev)
        ws = torch.empty(max(hgnn.hgnn_logprob_workspace(30, C, 3), 16), dtype=torch.uint8, device=dev)
        make = lambda *s: torch.full(s, FILL, device=dev)  # noqa: E731
        lp, st, en, tv, tc = make(30), make(30, 2), make(30), make(30, 3), torch.zeros((30, 3), dtype=torch.int32, device=dev)
        hgnn.hgnn_logprob(x, y, lp, stats=st, entropy=en, top_logprob=tv, top_class=tc, workspace=ws)
        a, b, c, d = make(30), make(30, 2), make(30), (make(30, 3), torch.zeros((30, 3), dtype=torch.int32, device=dev))
        hgnn.hgnn_logprob(x, y, a, workspace=ws)
        hgnn.hgnn_logprob(x, None, None, stats=b, workspace=ws)
        hgnn.hgnn_logprob(x, None, None, entropy=c, workspace=ws)
        hgnn.hgnn_logprob(x, None, None, top_logprob=d[0], top_class=d[1], workspace=ws)
        assert torch.equal(a, lp) and torch.equal(b, st) and torch.equal(c, en) and torch.equal(d[0], tv) and torch.equal(d[1], tc)
        # the entropy's gradient alone: labels are not needed
        dx, dz = torch.empty_like(x), torch.empty_like(x)
        h = torch.ones(30, device=dev)
        hgnn.hgnn_logprob_grad(x, None, st, None, dx, entropy=en, dentropy=h)
        hgnn.hgnn_logprob_grad(x, torch.full_like(y, -1), st, h, dz, entropy=en, dentropy=h)
        assert torch.equal(dx, dz)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("C", [6, 300, 5000])
def test_gradient_of_masked_rows(hgnn, dev, C, dtype):
    """A row of -inf alone has no gradient, whatever comes from above; a masked label has its row's."""
    x = np.full((4, C), -np.inf, NP[dtype])
    x[1, :3] = 1.0  # and the label 4 is masked
    x[3] = 0.5
    labels = np.array([1, 4, 0, -1], np.int32)
    t, y, out = run(hgnn, dev, x, labels, 0, C)
    g = np.array([np.nan, 2.0, np.inf, np.nan], np.float32)  # the last row has no label
    h = np.array([np.nan, 0.0, -np.inf, 0.0], np.float32)
    dx = torch.full_like(t, FILL)
    hgnn.hgnn_logprob_grad(t, y, out["stats"], up(g, dev), dx, entropy=out["entropy"], dentropy=up(h, dev))
    got = down(dx).astype(np.float64)
    assert np.all(got[[0, 2, 3]] == 0)
    want = np.zeros(C)
    want[:3], want[4] = -2 / 3, 2.0
    assert np.all(np.abs(got[1] - want) <= np.abs(want) * (2.0 ** -11 if dtype == torch.float16 else 16 * U))


def test_gradient_by_differences(hgnn, dev):
    """Of the values themselves: central differences of log probability and entropy in 64 bits of the host against the gradient of the call."""
    rng = np.random.default_rng(4)
    for C in (13, 777):
        x = rng.standard_normal((4, C)).astype(np.float32)
        labels = np.array([0, C - 1, -1, C // 2], np.int32)
        t, y, out = run(hgnn, dev, x, labels, 0, C)
        g, h = np.array([1, -2, 3, 0.5], np.float32), np.array([0.5, 0, -1, 2], np.float32)
        dx = torch.empty_like(t)
        hgnn.hgnn_logprob_grad(t, y, out["stats"], up(g, dev), dx, entropy=out["entropy"], dentropy=up(h, dev))
        got = down(dx)

        def value(z):
            r = reference(z)
            lp = np.array([r["lp"][i, labels[i]] if labels[i] >= 0 else 0 for i in range(4)])
            return g.astype(np.float64) * lp + h.astype(np.float64) * r["H"]
        step = 1e-4  # its square times the third derivative (below 3 here, weights up to 3) is the error of a central difference, 1e-16 / 1e-4 its rounding
        for c in rng.choice(C, 10, replace=False).tolist() + [0, C - 1, C // 2]:
            a, b = x.astype(np.float64), x.astype(np.float64)
            a[:, c] += step
            b[:, c] -= step
            diff = (value(a) - value(b)) / (2 * step)
            assert np.all(np.abs(got[:, c] - diff) <= 1e-7 + 64 * U * np.maximum(np.abs(diff), 4)), (C, c)


def test_far_rows(hgnn, dev):
    """Rows beyond 2^31 elements, read and written."""
    n, C = 2 ** 31 // 50000 + 40, 50000
    x = torch.zeros((n, C), dtype=torch.float16, device=dev)
    x[-1, 7] = 4.0
    y = torch.full((n,), 7, dtype=torch.int32, device=dev)
    lp, st = torch.empty(n, device=dev), torch.empty((n, 2), device=dev)
    need = hgnn.hgnn_logprob_workspace(n, C, 0)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    hgnn.hgnn_logprob(x, y, lp, stats=st, workspace=ws)
    hgnn.hgnn_logprob_grad(x, y, st, torch.ones(n, device=dev), x)
    got = down(lp)
    last = 4 - np.log(C - 1 + np.exp(4.0))
    assert abs(got[-1] - last) <= 500 * U * 12 and np.all(np.abs(got[:-1] + np.log(C)) <= 500 * U * 12)
    row = down(x[-1]).astype(np.float64)
    p = np.exp(last)
    assert abs(row[7] - (1 - p)) <= 2.0 ** -10 and np.all(np.abs(np.delete(row, 7) + np.exp(-np.log(C - 1 + np.exp(4.0)))) <= 2.0 ** -24)
