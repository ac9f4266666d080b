"""The forms that the log probabilities take by the numbers of rows and classes, each over several turns and with a partial last one, against the definitions in
64 bits, which the device evaluates here (rows are many).

Tolerances as in test_gpu_logprob.py, with the longest sum that a lane makes: a wave by itself adds C / 64 classes a lane, so D = C / 64 + 8 (and some 16 joins).
Powers of two below 2^-126, the least normal number, are zero to the hardware.  Of a class that far below the maximum the gradient, p times g and h (log p + H),
p = 2^-126 exp(-L) at most, is lost: no more than 2^-126 (|g| + |h| (|log p| + H)).  (Rows of more than 5600 rising or falling scores reach that: 87 of 469.)"""
import math

import pytest
import torch

from parity import down

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FILL = 7.0
HALF, SINGLE = torch.float16, torch.float32
CHUNK = 1 << 24  # elements that are looked at together


def placed(n, C, pitch, offset, dtype, dev):
    buf = torch.full((n * pitch + offset + 1,), FILL, dtype=dtype, device=dev)
    return torch.as_strided(buf, (n, C), (pitch, 1), offset), buf


def inputs(n, C, pitch, offset, dtype, dev):
    """Normal scores; rows that the mask leaves empty, or one or a few classes of, whose scores are equal, in part equal, rising, falling, the type's lowest value."""
    x, buf = placed(n, C, pitch, offset, dtype, dev)
    gen = torch.Generator(device=dev).manual_seed(n + C)
    for r in range(0, n, max(CHUNK // C, 1)):
        part = x[r:r + max(CHUNK // C, 1)]
        part.copy_(torch.randn(part.shape, generator=gen, device=dev) * 2)
    r = torch.arange(n, device=dev)
    x[r % 16 == 1] = x[r % 16 == 1].round()
    some = x[r % 16 == 2]
    x[r % 16 == 2] = some.masked_fill_(torch.rand(some.shape, generator=gen, device=dev) < 0.7, -math.inf)
    most = x[r % 64 == 3]
    x[r % 64 == 3] = most.masked_fill_(torch.rand(most.shape, generator=gen, device=dev) < 1 - 6 / C, -math.inf)
    x[5], x[n - 3] = -math.inf, 1.5
    x[6] = -math.inf
    x[6, C - 1] = 3.0
    x[7] = torch.arange(C, device=dev).to(dtype) / 64
    x[8] = -torch.arange(C, device=dev).to(dtype) / 64
    x[9] = torch.finfo(dtype).min
    x[n - 1] = torch.where(torch.rand(C, generator=gen, device=dev) < 0.5, -0.0, 0.0).to(dtype)
    labels = torch.randint(0, C, (n,), generator=gen, device=dev, dtype=torch.int32)
    labels[torch.rand(n, generator=gen, device=dev) < 0.2] = -1
    labels[:3] = torch.tensor([C, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device=dev)
    return x, buf, labels, gen


class Exact:
    """Of some rows, in 64 bits, with what the tolerances need."""

    def __init__(self, x):
        x = x.double()
        C = x.shape[1]
        self.m = x.amax(1)
        self.empty = torch.isneginf(self.m)
        self.d = x - torch.where(self.empty, 0.0, self.m)[:, None]
        S = self.d.exp().sum(1)
        self.L = torch.where(self.empty, 0.0, S.log())
        self.lp = self.d - self.L[:, None]
        self.p = torch.where(self.empty[:, None], 0.0, self.lp.exp())
        there = self.p > 0
        far = torch.where(there, self.d.abs(), 0.0)
        first, second = (self.p * far).sum(1), (self.p * far * far).sum(1)
        self.H = torch.where(self.empty, 0.0, self.L + first)
        D = -(-C // 64) + 8
        self.dL = (2 * D + 34 + 3 * first) * U + 2 * U * self.L.abs()
        self.dH = self.dL + (3 * second + (39 + 2 * D) * first) * U + 2 * U * (self.L.abs() + first)
        finite = lambda a: torch.where(torch.isfinite(a), a.abs(), 0.0)  # noqa: E731
        self.tol = self.dL[:, None] + 2 * U * (finite(self.d) + finite(self.lp))


def near(what, got, ref, tol):
    fine = torch.isfinite(ref)
    got = got.double()
    assert torch.equal(got[~fine], ref[~fine]), what
    over = (got[fine] - ref[fine]).abs() - tol[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (what, float(over.max()))


def forward(hgnn, dev, x, labels, k):
    n, C = x.shape
    need = hgnn.hgnn_logprob_workspace(n, C, k)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=dev) if need else None
    make = lambda *s: torch.full(s, FILL, device=dev)  # noqa: E731
    out = dict(logprob=make(n), stats=make(n, 2), entropy=make(n))
    if k:
        out.update(top_logprob=make(n, k), top_class=torch.full((n, k), -5, dtype=torch.int32, device=dev))
    hgnn.hgnn_logprob(x, labels, workspace=ws, **out)
    plain = {name: torch.full_like(t, 3) for name, t in out.items() if name != "entropy"}  # without the entropy: another form
    hgnn.hgnn_logprob(x, labels, workspace=ws, **plain)
    return out, plain


def check_forward(out, labels, x, k, step):
    n, C = x.shape
    for r in range(0, n, step):
        e = Exact(x[r:r + step])
        y = labels[r:r + step].long()
        real = (y >= 0) & (y < C)
        at = torch.where(real, y, 0)[:, None]
        near("logprob", out["logprob"][r:r + step], torch.where(real, e.lp.gather(1, at)[:, 0], 0.0), torch.where(real, e.tol.gather(1, at)[:, 0], 0.0))
        stats = out["stats"][r:r + step].double()
        assert torch.equal(stats[:, 0], e.m)
        near("stats", stats[:, 1], e.L, e.dL)
        if "entropy" in out:
            near("entropy", out["entropy"][r:r + step], e.H, e.dH)
        if k:
            best = torch.sort(x[r:r + step].double() + 0.0, dim=1, descending=True, stable=True).indices[:, :k]
            assert torch.equal(out["top_class"][r:r + step].long(), best)
            near("top_logprob", out["top_logprob"][r:r + step], e.lp.gather(1, best), e.tol.gather(1, best))


def check_grad(hgnn, dev, x, labels, out, gen, pitch, offset, with_entropy, step):
    n, C = x.shape
    g = torch.randn(n, generator=gen, device=dev)
    h = torch.randn(n, generator=gen, device=dev) if with_entropy else torch.zeros(n, device=dev)
    dx, buf = placed(n, C, pitch, offset, x.dtype, dev)
    more = dict(entropy=out["entropy"], dentropy=h) if with_entropy else {}
    hgnn.hgnn_logprob_grad(x, labels, out["stats"], g, dx, **more)
    for r in range(0, n, step):
        e = Exact(x[r:r + step])
        y = labels[r:r + step].long()
        real = (y >= 0) & (y < C) & ~e.empty
        g64, h64 = torch.where(real, g[r:r + step], 0.0).double()[:, None], h[r:r + step].double()[:, None]
        hot = torch.zeros_like(e.p).scatter_(1, torch.where(real, y, 0)[:, None], real.double()[:, None])
        there = e.p > 0
        lp = torch.where(there, e.lp, 0.0)
        ref = g64 * (hot - e.p) - h64 * e.p * torch.where(there, lp + e.H[:, None], 0.0)
        size = lp.abs() + e.H[:, None]
        rel = e.tol + (3 * lp.abs() + 4) * U
        tol = g64.abs() * (e.p * rel + U * (hot + e.p)) + h64.abs() * e.p * (size * (rel + 4 * U) + e.tol + e.dH[:, None]) + 4 * U * ref.abs()
        tol += 2.0 ** -126 * (1 + g64.abs() + h64.abs() * size)
        if x.dtype == HALF:
            tol = tol * (1 + 2.0 ** -11) + ref.abs() * 2.0 ** -11 + 2.0 ** -25
        near("dlogits", dx[r:r + step], ref, tol)
    again = torch.empty((n, C), dtype=x.dtype, device=dev).copy_(x)
    hgnn.hgnn_logprob_grad(again, labels, out["stats"], g, again, **more)  # in its own place
    assert torch.equal(again, dx)
    dx.fill_(FILL)
    assert bool((buf == FILL).all()), "something beside the rows was written"


FORMS = [  # n, C, pitch, offset, k: a wave to a row with alternatives, of one turn and of several, whose last is a single class or nearly a whole one
    (4099, 1021, 1023, 1, 5), (4096, 513, 513, 0, 1), (4097, 3001, 3003, 3, 8), (4096, 4096, 4096, 0, 32), (5000, 2049, 2050, 1, 20), (4200, 4095, 4097, 0, 2),
    # and without
    (4100, 2500, 2503, 1, 0), (4100, 4096, 4096, 0, 0), (4096, 2049, 2049, 3, 0),
    # lanes of a group with two and four pieces each
    (70, 777, 779, 1, 0), (33, 1024, 1024, 0, 0), (40, 1500, 1501, 1, 0), (40, 2048, 2048, 0, 0), (33, 1025, 1025, 0, 0),
    (33000, 511, 513, 1, 0), (40001, 257, 257, 0, 0), (140001, 57, 59, 3, 0), (262145, 31, 32, 0, 0), (70001, 200, 201, 1, 0),
    # workgroups to a row: a wave or two with classes, a last part that is short
    (3000, 1500, 1501, 1, 5), (700, 2500, 2501, 0, 9), (20, 30011, 30013, 1, 32), (1025, 4097, 4097, 0, 7),
    # very many short rows
    (17000003, 3, 3, 1, 2), (9000001, 9, 11, 0, 2), (9000001, 10, 10, 0, 7),
]


@pytest.mark.parametrize("dtype", [HALF, SINGLE])
@pytest.mark.parametrize("n,C,pitch,offset,k", FORMS)
def test_forms(hgnn, dev, n, C, pitch, offset, k, dtype):
    print(f"logprob n={n} C={C} pitch={pitch} k={k} {dtype}", flush=True)
    x, buf, labels, gen = inputs(n, C, pitch, offset, dtype, dev)
    step = max(CHUNK // C, 1)
    out, plain = forward(hgnn, dev, x, labels, k)
    check_forward(out, labels, x, k, step)
    check_forward(plain, labels, x, k, step)
    for with_entropy in (False, True):
        check_grad(hgnn, dev, x, labels, out, gen, pitch, offset, with_entropy, step)


@pytest.mark.parametrize("n,C,pitch,offset,dtype", [(130003, 777, 777, 1, HALF), (2100, 50021, 50023, 1, HALF), (1100, 50021, 50021, 0, SINGLE), (90001, 570, 571, 3, SINGLE)])
def test_gradients_past_the_caches(hgnn, dev, n, C, pitch, offset, dtype):
    """192 MB and more of them."""
    print(f"logprob gradient n={n} C={C} pitch={pitch} {dtype}", flush=True)
    assert n * C * (2 if dtype == HALF else 4) >= 192 << 20
    x, buf, labels, gen = inputs(n, C, pitch, offset, dtype, dev)
    out, _ = forward(hgnn, dev, x, labels, 0)
    for with_entropy in (False, True):
        check_grad(hgnn, dev, x, labels, out, gen, pitch, offset, with_entropy, max(CHUNK // C, 1))


@pytest.mark.parametrize("dtype", [HALF, SINGLE])
@pytest.mark.parametrize("n,C,k", [(4099, 1021, 5), (4097, 3001, 8), (4100, 2500, 0), (40, 1500, 0), (33000, 300, 0), (700, 2500, 9)])
def test_forms_without_numbers(hgnn, dev, n, C, k, dtype):
    """Rows with NaN or +inf are NaN everywhere, their alternatives some different classes; their neighbours do not notice."""
    x, buf, labels, gen = inputs(n, C, C, 0, dtype, dev)
    before, _ = forward(hgnn, dev, x, labels, k)
    x[11, C // 2], x[12, C - 1], x[13, 0], x[20] = math.nan, math.nan, math.inf, math.nan
    bad = torch.zeros(n, dtype=torch.bool, device=dev)
    bad[[11, 12, 13, 20]] = True
    labels[bad] = 1
    out, _ = forward(hgnn, dev, x, labels, k)
    for name, t in out.items():
        assert torch.equal(t[~bad], before[name][~bad]), name
        if name != "top_class":
            assert bool(torch.isnan(t[bad]).all()), name
        else:
            c = down(t[bad])
            assert c.min() >= 0 and c.max() < C and all(len(set(row)) == k for row in c.tolist())
    dx = torch.zeros_like(x)
    hgnn.hgnn_logprob_grad(x, labels, out["stats"], torch.ones(n, device=dev), dx, entropy=out["entropy"], dentropy=torch.ones(n, device=dev))
    assert bool(torch.isnan(dx[bad]).all()) and bool(torch.isfinite(dx[~bad]).all())
