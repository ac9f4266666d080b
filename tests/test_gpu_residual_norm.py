"""The norms around a block with its gate and residual, and their gradients, against 64 bits on the host.

Tolerances, u = 2^-24.  A sum over a row is eight elements of a lane in order and then at most ten levels of lanes and sixteen waves: 40 u of the sum of the
absolute values.  With xa = r (|x| + mean |x|), which is what xh = r (x - mean) is formed from, xh is off by 64 u xa (the mean, the difference, the variance and
its root), and N^T(d) = r (v - xh mean(v xh) - mean(v)), v = d w, by 128 u r (|v| + xa mean(|v| xa) + mean |v|).  Sums over rows go through chains of at most 256 in
a workgroup, 80 over the workgroups and as many rows as a lane takes, 512 u of the sum of the absolute values in all.  A store in fp16 adds 2^-11 of the value, or
2^-25.  Z is held against the norm of H as the call stored it."""
import numpy as np
import pytest
import torch

from parity import down

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5
FILL = 7.0
F16, F32 = np.float16, np.float32
NONE, RMS, LAYER = 0, 1, 2


def place(a, dev, pitch=None, offset=0, fill=FILL):
    """A device copy in a buffer of that pitch, `offset` elements in -> (view, buffer)"""
    t = torch.from_numpy(np.ascontiguousarray(a))
    n, F = t.shape
    pitch = F if pitch is None else pitch
    buf = torch.full((max(n - 1, 0) * pitch + (F if n else 0) + offset + 1,), fill, dtype=t.dtype, device=dev)
    v = torch.as_strided(buf, (n, F), (pitch, 1), offset)
    v.copy_(t)
    return v, buf


def untouched(view, buf):
    """Nothing beside the view has been written."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(mask, view.shape, view.stride(), view.storage_offset()).fill_(False)
    assert bool((buf[mask] == FILL).all()), "something beside the tensor was written"


def moments(x, kind):
    mean = x.mean(1, keepdims=True) if kind == LAYER else np.zeros((x.shape[0], 1))
    r = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + EPS)
    return (x - mean) * r, r, r * (np.abs(x) + (np.abs(x).mean(1, keepdims=True) if kind == LAYER else 0))


def back(d, w, xh, r, xa, kind):
    v = d * w
    out = r * (v - xh * (v * xh).mean(1, keepdims=True) - (v.mean(1, keepdims=True) if kind == LAYER else 0))
    mag = r * (np.abs(v) + xa * (np.abs(v) * xa).mean(1, keepdims=True) + (np.abs(v).mean(1, keepdims=True) if kind == LAYER else 0))
    return out, mag


def near(name, got, ref, tol):
    got = got.astype(np.float64)
    bad = ~(np.abs(got - ref) <= tol + (np.abs(ref) * 2.0 ** -11 + 2.0 ** -25 if name in HALVES else 2.0 ** -149 + U * np.abs(ref)))
    assert not bad.any(), (name, int(bad.sum()), got[bad][:3], np.broadcast_to(ref, got.shape)[bad][:3], np.broadcast_to(tol, got.shape)[bad][:3])


HALVES = set()


class Case:
    def __init__(self, n, F, stream=F16, post=LAYER, pre=LAYER, gate="feature", bias=True, alpha=0.7, weights=True, seed=0, mean=0.3, branch=True, residual=True):
        rng = np.random.default_rng(seed + 1000 * F + n)
        f = lambda *s: rng.standard_normal(s)  # noqa: E731
        self.n, self.F, self.stream, self.post, self.pre, self.gate_kind, self.alpha = n, F, stream, post, pre, gate, alpha
        self.R = (f(n, F) + mean).astype(stream) if residual else None
        self.Y = (f(n, F) * 0.8 + mean).astype(F16) if branch else None
        vec = lambda there, c: (c + 0.2 * f(F)).astype(F32) if there else None  # noqa: E731
        self.post_w, self.post_b = vec(post and weights, 1), vec(post and bias, 0)
        self.pre_w, self.pre_b = vec(pre and weights, 1), vec(pre and bias, 0)
        self.gate = {"none": None, "feature": vec(True, 0.5), "rows": (0.5 * f(n, F)).astype(F16)}[gate]
        self.H = (f(n, F) * 1.7 + mean).astype(stream)
        self.dH, self.dZ = f(n, F).astype(stream), f(n, F).astype(F16) if pre else None

    def kwargs(self, dev, pitch=None, offset=0):
        t = lambda a: None if a is None else torch.from_numpy(a).to(dev)  # noqa: E731
        gate = place(self.gate, dev, pitch, offset)[0] if self.gate_kind == "rows" else t(self.gate)
        return dict(post=self.post, post_w=t(self.post_w), post_b=t(self.post_b), gate=gate, alpha=self.alpha, pre=self.pre, pre_w=t(self.pre_w), pre_b=t(self.pre_b), eps=EPS)

    def wide(self):
        d = lambda a, c: c if a is None else a.astype(np.float64)  # noqa: E731
        return d(self.post_w, 1.0), d(self.post_b, 0.0), d(self.gate, 1.0), d(self.pre_w, 1.0), d(self.pre_b, 0.0)


def forward(hgnn, dev, c, pitch=None, offset=0, in_place=False):
    print(f"norm n={c.n} F={c.F} {c.stream.__name__} post={c.post} pre={c.pre} gate={c.gate_kind} pitch={pitch} offset={offset}", flush=True)
    HALVES.clear()
    HALVES.update({"Z"} | ({"H"} if c.stream == F16 else set()))
    R, Rb = place(c.R, dev, pitch, offset) if c.R is not None else (None, None)
    Y, Yb = place(c.Y, dev, pitch, offset) if c.Y is not None else (None, None)
    H, Hb = (R, Rb) if in_place else place(np.full((c.n, c.F), 3, c.stream), dev, pitch, offset)
    Z, Zb = place(np.full((c.n, c.F), 3, F16), dev, pitch, offset) if c.pre else (None, None)
    hgnn.hgnn_residual_norm(R, Y, H, Z, **c.kwargs(dev, pitch, offset))
    pw, pb, g, qw, qb = c.wide()
    h, mag = 0.0, 0.0
    if c.Y is not None:
        y = c.Y.astype(np.float64)
        xh, r, xa = moments(y, c.post) if c.post else (y, 1.0, np.abs(y))
        b = xh * pw + pb
        h, mag = g * b, np.abs(g) * (xa * np.abs(pw) + np.abs(pb))
    if c.R is not None:
        h, mag = h + c.alpha * c.R.astype(np.float64), mag + np.abs(c.alpha * c.R.astype(np.float64))
    got = down(H)
    near("H", got, h, 64 * U * mag)
    untouched(H, Hb)
    if c.pre:
        xh, r, xa = moments(got.astype(np.float64), c.pre)
        near("Z", down(Z), xh * qw + qb, 64 * U * (xa * np.abs(qw) + np.abs(qb)))
        untouched(Z, Zb)
    if Yb is not None:
        untouched(Y, Yb)
    return H, Z


def backward(hgnn, dev, c, pitch=None, offset=0, in_place=False, only=None, dH=True):
    print(f"norm grad n={c.n} F={c.F} {c.stream.__name__} post={c.post} pre={c.pre} gate={c.gate_kind} pitch={pitch} offset={offset} only={only}", flush=True)
    HALVES.clear()
    HALVES.update({"dY"} | ({"dR"} if c.stream == F16 else set()) | ({"dgate"} if c.gate_kind == "rows" else set()))
    H, Y = place(c.H, dev, pitch, offset)[0], place(c.Y, dev, pitch, offset)[0]
    gH, gHb = place(c.dH, dev, pitch, offset) if dH else (None, None)
    gZ = place(c.dZ, dev, pitch, offset)[0] if c.pre else None
    wanted = lambda name, there=True: there and (only is None or name in only)  # noqa: E731
    out = lambda name, dtype, there=True: place(np.full((c.n, c.F), 3, dtype), dev, pitch, offset) if wanted(name, there) else (None, None)  # noqa: E731
    dR, dRb = (gH, gHb) if in_place else out("dR", c.stream)
    dY, dYb = out("dY", F16)
    vec = lambda name, there: torch.full((c.F,), FILL, device=dev) if wanted(name, there) else None  # noqa: E731
    dgate, dgb = out("dgate", F16) if c.gate_kind == "rows" else (vec("dgate", c.gate_kind == "feature"), None)
    dpw, dpb, dqw, dqb = vec("dpost_w", c.post), vec("dpost_b", c.post), vec("dpre_w", c.pre), vec("dpre_b", c.pre)
    ws = torch.full((max(hgnn.hgnn_residual_norm_grad_workspace(c.n, c.F), 16),), 255, dtype=torch.uint8, device=dev)
    hgnn.hgnn_residual_norm_grad(H, Y, gH, gZ, dR, dY, ws, dgate=dgate, dpost_w=dpw, dpost_b=dpb, dpre_w=dqw, dpre_b=dqb, **c.kwargs(dev, pitch, offset))
    pw, pb, g, qw, qb = c.wide()
    e = c.dH.astype(np.float64) if dH else np.zeros((c.n, c.F))
    mag = np.abs(e)
    if c.pre:
        xh, r, xa = moments(c.H.astype(np.float64), c.pre)
        dz = c.dZ.astype(np.float64)
        through, m = back(dz, qw, xh, r, xa, c.pre)
        e, mag = e + through, mag + m
        if dqw is not None:
            near("dpre_w", down(dqw), (dz * xh).sum(0), 512 * U * (np.abs(dz) * xa).sum(0))
        if dqb is not None:
            near("dpre_b", down(dqb), dz.sum(0), 512 * U * np.abs(dz).sum(0))
    if dR is not None:
        near("dR", down(dR), c.alpha * e, 128 * U * abs(c.alpha) * mag)
        untouched(dR, dRb)
    y = c.Y.astype(np.float64)
    xh, r, xa = moments(y, c.post) if c.post else (y, 1.0, np.abs(y))
    b, bmag = xh * pw + pb, xa * np.abs(pw) + np.abs(pb)
    if dgate is not None:
        if c.gate_kind == "rows":
            near("dgate", down(dgate), e * b, 192 * U * mag * bmag)
            untouched(dgate, dgb)
        else:
            near("dgate", down(dgate), (e * b).sum(0), 640 * U * (mag * bmag).sum(0))
    db, dmag = e * g, mag * np.abs(g)
    if dpw is not None:
        near("dpost_w", down(dpw), (db * xh).sum(0), 640 * U * (dmag * xa).sum(0))
    if dpb is not None:
        near("dpost_b", down(dpb), db.sum(0), 640 * U * dmag.sum(0))
    if dY is not None:
        ref, m = back(db, pw, xh, r, xa, c.post) if c.post else (db, dmag)
        if c.post:  # what is off in e goes through, too
            m = m + back(dmag, np.abs(pw), xa, r, xa, NONE)[1]
        near("dY", down(dY), ref, 256 * U * m)
        untouched(dY, dYb)


SHAPES = [(1, 1), (5, 1), (2, 2), (3, 7), (1, 8), (300, 8), (77, 9), (1000, 16), (63, 24), (130, 33), (64, 42), (257, 64), (33, 100), (129, 128), (65, 129), (9, 255), (40, 256), (10, 257), (70, 333),
          (17, 512), (6, 513), (19, 608), (3, 1024), (21, 1025), (4, 2048), (5, 2049), (11, 3000), (2, 4096), (9, 4097), (1, 8191), (3, 8192)]


@pytest.mark.parametrize("n,F", SHAPES)
@pytest.mark.parametrize("stream", [F16, F32])
def test_widths(hgnn, dev, n, F, stream):
    c = Case(n, F, stream)
    forward(hgnn, dev, c)
    backward(hgnn, dev, c)
    c = Case(n, F, stream, post=RMS, pre=RMS, gate="rows", bias=False)
    forward(hgnn, dev, c, pitch=F + 3, offset=1)
    backward(hgnn, dev, c, pitch=F + 3, offset=1)


@pytest.mark.parametrize("post", [NONE, RMS, LAYER])
@pytest.mark.parametrize("pre", [NONE, RMS, LAYER])
@pytest.mark.parametrize("gate", ["none", "feature", "rows"])
def test_parts(hgnn, dev, post, pre, gate):
    """Every combination of norms and gates, with and without weights, in place and not."""
    for F, n in ((40, 37), (700, 5)):
        for weights, bias in ((True, True), (False, True), (True, False), (False, False)):
            c = Case(n, F, F16, post, pre, gate, bias, 1.0, weights)
            forward(hgnn, dev, c, pitch=F + 8)
            backward(hgnn, dev, c, pitch=F + 8)
        c = Case(n, F, F32, post, pre, gate)
        forward(hgnn, dev, c, in_place=True)
        backward(hgnn, dev, c, in_place=True)


def test_what_may_be_missing(hgnn, dev):
    """No branch, no residual, no H, no gradient of H, one output alone."""
    c = Case(50, 72, F16, NONE, RMS, "none", branch=False, alpha=1.0)
    forward(hgnn, dev, c)
    R = place(c.R, dev)[0]
    Z, Zb = place(np.full((50, 72), 3, F16), dev)
    hgnn.hgnn_residual_norm(R, None, None, Z, pre=RMS, pre_w=torch.from_numpy(c.pre_w).to(dev), pre_b=torch.from_numpy(c.pre_b).to(dev), eps=EPS)
    _, want = forward(hgnn, dev, c)
    assert torch.equal(Z, want)
    forward(hgnn, dev, Case(50, 72, F32, LAYER, LAYER, "feature", residual=False))
    c = Case(211, 72, F16)
    backward(hgnn, dev, c, dH=False)
    for name in ("dR", "dY", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b"):
        backward(hgnn, dev, c, only={name})
    # without sums over rows no workspace is asked for
    dR = torch.empty(211, 72, dtype=torch.float16, device=dev)
    hgnn.hgnn_residual_norm_grad(None, None, place(c.dH, dev)[0], None, dR, None, None, alpha=0.5)
    assert np.array_equal(down(dR), (c.dH.astype(F32) * F32(0.5)).astype(F16))


def test_no_rows(hgnn, dev):
    """Sums over no rows are zeros; nothing else is written."""
    e = torch.empty(0, 24, dtype=torch.float16, device=dev)
    hgnn.hgnn_residual_norm(e, e, e, e, pre=RMS)
    v = [torch.full((24,), FILL, device=dev) for _ in range(5)]
    ws = torch.empty(16, dtype=torch.uint8, device=dev)
    hgnn.hgnn_residual_norm_grad(e, e, e, e, e, e, ws, post=LAYER, post_w=v[0].clone(), post_b=v[0].clone(), gate=v[0].clone(), pre=LAYER, dgate=v[0], dpost_w=v[1], dpost_b=v[2],
                                 dpre_w=v[3], dpre_b=v[4])
    assert all(bool((x == 0).all()) for x in v)


def test_rows_of_zeros_and_what_is_not_finite(hgnn, dev):
    """A row of zeros has a norm of zeros; a row with NaN or infinity spoils itself alone, and what stands between rows reaches nothing."""
    n, F = 40, 42
    c = Case(n, F, F16, RMS, LAYER, "none", bias=False)
    c.Y[3], c.R[3] = 0, 0
    c.Y[5, 7], c.R[9, 0], c.Y[11, 41] = np.nan, np.inf, -np.inf
    wide = torch.full((n, 48), float("nan"), dtype=torch.float16, device=dev)
    R, Y = wide.clone()[:, :F], wide.clone()[:, :F]
    R.copy_(torch.from_numpy(c.R)), Y.copy_(torch.from_numpy(c.Y))
    H, Z = torch.zeros(n, 48, dtype=torch.float16, device=dev)[:, :F], torch.zeros(n, 48, dtype=torch.float16, device=dev)[:, :F]
    hgnn.hgnn_residual_norm(R, Y, H, Z, **c.kwargs(dev))
    clean = Case(n, F, F16, RMS, LAYER, "none", bias=False)
    clean.Y[3], clean.R[3] = 0, 0
    H2, Z2 = forward(hgnn, dev, clean)
    bad = torch.zeros(n, dtype=torch.bool, device=dev)
    bad[[5, 9, 11]] = True
    assert torch.equal(H[~bad], H2[~bad]) and torch.equal(Z[~bad], Z2[~bad])
    assert bool(Z[bad].isnan().all()) and bool((Z[3] == 0).all())


def test_gradients_against_differences(hgnn, dev):
    """The loss sum(cH H) + sum(cZ Z) in fp32 streams, differences of the formula in 64 bits on the host against the gradients of the call."""
    c = Case(6, 20, F32, LAYER, RMS, "feature", mean=0.1)
    # what the gradients start from is the stored H: take the forward's own
    y, pw, pb, g, qw, qb = c.Y.astype(np.float64), *c.wide()
    R = c.R.astype(np.float64)

    def h_of(R, y, pw, pb, g):
        return c.alpha * R + g * (moments(y, c.post)[0] * pw + pb)

    def loss(R, y, pw, pb, g, qw, qb):
        h = h_of(R, y, pw, pb, g)
        return (c.dH.astype(np.float64) * h).sum() + (c.dZ.astype(np.float64) * (moments(h, c.pre)[0] * qw + qb)).sum()
    c.H = h_of(R, y, pw, pb, g).astype(F32)
    backward(hgnn, dev, c)
    H, Y, dH, dZ = (place(a, dev)[0] for a in (c.H, c.Y, c.dH, c.dZ))
    dR, dY = torch.empty_like(dH), torch.empty_like(Y)
    v = [torch.empty(20, device=dev) for _ in range(5)]
    ws = torch.empty(hgnn.hgnn_residual_norm_grad_workspace(6, 20), dtype=torch.uint8, device=dev)
    hgnn.hgnn_residual_norm_grad(H, Y, dH, dZ, dR, dY, ws, dgate=v[0], dpost_w=v[1], dpost_b=v[2], dpre_w=v[3], dpre_b=v[4], **c.kwargs(dev))
    got = {0: dR, 1: dY, 2: v[1], 3: v[2], 4: v[0], 5: v[3], 6: v[4]}
    at = [R, y, pw, pb, g, qw, qb]
    rng = np.random.default_rng(1)
    for k, t in got.items():
        for _ in range(4):
            i = tuple(rng.integers(0, s) for s in at[k].shape)
            step = 1e-4  # a central difference is off by step^2 / 6 of the third derivative (some hundreds at most here) and 2^-52 of the loss (~100) over the step
            up, lo = [a.copy() for a in at], [a.copy() for a in at]
            up[k][i] += step
            lo[k][i] -= step
            want = (loss(*up) - loss(*lo)) / (2 * step)
            assert abs(down(t)[i] - want) <= 1e-5 + abs(want) * (2.0 ** -10 if k == 1 else 1e-5), (k, i, down(t)[i], want)


def test_many_rows(hgnn, dev):
    """More rows than a launch has places: lanes take several in turn, in both shapes."""
    for n, F in ((70001, 64), (5001, 600)):
        c = Case(n, F, F16)
        forward(hgnn, dev, c)
        backward(hgnn, dev, c)


def test_by_both_routes_in_a_graph_and_on_a_stream(hgnn, dev):
    """Captured and replayed with other data, on another stream, through ctypes and through the native module: the same bits."""
    c = Case(300, 100, F32, LAYER, RMS, "rows")
    kw = c.kwargs(dev)
    t = {k: place(getattr(c, k), dev)[0] for k in ("R", "Y", "H", "dH", "dZ")}
    out = {k: torch.empty_like(t[s]) for k, s in (("H2", "R"), ("Z", "Y"), ("dR", "R"), ("dY", "Y"), ("dgate", "Y"))}
    v = [torch.empty(100, device=dev) for _ in range(4)]
    ws = torch.empty(hgnn.hgnn_residual_norm_grad_workspace(300, 100), dtype=torch.uint8, device=dev)

    def call(stream=None):
        hgnn.hgnn_residual_norm(t["R"], t["Y"], out["H2"], out["Z"], stream=stream, **kw)
        hgnn.hgnn_residual_norm_grad(out["H2"], t["Y"], t["dH"], t["dZ"], out["dR"], out["dY"], ws, dgate=out["dgate"], dpost_w=v[0], dpost_b=v[1], dpre_w=v[2], dpre_b=v[3], stream=stream, **kw)

    def taken():
        torch.cuda.synchronize()
        return [x.clone() for x in [*out.values(), *v]]
    call()
    first = taken()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for x in [*out.values(), *v]:
        x.zero_()
    torch.cuda.synchronize()
    call(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, taken()))
    native, hgnn.binding._calls = hgnn.binding._calls, None
    try:
        for x in [*out.values(), *v]:
            x.zero_()
        call()
        assert native is not None and all(torch.equal(a, b) for a, b in zip(first, taken()))
    finally:
        hgnn.binding._calls = native
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        t["Y"].mul_(1.25)
        t["dZ"].add_(0.5)
        graph.replay()
        replayed = taken()
        call()
        assert all(torch.equal(a, b) for a, b in zip(replayed, taken())), k


def test_refusals_of_the_binding(hgnn, dev):
    h, f = torch.zeros(4, 8, dtype=torch.float16, device=dev), torch.zeros(4, 8, device=dev)
    w = torch.ones(8, device=dev)
    for bad in (lambda: hgnn.hgnn_residual_norm(h, h, f, None), lambda: hgnn.hgnn_residual_norm(h, f, h, None), lambda: hgnn.hgnn_residual_norm(h, h, h, None, pre=RMS),
                lambda: hgnn.hgnn_residual_norm(h, h, h, h), lambda: hgnn.hgnn_residual_norm(None, None, None, None), lambda: hgnn.hgnn_residual_norm(h, h[:, :7], h, None),
                lambda: hgnn.hgnn_residual_norm(h, h, h, None, post=3), lambda: hgnn.hgnn_residual_norm(h, h, h, None, post_w=w),
                lambda: hgnn.hgnn_residual_norm(h, h, h, None, gate=w[:7]), lambda: hgnn.hgnn_residual_norm(h, h, h, None, gate=f), lambda: hgnn.hgnn_residual_norm(h, h, h, h, pre=RMS, eps=0.0),
                lambda: hgnn.hgnn_residual_norm(h, None, h, None, gate=w), lambda: hgnn.hgnn_residual_norm(h, h, h, None, alpha=float("nan")),
                lambda: hgnn.hgnn_residual_norm(h.t(), h.t(), h.t(), None),
                lambda: hgnn.hgnn_residual_norm_grad(h, h, h, h, h, h, None, dgate=w), lambda: hgnn.hgnn_residual_norm_grad(h, h, h, None, h, h, None, pre=RMS),
                lambda: hgnn.hgnn_residual_norm_grad(h, None, h, None, None, h, None, post=RMS), lambda: hgnn.hgnn_residual_norm_grad(h, h, h, h, h, h, w[:1], pre=RMS, dpre_w=w),
                lambda: hgnn.hgnn_residual_norm_grad(h, h, h, None, h, h, None, gate=w, dgate=h)):
        with pytest.raises((hgnn.HgnnError, TypeError, ValueError)):
            bad()
