"""Norms around a block where workgroups of several waves take several rows in turn, and gradients whose outputs go past the caches, against 64 bits.  The
tolerances are those that test_gpu_residual_norm.py derives; a lane takes at most 40 rows here."""
import numpy as np
import pytest
import torch

from test_gpu_residual_norm import EPS, F16, F32, LAYER, NONE, RMS, U, Case, backward, forward

pytestmark = pytest.mark.gpu


# more rows than workgroups of 4, 8 and 16 waves, the last ones with a row fewer
@pytest.mark.parametrize("n,F", [(3001, 2048), (1301, 1025), (2101, 4096), (1500, 2049), (1501, 4097), (1101, 8191), (600, 8192)])
@pytest.mark.parametrize("stream", [F16, F32])
def test_rows_in_turn(hgnn, dev, n, F, stream):
    c = Case(n, F, stream)
    forward(hgnn, dev, c)
    backward(hgnn, dev, c)
    c = Case(n, F, stream, RMS, RMS, "rows", bias=False)
    forward(hgnn, dev, c, pitch=F + 3, offset=1)
    backward(hgnn, dev, c, pitch=F + 3, offset=1)


@pytest.mark.parametrize("post,pre,gate", [(NONE, LAYER, "none"), (LAYER, NONE, "feature"), (RMS, LAYER, "feature")])
@pytest.mark.parametrize("F", [1800, 3333, 6000])
def test_parts_in_turn(hgnn, dev, post, pre, gate, F):
    c = Case(1400, F, F16, post, pre, gate)
    forward(hgnn, dev, c, in_place=True)
    backward(hgnn, dev, c, in_place=True)
    backward(hgnn, dev, c, dH=pre == NONE, only={"dR"})


def normed(x, kind):
    mean = x.mean(1, keepdim=True) if kind == LAYER else x.new_zeros(())
    r = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    return (x - mean) * r, r, r * (x.abs() + (x.abs().mean(1, keepdim=True) if kind == LAYER else 0))


def back(d, w, xh, r, xa, kind):
    v = d * w
    layer = 1 if kind == LAYER else 0
    out = r * (v - xh * (v * xh).mean(1, keepdim=True) - layer * v.mean(1, keepdim=True))
    return out, r * (v.abs() + xa * (v.abs() * xa).mean(1, keepdim=True) + layer * v.abs().mean(1, keepdim=True))


@pytest.mark.parametrize("stream,n,F", [(torch.float16, 395009, 128), (torch.float32, 270001, 128), (torch.float16, 25003, 2048), (torch.float32, 8301, 4096), (torch.float16, 400007, 127)])
def test_outputs_past_the_caches(hgnn, dev, stream, n, F):
    """dR and dY of more than 192 MiB in whole lines (but for the last, whose rows are none): every element, and the sums over all rows."""
    print("past the caches", stream, n, F, flush=True)
    gen = torch.Generator(device=dev).manual_seed(n + F)
    f = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    half = torch.float16
    H, dH, Y, dZ = (f(n, F) * 1.7 + 0.3).to(stream), f(n, F).to(stream), (f(n, F) * 0.8 + 0.3).to(half), f(n, F).to(half)
    pw, pb, gate, qw, qb = 1 + 0.2 * f(F), 0.2 * f(F), 0.5 + 0.2 * f(F), 1 + 0.2 * f(F), 0.2 * f(F)
    dR, dY = torch.full_like(H, 3), torch.full_like(Y, 3)
    assert n * F * (dR.element_size() + 2) > 192 << 20
    got = [torch.full((F,), 7.0, device=dev) for _ in range(5)]
    ws = torch.full((hgnn.hgnn_residual_norm_grad_workspace(n, F),), 255, dtype=torch.uint8, device=dev)
    alpha = 0.7
    hgnn.hgnn_residual_norm_grad(H, Y, dH, dZ, dR, dY, ws, post=LAYER, post_w=pw, post_b=pb, gate=gate, alpha=alpha, pre=RMS, pre_w=qw, pre_b=qb, eps=EPS, dgate=got[0], dpost_w=got[1],
                                 dpost_b=got[2], dpre_w=got[3], dpre_b=got[4])
    wpw, wpb, wg, wqw = (t.double() for t in (pw, pb, gate, qw))
    sums, mags = [torch.zeros(F, dtype=torch.float64, device=dev) for _ in range(5)], [torch.zeros(F, dtype=torch.float64, device=dev) for _ in range(5)]

    def add(k, v, m):
        sums[k] += v.sum(0)
        mags[k] += m.sum(0)
    step = (1 << 23) // F
    for i in range(0, n, step):
        at = slice(i, i + step)
        h, e, y, dz = (t[at].double() for t in (H, dH, Y, dZ))
        mag = e.abs()
        xh, r, xa = normed(h, RMS)
        t, m = back(dz, wqw, xh, r, xa, RMS)
        add(3, dz * xh, dz.abs() * xa)
        add(4, dz, dz.abs())
        e, mag = e + t, mag + m
        a = np.float64(F32(alpha))
        bad = (dR[at].double() - a * e).abs() > 128 * U * a * mag + (2.0 ** -11 * (a * e).abs() + 2.0 ** -25 if stream == half else U * (a * e).abs())
        assert not bool(bad.any()), ("dR", i, bad.nonzero()[:3])
        xh, r, xa = normed(y, LAYER)
        b, bmag = xh * wpw + wpb, xa * wpw.abs() + wpb.abs()
        add(0, e * b, mag * bmag)
        db, dmag = e * wg, mag * wg.abs()
        add(1, db * xh, dmag * xa)
        add(2, db, dmag)
        t, m = back(db, wpw, xh, r, xa, LAYER)
        m = m + back(dmag, wpw.abs(), xa, r, xa, NONE)[1]
        bad = (dY[at].double() - t).abs() > 256 * U * m + 2.0 ** -11 * t.abs() + 2.0 ** -25
        assert not bool(bad.any()), ("dY", i, bad.nonzero()[:3])
    for k, name in enumerate(("dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b")):
        off = (got[k].double() - sums[k]).abs() - U * sums[k].abs()
        assert bool((off <= 640 * U * mags[k]).all()), (name, float((off / mags[k]).max()) / U)
