"""Whole steps of a network of gated blocks as a program makes them with these calls: norms, gated projections, projections, their gradients, clipping and orthogonal
updates, against the same steps in 64 bits on the host; captured and replayed; and two of them at once on streams of their own."""
import numpy as np
import pytest
import torch

from parity import down

pytestmark = pytest.mark.gpu
HALF = torch.float16
RMS, LAYER = 1, 2
COEF = [(3.4445, -4.775, 2.0315)] * 5


class Step:
    """Two blocks h <- 0.9 h + gate * norm(gated(norm(h)) W): what a program keeps, and one training step of it."""

    def __init__(self, hgnn, dev, n=700, D=96, F=136, blocks=2, seed=0):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s, sd=1.0, dtype=HALF: (torch.randn(*s, generator=g) * sd).to(dtype).to(dev)  # noqa: E731
        self.h, self.n, self.D, self.F, self.blocks = hgnn, n, D, F, blocks
        self.x = rnd(n, D, dtype=torch.float32)
        self.target = rnd(n, D, dtype=torch.float32)
        zeros = lambda *s, dtype=HALF: torch.zeros(*s, dtype=dtype, device=dev)  # noqa: E731
        f32 = torch.float32
        self.p, self.a, self.g = [], [], []
        for _ in range(blocks):
            self.p.append(dict(Wg=rnd(F, D, sd=D ** -0.5), Wu=rnd(F, D, sd=D ** -0.5), Wd=rnd(F, D, sd=F ** -0.5), pre=1 + rnd(D, sd=0.1, dtype=f32), post=1 + rnd(D, sd=0.1, dtype=f32),
                               gate=rnd(D, sd=0.5, dtype=f32)))
            self.a.append(dict(H=zeros(n, D, dtype=f32), Z=zeros(n, D), Y=zeros(n, F), B=zeros(n, D)))
            self.g.append(dict(Wg=zeros(F, D), Wu=zeros(F, D), Wd=zeros(F, D, dtype=f32), pre=zeros(D, dtype=f32), post=zeros(D, dtype=f32), gate=zeros(D, dtype=f32)))
        self.out = zeros(n, D, dtype=f32)
        self.dh, self.dB, self.dY, self.dZ = zeros(n, D, dtype=f32), zeros(n, D), zeros(n, F), zeros(n, D)
        self.norm = zeros(1, dtype=f32)
        self.updates = [zeros(F, D, dtype=f32) for _ in range(3 * blocks)]
        sizes = [hgnn.hgnn_gated_workspace(n, D, F), hgnn.hgnn_gated_grad_workspace(n, D, F), hgnn.hgnn_residual_norm_grad_workspace(n, D), hgnn.hgnn_linear_wgrad_workspace(F, D),
                 hgnn.hgnn_grad_norm_workspace(), hgnn.hgnn_orthogonalize_workspace(self.updates)]
        self.ws = torch.empty(max(sizes), dtype=torch.uint8, device=dev)

    def run(self, stream=None):
        h, s = self.h, dict(stream=stream)
        # h_0 = x, z_0 = pre(x); then h_{i+1} = 0.9 h_i + gate * post(b_i) and z_{i+1} = pre(h_{i+1})
        for i, (p, a) in enumerate(zip(self.p, self.a)):
            if i == 0:
                h.hgnn_residual_norm(self.x, None, a["H"], a["Z"], pre=RMS, pre_w=p["pre"], **s)
            h.hgnn_gated(a["Z"], p["Wg"], p["Wu"], a["Y"], act=h.HGNN_SILU, trans_w=True, workspace=self.ws, **s)
            h.hgnn_linear(a["Y"], p["Wd"], a["B"], **s)
            last = i + 1 == self.blocks
            after = {} if last else dict(pre=RMS, pre_w=self.p[i + 1]["pre"])
            h.hgnn_residual_norm(a["H"], a["B"], self.out if last else self.a[i + 1]["H"], None if last else self.a[i + 1]["Z"], post=LAYER, post_w=p["post"], gate=p["gate"], alpha=0.9, **after, **s)
        # the loss 0.5 |out - target|^2 / n, scaled by 64
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
            torch.sub(self.out, self.target, out=self.dh)
            self.dh.mul_(64.0 / self.n)
        for i in reversed(range(self.blocks)):
            p, a, g = self.p[i], self.a[i], self.g[i]
            last = i + 1 == self.blocks
            after = {} if last else dict(pre=RMS, pre_w=self.p[i + 1]["pre"], dpre_w=self.g[i + 1]["pre"])
            h.hgnn_residual_norm_grad(self.out if last else self.a[i + 1]["H"], a["B"], self.dh, None if last else self.dZ, self.dh, self.dB, self.ws, post=LAYER, post_w=p["post"], gate=p["gate"],
                                      alpha=0.9, dgate=g["gate"], dpost_w=g["post"], **after, **s)
            h.hgnn_linear(self.dB, p["Wd"], self.dY, trans_w=True, **s)
            h.hgnn_linear_wgrad(a["Y"], self.dB, g["Wd"], self.ws, **s)
            h.hgnn_gated_grad(a["Z"], p["Wg"], p["Wu"], self.dY, self.dZ, g["Wg"], g["Wu"], self.ws, act=h.HGNN_SILU, trans_w=True, **s)
        h.hgnn_residual_norm_grad(self.a[0]["H"], None, self.dh, self.dZ, self.dh, None, self.ws, pre=RMS, pre_w=self.p[0]["pre"], dpre_w=self.g[0]["pre"], **s)
        weights = [g[k] for g in self.g for k in ("Wg", "Wu", "Wd")]
        vectors = [g[k] for g in self.g for k in ("pre", "post", "gate")]
        h.hgnn_grad_clip(weights + vectors, 1.0, self.norm, self.ws, inv_scale=1 / 64.0, **s)
        h.hgnn_orthogonalize(weights, self.updates, COEF, self.ws, scales=[0.2] * len(weights), **s)

    def results(self):
        return [self.out, self.dh, self.norm, *self.updates, *(g[k] for g in self.g for k in g)]

    def reference(self):
        """The same in 64 bits by autograd on the host -> (out, gradients before clipping, of the weights and of x)."""
        leaf = lambda t: t.detach().cpu().double().requires_grad_(True)  # noqa: E731
        x, ps = leaf(self.x), [{k: leaf(v) for k, v in p.items()} for p in self.p]
        rms = lambda v: v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt()  # noqa: E731
        hh = x
        for p in ps:
            z = rms(hh) * p["pre"]
            b = (torch.nn.functional.silu(z @ p["Wg"].t()) * (z @ p["Wu"].t())) @ p["Wd"]
            c = b - b.mean(1, keepdim=True)
            hh = 0.9 * hh + p["gate"] * (rms(c) * p["post"])
        loss = 0.5 * (hh - self.target.cpu().double()).square().sum() / self.n
        loss.backward()
        return hh.detach(), [{k: v.grad for k, v in p.items()} for p in ps], x.grad


def rel(a, b):
    return float((a.cpu().double() - b).norm() / b.norm())


def test_a_step_against_64_bits(hgnn, dev):
    """Vertex-level values and gradients pass through fp16 some ten times on the way (2^-11 each, relative to their size): 2-norms within 16 x 2^-11 of the exact ones."""
    step = Step(hgnn, dev)
    step.run()
    torch.cuda.synchronize()
    out, grads, dx = step.reference()
    assert rel(step.out, out) <= 16 * 2.0 ** -11
    assert rel(step.dh / 64, dx) <= 16 * 2.0 ** -11
    norm = float(torch.sqrt(sum((v * v).sum() for g in grads for v in g.values())))
    assert abs(float(step.norm[0]) - norm) <= 16 * 2.0 ** -11 * norm
    factor = min(1.0, 1.0 / norm)
    for i, g in enumerate(grads):
        for k, v in g.items():
            assert rel(step.g[i][k], v * factor) <= 16 * 2.0 ** -11, (i, k)
    # orthogonal updates of what the clipped gradients are: singular values between 0.2 x 0.6 and 0.2 x 1.3 for all but the small ones
    for u in step.updates:
        s = torch.linalg.svdvals(u.double().cpu()) / 0.2
        assert float(s.max()) <= 1.3 and float(s.median()) >= 0.6


def test_captured_and_replayed(hgnn, dev):
    step = Step(hgnn, dev, seed=1)
    step.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for k in range(4):
        step.x.mul_(1.1)
        step.p[0]["Wu"].mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in step.results()]
        step.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, step.results())), k


def test_two_steps_at_once(hgnn, dev):
    """Two programs with memory of their own on two streams: what each gets alone."""
    steps = [Step(hgnn, dev, seed=s, n=500 + 300 * s) for s in (2, 3)]
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in s.results()])
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(3):
        for s, q in zip(steps, streams):
            s.run(q)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(w, s.results()))
