"""A training step from learned vertex features to clipped gradients: lookup, GCN layer, projection to class scores, loss, every gradient, clipping.  Every stage is held to its
definition in 64 bits on the values that the stage before it has left; the whole of it is captured, replayed and run beside other work."""
import ctypes

import numpy as np
import pytest
import torch

from parity import compare, down, rand_graph, up

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


class Step:
    """Buffers of a step on a graph of V vertices with learned features: K wide, C classes, scores in rows of pitch P."""

    def __init__(self, hgnn, dev, V=700, N=1500, K=40, C=13, seed=0, extra=None):
        self.h, self.dev = hgnn, dev
        r = np.random.default_rng(seed)
        rowptr, col = rand_graph(V, V, 6, seed, hubs=((3, 400),), empties=(5, V - 1))
        self.rowptr, self.col = rowptr, col
        self.g = hgnn.Csr(up(rowptr, dev), up(col, dev))
        self.gt = hgnn.hgnn_transpose(self.g)
        self.plan, self.plan_t = (hgnn.hgnn_plan_create(x, 256, 48, 1) for x in (self.g, self.gt))
        self.V, self.N, self.K, self.C, self.P = V, N, K, C, (C + 7) // 8 * 8
        half, single = torch.float16, torch.float32
        new = lambda *s, t=half: torch.full(s, 9.0, dtype=t, device=dev)  # noqa: E731
        self.table = up(r.standard_normal((N, K)).astype(np.float32), dev)  # fp32 master copy
        self.W = up((r.standard_normal((K, C)) / 6).astype(np.float16), dev)
        self.ids = torch.empty(V, dtype=torch.int32, device=dev)
        self.labels = torch.empty(V, dtype=torch.int32, device=dev)
        self.load(seed)
        self.x, self.y = new(V, K), new(V, K)
        self.logits, self.dlogits = (torch.zeros((V, self.P), dtype=half, device=dev)[:, :C] for _ in range(2))
        self.logprob, self.stats, self.entropy = new(V, t=single), new(V, 2, t=single), new(V, t=single)
        self.scale = 1024.0
        self.dlogprob = torch.full((V,), -self.scale / V, device=dev)
        self.dentropy = torch.full((V,), -0.01 * self.scale / V, device=dev)
        self.Wt = torch.zeros((K, self.P), dtype=half, device=dev)  # the weight in padded rows: dlogits . W^T reads K columns of it
        self.dy, self.dx = new(V, K), new(V, K)
        self.dW = torch.full((K, self.P), 9.0, device=dev)
        self.dT = new(N, K, t=single)
        self.dW_out, self.dT_out = new(K, C, t=half), new(N, K, t=single)
        self.norm = new(1, t=single)
        u8 = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device=dev)  # noqa: E731
        self.ws_w, self.ws_t = u8(hgnn.hgnn_linear_wgrad_workspace(K, self.P)), u8(hgnn.hgnn_embedding_grad_workspace(V, K, N))
        self.ws_s, self.ws_n = u8(hgnn.hgnn_logprob_workspace(V, C)), u8(hgnn.hgnn_grad_norm_workspace())

    def load(self, seed):
        """Another batch into the same buffers: ids with repeats and padding, labels with some missing."""
        r = np.random.default_rng(100 + seed)
        ids = np.where(r.random(self.V) < 0.3, r.integers(0, 5, self.V), r.integers(0, self.N, self.V))
        ids[r.random(self.V) < 0.05] = -1
        labels = r.integers(0, self.C, self.V)
        labels[r.random(self.V) < 0.2] = -1
        self.ids.copy_(torch.from_numpy(ids.astype(np.int32)))
        self.labels.copy_(torch.from_numpy(labels.astype(np.int32)))

    def run(self):
        h = self.h
        h.hgnn_embedding(self.ids, self.table, self.x, scale=0.5)
        h.hgnn_spmm_discretized(self.plan, self.g, None, 1, self.x, self.y, op=h.HGNN_MEAN)
        h.hgnn_linear(self.y, self.W, self.logits)
        h.hgnn_logprob(self.logits, self.labels, self.logprob, stats=self.stats, entropy=self.entropy, workspace=self.ws_s)
        h.hgnn_logprob_grad(self.logits, self.labels, self.stats, self.dlogprob, self.dlogits, entropy=self.entropy, dentropy=self.dentropy)
        full = torch.as_strided(self.dlogits, (self.V, self.P), (self.P, 1))  # the padding is zero
        h.hgnn_linear_wgrad(self.y, full, self.dW, self.ws_w)
        self.Wt[:, :self.C].copy_(self.W)
        h.hgnn_linear(full, self.Wt, self.dy, trans_w=True)
        h.hgnn_spmm_discretized(self.plan_t, self.gt, None, 1, self.dy, self.dx)
        h.hgnn_embedding_grad(self.ids, self.dx, self.dT, self.ws_t, scale=0.5)
        h.hgnn_grad_clip([self.dW[:, :self.C], self.dT], 0.25, self.norm, self.ws_n, outs=[self.dW_out, self.dT_out], inv_scale=1 / self.scale)

    def outputs(self):
        return [t.clone() for t in (self.x, self.y, self.logits, self.logprob, self.stats, self.entropy, self.dlogits, self.dW, self.dy, self.dx, self.dT, self.norm,
                                    self.dW_out, self.dT_out)]


def same(a, b):
    return all(torch.equal(x.view(torch.uint8) if x.is_contiguous() else x, y.view(torch.uint8) if y.is_contiguous() else y) for x, y in zip(a, b))


def test_every_stage(hgnn, dev):
    s = Step(hgnn, dev)
    s.run()
    d = {k: down(v).astype(np.float64) for k, v in vars(s).items() if isinstance(v, torch.Tensor)}
    ids, labels = down(s.ids), down(s.labels)
    real = ids >= 0
    x = np.where(real[:, None], d["table"][np.where(real, ids, 0)] * 0.5, 0)
    assert np.all(np.abs(d["x"] - x) <= np.abs(x) * 2.0 ** -11 + 2.0 ** -25)
    V, C = s.V, s.C
    A = np.zeros((V, V))
    np.add.at(A, (np.repeat(np.arange(V), np.diff(s.rowptr)), s.col), 1)
    deg = np.maximum(A.sum(1), 1)[:, None]
    compare("aggregation", down(s.y), A @ d["x"] / deg, (A @ np.abs(d["x"])) / deg)
    compare("scores", down(s.logits), d["y"] @ d["W"], np.abs(d["y"]) @ np.abs(d["W"]))
    z = d["logits"]
    lp = z - z.max(1, keepdims=True)
    lp -= np.log(np.exp(lp).sum(1, keepdims=True))
    p = np.exp(lp)
    labelled = labels >= 0
    at = np.where(labelled, labels, 0)
    tol = 64 * U * (1 + np.abs(lp).max(1))  # 13 classes: 2 D + 34 + 3 sum p |d| and the rest of test_gpu_logprob.py's, with D = 9, below 64 (1 + max |log p|)
    assert np.all(np.abs(d["logprob"] - np.where(labelled, lp[np.arange(V), at], 0)) <= tol)
    H = -(p * lp).sum(1)
    assert np.all(np.abs(d["entropy"] - H) <= 4 * tol)
    hot = np.zeros((V, C))
    hot[np.arange(V)[labelled], labels[labelled]] = 1
    g, h = np.where(labelled, d["dlogprob"], 0)[:, None], d["dentropy"][:, None]
    dz = g * (hot - p) - h * p * (lp + H[:, None])
    assert np.all(np.abs(d["dlogits"] - dz) <= np.abs(dz) * 2.0 ** -11 + 2.0 ** -25 + 8 * tol[:, None] * (np.abs(g) + np.abs(h)) * (1 + np.abs(lp)))
    dW = d["y"].T @ d["dlogits"]
    assert np.all(np.abs(d["dW"][:, :C] - dW) <= V * U * (np.abs(d["y"]).T @ np.abs(d["dlogits"])) + 1e-30)
    compare("gradient of the aggregated", down(s.dy), d["dlogits"] @ d["W"].T, np.abs(d["dlogits"]) @ np.abs(d["W"]).T)
    compare("gradient of the features", down(s.dx), A.T @ d["dy"], A.T @ np.abs(d["dy"]))
    dT, mag, m = np.zeros((s.N, s.K)), np.zeros((s.N, s.K)), np.zeros((s.N, 1))
    np.add.at(dT, ids[real], d["dx"][real] * 0.5)
    np.add.at(mag, ids[real], np.abs(d["dx"][real]) * 0.5)
    np.add.at(m, ids[real], 1)
    assert np.all(np.abs(d["dT"] - dT) <= (m + 3) * U * mag)
    norm = np.sqrt((d["dW"][:, :C] ** 2).sum() + (d["dT"] ** 2).sum()) / s.scale
    assert abs(d["norm"][0] - norm) <= 6 * U * norm
    for most in (0.25, norm / 2):  # as in the step, whose norm is less, and to half of it
        if most != 0.25:
            hgnn.hgnn_grad_clip([s.dW[:, :C], s.dT], most, s.norm, s.ws_n, outs=[s.dW_out, s.dT_out], inv_scale=1 / s.scale)
        got_w, got_t = down(s.dW_out).astype(np.float64), down(s.dT_out).astype(np.float64)
        f = min(1, most / norm) / s.scale
        assert np.all(np.abs(got_t - d["dT"] * f) <= 8 * U * np.abs(d["dT"] * f) + 2.0 ** -149)
        assert np.all(np.abs(got_w - d["dW"][:, :C] * f) <= np.abs(d["dW"][:, :C] * f) * (2.0 ** -11 + 8 * U) + 2.0 ** -25)


def test_captured_and_replayed(hgnn, dev):
    """Replays on other batches, with the program's own work and waits in between, give the bits of the eager step."""
    s = Step(hgnn, dev, seed=1)
    eager = []
    for batch in range(4):
        s.load(batch)
        s.run()
        torch.cuda.synchronize()
        eager.append(s.outputs())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for batch in (2, 0, 3, 1, 1, 2):
        s.load(batch)
        for t in (s.x, s.logprob, s.dT, s.norm, s.dT_out):
            t.fill_(float("nan"))
        for ws in (s.ws_w, s.ws_t, s.ws_s, s.ws_n):
            ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert same(s.outputs(), eager[batch]), batch
        if batch == 3:
            s.load(0)
            s.run()
            torch.cuda.synchronize()
            assert same(s.outputs(), eager[0])


def test_two_steps_at_once(hgnn, dev):
    """Two steps with buffers of their own on two streams, and one on a stream that is given by object and by number."""
    a, b = Step(hgnn, dev, seed=2), Step(hgnn, dev, V=900, N=300, K=32, C=21, seed=3)
    want = []
    for s in (a, b):
        s.run()
        torch.cuda.synchronize()
        want.append(s.outputs())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, t in zip((a, b), streams):
        for x in (s.x, s.dT, s.dT_out, s.logprob):
            x.zero_()
        t.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for s, t in zip((a, b), streams):
            with torch.cuda.stream(t):
                s.run()
    torch.cuda.synchronize()
    assert same(a.outputs(), want[0]) and same(b.outputs(), want[1])
    t = streams[0]
    for stream in (t, t.cuda_stream):
        a.dT.zero_(), a.logprob.zero_(), a.x.zero_(), a.norm.zero_(), a.dlogits.zero_()
        t.wait_stream(torch.cuda.current_stream())
        hgnn.hgnn_embedding(a.ids, a.table, a.x, scale=0.5, stream=stream)
        hgnn.hgnn_logprob(a.logits, a.labels, a.logprob, stats=a.stats, entropy=a.entropy, workspace=a.ws_s, stream=stream)
        hgnn.hgnn_logprob_grad(a.logits, a.labels, a.stats, a.dlogprob, a.dlogits, entropy=a.entropy, dentropy=a.dentropy, stream=stream)
        hgnn.hgnn_embedding_grad(a.ids, a.dx, a.dT, a.ws_t, scale=0.5, stream=stream)
        hgnn.hgnn_grad_norm([a.dW[:, :a.C], a.dT], a.norm, a.ws_n, inv_scale=1 / a.scale, stream=stream)
        t.synchronize()
        assert same(a.outputs(), want[0])


def test_an_overflowing_step_adds_nothing(hgnn, dev):
    s = Step(hgnn, dev, seed=4)
    s.dlogprob.fill_(-1e38)  # the scores' gradients overflow fp16
    s.run()
    assert not np.isfinite(down(s.norm)[0])
    assert not torch.count_nonzero(s.dT_out) and not torch.count_nonzero(s.dW_out)


def test_native_calls_and_ctypes_agree(hgnn, dev, monkeypatch):
    """The plain forms are taken by the native module; without it the same bits come by ctypes."""
    b = hgnn.binding
    assert b._calls is not None
    s = Step(hgnn, dev, seed=5)
    taken = []

    class Spy:
        def __getattr__(self, name):
            f = getattr(calls, name)

            def call(*a):
                st = f(*a)
                taken.append((name, st))
                return st
            return call
    calls = b._calls
    monkeypatch.setattr(b, "_calls", Spy())
    s.run()
    hgnn.hgnn_grad_norm((s.dT,), s.norm, s.ws_n)
    torch.cuda.synchronize()
    want = s.outputs()
    names = dict(taken)
    assert all(names[n] == 0 for n in ("embedding", "embedding_grad", "logprob", "logprob_grad", "grad_norm", "grad_clip")), taken
    monkeypatch.setattr(b, "_calls", None)
    s.run()
    hgnn.hgnn_grad_norm((s.dT,), s.norm, s.ws_n)
    torch.cuda.synchronize()
    assert same(s.outputs(), want)


REFUSED = {
    "ids of int64": lambda h, s: h.hgnn_embedding(s.ids.long(), s.table, s.x),
    "ids with a stride": lambda h, s: h.hgnn_embedding(s.ids.repeat(2)[::2], s.table, s.x),
    "a table in doubles": lambda h, s: h.hgnn_embedding(s.ids, s.table.double(), s.x),
    "a transposed table": lambda h, s: h.hgnn_embedding(s.ids, torch.empty((s.K, s.N), device=s.dev).t(), s.x),
    "an output in fp32": lambda h, s: h.hgnn_embedding(s.ids, s.table, s.x.float()),
    "an output of another width": lambda h, s: h.hgnn_embedding(s.ids, s.table, s.x[:, :8]),
    "fewer ids than rows": lambda h, s: h.hgnn_embedding(s.ids[:-1], s.table, s.x),
    "rows that are one row": lambda h, s: h.hgnn_embedding(s.ids, s.table, s.x[:1].expand(s.V, s.K)),
    "a gradient of another height": lambda h, s: h.hgnn_embedding_grad(s.ids, s.dx[:-1], s.dT, s.ws_t),
    "a gradient of another width": lambda h, s: h.hgnn_embedding_grad(s.ids, s.dx[:, :8], s.dT, s.ws_t),
    "no workspace": lambda h, s: h.hgnn_embedding_grad(s.ids, s.dx, s.dT, None),
    "a small workspace": lambda h, s: h.hgnn_embedding_grad(s.ids, s.dx, s.dT, s.ws_t[:1024]),
    "a workspace at an odd address": lambda h, s: h.hgnn_embedding_grad(s.ids, s.dx, s.dT, torch.empty(s.ws_t.numel() + 8, dtype=torch.uint8, device=s.dev)[8:]),
    "labels on the host": lambda h, s: h.hgnn_logprob(s.logits, s.labels.cpu(), s.logprob),
    "labels of int64": lambda h, s: h.hgnn_logprob(s.logits, s.labels.long(), s.logprob),
    "labels alone": lambda h, s: h.hgnn_logprob(s.logits, s.labels, None),
    "stats of another shape": lambda h, s: h.hgnn_logprob(s.logits, s.labels, s.logprob, stats=s.stats.t().contiguous()),
    "stats with a pitch": lambda h, s: h.hgnn_logprob(s.logits, s.labels, s.logprob, stats=torch.empty((s.V, 3), device=s.dev)[:, :2]),
    "values without classes": lambda h, s: h.hgnn_logprob(s.logits, s.labels, s.logprob, top_logprob=torch.empty((s.V, 2), device=s.dev)),
    "more alternatives than classes": lambda h, s: h.hgnn_logprob(s.logits, s.labels, s.logprob, top_logprob=torch.empty((s.V, 14), device=s.dev),
                                                                  top_class=torch.empty((s.V, 14), dtype=torch.int32, device=s.dev)),
    "scores in bfloat16": lambda h, s: h.hgnn_logprob(s.logits.bfloat16(), s.labels, s.logprob),
    "one vector of scores": lambda h, s: h.hgnn_logprob(s.logits[0], s.labels[:1], s.logprob[:1]),
    "a gradient of another type": lambda h, s: h.hgnn_logprob_grad(s.logits, s.labels, s.stats, s.dlogprob, s.dlogits.float()),
    "no stats": lambda h, s: h.hgnn_logprob_grad(s.logits, s.labels, None, s.dlogprob, s.dlogits),
    "the entropy's gradient without the entropy": lambda h, s: h.hgnn_logprob_grad(s.logits, s.labels, s.stats, s.dlogprob, s.dlogits, dentropy=s.dentropy),
    "a transposed gradient": lambda h, s: h.hgnn_grad_norm([s.dT.t()], s.norm, s.ws_n),
    "a broadcast gradient": lambda h, s: h.hgnn_grad_norm([s.dT[:1].expand(4, s.K)], s.norm, s.ws_n),
    "outputs of another number": lambda h, s: h.hgnn_grad_clip([s.dT], 1.0, s.norm, s.ws_n, outs=[]),
    "outputs of another shape": lambda h, s: h.hgnn_grad_clip([s.dT], 1.0, s.norm, s.ws_n, outs=[s.dW]),
    "the same tensor twice": lambda h, s: h.hgnn_grad_clip([s.dT, s.dT], 1.0, s.norm, s.ws_n),
    "a norm below zero": lambda h, s: h.hgnn_grad_clip([s.dT], -1.0, s.norm, s.ws_n),
    "no scale": lambda h, s: h.hgnn_grad_clip([s.dT], 1.0, s.norm, s.ws_n, inv_scale=0.0),
    "a norm in doubles": lambda h, s: h.hgnn_grad_norm([s.dT], s.norm.double(), s.ws_n),
    "a gradient in bfloat16": lambda h, s: h.hgnn_grad_norm([s.dT.bfloat16()], s.norm, s.ws_n),
}


@pytest.mark.parametrize("what", sorted(REFUSED))
def test_refusals_of_the_binding(hgnn, dev, what):
    """On the host, before anything is launched: nothing has changed."""
    s = Step(hgnn, dev, seed=6)
    before = s.outputs()
    with pytest.raises((TypeError, ValueError, hgnn.HgnnError, AttributeError)):
        REFUSED[what](hgnn, s)
    torch.cuda.synchronize()
    assert same(s.outputs(), before)


def test_tensors_of_another_device(hgnn, dev, monkeypatch):
    """Tensors of a device that is not the current one are refused by both routes (the streams and launches would be the current one's): nothing has changed."""
    b = hgnn.binding
    s = Step(hgnn, dev, seed=7)
    before = s.outputs()
    calls = [lambda: hgnn.hgnn_embedding(s.ids, s.table, s.x), lambda: hgnn.hgnn_embedding_grad(s.ids, s.dx, s.dT, s.ws_t),
             lambda: hgnn.hgnn_logprob(s.logits, s.labels, s.logprob, stats=s.stats), lambda: hgnn.hgnn_logprob_grad(s.logits, s.labels, s.stats, s.dlogprob, s.dlogits),
             lambda: hgnn.hgnn_grad_norm([s.dT], s.norm, s.ws_n), lambda: hgnn.hgnn_grad_clip([s.dT], 1.0, s.norm, s.ws_n)]
    native, addresses = b._calls, {n: ctypes.cast(getattr(hgnn.load(), n), ctypes.c_void_p).value for n in hgnn.EXPORTS}
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    native.bind(addresses, b._raw_stream, lambda: 1)
    try:
        for call in calls:
            with pytest.raises(ValueError, match="device 0 while device 1"):
                call()
    finally:
        native.bind(addresses, b._raw_stream, b._current_device)
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert same(s.outputs(), before)
    for call in calls:
        call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("native", [True, False])
def test_nothing_and_the_least(hgnn, dev, native, monkeypatch):
    """No positions, no rows, no classes asked for, no tensors, tensors without elements, of no axis or several: every one is a call like another."""
    if not native:
        monkeypatch.setattr(hgnn.binding, "_calls", None)
    zeros = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device=dev)  # noqa: E731
    ones = lambda *s, t=torch.float32: torch.ones(s, dtype=t, device=dev)  # noqa: E731
    h, i = torch.float16, torch.int32
    hgnn.hgnn_embedding(zeros(0, t=i), zeros(5, 8), zeros(0, 8, t=h))
    for table, want in ((zeros(0, 8), 0), (ones(1, 8), 24), (ones(2, 9)[:, 1:], 24)):
        out = ones(3, 8, t=h)
        hgnn.hgnn_embedding(zeros(3, t=i), table, out)
        assert float(out.sum()) == want
    dT = ones(5, 8)
    hgnn.hgnn_embedding_grad(zeros(0, t=i), zeros(0, 8, t=h), dT, None)
    assert float(dT.abs().sum()) == 0
    hgnn.hgnn_embedding_grad(zeros(3, t=i), zeros(3, 8, t=h), zeros(0, 8), zeros(4096, t=torch.uint8))
    hgnn.hgnn_logprob(zeros(0, 7, t=h), zeros(0, t=i), zeros(0), stats=zeros(0, 2), entropy=zeros(0), top_logprob=zeros(0, 3), top_class=zeros(0, 3, t=i))
    hgnn.hgnn_logprob(zeros(3, 7, t=h), None, None)
    hgnn.hgnn_logprob(zeros(3, 7, t=h), None, None, top_logprob=zeros(3, 0), top_class=zeros(3, 0, t=i))
    hgnn.hgnn_logprob_grad(zeros(0, 7, t=h), zeros(0, t=i), zeros(0, 2), zeros(0), zeros(0, 7, t=h))
    dx = ones(3, 7, t=h)
    hgnn.hgnn_logprob_grad(zeros(3, 7, t=h), None, zeros(3, 2), None, dx)
    assert float(dx.abs().sum()) == 0
    ws, norm = torch.empty(hgnn.hgnn_grad_norm_workspace(), dtype=torch.uint8, device=dev), ones(1)
    for tensors, want in (([], 0.0), ([zeros(0), zeros(4, 0), zeros(0, 4)], 0.0), ([zeros(0), ones(), ones(2, 3, 4)], 5.0), ([ones(5, 8)[:, :3], ones(1, t=h)], 4.0)):
        for call in (lambda: hgnn.hgnn_grad_norm(tensors, norm, ws), lambda: hgnn.hgnn_grad_clip(tensors, 2.0, norm, ws)):
            norm.fill_(7)
            call()
            assert float(norm) == want
        assert all(bool((t == min(1.0, 2.0 / max(want, 1e-9))).all()) for t in tensors)
    torch.cuda.synchronize()


def test_sizes_beyond_int32(hgnn, dev):
    """Rows and classes that a 32-bit number would cut to a few are refused, not cut."""
    far = torch.empty(2 ** 32 + 9, dtype=torch.float16, device=dev)
    single, ids = torch.zeros(1, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    stats, out = torch.zeros((1, 2), device=dev), torch.zeros((1, 1), dtype=torch.float16, device=dev)
    ws = torch.empty(4096, dtype=torch.uint8, device=dev)
    for call in (lambda: hgnn.hgnn_embedding(ids, far[:, None], out), lambda: hgnn.hgnn_embedding_grad(ids, out, far[:, None], ws),
                 lambda: hgnn.hgnn_logprob(far[None], ids, single), lambda: hgnn.hgnn_logprob_grad(far[None], ids, stats, single, far[None]),
                 lambda: hgnn.hgnn_embedding_grad_workspace(1, 1, 2 ** 32 + 9), lambda: hgnn.hgnn_logprob_workspace(1, 2 ** 32 + 9, 1)):
        with pytest.raises(ValueError, match="int32"):
            call()


def test_two_graphs_share_a_workspace(hgnn, dev):
    """Captured calls of different sizes with one workspace, replayed in turn: every one finds in it only what it has written itself."""
    rng = np.random.default_rng(8)
    norm_ws = torch.empty(hgnn.hgnn_grad_norm_workspace(), dtype=torch.uint8, device=dev)
    sizes = ((3000, 400, 24, 5003), (20011, 50, 40, 3001))
    need = max(max(hgnn.hgnn_embedding_grad_workspace(n, F, V), hgnn.hgnn_logprob_workspace(3, C, 20)) for n, V, F, C in sizes)
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    runs = []
    for n, V, F, C in sizes:
        ids = up(rng.integers(-1, V, n).astype(np.int32), dev)
        dY, x = up(rng.standard_normal((n, F)).astype(np.float16), dev), up(rng.standard_normal((3, C)).astype(np.float32), dev)
        y = up(rng.integers(0, C, 3).astype(np.int32), dev)
        outs = (torch.zeros((V, F), device=dev), torch.zeros(3, device=dev), torch.zeros((3, 20), device=dev), torch.zeros((3, 20), dtype=torch.int32, device=dev),
                torch.zeros(1, device=dev), torch.zeros((n, F), device=dev))

        def run(ids=ids, dY=dY, x=x, y=y, outs=outs):
            hgnn.hgnn_embedding_grad(ids, dY, outs[0], ws)
            hgnn.hgnn_logprob(x, y, outs[1], top_logprob=outs[2], top_class=outs[3], workspace=ws)
            hgnn.hgnn_grad_clip([dY], 1.0, outs[4], norm_ws, outs=[outs[5]])
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        runs.append((graph, run, outs, want))
    for turn in range(4):
        for graph, run, outs, want in runs if turn % 2 else runs[::-1]:
            for t in outs:
                t.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn
        runs[turn % 2][1]()  # and an eager one between them
