"""Clipping of 192 MB and more, whose outputs are written past the caches, from and into every type, in place and with gaps between rows, element by element on the device.

Tolerances as in test_gpu_grad_clip.py."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FILL = 7.0
HALF, SINGLE = torch.float16, torch.float32


def matrix(rows, cols, pitch, offset, dtype, dev):
    buf = torch.full((rows * pitch + offset + 1,), FILL, dtype=dtype, device=dev)
    return torch.as_strided(buf, (rows, cols), (pitch, 1), offset), buf


TENSORS = [  # rows, columns, pitch, offset, type of the gradient, of the output
    (300001, 100, 100, 0, SINGLE, SINGLE), (400003, 41, 41, 1, HALF, SINGLE), (1, 5000011, 5000011, 3, SINGLE, HALF), (200003, 42, 48, 0, SINGLE, SINGLE),
    (100003, 7, 9, 1, HALF, HALF), (300, 20003, 20005, 1, HALF, SINGLE), (70001, 33, 40, 0, SINGLE, HALF), (1, 3, 3, 1, HALF, HALF), (1, 1000003, 1000003, 0, HALF, HALF),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("inv_scale,max_norm", [(2.0 ** -10, 1.0), (1.0, math.inf)])
def test_outputs_past_the_caches(hgnn, dev, in_place, inv_scale, max_norm):
    print(f"clip past the caches, in place {in_place}, inv_scale {inv_scale} max_norm {max_norm}", flush=True)
    gen = torch.Generator(device=dev).manual_seed(3)
    grads, outs, buffers, copies = [], [], [], []
    for rows, cols, pitch, offset, a, b in TENSORS:
        g, gbuf = matrix(rows, cols, pitch, offset, a, dev)
        g.copy_(torch.randn((rows, cols), generator=gen, device=dev) * 100)
        o, obuf = (g, gbuf) if in_place else matrix(rows, cols, pitch + 2 if pitch > cols else pitch, offset, b, dev)
        grads.append(g), outs.append(o), buffers.append(obuf), copies.append(g.clone())
    assert sum(o.numel() * o.element_size() for o in outs) >= (192 << 20)
    ref = inv_scale * math.sqrt(sum(float(c.double().square().sum()) for c in copies))
    ws = torch.full((hgnn.hgnn_grad_norm_workspace(),), 255, dtype=torch.uint8, device=dev)
    norm = torch.full((1,), FILL, device=dev)
    hgnn.hgnn_grad_clip(grads, max_norm, norm, ws, outs=None if in_place else outs, inv_scale=inv_scale)
    assert abs(float(norm) - ref) <= 6 * U * ref
    factor = inv_scale * min(1.0, max_norm / ref)
    for c, g, o, buf in zip(copies, grads, outs, buffers):
        want = c.double() * factor
        tol = 8 * U * want.abs() + 2.0 ** -149
        if o.dtype == HALF:
            tol += want.abs() * 2.0 ** -11 + 2.0 ** -25
        assert bool(((o.double() - want).abs() <= tol).all()), (o.shape, o.dtype)
        if not in_place:
            assert torch.equal(g, c), "what was read is as it was"
        o.fill_(FILL)
        assert bool((buf == FILL).all()), "something beside the rows was written"


def test_many_tensors_captured(hgnn, dev):
    """Several launches of each pass in a graph, replayed over other gradients, with a number among them that is none and without."""
    gen = torch.Generator(device=dev).manual_seed(5)
    sizes = [1 + 977 * i % 4099 for i in range(230)] + [1500007]
    grads = [torch.zeros(n, dtype=(HALF, SINGLE)[i % 2], device=dev) for i, n in enumerate(sizes)]
    outs = [torch.empty(n, dtype=(SINGLE, HALF)[i % 3 == 0], device=dev) for i, n in enumerate(sizes)]
    ws = torch.empty(hgnn.hgnn_grad_norm_workspace(), dtype=torch.uint8, device=dev)
    norm, alone = torch.zeros(1, device=dev), torch.zeros(1, device=dev)
    call = lambda: (hgnn.hgnn_grad_clip(grads, 2.0, norm, ws, outs=outs, inv_scale=0.25), hgnn.hgnn_grad_norm(grads, alone, ws, inv_scale=0.25))  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for turn in range(5):
        for g in grads:
            g.copy_(torch.randn(g.shape, generator=gen, device=dev) * 3 ** turn)
        if turn == 2:
            grads[150][0] = math.nan
        graph.replay()
        torch.cuda.synchronize()
        got = [norm.clone(), alone.clone()] + [o.clone() for o in outs]
        for o in outs:
            o.fill_(FILL)
        call()
        assert all(torch.equal(a.nan_to_num(nan=-1.0), b.nan_to_num(nan=-1.0)) for a, b in zip(got, [norm, alone] + outs))
        if turn == 2:
            assert math.isnan(float(norm)) and all(bool((o == 0).all()) for o in outs)
            continue
        ref = 0.25 * math.sqrt(sum(float(g.double().square().sum()) for g in grads))
        assert abs(float(norm) - ref) <= 6 * U * ref and torch.equal(norm, alone)
        for g, o in zip(grads, outs):
            want = g.double() * (0.25 * min(1.0, 2.0 / ref))
            tol = 8 * U * want.abs() + 2.0 ** -149 + (want.abs() * 2.0 ** -11 + 2.0 ** -25 if o.dtype == HALF else 0.0)
            assert bool(((o.double() - want).abs() <= tol).all())
