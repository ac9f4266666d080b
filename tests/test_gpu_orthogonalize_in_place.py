"""Matrices divided by their norms without any step, in place and not, against 64 bits on the host.

Tolerance, elementwise: an element times 2048 / |G| is rounded once from 64 bits, scale / 2048 is a rounding or none, and their product one: 4 roundings of 2^-24 at
most, and the output's of 2^-11 (2^-25 below fp16's normal numbers) where that is fp16."""
import numpy as np
import pytest
import torch

from parity import down

pytestmark = pytest.mark.gpu
F16, F32 = np.float16, np.float32


def matrix(rows, cols, dtype, seed):
    return np.random.default_rng(seed).standard_normal((rows, cols)).astype(dtype)


LISTS = {"wide": [(64, 608)], "high": [(608, 64)], "one workgroup": [(64, 64)], "many": [(64, 4096)] * 20, "several launches": [(3 + i, 4096 - 100 * i) for i in range(30)],
         "with a large one": [(64, 4096), (100, 300), (4096, 7), (300, 90)]}


@pytest.mark.parametrize("sides", list(LISTS.values()), ids=list(LISTS))
@pytest.mark.parametrize("dtype", [F16, F32])
def test_no_steps(hgnn, dev, sides, dtype):
    print("no steps", sides, dtype.__name__, flush=True)
    mats = [matrix(*s, dtype, i) for i, s in enumerate(sides)]
    scales = [(-1) ** i * (0.5 + i) for i in range(len(mats))]
    grads = [torch.from_numpy(m).to(dev) for m in mats]
    outs = [torch.full_like(g, 3) for g in grads]
    ws = torch.full((hgnn.hgnn_orthogonalize_workspace(grads),), 255, dtype=torch.uint8, device=dev)
    hgnn.hgnn_orthogonalize(grads, outs, [], ws, scales=scales)
    for m, o, s in zip(mats, outs, scales):
        w = m.astype(np.float64)
        ref = s * w / np.sqrt((w * w).sum())
        room = 4 * 2.0 ** -24 * np.abs(ref) + (2.0 ** -11 * np.abs(ref) + 2.0 ** -25 if dtype == F16 else 2.0 ** -24 * np.abs(ref))
        assert (np.abs(down(o).astype(np.float64) - ref) <= room).all(), m.shape
    for _ in range(3):
        again = [torch.from_numpy(m).to(dev) for m in mats]
        ws.fill_(255)
        hgnn.hgnn_orthogonalize(again, None, [], ws, scales=scales)
        assert all(torch.equal(a, o) for a, o in zip(again, outs))
