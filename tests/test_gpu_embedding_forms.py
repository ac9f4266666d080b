"""Rows of a table where they are many: four of them to a group of lanes, through the caches and past them, compared on the device.

Tolerances as in test_gpu_embedding.py: a value takes the scale's product (2^-24 of it) and one rounding to fp16 (2^-11, half a subnormal step below the normal range)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

FILL = 7.0
HALF, SINGLE = torch.float16, torch.float32


def strided(rows, cols, pitch, offset, dtype, dev):
    buf = torch.full((rows * pitch + offset + 1,), FILL, dtype=dtype, device=dev)
    return torch.as_strided(buf, (rows, cols), (pitch, 1), offset), buf


LOOKUPS = [  # n, V, F, pitch of the table, of the output, offset into both
    (99991, 23300, 100, 104, 104, 0), (99991, 23300, 100, 100, 101, 1), (270001, 5000, 42, 43, 45, 3), (1100003, 300, 7, 7, 7, 0), (1100003, 20000, 8, 11, 9, 5), (33003, 999, 333, 335, 333, 1),
    (20001, 77, 1000, 1000, 1003, 0), (600001, 4097, 13, 16, 13, 0), (65537, 70000, 128, 128, 128, 0),
    (303001, 9000, 333, 334, 335, 1), (101003, 500, 1001, 1001, 1001, 0), (800003, 30000, 128, 128, 136, 0),  # 192 MB and more
]


@pytest.mark.parametrize("dtype", [HALF, SINGLE])
@pytest.mark.parametrize("n,V,F,ldt,ldo,offset", LOOKUPS)
def test_many_rows(hgnn, dev, n, V, F, ldt, ldo, offset, dtype):
    """With ids among them that are none."""
    print(f"lookup n={n} V={V} F={F} pitches {ldt} {ldo} {dtype}", flush=True)
    lanes = 1
    while lanes < 64 and 8 * lanes < F:
        lanes *= 2
    assert n * lanes >= 1 << 20
    gen = torch.Generator(device=dev).manual_seed(n + F)
    table, _ = strided(V, F, ldt, offset, dtype, dev)
    table.copy_(torch.randn((V, F), generator=gen, device=dev))
    ids = torch.randint(0, V, (n,), generator=gen, device=dev, dtype=torch.int32)
    none = torch.rand(n, generator=gen, device=dev) < 0.3
    ids = torch.where(none, torch.tensor([-1, V, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device=dev)[torch.arange(n, device=dev) % 4], ids)
    ids[-5:] = torch.tensor([V - 1, -1, 0, V, V - 1], dtype=torch.int32, device=dev)
    real = (ids >= 0) & (ids < V)
    out, buf = strided(n, F, ldo, offset, HALF, dev)
    for scale in (1.0, -0.375):  # (a number of few bits: the same in 32 and 64)
        out.fill_(3.0)
        hgnn.hgnn_embedding(ids, table, out, scale=scale)
        for r in range(0, n, 1 << 17):
            part = slice(r, min(r + (1 << 17), n))
            ref = torch.where(real[part, None], table[torch.where(real[part], ids[part], 0).long()].double() * scale, 0.0)
            got = out[part]
            if scale == 1.0:
                assert torch.equal(got, ref.to(HALF) if dtype == HALF else ref.float().to(HALF))
            assert bool(((got.double() - ref).abs() <= ref.abs() * (2.0 ** -11 + 2.0 ** -24) + 2.0 ** -25).all())
    out.fill_(FILL)
    assert bool((buf == FILL).all()), "something beside the rows was written"


@pytest.mark.parametrize("dtype", [HALF, SINGLE])
@pytest.mark.parametrize("n,V,F,ldy,ldt,offset", [(600011, 13292, 42, 48, 48, 0), (200003, 1001, 100, 101, 103, 1), (600011, 97, 7, 7, 9, 1), (70001, 40, 520, 523, 520, 0)])
def test_accumulated_gradients_of_many_positions(hgnn, dev, n, V, F, ldy, ldt, offset, dtype):
    """Whole numbers, whose sums are exact in fp32 in any order (n times 4 and 3 are below 2^24): one rounding to fp16 is all there is."""
    print(f"accumulated table gradient n={n} V={V} F={F} {dtype}", flush=True)
    gen = torch.Generator(device=dev).manual_seed(n + F)
    u = torch.rand(n, generator=gen, device=dev)
    ids = (V * u * u * u).to(torch.int32).clamp_(max=V - 1)
    ids[torch.rand(n, generator=gen, device=dev) < 0.05] = -1
    ids[ids == 5] = 6  # a row without a position
    dY, _ = strided(n, F, ldy, offset, HALF, dev)
    dY.copy_(torch.randint(-4, 5, (n, F), generator=gen, device=dev))
    T, buf = strided(V, F, ldt, offset, dtype, dev)
    T.copy_(torch.randint(-3, 4, (V, F), generator=gen, device=dev))
    real = ids >= 0
    want = T.double().index_add_(0, ids[real].long(), dY[real].double() * 0.5)
    ws = torch.full((hgnn.hgnn_embedding_grad_workspace(n, F, V),), 255, dtype=torch.uint8, device=dev)
    hgnn.hgnn_embedding_grad(ids, dY, T, ws, scale=0.5, accumulate=True)
    assert torch.equal(T, want.to(dtype))
    T.fill_(FILL)
    assert bool((buf == FILL).all()), "something beside the rows was written"


@pytest.mark.parametrize("n,V,F,ldy", [(26000003, 5003, 1, 1), (2 ** 24 + 77, 300007, 126, 130)])
@pytest.mark.parametrize("hub", [False, True])
def test_gradients_of_very_many_positions(hgnn, dev, n, V, F, ldy, hub):
    """More tiles of the sort than its sums are taken of at once, and rows of dY beyond 2^31 elements.  Whole numbers from -1 to 1, whose sums are
    exact in fp32 in any order while an id has fewer than 2^24 positions."""
    print(f"table gradient of {n} positions V={V} F={F} hub={hub}", flush=True)
    gen = torch.Generator(device=dev).manual_seed(n % 1000 + F)
    ids = torch.randint(0, V, (n,), generator=gen, device=dev, dtype=torch.int32)
    if hub:
        ids[torch.rand(n, generator=gen, device=dev) < 0.45] = V // 3
    ids[torch.rand(n, generator=gen, device=dev) < 0.01] = -1
    ids[-3:] = torch.tensor([V - 1, 0, V - 1], dtype=torch.int32, device=dev)
    assert int((ids == V // 3).sum()) < 1 << 24
    dY = torch.empty((n, ldy), dtype=HALF, device=dev)[:, :F]
    for r in range(0, n, 1 << 20):
        part = dY[r:r + (1 << 20)]
        part.copy_(torch.randint(-1, 2, part.shape, generator=gen, device=dev, dtype=torch.int8))
    T = torch.full((V, F), FILL, device=dev)
    ws = torch.full((hgnn.hgnn_embedding_grad_workspace(n, F, V),), 255, dtype=torch.uint8, device=dev)
    hgnn.hgnn_embedding_grad(ids, dY, T, ws)
    torch.cuda.synchronize()
    print("  sums on the device are there", flush=True)
    want = torch.zeros((V, F), dtype=torch.float64, device=dev)
    for r in range(0, n, 1 << 20):
        i, y = ids[r:r + (1 << 20)].long(), dY[r:r + (1 << 20)].double()
        rest = (i >= 0) & (i != V // 3)  # (torch adds rows of one index one by one: half a million of the same would take seconds)
        want.index_add_(0, i[rest], y[rest])
        want[V // 3] += y[i == V // 3].sum(0)
    assert torch.equal(T.double(), want)
