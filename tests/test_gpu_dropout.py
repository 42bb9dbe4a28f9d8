"""cel.dropout against the generator as published: which values stay is exact, and those are one product in 32
bits (the factor is off by half a step, the product by another: 2^-23 together), rounded once."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402
from block_reference import kept, randn, within  # noqa: E402

DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def check(x, p, seed, step=0, got=None):
    got = cel.dropout(x, p, seed, step=step) if got is None else got
    assert got.shape == x.shape and got.dtype == x.dtype
    columns = x.shape[-1] if x.dim() else 1
    if not x.numel():
        return got
    keep, by = kept(x.numel() // columns, columns, p, seed, int(step))
    want = torch.where(keep, x.double().cpu().reshape(-1, columns) * by, 0.0)
    within(got.reshape(-1, columns), want, 2.0 ** -23 * want.abs())
    assert not bool(got.cpu().reshape(-1, columns)[~keep].any())
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("columns", [1, 2, 7, 8, 9, 15, 64, 100, 1023, 1024, 1025, 2049])
def test_sizes(columns, dtype):
    for rows in (0, 1, 2, 33):
        check(randn(rows, columns, seed=columns).to(dtype).to(DEV), 0.1, 12345, rows)


@pytest.mark.parametrize("p", [0.0, 1e-6, 2.0 ** -17, 2.0 ** -16, 0.05, 0.1, 0.5, 0.9, 1 - 2.0 ** -16, 1 - 2.0 ** -18, 1.0])
def test_probabilities(p):
    x = randn(64, 520, seed=3).to(DEV)
    got = check(x, p, 99)
    if p < 2.0 ** -17:
        assert torch.equal(got, x)
    if p == 1.0:
        assert not bool(got.any())


@pytest.mark.parametrize("seed,step", [(0, 0), (2 ** 32, 0), (2 ** 63 + 5, 1), (2 ** 64 - 1, 2 ** 32), (1, -1), (-1, 2 ** 63 - 1), (7, -2 ** 63)])
def test_seeds_and_steps(seed, step):
    x = randn(20, 72).to(DEV)
    got = check(x, 0.3, seed, step)
    at = torch.tensor([step], dtype=torch.int64, device=DEV)
    assert torch.equal(cel.dropout(x, 0.3, seed, step=at), got)
    assert torch.equal(cel.dropout(x, 0.3, seed, step=at[0]), got)
    assert not torch.equal(cel.dropout(x, 0.3, seed, step=at + 1), got)


def test_share_and_independence():
    """About p of many values, within five deviations, in every column and every row; masks of two steps agree as two coins do."""
    n, p = 1 << 21, 0.25
    x = torch.ones(2048, 1024, device=DEV)
    one, two = cel.dropout(x, p, 5, step=0) > 0, cel.dropout(x, p, 5, step=1) > 0
    for m, share in ((one, 1 - p), (one & two, (1 - p) ** 2)):
        assert abs(float(m.double().mean()) - share) <= 5 * (share * (1 - share) / n) ** 0.5
    for dim, count in ((0, 2048), (1, 1024)):
        assert float((one.double().mean(dim) - 0.75).abs().max()) <= 6 * (0.1875 / count) ** 0.5


def test_shapes_and_strides():
    base = randn(12, 10, 96, seed=1).bfloat16().to(DEV)
    for x in (base, base[:, :, 1:70], base[::2], base[:, ::3], base.transpose(0, 1), base[..., ::2], base[:1].expand(12, 10, 96),
              base[3], base[3, 4], base[3, 4, 5], base[0, 0, :0], base[:, 0], base.flatten(), base[:, :, 0]):
        check(x, 0.4, 17)


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place_and_into_views(dtype):
    wide = randn(31, 100, seed=4).to(dtype).to(DEV)
    before = wide.clone()
    x = wide[:, 3:50]
    want = check(x, 0.2, 8)
    assert cel.dropout(x, 0.2, 8, out=x) is x
    assert torch.equal(x, want) and torch.equal(wide[:, :3], before[:, :3]) and torch.equal(wide[:, 50:], before[:, 50:])
    cel.dropout(x, 0.2, 9, out=wide[:, 53:])
    check(x, 0.2, 9, got=wide[:, 53:])
    assert torch.equal(x, want) and torch.equal(wide[:, 50:53], before[:, 50:53])


def test_what_is_dropped_is_zero_whatever_it_was():
    x = torch.full((16, 64), float("nan"), device=DEV)
    x[::2] = float("inf")
    got, (keep, _) = cel.dropout(x, 0.5, 3).cpu(), kept(16, 64, 0.5, 3, 0)
    assert not bool(got[~keep].any()) and not bool(torch.isfinite(got[keep]).any())


def test_its_gradient_is_the_same_call():
    """By differences: the operation is linear, so that <g, drop(x + h) - drop(x)> = <drop(g), h>."""
    x, h, g = (randn(9, 33, seed=s).to(DEV) for s in (1, 2, 3))
    d = cel.dropout(x + h, 0.3, 4).double() - cel.dropout(x, 0.3, 4).double()
    size = float((g.abs() * (x.abs() + h.abs())).sum()) / 0.7
    assert abs(float((d * g).sum()) - float((cel.dropout(g, 0.3, 4).double() * h).sum())) <= 8 * 2.0 ** -24 * size


def test_one_long_row():
    n = 40_000_003
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    got = cel.dropout(x, 0.5, 21) > 0
    for first in (0, 8 * (1 << 20), n // 8 * 8 - 80):
        blocks = first // 8
        import numpy as np
        from block_reference import philox
        c = [np.arange(blocks, blocks + 10, dtype=np.uint64), np.zeros(10, np.uint64), np.zeros(10, np.uint64), np.zeros(10, np.uint64)]
        words = np.stack(philox(c, 21), 1)
        bits = np.stack([words & np.uint64(0xffff), words >> np.uint64(16)], 2).reshape(-1) >= 32768
        assert bool((got[first:first + 80].cpu().numpy() == bits).all())


def test_more_pieces_than_one_launch_counts():
    """2^32 - 100 rows of one value: two launches, the second from row 2^32 - 257 on."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB of memory")
    n = (1 << 32) - 100
    x = torch.ones(n, 1, dtype=torch.bfloat16, device=DEV)
    got = cel.dropout(x, 0.5, 3, out=x)
    for first in (0, (1 << 31) - 7, n - 200):
        keep, _ = kept(200, 1, 0.5, 3, 0, row0=first)
        assert torch.equal(got[first:first + 200].cpu() > 0, keep)


def test_replayed_graphs_go_on():
    """A step on the device that the graph itself advances: each replay has its own mask."""
    x = randn(64, 200, seed=6).bfloat16().to(DEV)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    want = [cel.dropout(x, 0.1, 77, step=s) for s in range(5)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = cel.dropout(x, 0.1, 77, step=step)
        step.add_(1)
    step.zero_()
    for s in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[s])
        assert torch.equal(cel.dropout(x, 0.1, 77, step=step), want[s + 1])


def test_refusals():
    def refused(*a, **kw):
        with pytest.raises(cel.CelError) as e:
            cel.dropout(*a, **kw)
        assert e.value.code == -1

    x = randn(8, 16).to(DEV)
    for p in (-0.1, 1.5, float("nan")):
        refused(x, p, 1)
    refused(x.double(), 0.1, 1)
    refused(x.cpu(), 0.1, 1)
    refused(x, 0.1, 1, step=torch.zeros(2, dtype=torch.int64, device=DEV))
    refused(x, 0.1, 1, step=torch.zeros(1, dtype=torch.int32, device=DEV))
    refused(x, 0.1, 1, step=torch.zeros(1, dtype=torch.int64))
    refused(x, 0.1, 1, out=torch.empty(8, 15, device=DEV))
    refused(x, 0.1, 1, out=torch.empty(8, 16, device=DEV).half())
    refused(x, 0.1, 1, out=torch.empty(16, 8, device=DEV).T)
    wide = torch.zeros(9, 16, device=DEV)
    refused(wide[:8], 0.1, 1, out=wide[1:])
    refused(wide.flatten()[:128], 0.1, 1, out=wide.flatten()[1:129])
    refused(wide[:4, :8], 0.1, 1, out=wide.flatten()[4:36].view(4, 8))  # rows of another stride between
    cel.dropout(wide[:4, :8], 0.1, 1, out=wide[:4, 8:])
    import numpy as np
    assert torch.equal(cel.dropout(x, 0.5, np.int64(-3), step=np.int64(-1)), cel.dropout(x, 0.5, -3, step=-1))
    refused(x.clone().requires_grad_(), 0.1, 1)
