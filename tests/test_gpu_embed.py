"""cel.embed and cel.embed_grad against the definition.

The lookup is one 32-bit product, rounded once: equal to the same product taken
by the CPU.  A gradient's element is a 32-bit sum of n products, in some order,
scaled and rounded once: off by at most (n + 1) 2^-24 scale sum |dx| and u |it|
(u = 2^-8 bfloat16, 2^-11 float16, 2^-24 float32; 2^-25 below float16's normal
range), to first order; 1 % is added for the higher ones.
"""
from __future__ import annotations

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402

DEV = "cuda:0"
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TYPES = list(UNIT)


def zipf(T, V, seed):
    u = np.random.default_rng([5, seed]).random(T)
    return torch.from_numpy(np.minimum((V + 1.0) ** u - 1.0, V - 1).astype(np.int64))


def randn(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def ref_embed(table, ids, scale):
    ids, table = ids.long().cpu(), table.cpu()
    there = (ids >= 0) & (ids < table.shape[0])
    rows = table[ids.clamp(0, table.shape[0] - 1)].float() * torch.tensor(scale, dtype=torch.float32)
    return torch.where(there[:, None], rows, torch.zeros(())).to(table.dtype)


def check_grad(dx, ids, V, scale, dtype, grad=None):
    grad = cel.embed_grad(dx, ids, V, scale=scale, dtype=dtype) if grad is None else grad
    out_type = dtype or dx.dtype
    assert grad.shape == (V, dx.shape[1]) and grad.dtype == out_type
    ids, x = ids.long().cpu(), dx.double().cpu()
    there = (ids >= 0) & (ids < V)
    ids, x = ids[there], x[there]
    want = torch.zeros(V, dx.shape[1], dtype=torch.float64).index_add_(0, ids, x) * scale
    size = torch.zeros_like(want).index_add_(0, ids, x.abs()) * abs(scale)
    n = torch.bincount(ids, minlength=V).double()[:, None]
    bound = 1.01 * ((n + 1) * 2.0 ** -24 * size + UNIT[out_type] * want.abs())
    if out_type == torch.float16:
        bound += 2.0 ** -25
    assert bool(((grad.double().cpu() - want).abs() <= bound).all())
    assert not grad.cpu()[(n == 0)[:, 0]].any()
    return grad


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("h", [1, 3, 7, 8, 9, 64, 100, 255, 1024, 2049, 8192])
def test_lookup(h, dtype):
    V, T = 300, 77
    table = randn(V, h, seed=h).to(dtype).to(DEV)
    for ids in (zipf(T, V, h), zipf(T, V, h).int()):
        ids = ids.clone()
        ids[3], ids[40], ids[41] = -1, V, 2 ** 31 - 1
        got = cel.embed(table, ids.to(DEV), scale=math.sqrt(h))
        assert torch.equal(got.cpu(), ref_embed(table, ids, math.sqrt(h)))
    assert torch.equal(cel.embed(table, ids.to(DEV)).cpu(), ref_embed(table, ids, 1.0))


@pytest.mark.parametrize("T", [0, 1, 2, 1000])
def test_lookup_lengths_and_one_row(T):
    table = randn(1, 24).to(DEV)
    ids = torch.zeros(T, dtype=torch.int64, device=DEV)
    assert torch.equal(cel.embed(table, ids, scale=2.0), table.repeat(T, 1) * 2.0)


def test_lookup_strides():
    wide = randn(50, 96).to(torch.bfloat16).to(DEV)
    ids = zipf(30, 50, 1)
    for table in (wide[:, 8:72], wide[:, 5:70], wide[::2], wide.T.contiguous().T, wide[:, ::3]):
        ids_ = ids.clamp(max=table.shape[0] - 1)
        assert torch.equal(cel.embed(table, ids_.to(DEV), scale=3.0).cpu(), ref_embed(table, ids_, 3.0))
    every = torch.stack([ids, ids], 1).to(DEV)
    assert torch.equal(cel.embed(wide, every[:, 0]).cpu(), ref_embed(wide, ids, 1.0))


def test_lookup_keeps_infinities():
    table = randn(4, 16).to(DEV)
    table[1], table[2] = float("inf"), float("nan")
    got = cel.embed(table, torch.tensor([1, 2, -1, 3], device=DEV), scale=0.5)
    assert bool(torch.isinf(got[0]).all()) and bool(torch.isnan(got[1]).all())
    assert not got[2].any() and torch.equal(got[3], table[3] * 0.5)


@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, None), (torch.bfloat16, torch.float32), (torch.float16, None),
                                       (torch.float16, torch.float32), (torch.float32, None)])
@pytest.mark.parametrize("h", [1, 5, 8, 72, 1000, 2049])
def test_gradient(h, dtype, out):
    V, T = 500, 700
    ids = zipf(T, V, h)
    ids[::50] = -1
    ids[7], ids[8] = V, 10 ** 9
    dx = randn(T, h, seed=h).to(dtype).to(DEV)
    for i in (ids, ids.int()):
        check_grad(dx, i.to(DEV), V, 1.7, out)


@pytest.mark.parametrize("T", [0, 1, 2, 63, 64, 65, 128, 1023, 1025, 8191, 8192, 8193, 10240, 20000, 70001])
def test_gradient_lengths(T):
    """Both sorts, and the border between them."""
    V = 3000
    check_grad(randn(T, 16, seed=T).to(DEV), zipf(T, V, T).to(DEV), V, 0.5, None)


@pytest.mark.parametrize("V", [1, 2, 511, 512, 513, 262143, 262144, 400001])
@pytest.mark.parametrize("T", [600, 9000])
def test_gradient_vocabularies(V, T):
    """One, two and three passes of the sort."""
    ids = torch.from_numpy(np.random.default_rng(V).integers(0, V, T))
    check_grad(randn(T, 8, seed=V).to(torch.bfloat16).to(DEV), ids.to(DEV), V, 1.0, torch.float32)


@pytest.mark.parametrize("T", [64, 200, 5000, 12345])
def test_gradient_of_one_word(T):
    ids = torch.full((T,), 5, dtype=torch.int32, device=DEV)
    check_grad(randn(T, 40, seed=1).to(DEV), ids, 9, 1.0, None)
    ids[T // 3:T // 2] = 2  # words that begin and end inside a chunk
    check_grad(randn(T, 40, seed=2).to(DEV), ids, 9, -2.0, None)
    check_grad(randn(T, 40, seed=3).to(DEV), torch.full_like(ids, -1), 9, 1.0, None)


def test_gradient_strides():
    wide = randn(900, 200).to(torch.float16).to(DEV)
    ids = zipf(900, 100, 4).to(DEV)
    for dx in (wide[:, 16:80], wide[:, 3:77], wide.T.contiguous().T):
        check_grad(dx, ids, 100, 1.0, torch.float32)


def test_a_word_keeps_its_infinities_to_itself():
    ids = zipf(2000, 50, 3)
    dx = randn(2000, 24).to(DEV)
    plain = cel.embed_grad(dx, ids.to(DEV), 50)
    dx[int((ids == 7).nonzero()[0])] = float("nan")
    got = cel.embed_grad(dx, ids.to(DEV), 50)
    others = torch.arange(50, device=DEV) != 7
    assert torch.equal(got[others], plain[others]) and bool(torch.isnan(got[7]).all())
    ids[ids == 7] = -1
    assert torch.equal(cel.embed_grad(dx, ids.to(DEV), 50)[others], plain[others])


@pytest.mark.parametrize("T", [3000, 30000])
def test_the_same_bits_every_time(T):
    ids, dx = zipf(T, 1000, 1).to(DEV), randn(T, 64).to(torch.bfloat16).to(DEV)
    first = cel.embed_grad(dx, ids, 1000)
    for _ in range(3):
        assert torch.equal(cel.embed_grad(dx, ids, 1000), first)


def test_gradient_is_the_lookups_transpose():
    """<dx, embed(E)> = <embed_grad(dx), E> for every E: the lookup is linear in its table."""
    V, T, h = 200, 300, 32
    ids, dx, E = zipf(T, V, 9).to(DEV), randn(T, h, seed=1).to(DEV), randn(V, h, seed=2).to(DEV)
    a = float((dx.double() * cel.embed(E, ids, scale=1.5).double()).sum())
    b = float((cel.embed_grad(dx, ids, V, scale=1.5).double() * E.double()).sum())
    # every one of T h products carries at most 300 roundings of 2^-24 of its size
    size = float((dx.double().abs() * 1.5 * E[ids].double().abs()).sum())
    assert abs(a - b) <= 302 * 2.0 ** -24 * size


@pytest.mark.parametrize("T", [500, 20000])
def test_on_another_stream_and_in_a_graph(T):
    V, h = 400, 48
    ids, dx, table = zipf(T, V, 2).to(DEV), randn(T, h).to(DEV), randn(V, h, seed=1).to(DEV)

    def step():
        return cel.embed(table, ids, scale=2.0), cel.embed_grad(dx, ids, V)

    plain = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, plain))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for n in range(3):
        ids.copy_(zipf(T, V, 30 + n))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))


def test_refusals():
    table, ids = randn(10, 8).to(DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    dx = randn(4, 8).to(DEV)

    def refused(f, *a, **kw):
        with pytest.raises(cel.CelError) as e:
            f(*a, **kw)
        assert e.value.code == -1

    refused(cel.embed, table.double(), ids)
    refused(cel.embed, table[0], ids)
    refused(cel.embed, table.cpu(), ids)
    refused(cel.embed, table, ids.cpu())
    refused(cel.embed, table, ids.float())
    refused(cel.embed, table, ids.view(2, 2))
    refused(cel.embed, table[:0], ids)
    refused(cel.embed, table[:, :0], ids)
    refused(cel.embed, table, ids, scale=float("nan"))
    refused(cel.embed_grad, dx[:3], ids, 10)
    refused(cel.embed_grad, dx, ids, 0)
    refused(cel.embed_grad, dx, ids, 2 ** 31)
    refused(cel.embed_grad, dx, ids, 10, dtype=torch.bfloat16)
    refused(cel.embed_grad, dx.double(), ids, 10)
    refused(cel.embed_grad, dx, ids, 10, scale=float("inf"))


def test_views_of_a_buffer_beyond_32_bits():
    """Rows 2^22 and 2^23 values apart: the last of them lie past 2^32 bytes."""
    V, T, h = 600, 700, 72
    table, dx, ids = randn(V, h, seed=40).bfloat16(), randn(T, h, seed=41).bfloat16(), zipf(T, V, 42)
    wide = torch.empty(T * 2 ** 22 + V * 2 ** 22, dtype=torch.bfloat16, device=DEV)
    far = wide.as_strided((V, h), (2 ** 23, 1))
    far.copy_(table)
    ids[-3:] = torch.tensor([V - 1, V, V - 2])
    assert torch.equal(cel.embed(far, ids.to(DEV)).cpu(), ref_embed(table, ids, 1.0))
    far = wide.as_strided((T, h), (2 ** 22, 1))
    far.copy_(dx)
    check_grad(far, ids.to(DEV), V, 1.0, None)


@pytest.mark.parametrize("T", [8191, 8192, 8193])
def test_gradient_where_the_sort_changes(T):
    check_grad(randn(T, 24, seed=T).bfloat16().to(DEV), zipf(T, 9000, T).to(DEV), 9000, 1.0, None)


@pytest.mark.parametrize("V,h", [(16384, 8), (16385, 8), (8192, 1024), (8193, 1000)])
def test_gradient_where_a_waves_rows_change(V, h):
    check_grad(randn(900, h, seed=V).bfloat16().to(DEV), zipf(900, V, V).to(DEV), V, 1.0, torch.float32)
