"""cel.embed and cel.embed_grad whose results are larger than the 256 MiB up to which
they are kept in the caches: every row of the lookup and sampled rows of the gradient."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402

DEV = "cuda:0"
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TYPES = list(UNIT)


def rows_past(h, dtype):
    return (256 << 20) // (h * torch.empty(0, dtype=dtype).element_size()) + 3


@pytest.mark.parametrize("h", [1023, 2049, 1024])
@pytest.mark.parametrize("dtype", TYPES)
def test_lookup(h, dtype):
    V, T = 211, rows_past(h, dtype)
    table = torch.randn(V, h, generator=torch.Generator().manual_seed(h)).to(dtype).to(DEV)
    ids = torch.randint(-1, V + 1, (T,), generator=torch.Generator().manual_seed(1)).to(DEV)
    got = cel.embed(table, ids, scale=1.5)
    want = torch.cat([(table.float() * 1.5).to(dtype), torch.zeros(2, h, dtype=dtype, device=DEV)])
    for a in range(0, T, 8192):
        assert torch.equal(got[a:a + 8192], want[ids[a:a + 8192].clamp(max=V)])


@pytest.mark.parametrize("h", [1023, 2049, 1024])
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                       (torch.float16, torch.float16), (torch.float32, torch.float32)])
def test_gradient(h, dtype, out):
    """Sums of n terms in 32 bits, in some order, scaled and rounded once: (n + 1) 2^-24 of the
    sizes, and the result's rounding, with 1 % for higher orders."""
    V, T = rows_past(h, out), 1500
    gen = torch.Generator().manual_seed(h)
    dx = torch.randn(T, h, generator=gen).to(dtype)
    ids = torch.randint(0, V, (T,), generator=gen)
    ids[:200], ids[200:240], ids[240:250] = V - 1, 0, -1
    grad = cel.embed_grad(dx.to(DEV), ids.to(DEV), V, scale=1.5, dtype=out)
    assert grad.shape == (V, h) and grad.dtype == out
    words, at = ids[ids >= 0].unique(return_inverse=True)
    x = dx[ids >= 0].double()
    want, size = (torch.zeros(len(words), h, dtype=torch.float64).index_add_(0, at, y) * 1.5 for y in (x, x.abs()))
    n = torch.bincount(at).double()[:, None]
    bound = 1.01 * ((n + 1) * 2.0 ** -24 * size + UNIT[out] * want.abs()) + (2.0 ** -25 if out == torch.float16 else 0.0)
    assert bool(((grad[words.to(DEV)].double().cpu() - want).abs() <= bound).all())
    grad[words.to(DEV)] = 0
    assert not grad.any()
