"""cel.embed and cel.embed_grad beyond 2^24 workgroups, which one row of a launch's grid does not take."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402

DEV = "cuda:0"


def test_lookup():
    T = 2 ** 28 + 5
    table = torch.arange(1, 8, device=DEV, dtype=torch.float32).to(torch.bfloat16)[:, None]
    ids = torch.arange(2 ** 14, device=DEV, dtype=torch.int32).mul_(31).remainder_(7).repeat(2 ** 14)
    ids = torch.cat([ids, ids[:5].flip(0)])
    got = cel.embed(table, ids)
    assert got.shape == (T, 1)
    for a in range(0, T, 2 ** 26):
        assert torch.equal(got[a:a + 2 ** 26, 0].float(), ids[a:a + 2 ** 26].float() + 1.0)


def test_gradient():
    V = 2 ** 28 + 9
    ids = torch.tensor([0, 5, V - 1, 2 ** 27, V - 1, V - 2, 5, 2 ** 28 - 1, 2 ** 28], device=DEV)
    dx = torch.arange(1, 10, device=DEV, dtype=torch.float32).to(torch.bfloat16)[:, None]
    grad = cel.embed_grad(dx, ids, V)
    assert grad.shape == (V, 1)
    at = torch.tensor([0, 5, 2 ** 27, 2 ** 28 - 1, 2 ** 28, V - 2, V - 1], device=DEV)
    assert grad[at, 0].tolist() == [1.0, 9.0, 4.0, 8.0, 9.0, 6.0, 8.0]
    assert int(grad.count_nonzero()) == 7
