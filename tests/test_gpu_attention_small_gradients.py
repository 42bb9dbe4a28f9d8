"""Attention's gradient in float16 over the sizes that a loss and its scale give it: the
operation is linear in dout, and so is its accuracy until the results themselves leave
float16's range.  Every element against its own bound (attention_bounds)."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402
from attention_bounds import definition, outside  # noqa: E402

DEV = "cuda:0"


def check(q, k, v, dout, lengths):
    expected = definition(q, k, v, dout, lengths)
    assert max(float(expected[n][0].abs().max()) for n in ("out", "dq", "dk", "dv")) < 65504
    ptr = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32), device=DEV)
    q, k, v, dout = (x.to(DEV) for x in (q, k, v, dout))
    out, lse = cel.attention(q, k, v, ptr)
    dq, dk, dv = cel.attention_grad(dout, q, k, v, out, lse, ptr)
    bad = {n: outside(expected, n, x) for n, x in dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv).items()}
    assert not any(n for n, _ in bad.values()), bad


def batch(T, H, K, d, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(T, n, d, generator=g) for n in (H, K, K, H)]


# the sizes of a batch, and its tiles: keys of one group of waves or of two, one head's rows in a part or all
SHAPES = [([250, 60, 1, 100], 2, 1, 64), ([700], 2, 2, 64), ([4096], 1, 1, 64), ([2500, 500], 2, 1, 128), ([500, 600], 32, 32, 32),
          ([333, 90], 3, 1, 80)]


@pytest.mark.parametrize("lengths,H,K,d", SHAPES)
@pytest.mark.parametrize("by", [-14, -12, -6, 0])
def test_small(lengths, H, K, d, by):
    q, k, v, g = batch(sum(lengths), H, K, d, 100 + d)
    check(q.half(), k.half(), v.half(), (g * 2.0 ** by).half(), lengths)


@pytest.mark.parametrize("lengths,H,K,d", [([250, 60, 1, 100], 2, 1, 64), ([600], 2, 2, 128), ([500, 600], 32, 32, 32)])
def test_large(lengths, H, K, d):
    """dp passes float16's range, the gradients do not."""
    q, k, v, g = batch(sum(lengths), H, K, d, 200 + d)
    q, k, v, g = (q / 8).half(), (k / 8).half(), (v * 64).half(), (g * 512).half()
    assert float((g[:, 0].double() @ v[:, 0].double().T).abs().max()) > 65504
    check(q, k, v, g, lengths)


@pytest.mark.parametrize("lengths,H,K,d", SHAPES)
def test_rows_of_different_sizes(lengths, H, K, d):
    """Every token's dout of a size of its own, 2^-14 to 2^3, in no order, falling and rising."""
    T = sum(lengths)
    q, k, v, g = batch(T, H, K, d, 300 + d)
    sizes = torch.rand(T, generator=torch.Generator().manual_seed(d)) * 17 - 14
    for s in (sizes, sizes.sort().values, sizes.sort(descending=True).values):
        check(q.half(), k.half(), v.half(), (g * torch.exp2(s)[:, None, None]).half(), lengths)


def test_none_and_one():
    """Gradients of 0 stay 0, and one token's alone reaches the others."""
    lengths = [100, 150]
    q, k, v, g = (x.half() for x in batch(250, 2, 1, 64, 7))
    check(q, k, v, torch.zeros_like(g), lengths)
    one = torch.zeros_like(g)
    one[180] = g[180] * 2.0 ** -10
    check(q, k, v, one, lengths)
