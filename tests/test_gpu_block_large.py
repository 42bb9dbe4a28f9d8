"""A block's operations on arrays of more than 2^32 bytes: the last rows are those of a call on them alone."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402
from attention_bounds import outside  # noqa: E402
from block_reference import Joint, randn, within  # noqa: E402
from cross_bounds import definition  # noqa: E402

DEV = "cuda:0"
T, LAST = 300_007, 40


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GiB of memory")
    yield
    torch.cuda.empty_cache()


def big(small):
    """Rows of zeros, and behind them small's."""
    x = torch.zeros(T, *small.shape[1:], dtype=small.dtype, device=DEV)
    x[-len(small):] = small.to(DEV)
    return x


def test_rotary():
    small = randn(LAST, 64, 128, seed=1).bfloat16()
    pos, freqs = torch.arange(T, device=DEV), torch.rand(64, device=DEV)
    got = cel.rotary(big(small), pos, freqs)
    assert torch.equal(got[-LAST:], cel.rotary(small.to(DEV), pos[-LAST:], freqs)) and not bool(got[:5].any())


def test_norms():
    h = 8192
    f, x, dy, dz = (randn(LAST, h, seed=i).bfloat16() for i in range(4))
    w = randn(h, seed=5, at=1.0).to(DEV)
    how = dict(post=w, gate=w, eps=1e-3)
    F, X = big(f), big(x)
    y, z = cel.residual_norm(F, X, w, **how)
    y1, z1 = cel.residual_norm(f.to(DEV), x.to(DEV), w, **how)
    assert torch.equal(y[-LAST:], y1) and torch.equal(z[-LAST:], z1) and not bool(z[:5].any())
    del X, z
    DY, DZ = big(dy), big(dz)
    dx, df, grads = cel.residual_norm_grad(DY, DZ, F, y, w, **how)
    dx1, df1, grads1 = cel.residual_norm_grad(dy.to(DEV), dz.to(DEV), f.to(DEV), y1, w, **how)
    assert torch.equal(dx[-LAST:], dx1) and torch.equal(df[-LAST:], df1)
    want = Joint(w, **how).backward(dy, dz, f, y1.cpu())
    for n in grads:  # the other rows add zeros: the last ones' sums, in some order
        within(grads[n], *want[n])


def test_cross_attention():
    """States behind 2^32 bytes of others."""
    H, d, n = 64, 128, 70
    q, k, v = (randn(m, H, d, seed=m).bfloat16() for m in (5, n, n + 1))
    K, V = big(k), big(v[:n])
    ptr = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    out, lse = cel.cross_attention(q.to(DEV), K, V, ptr(0, 5), ptr(T - n, T))
    out1, lse1 = cel.cross_attention(q.to(DEV), k.to(DEV), v[:n].to(DEV), ptr(0, 5), ptr(0, n))
    want = definition(q, k, v[:n], torch.zeros_like(q), [5], [n])
    for got in ((out, lse), (out1, lse1)):
        for name, x in zip(("out", "lse"), got):
            assert outside(want, name, x)[0] == 0, name
