"""Which views of memory attention's gradients may be written to (CPU only: the binding's
arithmetic on addresses against every element's own)."""
import itertools
import random

import pytest

pytest.importorskip("torch")

from paper_2208_00184_amd import _binding as b  # noqa: E402


def elements(at, row, head, T, H, d):
    return [at + t * row + h * head + c for t in range(T) for h in range(H) for c in range(d)]


def block(at, row, head, T, H, d):
    return b._block(b._Rows(2 * at, row, head), T, H, d)


def test_values_of_one_view():
    for T, H, d in itertools.product((1, 2, 5), (1, 2, 3, 6), (8, 16)):
        for row, head in itertools.product(range(d, 140, 8), range(0, 140, 8)):
            e = elements(64, row, head, T, H, d)
            assert b._folded(block(64, row, head, T, H, d), T, d) == (len(set(e)) < len(e)), (T, H, d, row, head)


def test_two_views():
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(20000):
        T, d, H, K = rng.choice((1, 2, 5)), rng.choice((8, 16)), rng.choice((1, 2, 4)), rng.choice((1, 2))
        row = rng.randrange(d, 200, 8)
        at, to = (8 * rng.randrange(0, 60) for _ in range(2))
        x = (at, row, rng.choice((d, 2 * d, 3 * d, row * T)), T, H, d)
        y = (to, row, rng.choice((d, 2 * d, 3 * d, row * T)), T, K, d)
        meet = bool(set(elements(*x)) & set(elements(*y)))
        seen[meet] += 1
        assert b._meet(block(*x), block(*y), T, d) == meet, (x, y)
        assert b._meet(block(*y), block(*x), T, d) == meet, (x, y)
    assert min(seen) > 2000


def test_two_views_of_different_rows():
    x = (0, 64, 16, 4, 2, 16)
    assert b._meet(block(*x), block(0, 128, 16, 4, 2, 16), 4, 16)
    assert not b._meet(block(*x), block(400, 128, 16, 4, 2, 16), 4, 16)
    assert not b._meet(block(*x), block(32, 128, 16, 4, 2, 16), 4, 16)


def test_the_binding_refuses_them(monkeypatch):
    """attention_grad, up to where it would ask for scratch."""
    import torch

    class Reached(Exception):
        pass

    def reached(*_):
        raise Reached

    monkeypatch.setattr(b, "_device_of", lambda fn, **tensors: 0)
    monkeypatch.setattr(b, "_on", lambda index: b.nullcontext())
    monkeypatch.setattr(b, "lib", reached)
    T, H, K, d = 40, 4, 2, 64
    q, dout, out, dq = (torch.zeros(T, H, d, dtype=torch.bfloat16) for _ in range(4))
    k, v, dk, dv = (torch.zeros(T, K, d, dtype=torch.bfloat16) for _ in range(4))
    lse, ptr = torch.zeros(H, T), torch.tensor([0, T], dtype=torch.int32)

    def call(*grads):
        return b.attention_grad(dout, q, k, v, out, lse, ptr, grads=grads)

    def refused(what, *grads):
        with pytest.raises(b.CelError, match=what) as e:
            call(*grads)
        assert e.value.code == b.E_ARG

    fused = torch.zeros(T, (H + 2 * K) * d, dtype=torch.bfloat16)
    parts = [x.view(T, -1, d) for x in fused.split([H * d, K * d, K * d], 1)]
    for grads in ((dq, dk, dv), parts):
        with pytest.raises(Reached):
            call(*grads)
    refused("dq share memory", torch.zeros(T, 1, d, dtype=torch.bfloat16).expand(T, H, d), dk, dv)
    refused("dk share memory", dq, torch.zeros(T, 1, d, dtype=torch.bfloat16).expand(T, K, d), dv)
    refused("dv share memory", dq, dk, torch.zeros(T * d + d, dtype=torch.bfloat16).as_strided((T, K, d), (d, d, 1)))
    refused("dv shares memory with dk", dq, dk, dk)
    refused("dv shares memory with dk", parts[0], parts[1], fused[:, (H + 1) * d:(H + 3) * d].view(T, K, d))
    refused("dq shares memory with q", q, dk, dv)
    refused("dk shares memory with k", dq, k, dv)
    refused("dv shares memory with v", dq, dk, v)
    refused("dq shares memory with dout", dout, dk, dv)
    refused("dq shares memory with out", out, dk, dv)
