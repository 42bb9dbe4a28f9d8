"""What the binding of the training-step operations refuses and accepts besides the sizes and types."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402

DEV = "cuda:0"


def refused(f, *a, **kw):
    with pytest.raises(cel.CelError) as e:
        f(*a, **kw)
    assert e.value.code == -1


def batch(T=40, H=4, K=2, d=64, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(T, n, d, generator=g).bfloat16().to(DEV) for n in (H, K, K, H)] + [
        torch.tensor([0, T], dtype=torch.int32, device=DEV)]


def test_tensors_that_ask_for_a_gradient():
    q, k, v, g, ptr = batch()
    out, lse = cel.attention(q, k, v, ptr)
    plain = cel.attention_grad(g, q, k, v, out, lse, ptr)
    ids, table, dx = torch.arange(5, device=DEV), torch.randn(7, 16, device=DEV), torch.randn(5, 16, device=DEV)
    rows, dtable = cel.embed(table, ids), cel.embed_grad(dx, ids, 7)
    for t in (q, k, v, table, dx, g):
        t.requires_grad_()
    for x in ((q, k.detach(), v.detach()), (q.detach(), k, v.detach()), (q.detach(), k.detach(), v)):
        refused(cel.attention, *x, ptr)
        refused(cel.attention_grad, g.detach(), *x, out, lse, ptr)
    x = [t.detach() for t in (q, k, v)]
    refused(cel.attention_grad, g, *x, out, lse, ptr)
    refused(cel.attention_grad, g.detach(), *x, out, lse, ptr, grads=[torch.zeros_like(t).requires_grad_() for t in x])
    refused(cel.embed, table, ids)
    refused(cel.embed_grad, dx, ids, 7)
    with torch.no_grad():
        again, _ = cel.attention(q, k, v, ptr)
        assert torch.equal(again, out)
        assert all(torch.equal(a, b) for a, b in zip(cel.attention_grad(g, q, k, v, out, lse, ptr), plain))
        assert torch.equal(cel.embed(table, ids), rows) and torch.equal(cel.embed_grad(dx, ids, 7), dtable)


def test_inside_a_function_of_torch():
    """The two together as a differentiable operation, which a user makes of them."""

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, ptr):
            out, lse = cel.attention(q, k, v, ptr)
            ctx.save_for_backward(q, k, v, ptr, out, lse)
            return out

        @staticmethod
        def backward(ctx, dout):
            q, k, v, ptr, out, lse = ctx.saved_tensors
            return (*cel.attention_grad(dout, q, k, v, out, lse, ptr), None)

    q, k, v, g, ptr = batch()
    out, lse = cel.attention(q, k, v, ptr)
    plain = cel.attention_grad(g, q, k, v, out, lse, ptr)
    x = [t.clone().requires_grad_() for t in (q, k, v)]
    Attention.apply(*x, ptr).backward(g)
    assert all(torch.equal(t.grad, p) for t, p in zip(x, plain))


def test_tensors_without_dimensions():
    one, ids = torch.zeros((), device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV)
    q, k, v, g, ptr = batch()
    refused(cel.embed, one, ids)
    refused(cel.embed, torch.zeros(4, 8, device=DEV), ids[0])
    refused(cel.embed_grad, one, ids, 4)
    refused(cel.attention, one, one, one, ptr)
    refused(cel.attention, q, k, v, ptr[0])


@pytest.mark.parametrize("T,H,K", [(1, 4, 2), (40, 1, 1), (1, 1, 1)])
def test_strides_that_are_never_taken(T, H, K):
    """One token's or one head's, which torch leaves at anything, also of gradients written in place."""
    x = batch(T, H, K)
    q, k, v, g, ptr = x

    def odd(t):
        row, head, _ = t.stride()
        row, head = row if T > 1 else 3, head if t.shape[1] > 1 else 5
        return torch.zeros(2 * T * t.shape[1] * 64, dtype=t.dtype, device=DEV).as_strided(t.shape, (row, head, 1)).copy_(t)

    out, lse = cel.attention(q, k, v, ptr)
    plain = cel.attention_grad(g, q, k, v, out, lse, ptr)
    into = [odd(torch.zeros_like(t)) for t in (q, k, v)]
    again, lse2 = cel.attention(odd(q), odd(k), odd(v), ptr)
    assert torch.equal(again, out) and torch.equal(lse2, lse)
    got = cel.attention_grad(odd(g), odd(q), odd(k), odd(v), odd(out), lse, ptr, grads=into)
    assert all(a is b for a, b in zip(got, into)) and all(torch.equal(a, b) for a, b in zip(got, plain))


def test_timing_and_capture():
    """Launches that become part of a graph are not timed, and leave no error to a later call."""
    q, k, v, g, ptr = batch()
    ids, table = torch.arange(5, device=DEV), torch.randn(7, 16, device=DEV)

    def step():
        out, lse = cel.attention(q, k, v, ptr)
        return (out, lse, *cel.attention_grad(g, q, k, v, out, lse, ptr), cel.embed(table, ids))

    plain = step()
    torch.cuda.synchronize()
    before = cel.timing(True)
    try:
        cel.kernel_stats(reset=True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        assert cel.kernel_stats() == {}
        for _ in range(3):
            for t in held:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, plain))
            assert all(torch.equal(a, b) for a, b in zip(step(), plain))
        stats = cel.kernel_stats(reset=True)
        assert stats["k_attention"][0] == 3 and stats["k_embed"][0] == 3
    finally:
        cel.timing(before)
