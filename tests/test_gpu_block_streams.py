"""A block's operations on other streams than the default one, several at once, and captured into graphs whose
replays share them: every result has the bits of a call by itself."""
from __future__ import annotations

import threading

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402
from block_reference import randn  # noqa: E402

DEV = "cuda:0"


def ptr(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def work(seed, h=8192):
    """-> a function that runs every operation once and returns all results"""
    T, H, d = 96, 8, 64
    f, x, dy, dz = (randn(T, h, seed=10 * seed + i).bfloat16().to(DEV) for i in range(4))
    pre, post, bias, post_bias = (randn(h, seed=10 * seed + i, at=1.0).to(DEV) for i in range(4, 8))
    gate, seqs = randn(3, h, seed=seed).to(DEV), ptr(0, 30, 31, 90)
    q, k, v, g = (randn(n, m, d, seed=seed + i).bfloat16().to(DEV) for i, (n, m) in enumerate(((700, H), (3000, 2), (3000, 2), (700, H))))
    few = q[:5].contiguous(), ptr(0, 2, 5), ptr(0, 1000, 3000)
    pos, freqs = torch.arange(700, device=DEV), torch.rand(32, device=DEV)
    how = dict(post=post, gate=gate, seq_ptr=seqs, pre_bias=bias, post_bias=post_bias, p=0.2, seed=seed, center=bool(seed % 2))

    def run():
        y, z = cel.residual_norm(f, x, pre, **how)
        dx, df, grads = cel.residual_norm_grad(dy, dz, f, y, pre, **how)
        out, lse = cel.cross_attention(q, k, v, ptrs[0], ptrs[1])
        dq, dk, dv = cel.cross_attention_grad(g, q, k, v, out, lse, *ptrs)
        one = cel.cross_attention(few[0], k, v, *few[1:])
        return [y, z, dx, df, *grads.values(), out, lse, dq, dk, dv, *one, cel.rotary(q, pos, freqs), cel.rotary_grad(q, pos, freqs),
                cel.dropout(x, 0.3, seed)]

    ptrs = ptr(0, 300, 320, 700), ptr(0, 100, 2500, 3000)
    return run


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_on_streams_at_once():
    runs = [work(s) for s in range(3)]
    want = [r() for r in runs]
    torch.cuda.synchronize()
    errors = []

    def thread(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(5):
                    got = runs[i]()
                    s.synchronize()
                    assert same(got, want[i])
        except BaseException as e:  # noqa: BLE001 (reported by the test's thread)
            errors.append(repr(e))

    ts = [threading.Thread(target=thread, args=(i,)) for i in range(3)]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    assert not errors, errors


def test_two_graphs():
    """Two captured passes, replayed in turn, with eager work between."""
    runs = [work(s) for s in (5, 6)]
    want = [r() for r in runs]
    torch.cuda.synchronize()
    graphs, held = [], []
    for r in runs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.append(r())
        graphs.append(graph)
    for turn in range(3):
        for t in held[0] + held[1]:
            t.zero_()
        for i in (0, 1) if turn % 2 else (1, 0):
            graphs[i].replay()
        if turn == 1:
            assert same(runs[0](), want[0])
        torch.cuda.synchronize()
        assert same(held[0], want[0]) and same(held[1], want[1])
