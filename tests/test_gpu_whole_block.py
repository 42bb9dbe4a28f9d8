"""The operations of a whole decoder block together, as the example's training step uses them: its gradients
against torch's own of the same step in 64 bits, with the same masks."""
from __future__ import annotations

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

from block_reference import kept  # noqa: E402

DEV = "cuda:0"
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "measure_and_place.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("measure_and_place", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def attend(q, k, v, lengths, sources, causal):
    """[T, H, d] over [U, K, d] in 64 bits."""
    (T, H, d), K = q.shape, k.shape[1]
    out, at, k_at = [], 0, 0
    for L, M in zip(lengths, sources):
        Q, KK, V = (x.transpose(0, 1) for x in (q[at:at + L], k[k_at:k_at + M].repeat_interleave(H // K, 1), v[k_at:k_at + M].repeat_interleave(H // K, 1)))
        s = Q @ KK.transpose(1, 2) * d ** -0.5
        if causal:
            s = s.masked_fill(torch.ones(L, L, dtype=torch.bool).triu(1), -1e300)
        out.append((torch.softmax(s, 2) @ V).transpose(0, 1))
        at, k_at = at + L, k_at + M
    return torch.cat(out)


def plain_step(E, freqs, last, layers, ids, targets, states, lengths, sources, positions, H, K, drop, step):
    hidden, T = E.shape[1], len(ids)
    d = hidden // H

    def norm(v, w):
        return v / (v.square().mean(1, keepdim=True) + float(torch.tensor(1e-6))).sqrt() * w

    def dropped(v, seed):
        keep, by = kept(*v.shape, drop, seed, step)
        return torch.where(keep, v * by, 0.0)

    def turned(x):
        a = (positions.double()[:, None] * freqs)[:, None]
        u, v = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()], 2)

    x = E[ids] * hidden ** 0.5
    for n, w in enumerate(layers):
        for j, joint in enumerate(("self", "cross", "inner")):
            z = norm(x, w[f"pre {joint}"])
            if joint == "self":
                q, k, v = (t.reshape(T, -1, d) for t in (z @ w["qkv"]).split([H * d, K * d, K * d], 1))
                f = attend(turned(q), turned(k), v, lengths, lengths, True).reshape(T, hidden) @ w["out"]
            elif joint == "cross":
                k, v = (t.reshape(len(states), K, d) for t in (states @ w["states"]).split([K * d, K * d], 1))
                f = attend((z @ w["query"]).view(T, H, d), k, v, lengths, sources, False).reshape(T, hidden) @ w["cross"]
            else:
                f = dropped(torch.nn.functional.silu(z @ w["up"]), 1000 + n) @ w["down"]
            x = x + w[f"gate {joint}"] * dropped(norm(f, w[f"post {joint}"]), 3 * n + j)
    return torch.nn.functional.cross_entropy(norm(x, last) @ E.T, targets)


def test_gradients_of_a_whole_step(example):
    """A gradient of a weight of each kind.  Results between the operations are bfloat16: on the way forward and back
    through two blocks some 3 x 5 x 2 roundings each way, independent ones, of at most 2^-8 (a third of which is
    the mean error): sqrt(60) 2^-8 / 2 of the norm, twice that is allowed."""
    H, K, h, V, T, U = 4, 2, 64, 200, 150, 110
    lengths, sources = [90, 60], [30, 80]
    table, freqs, last, layers = example.whole_parameters(2, h, H, K, V, seed=3)
    gen = torch.Generator().manual_seed(1)
    ids = torch.randint(0, V, (T,), generator=gen)
    states = torch.randn(U, h, generator=gen).bfloat16()
    positions = torch.cat([torch.arange(n) for n in lengths])
    ptr, state_ptr = (torch.tensor([0, x[0], sum(x)], dtype=torch.int32, device=DEV) for x in (lengths, sources))
    step = torch.tensor([7], dtype=torch.int64, device=DEV)
    loss, dtable, dlast, dstates, grads = example.whole_step(
        example.Recorder(), table, freqs, last, layers, ids.to(DEV), ids.roll(-1).to(DEV), states.to(DEV), ptr, state_ptr,
        positions.to(DEV), H, K, 0.2, step)
    up = lambda t: t.double().cpu().requires_grad_()  # noqa: E731
    E, l, s, w = up(table), up(last), up(states), [{n: up(t) for n, t in layer.items()} for layer in layers]
    want = plain_step(E, freqs.cpu(), l, w, ids, ids.roll(-1), s, lengths, sources, positions, H, K, 0.2, 7)
    want.backward()
    bound = 60 ** 0.5 * 2.0 ** -8
    assert abs(loss - float(want)) <= bound * float(want)
    pairs = [("table", dtable, E), ("last", dlast, l), ("states", dstates, s)]
    pairs += [(f"{name} {n}", grads[n][name], w[n][name]) for n in range(2) for name in w[n]]
    off = {name: float((got.double().cpu() - t.grad).norm() / t.grad.norm()) for name, got, t in pairs}
    assert max(off.values()) <= bound, off


def test_the_step_runs_and_is_placed(example):
    losses, wl, ms, node_dev = example.main(
        "--whole --blocks 2 --hidden 128 --heads 4 --kv-heads 2 --vocab 500 --tokens 300 --states 200 --sequences 5 --devices 3 --steps 2".split())
    assert all(x == x and x < 100 for x in losses)
    # table, ids, states and 16 weights a block; embed and norm; 5, 5 and 4 operations of a block's parts; the loss and its two;
    # backwards 6, 8 and 6, then norm, embed and table
    assert wl.n == 3 + 2 * 16 + 2 + 2 * 14 + 3 + 2 * 20 + 3
    assert node_dev.shape[0] == wl.n and int(node_dev.max()) < 3 and int(wl.w.sum()) // 3 <= ms


def test_every_source_is_read_by_an_operation(example):
    """The vectors of the norms and gates among them: whoever reads one has an edge from it, forward and backward."""
    _, wl, _, _ = example.main(
        "--whole --blocks 2 --hidden 128 --heads 4 --kv-heads 2 --vocab 500 --tokens 300 --states 200 --sequences 5 --devices 3 --steps 1".split())
    src, _ = wl.edges()
    readers = [int((src == n).sum()) for n in range(3 + 2 * 16)]
    assert min(readers) >= 1 and min(readers[3:]) >= 2, readers  # each weight and vector forward and backward
