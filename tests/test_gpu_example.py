"""The example that measures a training step and places it, at a small size."""
from __future__ import annotations

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "measure_and_place.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("measure_and_place", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_step_learns_and_is_placed(example):
    losses, wl, ms, node_dev = example.main(
        "--blocks 2 --hidden 128 --heads 4 --kv-heads 2 --vocab 500 --tokens 300 --sequences 5 --devices 3 --steps 4".split())
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
    assert wl.n == 2 + 2 * 2 + 1 + 3 * 2 + 3 + 5 * 2 + 2
    work = int(wl.w.sum())
    assert node_dev.shape[0] == wl.n and int(node_dev.max()) < 3
    assert work // 3 <= ms  # three devices cannot do more than a third each


def test_the_steps_gradients_are_the_losss(example):
    """The step's gradient of a weight of each kind against torch's own over the same
    operations in 32 bits (bfloat16 results in between: eight roundings of 2^-8 on the way)."""
    H, K, h, V, T = 4, 2, 64, 200, 150
    d = h // H
    table, layers = example.parameters(1, h, H, K, V, seed=3)
    ids = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(1)).to("cuda:0")
    targets = ids.roll(-1)
    ptr = torch.tensor([0, 90, 150], dtype=torch.int32, device="cuda:0")
    loss, dtable, grads = example.training_step(example.Recorder(), table, layers, ids, targets, ptr, H, K)
    E, A, B = (t.float().cpu().requires_grad_() for t in (table, *layers[0]))
    x = E[ids.cpu()] * h ** 0.5
    q, k, v = (x @ A).split([H * d, K * d, K * d], 1)
    out = torch.zeros(T, H, d)
    for r in (slice(0, 90), slice(90, 150)):
        n = r.stop - r.start
        for i in range(H):
            cols, kv = slice(i * d, i * d + d), slice(i // 2 * d, i // 2 * d + d)
            s = (q[r, cols] @ k[r, kv].T * d ** -0.5).masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -1e30)
            out[r, i] = torch.softmax(s, 1) @ v[r, kv]
    y = x + out.reshape(T, h) @ B
    want = torch.nn.functional.cross_entropy(y @ E.T, targets.cpu())
    want.backward()
    assert abs(loss - float(want)) <= 8 * 2.0 ** -8 * float(want)
    for got, t in ((dtable, E), (grads[0][0], A), (grads[0][1], B)):
        assert float((got.float().cpu() - t.grad).norm()) <= 8 * 2.0 ** -8 * float(t.grad.norm())
