"""Measure a transformer's training step on this GPU, then place it on several.

A placement is only as good as the costs of its graph (Section 4.2.1 of the paper:
run the operations, take their times).  Here the step runs for real: a packed batch of
token sequences through the embedding lookup, blocks of causal attention between two
linear layers, a loss over the vocabulary, and backwards through all of it with
``cel.attention_grad`` and ``cel.embed_grad``.  Every operation is timed where it
stands, and becomes a node with that time and the bytes of its result; the graph goes through
levels, b-levels, CPD-TOPO, clustering, Adjusting Placement and the makespan.

    python examples/measure_and_place.py --blocks 4 --hidden 1024 --heads 16 --devices 4
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2208_00184_amd as cel  # noqa: E402
from workloads import from_edges  # noqa: E402

DEVICE = "cuda:0"


class Recorder:
    """Runs operations one by one; what ran, for how long, on what and into how many bytes."""

    def __init__(self):
        self.names, self.times, self.bytes, self.edges = [], [], [], []
        self.made = {}  # id of a tensor -> (the tensor, the node that made it)

    def source(self, name, t):
        """A tensor that the step starts from (a parameter, the batch): a node without cost."""
        self._node(name, 0, [], [t])
        return t

    def run(self, name, f, *args):
        f(*args)  # the first call may allocate
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        out = f(*args)
        b.record()
        b.synchronize()
        made = out if isinstance(out, tuple) else (out,)
        self._node(name, max(1, round(a.elapsed_time(b) * 1e6)), args, made)
        return out

    def _node(self, name, ns, args, made):
        at = len(self.names)
        self.names.append(name)
        self.times.append(ns)
        self.bytes.append(sum(t.numel() * t.element_size() for t in made))
        for x in args:
            if isinstance(x, torch.Tensor) and id(x) in self.made:
                self.edges.append((self.made[id(x)][1], at))
        for t in made:
            self.made[id(t)] = (t, at)

    def workload(self, devices, bandwidth, latency):
        """The step as the library takes it: times in ns, bytes, devices that hold two thirds of all
        memory each (where there are two, all of it, and a single one twice that)."""
        cap = np.full(devices, 2 * sum(self.bytes) // max(1, min(devices, 3)), np.int64)
        return from_edges(len(self.names), self.edges, self.times, self.bytes, devices, cap, bandwidth, latency,
                          name="measured")


def parameters(blocks, hidden, heads, kv_heads, vocab, seed=0):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)

    def weight(*shape, by):
        return (torch.randn(shape, generator=gen, device=DEVICE) * by).bfloat16()

    d = hidden // heads
    layers = [(weight(hidden, (heads + 2 * kv_heads) * d, by=hidden ** -0.5), weight(hidden, hidden, by=hidden ** -0.5))
              for _ in range(blocks)]
    return weight(vocab, hidden, by=1 / hidden), layers


def training_step(rec, table, layers, ids, targets, seq_ptr, heads, kv_heads):
    """Forward and backward -> (loss, gradient of the table, gradients of the layers)."""
    hidden = table.shape[1]
    d, c = hidden // heads, math.sqrt(hidden)

    def split(fused):
        return tuple(x.view(x.shape[0], -1, d) for x in fused.split([heads * d, kv_heads * d, kv_heads * d], 1))

    def attend_backward(dout, fused, out, lse):
        grad = torch.empty_like(fused)
        cel.attention_grad(dout, *split(fused), out, lse, seq_ptr, grads=split(grad))
        return grad

    def loss_and_gradient(x, table):
        logits = (x @ table.T).float()
        p = torch.softmax(logits, 1)
        loss = -torch.log(p.gather(1, targets[:, None]).clamp_min(1e-30)).mean()
        p.scatter_add_(1, targets[:, None], torch.full_like(p[:, :1], -1.0))
        return loss, (p / len(targets)).bfloat16()

    x = rec.run("embed", lambda t, i: cel.embed(t, i, scale=c), table, ids)
    saved = []
    for n, (w_in, w_out) in enumerate(layers):
        fused = rec.run(f"qkv {n}", torch.mm, x, w_in)
        out, lse = rec.run(f"attention {n}", lambda f: cel.attention(*split(f), seq_ptr), fused)
        flat = out.view(out.shape[0], hidden)
        rec.made[id(flat)] = (flat, rec.made[id(out)][1])
        y = rec.run(f"projection {n}", torch.addmm, x, flat, w_out)
        saved.append((x, fused, out, lse, flat))
        x = y
    loss, dlogits = rec.run("loss", loss_and_gradient, x, table)
    dx = rec.run("loss' rows", torch.mm, dlogits, table)
    out_grad = rec.run("loss' table", lambda g, x: torch.mm(g.T, x), dlogits, x)
    grads = []
    for n in reversed(range(len(layers))):
        w_in, w_out = layers[n]
        x, fused, out, lse, flat = saved[n]
        dflat = rec.run(f"projection' {n}", lambda g, w: torch.mm(g, w.T), dx, w_out)
        dw_out = rec.run(f"projection weight' {n}", lambda f, g: torch.mm(f.T, g), flat, dx)
        dout = dflat.view_as(out)
        rec.made[id(dout)] = (dout, rec.made[id(dflat)][1])
        dfused = rec.run(f"attention' {n}", attend_backward, dout, fused, out, lse)
        dw_in = rec.run(f"qkv weight' {n}", lambda x, g: torch.mm(x.T, g), x, dfused)
        dx = rec.run(f"qkv' {n}", lambda d, g, w: torch.addmm(d, g, w.T), dx, dfused, w_in)
        grads.append((dw_in, dw_out))
    in_grad = rec.run("embed'", lambda g, i: cel.embed_grad(g, i, table.shape[0], scale=c, dtype=torch.float32), dx, ids)
    dtable = rec.run("table'", lambda a, b: a + b, in_grad, out_grad)
    return float(loss), dtable, grads[::-1]


def place(wl):
    """Adjusting Placement of a measured step -> (makespan on all devices, clusters, device of each node)."""
    g, dev = cel.Graph.from_arrays(wl, DEVICE), cel.Devices.from_arrays(wl)
    lev, order_id, level_ptr, L = cel.topo_levels(g)
    bl, tl, prio, _ = cel.blevel(g, dev, lev, level_ptr, order_id, L, want_tlevel=True)
    cid, C, _ = cel.cluster(g, dev, cel.cpd_order(g, bl, tl), 200, -1)
    _, node_dev, _, _ = cel.place(g, dev, cid, C)
    ms, _, _ = cel.makespan(g, dev, prio, lev, level_ptr, L, node_dev)
    return int(ms[0]), C, node_dev


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("blocks", 4), ("hidden", 1024), ("heads", 16), ("kv-heads", 4), ("vocab", 32000), ("tokens", 4096),
                        ("sequences", 9), ("devices", 4), ("bandwidth", 150), ("latency", 2000), ("steps", 3)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--rate", type=float, default=0.5, help="of the plain gradient steps in between")
    a = p.parse_args(argv)
    rng = np.random.default_rng(0)
    cuts = np.sort(rng.choice(np.arange(1, a.tokens), a.sequences - 1, replace=False))
    seq_ptr = torch.tensor(np.concatenate([[0], cuts, [a.tokens]]).astype(np.int32), device=DEVICE)
    words = torch.from_numpy(((a.vocab + 1.0) ** rng.random(a.tokens + 1) - 1).astype(np.int64)).clamp_max(a.vocab - 1)
    ids, targets = words[:-1].to(DEVICE), words[1:].to(DEVICE)
    table, layers = parameters(a.blocks, a.hidden, a.heads, a.kv_heads, a.vocab)
    losses = []
    for _ in range(a.steps):
        rec = Recorder()
        rec.source("table", table), rec.source("ids", ids)
        for n, (w_in, w_out) in enumerate(layers):
            rec.source(f"qkv weight {n}", w_in), rec.source(f"projection weight {n}", w_out)
        loss, dtable, grads = training_step(rec, table, layers, ids, targets, seq_ptr, a.heads, a.kv_heads)
        losses.append(loss)
        table.sub_((a.rate * dtable).to(table.dtype))
        for (w_in, w_out), (g_in, g_out) in zip(layers, grads):
            w_in.sub_(a.rate * g_in), w_out.sub_(a.rate * g_out)
    wl = rec.workload(a.devices, a.bandwidth, a.latency)
    ms, clusters, node_dev = place(wl)
    print(f"loss {' '.join('%.4f' % x for x in losses)}")
    for name, ns in sorted(zip(rec.names, rec.times), key=lambda x: -x[1])[:8]:
        print(f"{name:24s} {ns / 1e3:9.1f} us")
    print(f"{wl.n} operations, {wl.m} tensors, {sum(rec.times) / 1e6:.3f} ms on one device; "
          f"{ms / 1e6:.3f} ms placed on {a.devices} as {clusters} clusters")
    return losses, wl, ms, node_dev


if __name__ == "__main__":
    main()
