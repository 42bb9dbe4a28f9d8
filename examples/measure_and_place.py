"""Measure a transformer's training step on this GPU, then place it on several.

A placement is only as good as the costs of its graph (Section 4.2.1 of the paper:
run the operations, take their times).  Here the step runs for real: a packed batch of
token sequences through the embedding lookup, blocks of causal attention between two
linear layers, a loss over the vocabulary, and backwards through all of it with
``cel.attention_grad`` and ``cel.embed_grad``.  Every operation is timed where it
stands, and becomes a node with that time and the bytes of its result; the graph goes through
levels, b-levels, CPD-TOPO, clustering, Adjusting Placement and the makespan.

    python examples/measure_and_place.py --blocks 4 --hidden 1024 --heads 16 --devices 4

With ``--whole`` a block is a translator's decoder block, whole: rotary positions and causal attention, attention
to an encoder's states, a layer inside with dropout, and around each of the three a norm before, a norm behind with
a gate, dropout and the residual stream (``cel.rotary``, ``cel.cross_attention``, ``cel.dropout``, ``cel.residual_norm``).
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

    def view(self, t, of):
        """t, a view of a tensor that an operation made."""
        self.made[id(t)] = (t, self.made[id(of)][1])
        return t

    def _node(self, name, ns, args, made):
        at = len(self.names)
        self.names.append(name)
        self.times.append(ns)
        self.bytes.append(sum(t.numel() * t.element_size() for t in made if t is not None))
        for x in args:
            if isinstance(x, torch.Tensor) and id(x) in self.made:
                self.edges.append((self.made[id(x)][1], at))
        for t in made:
            if t is not None:
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


JOINTS = ("self", "cross", "inner")  # the three parts of a whole block


def whole_parameters(blocks, hidden, heads, kv_heads, vocab, seed=0):
    """-> (table, rotary frequencies, the last norm, weights of each block by name)"""
    gen = torch.Generator(device=DEVICE).manual_seed(seed)

    def weight(*shape):
        return (torch.randn(shape, generator=gen, device=DEVICE) * shape[0] ** -0.5).bfloat16()

    def vector(at, by=0.05):
        return at + by * torch.randn(hidden, generator=gen, device=DEVICE)

    d = hidden // heads
    layers = []
    for _ in range(blocks):
        layer = dict(qkv=weight(hidden, (heads + 2 * kv_heads) * d), out=weight(hidden, hidden), query=weight(hidden, hidden),
                     states=weight(hidden, 2 * kv_heads * d), cross=weight(hidden, hidden), up=weight(hidden, 4 * hidden),
                     down=weight(4 * hidden, hidden))
        for joint in JOINTS:
            layer.update({f"pre {joint}": vector(1.0), f"post {joint}": vector(1.0), f"gate {joint}": vector(0.5)})
        layers.append(layer)
    freqs = 10000.0 ** (-torch.arange(d // 2, device=DEVICE, dtype=torch.float64) / (d // 2))
    return (torch.randn(vocab, hidden, generator=gen, device=DEVICE) / hidden).bfloat16(), freqs, vector(1.0), layers


def whole_step(rec, table, freqs, last, layers, ids, targets, states, seq_ptr, state_ptr, positions, heads, kv_heads, drop, step):
    """Forward and backward -> (loss, gradients of table, last norm, states, and of each block's weights by name)."""
    (hidden, T), mm = (table.shape[1], len(ids)), torch.mm
    d, H, K, c = hidden // heads, heads, kv_heads, math.sqrt(hidden)

    def tmm(a, b):
        return mm(a.T, b)

    def mmt(a, b):
        return mm(a, b.T)

    def in_order(dx, df, g):
        return dx, df, g["pre"], g.get("post"), g.get("gate")

    def join(n, joint):  # how part `joint` of block n ends: the mask's seed is the joint's own
        return dict(p=drop, seed=3 * n + JOINTS.index(joint), step=step)

    def split(fused, *counts):  # heads side by side, of one projection
        return tuple(x.view(fused.shape[0], -1, d) for x in fused.split([k * d for k in counts], 1))

    x = rec.run("embed", lambda t, i: cel.embed(t, i, scale=c), table, ids)
    names = [(n, j) for n in range(len(layers)) for j in JOINTS]
    following = [layers[n][f"pre {j}"] for n, j in names[1:]] + [last]  # the norm behind each part
    x, z = rec.run("norm", lambda x, w: cel.residual_norm(None, x, w), x, layers[0]["pre self"])
    saved, first = [], x
    for (n, joint), after in zip(names, following):
        w = layers[n]
        if joint == "self":
            fused = rec.run(f"qkv {n}", mm, z, w["qkv"])
            turned = rec.run(f"rotary {n}", lambda f: cel.rotary(split(f, H + K, K)[0], positions, freqs), fused)
            out, lse = rec.run(f"attention {n}", lambda t, f: cel.attention(t[:, :H], t[:, H:], split(f, H + K, K)[1], seq_ptr), turned, fused)
            kept = z, fused, turned, out, lse
            inner = rec.view(out.view(T, hidden), out)
            f = rec.run(f"projection {n}", mm, inner, w["out"])
        elif joint == "cross":
            q = rec.run(f"query {n}", mm, z, w["query"])
            kv = rec.run(f"states {n}", mm, states, w["states"])
            out, lse = rec.run(f"cross attention {n}", lambda q, kv: cel.cross_attention(q.view(T, H, d), *split(kv, K, K), seq_ptr, state_ptr), q, kv)
            kept = z, q, kv, out, lse
            inner = rec.view(out.view(T, hidden), out)
            f = rec.run(f"cross projection {n}", mm, inner, w["cross"])
        else:
            u = rec.run(f"up {n}", mm, z, w["up"])
            inner = rec.run(f"dropout {n}", lambda u: cel.dropout(torch.nn.functional.silu(u), drop, 1000 + n, step=step), u)
            kept = z, u
            f = rec.run(f"down {n}", mm, inner, w["down"])
        x, z = rec.run(f"joint {joint} {n}", lambda f, x, after, post, gate: cel.residual_norm(f, x, after, post=post, gate=gate, **join(n, joint)),
                       f, x, after, w[f"post {joint}"], w[f"gate {joint}"])
        saved.append((kept, inner, f, x))

    def loss_and_gradient(z, table):
        p = torch.softmax((z @ table.T).float(), 1)
        loss = -torch.log(p.gather(1, targets[:, None]).clamp_min(1e-30)).mean()
        p.scatter_add_(1, targets[:, None], torch.full_like(p[:, :1], -1.0))
        return loss, (p / T).bfloat16()

    loss, dlogits = rec.run("loss", loss_and_gradient, z, table)
    dz, out_grad = rec.run("loss' rows", mm, dlogits, table), rec.run("loss' table", tmm, dlogits, z)
    dx, dstates, grads, vectors = None, torch.zeros_like(states), [{} for _ in layers], {}
    for (n, joint), after, (kept, inner, f, y) in reversed(list(zip(names, following, saved))):
        w, g = layers[n], grads[n]
        dx, df, dpre, g[f"post {joint}"], g[f"gate {joint}"] = rec.run(
            f"joint' {joint} {n}", lambda *a: in_order(*cel.residual_norm_grad(*a, **join(n, joint))), dx, dz, f, y, after,
            w[f"post {joint}"], w[f"gate {joint}"])
        vectors[n, joint] = dpre  # of the part behind this one
        out_weight, in_weight = dict(self=("out", "qkv"), cross=("cross", "query"), inner=("down", "up"))[joint]
        g[out_weight] = rec.run(f"{out_weight} weight' {n}", tmm, inner, df)
        dinner = rec.run(f"{out_weight}' {n}", mmt, df, w[out_weight])
        if joint == "self":
            z, fused, turned, out, lse = kept

            def attend(dout, turned, fused, out, lse):
                dfused = torch.empty_like(fused)
                q, k, v = split(dfused, H, K, K)
                cel.attention_grad(dout.view(T, H, d), turned[:, :H], turned[:, H:], split(fused, H + K, K)[1], out, lse, seq_ptr, grads=(q, k, v))
                both = split(dfused, H + K, K)[0]
                cel.rotary_grad(both, positions, freqs, out=both)
                return dfused

            din = rec.run(f"attention' {n}", attend, dinner, turned, fused, out, lse)
        elif joint == "cross":
            z, q, kv, out, lse = kept

            def attend_states(dout, q, kv, out, lse):
                dq, dkv = torch.empty_like(q), torch.empty_like(kv)
                k, v = split(kv, K, K)
                cel.cross_attention_grad(dout.view(T, H, d), q.view(T, H, d), k, v, out, lse, seq_ptr, state_ptr,
                                         grads=(dq.view(T, H, d), *split(dkv, K, K)))
                return dq, dkv

            din, dkv = rec.run(f"cross attention' {n}", attend_states, dinner, q, kv, out, lse)
            g["states"] = rec.run(f"states weight' {n}", tmm, states, dkv)
            dstates = rec.run(f"states' {n}", lambda a, g, w: torch.addmm(a, g, w.T), dstates, dkv, w["states"])
        else:
            z, u = kept
            din = rec.run(f"dropout' {n}", lambda g, u: torch.ops.aten.silu_backward(cel.dropout(g, drop, 1000 + n, step=step), u), dinner, u)
        g[in_weight] = rec.run(f"{in_weight} weight' {n}", tmm, z, din)
        dz = rec.run(f"{in_weight}' {n}", mmt, din, w[in_weight])
    dx, _, dpre, _, _ = rec.run("norm'", lambda dx, dz, x, w: in_order(*cel.residual_norm_grad(dx, dz, None, x, w)), dx, dz, first, layers[0]["pre self"])
    for (n, joint), before in zip(names, [dpre] + [vectors[k] for k in names[:-1]]):
        grads[n][f"pre {joint}"] = before
    in_grad = rec.run("embed'", lambda g, i: cel.embed_grad(g, i, table.shape[0], scale=c, dtype=torch.float32), dx, ids)
    return float(loss), rec.run("table'", lambda a, b: a + b, in_grad, out_grad), vectors[names[-1]], dstates, grads


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
    p.add_argument("--rate", type=float, help="of the plain gradient steps in between (0.5, whole blocks 0.02)")
    p.add_argument("--whole", action="store_true", help="whole decoder blocks, over an encoder's states")
    p.add_argument("--states", type=int, default=3000, help="an encoder's, of all sequences together")
    p.add_argument("--drop", type=float, default=0.1)
    a = p.parse_args(argv)
    rate = a.rate if a.rate is not None else 0.02 if a.whole else 0.5
    rng = np.random.default_rng(0)
    cuts = np.sort(rng.choice(np.arange(1, a.tokens), a.sequences - 1, replace=False))
    seq_ptr = torch.tensor(np.concatenate([[0], cuts, [a.tokens]]).astype(np.int32), device=DEVICE)
    words = torch.from_numpy(((a.vocab + 1.0) ** rng.random(a.tokens + 1) - 1).astype(np.int64)).clamp_max(a.vocab - 1)
    ids, targets = words[:-1].to(DEVICE), words[1:].to(DEVICE)
    losses = []
    if a.whole:
        table, freqs, last, layers = whole_parameters(a.blocks, a.hidden, a.heads, a.kv_heads, a.vocab)
        cuts = np.sort(rng.choice(np.arange(1, a.states), a.sequences - 1, replace=False))
        state_ptr = torch.tensor(np.concatenate([[0], cuts, [a.states]]).astype(np.int32), device=DEVICE)
        states = torch.randn(a.states, a.hidden, device=DEVICE, generator=torch.Generator(device=DEVICE).manual_seed(1)).bfloat16()
        starts = torch.repeat_interleave(seq_ptr[:-1], torch.diff(seq_ptr))
        positions = torch.arange(a.tokens, device=DEVICE, dtype=torch.int32) - starts
        step = torch.zeros(1, dtype=torch.int64, device=DEVICE)
    else:
        table, layers = parameters(a.blocks, a.hidden, a.heads, a.kv_heads, a.vocab)
    for _ in range(a.steps):
        rec = Recorder()
        if a.whole:
            rec.source("table", table), rec.source("ids", ids), rec.source("states", states)
            for n, layer in enumerate(layers):
                for name, w in layer.items():
                    rec.source(f"{name} {n}", w)
            loss, dtable, dlast, _, grads = whole_step(rec, table, freqs, last, layers, ids, targets, states, seq_ptr, state_ptr, positions,
                                                       a.heads, a.kv_heads, a.drop, step)
            losses.append(loss)
            table.sub_((rate * dtable).to(table.dtype))
            last.sub_(rate * dlast)
            for layer, g in zip(layers, grads):
                for name, w in layer.items():
                    w.sub_((rate * g[name]).to(w.dtype))
            step.add_(1)
            continue
        rec.source("table", table), rec.source("ids", ids)
        for n, (w_in, w_out) in enumerate(layers):
            rec.source(f"qkv weight {n}", w_in), rec.source(f"projection weight {n}", w_out)
        loss, dtable, grads = training_step(rec, table, layers, ids, targets, seq_ptr, a.heads, a.kv_heads)
        losses.append(loss)
        table.sub_((rate * dtable).to(table.dtype))
        for (w_in, w_out), (g_in, g_out) in zip(layers, grads):
            w_in.sub_(rate * g_in), w_out.sub_(rate * g_out)
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
