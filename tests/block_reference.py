"""Plain 64-bit forms of a block's operations, and how far a result may be from them."""
from __future__ import annotations

import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}  # half a step
SMALLEST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # below normal numbers


def randn(*shape, seed=0, by=1.0, at=0.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * by + at


def within(got, want, error, dtype=None):
    """got is want, rounded once to its type, but for `error` before that."""
    dtype = dtype or got.dtype
    got, error = got.detach().double().cpu(), torch.as_tensor(error, dtype=torch.float64)
    bound = 1.01 * (error + UNIT[dtype] * (want.abs() + error) + SMALLEST[dtype])
    off = (got - want).abs()
    assert bool((off <= bound).all()), (float((off / bound).max()), int((off > bound).sum()))


def philox(c, k, rounds=10):
    """The generator's four words for counters c [4][...] and a key, as published, in Python's integers' range."""
    c = [np.asarray(x, np.uint64) for x in c]
    low, k0, k1 = np.uint64(0xffffffff), k & 0xffffffff, k >> 32 & 0xffffffff
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xd2511f53), c[2] * np.uint64(0xcd9e8d57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9e3779b9) & 0xffffffff, (k1 + 0xbb67ae85) & 0xffffffff
    return c


def kept(rows, columns, p, seed, step, row0=0):
    """-> (which values stay [rows, columns], the factor of those)"""
    blocks = (columns + 7) // 8
    step %= 1 << 64
    c = np.broadcast_arrays(np.arange(blocks, dtype=np.uint64)[None], np.arange(row0, row0 + rows, dtype=np.uint64)[:, None],
                            np.uint64(step & 0xffffffff), np.uint64(step >> 32))
    words = np.stack(philox(c, seed % (1 << 64)), 2)
    bits = np.stack([words & np.uint64(0xffff), words >> np.uint64(16)], 3).reshape(rows, 8 * blocks)[:, :columns]
    least = int(p * 65536 + 0.5)
    return torch.from_numpy(bits >= least), (0.0 if least == 65536 else 1.0 / (1.0 - least / 65536.0))


def turn(x, positions, freqs, axes=None, pairs=False, back=False):
    """-> (x turned, the size of each value's pair)"""
    x, P = x.detach().double().cpu(), freqs.numel()
    pos = positions.cpu().double()
    pos = pos[None] if pos.dim() == 1 else pos
    axis = torch.zeros(P, dtype=torch.int64) if axes is None else axes.long().cpu()
    there = (axis >= 0) & (axis < pos.shape[0])
    a = pos[axis.clamp(0, pos.shape[0] - 1)].T * freqs.double().cpu() * there
    a = (-a if back else a)[:, None]
    u, v = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if pairs else (x[..., :P], x[..., P:2 * P])
    one, two, size = u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin(), u.abs() + v.abs()
    out, sizes = x.clone(), torch.zeros_like(x)
    if pairs:
        out[..., 0:2 * P:2], out[..., 1:2 * P:2] = one, two
        sizes[..., 0:2 * P:2] = sizes[..., 1:2 * P:2] = size
    else:
        out[..., :P], out[..., P:2 * P] = one, two
        sizes[..., :P] = sizes[..., P:2 * P] = size
    return out, sizes


U = 2.0 ** -24
ADDS = 48  # additions that a row's sum passes through at most: 16 in a lane, 6 over lanes, 16 over waves, and what is done to it


class Unit:
    """norm(v) of rows in 64 bits from values with errors e: the value, its factor r, and the value's error
    in 32 bits.  A sum of squares is off by ADDS u of itself, r by half of that and its own three roundings; a mean by
    ADDS u of the mean size; and an error e moves the value by r (e - [mean e] - V mean(V e))."""

    def __init__(self, v, eps, center, e=0.0):
        e = torch.as_tensor(e, dtype=torch.float64).expand(v.shape)
        w = v - v.mean(1, keepdim=True) if center else v
        self.r = 1.0 / ((w * w).mean(1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32))).sqrt()
        self.v = V = w * self.r
        e = e + (U * w.abs() + ADDS * U * v.abs().mean(1, keepdim=True) if center else 0.0)
        self.er = (ADDS / 2 + 4) * U  # of r
        self.e = (self.er + 2 * U) * V.abs() + self.r * (e + e.mean(1, keepdim=True) * center + V.abs() * (V.abs() * e).mean(1, keepdim=True))
        self.center = center

    def back(self, g, eg):
        """The gradient of v at g, known to eg -> (gradient, error)"""
        V, r, m = self.v, self.r, lambda x: x.mean(1, keepdim=True)
        c, b = m(g * V), m(g) * self.center
        ec = m(g.abs() * self.e + eg * V.abs()) + ADDS * U * m((g * V).abs())
        eb = (m(eg) + ADDS * U * m(g.abs())) * self.center
        size = g.abs() + b.abs() + (V * c).abs()
        return r * (g - b - V * c), r * ((self.er + 4 * U) * size + eg + eb + self.e * c.abs() + V.abs() * ec)


def gates(gate, seq_ptr, rows):
    """-> (each row's gate [rows, h], each row's sequence or -1)"""
    gate = gate.double().cpu()
    if seq_ptr is None:
        return gate.expand(rows, -1), torch.zeros(rows, dtype=torch.int64)
    ptr, of = seq_ptr.cpu().tolist(), torch.full((rows,), -1, dtype=torch.int64)
    for s, (a, b) in enumerate(zip(ptr, ptr[1:])):
        of[a:b] = s
    return torch.where(of[:, None] >= 0, gate[of.clamp(min=0)] if len(gate) else torch.zeros(rows, gate.shape[1]).double(), 0.0), of


class Joint:
    """residual_norm and its gradient in 64 bits, each with its error."""

    def __init__(self, pre, post=None, gate=None, seq_ptr=None, pre_bias=None, post_bias=None, scale=1.0, p=0.0, seed=0, step=0,
                 eps=1e-6, center=False):
        up = lambda t: None if t is None else t.detach().double().cpu()  # noqa: E731
        self.pre, self.post, self.pre_bias, self.post_bias = up(pre), up(post), up(pre_bias), up(post_bias)
        self.gate, self.seq_ptr, self.scale = gate, seq_ptr, float(torch.tensor(scale, dtype=torch.float32))
        self.p, self.seed, self.step, self.eps, self.center = p, seed, int(step), eps, center

    def drop(self, x, e):
        if not int(self.p * 65536 + 0.5):
            return x, e
        keep, by = kept(*x.shape, self.p, self.seed, self.step)
        return torch.where(keep, x * by, 0.0), torch.where(keep, e * by + 2 * U * (x * by).abs(), 0.0)

    @staticmethod
    def affine(unit, w, b):
        n = unit.v * w
        e = unit.e * w.abs() + 2 * U * n.abs()
        return (n, e) if b is None else (n + b, e + U * (n + b).abs())

    def branch(self, f):
        """-> (norm(f) or None, drop(n), its error)"""
        f = f.double().cpu()
        unit, n, e = None, f, torch.zeros_like(f)
        if self.post is not None:
            unit = Unit(f, self.eps, self.center)
            n, e = self.affine(unit, self.post, self.post_bias)
        return (unit, *self.drop(n, e))

    def forward(self, f, x):
        y, e = x.double().cpu(), torch.zeros(x.shape, dtype=torch.float64)
        if f is not None:
            _, n, en = self.branch(f)
            if self.gate is not None:
                g, of = gates(self.gate, self.seq_ptr, len(x))
                n, en = torch.where(of[:, None] >= 0, n * g, 0.0), torch.where(of[:, None] >= 0, en * g.abs() + U * (n * g).abs(), 0.0)
            e = en + 2 * U * ((y * self.scale).abs() + n.abs())
            y = y * self.scale + n
        if self.pre is None:
            return (y, e), None
        return (y, e), self.affine(Unit(y, self.eps, self.center, e), self.pre, self.pre_bias)

    def backward(self, dy, dz, f, y):
        """-> {name: (gradient, error)}"""
        out, T = {}, len(y)
        total = lambda x, e: (x.sum(0), e.sum(0) + (T + 4) * U * x.abs().sum(0))  # noqa: E731
        t = torch.zeros(y.shape, dtype=torch.float64) if dy is None else dy.double().cpu()
        et = torch.zeros_like(t)
        if self.pre is not None:
            unit, dz = Unit(y.double().cpu(), self.eps, self.center), dz.double().cpu()
            g, e = unit.back(dz * self.pre, U * (dz * self.pre).abs())
            t, et = t + g, e + U * (t + g).abs()
            out["pre"] = total(dz * unit.v, dz.abs() * unit.e)
            if self.pre_bias is not None:
                out["pre_bias"] = total(dz, 0 * dz)
        out["dx"] = t * self.scale, abs(self.scale) * et + U * (t * self.scale).abs()
        if f is None:
            return out
        unit, n, en = self.branch(f)
        e, ee = t, et
        if self.gate is not None:
            g, of = gates(self.gate, self.seq_ptr, T)
            per, eper = t * n, et * n.abs() + t.abs() * en
            if self.seq_ptr is None:
                out["gate"] = total(per, eper)
            else:
                there, S = of >= 0, len(self.gate)
                add = lambda x: torch.zeros(S, x.shape[1], dtype=torch.float64).index_add_(0, of[there], x[there])  # noqa: E731
                out["gate"] = add(per), add(eper + (T + 4) * U * per.abs())
            live = of[:, None] >= 0
            e, ee = torch.where(live, t * g, 0.0), torch.where(live, et * g.abs() + U * (t * g).abs(), 0.0)
        e, ee = self.drop(e, ee)
        if self.post is not None:
            live = torch.ones(T, 1, dtype=torch.bool) if self.gate is None else live
            out["post"] = total(torch.where(live, e * unit.v, 0.0), torch.where(live, ee * unit.v.abs() + e.abs() * unit.e, 0.0))
            if self.post_bias is not None:
                out["post_bias"] = total(e, ee)
            g, eg = e * self.post, ee * self.post.abs() + U * (e * self.post).abs()
            e, ee = (torch.where(live, x, 0.0) for x in unit.back(g, eg))
        out["df"] = e, ee
        return out
