"""Attention and its gradient in 64 bits, with how far each element of a result may be off.

The bounds follow the roundings of cel.attention and cel.attention_grad, with u the unit
round-off of the rows' type (2^-8 bfloat16, 2^-11 float16).  Roundings of different
values are taken as independent: a sum of n rounded terms x is off by at most 6 u times the root of
the sum of x^2 (each is off by at most u |x|, so this holds for any signs up to 36 terms, and is more than ten
standard deviations of independent ones beyond).

- p is rounded as the operand of out and dv, out once more, and D = <dout, out> carries both;
- ds = p (dp - D) is rounded as the operand of dq and dk, which carry D's error too: dq the
  same for all of a row's keys, dk one of each row's;
- all else is 32 bit: scores and dp off by 6 sqrt(d) 2^-24 of the sum of their products' sizes,
  sums of n products by 6 sqrt(n) 2^-24, exponentials and logarithms by 2^-20;
- float16 has no values below 2^-24, half of which an operand or a result may be off: a weight
  of out stands relative to its row's largest, one of dv is 2^8 times p, ds at least 2^8 where its row's
  (dq) or its key's (dk) largest is.
5 % are added for products of errors.
"""
from __future__ import annotations

import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _norm(x, dim):
    return x.square().sum(dim).sqrt()


def definition(q, k, v, dout, lengths, first=0, scale=None, wide=None):
    """-> {name: (value, bound)} for out, lse, dq, dk, dv, on the CPU in 64 bits.  wide: the tokens
    [T] whose D is a sum in 32 bits and carries no rounding of out (none by default)."""
    dtype, u = q.dtype, UNIT[q.dtype]
    half = dtype == torch.float16
    q, k, v, dout = (x.double().cpu() for x in (q, k, v, dout))
    T, H, d = q.shape
    K, c = k.shape[1], d ** -0.5 if scale is None else scale
    least = 2.0 ** -25 if half else 0.0
    r32 = 6 * math.sqrt(d) * 2.0 ** -24

    def pair(*shape, fill=0.0):
        return torch.full(shape, fill, dtype=torch.float64), torch.zeros(shape, dtype=torch.float64)

    out, b_out = pair(T, H, d)
    lse, b_lse = pair(H, T, fill=-math.inf)
    (dq, b_dq), (dk, b_dk), (dv, b_dv) = pair(T, H, d), pair(T, K, d), pair(T, K, d)
    at = first
    for L in lengths:
        r = slice(at, at + L)
        at += L
        if not L:
            continue
        Q, G = q[r].transpose(0, 1), dout[r].transpose(0, 1)  # [H, L, d]
        KK, V = (x[r].transpose(0, 1).repeat_interleave(H // K, 0) for x in (k, v))

        def over(a, b):  # sum over the middle axis of a [H, L, L] and b [H, L, d]
            return a @ b

        seen = torch.ones(L, L, dtype=torch.bool).tril()
        s = (Q @ KK.transpose(1, 2) * c).masked_fill(~seen, -math.inf)
        z = torch.logsumexp(s, 2, keepdim=True)
        p = torch.exp(s - z)
        sizes = (Q.abs() @ KK.abs().transpose(1, 2)) * c
        off_s = (r32 * sizes).masked_fill(~seen, 0.0).amax((1, 2), keepdim=True)  # of a score, in each head
        w = 2 * off_s + 2.0 ** -20 + 2.0 ** -22 * z.abs() + 6 * math.sqrt(L * H / K) * 2.0 ** -24  # of p and sums, [H, L, 1]
        w = w.amax(1, keepdim=True)
        pv, pv2 = over(p, V.abs()), over(p ** 2, V ** 2).sqrt()
        o = over(p, V)
        e_o = 6 * u * pv2 + w * pv + u * o.abs() + least
        if half:
            e_o = e_o + 2.0 ** -25 * p.amax(2, keepdim=True) * over(seen.double().expand_as(p), V.abs())
        out[r], b_out[r] = o.transpose(0, 1), e_o.transpose(0, 1)
        lse[:, r], b_lse[:, r] = z[..., 0], (w + 0 * z)[..., 0]

        dp = G @ V.transpose(1, 2)
        dp_sizes = G.abs() @ V.abs().transpose(1, 2)
        D = (G * o).sum(2, keepdim=True)
        e_D = 6 * u * (_norm(p * dp, 2)[..., None] + _norm(G * o, 2)[..., None]) + (least * G.abs()).sum(2, keepdim=True)
        if half:
            e_D = e_D + (2.0 ** -25 * p.amax(2, keepdim=True) * (seen * dp_sizes).sum(2, keepdim=True))
        if wide is not None:
            e_D = e_D * ~wide[r, None]
        e_D = e_D + (w + r32) * ((p * dp_sizes).sum(2, keepdim=True))
        ds = p * (dp - D)
        e_32 = p * ((w + r32) * dp_sizes + w * D.abs())
        tp, tds, t32 = p.transpose(1, 2), ds.transpose(1, 2), e_32.transpose(1, 2)

        x = c * over(ds, KK)
        e = c * (6 * u * over(ds ** 2, KK ** 2).sqrt() + e_D * over(p, KK).abs() + over(e_32, KK.abs())) + u * x.abs() + least
        if half:
            e = e + c * 2.0 ** -32 * ds.abs().amax(2, keepdim=True) * over(seen.double().expand_as(p), KK.abs())
        dq[r], b_dq[r] = x.transpose(0, 1), e.transpose(0, 1)

        def group(y):  # [H, L, d] summed over the heads that share a key/value head, as [L, K, d]
            return y.reshape(K, H // K, L, d).sum(1).transpose(0, 1)

        tseen = seen.T.double().expand_as(p)
        x = group(c * over(tds, Q))
        e = c * group((6 * u) ** 2 * over(tds ** 2, Q ** 2) + over(tp ** 2, (e_D * Q) ** 2)).sqrt() + group(c * over(t32, Q.abs()))
        e = e + u * x.abs() + least
        if half:
            top = tds.abs().amax(2, keepdim=True).reshape(K, H // K, L, 1).amax(1, keepdim=True).expand(K, H // K, L, 1).reshape(H, L, 1)
            e = e + group(c * 2.0 ** -32 * top * over(tseen, Q.abs()))
        dk[r], b_dk[r] = x, e
        x = group(over(tp, G))
        e = 6 * u * group(over(tp ** 2, G ** 2)).sqrt() + group(w * over(tp, G.abs())) + u * x.abs() + least
        if half:
            e = e + group(2.0 ** -33 * over(tseen, G.abs()))
        dv[r], b_dv[r] = x, e
    return dict(out=(out, 1.05 * b_out), lse=(lse, 1.05 * b_lse), dq=(dq, 1.05 * b_dq), dk=(dk, 1.05 * b_dk),
                dv=(dv, 1.05 * b_dv))


def unseen_zero_rows(expected, name):
    """How many rows (token, head) that hold anything would pass as zeros."""
    value, bound = expected[name]
    return int(((value.abs() <= bound).all(-1) & (value != 0).any(-1)).sum())


def outside(expected, name, got):
    """How many elements of a result are off by more than their bound, and the largest share of it."""
    value, bound = expected[name]
    got = got.double().cpu()
    same = got == value  # infinities, and padding's zeros
    off = torch.where(same, torch.zeros_like(value), (got - value).abs())
    bad = ~(off <= bound)
    return int(bad.sum()), float((off / bound.clamp_min(1e-300)).nan_to_num(nan=math.inf).max()) if off.numel() else 0.0
