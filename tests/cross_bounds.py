"""Cross attention and its gradient in 64 bits, with how far each element of a result may be off: the roundings
and bounds that attention_bounds describes, of tokens that see all the states of their sequence."""
from __future__ import annotations

import math

import torch

from attention_bounds import UNIT, _norm


def definition(q, k, v, dout, lengths, sources, first=0, k_first=0, scale=None):
    """-> {name: (value, bound)} for out, lse, dq, dk, dv, on the CPU in 64 bits."""
    dtype, u = q.dtype, UNIT[q.dtype]
    half = dtype == torch.float16
    q, k, v, dout = (x.double().cpu() for x in (q, k, v, dout))
    (T, H, d), (U, K) = q.shape, k.shape[:2]
    c = d ** -0.5 if scale is None else scale
    least = 2.0 ** -25 if half else 0.0
    r32 = 6 * math.sqrt(d) * 2.0 ** -24

    def pair(*shape, fill=0.0):
        return torch.full(shape, fill, dtype=torch.float64), torch.zeros(shape, dtype=torch.float64)

    out, b_out = pair(T, H, d)
    lse, b_lse = pair(H, T, fill=-math.inf)
    (dq, b_dq), (dk, b_dk), (dv, b_dv) = pair(T, H, d), pair(U, K, d), pair(U, K, d)
    at, k_at = first, k_first
    for L, M in zip(lengths, sources):
        r, kr = slice(at, at + L), slice(k_at, k_at + M)
        at, k_at = at + L, k_at + M
        if not L or not M:
            continue
        Q, G = q[r].transpose(0, 1), dout[r].transpose(0, 1)  # [H, L, d]
        KK, V = (x[kr].transpose(0, 1).repeat_interleave(H // K, 0) for x in (k, v))  # [H, M, d]
        s = Q @ KK.transpose(1, 2) * c
        z = torch.logsumexp(s, 2, keepdim=True)
        p = torch.exp(s - z)
        off_s = (r32 * c * (Q.abs() @ KK.abs().transpose(1, 2))).amax((1, 2), keepdim=True)
        w = 2 * off_s + 2.0 ** -20 + 2.0 ** -22 * z.abs() + 6 * math.sqrt(max(L, M) * H / K) * 2.0 ** -24
        w = w.amax(1, keepdim=True)
        pv, pv2, o = p @ V.abs(), (p ** 2 @ V ** 2).sqrt(), p @ V
        e_o = 6 * u * pv2 + w * pv + u * o.abs() + least
        every = torch.ones_like(p)
        if half:
            e_o = e_o + 2.0 ** -25 * p.amax(2, keepdim=True) * (every @ V.abs())
        out[r], b_out[r] = o.transpose(0, 1), e_o.transpose(0, 1)
        lse[:, r], b_lse[:, r] = z[..., 0], (w + 0 * z)[..., 0]

        dp, dp_sizes = G @ V.transpose(1, 2), G.abs() @ V.abs().transpose(1, 2)
        D = (G * o).sum(2, keepdim=True)
        e_D = 6 * u * (_norm(p * dp, 2)[..., None] + _norm(G * o, 2)[..., None]) + (least * G.abs()).sum(2, keepdim=True)
        if half:
            e_D = e_D + (2.0 ** -25 * p.amax(2, keepdim=True) * dp_sizes.sum(2, keepdim=True))
        e_D = e_D + (w + r32) * ((p * dp_sizes).sum(2, keepdim=True))
        ds = p * (dp - D)
        e_32 = p * ((w + r32) * dp_sizes + w * D.abs())
        tp, tds, t32, tall = (x.transpose(1, 2) for x in (p, ds, e_32, every))
        x = c * (ds @ KK)
        e = c * (6 * u * (ds ** 2 @ KK ** 2).sqrt() + e_D * (p @ KK).abs() + e_32 @ KK.abs()) + u * x.abs() + least
        if half:
            e = e + c * 2.0 ** -32 * ds.abs().amax(2, keepdim=True) * (every @ KK.abs())
        dq[r], b_dq[r] = x.transpose(0, 1), e.transpose(0, 1)

        def group(y):  # [H, M, d] summed over the heads that share a key/value head, as [M, K, d]
            return y.reshape(K, H // K, M, d).sum(1).transpose(0, 1)

        x = group(c * (tds @ Q))
        e = c * group((6 * u) ** 2 * (tds ** 2 @ Q ** 2) + tp ** 2 @ (e_D * Q) ** 2).sqrt() + group(c * (t32 @ Q.abs()))
        e = e + u * x.abs() + least
        if half:
            top = tds.abs().amax(2, keepdim=True).reshape(K, H // K, M, 1).amax(1, keepdim=True).expand(K, H // K, M, 1).reshape(H, M, 1)
            e = e + group(c * 2.0 ** -32 * top * (tall @ Q.abs()))
        dk[kr], b_dk[kr] = x, e
        x = group(tp @ G)
        e = 6 * u * group(tp ** 2 @ G ** 2).sqrt() + group(w * (tp @ G.abs())) + u * x.abs() + least
        if half:
            e = e + group(2.0 ** -33 * (tall @ G.abs()))
        dv[kr], b_dv[kr] = x, e
    return dict(out=(out, 1.05 * b_out), lse=(lse, 1.05 * b_lse), dq=(dq, 1.05 * b_dq), dk=(dk, 1.05 * b_dk), dv=(dv, 1.05 * b_dv))
