"""cel.attention and cel.attention_grad against the definition in 64 bits.

Tolerances (2-norm of the difference over the 2-norm of the reference), with u
the unit round-off of the rows' type (2^-8 bfloat16, 2^-11 float16: what a
rounding to nearest is off by at most, relative):
- out: the weights p are rounded once, which moves out by at most u |out|
  where the roundings' signs are independent, and out once: 2 u.
- lse: 32-bit sums of at most a few thousand products and exponentials, a few
  times 2^-24 each: 1e-5 absolute, of values around 1 to 10.
- gradients: their own rounding, that of p or ds, and out's in D = <dout, out>,
  u |dout| |out| at most next to <dout, v>: u each, and one u for the 32-bit
  sums between them: 4 u.
"""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402

DEV = "cuda:0"
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.bfloat16, torch.float16]


def ptr_of(lengths, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lengths)]).astype(np.int32), device=DEV)


def batch(T, H, K, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(T, n, d, generator=g).to(dtype).to(DEV) for n in (H, K, K, H)]


def reference(q, k, v, dout, lengths, first=0, scale=None):
    """out, lse, dq, dk, dv in float64 on the CPU, token by token's definition."""
    q, k, v, dout = (x.double().cpu() for x in (q, k, v, dout))
    T, H, d = q.shape
    K, c = k.shape[1], d ** -0.5 if scale is None else scale
    out, lse = torch.zeros(T, H, d, dtype=torch.float64), torch.full((H, T), -float("inf"), dtype=torch.float64)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    at = first
    for L in lengths:
        r = slice(at, at + L)
        at += L
        seen = torch.tril(torch.ones(L, L, dtype=torch.bool))
        for h in range(H):
            kv = h // (H // K)
            s = (q[r, h] @ k[r, kv].T * c).masked_fill(~seen, -float("inf"))
            z = torch.logsumexp(s, 1) if L else s.sum(1)
            p = torch.exp(s - z[:, None])
            out[r, h], lse[h, r] = p @ v[r, kv], z
            ds = p * (dout[r, h] @ v[r, kv].T - (dout[r, h] * out[r, h]).sum(1, keepdim=True))
            dq[r, h] = c * ds @ k[r, kv]
            dk[r, kv] += c * ds.T @ q[r, h]
            dv[r, kv] += p.T @ dout[r, h]
    return out, lse, dq, dk, dv


def off(x, y):
    x, y = x.double().cpu(), y.double().cpu()
    n = float(y.norm())
    return float((x - y).norm()) / n if n else float((x - y).norm())


def check(q, k, v, dout, lengths, first=0, scale=None):
    ptr, u = ptr_of(lengths, first), UNIT[q.dtype]
    out, lse = cel.attention(q, k, v, ptr, scale=scale)
    grads = cel.attention_grad(dout, q, k, v, out, lse, ptr, scale=scale)
    r_out, r_lse, *r_grads = reference(q, k, v, dout, lengths, first, scale)
    assert off(out, r_out) <= 2 * u
    fin = torch.isfinite(r_lse)
    assert torch.equal(torch.isfinite(lse).cpu(), fin)
    assert (lse.double().cpu()[fin] - r_lse[fin]).abs().max() <= 1e-5 if fin.any() else True
    assert bool((lse.cpu()[~fin] == -float("inf")).all())
    for name, x, y in zip(("dq", "dk", "dv"), grads, r_grads):
        assert torch.isfinite(x).all() and off(x, y) <= 4 * u, name
    none = torch.ones(q.shape[0], dtype=torch.bool)
    none[first:first + sum(lengths)] = False
    for x in (out, *grads):
        assert not x[none.to(DEV)].any()
    return out, lse, grads


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [8, 24, 32, 40, 64, 72, 80, 96, 104, 128])
def test_dimensions(d, dtype):
    lengths = [150, 1, 33, 64]
    check(*batch(sum(lengths), 4, 2, d, dtype, d), lengths)


@pytest.mark.parametrize("lengths", [[1], [2], [31], [32], [33], [63], [64], [65], [127], [128], [129], [191], [192],
                                     [193], [257], [700], [1] * 40, [0, 5, 0, 0, 130, 0], [64] * 5, [3, 500, 2, 128, 1]])
def test_lengths(lengths):
    check(*batch(sum(lengths), 2, 1, 64, torch.bfloat16, sum(lengths)), lengths)
    check(*batch(sum(lengths), 2, 2, 128, torch.float16, sum(lengths)), lengths)


@pytest.mark.parametrize("H,K", [(1, 1), (3, 1), (5, 5), (6, 3), (16, 2), (24, 8)])
def test_head_groups(H, K):
    lengths = [90, 47]
    check(*batch(137, H, K, 64, torch.bfloat16, H), lengths)


@pytest.mark.parametrize("T,first,lengths", [(300, 7, [100, 50]), (200, 0, []), (200, 130, [1]), (129, 0, [128]),
                                             (400, 200, [0, 200, 0])])
def test_tokens_of_no_sequence(T, first, lengths):
    check(*batch(T, 2, 1, 64, torch.bfloat16, T), lengths, first)


def test_no_tokens_and_no_sequences():
    q, k, v, g = batch(0, 2, 1, 64, torch.bfloat16)
    out, lse = cel.attention(q, k, v, ptr_of([]))
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)
    assert [x.shape[0] for x in cel.attention_grad(g, q, k, v, out, lse, ptr_of([]))] == [0, 0, 0]


@pytest.mark.parametrize("dtype", TYPES)
def test_long_sequence(dtype):
    check(*batch(3000, 2, 1, 128, dtype, 5), [2500, 500])


def test_scale_and_large_scores():
    """Scores of some hundreds: the running maximum moves far and weights vanish."""
    q, k, v, g = batch(333, 2, 2, 64, torch.float16, 3)
    check(q, k, v, g, [333], scale=0.01)
    out, lse = cel.attention(q * 8, k * 8, v, ptr_of([333]), scale=1.0)
    r_out, r_lse, *_ = reference(q * 8, k * 8, v, g, [333], scale=1.0)
    assert off(out, r_out) <= 2 * UNIT[torch.float16]
    # products of up to 64 * 600 in 32 bits: 2^-24 of sums of magnitudes below 64 * 64 * 16 a few times over
    assert (lse.double().cpu() - r_lse).abs().max() <= 1e-2


def test_strides_and_fused_views():
    T, H, K, d = 200, 4, 2, 64
    lengths = [120, 80]
    q, k, v, g = batch(T, H, K, d, torch.bfloat16, 9)
    plain = check(q, k, v, g, lengths)
    fused = torch.cat([x.reshape(T, -1) for x in (q, k, v)], 1)
    fq, fk, fv = (x.view(T, -1, d) for x in fused.split([H * d, K * d, K * d], 1))
    heads_first = g.transpose(0, 1).contiguous().transpose(0, 1)
    ptr = ptr_of(lengths)
    out, lse = cel.attention(fq, fk, fv, ptr)
    into = torch.full((T, (H + 2 * K) * d), 7.0, dtype=q.dtype, device=DEV)
    views = [x.view(T, -1, d) for x in into.split([H * d, K * d, K * d], 1)]
    got = cel.attention_grad(heads_first, fq, fk, fv, out, lse, ptr, grads=views)
    assert torch.equal(out, plain[0]) and torch.equal(lse, plain[1])
    for a, b in zip(got, plain[2]):
        assert torch.equal(a, b)
    # values not contiguous, and addresses off 16 bytes: copied by the call
    odd = torch.empty(T * K * d + 1, dtype=q.dtype, device=DEV)[1:].view(T, K, d).copy_(k)
    turned = v.transpose(1, 2).contiguous().transpose(1, 2)
    again, _ = cel.attention(q, odd, turned, ptr)
    assert torch.equal(again, plain[0])


def test_the_same_bits_every_time():
    lengths = [700, 3, 260, 37]
    q, k, v, g = batch(1000, 8, 2, 80, torch.bfloat16, 11)
    ptr = ptr_of(lengths)
    first = None
    for _ in range(3):
        out, lse = cel.attention(q, k, v, ptr)
        got = (out, lse, *cel.attention_grad(g, q, k, v, out, lse, ptr))
        assert first is None or all(torch.equal(a, b) for a, b in zip(got, first))
        first = got


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_row_does_not_see_stays_out(bad, d):
    """A token full of infinities or NaN reaches the later tokens of its own
    sequence only (forward: through k and v; backward: k and v's gradients of
    earlier tokens see q and dout, dq of later ones see k and v)."""
    lengths, at = [60, 200, 90], 60 + 97  # in the middle sequence
    T = sum(lengths)
    q, k, v, g = batch(T, 2, 1, d, torch.bfloat16, 4)
    ptr = ptr_of(lengths)
    out0, lse0 = cel.attention(q, k, v, ptr)
    g0 = cel.attention_grad(g, q, k, v, out0, lse0, ptr)
    before, behind = slice(0, at), slice(260, T)
    k2, v2 = k.clone(), v.clone()
    k2[at], v2[at] = bad, bad
    out, lse = cel.attention(q, k2, v2, ptr)
    for rows in (before, behind):
        assert torch.equal(out[rows], out0[rows]) and torch.equal(lse[:, rows], lse0[:, rows])
    assert not torch.isfinite(out[at:260].float()).all()
    dq, dk, dv = cel.attention_grad(g, q, k2, v2, out, lse, ptr)
    assert torch.equal(dq[before], g0[0][before]) and torch.equal(dq[behind], g0[0][behind])
    assert torch.equal(dk[behind], g0[1][behind]) and torch.equal(dv[behind], g0[2][behind])
    # q and dout of one token: keys behind it, and other sequences, do not see them
    q2, g2 = q.clone(), g.clone()
    q2[at], g2[at] = bad, bad
    out, lse = cel.attention(q2, k, v, ptr)
    others = torch.arange(T, device=DEV) != at
    assert torch.equal(out[others], out0[others])
    dq, dk, dv = cel.attention_grad(g2, q2, k, v, out, lse, ptr)
    assert torch.equal(dq[others], g0[0][others])
    for x, y in ((dk, g0[1]), (dv, g0[2])):
        assert torch.equal(x[:60], y[:60]) and torch.equal(x[at + 1:], y[at + 1:])
    assert not torch.isfinite(dk[60:at + 1].float()).all()


def test_padding_may_hold_anything():
    q, k, v, g = batch(300, 2, 2, 64, torch.bfloat16, 6)
    plain = check(q, k, v, g, [100, 130], 20)
    for x in (q, k, v, g):
        x[:20] = float("nan")
        x[250:] = float("inf")
    ptr = ptr_of([100, 130], 20)
    out, lse = cel.attention(q, k, v, ptr)
    assert torch.equal(out, plain[0]) and torch.equal(lse, plain[1])
    for a, b in zip(cel.attention_grad(g, q, k, v, out, lse, ptr), plain[2]):
        assert torch.equal(a, b)


def test_gradient_against_differences():
    """The directional derivative of <dout, out> by central differences of the 64-bit
    definition, along random directions: 4 u of |gradient| |direction|."""
    lengths = [70, 30]
    q, k, v, g = batch(100, 2, 1, 64, torch.float16, 8)
    ptr = ptr_of(lengths)
    out, lse = cel.attention(q, k, v, ptr)
    grads = cel.attention_grad(g, q, k, v, out, lse, ptr)
    rng = torch.Generator().manual_seed(1)
    x = [t.double().cpu() for t in (q, k, v)]
    for n in range(3):
        step = torch.randn(x[n].shape, generator=rng, dtype=torch.float64)
        value = []
        for e in (1e-4, -1e-4):
            y = list(x)
            y[n] = x[n] + e * step
            value.append(float((reference(*y, g, lengths)[0] * g.double().cpu()).sum()))
        slope = (value[0] - value[1]) / 2e-4
        mine = float((grads[n].double().cpu() * step).sum())
        bound = 4 * UNIT[torch.float16] * float(grads[n].double().norm()) * float(step.norm())
        assert abs(mine - slope) <= bound


def test_on_another_stream_and_in_a_graph():
    lengths = [200, 56]
    q, k, v, g = batch(256, 4, 2, 64, torch.bfloat16, 2)
    ptr = ptr_of(lengths)

    def step():
        out, lse = cel.attention(q, k, v, ptr)
        return (out, lse, *cel.attention_grad(g, q, k, v, out, lse, ptr))

    plain = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, plain))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for n in range(3):
        q.copy_(batch(256, 4, 2, 64, torch.bfloat16, 20 + n)[0])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))


def test_malformed_seq_ptr_stays_in_bounds():
    q, k, v, g = batch(200, 2, 1, 64, torch.bfloat16, 2)
    for p in ([5, 100, 20, 200], [-50, 100, 1 << 30], [300, 400], [0, 1 << 30], [150, 90]):
        ptr = torch.tensor(p, dtype=torch.int32, device=DEV)
        out, lse = cel.attention(q, k, v, ptr)
        cel.attention_grad(g, q, k, v, out, lse, ptr)
        torch.cuda.synchronize()


def test_refusals():
    q, k, v, g = batch(64, 4, 2, 64, torch.bfloat16)
    ptr = ptr_of([64])
    out, lse = cel.attention(q, k, v, ptr)

    def refused(f, *a, **kw):
        with pytest.raises(cel.CelError) as e:
            f(*a, **kw)
        assert e.value.code == -1

    refused(cel.attention, q.float(), k.float(), v.float(), ptr)
    refused(cel.attention, q, k.half(), v, ptr)
    refused(cel.attention, q, k[:63], v[:63], ptr)
    refused(cel.attention, q[:, :3], k, v, ptr)
    refused(cel.attention, q, k, v[:, :1], ptr)
    refused(cel.attention, q[0], k, v, ptr)
    refused(cel.attention, q[..., :60], k[..., :60], v[..., :60], ptr)
    refused(cel.attention, *(torch.zeros(4, 2, 136, dtype=torch.bfloat16, device=DEV),) * 3, ptr)
    refused(cel.attention, q, k, v, ptr.long())
    refused(cel.attention, q, k, v, ptr.cpu())
    refused(cel.attention, q.cpu(), k, v, ptr)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        refused(cel.attention, q, k, v, ptr, scale=scale)
    refused(cel.attention_grad, g[:, :2], q, k, v, out, lse, ptr)
    refused(cel.attention_grad, g, q, k, v, out, lse.T.contiguous(), ptr)
    refused(cel.attention_grad, g, q, k, v, out, lse.double(), ptr)
    refused(cel.attention_grad, g, q, k, v, out, lse, ptr, grads=(q[:, :, ::2], k, v))
    odd = torch.empty(q.numel() + 1, dtype=q.dtype, device=DEV)[1:].view(q.shape)
    refused(cel.attention_grad, g, q, k, v, out, lse, ptr, grads=(odd, torch.empty_like(k), torch.empty_like(v)))


@pytest.mark.parametrize("lengths", [[512], [513], [640], [1100], [1000, 24], [0, 511, 1], [1] * 600, [30] * 20,
                                     [70, 40, 500, 64, 130]])
@pytest.mark.parametrize("d,dtype", [(32, torch.float16), (64, torch.bfloat16), (96, torch.bfloat16), (128, torch.float16)])
def test_few_tiles_of_many_keys(lengths, d, dtype):
    """Few rows' tiles over 512 tokens and more: a tile's keys are dealt out and joined."""
    check(*batch(sum(lengths), 2, 1, d, dtype, d + len(lengths)), lengths)


def test_few_tiles_with_tokens_of_no_sequence():
    for T, first, lengths in [(700, 0, []), (700, 650, [3]), (900, 130, [260, 0, 300])]:
        check(*batch(T, 2, 2, 64, torch.bfloat16, T), lengths, first)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [150, 250, 380])
def test_few_tiles_and_what_a_row_does_not_see(bad, at):
    """Infinities and NaN in one token's k and v, in either half of the keys' tiles."""
    lengths = [100, 400, 200]
    q, k, v, g = batch(700, 2, 1, 64, torch.bfloat16, 6)
    ptr = ptr_of(lengths)
    out0, lse0 = cel.attention(q, k, v, ptr)
    g0 = cel.attention_grad(g, q, k, v, out0, lse0, ptr)
    k2, v2 = k.clone(), v.clone()
    k2[at], v2[at] = bad, bad
    out, lse = cel.attention(q, k2, v2, ptr)
    dq, dk, dv = cel.attention_grad(g, q, k2, v2, out, lse, ptr)
    for rows in (slice(0, at), slice(500, 700)):
        assert torch.equal(out[rows], out0[rows]) and torch.equal(lse[:, rows], lse0[:, rows])
        assert torch.equal(dq[rows], g0[0][rows])
    assert torch.equal(dk[500:], g0[1][500:]) and torch.equal(dv[500:], g0[2][500:])
    assert not torch.isfinite(out[at:500].float()).all()


def test_views_of_a_buffer_beyond_32_bits():
    """Rows 2^23 values apart: the last of them lie past 2^32 bytes."""
    T, d, lengths = 600, 64, [90, 510]
    q, k, v, g = batch(T, 2, 1, d, torch.bfloat16, 12)
    plain = check(q, k, v, g, lengths)
    wide = torch.empty(T * 2 ** 23, dtype=q.dtype, device=DEV)
    views = [wide.as_strided((T, x.shape[1], d), (2 ** 23, d, 1), 64 * 1000 * n) for n, x in enumerate((q, k, v, g))]
    for view, x in zip(views, (q, k, v, g)):
        view.copy_(x)
    into = [wide.as_strided((T, x.shape[1], d), (2 ** 23, d, 1), 64 * 1000 * n + 64 * 500) for n, x in enumerate((q, k, v))]
    ptr = ptr_of(lengths)
    out, lse = cel.attention(*views[:3], ptr)
    got = cel.attention_grad(views[3], *views[:3], out, lse, ptr, grads=into)
    assert torch.equal(out, plain[0]) and torch.equal(lse, plain[1])
    for a, b in zip(got, plain[2]):
        assert torch.equal(a, b)
