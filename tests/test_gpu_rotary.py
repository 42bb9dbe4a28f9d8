"""cel.rotary and cel.rotary_grad against the definition in 64 bits.

A value is two products and a sum in 32 bits (three roundings, of at most |u| + |v| each), of a sine and
a cosine.  These are the library's of a part of a turn rounded to 32 bits: off by 2^-25 of half a turn, pi 2^-25,
and by two of their own steps, 2^-23.  Together 6 2^-24 (|u| + |v|) at most, before the one rounding.
"""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402
from block_reference import randn, turn, within  # noqa: E402

DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]
STEP = 6 * 2.0 ** -24


def freqs_of(P, dtype=torch.float32):
    return (10000.0 ** (-torch.arange(P, dtype=torch.float64) / max(P, 1))).to(dtype).to(DEV)


def check(x, positions, freqs, axes=None, pairs=False, error=STEP):
    for f, back in ((cel.rotary, False), (cel.rotary_grad, True)):
        got = f(x, positions, freqs, axes=axes, pairs=pairs)
        want, size = turn(x, positions, freqs, axes, pairs, back)
        assert got.shape == x.shape and got.dtype == x.dtype
        within(got, want, error * size)
        P2 = 2 * freqs.numel()
        assert torch.equal(got[..., P2:], x[..., P2:])


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,P", [(64, 32), (128, 64), (80, 32), (96, 48), (40, 20), (1, 0), (2, 1), (3, 1), (7, 3), (17, 8),
                                 (33, 9), (255, 127), (256, 64), (64, 0), (4096, 2048), (4096, 0), (4095, 1500)])
def test_sizes(d, P, dtype, pairs):
    x = randn(37, 5, d, seed=d).to(dtype).to(DEV)
    check(x, torch.arange(37, device=DEV), freqs_of(P), pairs=pairs)


@pytest.mark.parametrize("T", [0, 1, 2, 3, 64, 1000, 4097])
@pytest.mark.parametrize("H", [1, 8, 9, 31])
def test_lengths_and_heads(T, H):
    check(randn(T, H, 64, seed=T + H).bfloat16().to(DEV), torch.arange(T, device=DEV, dtype=torch.int32) + 7, freqs_of(32))


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("A,split", [(2, (8, 8)), (3, (16, 24, 24)), (3, (0, 5, 11)), (4, (1, 2, 3, 4))])
def test_axes(A, split, pairs):
    P, T = sum(split), 203
    axes = torch.repeat_interleave(torch.arange(A), torch.tensor(split)).int()
    pos = torch.randint(-50, 5000, (A, T), generator=torch.Generator().manual_seed(A))
    for order in (axes, axes[torch.randperm(P, generator=torch.Generator().manual_seed(1))]):
        for p in (pos, pos.int()):
            check(randn(T, 3, 2 * P + 3, seed=P).to(DEV), p.to(DEV), freqs_of(P), axes=order.to(DEV), pairs=pairs)


def test_positions_with_strides():
    wide = torch.randint(0, 4000, (6, 300), generator=torch.Generator().manual_seed(3)).to(DEV)
    axes = (torch.arange(32) % 3).int().to(DEV)
    x = randn(100, 2, 64).to(DEV)
    for pos in (wide[::2, 50:150], wide[:3, ::3], wide.T.contiguous().T[:3, 7:107], wide[:1, :100].expand(3, 100)):
        check(x, pos, freqs_of(32), axes=axes)


def test_axes_that_do_not_exist():
    axes = torch.tensor([0, 1, -1, 2, 0, 2 ** 31 - 1, 1, -2 ** 31], dtype=torch.int32, device=DEV)
    x = randn(50, 2, 16).to(DEV)
    pos = torch.randint(0, 999, (2, 50), generator=torch.Generator().manual_seed(3)).to(DEV)
    check(x, pos, freqs_of(8), axes=axes)
    got = cel.rotary(x, pos, freqs_of(8), axes=axes)
    assert torch.equal(got[..., [2, 10]], x[..., [2, 10]])


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,P", [(64, 32), (40, 13), (7, 3), (256, 128)])
def test_pairs_without_an_axis_keep_their_bits(d, P, dtype, pairs):
    """Whatever their other value is: infinities, NaN, and the sign of zero."""
    x = randn(29, 3, d, seed=d)
    for n, odd in enumerate((float("inf"), float("nan"), -float("inf"), -0.0, 0.0)):
        x.flatten()[n::7] = odd
    x = x.to(dtype).to(DEV)
    axes = torch.tensor([(-1, 0, 2, 1, 2 ** 31 - 1)[p % 5] for p in range(P)], dtype=torch.int32, device=DEV)
    positions = torch.arange(58, device=DEV).view(2, 29)
    still = torch.zeros(d, dtype=torch.bool, device=DEV)
    for p in range(P):
        if p % 5 in (0, 2, 4):
            still[[2 * p, 2 * p + 1] if pairs else [p, p + P]] = True
    still[2 * P:] = True
    bits = {2: torch.int16, 4: torch.int32}[x.element_size()]
    for f in (cel.rotary, cel.rotary_grad):
        got = f(x, positions, freqs_of(P), axes=axes, pairs=pairs)
        assert torch.equal(got[..., still].view(bits), x[..., still].view(bits))
        clean = f(x.nan_to_num(0.0, 0.0, 0.0), positions, freqs_of(P), axes=axes, pairs=pairs)
        both = torch.isfinite(got) & torch.isfinite(x)
        assert torch.equal(got[both], clean[both])  # the others turn as ever
        again = x.clone()
        f(again, positions, freqs_of(P), axes=axes, pairs=pairs, out=again)
        assert torch.equal(again.view(bits), got.view(bits))


@pytest.mark.parametrize("far", [2 ** 20, 2 ** 31 - 64, 2 ** 40, 2 ** 52, -2 ** 45])
def test_far_positions(far):
    """Against angles of numpy's long doubles (64 bits of fraction): at 2^52 a product in 64 bits alone is off by half a turn."""
    T, P = 63, 32
    x, f = randn(T, 2, 2 * P).to(DEV), freqs_of(P)
    pos = torch.arange(T) + far
    got = cel.rotary(x, pos.to(DEV), f)
    a = pos.numpy().astype(np.longdouble)[:, None] * f.cpu().double().numpy().astype(np.longdouble)[None]
    # a has 64 bits: exact for 53 of the position less 24 of the frequency where that fits, else off by 2^-64 of it
    two_pi = np.longdouble(6.283185307179586) + np.longdouble(2.4492935982947064e-16)
    r = a - np.rint(a / two_pi) * two_pi
    off = abs(float(far)) * (2.0 ** -64 * 2 + 2.0 ** -104)  # of a, and of two_pi's own rest
    c, s = (torch.from_numpy(g(r).astype(np.float64))[:, None] for g in (np.cos, np.sin))
    u, v = x.double().cpu()[..., :P], x.double().cpu()[..., P:]
    size = (u.abs() + v.abs()).repeat(1, 1, 2)
    within(got, torch.cat([u * c - v * s, v * c + u * s], 2), (STEP + off) * size)


def test_frequencies_of_64_bits():
    check(randn(100, 2, 64).to(DEV), torch.arange(100, device=DEV) * 1000, freqs_of(32, torch.float64))


def test_strides_and_copies():
    T, H, d = 90, 6, 64
    pos, f = torch.arange(T, device=DEV), freqs_of(32)
    fused = randn(T, (H + 4) * d + 3, seed=1).bfloat16().to(DEV)
    views = [fused[:, 1:1 + H * d].view(T, H, d), fused[:, :H * d].view(T, H, d), fused[:, :2 * H * d:2][:, :d * 3].reshape(T, 3, d),
             randn(T, d, H).bfloat16().to(DEV).transpose(1, 2), randn(H, T, d).bfloat16().to(DEV).transpose(0, 1),
             randn(1, H, d).bfloat16().to(DEV).expand(T, H, d), randn(T, H, 2 * d).bfloat16().to(DEV)[..., ::2]]
    for x in views:
        check(x, pos, f)
        check(x, pos, f, pairs=True)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_in_place(dtype, pairs):
    T, H, K, d = 70, 4, 2, 48
    fused = randn(T, (H + 2 * K) * d, seed=2).to(dtype).to(DEV)
    pos, f, before = torch.arange(T, device=DEV), freqs_of(20), fused.clone()
    both = fused[:, :(H + K) * d].view(T, H + K, d)
    want = cel.rotary(both, pos, f, pairs=pairs)
    assert cel.rotary(both, pos, f, pairs=pairs, out=both) is both
    assert torch.equal(both, want) and torch.equal(fused[:, (H + K) * d:], before[:, (H + K) * d:])
    other = torch.full((T, 2 * (H + K), d), 7.0, dtype=dtype, device=DEV)
    cel.rotary_grad(both, pos, f, pairs=pairs, out=other[:, ::2])
    assert torch.equal(other[:, ::2], cel.rotary_grad(both, pos, f, pairs=pairs)) and bool((other[:, 1::2] == 7).all())


def test_infinities_stay_in_their_pair():
    x = randn(10, 2, 64).to(DEV)
    x[3, 1, 5], x[4, 0, 40] = float("inf"), float("nan")
    got, plain = cel.rotary(x, torch.arange(10, device=DEV), freqs_of(32)), torch.isfinite(x)
    touched = ~torch.isfinite(got)
    assert bool(touched[3, 1, [5, 37]].all()) and bool(touched[4, 0, [8, 40]].all()) and int(touched.sum()) == 4
    assert int((~plain).sum()) == 2


def test_many_pieces_of_one_call():
    """More threads' work than a workgroup deals with, at every deal of the heads."""
    for T, H in ((3000, 1), (3000, 40), (20000, 40)):
        x = randn(64, H, 32, seed=H).bfloat16().to(DEV).repeat(-(-T // 64), 1, 1)[:T]
        pos = (torch.arange(T, device=DEV) % 64)
        got = cel.rotary(x, pos, freqs_of(16))
        want, size = turn(x[:64], pos[:64], freqs_of(16))
        within(got[:64], want, STEP * size)
        assert torch.equal(got, got[:64].repeat(-(-T // 64), 1, 1)[:T])


def test_the_gradient_is_the_transpose():
    x, g = randn(40, 3, 24, seed=1).to(DEV), randn(40, 3, 24, seed=2).to(DEV)
    pos, f = torch.arange(40, device=DEV) * 3, freqs_of(10)
    one = float((cel.rotary(x, pos, f).double() * g.double()).sum())
    two = float((x.double() * cel.rotary_grad(g, pos, f).double()).sum())
    assert abs(one - two) <= 8 * 2.0 ** -24 * 2 * float((x.double().abs().sum() * g.double().abs().max()))


def test_refusals():
    def refused(*a, **kw):
        with pytest.raises(cel.CelError) as e:
            cel.rotary(*a, **kw)
        assert e.value.code == -1

    x, pos, f = randn(8, 2, 16).to(DEV), torch.arange(8, device=DEV), freqs_of(8)
    axes = torch.zeros(8, dtype=torch.int32, device=DEV)
    refused(x[0], pos, f)
    refused(x.double(), pos, f)
    refused(x.cpu(), pos, f)
    refused(x, pos.cpu(), f)
    refused(x, pos[:7], f)
    refused(x, pos.float(), f)
    refused(x, pos.repeat(2, 1), f)  # two axes, and nothing says which pair has which
    refused(x, pos, f.half())
    refused(x, pos, freqs_of(9))
    refused(x, pos, f, axes=axes[:7])
    refused(x, pos, f, axes=axes.long())
    refused(x, pos[:0].reshape(0, 8) if False else torch.zeros(0, 8, dtype=torch.int64, device=DEV), f, axes=axes)
    refused(x, pos, f, out=torch.empty(8, 2, 15, device=DEV))
    refused(x, pos, f, out=torch.empty(8, 2, 16, device=DEV).half())
    refused(x, pos, f, out=torch.empty(8, 2, 32, device=DEV)[..., ::2])
    refused(x, pos, f, out=torch.empty(1, 2, 16, device=DEV).expand(8, 2, 16))
    wide = torch.zeros(9, 2, 16, device=DEV)
    refused(wide[:8], pos, f, out=wide[1:])
    refused(wide[:8], pos, f, out=wide.flatten()[8:264].view(8, 2, 16))
    both = torch.zeros(8, 3, 2, 16, device=DEV)
    refused(both[:, 0], pos, f, out=both.flatten()[32:288].view(8, 2, 16))  # rows of another stride between
    cel.rotary(both[:, 0], pos, f, out=both[:, 2])
    refused(x, pos, f, out=x.flip(0)[:8].transpose(0, 1).contiguous().transpose(0, 1)[:, :1])
    refused(x.clone().requires_grad_(), pos, f)
