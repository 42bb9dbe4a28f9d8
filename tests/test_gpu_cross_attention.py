"""cel.cross_attention and cel.cross_attention_grad element by element against the definition in 64 bits
(cross_bounds): each value against a bound of its own."""
from __future__ import annotations

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402
from attention_bounds import outside, unseen_zero_rows  # noqa: E402
from cross_bounds import definition  # noqa: E402

DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16]


def ptr_of(lengths, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lengths)]).astype(np.int32), device=DEV)


def batch(T, U, H, K, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, heads, d, generator=g).to(dtype).to(DEV) for n, heads in ((T, H), (U, K), (U, K), (T, H))]


def run(q, k, v, dout, p, kp, **how):
    out, lse = cel.cross_attention(q, k, v, p, kp, **how)
    dq, dk, dv = cel.cross_attention_grad(dout, q, k, v, out, lse, p, kp, **how)
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)


def check(q, k, v, dout, lengths, sources, first=0, k_first=0, scale=None):
    expected = definition(q, k, v, dout, lengths, sources, first, k_first, scale)
    got = run(q, k, v, dout, ptr_of(lengths, first), ptr_of(sources, k_first), scale=scale)
    for n in ("out", "dq", "dk", "dv"):  # the bounds see a missing row, but for one in a hundred at most
        assert unseen_zero_rows(expected, n) <= expected[n][0].shape[0] * expected[n][0].shape[1] // 100
    bad = {n: outside(expected, n, x) for n, x in got.items()}
    assert not any(n for n, _ in bad.values()), bad
    return got


def mixed(n, total, least, seed):
    rng = np.random.default_rng(seed)
    cuts = np.sort(rng.integers(0, total - least * n + 1, n - 1))
    return [int(x) + least for x in np.diff(np.concatenate([[0], cuts, [total - least * n]]))]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [8, 24, 32, 40, 64, 72, 80, 96, 104, 128])
def test_dimensions(d, dtype):
    lengths, sources = [150, 1, 0, 33, 64], [70, 129, 11, 0, 200]
    check(*batch(251, 413, 4, 2, d, dtype, d), lengths, sources, 1, 2)


@pytest.mark.parametrize("L", [1, 2, 31, 33, 64, 65, 127, 129, 300])
@pytest.mark.parametrize("M", [1, 2, 16, 63, 64, 65, 128, 191, 700])
def test_lengths(L, M):
    check(*batch(L, M, 2, 1, 64, torch.bfloat16, L + M), [L], [M])
    check(*batch(L, M, 2, 2, 128, torch.float16, L + M), [L], [M])


@pytest.mark.parametrize("lengths,sources", [
    ([1] * 40, [5] * 40), ([1] * 70, list(range(70))), ([5] * 40, [1] * 40), ([0, 5, 0, 0, 130, 0], [3, 0, 200, 0, 1, 64]),
    ([64] * 5, [64] * 5), ([3, 500, 2, 128, 1], [700, 2, 65, 1, 33]), ([200, 1], [0, 0]), ([0, 0], [40, 50]), ([128, 128], [0, 300])])
def test_batches(lengths, sources):
    T, U = sum(lengths), sum(sources)
    check(*batch(T, U, 4, 2, 64, torch.float16, T), lengths, sources)
    check(*batch(T + 9, U + 150, 3, 1, 96, torch.bfloat16, T), lengths, sources, 4, 140)


@pytest.mark.parametrize("H,K", [(1, 1), (3, 1), (5, 5), (6, 3), (16, 2), (24, 8), (65, 5)])
def test_head_groups(H, K):
    check(*batch(137, 211, H, K, 64, torch.bfloat16, H), [90, 47], [11, 200])


@pytest.mark.parametrize("T,U,n,H,K", [
    (1100, 900, 9, 32, 32),    # keys with one group of waves
    (6301, 3001, 90, 40, 8),   # five query heads a key/value head, dealt out unevenly
    (2049, 12289, 60, 16, 8),
    (4097, 1023, 40, 5, 1),    # an odd number of rows in the scratch
    (700, 5000, 3, 2, 1)])     # two groups of waves share a sequence's keys
@pytest.mark.parametrize("d,dtype", [(64, torch.bfloat16), (128, torch.float16)])
def test_large_launches(T, U, n, H, K, d, dtype):
    lengths, sources = mixed(n, T - 9, 0, T + H), mixed(n, U - 5, 0, U)
    check(*batch(T, U, H, K, d, dtype, T), lengths, sources, 4, 3)


@pytest.mark.parametrize("T,U,n", [(5000, 3000, 300), (3000, 9000, 2), (20000, 70, 60), (70, 20000, 60)])
def test_tiles_in_order_of_their_length(T, U, n):
    """Launches whose tiles are put in order, on one side or both: each is dealt with once."""
    lengths, sources = mixed(n, T, 0, T + n), mixed(n, U, 0, U + n)
    check(*batch(T, U, 64, 16, 32, torch.bfloat16, T), lengths, sources)


FEW = [([1], [6000]), ([1, 1, 1], [3000, 0, 4000]), ([40], [2000]), ([5, 0, 130, 2], [900, 700, 3000, 1]), ([17, 90], [5000, 60])]


@pytest.mark.parametrize("lengths,sources", FEW)
@pytest.mark.parametrize("d,dtype,H,K", [(64, torch.bfloat16, 4, 2), (128, torch.float16, 2, 2), (40, torch.float16, 6, 1), (96, torch.bfloat16, 1, 1)])
def test_few_rows_share_their_keys(lengths, sources, d, dtype, H, K):
    """Rows whose keys are dealt out to several workgroups, single tokens among them, and the other way round."""
    T, U = sum(lengths), sum(sources)
    got = check(*batch(T + 3, U + 70, H, K, d, dtype, T), lengths, sources, 2, 64)
    check(*batch(U + 70, T + 3, H, K, d, dtype, T), sources, lengths, 64, 2)
    again = run(*batch(T + 3, U + 70, H, K, d, dtype, T), ptr_of(lengths, 2), ptr_of(sources, 64))
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan_where_keys_are_shared(dtype):
    lengths, sources = [3, 2], [3000, 2500]
    q, k, v, g = batch(5, 5500, 2, 1, 64, dtype, 7)
    plain = run(q, k, v, g, ptr_of(lengths), ptr_of(sources))
    k[3100], v[4000], g[4] = math.nan, math.inf, math.nan
    got = run(q, k, v, g, ptr_of(lengths), ptr_of(sources))
    for n, at in (("out", slice(0, 3)), ("dq", slice(0, 3)), ("dk", slice(0, 3000)), ("dv", slice(0, 3000))):
        assert torch.equal(got[n][at], plain[n][at]), n
    assert torch.equal(got["lse"][:, :3], plain["lse"][:, :3]) and bool(torch.isnan(got["out"][3:]).any())


@pytest.mark.parametrize("dtype,H,K,d", [(torch.bfloat16, 2, 1, 64), (torch.float16, 4, 4, 128), (torch.bfloat16, 16, 4, 40)])
def test_no_numbers_in_all_that_a_row_sees_of_a_share(dtype, H, K, d):
    """Each row's keys are 2,753 and 2,747, dealt out 512 or more to a workgroup: of a share, the first three rows
    see key 2,752 alone (where 86 tiles are shared by ten), or all keys are no numbers.  A weight that is no number
    makes the row's result none, as for few keys."""
    lengths, sources = [3, 2], [2753, 2747]
    p, kp = ptr_of(lengths), ptr_of(sources)
    q, k, v, g = batch(5, 5500, H, K, d, dtype, 8)
    plain = run(q, k, v, g, p, kp)
    for keys in (slice(2752, 2753), slice(0, 2753), slice(512, 1600), slice(1000, 1001)):
        bad = k.clone()
        bad[keys] = math.nan
        got = run(q, bad, v, g, p, kp)
        for n in ("out", "dq"):
            assert bool(torch.isnan(got[n][:3]).all()) and torch.equal(got[n][3:], plain[n][3:]), (keys, n)
        assert bool(torch.isnan(got["lse"][:, :3]).all()) and torch.equal(got["lse"][:, 3:], plain["lse"][:, 3:]), keys
        for n in ("dk", "dv"):
            assert bool(torch.isnan(got[n][:2753]).all()) and torch.equal(got[n][2753:], plain[n][2753:]), (keys, n)


@pytest.mark.parametrize("U", [60, 700, 16384])
def test_one_token_and_no_numbers(U):
    """The same pattern however many keys there are, and so workgroups that share them."""
    q, k, v, g = batch(1, U, 2, 1, 64, torch.bfloat16, U)
    p, kp = ptr_of([1]), ptr_of([U])
    bad = k.clone()
    bad[U // 3:2 * U // 3] = math.nan
    out, lse = cel.cross_attention(q, bad, v, p, kp)
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())
    out, lse = cel.cross_attention(q * math.nan, k, v, p, kp)
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())
    # keys of weight 0 with infinite values: 0 times infinity
    q[:], low, wide = 1.0, k.clone(), v.clone()
    low[U // 3:2 * U // 3], wide[U // 2, :, 5] = -math.inf, math.inf
    out, lse = cel.cross_attention(q, low, wide, p, kp)
    assert bool(torch.isnan(out[..., 5]).all()) and bool(torch.isfinite(out[..., :5]).all()) and bool(torch.isfinite(out[..., 6:]).all())
    assert bool(torch.isfinite(lse).all())


def test_scores_of_minus_infinity():
    """A row all of whose scores are minus infinity has no weights (0 / 0), whether its keys are shared or not; one
    with another score has that one's alone."""
    for U in (60, 6000):
        q, k, v, g = batch(2, U, 1, 1, 64, torch.bfloat16, 9)
        q[:], k[:] = 1.0, -math.inf
        out, lse = cel.cross_attention(q, k, v, ptr_of([2]), ptr_of([U]))
        assert bool(torch.isnan(out).all()) and bool((lse == -math.inf).all())
        k[U // 2] = 0.5
        out, lse = cel.cross_attention(q, k, v, ptr_of([2]), ptr_of([U]))
        assert torch.equal(out, v[U // 2].expand(2, 1, 64)) and float((lse - 4.0).abs().max()) <= 1e-5


def test_as_many_keys_as_fit_one_tile_in_odd_places():
    """D is a sum in 32 bits for rows whose keys lie in one tile, wherever that tile is among a workgroup's."""
    lengths, sources = [1, 90, 2, 30, 128, 7], [100, 3, 64, 60, 1, 130]
    for H, K, U in ((2, 1, 0), (40, 8, 0), (1, 1, 600)):
        s = sources[:-1] + [sources[-1] + U]
        check(*batch(sum(lengths), sum(s), H, K, 64, torch.float16, H), lengths, s)


def test_no_rows_no_keys_no_sequences():
    for T, U in ((0, 0), (0, 70), (70, 0), (0, 5000)):
        q, k, v, g = batch(T, U, 8, 2, 64, torch.bfloat16)
        for n in (0, 2):
            got = run(q, k, v, g, ptr_of([0] * n), ptr_of([0] * n))
            assert not any(bool(got[x].any()) for x in ("out", "dq", "dk", "dv")) and bool((got["lse"] == -math.inf).all())
    q, k, v, g = batch(70, 90, 4, 2, 64, torch.bfloat16)
    got = run(q, k, v, g, ptr_of([70]), ptr_of([0], 90))
    assert not any(bool(got[x].any()) for x in ("out", "dq", "dk", "dv")) and bool((got["lse"] == -math.inf).all())


def test_the_same_batch_as_both_sides():
    """States that are the tokens': attention without the causal mask, of which a sequence's last token is the same."""
    q, k, v, g = batch(300, 300, 4, 2, 64, torch.bfloat16, 5)
    lengths = [100, 37, 163]
    ptr, last = ptr_of(lengths), torch.tensor([99, 136, 299], device=DEV)
    out, lse = cel.cross_attention(q, k, v, ptr, ptr)
    causal, c_lse = cel.attention(q, k, v, ptr)
    assert float((out[last].float() - causal[last].float()).abs().max()) <= 2 * 2.0 ** -8 * float(causal[last].float().abs().max())
    assert float((lse[:, last] - c_lse[:, last]).abs().max()) <= 1e-5


def test_malformed_pointers_stay_in_bounds():
    q, k, v, g = batch(100, 200, 4, 2, 64, torch.bfloat16)
    for a, b in (([0, 500, 100], [0, 100, 200]), ([0, 50, 100], [150, 20, 2 ** 30]), ([-7, 50, 100], [-3, 100, 201]),
                 ([100, 0, 100], [200, 0, 200]), ([2 ** 31 - 1, 0, -2 ** 31], [-2 ** 31, 2 ** 31 - 1, 5])):
        run(q, k, v, g, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (a, b)))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_infinities_and_nan_of_other_sequences_stay_out(d, dtype):
    lengths, sources = [50, 30, 90], [40, 100, 70]
    q, k, v, g = batch(170, 210, 4, 2, d, dtype, d)
    plain = run(q, k, v, g, ptr_of(lengths), ptr_of(sources))
    k[60], v[70], v[80] = math.nan, math.inf, -math.inf  # states of the second
    q[60], g[55] = math.nan, math.inf  # and tokens of it
    got = run(q, k, v, g, ptr_of(lengths), ptr_of(sources))
    rows = torch.cat([torch.arange(50), torch.arange(80, 170)]).to(DEV)
    keys = torch.cat([torch.arange(40), torch.arange(140, 210)]).to(DEV)
    for n, at in (("out", rows), ("dq", rows), ("dk", keys), ("dv", keys)):
        assert torch.equal(got[n][at], plain[n][at]), n
    assert torch.equal(got["lse"][:, rows], plain["lse"][:, rows])
    assert not bool(torch.isfinite(got["out"][50:80]).all())


def test_strides_copies_and_gradients_in_place():
    T, U, H, K, d = 90, 130, 4, 2, 64
    q, k, v, g = batch(T, U, H, K, d, torch.bfloat16, 3)
    p, kp = ptr_of([50, 40]), ptr_of([100, 30])
    plain = run(q, k, v, g, p, kp)
    fused = torch.cat([k.view(U, -1), v.view(U, -1)], 1)
    views = [(q, fused[:, :K * d].view(U, K, d), fused[:, K * d:].view(U, K, d), g),
             tuple(x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, g)),
             tuple(torch.stack([x, x], -1)[..., 0] for x in (q, k, v, g))]
    for x in views:
        got = run(*x, torch.stack([p, p], 1)[:, 0], kp)
        assert all(torch.equal(got[n], plain[n]) for n in plain)
    dfused, dq = torch.zeros_like(fused), torch.zeros_like(q)
    into = dq, dfused[:, :K * d].view(U, K, d), dfused[:, K * d:].view(U, K, d)
    got = cel.cross_attention_grad(g, q, k, v, plain["out"], plain["lse"], p, kp, grads=into)
    assert all(a is b for a, b in zip(got, into)) and all(torch.equal(a, plain[n]) for a, n in zip(got, ("dq", "dk", "dv")))
    with pytest.raises(cel.CelError):
        cel.cross_attention_grad(g, q, k, v, plain["out"], plain["lse"], p, kp, grads=(q, into[1], into[2]))
    with pytest.raises(cel.CelError):
        cel.cross_attention_grad(g, q, k, v, plain["out"], plain["lse"], p, kp, grads=(dq, into[1], into[1]))
    with pytest.raises(cel.CelError):
        cel.cross_attention_grad(g, q, k, v, plain["out"], plain["lse"], p, kp, grads=(dq, dfused[:1, :K * d].view(1, K, d).expand(U, K, d), into[2]))


def test_inside_a_graph():
    q, k, v, g = batch(600, 900, 8, 2, 64, torch.float16, 8)
    p, kp = ptr_of([100, 500]), ptr_of([700, 200])
    want = run(q, k, v, g, p, kp)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run(q, k, v, g, p, kp)
    for _ in range(3):
        for t in held.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(held[n], want[n]) for n in want)
        assert all(torch.equal(x, want[n]) for n, x in run(q, k, v, g, p, kp).items())


def test_kernel_times_do_not_hold_each_other():
    """Of one token on many states, whose keys are shared: the kernels' times together are no longer than the calls'."""
    q, k, v, g = batch(1, 16384, 16, 4, 128, torch.bfloat16, 2)
    p, kp = ptr_of([1]), ptr_of([16384])
    run(q, k, v, g, p, kp)
    torch.cuda.synchronize()
    was = cel.timing(True)
    try:
        cel.kernel_stats(reset=True)
        whole = 0.0
        for _ in range(50):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            run(q, k, v, g, p, kp)
            b.record()
            b.synchronize()
            whole += a.elapsed_time(b)
        stats = cel.kernel_stats(reset=True)
    finally:
        cel.timing(was)
    assert stats["k_attention"][0] == stats["k_attention_dq"][0] == 50 and stats["k_attention_unite"][0] == 100
    assert sum(ms for _, ms in stats.values()) <= whole


def test_gradients_against_differences():
    """Of sums of float16 results at steps that 16 bits hold exactly: out's own roundings leave 2^-11 |out| of a value,
    independent ones, over the step; the second-order term is step^2 times the size of third derivatives."""
    T, U, H, K, d = 20, 30, 2, 1, 32
    q, k, v, g = batch(T, U, H, K, d, torch.float16, 4)
    q, k = (q / 2).half(), (k / 2).half()
    p, kp = ptr_of([12, 8]), ptr_of([17, 13])
    got = run(q, k, v, g, p, kp)
    total = lambda *x: float((cel.cross_attention(*x, p, kp)[0].double() * g.double()).sum())  # noqa: E731
    h = 0.125
    for n, name in enumerate(("dq", "dk", "dv")):
        sign = torch.randint(0, 2, got[name].shape, generator=torch.Generator().manual_seed(n)).to(DEV) * 2 - 1
        one, two = [[q, k, v] for _ in range(2)]
        base = ((q, k, v)[n].double() * 1024).round() / 1024
        one[n], two[n] = (base + h * sign).half(), (base - h * sign).half()
        by = one[n].double() - two[n].double()
        slope, want = total(*one) - total(*two), float((got[name].double() * by).sum())
        rounding = 6 * 2.0 ** -11 * float((got["out"].double() * g.double()).norm()) * 2 ** 0.5 + 2.0 ** -10 * float((got[name].double() * by).norm()) * 6
        assert abs(slope - want) <= rounding + 0.1 * float((got[name].double() * by).norm()), name


def test_refusals():
    def refused(f, *a, **kw):
        with pytest.raises(cel.CelError) as e:
            f(*a, **kw)
        assert e.value.code == -1

    q, k, v, g = batch(40, 50, 4, 2, 64, torch.bfloat16)
    p, kp = ptr_of([40]), ptr_of([50])
    out, lse = cel.cross_attention(q, k, v, p, kp)
    f, b = cel.cross_attention, cel.cross_attention_grad
    refused(f, q, k[:49], v, p, kp)
    refused(f, q, k[..., :56], v[..., :56], p, kp)
    refused(f, q, k.half(), v, p, kp)
    refused(f, q, k.repeat(1, 3, 1)[:, :3], v.repeat(1, 3, 1)[:, :3], p, kp)
    refused(f, q, k, v, p, ptr_of([20, 30]))
    refused(f, q, k, v, p, kp.long())
    refused(f, q, k, v, p.long(), kp)
    refused(f, q, k, v, p, kp.cpu())
    refused(f, q, k, v, p, kp, scale=0.0)
    refused(f, q.clone().requires_grad_(), k, v, p, kp)
    refused(b, g[:39], q, k, v, out, lse, p, kp)
    refused(b, g, q, k, v, out, lse[:, :39], p, kp)
    refused(b, g, q, k, v, out, lse.half(), p, kp)
    refused(b, g, q, k, v, out, lse, p, kp, grads=(q.clone(), k.clone()))
    refused(b, g, q, k, v, out, lse, p, kp, grads=(q.clone(), q.clone(), v.clone()))
