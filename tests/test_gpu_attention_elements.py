"""cel.attention and cel.attention_grad element by element (attention_bounds): every value
against a bound of its own, so that no row hides behind the others; batches whose
launches are large, where workgroups take their tiles in another order and key/value heads
deal out their query heads unevenly; and infinities and NaN in every type and kernel."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU, skipped there
    pytest.skip("needs a ROCm GPU", allow_module_level=True)

import paper_2208_00184_amd as cel  # noqa: E402
from attention_bounds import definition, outside, unseen_zero_rows  # noqa: E402

DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16]


def batch(T, H, K, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(T, n, d, generator=g).to(dtype) for n in (H, K, K, H)]


def run(q, k, v, dout, ptr):
    q, k, v, dout = (x.to(DEV) for x in (q, k, v, dout))
    out, lse = cel.attention(q, k, v, ptr)
    dq, dk, dv = cel.attention_grad(dout, q, k, v, out, lse, ptr)
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)


def ptr_of(lengths, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lengths)]).astype(np.int32), device=DEV)


def check(q, k, v, dout, lengths, first=0):
    expected = definition(q, k, v, dout, lengths, first)
    for n in ("out", "dq", "dk", "dv"):  # the bounds see a missing row, but for one in a hundred at most
        assert unseen_zero_rows(expected, n) <= q.shape[0] * q.shape[1] // 100
    got = run(q, k, v, dout, ptr_of(lengths, first))
    bad = {n: outside(expected, n, x) for n, x in got.items()}
    assert not any(n for n, _ in bad.values()), bad


def ragged(total, mean, seed):
    """Lengths around `mean`, some of one token and of none, and one of more than 600."""
    rng = np.random.default_rng(seed)
    out = [617, 1, 0]
    while sum(out) < total:
        out.append(min(int(rng.integers(1, 2 * mean)), total - sum(out)))
    return [int(x) for x in rng.permutation(out)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [8, 32, 40, 64, 80, 96, 128])
def test_dimensions(d, dtype):
    check(*batch(410, 4, 2, d, dtype, d), [150, 1, 0, 33, 64, 129, 30], 3)


@pytest.mark.parametrize("lengths", [[1], [2], [31], [33], [63], [64], [65], [127], [129], [191], [193], [257], [700], [1] * 70,
                                     [511, 1], [1100], [2500, 500]])
@pytest.mark.parametrize("d,dtype", [(64, torch.bfloat16), (128, torch.float16), (32, torch.float16), (96, torch.bfloat16)])
def test_lengths(lengths, d, dtype):
    check(*batch(sum(lengths), 2, 1, d, dtype, sum(lengths)), lengths)


@pytest.mark.parametrize("T,mean,H,K", [
    (1100, 100, 32, 32),   # 288 workgroups: keys with one group of waves; dies take theirs forwards and backwards
    (6301, 60, 40, 8),     # five query heads a key/value head, dealt out 2, 2, 1; 2,000 workgroups forward
    (12289, 60, 16, 8),    # two query heads a key/value head, in one part
    (4097, 90, 5, 1),      # five in five parts, behind an odd number of rows in the scratch
    (2049, 200, 33, 3)])   # heads that no power of two divides
@pytest.mark.parametrize("d,dtype", [(64, torch.bfloat16), (128, torch.float16)])
def test_large_launches(T, mean, H, K, d, dtype):
    lengths = ragged(T - 9, mean, T + H)
    check(*batch(T, H, K, d, dtype, T), lengths, 4)


def test_four_whole_sequences():
    """512 workgroups, two a compute unit: the order whose second half comes backwards."""
    check(*batch(4096, 16, 16, 64, torch.bfloat16, 5), [1024] * 4)


# keys with one group of waves (few tokens, or many heads) and with two
BATCHES = [([60, 200, 90], 2, 1), ([100, 400, 200], 2, 1), ([100, 400, 60], 64, 32)]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("lengths,H,K", BATCHES)
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("dtype", TYPES)
def test_one_value_that_is_no_number(dtype, d, lengths, H, K, bad):
    """In one dimension of one token of v, then of dout: which elements are finite follows
    from the formulas, and those that are keep their bits."""
    T, at, c = sum(lengths), lengths[0] + 97, 5
    q, k, v, g = batch(T, H, K, d, dtype, d + T)
    ptr = ptr_of(lengths)
    plain = run(q, k, v, g, ptr)
    first, end = lengths[0], lengths[0] + lengths[1]  # the second sequence
    kv, group = K - 1, H // K
    heads = torch.zeros(H, dtype=torch.bool)
    heads[kv * group:] = True

    def same(name, got, touched):
        touched = touched.to(DEV)
        assert torch.equal(got[~touched], plain[name][~touched]), name
        assert not torch.isfinite(got[touched]).any(), name

    # v: out of the rows that see it, in that dimension alone; lse and dv hold no v; D of those rows, so all
    # of their dq, and dk of every key that they see
    v2 = v.clone()
    v2[at, kv, c] = bad
    got = run(q, k, v2, g, ptr)
    rows = torch.zeros(T, H, d, dtype=torch.bool)
    rows[at:end] = heads[:, None]
    touched = rows.clone()
    touched[:, :, :c] = False
    touched[:, :, c + 1:] = False
    same("out", got["out"], touched)
    assert torch.equal(got["lse"], plain["lse"]) and torch.equal(got["dv"], plain["dv"])
    same("dq", got["dq"], rows)
    keys = torch.zeros(T, K, d, dtype=torch.bool)
    keys[first:end, kv] = True  # the sequence's last row sees all of it
    same("dk", got["dk"], keys)
    # dout: D and dp of its own row, so its dq, and dk of the keys it sees; dv of those keys in that dimension alone
    g2 = g.clone()
    h = H - 1
    g2[at, h, c] = bad
    got = run(q, k, v, g2, ptr)
    assert torch.equal(got["out"], plain["out"]) and torch.equal(got["lse"], plain["lse"])
    rows = torch.zeros(T, H, d, dtype=torch.bool)
    rows[at, h] = True
    same("dq", got["dq"], rows)
    keys = torch.zeros(T, K, d, dtype=torch.bool)
    keys[first:at + 1, kv] = True
    same("dk", got["dk"], keys)
    keys[:, :, :c] = False
    keys[:, :, c + 1:] = False
    same("dv", got["dv"], keys)


@pytest.mark.parametrize("lengths,H,K", BATCHES)
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("dtype", TYPES)
def test_padding_may_hold_anything(dtype, d, lengths, H, K):
    first, T = 20, sum(lengths) + 45
    x = batch(T, H, K, d, dtype, d)
    ptr = ptr_of(lengths, first)
    plain = run(*x, ptr)
    for t in x:
        t[:first] = float("nan")
        t[first + sum(lengths):] = float("inf")
    for n, got in run(*x, ptr).items():
        assert torch.equal(got, plain[n]), n


@pytest.mark.parametrize("lengths,H,K", BATCHES)
@pytest.mark.parametrize("d,dtype", [(64, torch.bfloat16), (128, torch.float16)])
@pytest.mark.parametrize("by", [30.0, -30.0, 0.0])
def test_a_row_does_not_hang_on_its_neighbours(by, d, dtype, lengths, H, K):
    """Other tokens' queries and gradients, and later tokens' keys and values, change no bit of a row, also
    where their scores are large."""
    T, at = sum(lengths), lengths[0] + 97
    q, k, v, g = batch(T, H, K, d, dtype, 3 * d + T)
    ptr = ptr_of(lengths)
    plain = run(q, k, v, g, ptr)
    others = (torch.arange(T) % 7 != 3).to(DEV)
    q2, g2 = q.clone(), g.clone()
    q2[~others.cpu()] *= by
    g2[~others.cpu()] *= by
    got = run(q2, k, v, g2, ptr)
    for n in ("out", "dq"):
        assert torch.equal(got[n][others], plain[n][others]), n
    assert torch.equal(got["lse"][:, others], plain["lse"][:, others])
    k2, v2 = k.clone(), v.clone()
    k2[at:at + 3] *= by
    v2[at:at + 3] *= by
    got = run(q, k2, v2, g, ptr)
    before = slice(0, at)
    assert torch.equal(got["out"][before], plain["out"][before]) and torch.equal(got["dq"][before], plain["dq"][before])
    assert torch.equal(got["lse"][:, before], plain["lse"][:, before])
    end = lengths[0] + lengths[1]
    for n in ("out", "dq", "dk", "dv"):
        assert torch.equal(got[n][end:], plain[n][end:]), n


@pytest.mark.parametrize("lengths", [[90, 20, 10], [30, 34, 40, 24], [128], [70, 1, 2, 3, 4, 5, 6, 7], [64, 64], [60, 3, 1, 50]])
@pytest.mark.parametrize("H,K,d", [(2, 1, 64), (3, 3, 128), (4, 2, 80)])
@pytest.mark.parametrize("more", [0, 600])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_few_keys(dtype, more, H, K, d, lengths):
    """D of a row whose keys lie in one tile of 64 is a sum in 32 bits: where few values are averaged out is
    as large as they are, and its rounding would weigh as much as all else.  Within one block of 128 tokens
    the tiles are the tokens 0 to 63 and 64 to 127; `more` others in front make a block of their own."""
    assert sum(lengths) <= 128
    ends = np.cumsum(lengths)
    starts = ends - lengths
    wide = torch.zeros(more + 128, dtype=torch.bool)
    for a, b in zip(starts, ends):
        for t in range(a, b):
            wide[more + int(t)] = int(a) // 64 == int(t) // 64
    before = [more] if more else []
    # the block of 128 tokens has to begin with its sequences
    first = -more % 128
    T = first + more + 128
    q, k, v, g = batch(T, H, K, d, dtype, d + more + len(lengths))
    expected = definition(q, k, v, g, before + lengths, first, wide=torch.cat([torch.zeros(first, dtype=torch.bool), wide]))
    got = run(q, k, v, g, ptr_of(before + lengths, first))
    bad = {n: outside(expected, n, x) for n, x in got.items()}
    assert not any(n for n, _ in bad.values()), bad
