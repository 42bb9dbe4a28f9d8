"""What the C entry points of a block's operations refuse, and the scratch they ask for (CPU only:
every call ends before anything is enqueued)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2208_00184_amd", "libcel.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libcel.so not built")

ARG = -1
SOME = 1 << 20  # an address that is never looked at
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    pytest.importorskip("torch")
    from paper_2208_00184_amd import _binding
    return _binding.lib()


def b():
    from paper_2208_00184_amd import _binding
    return _binding


def rotary(**kw):
    d = dict(type=0, tokens=100, heads=4, dim=64, pairs=32, interleaved=0, n_axes=3, position_bytes=4, freq_bytes=4,
             positions=SOME, axis_stride=100, freqs=SOME, axes=SOME)
    d.update(kw)
    return b()._Rotary(*d.values())


def rows(p=SOME, row=4 * 64, head=64):
    return b()._Rows(p, row, head)


def matrix(p=SOME, stride=64):
    return ctypes.byref(b()._Matrix(p, stride))


def dropout(**kw):
    d = dict(type=0, rows=100, columns=64, p=0.1, seed=1, step=0, step_at=None)
    d.update(kw)
    mask = b()._Mask(d.pop("p"), d.pop("seed"), d.pop("step"), d.pop("step_at"))
    return b()._Dropout(*d.values(), mask)


def norm(**kw):
    d = dict(type=0, stream_type=0, param_type=2, center=0, rows=100, hidden=64, n_seq=0, seq_ptr=None, eps=1e-5, scale=1.0,
             pre=SOME, pre_bias=None, post=None, post_bias=None, gate=None, p=0.0)
    d.update(kw)
    return b()._Norm(*d.values()) if isinstance(d["p"], b()._Mask) else b()._Norm(*list(d.values())[:-1], b()._Mask(d["p"], 0, 0, None))


@pytest.mark.parametrize("bad", [dict(type=3), dict(type=-1), dict(tokens=-1), dict(heads=-1), dict(heads=65536), dict(dim=0),
                                 dict(dim=4097), dict(pairs=-1), dict(pairs=33), dict(n_axes=0), dict(axes=None),
                                 dict(axis_stride=-1), dict(position_bytes=2), dict(freq_bytes=2), dict(positions=None),
                                 dict(freqs=None)])
def test_rotary_descriptors(lib, bad):
    a, r = ctypes.byref(rotary(**bad)), ctypes.byref(rows())
    assert lib.cel_rotary(a, r, r, None) == ARG and lib.cel_rotary_grad(a, r, r, None) == ARG


@pytest.mark.parametrize("bad", [dict(p=None), dict(p=SOME + 1), dict(row=-1), dict(head=-1), dict(row=2 ** 41), dict(head=2 ** 41)])
def test_rotary_views(lib, bad):
    a, good, r = ctypes.byref(rotary()), ctypes.byref(rows()), ctypes.byref(rows(**bad))
    assert lib.cel_rotary(a, r, good, None) == ARG and lib.cel_rotary(a, good, r, None) == ARG
    assert lib.cel_rotary(a, None, good, None) == ARG and lib.cel_rotary(None, good, good, None) == ARG


@pytest.mark.parametrize("bad", [dict(type=3), dict(type=-1), dict(rows=-1), dict(rows=2 ** 32), dict(columns=-1),
                                 dict(columns=2 ** 31), dict(p=-0.1), dict(p=1.1), dict(p=NAN)])
def test_dropout_descriptors(lib, bad):
    assert lib.cel_dropout(ctypes.byref(dropout(**bad)), matrix(), matrix(), None) == ARG


def test_dropout_other_arguments(lib):
    a = ctypes.byref(dropout())
    assert lib.cel_dropout(None, matrix(), matrix(), None) == ARG
    for bad in (None, matrix(p=None), matrix(p=SOME + 1), matrix(stride=63), matrix(stride=2 ** 41)):
        assert lib.cel_dropout(a, bad, matrix(), None) == ARG and lib.cel_dropout(a, matrix(), bad, None) == ARG


BAD_NORM = [dict(type=3), dict(type=-1), dict(stream_type=1), dict(param_type=1), dict(type=2, stream_type=0), dict(rows=-1),
            dict(rows=2 ** 31), dict(hidden=0), dict(hidden=16385), dict(eps=-1e-6), dict(eps=NAN), dict(eps=INF),
            dict(scale=NAN), dict(scale=INF), dict(seq_ptr=SOME, n_seq=3), dict(seq_ptr=SOME, n_seq=-1, gate=SOME),
            dict(seq_ptr=SOME, n_seq=65531, gate=SOME), dict(pre=None, pre_bias=SOME), dict(post_bias=SOME), dict(p=1.5)]


@pytest.mark.parametrize("bad", BAD_NORM)
def test_norm_descriptors(lib, bad):
    a, m = ctypes.byref(norm(**bad)), matrix()
    g = ctypes.byref(b()._NormGrads(*[SOME] * 5))
    assert lib.cel_residual_norm_grad_scratch(a) == ARG
    assert lib.cel_residual_norm(a, m, m, m, m, None) == ARG
    assert lib.cel_residual_norm_grad(a, m, m, m, m, SOME, m, m, g, None) == ARG


def test_norm_other_arguments(lib):
    m = matrix()
    everything = dict(pre_bias=SOME, post=SOME, post_bias=SOME, gate=SOME)
    a = ctypes.byref(norm(**everything))
    g = ctypes.byref(b()._NormGrads(*[SOME] * 5))
    assert lib.cel_residual_norm(None, m, m, m, m, None) == ARG and lib.cel_residual_norm_grad_scratch(None) == ARG
    for bad in (None, matrix(p=None), matrix(p=SOME + 1), matrix(stride=63)):
        for at in range(4):
            args = [m] * 4
            args[at] = bad
            assert lib.cel_residual_norm(a, *args, None) == ARG
        for at in (0, 1, 2, 3, 5, 6):
            if at == 0 and bad is None:
                continue  # dy may be NULL
            args = [m, m, m, m, SOME, m, m]
            args[at] = bad
            assert lib.cel_residual_norm_grad(a, *args, g, None) == ARG
    assert lib.cel_residual_norm_grad(a, m, m, m, m, None, m, m, g, None) == ARG
    assert lib.cel_residual_norm_grad(a, m, m, m, m, SOME, m, m, None, None) == ARG
    for at in range(5):
        few = [SOME] * 5
        few[at] = None
        assert lib.cel_residual_norm_grad(a, m, m, m, m, SOME, m, m, ctypes.byref(b()._NormGrads(*few)), None) == ARG
    for alone in (dict(post=SOME), dict(gate=SOME), dict(p=0.5), dict(scale=2.0), dict(pre=None)):  # without a block's output
        a = ctypes.byref(norm(**alone))
        assert lib.cel_residual_norm(a, None, m, m, m, None) == ARG
        assert lib.cel_residual_norm_grad(a, m, m, None, m, SOME, m, None, g, None) == ARG
    none = ctypes.byref(norm(pre=None))
    assert lib.cel_residual_norm_grad(none, None, None, m, m, SOME, m, m, g, None) == ARG  # no gradient at all


def test_norm_scratch(lib):
    """Sums of five vectors of up to 256 workgroups, and one more of each sequence."""
    size = lambda **kw: lib.cel_residual_norm_grad_scratch(ctypes.byref(norm(**kw)))  # noqa: E731
    assert size() == 5 * 4 * 256 * 64
    assert size(gate=SOME, seq_ptr=SOME, n_seq=7, hidden=33) == 5 * 4 * 263 * 33
    assert size(rows=0, hidden=16384) == 5 * 4 * 256 * 16384


def test_the_tests_own_generator_is_the_published_one():
    """The known answers that its authors publish for Philox4x32 with ten rounds (and with seven)."""
    np = pytest.importorskip("numpy")
    from block_reference import philox
    ones = 0xffffffff
    for counter, key, rounds, want in (
            ([0] * 4, 0, 10, (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ([ones] * 4, ones << 32 | ones, 10, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], 0x299f31d0 << 32 | 0xa4093822, 10,
             (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
            ([0] * 4, 0, 7, (0x5f6fb709, 0x0d893f64, 0x4f121f81, 0x4f730a48))):
        assert tuple(int(x) for x in philox([np.uint64(c) for c in counter], key, rounds)) == want


def cross(**kw):
    r = rows()
    d = dict(type=0, tokens=100, keys=70, n_seq=2, heads=4, kv_heads=2, dim=64, scale=0.125, seq_ptr=SOME, key_ptr=SOME, q=r, k=r, v=r)
    d.update(kw)
    return b()._Cross(*d.values())


@pytest.mark.parametrize("bad", [dict(type=2), dict(tokens=-1), dict(keys=-1), dict(keys=2 ** 31 - 1), dict(n_seq=-1), dict(heads=0),
                                 dict(heads=5), dict(dim=12), dict(dim=136), dict(scale=0.0), dict(scale=NAN)])
def test_cross_descriptors(lib, bad):
    a, r = ctypes.byref(cross(**bad)), ctypes.byref(rows())
    assert lib.cel_cross_attention_grad_scratch(a) == ARG
    assert lib.cel_cross_attention(a, r, SOME, SOME, None) == ARG
    assert lib.cel_cross_attention_grad(a, r, SOME, r, SOME, r, r, r, None) == ARG


def test_cross_other_arguments(lib):
    r = ctypes.byref(rows())
    assert lib.cel_cross_attention_grad_scratch(None) == ARG
    assert lib.cel_cross_attention(None, r, SOME, SOME, None) == ARG
    assert lib.cel_cross_attention_grad(None, r, SOME, r, SOME, r, r, r, None) == ARG
    for bad in (dict(seq_ptr=None), dict(key_ptr=None), dict(q=rows(p=None)), dict(k=rows(p=SOME + 8)), dict(v=rows(row=60))):
        a = ctypes.byref(cross(**bad))
        assert lib.cel_cross_attention(a, r, SOME, SOME, None) == ARG
        assert lib.cel_cross_attention_grad(a, r, SOME, r, SOME, r, r, r, None) == ARG
    a = ctypes.byref(cross())
    assert lib.cel_cross_attention(a, None, SOME, SOME, None) == ARG and lib.cel_cross_attention(a, r, None, SOME, None) == ARG
    for at in range(7):
        args = [r, SOME, r, SOME, r, r, r]
        args[at] = None
        assert lib.cel_cross_attention_grad(a, *args, None) == ARG
    # 2^24 workgroups of the keys' launch
    big = ctypes.byref(cross(keys=2 ** 24, heads=64, kv_heads=8))
    assert lib.cel_cross_attention_grad_scratch(big) == ARG
    assert lib.cel_cross_attention_grad(big, r, SOME, r, SOME, r, r, r, None) == ARG


def test_cross_scratch(lib):
    size = lambda **kw: lib.cel_cross_attention_grad_scratch(ctypes.byref(cross(**kw)))  # noqa: E731
    assert size() == 4 * (2 * 4 * 100 + 2 * 2 * 70 * 2 * 64)
    assert size(kv_heads=4) == 4 * 2 * 4 * 100
    assert size(tokens=0, kv_heads=4) == 0 and size(tokens=0, keys=0) == 0
    few = lambda **kw: lib.cel_cross_attention_scratch(ctypes.byref(cross(**kw)))  # noqa: E731
    assert few() == 0 and lib.cel_cross_attention_scratch(None) == ARG and few(tokens=-1) == ARG
    # more workgroups than fit at once: the tiles' order, of rows, and in the gradient of keys too
    big = dict(tokens=10000, keys=20000, heads=64, kv_heads=64)
    assert few(**big) == 4 * 79 and few(n_seq=1, **big) == 0 and few(**{**big, "tokens": 4097 * 128}) == 0
    assert size(**big) == 4 * (2 * 64 * 10000 + 79 + 313)
    a, r = ctypes.byref(cross(**big, q=rows(row=64 * 64), k=rows(row=64 * 64), v=rows(row=64 * 64))), ctypes.byref(rows(row=64 * 64))
    assert lib.cel_cross_attention(a, r, SOME, None, None) == ARG
