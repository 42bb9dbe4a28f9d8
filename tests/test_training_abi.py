"""What the C entry points of the training-step operations refuse, and the scratch
they ask for (CPU only: every call ends before anything is enqueued)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2208_00184_amd", "libcel.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libcel.so not built")

ARG = -1
SOME = 1 << 20  # an address that is never looked at


@pytest.fixture(scope="module")
def lib():
    pytest.importorskip("torch")
    from paper_2208_00184_amd import _binding
    return _binding.lib()


def attn(**kw):
    from paper_2208_00184_amd import _binding as b
    rows = b._Rows(SOME, 4 * 64, 64)
    d = dict(type=0, tokens=100, n_seq=2, heads=4, kv_heads=2, dim=64, scale=0.125, seq_ptr=SOME, q=rows, k=rows, v=rows)
    d.update(kw)
    return b._Attn(*d.values())


def embed(**kw):
    from paper_2208_00184_amd import _binding as b
    d = dict(type=0, id_bytes=4, tokens=100, vocab=50, hidden=24, stride=24, ids=SOME, scale=1.0)
    d.update(kw)
    return b._Embed(*d.values())


def rows(p=SOME, row=4 * 64, head=64):
    from paper_2208_00184_amd import _binding as b
    return b._Rows(p, row, head)


BAD_ATTN = [dict(type=2), dict(type=-1), dict(tokens=-1), dict(n_seq=-1), dict(heads=0), dict(kv_heads=0),
            dict(heads=5), dict(dim=0), dict(dim=12), dict(dim=136), dict(scale=0.0), dict(scale=-1.0),
            dict(scale=float("nan")), dict(scale=float("inf")), dict(tokens=2 ** 31 - 5000, heads=65534)]


@pytest.mark.parametrize("bad", BAD_ATTN)
def test_attention_descriptors(lib, bad):
    a, r = attn(**bad), ctypes.byref(rows())
    assert lib.cel_attention_grad_scratch(ctypes.byref(a)) == ARG
    assert lib.cel_attention(ctypes.byref(a), r, ctypes.c_void_p(SOME), None) == ARG
    p = ctypes.c_void_p(SOME)
    assert lib.cel_attention_grad(ctypes.byref(a), r, p, r, p, r, r, r, None) == ARG


@pytest.mark.parametrize("bad", [dict(p=None), dict(p=SOME + 8), dict(row=4 * 64 + 4), dict(head=68), dict(row=56),
                                 dict(head=-8), dict(row=2 ** 23 + 8)])
def test_attention_views(lib, bad):
    p, good, r = ctypes.c_void_p(SOME), rows(), rows(**bad)
    for name in ("q", "k", "v"):
        a = attn(**{name: r})
        assert lib.cel_attention(ctypes.byref(a), ctypes.byref(good), p, None) == ARG
    a = attn()
    assert lib.cel_attention(ctypes.byref(a), ctypes.byref(r), p, None) == ARG
    for at in (1, 3, 5, 6, 7):
        args = [ctypes.byref(a), ctypes.byref(good), p, ctypes.byref(good), p] + [ctypes.byref(good)] * 3 + [None]
        args[at] = ctypes.byref(r)
        assert lib.cel_attention_grad(*args) == ARG


def test_attention_null_arguments(lib):
    a, r, p = ctypes.byref(attn()), ctypes.byref(rows()), ctypes.c_void_p(SOME)
    assert lib.cel_attention_grad_scratch(None) == ARG
    assert lib.cel_attention(None, r, p, None) == ARG
    assert lib.cel_attention(a, None, p, None) == ARG
    assert lib.cel_attention(a, r, None, None) == ARG
    assert lib.cel_attention(ctypes.byref(attn(seq_ptr=None)), r, p, None) == ARG
    for at in range(8):
        args = [a, r, p, r, p, r, r, r]
        args[at] = None
        assert lib.cel_attention_grad(*args, None) == ARG


def test_attention_scratch(lib):
    """lse and D of every row; from 2 parts on, dk and dv of every part in 32 bits."""
    assert lib.cel_attention_grad_scratch(ctypes.byref(attn(kv_heads=4, seq_ptr=None))) == 4 * 2 * 4 * 100
    assert lib.cel_attention_grad_scratch(ctypes.byref(attn(tokens=0))) == 0
    few = lib.cel_attention_grad_scratch(ctypes.byref(attn()))
    assert few == 4 * (2 * 4 * 100 + 2 * 2 * 100 * 2 * 64)


@pytest.mark.parametrize("bad", [dict(type=3), dict(type=-1), dict(id_bytes=2), dict(tokens=-1), dict(tokens=2 ** 31),
                                 dict(vocab=0), dict(vocab=2 ** 31), dict(hidden=0), dict(hidden=2 ** 24 + 1),
                                 dict(stride=23), dict(ids=None), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_embed_descriptors(lib, bad):
    e, p = ctypes.byref(embed(**bad)), ctypes.c_void_p(SOME)
    assert lib.cel_embed(e, p, p, None) == ARG
    assert lib.cel_embed_grad(e, p, p, 2, p, None) == ARG


def test_embed_other_arguments(lib):
    e, p = ctypes.byref(embed()), ctypes.c_void_p(SOME)
    assert lib.cel_embed(None, p, p, None) == ARG
    assert lib.cel_embed(e, None, p, None) == ARG and lib.cel_embed(e, p, None, None) == ARG
    assert lib.cel_embed_grad(None, p, p, 2, p, None) == ARG
    assert lib.cel_embed_grad(e, None, p, 2, p, None) == ARG
    assert lib.cel_embed_grad(e, p, None, 2, p, None) == ARG
    assert lib.cel_embed_grad(e, p, p, 2, None, None) == ARG
    assert lib.cel_embed_grad(e, p, p, 1, p, None) == ARG  # bfloat16 rows, float16 gradient
    assert lib.cel_embed_grad_scratch(-1, 10, 10) == ARG
    assert lib.cel_embed_grad_scratch(10, 0, 10) == ARG
    assert lib.cel_embed_grad_scratch(10, 10, 0) == ARG
    assert lib.cel_embed_grad_scratch(0, 10, 10) >= 4 * 11


def test_attention_scratch_of_an_odd_number_of_rows(lib):
    """The parts lie behind 2 x 3 x 137 numbers, rounded up to 16 bytes for their vectors of four."""
    a = attn(tokens=137, heads=3, kv_heads=1, q=rows(row=3 * 64), seq_ptr=None)
    assert lib.cel_attention_grad_scratch(ctypes.byref(a)) == 4 * (824 + 2 * 3 * 137 * 64)


def test_attention_launches_stay_below_what_a_grid_takes(lib):
    """2^24 workgroups of 256 threads are one too many: refused before anything is enqueued."""
    r, p = ctypes.byref(rows()), ctypes.c_void_p(SOME)
    for kw, forward in ((dict(tokens=2 ** 26, heads=64, kv_heads=64), True), (dict(tokens=2 ** 24, heads=64, kv_heads=8), False)):
        a = attn(**kw)
        assert lib.cel_attention_grad_scratch(ctypes.byref(a)) == ARG
        assert lib.cel_attention_grad(ctypes.byref(a), r, p, r, p, r, r, r, None) == ARG
        if forward:
            assert lib.cel_attention(ctypes.byref(a), r, p, None) == ARG
    assert lib.cel_attention_grad_scratch(ctypes.byref(attn(tokens=2 ** 24 - 64, heads=64, kv_heads=64))) > 0


@pytest.mark.parametrize("scale", [3e38, 2.5e38, 1e-38, 1e-45])
def test_attention_scales_that_exponents_do_not_hold(lib, scale):
    """log2(e) times the scale, or 8 over it, is not finite in 32 bits."""
    a, r, p = attn(scale=scale), ctypes.byref(rows()), ctypes.c_void_p(SOME)
    assert lib.cel_attention_grad_scratch(ctypes.byref(a)) == ARG
    assert lib.cel_attention(ctypes.byref(a), r, p, None) == ARG
    assert lib.cel_attention_grad(ctypes.byref(a), r, p, r, p, r, r, r, None) == ARG
