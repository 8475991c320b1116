"""Argument checks of the cache and attention calls, which end before anything touches a device, and the definitions that the GPU tests
compare with (no GPU)."""
import ctypes as C

import numpy as np
import pytest

import _attention as ref
from test_abi import LIB

EINVAL, ESHAPE = -1, -2
I = C.c_int64
BUF = C.c_void_p(4096)          # never dereferenced: validation fails first, or there is nothing to do
F = C.c_float


@pytest.fixture(scope="module")
def lib():
    return C.CDLL(LIB)


def test_page_bytes(lib):
    lib.pipe_cache_page_bytes.restype = I
    for P in (16, 32, 64, 128, 256):
        for D in (64, 128):
            assert lib.pipe_cache_page_bytes(3, D, P) == 3 * P * (D + 8)
    for bad in ((0, 64, 16), (1, 80, 16), (1, 64, 48), (1, 64, 8), (1, 64, 512), (70000, 64, 16)):
        assert lib.pipe_cache_page_bytes(*bad) == 0


def plan(lib, **o):
    a = dict(cached=BUF, fresh=BUF, B=4, P=16, free=BUF, n_free=8, used=BUF, table=BUF, width=4, T=4, lengths=BUF, starts=BUF, slots=BUF,
             positions=BUF, counts=C.c_void_p(8192))
    a.update(o)
    return lib.pipe_cache_plan(*a.values(), None)


def test_plan_refusals(lib):
    for name in ("cached", "fresh", "used", "table", "lengths", "starts", "slots", "positions", "counts", "free"):
        assert plan(lib, **{name: None}) == EINVAL, name
    assert plan(lib, P=17) == EINVAL and plan(lib, P=0) == EINVAL and plan(lib, P=-16) == EINVAL
    for bad in (dict(B=0), dict(B=4097), dict(T=-1), dict(width=0), dict(n_free=-1)):
        assert plan(lib, **bad) == ESHAPE, bad
    for at in (4096 - 8, 4096 - 4, 4096):            # counts over used
        assert plan(lib, counts=C.c_void_p(at)) == EINVAL


def write(lib, **o):
    a = dict(k=BUF, v=BUF, type=2, T=4, H=2, D=64, kt=I(128), kh=I(64), vt=I(128), vh=I(64), slots=BUF, cache=BUF, pages=4, P=16)
    a.update(o)
    return lib.pipe_cache_write(*a.values(), None)


def read(lib, **o):
    a = dict(cache=BUF, pages=4, P=16, slots=BUF, T=4, H=2, D=64, type=0, k=BUF, v=BUF)
    a.update(o)
    return lib.pipe_cache_read(*a.values(), None)


def test_write_and_read_refusals(lib):
    for f in (write, read):
        for name in ("k", "v", "slots", "cache"):
            assert f(lib, **{name: None}) == EINVAL, name
        for bad in (dict(type=3), dict(type=-1), dict(P=20), dict(cache=C.c_void_p(4100))):
            assert f(lib, **bad) == EINVAL, bad
        for bad in (dict(T=-1), dict(H=0), dict(D=96), dict(pages=0), dict(pages=1 << 27), dict(T=1 << 30, H=4)):
            assert f(lib, **bad) == ESHAPE, bad
        assert f(lib, T=0, k=None, v=None, slots=None) == 0
    for name in ("kt", "kh", "vt", "vh"):
        assert write(lib, **{name: I(-1)}) == ESHAPE
    assert read(lib, k=C.c_void_p(4104)) == EINVAL


def attend(lib, **o):
    a = dict(q=BUF, type=0, T=4, Hq=8, Hkv=2, D=64, qt=I(512), qh=I(64), starts=BUF, lengths=BUF, B=2, cache=BUF, pages=4, P=16, table=BUF, width=2,
             scale=F(0.1), hint=0, out=BUF)
    a.update(o)
    return lib.pipe_cache_attention(*a.values(), None)


def prompt(lib, **o):
    a = dict(q=BUF, k=BUF, v=BUF, type=0, Tq=4, Tk=4, Hq=8, Hkv=2, D=64, qt=I(512), qh=I(64), kt=I(128), kh=I(64), vt=I(128), vh=I(64), qs=BUF,
             ks=None, B=2, causal=1, scale=F(0.1), out=BUF)
    a.update(o)
    return lib.pipe_prompt_attention(*a.values(), None)


def test_attention_refusals(lib):
    for f, names in ((attend, ("q", "starts", "lengths", "cache", "table", "out")), (prompt, ("q", "k", "v", "qs", "out"))):
        for name in names:
            assert f(lib, **{name: None}) == EINVAL, name
        for bad in (dict(type=5), dict(scale=F(float("nan"))), dict(scale=F(float("inf"))), dict(out=C.c_void_p(4104))):
            assert f(lib, **bad) == EINVAL, bad
        for bad in (dict(Hq=7), dict(Hkv=0), dict(Hq=1), dict(D=32), dict(B=0), dict(qt=I(-1)), dict(qh=I(-64))):
            assert f(lib, **bad) == ESHAPE, bad
    for bad in (dict(T=-1), dict(width=0), dict(hint=-1), dict(pages=0), dict(T=1 << 29)):
        assert attend(lib, **bad) == ESHAPE, bad
    assert attend(lib, P=40) == EINVAL
    assert attend(lib, T=100000, width=1 << 30) == ESHAPE               # more steps than a launch counts
    for bad in (dict(Tq=-1), dict(Tk=-1), dict(Tk=5), dict(kt=I(-1)), dict(vh=I(-1)), dict(Tq=1 << 29, Tk=1 << 29)):
        assert prompt(lib, **bad) == ESHAPE, bad
    assert prompt(lib, causal=2) == EINVAL
    assert attend(lib, T=0) == 0 and prompt(lib, Tq=0, Tk=0) == 0       # nothing to do
    assert lib.pipe_prepare_cache_attention(0, 8, 2, 64, 1, 100, None) == EINVAL
    assert lib.pipe_prepare_cache_attention(4, 8, 2, 64, 1, 0, None) == EINVAL
    assert lib.pipe_prepare_cache_attention(4, 8, 2, 96, 1, 100, None) == ESHAPE


def test_rows_are_held_to_half_a_step():
    """The definition itself: every value of a finite row lies within half a step of what its code stands for."""
    rng = np.random.default_rng(0)
    for gain in (1e-30, 1e-3, 1.0, 7e8, 1e37):
        x = (rng.standard_normal((200, 64)) * gain).astype(np.float32)
        c, s, m = ref.quantize_rows(x)
        assert c.max() == 15 and c.min() == 0
        err = np.abs(s.astype(np.float64) * c + m - x)
        assert np.all(err <= 0.5 * s + 16 * ref.U32 * (15 * s.astype(np.float64) + np.abs(m)))


def test_attend_of_rows_that_see_nothing():
    q = np.ones((3, 2, 4))
    k = v = np.ones((2, 1, 4))
    out = ref.attend(q, k, v, 0.5, [-1, 0, 1])
    assert not out[:2].any() and np.allclose(out[2], 1.0)
