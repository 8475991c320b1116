"""Argument checks of the calls with a scale for each token and of the experts' calls, which end before anything touches a device, and the definitions that the
GPU tests compare with (no GPU)."""
import ctypes as C
import os

import numpy as np
import pytest

import _experts as ref
from test_abi import LIB, ROOT

EINVAL, ESHAPE = -1, -2
I = C.c_int64
BUF = C.c_void_p(4096)          # never dereferenced: validation fails first, or there is nothing to do
ODD = C.c_void_p(4104)


@pytest.fixture(scope="module")
def lib():
    return C.CDLL(LIB)


def test_sizes(lib):
    lib.pipe_token_scratch.restype = I
    for n, pitch in ((1, 128), (127, 128), (128, 128), (129, 256), (4096, 4096), (130944, 130944)):
        assert lib.pipe_token_pitch(n) == pitch
        assert lib.pipe_token_scratch(I(7), n) == 7 * (pitch + 4)
    assert lib.pipe_token_pitch(0) == 0 and lib.pipe_token_pitch(-5) == 0 and lib.pipe_token_pitch(130945) == 0
    assert lib.pipe_token_scratch(I(0), 8) == 0 and lib.pipe_token_scratch(I(-1), 8) == -1 and lib.pipe_token_scratch(I(3), 0) == -1
    assert lib.pipe_token_scratch(I(1 << 30), 8) == -1
    assert 127 * 127 * 130944 < 2 ** 31 and 127 * 128 * 130944 < 2 ** 31


def quantize(lib, **o):
    a = dict(x=BUF, type=2, rows=I(4), n=100, stride=I(100), codes=BUF, scales=BUF)
    a.update(o)
    return lib.pipe_token_quantize(*a.values(), None)


def test_quantize_refusals(lib):
    for name in ("x", "codes", "scales"):
        assert quantize(lib, **{name: None}) == EINVAL, name
    for bad in (dict(type=3), dict(type=-1), dict(codes=ODD)):
        assert quantize(lib, **bad) == EINVAL, bad
    for bad in (dict(rows=I(-1)), dict(rows=I(1 << 30)), dict(n=0), dict(n=130945), dict(stride=I(-1))):
        assert quantize(lib, **bad) == ESHAPE, bad
    assert quantize(lib, rows=I(0), x=None, codes=None, scales=None) == 0


def forward(lib, **o):
    a = dict(x=BUF, type=2, T=I(4), n=100, stride=I(100), codes=BUF, scales=BUF, bias=None, out=33, act=0, scratch=BUF, y=BUF)
    a.update(o)
    return lib.pipe_token_forward(*a.values(), None)


def experts(lib, **o):
    a = dict(x=BUF, type=2, T=I(4), n=100, stride=I(100), codes=BUF, scales=BUF, bias=None, E=3, out=33, starts=BUF, order=BUF, rows=I(8), k=2, act=0,
             scratch=BUF, y=BUF)
    a.update(o)
    return lib.pipe_expert_forward(*a.values(), None)


def test_layer_refusals(lib):
    for f in (forward, experts):
        for name in ("x", "codes", "scales", "y"):
            assert f(lib, **{name: None}) == EINVAL, name
        for T in (65, 100000):                   # more than 8192 codes need room
            assert f(lib, T=I(T), scratch=None, **({"rows": I(2 * T)} if f is experts else {})) == EINVAL
        for bad in (dict(type=4), dict(act=4), dict(act=-1), dict(codes=ODD), dict(y=ODD), dict(scratch=ODD)):
            assert f(lib, **bad) == EINVAL, bad
        for bad in (dict(T=I(-1)), dict(T=I(1 << 30)), dict(n=0), dict(n=131000), dict(stride=I(-1)), dict(out=0), dict(out=(1 << 28) + 1)):
            assert f(lib, **bad) == ESHAPE, bad
    assert forward(lib, T=I(0), x=None, y=None, scratch=None) == 0
    assert experts(lib, rows=I(0), x=None, y=None, scratch=None, starts=None) == 0
    assert experts(lib, starts=None) == EINVAL
    for bad in (dict(E=0), dict(E=1025), dict(k=0), dict(k=33), dict(rows=I(-1)), dict(rows=I(1 << 30)), dict(order=None), dict(T=I(0))):
        assert experts(lib, **bad) == ESHAPE, bad


def test_layers_without_scratch(lib):
    """NULL for the scratch is refused wherever the codes have a launch of their own: of few codes too, where outputs are many, lie over the input, or the kernel is set."""
    apart = dict(x=C.c_void_p(1 << 20), y=C.c_void_p(1 << 30), scratch=None)
    for f, one in ((forward, {}), (experts, dict(E=3, rows=I(1), order=BUF, k=1))):
        for out in (16385, 40000, 1 << 28):
            assert f(lib, **apart, T=I(1), n=4096, out=out, **one) == EINVAL
        assert f(lib, **apart, T=I(3), n=4096, out=8, **(dict(one, rows=I(3)) if one else {})) == EINVAL
        for shift, out in ((0, 8), (16, 8), (192, 8), (-16, 16)):                # a row of 100 fp16 values, 200 bytes
            assert f(lib, **dict(apart, y=C.c_void_p((1 << 20) + shift)), T=I(1), out=out, type=1, **one) == EINVAL
        try:
            for which in (2, 3, 4):
                assert lib.pipe_set_token_kernel(which) == 0
                assert f(lib, **apart, T=I(1), out=8, **one) == EINVAL
        finally:
            assert lib.pipe_set_token_kernel(0) == 0
    # experts: a tile for each that may have a row
    assert experts(lib, **apart, T=I(30), n=100, E=1024, rows=I(60), order=BUF, k=2, out=257) == EINVAL


def route(lib, **o):
    a = dict(logits=BUF, type=0, T=4, E=8, stride=I(8), k=2, renormalize=1, experts=BUF, weights=BUF, starts=BUF, order=BUF, places=BUF, scratch=BUF)
    a.update(o)
    return lib.pipe_expert_route(*a.values(), None)


def sort(lib, **o):
    a = dict(experts=BUF, T=4, k=2, E=8, starts=BUF, order=BUF, places=BUF, scratch=BUF)
    a.update(o)
    return lib.pipe_expert_sort(*a.values(), None)


def combine(lib, **o):
    a = dict(y=BUF, type=1, rows=I(8), out=100, stride=I(100), places=BUF, weights=BUF, T=4, k=2, dst=BUF)
    a.update(o)
    return lib.pipe_expert_combine(*a.values(), None)


def test_router_refusals(lib):
    for f, names in ((route, ("logits", "experts", "weights", "starts", "order", "places")), (sort, ("experts", "starts", "order", "places")),
                     (combine, ("y", "places", "weights", "dst"))):
        for name in names:
            assert f(lib, **{name: None}) == EINVAL, name
        for bad in (dict(T=-1), dict(k=0), dict(k=33), dict(T=1 << 29)):
            assert f(lib, **bad) == ESHAPE, bad
    for f in (route, sort):
        for bad in (dict(E=0), dict(E=1025)):
            assert f(lib, **bad) == ESHAPE, bad
        assert f(lib, T=600, scratch=None) == EINVAL and f(lib, T=600, scratch=ODD) == EINVAL
    lib.pipe_expert_scratch.restype = I
    for k in range(1, 33):                       # whole tokens of up to 512 pairs a block
        assert lib.pipe_expert_scratch(481 // k, k, 8) == 0 and lib.pipe_expert_scratch(512 // k, k, 8) == 0
        assert lib.pipe_expert_scratch(512 // k + 1, k, 8) == 2 * 12 * 2
    assert lib.pipe_expert_scratch(0, 3, 5) == 0
    assert lib.pipe_expert_scratch(128 * 256, 2, 8) == 128 * 12 * 2 and lib.pipe_expert_scratch(128 * 256 + 1, 2, 8) == 3104
    # sums by a launch of their own: of more than 512 blocks, and of more than 36864 counts
    assert lib.pipe_expert_scratch(512 * 256, 2, 8) == 512 * 12 * 2 and lib.pipe_expert_scratch(512 * 256 + 1, 2, 8) == 12320 + 514 * 12 * 4
    assert lib.pipe_expert_scratch(354 * 64, 8, 100) == 73632 and lib.pipe_expert_scratch(354 * 64 + 1, 8, 100) == 73840 + 356 * 104 * 4
    for bad in ((-1, 2, 8), (4, 0, 8), (4, 33, 8), (4, 2, 0), (4, 2, 1025), (1 << 29, 2, 8)):
        assert lib.pipe_expert_scratch(*bad) == -1
    for bad in (dict(type=3), dict(renormalize=2)):
        assert route(lib, **bad) == EINVAL
    for bad in (dict(k=9), dict(stride=I(-1))):
        assert route(lib, **bad) == ESHAPE
    assert combine(lib, type=-1) == EINVAL
    for bad in (dict(rows=I(-1)), dict(rows=I(1 << 30)), dict(out=0), dict(stride=I(-1))):
        assert combine(lib, **bad) == ESHAPE, bad
    assert combine(lib, T=0, places=None, weights=None, dst=None) == 0


def test_512_pairs_need_no_scratch(lib):
    lib.pipe_expert_scratch.restype = I
    for k in range(1, 33):
        assert all(lib.pipe_expert_scratch(T, k, 1024) == 0 for T in range(512 // k + 1))
    header = open(os.path.join(ROOT, "include", "pipe.h")).read()
    assert "T * top_k <= 512; -1: no such router" in header


def test_quantize_definition():
    rng = np.random.default_rng(0)
    for gain in (1e-37, 1e-3, 1.0, 1e38):
        x = (rng.uniform(-1, 1, (50, 300)) * gain).astype(np.float32)
        c, s = ref.quantize(x)
        s = s.astype(np.float64)[:, None]
        live = s[:, 0] > 0           # (1e-37 / 127 is under 2^-126: such rows are zeros by definition)
        assert live.all() == (gain > 1e-36) and np.all(np.abs(c[live]).max(1) == 127) and not c[~live].any()
        assert np.all(np.abs(c * s - x) <= np.where(s > 0, s * (0.5 + 128 * 2.0 ** -23), 127 * 2.0 ** -126))
    c, s = ref.quantize(np.array([[0, 0], [np.nan, 1], [np.inf, 1], [1e-40, 0]], np.float32))
    assert not c.any() and s[0] == 0 and s[3] == 0 and np.isnan(s[1:3]).all()


def test_route_and_sort_definitions():
    e, w = ref.route(np.array([[1.0, 3.0, 3.0, -np.inf], [-np.inf] * 4, [-np.inf, 0.0, -np.inf, np.nan]]), 3, True)
    assert e.tolist() == [[1, 2, 0], [-1, -1, -1], [1, -1, -1]]
    assert np.allclose(w.sum(1), [1, 0, 1])
    starts, order, places = ref.sort(np.array([[2, 0], [0, -1], [5, 2]]), 3)
    assert starts.tolist() == [0, 2, 2, 4] and order.tolist() == [1, 2, 0, 5, -1, -1] and places.tolist() == [[2, 0], [1, -1], [-1, 3]]
