"""Attention at the edges of its number range: zero, constant, huge and infinite keys and values, empty and tiny queries, scales far from one;
and what the binding refuses.  Against the definitions in numpy."""
import ctypes

import numpy as np
import pytest
import torch

import _attention as ref
from test_gpu_attention import DT, cache_reference, ints, pipe, prompt_reference, random_cache, typed  # noqa: F401

pytestmark = pytest.mark.gpu


def prompt_limit(kind, q, k, v, scale):
    D, n = q.shape[-1], k.shape[0]
    a = abs(scale) * float(np.abs(q).max()) * float(np.abs(k).sum(-1).max())
    return ref.far(kind, D, n, a, float(np.abs(v).max()))


# ------------------------------------------------------------------ prompts

ZEROS = {
    "all": lambda v: v.zero_(),
    "first": lambda v: v[0].zero_(),
    "a tile": lambda v: v[:32].zero_(),
    "two tiles": lambda v: v[:64].zero_(),
    "one head": lambda v: v[:, 1].zero_(),
}


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("zero", ZEROS)
@pytest.mark.parametrize("D,causal,n", [(64, True, 100), (128, True, 100), (64, False, 70), (128, False, 5)])
def test_prompts_of_zero_values(pipe, kind, zero, D, causal, n):
    rng = np.random.default_rng(D + n)
    q, qf = typed(rng, (n, 4, D), kind)
    k, kf = typed(rng, (n, 2, D), kind)
    v, _ = typed(rng, (n, 2, D), kind)
    ZEROS[zero](v)
    vf = v.double().cpu().numpy()
    got = pipe.pipe_prompt_attention(q, k, v, ints([0, n]), causal=causal).double().cpu().numpy()
    want = prompt_reference(qf, kf, vf, [n], [n], causal, D ** -0.5)
    assert np.abs(got - want).max() <= prompt_limit(kind, qf, kf, vf, D ** -0.5)


@pytest.mark.parametrize("gain", [1e-30, 1.5e-33, 1e-35, 1e-37])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_of_tiny_values(pipe, D, gain):
    """Weights times values of that size are multiples of some 2^-149: 2^-22 a key beside the bound of other values."""
    n = 90
    rng = np.random.default_rng(D)
    q, qf = typed(rng, (n, 2, D), "f32")
    k, kf = typed(rng, (n, 2, D), "f32")
    v, vf = typed(rng, (n, 2, D), "f32", gain=gain)
    got = pipe.pipe_prompt_attention(q, k, v, ints([0, n])).double().cpu().numpy()
    want = prompt_reference(qf, kf, vf, [n], [n], True, D ** -0.5)
    top = float(np.abs(vf).max())
    assert np.abs(got - want).max() <= prompt_limit("f32", qf, kf, vf, D ** -0.5) + n * 2.0 ** -22 * top + 2.0 ** -140


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("scale", [1e-8, -1e-20, 1e-44])
def test_prompts_of_zero_queries_and_small_scales(pipe, kind, scale):
    """Scores of (next to) nothing: every query gives the mean of the values it sees."""
    D, n = 64, 80
    rng = np.random.default_rng(3)
    q, _ = typed(rng, (n, 2, D), kind)
    q[::2] = 0
    qf = q.double().cpu().numpy()
    k, kf = typed(rng, (n, 2, D), kind)
    v, vf = typed(rng, (n, 2, D), kind)
    got = pipe.pipe_prompt_attention(q, k, v, ints([0, n]), scale=scale).double().cpu().numpy()
    want = prompt_reference(qf, kf, vf, [n], [n], True, scale)
    assert np.abs(got - want).max() <= prompt_limit(kind, qf, kf, vf, scale)


def far_factors(pipe, kind, q_gain, k_gain, scale, D):
    n = 70
    rng = np.random.default_rng(4)
    q, qf = typed(rng, (n, 2, D), kind, gain=q_gain)
    k, kf = typed(rng, (n, 2, D), kind, gain=k_gain)
    v, vf = typed(rng, (n, 2, D), kind)
    got = pipe.pipe_prompt_attention(q, k, v, ints([0, n]), scale=scale).double().cpu().numpy()
    want = prompt_reference(qf, kf, vf, [n], [n], True, scale)
    assert np.abs(got - want).max() <= prompt_limit(kind, qf, kf, vf, scale)


@pytest.mark.parametrize("kind,q_gain,k_gain,scale", [("f32", 1e-38, 1.0, 3e38), ("f32", 1e-20, 1e-20, 1e38), ("f32", 0.0, 1.0, -3e38), ("bf16", 0.0, 1.0, 3e38),
                                                      ("f16", 1e-4, 1e-3, 1e6)])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_of_huge_scales(pipe, kind, q_gain, k_gain, scale, D):
    far_factors(pipe, kind, q_gain, k_gain, scale, D)


@pytest.mark.parametrize("kind,q_gain,k_gain", [("f32", 1e-33, 1e33), ("f32", 1e33, 1e-33), ("f32", 1e-37, 6e37), ("bf16", 1e-33, 1e33), ("bf16", 1e30, 1e-30)])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_of_far_factors(pipe, kind, q_gain, k_gain, D):
    """Factors at the ends of the range whose product is an ordinary score."""
    far_factors(pipe, kind, q_gain, k_gain, D ** -0.5, D)


@pytest.mark.parametrize("kind,gain", [("f32", 3e37), ("bf16", 3e37), ("f16", 1.3e4)])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_of_huge_values(pipe, kind, gain, D):
    """Sums over values next to the type's largest: the result is one of them on average, though their sum is beyond fp32."""
    n = 150
    rng = np.random.default_rng(5)
    q, qf = typed(rng, (n, 2, D), kind)
    k, kf = typed(rng, (n, 2, D), kind)
    v = torch.from_numpy(np.clip(rng.standard_normal((n, 2, D)), -4, 4).astype(np.float32) * np.float32(gain)).to(DT[kind]).abs().cuda()
    vf = v.double().cpu().numpy()
    got = pipe.pipe_prompt_attention(q, k, v, ints([0, n])).double().cpu().numpy()
    want = prompt_reference(qf, kf, vf, [n], [n], True, D ** -0.5)
    assert np.abs(got - want).max() <= prompt_limit(kind, qf, kf, vf, D ** -0.5)


def close(got, want, limit):
    """Equal where not finite, within the limit elsewhere."""
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True)
    assert np.isfinite(got[~odd]).all() and np.abs(got[~odd] - want[~odd]).max() <= limit


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [0, 40, 149])
@pytest.mark.parametrize("scale", [None, -0.1])
def test_prompts_with_an_infinite_key(pipe, kind, D, at, scale):
    """A key with an infinity: a score of -infinity is a weight of 0, one of +infinity is NaN."""
    n, H = 150, 2
    rng = np.random.default_rng(at + D)
    q, qf = typed(rng, (n, H, D), kind)
    k, kf = typed(rng, (n, H, D), kind)
    v, vf = typed(rng, (n, H, D), kind)
    sc = D ** -0.5 if scale is None else scale
    limit = prompt_limit(kind, qf, kf, vf, sc)
    k[at, 0, 5], k[at, 1, 3] = float("inf"), -float("inf")
    kf[at, 0, 5], kf[at, 1, 3] = np.inf, -np.inf
    got = pipe.pipe_prompt_attention(q, k, v, ints([0, n]), scale=scale).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = prompt_reference(qf, kf, vf, [n], [n], True, sc)
    if at == 0:
        got, want = got[1:], want[1:]            # (a query whose only score is -infinity has no weights at all)
    assert at == 149 or (np.isnan(want).any() and np.isfinite(want[at:]).any())
    close(got, want, limit)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("at", [0, 31, 70, 299])
def test_prompts_with_an_infinite_value(pipe, kind, D, causal, at):
    """An infinity of V is one in its column of every query that sees it, wherever its tile lies, and nowhere else."""
    n, H = 300, 2
    rng = np.random.default_rng(at + D)
    q, qf = typed(rng, (n, H, D), kind)
    k, kf = typed(rng, (n, H, D), kind)
    v, vf = typed(rng, (n, H, D), kind)
    limit = prompt_limit(kind, qf, kf, vf, D ** -0.5)
    v[at, 0, 5], v[at, 1, 3] = float("inf"), -float("inf")
    vf[at, 0, 5], vf[at, 1, 3] = np.inf, -np.inf
    got = pipe.pipe_prompt_attention(q, k, v, ints([0, n]), causal=causal).double().cpu().numpy()
    close(got, prompt_reference(qf, kf, vf, [n], [n], causal, D ** -0.5), limit)


# ------------------------------------------------------------------ the cache

def filled(pipe, k, v, P):
    """(cache, table, K and V as the cache holds them in fp64) of one request with the rows k and v [n, Hkv, D], fp32."""
    n, Hkv, D = k.shape
    pages = -(-n // P)
    cache = torch.zeros((pages, pipe.pipe_cache_page_bytes(Hkv, D, P)), dtype=torch.uint8, device="cuda")
    slots = ints(np.arange(n))
    pipe.pipe_cache_write(torch.from_numpy(k.astype(np.float32)).cuda(), torch.from_numpy(v.astype(np.float32)).cuda(), slots, cache, P)
    kk, vv = (x.double().cpu().numpy() for x in pipe.pipe_cache_read(slots, cache, P, Hkv, D))
    return cache, ints(np.arange(pages)[None]), kk, vv


CONSTANTS = (2.0 ** -90, 1.0, 1000.0, 2.0 ** 20, -2.0 ** 100, 2.0 ** 126)


@pytest.mark.parametrize("kind,values", [("f32", CONSTANTS), ("bf16", CONSTANTS), ("f16", (1.0, 1000.0, 57344.0))])
@pytest.mark.parametrize("n", [3, 1100, 20000])
@pytest.mark.parametrize("rise", [0.0, 0.003])
@pytest.mark.parametrize("D", [64, 128])
def test_cache_of_constant_values(pipe, kind, values, n, rise, D):
    """Rows of V without a scale, under equal scores and under slowly rising (for other queries falling) ones."""
    P, Hq, Hkv = 64, 4, 2
    rng = np.random.default_rng(n)
    k = np.broadcast_to((np.arange(n) * rise)[:, None, None], (n, Hkv, D))
    q, qf = typed(rng, (1, Hq, D), kind)
    limit = 2 * ref.UNIT[kind] + 2 * (n + 16) * ref.U32
    for c in values:
        cache, table, _, vv = filled(pipe, k, np.full((n, Hkv, D), c), P)
        assert (vv == c).all()
        for hint in (0, 1):
            got = pipe.pipe_cache_attention(q, ints([0, 1]), ints([n]), cache, table, P, Hkv, scale=0.1, max_length=hint).double().cpu().numpy()
            assert np.abs(got / c - 1).max() <= limit, (c, hint)


@pytest.mark.parametrize("kind,gain", [(k, g) for k in ("f32", "bf16") for g in (1e-36, 1e-30, 1e-20, 1e30, 3e37)] + [("f16", 1e-4), ("f16", 1.5e4)])
@pytest.mark.parametrize("D", [64, 128])
def test_cache_of_small_and_large_values(pipe, kind, gain, D):
    """Values of any size keep their digits, in one piece and in parts."""
    P, Hq, Hkv, n, fresh = 32, 4, 2, 1500, 2
    rng = np.random.default_rng(D)
    cache, table, kk, vv = filled(pipe, rng.standard_normal((n, Hkv, D)), np.clip(rng.standard_normal((n, Hkv, D)), -4, 4) * gain, P)
    q, qf = typed(rng, (fresh, Hq, D), kind)
    want = cache_reference(qf, [fresh], [n], [(kk, vv)], D ** -0.5)
    a = D ** -0.5 * float(np.abs(qf).sum(-1).max()) * 2 * float(np.abs(kk).max())
    limit = ref.far(kind, D, n, a, 2 * float(np.abs(vv).max()))
    if kind == "f16":
        limit += 2.0 ** -25                     # (an output under 2^-14 is rounded to a multiple of 2^-24)
    for hint in (0, 1):
        got = pipe.pipe_cache_attention(q, ints([0, fresh]), ints([n]), cache, table, P, Hkv, max_length=hint).double().cpu().numpy()
        assert np.abs(got - want).max() <= limit, hint


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("huge", [1e9, 1e30])
@pytest.mark.parametrize("n", [5, 300, 317])
def test_a_later_draft_stays_out_of_earlier_ones(pipe, kind, D, huge, n):
    """Values of the last fresh tokens that are far beyond the others' reach the queries that see them and leave the others' digits alone."""
    P, Hq, Hkv, fresh = 16, 4, 2, 4
    rng = np.random.default_rng(n)
    k, v = rng.standard_normal((n, Hkv, D)), rng.standard_normal((n, Hkv, D))
    v[-2:] *= huge
    cache, table, kk, vv = filled(pipe, k, v, P)
    q, qf = typed(rng, (fresh, Hq, D), kind)
    got = pipe.pipe_cache_attention(q, ints([0, fresh]), ints([n]), cache, table, P, Hkv).double().cpu().numpy()
    want = cache_reference(qf, [fresh], [n], [(kk, vv)], D ** -0.5)
    a = D ** -0.5 * float(np.abs(qf).sum(-1).max()) * 2 * float(np.abs(kk).max())
    for i in range(fresh):
        top = 2 * float(np.abs(vv[:n - fresh + i + 1]).max())
        assert np.abs(got[i] - want[i]).max() <= ref.far(kind, D, n, a, top), i


@pytest.mark.parametrize("kind,q_gain,k_gain,scale", [
    ("f32", 1e-33, 1e33, None), ("f32", 1e33, 1e-33, None), ("f32", 1e-37, 3e37, None), ("f32", 1e-30, 1.0, 1e-20), ("f32", 1e-38, 1.0, 3e38),
    ("f32", 0.0, 1.0, 1e-44), ("bf16", 1e33, 1e-33, None), ("bf16", 1e-33, 1e33, None), ("bf16", 1e-37, 3e37, None), ("bf16", 1e-30, 1.0, 1e-20), ("f16", 0.0, 1.0, 1e-44)])
def test_cache_of_far_factors(pipe, kind, q_gain, k_gain, scale):
    """Factors at the ends of the range whose product is an ordinary score, or none at all."""
    P, Hq, Hkv, D, n, fresh = 16, 4, 2, 64, 75, 3
    rng = np.random.default_rng(7)
    cache, table, kk, vv = filled(pipe, np.clip(rng.standard_normal((n, Hkv, D)), -4, 4) * k_gain, rng.standard_normal((n, Hkv, D)), P)
    q, qf = typed(rng, (fresh, Hq, D), kind, gain=q_gain)
    sc = D ** -0.5 if scale is None else scale
    got = pipe.pipe_cache_attention(q, ints([0, fresh]), ints([n]), cache, table, P, Hkv, scale=scale).double().cpu().numpy()
    want = cache_reference(qf, [fresh], [n], [(kk, vv)], sc)
    a = sc * float(np.abs(qf).sum(-1).max()) * 2 * float(np.abs(kk).max())
    assert np.abs(got - want).max() <= ref.far(kind, D, n, a, 2 * float(np.abs(vv).max()))


# ------------------------------------------------------------------ graphs

def fresh_stream():
    """A stream that no earlier call can have used (torch's own come from a pool)."""
    hip = ctypes.CDLL("libamdhip64.so")
    s = ctypes.c_void_p()
    assert hip.hipStreamCreate(ctypes.byref(s)) == 0
    return torch.cuda.ExternalStream(s.value)


def test_a_stream_without_scratch_is_refused_in_a_capture_and_served_once_prepared(pipe):
    rng = np.random.default_rng(1)
    lens = [2000, 300]
    cache, table, _ = random_cache(pipe, rng, lens, 2, 64, 16)
    q, _ = typed(rng, (2, 8, 64), "f32")
    starts, lengths = ints([0, 1, 2]), ints(lens)
    want = pipe.pipe_cache_attention(q, starts, lengths, cache, table, 16, 2)
    out = torch.full_like(want, float("nan"))
    side = fresh_stream()
    torch.cuda.synchronize()
    codes = []
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        try:
            pipe.pipe_cache_attention(q, starts, lengths, cache, table, 16, 2, out=out)
        except pipe.PipeError as e:
            codes.append(e.code)
        q.add(1)
    assert codes == [-6]
    with torch.cuda.stream(side):
        pipe.pipe_prepare_cache_attention(2, 8, 2, 64, 2, max(lens))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pipe.pipe_cache_attention(q, starts, lengths, cache, table, 16, 2, out=out)
    for _ in range(4):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_prompts_in_a_graph(pipe, kind):
    """Captured once, replayed on other values and other lengths, with the caller's work between."""
    n, D = 200, 64
    rng = np.random.default_rng(2)
    x, _ = typed(rng, (n, 8, D), kind)
    starts = ints([0, 50, 120, n])
    out = torch.empty((n, 4, D), dtype=DT[kind], device="cuda")
    call = lambda o=None: pipe.pipe_prompt_attention(x[:, :4], x[:, 4:6], x[:, 6:], starts, out=o)      # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(4):
        x.copy_(typed(rng, (n, 8, D), kind)[0])
        starts.copy_(ints([0, 10 * i, 60 + 35 * i, n - i]))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, call()), i


# ------------------------------------------------------------------ refusals

def small_call(pipe):
    """What a call of each kind takes: two requests of one fresh token."""
    q, k = torch.randn(2, 4, 64, device="cuda"), torch.randn(2, 2, 64, device="cuda")
    cache = torch.zeros((4, pipe.pipe_cache_page_bytes(2, 64, 16)), dtype=torch.uint8, device="cuda")
    starts, lengths, table, slots = ints([0, 1, 2]), ints([1, 1]), ints([[0], [1]]), ints([0, 16])
    return q, k, cache, starts, lengths, table, slots


def test_tables_of_other_ranks_are_refused(pipe):
    q, k, cache, starts, lengths, table, slots = small_call(pipe)
    pipe.pipe_cache_write(k, k, slots, cache, 16)
    for bad in (slots[None], slots[:, None], slots.view(2, 1, 1), slots[0]):
        with pytest.raises(ValueError):
            pipe.pipe_cache_read(bad, cache, 16, 2, 64)
        with pytest.raises(ValueError):
            pipe.pipe_cache_write(k, k, bad, cache, 16)
    for bad in (lengths[:, None], torch.stack([lengths, lengths], dim=1), lengths[0]):
        with pytest.raises(ValueError):
            pipe.pipe_cache_attention(q, starts, bad, cache, table, 16, 2)
    for bad in (starts[:, None], starts[0], starts[None]):
        with pytest.raises(ValueError):
            pipe.pipe_prompt_attention(q, k, k, bad)
    for bad in (lengths[:, None], lengths[0]):
        with pytest.raises(ValueError):
            pipe.pipe_cache_plan(bad, bad, 16, slots, ints([0]), table, 2)


def test_tensors_of_another_device_than_the_current_one_are_refused(pipe, monkeypatch):
    """The kernels run on the current device; one card is enough to ask: another one is said to be current."""
    q, k, cache, starts, lengths, table, slots = small_call(pipe)
    calls = [lambda: pipe.pipe_cache_plan(lengths, lengths, 16, slots, ints([0]), table, 2), lambda: pipe.pipe_cache_write(k, k, slots, cache, 16),
             lambda: pipe.pipe_cache_read(slots, cache, 16, 2, 64), lambda: pipe.pipe_cache_attention(q, starts, lengths, cache, table, 16, 2),
             lambda: pipe.pipe_prompt_attention(q, k, k, starts)]
    for call in calls:
        call()
    monkeypatch.setattr(pipe, "_device", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError):
            call()
