"""Page planning, the 4-bit cache, attention over it and over packed prompts, against their definitions in numpy."""
import numpy as np
import pytest
import torch

import _attention as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def pipe():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_2311_15806_amd.binding as b
    return b


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def typed(rng, shape, kind, gain=1.0):
    """(device tensor, the same values in fp64)"""
    t = torch.from_numpy((rng.standard_normal(shape) * gain).astype(np.float32)).to(DT[kind])
    return t.cuda(), t.double().numpy()


# ------------------------------------------------------------------ tables

PLANS = [
    # B, P, cached, fresh, free pages, used, width, T beyond the total (negative: cut), step
    (1, 16, (0, 0), (1, 1), 4, 0, 1, 0),
    (1, 16, (16, 16), (1, 1), 1, 0, 2, 3),
    (3, 32, (0, 100), (0, 70), 40, 2, 8, 0),
    (64, 16, (1, 900), (1, 1), 64, 5, 60, 0),
    (65, 64, (0, 300), (0, 200), 500, 0, 9, 17),
    (257, 128, (0, 1000), (0, 40), 500, 0, 10, 0),
    (300, 256, (0, 700), (0, 100), 40, 0, 4, 0),        # the free list ends
    (40, 16, (0, 100), (0, 100), 900, 0, 5, 0),         # the table's width ends
    (33, 16, (0, 50), (1, 60), 300, 1, 20, -400),       # more tokens than T
    (2, 16, (0, 0), (9000, 9001), 1200, 0, 600, 0),     # several workgroups
    (4096, 16, (0, 40), (0, 3), 9000, 0, 5, 5),
]


@pytest.mark.parametrize("case", PLANS, ids=range(len(PLANS)))
def test_plan(pipe, case):
    B, P, (c0, c1), (f0, f1), n_free, used, width, spare = case
    rng = np.random.default_rng(B * 7 + P)
    cached, fresh = rng.integers(c0, c1 + 1, B), rng.integers(f0, f1 + 1, B)
    T = max(0, int(fresh.sum()) + spare)
    free = rng.permutation(n_free + 100)[:n_free]
    table = np.full((B, width), 777777)
    for b in range(B):
        have = min(width, -(-int(cached[b]) // P))
        table[b, :have] = rng.integers(0, 5000, have)
    want = ref.plan(cached, fresh, P, free, used, table, T)
    d_table = ints(table)
    got = pipe.pipe_cache_plan(ints(cached), ints(fresh), P, ints(free), ints([used]), d_table, T)
    for name, g, w in zip(("lengths", "starts", "slots", "positions", "counts", "table"), (*got, d_table), want):
        assert np.array_equal(g.cpu().numpy(), w), name


def test_plan_of_negative_counts_and_steps_in_a_row(pipe):
    B, P, width = 5, 16, 7
    rng = np.random.default_rng(3)
    cached, table, free, used = np.array([-4, 0, 15, 16, 17]), np.full((B, width), -1), rng.permutation(60), 0
    table[2, 0], table[3, 0], table[4, :2] = 90, 91, (92, 93)
    d_cached, d_table, d_used, d_free = ints(cached), ints(table), ints([used, 0, 0]), ints(free)
    for step in range(6):
        fresh = rng.integers(-2, 20, B)
        T = 80
        want = ref.plan(cached, fresh, P, free, used, table, T)
        got = pipe.pipe_cache_plan(d_cached, ints(fresh), P, d_free, d_used, d_table, T)
        for g, w in zip((*got, d_table), want):
            assert np.array_equal(g.cpu().numpy(), w), step
        cached, used, table = want[0], int(want[4][0]), want[5]
        d_cached, d_used = got[0], got[4]


# ------------------------------------------------------------------ the cache

def expected_cache(before, slots, k, v, P, H, D):
    out = before.copy().reshape(before.shape[0], H, P * (D + 8))
    ck, sk, mk = ref.quantize_rows(k)
    cv, sv, mv = ref.quantize_rows(v)
    for t, slot in enumerate(slots):
        if slot < 0 or slot // P >= before.shape[0]:
            continue
        page, off = slot // P, slot % P
        for h in range(H):
            one = ref.block_of(ck[t, h][None], cv[t, h][None], np.concatenate([sk[t, h], mk[t, h]])[None],
                               np.concatenate([sv[t, h], mv[t, h]])[None])
            blk = out[page, h]
            blk[off * D // 2:(off + 1) * D // 2] = one[:D // 2]
            blk[P * D // 2 + off * D // 2:P * D // 2 + (off + 1) * D // 2] = one[D // 2:D]
            blk[P * D + 4 * off:P * D + 4 * off + 4] = one[D:D + 4]
            blk[P * D + 4 * P + 4 * off:P * D + 4 * P + 4 * off + 4] = one[D + 4:]
    return out.reshape(before.shape)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,H,P,T,layout", [(64, 1, 16, 1, "own"), (64, 12, 64, 33, "fused"), (128, 8, 16, 50, "fused"), (128, 3, 32, 7, "own"),
                                            (128, 2, 256, 20, "odd"), (64, 5, 128, 19, "odd")])
def test_write_and_read(pipe, kind, D, H, P, T, layout):
    rng = np.random.default_rng(T + D)
    pages = -(-T // P) + 3
    if layout == "odd":              # addresses and strides that no wide load fits
        flat = torch.from_numpy(rng.standard_normal(2 + T * (H * (D + 1) + 3) * 2).astype(np.float32)).to(DT[kind]).cuda()
        k = flat[1:].as_strided((T, H, D), (H * (D + 1) + 3, D + 1, 1))
        v = flat[1 + T * (H * (D + 1) + 3):].as_strided((T, H, D), (H * (D + 1) + 3, D + 1, 1))
    else:
        x, _ = typed(rng, (T, 2 * H + 4, D), kind)
        k, v = (x[:, 4:4 + H], x[:, 4 + H:]) if layout == "fused" else (x[:, :H].contiguous(), x[:, H:2 * H].contiguous())
    slots = rng.permutation(pages * P)[:T]
    if T > 4:
        slots[1], slots[3] = -1, pages * P + 5         # outside: skipped
    before = rng.integers(0, 256, (pages, pipe.pipe_cache_page_bytes(H, D, P))).astype(np.uint8)
    cache = torch.from_numpy(before).cuda()
    pipe.pipe_cache_write(k, v, ints(slots), cache, P)
    kf, vf = k.float().cpu().numpy(), v.float().cpu().numpy()
    assert np.array_equal(cache.cpu().numpy(), expected_cache(before, slots, kf, vf, P, H, D))
    for back in DT:
        rk, rv = pipe.pipe_cache_read(ints(slots), cache, P, H, D, DT[back])
        for got, x in ((rk, kf), (rv, vf)):
            c, s, m = ref.quantize_rows(x)
            exact = s.astype(np.float64) * c + m
            exact[(slots < 0) | (slots >= pages * P)] = 0
            want = torch.from_numpy(exact.astype(np.float32)).to(DT[back])
            assert torch.equal(got.cpu(), want), back
        # every value within half a step of what was written (and the fp32 roundings of its way there)
        c, s, m = ref.quantize_rows(kf)
        live = (slots >= 0) & (slots < pages * P)
        assert np.all(np.abs(s.astype(np.float64) * c + m - kf)[live] <= (0.5 * s + 16 * ref.U32 * (15 * s + np.abs(m)))[live])


def test_write_of_special_rows(pipe):
    D, P = 64, 16
    rng = np.random.default_rng(11)
    rows = rng.standard_normal((16, 1, D)).astype(np.float32)
    rows[0] = 0.0
    rows[1] = -3.7                                # one value: scale of the offset's own rounding
    rows[2] = 1.0                                 # exact in bf16: scale 0
    rows[3, 0, 5] = np.nan
    rows[4, 0, 63] = np.inf
    rows[5, 0, 0] = -np.inf
    rows[6] *= 3e38
    rows[6, 0, :2] = (3e38, -3e38)                # range beyond fp32
    rows[7] *= 1e-38                              # scales under 2^-126
    rows[8] *= 1e-44
    rows[9] *= 1e30
    rows[10] = np.linspace(100.0, 100.01, D)      # narrow beside its offset
    rows[11] = np.where(np.arange(D) % 2, -0.0, 0.0)
    rows[12] = -np.abs(rows[12])
    rows[13] = np.arange(D) % 16                  # the codes themselves
    rows[14, 0, :] = np.float32(-3.4e38)          # rounds down to -inf in bf16
    rows[15] = (np.arange(D) % 16 + 0.5) / 2      # halves between codes
    vals = np.roll(rows, 1, axis=0)
    cache = torch.zeros((2, pipe.pipe_cache_page_bytes(1, D, P)), dtype=torch.uint8, device="cuda")
    slots = np.arange(16) + P
    pipe.pipe_cache_write(torch.from_numpy(rows).cuda(), torch.from_numpy(vals).cuda(), ints(slots), cache, P)
    k, v = pipe.pipe_cache_read(ints(slots), cache, P, 1, D)
    for got, x in ((k, rows), (v, vals)):
        c, s, m = ref.quantize_rows(x)
        want = (s.astype(np.float64) * c + m).astype(np.float32)
        assert np.array_equal(got.cpu().numpy(), want, equal_nan=True)
    bad = np.isnan(k.cpu().numpy()).all(axis=(1, 2))
    assert list(np.nonzero(bad)[0]) == [3, 4, 5, 6, 14]


# ------------------------------------------------------------------ attention over the cache

def random_cache(pipe, rng, lens, H, D, P, spoil=True):
    """(cache, table, K and V per request in fp64): pages in random order; what no request holds is NaN or noise."""
    need = [-(-n // P) for n in lens]
    pages = sum(need) + 2
    cache = rng.integers(0, 256, (pages, H, P * (D + 8))).astype(np.uint8)
    if spoil:
        cache[:, :, P * D:] = np.array([0xc0, 0x7f] * (4 * P), np.uint8)      # NaN scales and offsets
    order = rng.permutation(pages)
    table = np.full((len(lens), max(need + [1]) + 1), -1)
    at, kv = 0, []
    for b, n in enumerate(lens):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        both = []
        for side in range(2):
            c = rng.integers(0, 16, (n, H, D)).astype(np.uint8)
            s = ref._bf16(0.2 + 0.2 * rng.random((n, H, 1)), True)
            m = ref._bf16(-7.5 * s + 0.3 * rng.standard_normal((n, H, 1)), False)
            for t in range(n):
                page, off = table[b, t // P], t % P
                word = (s[t].view(np.uint32) >> 16 | m[t].view(np.uint32) & 0xffff0000).view(np.uint8)
                cache[page, :, side * P * D // 2 + off * D // 2:side * P * D // 2 + (off + 1) * D // 2] = c[t, :, 0::2] | c[t, :, 1::2] << 4
                cache[page, :, P * D + 4 * P * side + 4 * off:P * D + 4 * P * side + 4 * off + 4] = word
            both.append(s.astype(np.float64) * c + m)
        kv.append(both)
    return torch.from_numpy(cache.reshape(pages, -1)).cuda(), ints(table), kv


def cache_reference(q, fresh, lens, kv, scale):
    out, a, v = np.zeros(q.shape), 0.0, 0.0
    at = 0
    for n, L, (k, val) in zip(fresh, lens, kv):
        seen = L - n + np.arange(n) + 1
        if n:
            out[at:at + n] = ref.attend(q[at:at + n], k, val, scale, seen)
        at += n
    return out


def cache_far(kind, D, q, lens, scale):
    # |s c + m| <= 15 s + |m| <= 6 + 4.5 of both K and V (scales up to 0.4, offsets -7.5 s and 5 deviations of 0.3)
    a = abs(scale) * float(np.abs(q).sum(-1).max()) * 10.5
    return ref.far(kind, D, max(lens), a, 10.5)


CACHES = [
    # Hq, Hkv, D, P, lengths, fresh
    (4, 1, 64, 16, [1], [1]),
    (8, 2, 128, 16, [1, 15, 16, 17, 0, 33], [1, 1, 1, 1, 1, 1]),
    (8, 8, 64, 32, [63, 64, 65, 300], [1, 1, 0, 1]),
    (7, 1, 128, 64, [129, 400], [3, 1]),
    (32, 1, 128, 32, [200, 31], [1, 1]),
    (12, 1, 64, 16, [100, 5, 77], [5, 5, 2]),
    (4, 2, 128, 128, [255, 256, 257], [1, 16, 17]),
    (2, 2, 64, 256, [600], [40]),
    (16, 8, 128, 16, [1030, 3], [1, 7]),           # more queries than cached tokens: the first ones see nothing
]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", CACHES, ids=range(len(CACHES)))
def test_cache_attention(pipe, kind, case):
    Hq, Hkv, D, P, lens, fresh = case
    rng = np.random.default_rng(sum(lens) + D)
    cache, table, kv = random_cache(pipe, rng, lens, Hkv, D, P)
    q, qf = typed(rng, (sum(fresh), Hq, D), kind)
    starts = np.concatenate([[0], np.cumsum(fresh)])
    for scale in (None, 0.3):
        sc = D ** -0.5 if scale is None else scale
        want = cache_reference(qf, fresh, lens, kv, sc)
        limit = cache_far(kind, D, qf, lens, sc)
        for hint in (0, max(lens), 64, 5000):
            got = pipe.pipe_cache_attention(q, ints(starts), ints(lens), cache, table, P, Hkv, scale=scale, max_length=hint)
            assert got.dtype == q.dtype
            err = np.abs(got.double().cpu().numpy() - want).max()
            assert err <= limit, (hint, err, limit)
            again = pipe.pipe_cache_attention(q, ints(starts), ints(lens), cache, table, P, Hkv, scale=scale, max_length=hint)
            assert torch.equal(got, again)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_cache_attention_of_a_long_request(pipe, kind):
    Hq, Hkv, D, P, lens = 4, 1, 128, 64, [9001, 2]
    rng = np.random.default_rng(5)
    cache, table, kv = random_cache(pipe, rng, lens, Hkv, D, P)
    q, qf = typed(rng, (2, Hq, D), kind)
    want = cache_reference(qf, [1, 1], lens, kv, D ** -0.5)
    limit = cache_far(kind, D, qf, lens, D ** -0.5)
    for hint in (0, 9001, 1, 100000):
        got = pipe.pipe_cache_attention(q, ints([0, 1, 2]), ints(lens), cache, table, P, Hkv, max_length=hint)
        assert np.abs(got.double().cpu().numpy() - want).max() <= limit


@pytest.mark.parametrize("B", [62, 63, 64, 65, 300, 1100])
def test_cache_attention_of_many_requests(pipe, B):
    """A share finds its place among up to 63 requests in one wave, among more in the workgroup; some hold nothing, some bring nothing."""
    Hq, Hkv, D, P = 3, 1, 64, 16
    rng = np.random.default_rng(B)
    fresh = rng.integers(0, 3, B)
    lens = np.where(rng.random(B) < 0.2, 0, rng.integers(0, 60, B))
    lens[B // 2], lens[-1], fresh[0], fresh[-1] = 700, 150, 0, 2
    cache, table, kv = random_cache(pipe, rng, list(lens), Hkv, D, P)
    q, qf = typed(rng, (int(fresh.sum()) + 2, Hq, D), "f32")
    starts = np.concatenate([[0], np.cumsum(fresh)])
    want = cache_reference(qf, fresh, lens, kv, D ** -0.5)
    limit = cache_far("f32", D, qf, list(lens), D ** -0.5)
    for hint in (0, 700, 10, 100000):
        got = pipe.pipe_cache_attention(q, ints(starts), ints(lens), cache, table, P, Hkv, max_length=hint).double().cpu().numpy()
        assert np.abs(got - want).max() <= limit, hint
        assert not got[int(fresh.sum()):].any()


SHARES = {
    # Hq, Hkv, lengths, fresh: what a workgroup gets
    "one tile each": (32, 32, [640 + 7 * i for i in range(16)], [1] * 16),
    "parts of one tile": (8, 2, [100, 2000, 3001], [1, 1, 1]),
    "parts of requests of several tiles": (4, 2, [2000, 130, 900], [40, 1, 3]),
    "equal shares": (8, 8, [300 + 150 * (i % 7) + 3200 * (i % 9 == 0) for i in range(60)], [1 + (i % 5 == 0) for i in range(60)]),
}


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shares", SHARES)
def test_cache_attention_in_shares(pipe, kind, shares):
    Hq, Hkv, lens, fresh = SHARES[shares]
    D, P = 64, 16
    rng = np.random.default_rng(len(lens))
    cache, table, kv = random_cache(pipe, rng, lens, Hkv, D, P)
    q, qf = typed(rng, (sum(fresh) + 3, Hq, D), kind)        # rows of no request behind them
    starts = ints(np.concatenate([[0], np.cumsum(fresh)]))
    got = pipe.pipe_cache_attention(q, starts, ints(lens), cache, table, P, Hkv, max_length=max(lens))
    want = cache_reference(qf, fresh, lens, kv, D ** -0.5)
    assert np.abs(got.double().cpu().numpy() - want).max() <= cache_far(kind, D, qf, lens, D ** -0.5)
    for _ in range(3):                                       # the counts of parts are back at zero, and the order of arrival does not matter
        assert torch.equal(got, pipe.pipe_cache_attention(q, starts, ints(lens), cache, table, P, Hkv, max_length=max(lens)))


def test_cache_attention_of_padded_steps_missing_pages_and_strided_queries(pipe):
    Hq, Hkv, D, P, lens = 8, 2, 64, 16, [40, 70]
    rng = np.random.default_rng(9)
    cache, table, kv = random_cache(pipe, rng, lens, Hkv, D, P)
    wide, _ = typed(rng, (6, Hq + 3, D), "f16")
    q = wide[:, 2:2 + Hq]
    qf = q.double().cpu().numpy()
    limit = cache_far("f16", D, qf, lens, D ** -0.5)
    full = cache_reference(qf, [1, 2], lens, kv, D ** -0.5)
    got = pipe.pipe_cache_attention(q, ints([0, 1, 3]), ints(lens), cache, table, P, Hkv).double().cpu().numpy()
    assert np.abs(got - full).max() <= limit and not got[3:].any()          # rows of no request: zeros
    # a page that is not there is left out: the same as a request without those tokens
    for missing in (-1, 10 ** 6, cache.shape[0]):
        t2 = table.clone()
        t2[1, 1] = missing
        k, v = (np.delete(x, range(16, 32), axis=0) for x in kv[1])
        short = cache_reference(qf, [1, 2], [40, 54], [kv[0], [k, v]], D ** -0.5)
        got = pipe.pipe_cache_attention(q, ints([0, 1, 3]), ints(lens), cache, t2, P, Hkv).double().cpu().numpy()
        assert np.abs(got - short).max() <= limit
    # a request all of whose pages are missing, and a length beyond the table
    t2 = table.clone()
    t2[0] = -1
    got = pipe.pipe_cache_attention(q, ints([0, 1, 3]), ints([40, 70]), cache, t2, P, Hkv).double().cpu().numpy()
    assert not got[0].any() and np.abs(got[1:3] - full[1:3]).max() <= limit


def test_cache_attention_keeps_a_bad_row_to_its_readers(pipe):
    """A NaN row reaches the queries that see it and no others; values that span the type's range; scores far apart."""
    Hq, Hkv, D, P = 2, 1, 64, 16
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((40, 1, D)).astype(np.float32), rng.standard_normal((40, 1, D)).astype(np.float32)
    k[30, 0, 3], v[:, 0, 7] = np.nan, 1e30
    cache = torch.zeros((3, pipe.pipe_cache_page_bytes(Hkv, D, P)), dtype=torch.uint8, device="cuda")
    pipe.pipe_cache_write(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), ints(np.arange(40)), cache, P)
    kk, vv = (x.double().cpu().numpy() for x in pipe.pipe_cache_read(ints(np.arange(40)), cache, P, Hkv, D))
    q, qf = typed(rng, (20, Hq, D), "f32", gain=40.0)
    got = pipe.pipe_cache_attention(q, ints([0, 20]), ints([40]), cache, ints([[0, 1, 2]]), P, Hkv).double().cpu().numpy()
    want = ref.attend(qf[:10], kk, vv, D ** -0.5, np.arange(21, 31))
    assert np.isnan(got[10:]).all() and np.isfinite(got[:10]).all()
    a = D ** -0.5 * float(np.abs(qf).sum(-1).max()) * 10
    assert np.abs(got[:10] - want).max() <= ref.far("f32", D, 40, a, float(np.abs(vv[:30]).max()))


def test_cache_beyond_four_gib(pipe):
    """Pages whose bytes lie beyond 2^32."""
    Hq, Hkv, D, P, L = 8, 8, 128, 256, 700
    per = pipe.pipe_cache_page_bytes(Hkv, D, P)
    pages = (1 << 32) // per + 40
    cache = torch.empty((pages, per), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(4)
    at = [pages - 1, 3, pages - 17]
    k, _ = typed(rng, (L, Hkv, D), "bf16")
    v, _ = typed(rng, (L, Hkv, D), "bf16")
    slots = np.array([at[t // P] * P + t % P for t in range(L)])
    pipe.pipe_cache_write(k, v, ints(slots), cache, P)
    kk, vv = (x.double().cpu().numpy() for x in pipe.pipe_cache_read(ints(slots), cache, P, Hkv, D))
    c, s, m = ref.quantize_rows(k.float().cpu().numpy())
    assert np.array_equal(kk, s.astype(np.float64) * c + m)
    q, qf = typed(rng, (1, Hq, D), "bf16")
    got = pipe.pipe_cache_attention(q, ints([0, 1]), ints([L]), cache, ints([at]), P, Hkv).double().cpu().numpy()
    want = ref.attend(qf, kk, vv, D ** -0.5, [L])
    a = D ** -0.5 * float(np.abs(qf).sum(-1).max()) * float(np.abs(kk).max()) * 2
    assert np.abs(got - want).max() <= ref.far("bf16", D, L, a, 2 * float(np.abs(vv).max()))


# ------------------------------------------------------------------ attention over prompts

PROMPTS = [
    # Hq, Hkv, D, query lengths, key lengths (None: the same), causal
    (2, 1, 64, [1], None, True),
    (4, 4, 128, [5, 0, 64, 65], None, True),
    (8, 2, 128, [127, 1, 130], None, True),
    (7, 1, 64, [33, 200], None, True),
    (3, 3, 64, [300], None, True),
    (4, 2, 128, [31, 70], None, False),
    (4, 2, 64, [10, 3, 90], [100, 3, 257], True),      # new tokens behind a prefix
    (4, 1, 128, [9, 150, 20], [0, 40, 7], True),       # more queries than keys: the first see nothing
    (4, 1, 64, [9, 40], [0, 129], False),
]


def prompt_reference(q, k, v, nq, nk, causal, scale):
    out = np.zeros(q.shape)
    a = b = 0
    for n, m in zip(nq, nk):
        seen = m - n + np.arange(n) + 1 if causal else np.full(n, m)
        out[a:a + n] = ref.attend(q[a:a + n], k[b:b + m], v[b:b + m], scale, seen)
        a, b = a + n, b + m
    return out


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["fused", "own", "odd"])
@pytest.mark.parametrize("case", PROMPTS, ids=range(len(PROMPTS)))
def test_prompt_attention(pipe, kind, layout, case):
    Hq, Hkv, D, nq, nk, causal = case
    rng = np.random.default_rng(sum(nq) + D)
    Tq, Tk = sum(nq), sum(nk or nq)
    if layout == "fused" and nk is None:
        x, _ = typed(rng, (Tq, Hq + 2 * Hkv, D), kind)
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    elif layout == "odd":
        def odd(T, H):
            flat = torch.from_numpy(rng.standard_normal(1 + T * (H * (D + 1) + 1) + D).astype(np.float32)).to(DT[kind]).cuda()
            return flat[1:].as_strided((T, H, D), (H * (D + 1) + 1, D + 1, 1))
        q, k, v = odd(Tq, Hq), odd(Tk, Hkv), odd(Tk, Hkv)
    else:
        q, k, v = (typed(rng, (T, H, D), kind)[0] for T, H in ((Tq, Hq), (Tk, Hkv), (Tk, Hkv)))
    qf, kf, vf = (x.double().cpu().numpy() for x in (q, k, v))
    starts = ints(np.concatenate([[0], np.cumsum(nq)]))
    starts_k = None if nk is None else ints(np.concatenate([[0], np.cumsum(nk)]))
    got = pipe.pipe_prompt_attention(q, k, v, starts, starts_k, causal=causal)
    want = prompt_reference(qf, kf, vf, nq, nk or nq, causal, D ** -0.5)
    a = D ** -0.5 * float(max((np.abs(qf[i]).max() for i in range(Tq)), default=0)) * float(np.abs(kf).sum(-1).max())
    err = np.abs(got.double().cpu().numpy() - want).max()
    assert err <= ref.far(kind, D, max(nk or nq), a, float(np.abs(vf).max())), err
    assert torch.equal(got, pipe.pipe_prompt_attention(q, k, v, starts, starts_k, causal=causal))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("B", [63, 64, 65, 200])
def test_prompt_attention_of_many_sequences(pipe, B, kind):
    Hq, Hkv, D = 3, 1, 64
    rng = np.random.default_rng(B)
    nq, nk = rng.integers(0, 9, B), rng.integers(0, 12, B)
    nq[B // 3] = 140
    q, qf = typed(rng, (int(nq.sum()) + 1, Hq, D), kind)
    k, kf = typed(rng, (int(nk.sum()), Hkv, D), kind)
    v, vf = typed(rng, (int(nk.sum()), Hkv, D), kind)
    starts, starts_k = (ints(np.concatenate([[0], np.cumsum(n)])) for n in (nq, nk))
    got = pipe.pipe_prompt_attention(q, k, v, starts, starts_k).double().cpu().numpy()
    want = prompt_reference(qf, kf, vf, nq, nk, True, D ** -0.5)
    a = D ** -0.5 * float(np.abs(qf).max()) * float(np.abs(kf).sum(-1).max())
    assert np.abs(got - want).max() <= ref.far(kind, D, 12, a, float(np.abs(vf).max()))
    assert not got[-1].any()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_prompt_attention_never_looks_ahead(pipe, kind):
    """What comes later may hold anything -- infinities, NaN, the type's largest values -- within a tile and beyond it, in another
    sequence too; a query that sees a NaN gives NaN."""
    Hq, Hkv, D, n = 4, 2, 128, 150
    rng = np.random.default_rng(1)
    q, qf = typed(rng, (2 * n, Hq, D), kind)
    k, kf = typed(rng, (2 * n, Hkv, D), kind)
    v, vf = typed(rng, (2 * n, Hkv, D), kind)
    limit = ref.far(kind, D, n, D ** -0.5 * float(np.abs(qf).max()) * float(np.abs(kf).sum(-1).max()), float(np.abs(vf).max()))
    want = prompt_reference(qf, kf, vf, [n, n], [n, n], True, D ** -0.5)
    top = torch.finfo(DT[kind]).max
    for at in (100, 127, 128, 149):
        for value in (float("nan"), float("inf"), -float("inf"), top, -top):
            k2, v2 = k.clone(), v.clone()
            k2[at, 1, 5], v2[at, 0, 9] = value, value
            got = pipe.pipe_prompt_attention(q, k2, v2, ints([0, n, 2 * n])).double().cpu().numpy()
            assert np.abs(got[:at] - want[:at]).max() <= limit
            assert np.abs(got[n:] - want[n:]).max() <= limit
            if value != value:
                assert np.isnan(got[at:n, 2:]).all()


def test_prompt_attention_of_large_scores(pipe):
    """Scores of some thousands: the running maximum does its work, one key takes all."""
    Hq, D, n = 2, 64, 200
    rng = np.random.default_rng(8)
    q, qf = typed(rng, (n, Hq, D), "f32", gain=30.0)
    k, kf = typed(rng, (n, Hq, D), "f32", gain=30.0)
    v, vf = typed(rng, (n, Hq, D), "f32")
    got = pipe.pipe_prompt_attention(q, k, v, ints([0, n])).double().cpu().numpy()
    want = prompt_reference(qf, kf, vf, [n], [n], True, D ** -0.5)
    a = D ** -0.5 * float((np.abs(qf).max()) * np.abs(kf).sum(-1).max())
    assert np.abs(got - want).max() <= ref.far("f32", D, n, a, float(np.abs(vf).max()))


def test_rows_of_no_sequence_are_zeros(pipe):
    q, k, v = (torch.randn(20, 2, 64, device="cuda") for _ in range(3))
    out = torch.full((20, 2, 64), float("nan"), device="cuda")
    pipe.pipe_prompt_attention(q, k, v, ints([0, 7, 11]), out=out)
    assert torch.isfinite(out).all() and not out[11:].any() and out[:11].any()


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("first", [3, 40])
def test_rows_before_the_first_sequence_are_zeros(pipe, kind, causal, first):
    Hq, Hkv, D, nq, nk = 4, 2, 64, [50, 9], [130, 9]
    rng = np.random.default_rng(first)
    q, qf = typed(rng, (first + sum(nq), Hq, D), kind)
    k, kf = typed(rng, (5 + sum(nk), Hkv, D), kind)
    v, vf = typed(rng, (5 + sum(nk), Hkv, D), kind)
    got = pipe.pipe_prompt_attention(q, k, v, ints(first + np.array([0, 50, 59])), ints(5 + np.array([0, 130, 139])), causal=causal)
    got = got.double().cpu().numpy()
    want = prompt_reference(qf[first:], kf[5:], vf[5:], nq, nk, causal, D ** -0.5)
    a = D ** -0.5 * float(np.abs(qf).max()) * float(np.abs(kf).sum(-1).max())
    assert not got[:first].any()
    assert np.abs(got[first:] - want).max() <= ref.far(kind, D, 130, a, float(np.abs(vf).max()))


@pytest.mark.parametrize("B", [2, 70])
@pytest.mark.parametrize("first", [3, 40])
def test_rows_before_the_first_request_are_zeros(pipe, B, first):
    Hq, Hkv, D, P = 8, 2, 64, 16
    rng = np.random.default_rng(B + first)
    lens = [200] + list(rng.integers(1, 300, B - 1))
    cache, table, kv = random_cache(pipe, rng, lens, Hkv, D, P)
    q, qf = typed(rng, (first + B, Hq, D), "f16")
    got = pipe.pipe_cache_attention(q, ints(first + np.arange(B + 1)), ints(lens), cache, table, P, Hkv).double().cpu().numpy()
    want = cache_reference(qf[first:], [1] * B, lens, kv, D ** -0.5)
    assert not got[:first].any()
    assert np.abs(got[first:] - want).max() <= cache_far("f16", D, qf, lens, D ** -0.5)


def lengths_of_many_tiles(B, T, rng):
    n = np.floor(rng.dirichlet(np.full(B, 0.5)) * T).astype(int)
    if B > 2:
        n[B // 2] = 0
    return list(n)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("B", [2, 9, 31])
def test_prompt_attention_of_many_tiles(pipe, B, causal, kind):
    """More tiles than the chip holds at once, of sequences of very different lengths, some with a prefix, some with fewer keys than queries,
    rows of none before and behind them: every row is computed once, by the tile that owns it.  Heads repeat, so that one reference serves."""
    Hkv, G, D, T = 150, 2, 64, 600
    rng = np.random.default_rng(B)
    nq = lengths_of_many_tiles(B, T, rng)
    nk = [int(n * f) for n, f in zip(nq, rng.choice([0.5, 1.0, 1.0, 2.5], B))]
    first, Tq, Tk = 2, 5 + sum(nq), sum(nk)
    q1, qf = typed(rng, (Tq, G, D), kind)
    k1, kf = typed(rng, (Tk, 1, D), kind)
    v1, vf = typed(rng, (Tk, 1, D), kind)
    assert (Tq * G // 128 + B + 1) * Hkv > 512
    q, k, v = q1.repeat(1, Hkv, 1), k1.expand(Tk, Hkv, D), v1.expand(Tk, Hkv, D)
    starts, starts_k = ints(first + np.concatenate([[0], np.cumsum(nq)])), ints(np.concatenate([[0], np.cumsum(nk)]))
    out = torch.full((Tq, Hkv * G, D), float("nan"), dtype=DT[kind], device="cuda")
    pipe.pipe_prompt_attention(q, k, v, starts, starts_k, causal=causal, out=out)
    got = out.view(Tq, Hkv, G, D)
    assert torch.equal(got, got[:, :1].expand_as(got))
    got = got[:, 0].double().cpu().numpy()
    want = prompt_reference(qf[first:], kf, vf, nq, nk, causal, D ** -0.5)
    a = D ** -0.5 * float(np.abs(qf).max()) * float(np.abs(kf).sum(-1).max())
    n = first + sum(nq)
    assert not got[:first].any() and not got[n:].any()
    assert np.abs(got[first:n] - want[:sum(nq)]).max() <= ref.far(kind, D, max(nk), a, float(np.abs(vf).max()))


# ------------------------------------------------------------------ graphs, streams, refusals

def test_a_step_in_a_graph(pipe):
    """Plan, write and attend captured once, replayed over several steps with the caller's work between them."""
    B, Hq, Hkv, D, P, T = 3, 4, 2, 64, 16, 8
    rng = np.random.default_rng(6)
    cached, fresh, used = ints([0, 14, 31]), ints([1, 1, 1]), ints([0, 0, 0])
    free = ints(rng.permutation(30)[:24] + 4)
    table = torch.full((B, 6), -1, dtype=torch.int32, device="cuda")
    table[1, 0], table[2, 0], table[2, 1] = 0, 1, 2
    cache = torch.zeros((34, pipe.pipe_cache_page_bytes(Hkv, D, P)), dtype=torch.uint8, device="cuda")
    x = torch.zeros((T, Hq + 2 * Hkv, D), device="cuda")

    def step():
        lengths, starts, slots, _, counts = pipe.pipe_cache_plan(cached, fresh, P, free, used, table, T)
        pipe.pipe_cache_write(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], slots, cache, P)
        y = pipe.pipe_cache_attention(x[:, :Hq], starts, lengths, cache, table, P, Hkv, max_length=96)
        return y, lengths, counts

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pipe.pipe_prepare_cache_attention(T, Hq, Hkv, D, B, 96)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y, lengths, counts = step()
    torch.cuda.current_stream().wait_stream(side)
    cache.zero_()
    for i in range(5):
        x.copy_(torch.from_numpy(rng.standard_normal(x.shape).astype(np.float32)))
        fresh.copy_(ints(rng.integers(0, 3, B)))
        keep_table, keep_cache = table.clone(), cache.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, lengths, counts, table, cache)]
        table.copy_(keep_table)
        cache.copy_(keep_cache)
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, (*want, table, cache)):
            assert torch.equal(a, b), i
        cached.copy_(lengths)
        used.copy_(counts)


def test_unprepared_capture_is_refused(pipe):
    q = torch.randn(2, 8, 64, device="cuda")
    cache = torch.zeros((4, pipe.pipe_cache_page_bytes(2, 64, 16)), dtype=torch.uint8, device="cuda")
    starts, lengths, table = ints([0, 1, 2]), ints([20, 30]), ints([[0, 1], [2, 3]])
    side = torch.cuda.Stream()
    codes = []
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            try:
                pipe.pipe_cache_attention(q, starts, lengths, cache, table, 16, 2, max_length=1 << 20)
            except pipe.PipeError as e:
                codes.append(e.code)
            q.add(1)
    assert codes in ([], [-6])      # served where no scratch is needed, refused where it would grow


def test_another_stream(pipe):
    rng = np.random.default_rng(12)
    lens = [500, 70]
    cache, table, kv = random_cache(pipe, rng, lens, 2, 64, 16)
    q, qf = typed(rng, (2, 4, 64), "f16")
    want = pipe.pipe_cache_attention(q, ints([0, 1, 2]), ints(lens), cache, table, 16, 2)
    starts, lengths = ints([0, 1, 2]), ints(lens)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(pipe.pipe_cache_attention(q, starts, lengths, cache, table, 16, 2))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_refusals(pipe):
    q, k = torch.randn(4, 4, 64, device="cuda"), torch.randn(4, 2, 64, device="cuda")
    cache = torch.zeros((4, pipe.pipe_cache_page_bytes(2, 64, 16)), dtype=torch.uint8, device="cuda")
    starts, lengths, table, slots = ints([0, 4]), ints([4]), ints([[0]]), ints([0, 1, 2, 3])
    attend = lambda **o: pipe.pipe_cache_attention(**{**dict(q=q, starts=starts, lengths=lengths, cache=cache, table=table,   # noqa: E731
                                                             page_size=16, kv_heads=2), **o})
    prompt = lambda **o: pipe.pipe_prompt_attention(**{**dict(q=q, k=k, v=k, starts=starts), **o})                            # noqa: E731
    for bad in (dict(q=q.double()), dict(q=q.cpu()), dict(q=q[0]), dict(q=q.transpose(1, 2)), dict(starts=starts.long()), dict(starts=ints([0])),
                dict(table=ints([[0], [1]])), dict(page_size=32), dict(kv_heads=4), dict(cache=cache.float()), dict(out=q.half())):
        with pytest.raises(ValueError):
            attend(**bad)
    for bad in (dict(k=k.half()), dict(v=k[:3]), dict(starts=ints([4])), dict(starts_k=ints([0, 2, 4])), dict(q=q[..., :32])):
        with pytest.raises(ValueError):
            prompt(**bad)
    for bad, code in ((dict(scale=float("nan")), -1), (dict(max_length=-1), -2), (dict(q=q[:, :3].contiguous()), -2)):
        with pytest.raises(pipe.PipeError) as e:
            attend(**bad)
        assert e.value.code == code
    for bad, code in ((dict(scale=float("inf")), -1), (dict(q=q[:, :3].contiguous()), -2), (dict(k=k[:3], v=k[:3]), -2),
                      (dict(q=q[..., :32].contiguous(), k=k[..., :32].contiguous(), v=k[..., :32].contiguous()), -2)):
        with pytest.raises(pipe.PipeError) as e:
            prompt(**bad)
        assert e.value.code == code
    for args in ((2, 96, 16), (2, 64, 8), (0, 64, 16)):
        with pytest.raises(ValueError):
            pipe.pipe_cache_page_bytes(*args)
    with pytest.raises(ValueError):
        pipe.pipe_cache_write(k, k, ints([0, 1]), cache, 16)
    with pytest.raises(ValueError):
        pipe.pipe_cache_write(k, k.half(), slots, cache, 16)
    with pytest.raises(ValueError):
        pipe.pipe_cache_plan(ints([0]), ints([1, 2]), 16, ints([0]), ints([0]), table, 4)
    with pytest.raises(pipe.PipeError) as e:
        pipe.pipe_cache_plan(ints([0]), ints([1]), 24, ints([0]), ints([0]), table, 4)
    assert e.value.code == -1
    n = 4097
    with pytest.raises(pipe.PipeError) as e:
        pipe.pipe_cache_plan(ints([0] * n), ints([1] * n), 16, ints([0]), ints([0]), ints([[0]] * n), 4)
    assert e.value.code == -2
    # nothing to do is no error
    assert attend(q=q[:0], starts=ints([0, 0])).shape == (0, 4, 64) and prompt(q=q[:0], k=k[:0], v=k[:0], starts=ints([0, 0])).shape == (0, 4, 64)
    pipe.pipe_cache_write(k[:0], k[:0], slots[:0], cache, 16)
    assert pipe.pipe_cache_read(slots[:0], cache, 16, 2, 64)[0].shape == (0, 2, 64)
