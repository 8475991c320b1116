"""The operators around attention from their definitions, in numpy: whole numbers for the tables, fp32 steps for the codes (each rounded
once, as the definition says), fp64 for the attentions; and how far fp32 arithmetic may be from it."""
import numpy as np

U32 = 2.0 ** -24                                             # unit roundoff of fp32
UNIT = {"f32": 2.0 ** -22, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # of a softmax weight and of an output (fp32: two fp16 terms)


def plan(cached, fresh, P, free, used, table, T):
    """(lengths, starts, slots, positions, counts, table)"""
    table = table.copy()
    width = table.shape[1]
    lengths, starts, nxt, missing, cut = [], [0], min(max(used, 0), len(free)), 0, 0
    slots, pos = np.full(T, -1, np.int64), np.full(T, -1, np.int64)
    for b in range(len(cached)):
        c, want = max(0, int(cached[b])), max(0, int(fresh[b]))
        n = min(want, T - starts[-1])
        cut += want - n
        for j in range(-(-c // P), -(-(c + n) // P)):
            if j >= width:
                missing += 1
            elif nxt < len(free):
                table[b, j], nxt = free[nxt], nxt + 1
            else:
                table[b, j], missing = -1, missing + 1
        for i in range(n):
            p = c + i
            page = int(table[b, p // P]) if p // P < width else -1
            slots[starts[-1] + i] = page * P + p % P if page >= 0 else -1
            pos[starts[-1] + i] = p
        lengths.append(c + n)
        starts.append(starts[-1] + n)
    return (np.array(lengths), np.array(starts), slots, pos, np.array([nxt, missing, cut]), table)


def _bf16(x, up):
    """The bf16 value next to x below or equal / above or equal, as fp32."""
    x = np.ascontiguousarray(x, np.float32)
    cut = (x.view(np.uint32) & 0xffff0000).view(np.float32)   # towards zero
    away = (x.view(np.uint32) & 0xffff) != 0
    step = away & ((x > 0) if up else (x < 0))
    return np.where(step, (cut.view(np.uint32) + np.uint32(0x10000)).view(np.float32), cut)


def quantize_rows(x):
    """(codes uint8, scale fp32, offset fp32) of the rows x [..., D] (fp32 values); NaN scale and offset for a bad row."""
    f = np.float32
    x = np.asarray(x, f)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
        m = _bf16(lo, False)
        s = _bf16((hi - m).astype(f) / f(15), True)
        s = np.where(s < f(2.0 ** -126), f(0), s)
        r = np.where(s > 0, f(1) / np.where(s > 0, s, f(1)), f(0)).astype(f)
        c = np.clip(np.rint(((x - m).astype(f) * r).astype(f)), 0, 15)
    bad = ~np.isfinite(x).all(-1, keepdims=True) | ~np.isfinite(s) | ~np.isfinite(m)
    c = np.where(bad, 0, np.nan_to_num(c)).astype(np.uint8)
    return c, np.where(bad, f(np.nan), s).astype(f), np.where(bad, f(np.nan), m).astype(f)


def block_of(k_codes, v_codes, k_sm, v_sm):
    """One head's part of a page: codes [P, D] and (scale, offset) [P, 2] of K and V -> uint8 [P * (D + 8)]."""
    def nib(c):
        return (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8).reshape(-1)

    def words(sm):
        u = np.ascontiguousarray(sm, np.float32).view(np.uint32)
        return ((u[:, 0] >> 16) | (u[:, 1] & 0xffff0000)).astype(np.uint32).view(np.uint8)

    return np.concatenate([nib(k_codes), nib(v_codes), words(k_sm), words(v_sm)])


def attend(q, k, v, scale, seen):
    """q [n, H, D], k and v [m, Hkv, D] in fp64, seen [n]: how many keys a query sees -> [n, H, D]; zeros where it sees none."""
    n, H, D = q.shape
    G = H // k.shape[1]
    out = np.zeros((n, H, D))
    for i in range(n):
        s = int(max(0, seen[i]))
        if s == 0:
            continue
        for h in range(H):
            S = scale * (k[:s, h // G] @ q[i, h])
            p = np.exp(S - S.max())
            out[i, h] = (p @ v[:s, h // G]) / p.sum()
    return out


def far(kind, D, n, a, v):
    """How far an output may be from the exact one.  a: the largest sum of magnitudes that a score is summed from (scaled), v: the
    largest magnitude of a value, n: keys.  A score of D + 8 roundings is off by (D + 8) u a, which is the relative error of its weight
    in the numerator and in the sum; the weight and the output are rounded to the type; n additions; fp32 splits q into two fp16 terms."""
    split = 2.0 ** -21 * a
    return v * (2 * UNIT[kind] + 2 * (D + 8) * U32 * a + 2 * split + 2 * (n + 16) * U32)
