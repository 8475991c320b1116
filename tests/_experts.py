"""The layers with a scale for each token and the experts' operators from their definitions, in numpy: codes by fp32 steps (each rounded once, as the
definition says), everything else in fp64; and how far fp32 arithmetic may be from it."""
import numpy as np
from scipy.special import erfc

U32 = 2.0 ** -24                                                   # half a step of fp32, relative
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # ... of an output
LEAST = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}   # ... of the smallest ones, absolute
ACTS = {"none": 0, "gelu": 1, "gated": 2, "relu": 3}


def quantize(x):
    """(codes int8 [rows, n], scales fp32 [rows]) of rows of fp32 values."""
    f = np.float32
    x = np.asarray(x, f)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(x).all(1)
        top = np.abs(np.where(bad[:, None], f(0), x)).max(1, initial=0)
        s = (top / f(127)).astype(f)
        s = np.where(s < f(2.0 ** -126), f(0), s)
        q = np.rint((x / np.where(s > 0, s, f(1))[:, None]).astype(f))
        c = np.where((s > 0)[:, None] & ~bad[:, None], np.clip(q, -127, 127), 0).astype(np.int8)
    return c, np.where(bad, f(np.nan), s).astype(f)


def sums(c, w):
    """Exact whole sums [T, rows] (fp64 holds them)."""
    return c.astype(np.float64) @ w.astype(np.float64).T


def layer(acc, sx, sw, bias, act, kind):
    """(y, how far an output may be from it): z = (acc rounded) * two mantissas, a bias added: three roundings of the product and one of the sum."""
    with np.errstate(all="ignore"):
        z0 = acc * sx.astype(np.float64)[:, None] * sw.astype(np.float64)[None]
        z = z0 if bias is None else z0 + bias.astype(np.float64)[None]
        # (a product under fp32's normal range is rounded to its smallest step)
        dz = 3.01 * U32 * np.abs(z0) + (1.01 * U32 * np.abs(z) if bias is not None else 0) + 2.0 ** -149
        if act == "gelu":
            y = 0.5 * z * erfc(-z / np.sqrt(2.0))
            # its slope is at most 1.13; the polynomial's error is 2e-8 of the argument at most (stated beside it), some roundings more
            dy = 1.13 * dz + 8 * U32 * np.abs(z)
        elif act == "relu":
            y, dy = np.where(z < 0, 0.0, z), dz
        elif act == "gated":
            h = z.shape[1] // 2
            g, u, dg, du = z[:, :h], z[:, h:], dz[:, :h], dz[:, h:]
            s = g / (1.0 + np.exp(-g))
            # slope of SiLU at most 1.1; exp is within two steps, 1 + exp and the quotient one rounding each, the product one
            dy = np.abs(u) * (1.1 * dg + 8 * U32 * np.abs(s) + 2.0 ** -149) + np.abs(s) * du * (1 + 1e-6)
            y = s * u
        else:
            y, dy = z, dz
        return y, dy + HALF[kind] * (np.abs(y) + dy) + LEAST[kind]


def linear(x, w, sw, bias, act, kind):
    c, s = quantize(x)
    return layer(sums(c, w), s, sw, bias, act, kind)


def sort(experts, E):
    flat = experts.reshape(-1)
    here = (flat >= 0) & (flat < E)
    key = np.where(here, flat, E)
    order = np.argsort(key, kind="stable")
    starts = np.concatenate([[0], np.cumsum(np.bincount(key, minlength=E + 1)[:E])])
    places = np.full(flat.shape, -1)
    n = starts[-1]
    places[order[:n]] = np.arange(n)
    return starts, np.where(np.arange(flat.size) < n, order, -1), places.reshape(experts.shape)


def route(logits, k, renormalize):
    """(experts, weights) of fp64 logits."""
    T, E = logits.shape
    experts, weights = np.full((T, k), -1), np.zeros((T, k))
    for t in range(T):
        l = np.where(np.isnan(logits[t]), -np.inf, logits[t])
        chosen = [e for e in sorted(range(E), key=lambda e: (-l[e], e))[:k] if l[e] > -np.inf]
        experts[t, :len(chosen)] = chosen
        if chosen:
            with np.errstate(all="ignore"):
                p = np.exp(logits[t] - l[chosen[0]])
            weights[t, :len(chosen)] = p[chosen] / (p[chosen].sum() if renormalize else p.sum())
    return experts, weights


def experts_layer(x, w, sw, bias, starts, order, k, n, act, kind):
    """Rows [n, out] and how far they may be: expert e's layer on its rows, zeros elsewhere."""
    out = w.shape[1] // (2 if act == "gated" else 1)
    y, far = np.zeros((n, out)), np.zeros((n, out))
    for e in range(w.shape[0]):
        r = np.arange(starts[e], starts[e + 1])
        src = r if order is None else order[r] // k
        ok = (src >= 0) & (src < x.shape[0])
        r, src = r[ok], src[ok]
        if r.size:
            y[r], far[r] = linear(x[src], w[e], sw[e], None if bias is None else bias[e], act, kind)
    return y, far


def combine(y, places, weights, kind):
    """(out, how far it may be): a product and a sum of k terms in fp32, one rounding to the type."""
    T, k = places.shape
    out, size = np.zeros((T, y.shape[1])), np.zeros((T, y.shape[1]))
    for j in range(k):
        t = np.nonzero((places[:, j] >= 0) & (places[:, j] < y.shape[0]))[0]
        term = weights[t, j, None] * y[places[t, j]]
        out[t] += term
        size[t] += np.abs(term)
    far = (k + 1) * U32 * size
    return out, far + HALF[kind] * (np.abs(out) + far) + LEAST[kind]
