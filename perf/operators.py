"""The operators around attention -- planning the pages of a 4-bit key/value cache, writing and reading it, attention over it and
attention over packed prompts -- as cases for measuring their speed.

listed() gives the cases, draw() more of the same ranges.  prepare() makes what a program holds before the call, run() is one pass
through an operator: the package's calls where `own` is true, the same in elementary torch operations in 32 bits where it is false.
exact() is the operators' definition in 64 bits.

A cache is uint8 [pages, bytes of a page]; a page holds, for every key/value head, P tokens: K codes [P][D/2], V codes [P][D/2] (two
4-bit codes a byte, the even value in the low half), and per token a 32-bit word of K and then of V with the row's scale in bf16 (low
half) and its offset in bf16 (high half).  A value is scale * code + offset.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # the tables of one generation step of 64 conversations: a handful of numbers, all latency
        dict(name="plan_step_b64", op="plan", B=64, fresh_lo=1, fresh_hi=1, cached_lo=1, cached_hi=4000, P=16, spare=0),
        # the tables of a batch of new prompts of very different lengths
        dict(name="plan_prompts_b200", op="plan", B=200, fresh_lo=1, fresh_hi=1900, cached_lo=0, cached_hi=0, P=32, spare=513),
        # keys and values of one generation step into the cache and back, bf16, grouped heads of a 7B-sized layer
        dict(name="cache_step_bf16_t64", op="cache", T=64, Hkv=8, D=128, P=16, dtype="bf16", fused=24),
        # a prompt of a 12-head layer of width 768 of an odd length, fp16
        dict(name="cache_prompt_f16_t4999", op="cache", T=4999, Hkv=12, D=64, P=64, dtype="f16", fused=24),
        # prompts as the package's own layers emit them: fp32, keys and values as two tensors
        dict(name="cache_prompts_f32_t16384", op="cache", T=16384, Hkv=8, D=128, P=32, dtype="f32", fused=0),
        # one conversation, one new token: the time to the next token
        dict(name="decode_one_bf16_777", op="decode", B=1, fresh=1, lo=777, hi=777, Hq=32, Hkv=8, D=128, P=16, dtype="bf16"),
        # a batch of conversations of very different lengths
        dict(name="decode_b48_bf16_ragged", op="decode", B=48, fresh=1, lo=33, hi=8000, Hq=32, Hkv=8, D=128, P=16, dtype="bf16"),
        # two long documents
        dict(name="decode_b2_f16_131072", op="decode", B=2, fresh=1, lo=130001, hi=131072, Hq=32, Hkv=8, D=128, P=64, dtype="f16"),
        # five drafted tokens a conversation to be verified, ungrouped heads of width 64, fp32 as the package's layers emit them
        dict(name="decode_drafts_f32_b16", op="decode", B=16, fresh=5, lo=100, hi=3000, Hq=32, Hkv=32, D=64, P=32, dtype="f32"),
        # one short prompt in a 12-head layer of width 768
        dict(name="prompt_f32_97", op="prompt", B=1, lo=97, hi=97, Hq=12, Hkv=12, D=64, dtype="f32", fused=True),
        # packed prompts of different lengths
        dict(name="prompt_f16_packed_b7", op="prompt", B=7, lo=3, hi=2500, Hq=32, Hkv=8, D=128, dtype="f16", fused=True),
        # one long document
        dict(name="prompt_bf16_8192", op="prompt", B=1, lo=8192, hi=8192, Hq=32, Hkv=8, D=128, dtype="bf16", fused=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; sizes are spread over their logarithm, odd ones among them."""
    op = rng.choice(["plan", "cache", "decode", "decode", "decode", "prompt", "prompt", "prompt"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    D, P = rng.choice([64, 128]), rng.choice([16, 32, 64])
    if op == "plan":
        B = _log_int(rng, 1, 500)
        step = rng.random() < 0.5
        hi = 1 if step else _log_int(rng, 2, max(3, 200000 // B))
        return dict(op="plan", B=B, fresh_lo=1, fresh_hi=hi, cached_lo=rng.choice([0, 1]), cached_hi=_log_int(rng, 1, 5000), P=P,
                    spare=rng.choice([0, 0, rng.randint(1, 1000)]))
    if op == "cache":
        Hkv = rng.choice([1, 4, 8, 12, 32])
        return dict(op="cache", T=_log_int(rng, 1, 16384 * 8 * 128 // (Hkv * D)), Hkv=Hkv, D=D, P=P, dtype=dtype,
                    fused=rng.choice([0, Hkv * 2]))
    if op == "decode":
        Hkv, G = rng.choice([(8, 4), (8, 8), (4, 7), (32, 1), (1, 16), (2, 12)])
        fresh = rng.choice([1, 1, 1, 2, 5, 8])
        B = _log_int(rng, 1, 64)
        top = max(64, min(131072, 48 * 8000 * 8 * 128 // (B * Hkv * D)))
        hi = _log_int(rng, 16, top)
        return dict(op="decode", B=B, fresh=fresh, lo=rng.choice([fresh, max(fresh, hi // 2), max(fresh, hi)]), hi=max(fresh, hi),
                    Hq=Hkv * G, Hkv=Hkv, D=D, P=P, dtype=dtype)
    Hkv, G = rng.choice([(8, 4), (8, 8), (4, 7), (12, 1), (32, 1), (2, 16)])
    B = _log_int(rng, 1, 16)
    top = int(math.sqrt(8192.0 ** 2 * 32 / (B * Hkv * G)))
    hi = _log_int(rng, 1, min(top, 8192 if dtype != "f32" else 4096))
    return dict(op="prompt", B=B, lo=rng.choice([1, max(1, hi // 2), hi]), hi=hi, Hq=Hkv * G, Hkv=Hkv, D=D, dtype=dtype,
                fused=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------ inputs


def _spread(n, lo, hi, salt):
    """n whole numbers of [lo, hi], spread evenly in a scattered order; the last one is hi."""
    v = [lo + ((i + 1) * 2654435761 + salt * 40503) % 4294967296 * (hi - lo + 1) // 4294967296 for i in range(n)]
    v[-1] = hi
    return v


def _gen(seed):
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return g, dev


def _ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _starts(lens, dev):
    return _ints([0] + list(np.cumsum(lens)), dev)


def _heads(g, dev, T, counts, D, dtype, fused):
    """Activations of head groups [T, H, D] -- slices of one projection's output where `fused`.  N(0, 1) with a few channels of a
    head larger than the rest, as keys have them."""
    gain = torch.ones(D, device=dev)
    gain[torch.randperm(D, generator=g, device=dev)[:2]] = 6.0
    if fused:
        x = torch.randn(T, sum(counts), D, generator=g, device=dev).mul_(gain).to(dtype)
        return list(x.split(counts, dim=1))
    return [torch.randn(T, n, D, generator=g, device=dev).mul_(gain).to(dtype) for n in counts]


def _plan_lens(case):
    return _spread(case["B"], case["cached_lo"], case["cached_hi"], 1), _spread(case["B"], case["fresh_lo"], case["fresh_hi"], 2)


def _page_bytes(case):
    return case["Hkv"] * case["P"] * (case["D"] + 8)


def _decode_lens(case):
    return _spread(case["B"], case["lo"], case["hi"], 3)


def prepare(case, seed):
    g, dev = _gen(seed)
    op = case["op"]
    s = dict(case=case)
    if op == "plan":
        cached, fresh = _plan_lens(case)
        P = case["P"]
        have, need = [-(-c // P) for c in cached], [-(-(c + f) // P) for c, f in zip(cached, fresh)]
        width = max(need) + 3
        pool = torch.randperm(sum(need) + 17, generator=g, device=dev).int()
        table = torch.full((case["B"], width), -1, dtype=torch.int32, device=dev)
        held = torch.arange(width, device=dev)[None] < torch.tensor(have, device=dev)[:, None]
        table[held] = pool[:sum(have)]
        s.update(cached=_ints(cached, dev), fresh=_ints(fresh, dev), table=table, free=pool[sum(have):].contiguous(),
                 used=_ints([3, 0, 0], dev), tokens=sum(fresh) + case["spare"])
        return s
    P, D, Hkv, dtype = case["P"] if "P" in case else 0, case["D"], case["Hkv"], DTYPES[case["dtype"]]
    if op == "cache":
        T = case["T"]
        pages = -(-T // P) + 5
        k, v = _heads(g, dev, T, [Hkv, Hkv] + ([case["fused"]] if case["fused"] else []), D, dtype, case["fused"] > 0)[:2]
        order = torch.randperm(pages, generator=g, device=dev)          # the pages of a pool that has been in use
        t = torch.arange(T, device=dev)
        s.update(k=k, v=v, slots=(order[t // P] * P + t % P).int(),
                 cache=torch.randint(0, 256, (pages, _page_bytes(case)), generator=g, device=dev, dtype=torch.uint8))
        return s
    if op == "decode":
        lens, B = _decode_lens(case), case["B"]
        need = [-(-n // P) for n in lens]
        width, pages = max(need) + 1, sum(need) + 2
        order = torch.randperm(pages, generator=g, device=dev).int()
        table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
        table[torch.arange(width, device=dev)[None] < torch.tensor(need, device=dev)[:, None]] = order[:sum(need)]
        cache = torch.randint(0, 256, (pages, Hkv, P * (D + 8)), generator=g, device=dev, dtype=torch.uint8)
        # scales and offsets of rows that are about N(0, 1)
        scale = (0.3 + 0.1 * torch.rand(pages, Hkv, 2 * P, generator=g, device=dev)).bfloat16()
        offset = (-7.5 * scale.float() + 0.2 * torch.randn(pages, Hkv, 2 * P, generator=g, device=dev)).bfloat16()
        cache[:, :, P * D:] = torch.stack([scale, offset], dim=-1).view(torch.uint8).reshape(pages, Hkv, 8 * P)
        T = B * case["fresh"]
        q = _heads(g, dev, T, [case["Hq"]], D, dtype, False)[0]
        s.update(q=q, starts=_starts([case["fresh"]] * B, dev), lengths=_ints(lens, dev), cache=cache.view(pages, -1), table=table)
        return s
    lens = _spread(case["B"], case["lo"], case["hi"], 4)
    q, k, v = _heads(g, dev, sum(lens), [case["Hq"], Hkv, Hkv], D, dtype, case["fused"])
    s.update(q=q, k=k, v=v, starts=_starts(lens, dev), longest=max(lens))
    return s


# ------------------------------------------------------------------------------------------ the operators' plain forms


def _plain_plan(s):
    cached, fresh, free, P = s["cached"].long(), s["fresh"].long(), s["free"], s["case"]["P"]
    table, T = s["table"], s["tokens"]
    width, n_free = table.shape[1], free.numel()
    zero = torch.zeros(1, dtype=torch.int64, device=table.device)
    starts = torch.cat([zero, fresh.cumsum(0)])
    total = cached + fresh
    have, need = (cached + P - 1) // P, (total + P - 1) // P
    base = torch.cat([zero, (need - have).cumsum(0)])
    col = torch.arange(width, device=table.device)[None]
    at = s["used"][0] + base[:-1, None] + col - have[:, None]
    page = torch.where(at < n_free, free[at.clamp(0, n_free - 1)], -1)
    table.copy_(torch.where((col >= have[:, None]) & (col < need[:, None]), page, table))
    marks = torch.zeros(T + 1, dtype=torch.int64, device=table.device)
    marks.index_add_(0, starts[1:-1].clamp(max=T), torch.ones_like(starts[1:-1]))
    t = torch.arange(T, device=table.device)
    b = marks.cumsum(0)[:T]
    pos = cached[b] + t - starts[b]
    page = table[b, (pos // P).clamp(0, width - 1)].long()
    live = t < starts[-1]
    slots = torch.where(live & (page >= 0), page * P + pos % P, -1)
    wanted = s["used"][0] + base[-1]
    counts = torch.stack([wanted.clamp(max=n_free), (wanted - n_free).clamp(min=0), zero[0]])
    return total.int(), starts.int(), slots.int(), torch.where(live, pos, -1).int(), counts.int(), table


def _plain_rows(x):
    """(codes, scale, offset) of rows in 4 bits."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    m = lo.bfloat16()
    m = torch.where(m.float() > lo, torch.nextafter(m, torch.full_like(m, -math.inf)), m).float()
    w = (hi - m) / torch.full_like(hi, 15.0)
    s = w.bfloat16()
    s = torch.where(s.float() < w, torch.nextafter(s, torch.full_like(s, math.inf)), s).float()
    s = torch.where(s < 2.0 ** -126, 0.0, s)
    r = torch.where(s > 0, 1.0 / s, 0.0)
    return ((x - m) * r).round().clamp(0, 15), s, m


def _plain_cache(s):
    case, slots = s["case"], s["slots"].long()
    P, D, Hkv, dtype = case["P"], case["D"], case["Hkv"], s["k"].dtype
    pages = s["cache"].shape[0]
    blocks = s["cache"].view(pages, Hkv, P * (D + 8))
    codes = blocks[:, :, :P * D].view(pages, Hkv, 2, P, D // 2)
    words = blocks[:, :, P * D:].view(torch.bfloat16).view(pages, Hkv, 2, P, 2)
    pg, off = slots // P, slots % P
    x = torch.stack([s["k"], s["v"]], dim=2)                                   # [T, Hkv, 2, D]
    c, sc, m = _plain_rows(x)
    c = c.to(torch.uint8).view(*c.shape[:-1], D // 2, 2)
    codes[pg, :, :, off] = c[..., 0] | (c[..., 1] << 4)
    words[pg, :, :, off] = torch.cat([sc, m], dim=-1).bfloat16()
    back, w = codes[pg, :, :, off], words[pg, :, :, off].float()               # and read back
    c = torch.stack([back & 15, back >> 4], dim=-1).flatten(-2).float()
    x = (w[..., :1] * c + w[..., 1:]).to(dtype)
    return x[:, :, 0], x[:, :, 1]


def _softmax_rows(S, seen):
    S = S.masked_fill(~seen, -math.inf)
    top = S.amax(-1, keepdim=True)
    p = torch.exp(S - torch.where(top == -math.inf, 0.0, top))
    return p / p.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_decode(s):
    case = s["case"]
    P, D, Hkv, n, B = case["P"], case["D"], case["Hkv"], case["fresh"], case["B"]
    G = case["Hq"] // Hkv
    W = -(-max(_decode_lens(case)) // P)
    pages = s["cache"].view(-1, Hkv, P * (D + 8))[s["table"][:, :W].long().clamp(min=0)]       # [B, W, Hkv, bytes]
    codes = pages[..., :P * D].reshape(B, W, Hkv, 2, P, D // 2)
    w = pages[..., P * D:].contiguous().view(torch.bfloat16).view(B, W, Hkv, 2, P, 2).float()
    x = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).float() * w[..., :1] + w[..., 1:]
    kv = x.permute(3, 0, 2, 1, 4, 5).reshape(2, B, Hkv, W * P, D)
    q = s["q"].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    S = torch.matmul(q, kv[0].transpose(-1, -2)) * D ** -0.5
    last = s["lengths"].long()[:, None] - n + torch.arange(n, device=q.device)[None]             # the last token that is seen
    seen = torch.arange(W * P, device=q.device) <= last.repeat_interleave(G, dim=1)[:, None, :, None]
    o = torch.matmul(_softmax_rows(S, seen), kv[1])
    return o.view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B * n, case["Hq"], D).to(s["q"].dtype)


def _plain_prompt(s):
    case, starts = s["case"], s["starts"].long()
    L, B, Hkv, D = s["longest"], case["B"], case["Hkv"], case["D"]
    G = case["Hq"] // Hkv
    at = torch.arange(L, device=starts.device)
    lens = starts[1:] - starts[:-1]
    rows = (starts[:-1, None] + at[None]).clamp(max=s["q"].shape[0] - 1)                        # [B, L]
    q = s["q"].float()[rows].view(B, L, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * L, D)
    k, v = (s[name].float()[rows].transpose(1, 2) for name in ("k", "v"))                       # [B, Hkv, L, D]
    S = torch.matmul(q, k.transpose(-1, -2)) * D ** -0.5
    seen = (at[None, :] <= at[:, None])[None] & (at[None, None, :] < lens[:, None, None])
    o = torch.matmul(_softmax_rows(S.view(B, Hkv, G, L, L), seen[:, None, None]).view(B, Hkv, G * L, L), v)
    o = o.view(B, Hkv, G, L, D).permute(0, 3, 1, 2, 4).reshape(B, L, case["Hq"], D)
    return o[at[None] < lens[:, None]].to(s["q"].dtype)


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"plan": _plain_plan, "cache": _plain_cache, "decode": _plain_decode, "prompt": _plain_prompt}[op](s)
    import paper_2311_15806_amd.binding as pipe
    case = s["case"]
    if op == "plan":
        return (*pipe.pipe_cache_plan(s["cached"], s["fresh"], case["P"], s["free"], s["used"], s["table"], s["tokens"]), s["table"])
    if op == "cache":
        pipe.pipe_cache_write(s["k"], s["v"], s["slots"], s["cache"], case["P"])
        return pipe.pipe_cache_read(s["slots"], s["cache"], case["P"], case["Hkv"], case["D"], s["k"].dtype)
    if op == "decode":
        return pipe.pipe_cache_attention(s["q"], s["starts"], s["lengths"], s["cache"], s["table"], case["P"], case["Hkv"],
                                         max_length=case["hi"])
    return pipe.pipe_prompt_attention(s["q"], s["k"], s["v"], s["starts"])


# ------------------------------------------------------------------------------------------ what they cannot do without


def work(case):
    """Every input once, every output once; two operations per multiply-add of the two products over the visible pairs."""
    op = case["op"]
    if op == "plan":
        cached, fresh = _plan_lens(case)
        new = sum(-(-(c + f) // case["P"]) - -(-c // case["P"]) for c, f in zip(cached, fresh))
        return {"bytes": 4 * (2 * case["B"] + 2 * case["B"] + 1 + 6 + 2 * (sum(fresh) + case["spare"]) + 2 * new), "flops": 0}
    size, D = 4 if case["dtype"] == "f32" else 2, case["D"]
    if op == "cache":
        rows = 2 * case["T"] * case["Hkv"]
        return {"bytes": rows * (2 * D * size + 2 * (D / 2 + 4)) + 8 * case["T"], "flops": 0}
    if op == "decode":
        lens, n = _decode_lens(case), case["fresh"]
        pairs = sum(n * L - n * (n - 1) // 2 for L in lens)
        table = 4 * sum(-(-L // case["P"]) for L in lens)
        return {"bytes": sum(lens) * case["Hkv"] * (D + 8) + 2 * case["B"] * n * case["Hq"] * D * size + table + 8 * case["B"],
                "flops": 4.0 * D * case["Hq"] * pairs}
    lens = _spread(case["B"], case["lo"], case["hi"], 4)
    return {"bytes": 2 * sum(lens) * (case["Hq"] + case["Hkv"]) * D * size + 4 * case["B"],
            "flops": 4.0 * D * case["Hq"] * sum(L * (L + 1) // 2 for L in lens)}


# ------------------------------------------------------------------------------------------ the same in 64 bits


def _exact_plan(s):
    case = s["case"]
    P, T = case["P"], s["tokens"]
    cached, fresh, free, table = (s[name].cpu().numpy().astype(np.int64) for name in ("cached", "fresh", "free", "table"))
    starts, slots, positions, nxt, missing = [0], np.full(T, -1), np.full(T, -1), int(s["used"][0]), 0
    for b in range(case["B"]):
        for j in range(-(-int(cached[b]) // P), -(-int(cached[b] + fresh[b]) // P)):
            if nxt < len(free):
                table[b, j], nxt = free[nxt], nxt + 1
            else:
                table[b, j], missing = -1, missing + 1
        p = cached[b] + np.arange(fresh[b])
        at = slice(starts[-1], starts[-1] + int(fresh[b]))
        positions[at] = p
        page = table[b, p // P]
        slots[at] = np.where(page >= 0, page * P + p % P, -1)
        starts.append(at.stop)
    out = (cached + fresh, starts, slots, positions, [nxt, missing, 0], table)
    return tuple(torch.from_numpy(np.asarray(v).astype(np.int32)) for v in out)


def _to_bf16(x, up):
    """fp64 values that are fp32 ones, to the bf16 value next to them below or above, by the bits."""
    u = x.float().contiguous().view(torch.int32).cpu().numpy().view(np.uint32).astype(np.int64)
    cut = (u & 0xffff) != 0
    away = cut & ((u >> 31 == 0) if up else (u >> 31 == 1))
    u = (u & 0xffff0000) + np.where(away, 0x10000, 0)
    return torch.from_numpy(u.astype(np.uint32).view(np.float32).astype(np.float64)).to(x.device)


def _exact_rows(x):
    """The values that 4-bit rows stand for: the codes follow by definition from arithmetic that is rounded to fp32."""
    f = lambda t: t.float().double()                                           # noqa: E731
    x = x.double()
    m = _to_bf16(x.min(-1, keepdim=True).values, False)
    s = _to_bf16(f(f(x.max(-1, keepdim=True).values - m) / 15.0), True)
    s = torch.where(s < 2.0 ** -126, torch.zeros_like(s), s)
    r = torch.where(s > 0, f(1.0 / s), torch.zeros_like(s))
    return s * torch.round(f(f(x - m) * r)).clamp(0, 15) + m


def _exact_attend(q, k, v, last):
    """q [n, H, D], k and v [t, H, D] in fp64; last [n]: the last key a query sees."""
    S = torch.einsum("nhd,thd->hnt", q, k) * q.shape[-1] ** -0.5
    S = S.masked_fill(torch.arange(k.shape[0], device=q.device)[None, None] > last[None, :, None], -math.inf)
    return torch.einsum("hnt,thd->nhd", torch.softmax(S, dim=-1), v)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "plan":
        return _exact_plan(s)
    if op == "cache":
        return _exact_rows(s["k"]), _exact_rows(s["v"])
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    G, out = Hq // Hkv, []
    if op == "decode":
        P, n = case["P"], case["fresh"]
        for b, L in enumerate(_decode_lens(case)):
            pages = s["cache"][s["table"][b, :-(-L // P)].long()].view(-1, Hkv, P * (D + 8))
            q = s["q"][b * n:(b + 1) * n].double()
            last = L - n + torch.arange(n, device=q.device)
            for h in range(Hkv):
                kv = []
                for side in range(2):
                    c = pages[:, h, side * P * D // 2:(side + 1) * P * D // 2].reshape(-1, D // 2)
                    w = pages[:, h, P * D + 4 * P * side:P * D + 4 * P * (side + 1)].reshape(-1, 4).contiguous().view(torch.bfloat16).double()
                    x = torch.empty(c.shape[0], D, dtype=torch.float64, device=c.device)
                    x[:, 0::2], x[:, 1::2] = c % 16, c // 16
                    kv.append((x * w[:, :1] + w[:, 1:])[:L, None].expand(-1, G, -1))
                out.append(_exact_attend(q[:, h * G:(h + 1) * G], *kv, last))
        return torch.cat([torch.cat(out[i:i + Hkv], dim=1) for i in range(0, len(out), Hkv)])
    starts = s["starts"].tolist()
    for a, e in zip(starts, starts[1:]):
        parts = []
        for h in range(Hq):
            parts.append(_exact_attend(s["q"][a:e, h:h + 1].double(), s["k"][a:e, h // G:h // G + 1].double(),
                                       s["v"][a:e, h // G:h // G + 1].double(), torch.arange(e - a, device=s["q"].device)))
        out.append(torch.cat(parts, dim=1))
    return torch.cat(out)
