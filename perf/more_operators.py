"""Products in 8-bit integers with a scale for each token and channel, and the same with a router's experts -- choosing the experts and
sorting the tokens by them, the experts' products, their weighted sum for each token -- as cases for measuring their speed.

listed() gives the cases, draw() more of the same ranges.  prepare() makes what a program holds before the call, run() is one pass
through an operator: the package's calls where `own` is true, the same in elementary torch operations in 32 bits where it is false.
exact() is the operators' definition in 64 bits.

Codes of weights are int8 [.., out, pitch], pitch the number of inputs rounded up to 128; a layer with a gate has the gate's rows first, then
as many of the other half.  An input row's scale is the largest magnitude / 127, its codes are the quotients by it to the nearest integer, half to even.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = {"none": 0, "gelu": 1, "gated": 2, "relu": 3}


def listed():
    return [
        # a projection of the next token of one conversation
        dict(name="linear_bf16_t1", op="linear", T=1, n_in=4096, n_out=4096, act="none", bias=False, dtype="bf16"),
        # the gated layer of a 7B-sized MLP for one generation step of 16 conversations
        dict(name="linear_gated_bf16_t16", op="linear", T=16, n_in=4096, n_out=11008, act="gated", bias=False, dtype="bf16"),
        # sizes that fit no tile, with everything an epilogue does
        dict(name="linear_gelu_f16_t333_odd", op="linear", T=333, n_in=1000, n_out=1537, act="gelu", bias=True, dtype="f16"),
        # prompts through a 7B-sized layer in the package's own type
        dict(name="linear_f32_t4096", op="linear", T=4096, n_in=4096, n_out=11008, act="none", bias=True, dtype="f32"),
        # a generation step's choice of experts: all latency
        dict(name="route_f32_t48_e64", op="route", T=48, E=64, k=6, renormalize=True, masked=0, dtype="f32"),
        # prompts' choice, with experts that are switched off
        dict(name="route_bf16_t16384_e128", op="route", T=16384, E=128, k=8, renormalize=False, masked=3, dtype="bf16"),
        # one token's two experts of eight
        dict(name="experts_f16_t1_e8", op="experts", T=1, k=2, E=8, absent=0, n_in=4096, n_out=4096, act="none", bias=False, gather=True, dtype="f16"),
        # a generation step through many small gated experts, most of which get a few tokens
        dict(name="experts_gated_bf16_t32_e64", op="experts", T=32, k=6, E=64, absent=0, n_in=2048, n_out=1408, act="gated", bias=False, gather=True, dtype="bf16"),
        # rows that lie by expert already (a layer's second product), a part of the experts on another device, fp32
        dict(name="experts_f32_t1001_e12", op="experts", T=1001, k=4, E=12, absent=4, n_in=1408, n_out=2048, act="none", bias=True, gather=False, dtype="f32"),
        # prompts through a layer of eight 7B-sized gated experts
        dict(name="experts_gated_bf16_t4096_e8", op="experts", T=4096, k=2, E=8, absent=0, n_in=4096, n_out=11008, act="gated", bias=False, gather=True, dtype="bf16"),
        # a generation step's results back in their tokens' order
        dict(name="combine_bf16_t32", op="combine", T=32, k=6, H=2048, absent=0, dtype="bf16"),
        # prompts' results, a quarter of the experts on another device
        dict(name="combine_f16_t8192", op="combine", T=8192, k=8, H=4096, absent=4, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """A layer's width: mostly of a multiple of 64, as layers have them, else any number."""
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.7 else n


def draw(rng):
    """One more case of the ranges above; sizes are spread over their logarithm, odd ones among them."""
    op = rng.choice(["linear", "linear", "linear", "route", "experts", "experts", "experts", "combine"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    if op == "route":
        E = _log_int(rng, 2, 256)
        k = rng.randint(1, min(8, E))
        return dict(op="route", T=_log_int(rng, 1, 16384), E=E, k=k, renormalize=rng.random() < 0.5,
                    masked=rng.choice([0, 0, rng.randint(0, E - 1)]), dtype=dtype)
    if op == "combine":
        k, H = rng.randint(1, 8), _width(rng, 64, 8192)
        return dict(op="combine", T=_log_int(rng, 1, 8192 * 8 * 4096 // (k * H) if dtype != "f32" else 4096 * 8 * 4096 // (k * H)), k=k, H=H,
                    absent=rng.choice([0, 0, 2, 8]), dtype=dtype)
    act = rng.choice(["none", "none", "gelu", "gated", "relu"])
    n_in, n_out = _width(rng, 64, 8192), _width(rng, 64, 11008)
    rows = n_out * (2 if act == "gated" else 1)
    if op == "linear":
        return dict(op="linear", T=_log_int(rng, 1, min(8192, 4096 * 4096 * 11008 // (n_in * rows))), n_in=n_in, n_out=n_out, act=act,
                    bias=rng.random() < 0.5, dtype=dtype)
    n_in, n_out = min(n_in, 4096), min(n_out, 4096)
    rows = n_out * (2 if act == "gated" else 1)
    E = _log_int(rng, 2, max(2, min(128, 400_000_000 // (n_in * rows))))
    k = rng.randint(1, min(8, E))
    return dict(op="experts", T=_log_int(rng, 1, max(1, min(8192, 4096 * 4096 * 11008 // (n_in * rows)) // k)), k=k, E=E, absent=rng.choice([0, 0, E // 3]),
                n_in=n_in, n_out=n_out, act=act, bias=rng.random() < 0.3, gather=rng.random() < 0.6, dtype=dtype)


# ------------------------------------------------------------------------------------------ inputs


def _gen(seed):
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return g, dev


def _pitch(n):
    return -(-n // 128) * 128


def _tokens(g, dev, T, n, dtype):
    """Activations: N(0, 1) of a size that differs by token, and a few channels larger than the rest."""
    gain = torch.ones(n, device=dev)
    gain[torch.randperm(n, generator=g, device=dev)[:max(1, n // 200)]] = 12.0
    size = torch.exp(torch.randn(T, 1, generator=g, device=dev) * 0.5)
    return (torch.randn(T, n, generator=g, device=dev) * gain * size).to(dtype)


def _weights(g, dev, lead, rows, n):
    """Codes [*lead, rows, pitch] of normal weights and the scales [*lead, rows]."""
    codes = torch.zeros(*lead, rows, _pitch(n), dtype=torch.int8, device=dev)
    flat = codes.view(-1, rows, codes.shape[-1])
    for e in range(flat.shape[0]):
        flat[e, :, :n] = torch.randn(rows, n, generator=g, device=dev).mul_(32).round_().clamp_(-127, 127).to(torch.int8)
    scales = (0.6 + 0.8 * torch.rand(*lead, rows, generator=g, device=dev)) / (32 * math.sqrt(n))
    return codes, scales


def _rows(case):
    return case["n_out"] * (2 if case["act"] == "gated" else 1)


def _choice(case):
    """Experts [T][k] of a case, -1 for one that is not here; low numbers are chosen more often."""
    every = case["E"] + case["absent"]
    out = []
    for t in range(case["T"]):
        u = ((t + 1) * 2654435761 % 4294967296) / 4294967296
        base = int(every * u ** 1.5)
        out.append([e if e < case["E"] else -1 for e in ((base + j) % every for j in range(case["k"]))])
    return out


def _counts(case):
    n = [0] * case["E"]
    for row in _choice(case):
        for e in row:
            if e >= 0:
                n[e] += 1
    return n


def prepare(case, seed):
    g, dev = _gen(seed)
    op, dtype = case["op"], DTYPES[case["dtype"]]
    s = dict(case=case)
    if op == "linear":
        codes, scales = _weights(g, dev, (), _rows(case), case["n_in"])
        s.update(x=_tokens(g, dev, case["T"], case["n_in"], dtype), codes=codes, scales=scales,
                 bias=torch.randn(_rows(case), generator=g, device=dev) * 0.1 if case["bias"] else None)
        return s
    if op == "route":
        logits = torch.randn(case["T"], case["E"], generator=g, device=dev) * 1.5 + torch.randn(case["E"], generator=g, device=dev)
        logits[:, torch.randperm(case["E"], generator=g, device=dev)[:case["masked"]]] = -math.inf
        s.update(logits=logits.to(dtype))
        return s
    T, k = case["T"], case["k"]
    if op == "combine":
        places = torch.randperm(T * k, generator=g, device=dev).int().view(T, k)
        if case["absent"]:
            places[torch.rand(T, k, generator=g, device=dev) < case["absent"] / 16.0] = -1
        weights = torch.softmax(torch.randn(T, k, generator=g, device=dev), dim=-1)
        s.update(y=torch.randn(T * k, case["H"], generator=g, device=dev).to(dtype), places=places, weights=weights)
        return s
    # the tables that the router gives, for a shuffled batch
    experts = torch.tensor(_choice(case), dtype=torch.int64, device=dev)[torch.randperm(T, generator=g, device=dev)]
    key = torch.where(experts < 0, case["E"], experts).flatten()
    order = torch.sort(key, stable=True).indices
    counts = _counts(case)
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    order[starts[-1]:] = -1
    n_x = T if case["gather"] else T * k
    codes, scales = _weights(g, dev, (case["E"],), _rows(case), case["n_in"])
    s.update(x=_tokens(g, dev, n_x, case["n_in"], dtype), codes=codes, scales=scales, starts_host=starts,
             starts=torch.tensor(starts, dtype=torch.int32, device=dev), order=order.int(),
             bias=torch.randn(case["E"], _rows(case), generator=g, device=dev) * 0.1 if case["bias"] else None)
    return s


# ------------------------------------------------------------------------------------------ the operators' plain forms


def _plain_quantize(x):
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    s = top / torch.full_like(top, 127.0)
    s = torch.where(s < 2.0 ** -126, 0.0, s)
    return torch.where(s > 0, (x / s).round().clamp(-127, 127), 0.0), s


def _plain_act(z, act):
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "relu":
        return z.clamp(min=0)
    if act == "gated":
        gate, up = z.chunk(2, dim=-1)
        return gate / (1.0 + torch.exp(-gate)) * up
    return z


def _plain_product(c, s, codes, scales, bias, act):
    z = torch.matmul(c, codes[:, :c.shape[1]].float().t()) * s * scales
    return _plain_act(z if bias is None else z + bias, act)


def _plain_linear(s):
    case = s["case"]
    c, sx = _plain_quantize(s["x"])
    return _plain_product(c, sx, s["codes"], s["scales"], s["bias"], case["act"]).to(s["x"].dtype)


def _plain_sort(experts, E):
    flat = experts.flatten().long()
    here = (flat >= 0) & (flat < E)
    order = torch.sort(torch.where(here, flat, E), stable=True).indices
    starts = torch.zeros(E + 2, dtype=torch.int64, device=flat.device).index_add_(0, torch.where(here, flat, E) + 1, torch.ones_like(flat)).cumsum(0)[:E + 1]
    row = torch.arange(flat.numel(), device=flat.device)
    places = torch.empty_like(flat)
    places[order] = torch.where(row < starts[E], row, -1)
    return starts.int(), torch.where(row < starts[E], order, -1).int(), places.view(experts.shape).int()


def _plain_route(s):
    case = s["case"]
    logits = s["logits"].float()
    top, experts = torch.sort(logits, dim=-1, descending=True, stable=True)
    top, experts = top[:, :case["k"]], experts[:, :case["k"]]
    there = top > -math.inf
    first = torch.where(there[:, :1], top[:, :1], 0.0)
    e = torch.exp(top - first)
    total = e.sum(-1, keepdim=True) if case["renormalize"] else torch.exp(logits - first).sum(-1, keepdim=True)
    weights = torch.where(there, e / total, 0.0)
    experts = torch.where(there, experts, -1).int()
    return (experts, weights, *_plain_sort(experts, case["E"]))


def _plain_experts(s):
    case, starts = s["case"], s["starts_host"]
    c, sx = _plain_quantize(s["x"])
    y = torch.zeros(s["order"].shape[0], case["n_out"], dtype=s["x"].dtype, device=c.device)
    for e in range(case["E"]):
        a, b = starts[e], starts[e + 1]
        if a == b:
            continue
        rows = s["order"][a:b].long() // case["k"] if case["gather"] else slice(a, b)
        y[a:b] = _plain_product(c[rows], sx[rows], s["codes"][e], s["scales"][e], None if s["bias"] is None else s["bias"][e], case["act"])
    return y


def _plain_combine(s):
    places = s["places"].long()
    w = torch.where(places >= 0, s["weights"], 0.0)
    out = torch.zeros(places.shape[0], s["y"].shape[1], device=places.device)
    for j in range(places.shape[1]):
        out += w[:, j:j + 1] * s["y"][places[:, j].clamp(min=0)].float()
    return out.to(s["y"].dtype)


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"linear": _plain_linear, "route": _plain_route, "experts": _plain_experts, "combine": _plain_combine}[op](s)
    import paper_2311_15806_amd.binding as pipe
    if op == "linear":
        return pipe.pipe_token_forward(s["x"], s["codes"], s["scales"], bias=s["bias"], act=ACTS[case["act"]])
    if op == "route":
        return pipe.pipe_expert_route(s["logits"], case["k"], renormalize=case["renormalize"])
    if op == "experts":
        return pipe.pipe_expert_forward(s["x"], s["codes"], s["scales"], s["starts"], order=s["order"] if case["gather"] else None,
                                        top_k=case["k"], bias=s["bias"], act=ACTS[case["act"]])
    return pipe.pipe_expert_combine(s["y"], s["places"], s["weights"])


# ------------------------------------------------------------------------------------------ what they cannot do without


def work(case):
    """Every input once (of the experts those that have a token), every output once; two operations per multiply-add."""
    op, size = case["op"], 4 if case["dtype"] == "f32" else 2
    if op == "route":
        T, k, E = case["T"], case["k"], case["E"]
        return {"bytes": T * E * size + 16 * T * k + 4 * (E + 1), "flops": 0}
    if op == "combine":
        T, k, H = case["T"], case["k"], case["H"]
        there = T * k * (1.0 - case["absent"] / 16.0)
        return {"bytes": (there + T) * H * size + 8 * T * k, "flops": 2.0 * there * H}
    n_in, rows = case["n_in"], _rows(case)
    row_bytes = rows * (n_in + 4 + (4 if case["bias"] else 0))
    if op == "linear":
        T = case["T"]
        return {"bytes": T * (n_in + case["n_out"]) * size + row_bytes, "flops": 2.0 * T * n_in * rows}
    counts = _counts(case)
    used, n = sum(c > 0 for c in counts), sum(counts)
    x_rows = case["T"] if case["gather"] else n
    return {"bytes": x_rows * n_in * size + case["T"] * case["k"] * (case["n_out"] * size + (4 if case["gather"] else 0)) + used * row_bytes,
            "flops": 2.0 * n * n_in * rows}


# ------------------------------------------------------------------------------------------ the same in 64 bits


def _fp32(t):
    return t.float().double()


def _exact_layer(x, codes, scales, bias, act):
    """One layer over rows x: the codes follow by definition from quotients that are rounded to fp32, everything else is in fp64."""
    n = x.shape[1]
    x = x.double()
    unit = _fp32(x.abs().max(dim=1).values / 127.0)
    unit = torch.where(unit < 2.0 ** -126, torch.zeros_like(unit), unit)
    q = torch.zeros_like(x)
    live = unit > 0
    q[live] = torch.round(_fp32(x[live] / unit[live, None])).clamp(-127, 127)
    w = codes[:, :n].double() * scales.double()[:, None]
    z = (q * unit[:, None]) @ w.t().contiguous()
    if bias is not None:
        z = z + bias.double()
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gated":
        h = z.shape[1] // 2
        return z[:, :h] * torch.sigmoid(z[:, :h]) * z[:, h:]
    return z


def _exact_route(s):
    case = s["case"]
    T, E, k = case["T"], case["E"], case["k"]
    logits = s["logits"].double().cpu()
    p = torch.softmax(logits, dim=-1)
    value = logits.clone()
    experts = torch.full((T, k), -1, dtype=torch.int32)
    weights = torch.zeros(T, k, dtype=torch.float64)
    index = torch.arange(E)[None]
    for j in range(k):
        top = value.max(dim=-1, keepdim=True).values
        e = torch.where(value == top, index, E).min(dim=-1).values             # the lowest of those that are largest
        ok = top[:, 0] > -math.inf
        experts[ok, j] = e[ok].int()
        weights[ok, j] = p[ok, e[ok]]
        value[torch.arange(T), e] = -math.inf
    if case["renormalize"]:
        weights = weights / weights.sum(dim=-1, keepdim=True)
    flat = experts.flatten()
    lists = [torch.nonzero(flat == e)[:, 0] for e in range(E)]
    starts = torch.tensor([0] + [len(v) for v in lists]).cumsum(0).int()
    order = torch.cat(lists + [torch.full((int((flat < 0).sum()),), -1)]).int()
    places = torch.full((T * k,), -1, dtype=torch.int32)
    for row, pair in enumerate(order.tolist()):
        if pair >= 0:
            places[pair] = row
    return experts, weights, starts, order, places.view(T, k)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "linear":
        return _exact_layer(s["x"], s["codes"], s["scales"], s["bias"], case["act"])
    if op == "route":
        return _exact_route(s)
    if op == "combine":
        y = torch.zeros(case["T"], case["H"], dtype=torch.float64, device=s["y"].device)
        for j in range(case["k"]):
            t = torch.nonzero(s["places"][:, j] >= 0)[:, 0]
            y[t] += s["weights"][t, j, None].double() * s["y"][s["places"][t, j].long()].double()
        return y
    out = torch.zeros(case["T"] * case["k"], case["n_out"], dtype=torch.float64, device=s["x"].device)
    first = 0
    for e, n in enumerate(_counts(case)):
        if n:
            at = torch.arange(first, first + n, device=out.device)
            x = s["x"][torch.div(s["order"][at], case["k"], rounding_mode="floor").long()] if case["gather"] else s["x"][at]
            out[at] = _exact_layer(x, s["codes"][e], s["scales"][e], s["bias"][e] if case["bias"] else None, case["act"])
            first += n
    return out
