"""The operators around a routed layer of experts and of its 8-bit form, as cases to be timed and compared.

A router's logits become experts and weights (scores, a bias for balance, groups, the largest few, renormalised), with the gradient;
the chosen experts become places, sorted by expert, and the ends of the experts' rows; rows go to their places and come back as
weighted sums, with the gradients of both.  In 8 bits: rows rotated and rounded to whole numbers with a scale for each row, the
product of two such operands, and both in one call, for one weight matrix or by expert, with the rows' way to their places inside.

``own = False`` computes the plain form, elementary torch operations in fp32 (keys that decide about an order, and quotients that
are rounded to whole numbers, in fp64) with one rounding at the end; ``own = True`` makes the library's calls on the same inputs.
``exact`` follows the definitions in fp64.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LARGEST = 2.3e12            # operations of the largest listed case
LARGEST_ROUTE = 1 << 24     # logits
LARGEST_MOVE = 1 << 28      # numbers at their places
SMALLEST_SCALE = 2.0 ** -126


# ---------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # decoding: one token's router, every feature of it in use (the calls themselves are what counts)
        {"name": "route_token", "kind": "route", "rows": 1, "experts": 256, "k": 8, "in": "f32", "score": "sigmoid", "bias": True, "groups": 8,
         "top_groups": 4, "group_top": 2, "renormalise": True, "scale": 2.5, "masked": False, "train": False},
        # a prompt through the same router, an odd number of tokens, padding at the end
        {"name": "route_prompt", "kind": "route", "rows": 16383, "experts": 256, "k": 8, "in": "bf16", "score": "sigmoid", "bias": True, "groups": 8,
         "top_groups": 4, "group_top": 2, "renormalise": True, "scale": 2.5, "masked": True, "train": False},
        # a training step's router: softmax over a few dozen experts, two of them taken, gradient of the logits
        {"name": "route_train", "kind": "route", "rows": 65536, "experts": 64, "k": 2, "in": "bf16", "score": "softmax", "bias": False, "groups": 1,
         "top_groups": 1, "group_top": 1, "renormalise": False, "scale": 1.0, "masked": False, "train": True},
        # as many experts as a call takes are near, an odd number of them, biased softmax, gradient in fp32
        {"name": "route_wide", "kind": "route", "rows": 8191, "experts": 999, "k": 11, "in": "f32", "score": "softmax", "bias": True, "groups": 1,
         "top_groups": 1, "group_top": 1, "renormalise": True, "scale": 1.0, "masked": False, "train": True},
        # decoding for a few sequences: their rows to the experts and back
        {"name": "exchange_tokens", "kind": "exchange", "rows": 24, "k": 8, "n": 2048, "in": "bf16", "train": False},
        # a training step's way there and back with the gradients of both, sizes beside whole pieces
        {"name": "exchange_odd", "kind": "exchange", "rows": 4099, "k": 6, "n": 1001, "in": "f16", "train": True},
        # the same for a large batch
        {"name": "exchange_train", "kind": "exchange", "rows": 16384, "k": 4, "n": 4096, "in": "bf16", "train": True},
        # a large fp32 weight matrix rounded to 8 bits and read back, as when a model is prepared for serving
        {"name": "quantise_weights", "kind": "quantise", "rows": 16384, "k": 8192, "block": 0, "in": "f32", "out": "bf16"},
        # decoding: one token through an 8-bit layer, the whole vector rotated
        {"name": "linear_token", "kind": "linear", "rows": 1, "k": 4096, "n": 16384, "experts": 0, "top": 0, "block": 4096, "in": "bf16"},
        # decoding for a few dozen sequences at once: odd numbers of them, of inputs and of outputs
        {"name": "linear_batch", "kind": "linear", "rows": 37, "k": 8191, "n": 10007, "experts": 0, "top": 0, "block": 0, "in": "f16"},
        # a prompt through a wide layer
        {"name": "linear_prompt", "kind": "linear", "rows": 16384, "k": 8192, "n": 8192, "experts": 0, "top": 0, "block": 512, "in": "bf16"},
        # a prompt through 8-bit experts of uneven load, two for each row
        {"name": "experts_prompt", "kind": "linear", "rows": 8191, "k": 4096, "n": 4096, "experts": 16, "top": 2, "block": 256, "in": "bf16"},
    ]


def _log_int(rng, lo, hi, unit=1):
    """A multiple of `unit` between lo and hi (in units), spread evenly over its logarithm."""
    return unit * max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("route", "route", "exchange", "exchange", "quantise", "product", "linear", "linear", "experts", "experts"))
    if kind == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        experts = _log_int(rng, 4, 1024 // groups, groups)
        top_groups = rng.randint(1, groups)
        rows = _log_int(rng, 1, min(65536, LARGEST_ROUTE // experts))
        return {"kind": kind, "rows": rows, "experts": experts, "k": rng.randint(1, min(16, experts // groups * top_groups)),
                "in": rng.choice(("f32", "bf16", "f16")), "score": rng.choice(("softmax", "sigmoid")), "bias": rng.random() < 0.5, "groups": groups,
                "top_groups": top_groups, "group_top": rng.choice((1, 2)), "renormalise": rng.random() < 0.6, "scale": rng.choice((1.0, 2.5)),
                "masked": rng.random() < 0.4, "train": rng.random() < 0.5}
    if kind == "exchange":
        k = rng.randint(1, 8)
        unit = rng.choice((1, 8, 8))
        n = _log_int(rng, 128 // unit, 8192 // unit, unit)
        return {"kind": kind, "rows": _log_int(rng, 1, min(65536, LARGEST_MOVE // (n * k))), "k": k, "n": n, "in": rng.choice(("f32", "bf16", "bf16", "f16")),
                "train": rng.random() < 0.6}
    block = rng.choice((0, 1)) * (1 << rng.randint(5, 12))
    width = _log_int(rng, max(1, 256 // block), 8192 // block, block) if block else _log_int(rng, 256, 8192)
    if kind == "quantise":
        return {"kind": kind, "rows": _log_int(rng, 1, (1 << 27) // width), "k": width, "block": block, "in": rng.choice(("f32", "bf16", "f16")),
                "out": "bf16" if block else rng.choice(("f32", "bf16"))}
    experts = _log_int(rng, 2, 64) if kind == "experts" else 0
    top = rng.randint(1, min(4, experts)) if kind == "experts" and rng.random() < 0.5 else 0
    n = _log_int(rng, 256, 4096 if experts else 16384)
    rows = _log_int(rng, 1, min(16384 // max(1, top), int(LARGEST / (4.0 * width * n * max(1, top)))))
    case = {"kind": "product" if kind == "product" else "linear", "rows": rows, "k": width, "n": n, "experts": experts}
    if kind == "product":
        return {**case, "out": rng.choice(("f32", "bf16", "f16"))}
    # (fp32 vectors go in as they are: what a rotation in fp32 leaves next to a border may become the whole number beside it)
    return {**case, "top": top, "block": block, "in": rng.choice(("bf16", "bf16", "f16") if block else ("bf16", "f16", "f32"))}


# ---------------------------------------------------------------------------------------------------------- the inputs
def _activations(gen, rows, k):
    """Coordinates of unit size, one in twenty ten times larger in every vector: what a layer's inputs look like."""
    x = torch.randn((rows, k), generator=gen, device=DEV)
    return x.mul_(torch.where(torch.rand(k, generator=gen, device=DEV) < 0.05, 10.0, 1.0))


def _choices(gen, rows, experts, k):
    """k different experts for each row, some of them taken much more often; one row in about sixty has none."""
    liked = torch.randn(experts, generator=gen, device=DEV)
    noise = torch.rand((rows, experts), generator=gen, device=DEV).clamp_(1e-6, 1 - 1e-6)
    chosen = (liked - torch.log(-torch.log(noise))).argsort(1, descending=True)[:, :k].int()
    chosen[rows - rows // 61:] = -1
    return chosen.contiguous()


def _ragged(gen, rows, experts):
    """Cumulative ends of uneven groups, some of them empty; one row in about sixty belongs to none."""
    share = torch.rand(experts, generator=gen, device=DEV).square().add_(1e-3)
    share = torch.where(torch.rand(experts, generator=gen, device=DEV) < 0.1, torch.zeros_like(share), share)
    share[0] += 1e-3
    used = rows - rows // 61
    ends = torch.floor(torch.cumsum(share, 0) / share.sum() * used + 0.5).long().clamp_(max=used)
    ends[-1] = used
    return ends


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, rows, k = case["kind"], case["rows"], case["k"]
    s = dict(case)
    if kind == "route":
        experts = case["experts"]
        # every token likes some experts, and some experts are liked by all
        liked = 0.7 * torch.randn(experts, generator=gen, device=DEV)
        s["logits"] = (1.5 * torch.randn((rows, experts), generator=gen, device=DEV) + liked).to(TYPES[case["in"]])
        s["b"] = (-0.1 if case["score"] == "sigmoid" else -0.5 / experts) * liked + 1e-3 * torch.randn(experts, generator=gen, device=DEV) if case["bias"] else None
        s["mask"] = torch.arange(rows, device=DEV) < rows - rows // 17 if case["masked"] else None
        s["dweights"] = torch.randn((rows, k), generator=gen, device=DEV) if case["train"] else None
        return s
    if kind == "exchange":
        dtype, n = TYPES[case["in"]], case["n"]
        s["places"] = _order(_choices(gen, rows, 16, k), 16)[0]
        s["weights"] = torch.softmax(torch.randn((rows, k), generator=gen, device=DEV), 1)
        s["x"] = torch.randn((rows, n), generator=gen, device=DEV).to(dtype)
        s["y"] = torch.randn((rows * k, n), generator=gen, device=DEV).to(dtype)
        if case["train"]:
            s["dx"] = torch.randn((rows * k, n), generator=gen, device=DEV).to(dtype)       # gradient of the rows at their places
            s["dout"] = torch.randn((rows, n), generator=gen, device=DEV).to(dtype)
        return s
    if kind == "quantise":
        s["x"] = _activations(gen, rows, k).to(TYPES[case["in"]])
        s["diag"] = torch.randint(0, 2, (k,), generator=gen, device=DEV).float() * 2 - 1 if case["block"] else None
        s["hadamard"] = _hadamard(case["block"], torch.float32) if case["block"] else None
        return s
    experts, n = case["experts"], case["n"]
    top = case.get("top", 0)
    if top:
        s["places"], s["ends"] = _order(_choices(gen, rows, experts, top), experts)
    elif experts:
        s["ends"] = _ragged(gen, rows, experts)
    if experts:
        # the most rows of a group: how far the plain form pads the groups
        s["most"] = max(1, int(torch.diff(s["ends"], prepend=s["ends"].new_zeros(1)).max()))
    s["w_codes"], s["w_scales"] = _pack(*_quantise(torch.randn((max(1, experts) * n, k), generator=gen, device=DEV)))
    if experts:
        s["w_codes"], s["w_scales"] = s["w_codes"].view(experts, n, -1), s["w_scales"].view(experts, n)
    if kind == "product":
        s["a_codes"], s["a_scales"] = _pack(*_quantise(_activations(gen, rows, k)))
        return s
    s["x"] = _activations(gen, rows, k).to(TYPES[case["in"]])
    s["diag"] = torch.randint(0, 2, (k,), generator=gen, device=DEV).float() * 2 - 1 if case["block"] else None
    s["hadamard"] = _hadamard(case["block"], torch.float32) if case["block"] else None
    return s


def _hadamard(b, dtype):
    """The L2-normalised Hadamard matrix in Sylvester order: entry (-1)^popcount(i & j) / sqrt(b)."""
    i = torch.arange(b, device=DEV)
    bits = i[:, None] & i[None, :]
    for shift in (8, 4, 2, 1):
        bits = bits ^ (bits >> shift)
    return (1 - 2 * (bits & 1)).to(dtype) / math.sqrt(b)


# ---------------------------------------------------------------------------------------------------------- the plain form
def _largest_first(keys, count):
    """Indices of the largest keys in falling order, equal ones in the order of their indices."""
    return torch.sort(keys, dim=1, descending=True, stable=True).indices[:, :count]


def _scores(logits, score):
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-logits))
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _route(s):
    """Weights and experts of every row; -1 and weight 0 in rows that the mask leaves out."""
    logits, far = s["logits"].float(), s["logits"].double()
    rows, experts, groups = s["rows"], s["experts"], s["groups"]
    keys = _scores(far, s["score"]) if s["b"] is not None or groups > 1 else far
    if s["b"] is not None:
        keys = keys + s["b"].double()
    if groups > 1:
        inside = keys.view(rows, groups, -1)
        best = torch.sort(inside, dim=2, descending=True).values[:, :, :s["group_top"]].sum(2)
        stay = torch.zeros((rows, groups), dtype=torch.bool, device=DEV).scatter_(1, _largest_first(best, s["top_groups"]), True)
        # without a bias the logits order experts as their scores do
        keys = (inside if s["b"] is not None else far.view(rows, groups, -1)).masked_fill(~stay[:, :, None], -math.inf).view(rows, experts)
    chosen = _largest_first(keys, s["k"])
    weights = _scores(logits, s["score"]).gather(1, chosen)
    if s["renormalise"]:
        weights = weights / weights.sum(1, keepdim=True)
    weights, chosen = weights * s["scale"], chosen.int()
    if s["mask"] is not None:
        weights, chosen = weights * s["mask"][:, None], torch.where(s["mask"][:, None], chosen, -1)
    return weights, chosen


def _route_grad(s, chosen):
    logits = s["logits"].float()
    there = chosen >= 0
    at = chosen.long().clamp(min=0)
    p, d = _scores(logits, s["score"]), s["dweights"] * s["scale"] * there
    if s["renormalise"]:
        q = p.gather(1, at)
        q = q / q.sum(1, keepdim=True)
        d = q * (d - (d * q).sum(1, keepdim=True)) * there
        if s["score"] == "sigmoid":
            d = d * (1 - p.gather(1, at))
        return torch.zeros_like(p).scatter_(1, at, d).to(s["logits"].dtype)
    d = torch.zeros_like(p).scatter_(1, at, d)
    if s["score"] == "sigmoid":
        d = d * p * (1 - p)
    else:
        d = p * (d - (d * p).sum(1, keepdim=True))
    return d.to(s["logits"].dtype)


def _order(chosen, experts):
    """The place of every choice in the order of the experts, and where each expert's places end."""
    flat = chosen.flatten().long()
    flat = torch.where((flat >= 0) & (flat < experts), flat, experts)
    order = torch.sort(flat, stable=True).indices
    places = torch.empty_like(flat)
    places[order] = torch.arange(flat.numel(), device=DEV)
    return places.int().view(chosen.shape), torch.cumsum(torch.bincount(flat, minlength=experts + 1), 0)[:experts]


def _quantise(v):
    """Whole numbers (in fp32) and scales of rows."""
    scale = (v.abs().amax(1) / 127).clamp_(min=SMALLEST_SCALE)
    return torch.round(v.double() / scale.double()[:, None]).float(), scale


def _pack(codes, scales):
    """Rows of whole pieces of 16 bytes, zeros behind the numbers."""
    return torch.nn.functional.pad(codes, (0, -codes.shape[1] % 16)).to(torch.int8), scales


def _rotated(s):
    x = s["x"].float()
    return ((x * s["diag"]).view(-1, s["block"]) @ s["hadamard"]).view(x.shape) if s["block"] else x


def _spread(rows, ends, most):
    """Places of the groups' rows in a table of `most` a group, whether there is one, and the way back."""
    starts = torch.cat((ends.new_zeros(1), ends[:-1]))
    at = starts[:, None] + torch.arange(most, device=DEV)
    row = torch.arange(rows, device=DEV)
    group = torch.searchsorted(ends, row, right=True)
    inside = group < ends.numel()
    group = group.clamp(max=ends.numel() - 1)
    return at.clamp(max=rows - 1), (at < ends[:, None])[..., None], group, (row - starts[group]).clamp(max=most - 1), inside[:, None]


def _products(x, w, ends, most):
    """x w^T of each group's rows with its own w, all in fp32; rows of no group are 0."""
    if ends is None:
        return x @ w.T
    at, there, group, place, inside = _spread(x.shape[0], ends, most)
    return torch.matmul(x[at] * there, w.transpose(1, 2))[group, place] * inside


def _plain(s):
    kind = s["kind"]
    if kind == "route":
        weights, chosen = _route(s)
        places, ends = _order(chosen, s["experts"])
        r = {"weights": weights, "experts": chosen, "places": places, "ends": ends}
        return {**r, "dlogits": _route_grad(s, chosen)} if s["train"] else r
    if kind == "exchange":
        at, w, dtype = s["places"].long(), s["weights"], s["x"].dtype
        out = torch.empty_like(s["y"])
        out[at] = s["x"][:, None]
        r = {"x": out, "y": (s["y"][at].float() * w[:, :, None]).sum(1).to(dtype)}
        if s["train"]:
            dy, dout = torch.empty_like(s["y"]), s["dout"].float()[:, None]
            dy[at] = (dout * w[:, :, None]).to(dtype)
            r.update(dx=s["dx"][at].float().sum(1).to(dtype), dy=dy, dweights=(s["y"][at].float() * dout).sum(2))
        return r
    if kind == "quantise":
        codes, scale = _quantise(_rotated(s))
        return (codes * scale[:, None]).to(TYPES[s["out"]])
    w = s["w_codes"].float() * s["w_scales"][..., None]
    if kind == "product":
        return _products(s["a_codes"].float() * s["a_scales"][:, None], w, s.get("ends"), s.get("most")).to(TYPES[s["out"]])
    codes, scale = _pack(*_quantise(_rotated(s)))
    x = codes.float() * scale[:, None]
    if s["top"]:
        spread = x.new_empty((s["places"].numel(), x.shape[1]))
        spread[s["places"].long()] = x[:, None]
        x = spread
    return _products(x, w, s.get("ends"), s.get("most")).to(s["x"].dtype)


# ---------------------------------------------------------------------------------------------------------- the library's calls
def run(s):
    if not own:
        return _plain(s)
    from paper_1610_06209_amd import binding as sp
    kind = s["kind"]
    if kind == "route":
        weights, chosen = sp.spinner_route(s["logits"], s["k"], s["b"], s["mask"], s["score"], s["groups"], s["top_groups"], s["group_top"], s["renormalise"], s["scale"])
        places, ends = sp.spinner_route_order(chosen, s["experts"])
        r = {"weights": weights, "experts": chosen, "places": places, "ends": ends}
        if s["train"]:
            r["dlogits"] = sp.spinner_route_grad(s["dweights"], s["logits"], chosen, s["score"], s["renormalise"], s["scale"])
        return r
    if kind == "exchange":
        r = {"x": sp.spinner_dispatch(s["x"], s["places"]), "y": sp.spinner_combine(s["y"], s["places"], s["weights"])}
        if s["train"]:
            r["dx"] = sp.spinner_combine(s["dx"], s["places"])
            r["dy"], r["dweights"] = sp.spinner_combine_grad(s["dout"], s["y"], s["places"], s["weights"])
        return r
    if kind == "quantise":
        codes, scales = sp.spinner_int_quantize(s["x"], s["diag"], s["block"])
        return sp.spinner_int_dequantize(codes, scales, TYPES[s["out"]], s["k"])
    if kind == "product":
        return sp.spinner_int_matmul(s["a_codes"], s["a_scales"], s["w_codes"], s["w_scales"], dtype=TYPES[s["out"]])
    return sp.spinner_int_linear(s["x"], s["w_codes"], s["w_scales"], s["diag"], s["block"], s.get("ends"), s.get("places"))


# ---------------------------------------------------------------------------------------------------------- what it takes
def _size(name):
    return 4 if name == "f32" else 2


def work(case):
    kind, rows, k = case["kind"], case["rows"], case["k"]
    if kind == "route":                         # logits read (and their gradient written), weights, experts and places written
        logits = rows * case["experts"] * _size(case["in"])
        return {"bytes": logits * (2 if case["train"] else 1) + rows * k * (16 if case["train"] else 12) + 8 * case["experts"], "flops": 0}
    if kind == "exchange":                      # x to its places, y and its weights to their sums; the same of the gradients, y once more
        row = (1 + k) * rows * case["n"] * _size(case["in"])
        return {"bytes": row * 2 + 8 * rows * k + (row * 2 + rows * k * 4 if case["train"] else 0), "flops": 0}
    if kind == "quantise":                      # written in 8 bits and read back
        return {"bytes": rows * k * (_size(case["in"]) + 2 + _size(case["out"])) + 8 * rows, "flops": 0}
    n, placed = case["n"], rows * max(1, case.get("top", 0))
    held = min(max(1, case["experts"]), placed) * n * (k + 4)      # no more experts than rows are read
    if kind == "product":
        return {"bytes": rows * (k + 4) + held + placed * n * _size(case["out"]), "flops": 2.0 * placed * n * k}
    return {"bytes": rows * k * _size(case["in"]) + held + placed * n * _size(case["in"]), "flops": 2.0 * placed * n * k}


# ---------------------------------------------------------------------------------------------------------- the definition in 64 bits
def _take_largest(keys, count):
    """The largest key again and again, the first of equal ones."""
    keys, n = keys.clone(), keys.shape[1]
    index = torch.arange(n, device=DEV).expand_as(keys)
    taken = []
    for _ in range(count):
        at = torch.where(keys == keys.max(1, keepdim=True).values, index, n).min(1, keepdim=True).values
        taken.append(at)
        keys.scatter_(1, at, -math.inf)
    return torch.cat(taken, 1)


def _exact_route(s):
    x, rows, experts, groups = s["logits"].double(), s["rows"], s["experts"], s["groups"]
    p = torch.sigmoid(x) if s["score"] == "sigmoid" else torch.softmax(x, 1)
    keys = (p + s["b"] if s["b"] is not None else p).clone()
    among = keys if s["b"] is not None else x
    if groups > 1:
        best = keys.view(rows, groups, -1).topk(min(s["group_top"], experts // groups), 2).values.sum(2)
        group = torch.arange(experts, device=DEV) // (experts // groups)
        stay = (_take_largest(best, s["top_groups"])[:, :, None] == group).any(1)
        among = torch.where(stay, among, -math.inf)
    chosen = _take_largest(among, s["k"])
    alive = torch.ones((rows, 1), dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"][:, None]
    value = torch.zeros((rows, s["k"]), dtype=torch.float64, device=DEV)
    for j in range(s["k"]):
        value[:, j] = p[torch.arange(rows, device=DEV), chosen[:, j]]
    total = value.sum(1, keepdim=True) if s["renormalise"] else 1.0
    weights = torch.where(alive, s["scale"] * value / total, 0.0)
    chosen = torch.where(alive, chosen, -1)
    # places: how many choices of smaller experts there are, and of the same expert in front
    flat = torch.where(chosen < 0, experts, chosen).flatten()
    counts = torch.zeros(experts + 1, dtype=torch.long, device=DEV).index_add_(0, flat, torch.ones_like(flat))
    ends = torch.cumsum(counts, 0)
    places = torch.empty_like(flat)
    for e in range(experts + 1):
        mine = (flat == e).nonzero()[:, 0]
        places[mine] = ends[e] - counts[e] + torch.arange(mine.numel(), device=DEV)
    r = {"weights": weights, "experts": chosen.int(), "places": places.int().view(rows, -1), "ends": ends[:experts]}
    if s["train"]:
        d = s["dweights"].double() * alive * s["scale"]
        dp = torch.zeros_like(p)
        for j in range(s["k"]):
            back = d[:, j] if not s["renormalise"] else (d[:, j] * total[:, 0] - (d * value).sum(1)) / total[:, 0] ** 2
            dp[torch.arange(rows, device=DEV), chosen[:, j].clamp(min=0)] += back
        r["dlogits"] = dp * p * (1 - p) if s["score"] == "sigmoid" else p * dp - p * (p * dp).sum(1, keepdim=True)
    return r


def _whole_numbers(v):
    """fp64 rows to what they become as whole numbers with a scale in fp32 each."""
    scale = torch.maximum((v.abs().max(1).values / 127).float(), torch.tensor(SMALLEST_SCALE, device=DEV)).double()[:, None]
    return torch.round(v / scale) * scale


def exact(case, seed):
    s = prepare(case, seed)
    kind, rows = case["kind"], case["rows"]
    if kind == "route":
        return _exact_route(s)
    if kind == "exchange":
        x, y, w, at = s["x"].double(), s["y"].double(), s["weights"].double(), s["places"].long()
        out, total = torch.empty_like(y), torch.zeros_like(x)
        for j in range(case["k"]):
            out[at[:, j]] = x
            total += w[:, j:j + 1] * y[at[:, j]]
        r = {"x": out, "y": total}
        if case["train"]:
            dout, dx, dy, dw = s["dout"].double(), torch.zeros_like(x), torch.empty_like(y), torch.empty_like(w)
            for j in range(case["k"]):
                dx += s["dx"][at[:, j]]
                dy[at[:, j]] = w[:, j:j + 1] * dout
                dw[:, j] = (dout * y[at[:, j]]).sum(1)
            r.update(dx=dx, dy=dy, dweights=dw)
        return r
    if kind == "product":
        return (s["a_codes"].double() * s["a_scales"].double()[:, None]) @ (s["w_codes"].double() * s["w_scales"].double()[:, None]).T
    x = s["x"].double()
    if case["block"]:
        x = ((x * s["diag"]).reshape(-1, case["block"]) @ _hadamard(case["block"], torch.float64)).reshape(x.shape)
    x = _whole_numbers(x)
    if kind == "quantise":
        return x
    w = s["w_codes"][..., :case["k"]].double() * s["w_scales"].double()[..., None]
    if not case["experts"]:
        return x @ w.T
    if case["top"]:
        slots = torch.empty((s["places"].numel(), x.shape[1]), dtype=torch.float64, device=DEV)
        for j in range(s["places"].shape[1]):
            slots[s["places"][:, j].long()] = x
        x = slots
    y = torch.zeros((x.shape[0], case["n"]), dtype=torch.float64, device=DEV)
    begin = 0
    for e, end in enumerate(s["ends"].tolist()):
        if end > begin:
            y[begin:end] = x[begin:end] @ w[e].T
        begin = end
    return y
