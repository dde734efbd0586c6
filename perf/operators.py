"""The operators that carry the framework's rotated vectors into a language model's linear layers, as cases to be timed and compared.

Microscaled 4-bit floating point: blocks of 32 numbers in e2m1 with a shared power of two, after the rotation H D that spreads
a vector's outliers; the quantisation, the product of quantised operands, and both in one call, for one weight matrix or for
groups of rows that each go to the weights of their own expert.  In 16 bits: the experts' products over ragged groups of rows
with the gradients of both operands.

``own = False`` computes the plain form, elementary torch operations in fp32 with one rounding at the end; ``own = True`` makes
the library's calls on the same inputs.  ``exact`` follows the definitions in fp64.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LARGEST = 3.4e12            # operations of the largest listed case


# ---------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # activations of one token on their way into 4 bits and back (the call itself is what counts)
        {"name": "quantise_token", "kind": "quantise", "rows": 1, "k": 4096, "in": "bf16", "out": "f32"},
        # a large fp32 weight matrix rounded to 4 bits and read back, as when a model is prepared for serving
        {"name": "quantise_weights", "kind": "quantise", "rows": 16384, "k": 16384, "in": "f32", "out": "bf16"},
        # quantised vectors against quantised stored ones: sizes that are no multiple of any tile, fp32 results
        {"name": "product_odd", "kind": "product", "rows": 1000, "k": 4128, "n": 10007, "experts": 0, "out": "f32"},
        # decoding: one token through a 4-bit layer, the whole vector rotated
        {"name": "linear_token", "kind": "linear", "rows": 1, "k": 4096, "n": 16384, "experts": 0, "block": 4096, "in": "bf16"},
        # decoding for a few dozen sequences at once, an odd number of them and of outputs
        {"name": "linear_batch", "kind": "linear", "rows": 37, "k": 8192, "n": 10007, "experts": 0, "block": 1024, "in": "f16"},
        # a prompt through a wide layer
        {"name": "linear_prompt", "kind": "linear", "rows": 16384, "k": 8192, "n": 8192, "experts": 0, "block": 512, "in": "bf16"},
        # decoding through 4-bit experts: a few rows for each, none for some
        {"name": "experts_tokens", "kind": "linear", "rows": 64, "k": 2048, "n": 4096, "experts": 32, "block": 2048, "in": "bf16"},
        # a prompt through 4-bit experts of uneven load
        {"name": "experts_prompt", "kind": "linear", "rows": 16383, "k": 4096, "n": 4096, "experts": 16, "block": 256, "in": "bf16"},
        # decoding through 16-bit experts
        {"name": "grouped_tokens", "kind": "grouped", "rows": 24, "k": 2048, "n": 8192, "experts": 8, "in": "bf16"},
        # a training step of a small layer of experts: products and both gradients, sizes beside the tiles
        {"name": "train_small", "kind": "train", "rows": 4099, "k": 1000, "n": 1032, "experts": 16, "in": "f16", "dw": "f16"},
        # a training step of a large one, weight gradients in fp32 for the optimiser
        {"name": "train_large", "kind": "train", "rows": 32768, "k": 4096, "n": 4096, "experts": 8, "in": "bf16", "dw": "f32"},
    ]


def _log_int(rng, lo, hi, unit=1):
    """A multiple of `unit` between lo and hi (in units), spread evenly over its logarithm; 3 * 2^10 is left out."""
    v = unit * max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return v - unit * (v == 3 << 10)


def draw(rng):
    kind = rng.choice(("quantise", "product", "linear", "linear", "experts", "experts", "grouped", "train", "train"))
    if kind == "quantise":
        k = _log_int(rng, 4, 512, 32)
        return {"kind": kind, "rows": _log_int(rng, 1, max(1, (1 << 28) // k)), "k": k, "in": rng.choice(("f32", "bf16", "f16")),
                "out": rng.choice(("f32", "bf16"))}
    if kind in ("product", "linear", "experts"):
        experts = _log_int(rng, 2, 64) if kind == "experts" else 0
        block = 1 << rng.randint(5, 12)
        k = _log_int(rng, max(1, 256 // block), 8192 // block, block) if kind != "product" else _log_int(rng, 4, 256, 32)
        n = _log_int(rng, 256, 16384 if not experts else 4096)
        rows = _log_int(rng, 1, min(16384, int(LARGEST / (4.0 * k * n))))
        case = {"kind": "product" if kind == "product" else "linear", "rows": rows, "k": k, "n": n, "experts": experts}
        if kind == "product":
            return {**case, "out": rng.choice(("f32", "bf16", "f16"))}
        return {**case, "block": rng.choice((0, block, block, block)), "in": rng.choice(("bf16", "bf16", "f16"))}
    even = rng.choice((1, 8, 8, 8))             # rows of whole 16-byte pieces, mostly
    k, n = _log_int(rng, 128 // even, 4096 // even, even), _log_int(rng, 128 // even, 4096 // even, even)
    rows = _log_int(rng, 1 if kind == "grouped" else 64, min(32768, int(LARGEST / (6.0 * k * n))))
    case = {"kind": kind, "rows": rows, "k": k, "n": n, "experts": _log_int(rng, 2, 64), "in": rng.choice(("bf16", "bf16", "f16"))}
    return {**case, "dw": rng.choice(("f32", case["in"]))} if kind == "train" else case


# ---------------------------------------------------------------------------------------------------------- the inputs
def _activations(gen, rows, k):
    """Coordinates of unit size, one in twenty ten times larger in every vector: what a layer's inputs look like."""
    x = torch.randn((rows, k), generator=gen, device=DEV)
    return x.mul_(torch.where(torch.rand(k, generator=gen, device=DEV) < 0.05, 10.0, 1.0))


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
    if kind == "quantise":
        s["x"] = _activations(gen, rows, k).to(TYPES[case["in"]])
        return s
    experts, n = case["experts"], case["n"]
    if experts:
        s["ends"] = _ragged(gen, rows, experts)
        # the most rows of a group: how far the plain form pads the groups
        s["most"] = max(1, int(torch.diff(s["ends"], prepend=s["ends"].new_zeros(1)).max()))
    w = torch.randn((max(1, experts) * n, k), generator=gen, device=DEV)
    if kind in ("product", "linear"):
        s["w_codes"], s["w_scales"] = _pack(*_quantise(w))
        if experts:
            s["w_codes"], s["w_scales"] = s["w_codes"].view(experts, n, k // 2), s["w_scales"].view(experts, n, k // 32)
    if kind == "product":
        s["a_codes"], s["a_scales"] = _pack(*_quantise(_activations(gen, rows, k)))
    elif kind == "linear":
        s["x"] = _activations(gen, rows, k).to(TYPES[case["in"]])
        s["diag"] = torch.randint(0, 2, (k,), generator=gen, device=DEV).float() * 2 - 1 if case["block"] else None
        s["hadamard"] = _hadamard(case["block"], torch.float32) if case["block"] else None
    else:
        dtype = TYPES[case["in"]]
        s["w"] = (w / math.sqrt(k)).view(experts, n, k).to(dtype)
        s["x"] = torch.randn((rows, k), generator=gen, device=DEV).to(dtype)
        if kind == "train":
            s["dy"] = torch.randn((rows, n), generator=gen, device=DEV).to(dtype)
    return s


def _hadamard(b, dtype):
    """The L2-normalised Hadamard matrix in Sylvester order: entry (-1)^popcount(i & j) / sqrt(b)."""
    i = torch.arange(b, device=DEV)
    bits = i[:, None] & i[None, :]
    for shift in (8, 4, 2, 1):
        bits = bits ^ (bits >> shift)
    return (1 - 2 * (bits & 1)).to(dtype) / math.sqrt(b)


# ---------------------------------------------------------------------------------------------------------- the plain form
def _quantise(v):
    """Numbers of 4 bits (as whole codes 0 .. 15) and exponents of their blocks of 32, both in int32."""
    v = v.float().view(*v.shape[:-1], -1, 32)
    a = v.abs()
    e = (torch.frexp(a.amax(-1)).exponent - 3).clamp(-127, 127)
    a = a * torch.exp2(-e.float())[..., None]
    # halfway points go to the even one of their two neighbours
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return code + 8 * torch.signbit(v), torch.where(a.amax(-1) > 0, e, -127)


def _values(code, e):
    """What the codes stand for, in fp32."""
    m = code & 7
    a = torch.where(m < 2, m * 0.5, (1 + 0.5 * (m & 1)) * torch.exp2(((m >> 1) - 1).float()))
    a = torch.where(code > 7, -a, a) * torch.exp2(e.float())[..., None]
    return a.flatten(-2)


def _pack(code, e):
    """Two codes a byte, the first in the low half, and a byte of exponent + 127 a block."""
    code = code.flatten(-2)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8), (e + 127).to(torch.uint8)


def _unpack(codes, scales):
    code = torch.stack((codes & 15, codes >> 4), -1).int()
    return _values(code.view(*scales.shape, 32), scales.int() - 127)


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
    if kind == "quantise":
        return _values(*_quantise(s["x"])).to(TYPES[s["out"]])
    if kind in ("product", "linear"):
        w = _unpack(s["w_codes"], s["w_scales"])
        if kind == "product":
            return _products(_unpack(s["a_codes"], s["a_scales"]), w, None, 0).to(TYPES[s["out"]])
        x = s["x"].float()
        if s["block"]:
            x = ((x * s["diag"]).view(-1, s["block"]) @ s["hadamard"]).view(x.shape)
        return _products(_values(*_quantise(x)), w, s.get("ends"), s.get("most")).to(s["x"].dtype)
    x, w = s["x"].float(), s["w"].float()
    if kind == "grouped":
        return _products(x, w, s["ends"], s["most"]).to(s["x"].dtype)
    at, there, group, place, inside = _spread(x.shape[0], s["ends"], s["most"])
    x, dy = x[at] * there, s["dy"].float()[at] * there
    y = torch.matmul(x, w.transpose(1, 2))[group, place] * inside
    dx = torch.matmul(dy, w)[group, place] * inside
    dw = torch.matmul(dy.transpose(1, 2), x)
    return {"y": y.to(s["x"].dtype), "dx": dx.to(s["x"].dtype), "dw": dw.to(TYPES[s["dw"]])}


# ---------------------------------------------------------------------------------------------------------- the library's calls
def run(s):
    if not own:
        return _plain(s)
    from paper_1610_06209_amd import binding as sp
    kind = s["kind"]
    if kind == "quantise":
        codes, scales = sp.spinner_mx_quantize(s["x"])
        return sp.spinner_mx_dequantize(codes, scales, TYPES[s["out"]])
    if kind == "product":
        return sp.spinner_mx_matmul(s["a_codes"], s["a_scales"], s["w_codes"], s["w_scales"], dtype=TYPES[s["out"]])
    if kind == "linear":
        return sp.spinner_mx_linear(s["x"], s["w_codes"], s["w_scales"], s["diag"], s["block"], s.get("ends"))
    y = sp.spinner_grouped_matmul(s["x"], s["w"], s["ends"])
    if kind == "grouped":
        return y
    dx = sp.spinner_grouped_matmul_dx(s["dy"], s["w"], s["ends"])
    return {"y": y, "dx": dx, "dw": sp.spinner_grouped_matmul_dw(s["dy"], s["x"], s["ends"], TYPES[s["dw"]])}


# ---------------------------------------------------------------------------------------------------------- what it takes
def _size(name):
    return 4 if name == "f32" else 2


def work(case):
    kind, rows, k = case["kind"], case["rows"], case["k"]
    mx = 17.0 / 32.0                            # bytes a number in 4 bits, with its share of the block's exponent
    if kind == "quantise":                      # written in 4 bits and read back
        return {"bytes": rows * k * (_size(case["in"]) + 2 * mx + _size(case["out"])), "flops": 0}
    n, all_w = case["n"], max(1, case["experts"]) * case["n"] * k
    held = min(max(1, case["experts"]), rows) * n * k          # no more experts than rows are read
    flops = 2.0 * rows * n * k
    if kind == "product":
        return {"bytes": (rows * k + held) * mx + rows * n * _size(case["out"]), "flops": flops}
    if kind == "linear":
        return {"bytes": 2 * rows * k + held * mx + 2 * rows * n, "flops": flops}
    if kind == "grouped":
        return {"bytes": 2 * (rows * k + held + rows * n), "flops": flops}
    # x, dy and w read, y, dx and dw written
    return {"bytes": 2 * (2 * rows * k + 2 * rows * n + held) + all_w * _size(case["dw"]), "flops": 3 * flops}


# ---------------------------------------------------------------------------------------------------------- the definition in 64 bits
def _e2m1(v):
    """fp64 numbers to what they become in 4 bits with a power of two for each 32."""
    v = v.double().unflatten(-1, (-1, 32))
    top = v.abs().amax(-1, keepdim=True)
    scale = torch.where(top > 0, torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2, -127.0).clamp(-127, 127)
    scale = torch.pow(torch.full_like(scale, 2.0), scale)
    u = (v / scale).abs()
    step = torch.where(u < 2, 0.5, torch.where(u < 4, 1.0, 2.0))        # between neighbours
    u = (torch.round(u / step) * step).clamp(max=6.0)                   # round() takes halves to the even multiple
    return (torch.copysign(u, v) * scale).flatten(-2)


def _from_bytes(codes, scales):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)
    table = torch.cat((table, -table))
    v = torch.empty((*codes.shape[:-1], 2 * codes.shape[-1]), dtype=torch.float64, device=DEV)
    v[..., 0::2], v[..., 1::2] = table[(codes % 16).long()], table[(codes // 16).long()]
    return v * torch.ldexp(torch.ones((), dtype=torch.float64, device=DEV), scales.int() - 127).repeat_interleave(32, -1)


def exact(case, seed):
    s = prepare(case, seed)
    kind, rows = case["kind"], case["rows"]
    if kind == "quantise":
        return _e2m1(s["x"])
    if kind == "product":
        return _from_bytes(s["a_codes"], s["a_scales"]) @ _from_bytes(s["w_codes"], s["w_scales"]).T
    if kind == "linear":
        x = s["x"].double()
        if case["block"]:
            x = ((x * s["diag"]).reshape(-1, case["block"]) @ _hadamard(case["block"], torch.float64)).reshape(x.shape)
        x = _e2m1(x)
        if not case["experts"]:
            return x @ _from_bytes(s["w_codes"], s["w_scales"]).T
    else:
        x = s["x"].double()
    y = torch.zeros((rows, case["n"]), dtype=torch.float64, device=DEV)
    dx = torch.zeros_like(x)
    dw = torch.zeros((case["experts"], case["n"], case["k"]), dtype=torch.float64, device=DEV) if kind == "train" else None
    begin = 0
    for e, end in enumerate(s["ends"].tolist()):
        if end > begin:
            w = s["w"][e].double() if kind != "linear" else _from_bytes(s["w_codes"][e], s["w_scales"][e])
            y[begin:end] = x[begin:end] @ w.T
            if kind == "train":
                dy = s["dy"][begin:end].double()
                dx[begin:end] = dy @ w
                dw[e] = dy.T @ x[begin:end]
        begin = end
    return {"y": y, "dx": dx, "dw": dw} if kind == "train" else y
