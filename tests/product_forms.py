"""Which form of the products' kernels sizes take, by the library's own rule (host code, reached by its C++ name), and sizes that take each of them through
more chunks of depth than lie in LDS at once."""
import ctypes
import os
import re

FORWARD, DX, DW = 0, 1, 2
FORMS = ["few rows", "256", "128", "128 deep", "64"]                # in the order of the library's enum
STAGES = {"256": 2, "128": 2, "128 deep": 4, "64": 4, "any 64": 2, "any 128": 2}
_TYPES = {"int": ctypes.c_int, "unsigned": ctypes.c_uint, "long long": ctypes.c_longlong}


def _params_class():
    """The parameters as the header declares them."""
    from paper_1610_06209_amd import build

    text = open(os.path.join(build.CSRC, "mx4.hpp")).read()
    assert re.search(r"enum \{ kFewRows, kTile256, kTile128, kTile128Deep, kTile64 \};", text)
    fields = []
    for line in re.search(r"struct ProductParams \{(.*?)\n\};", text, re.S).group(1).splitlines():
        line = line.split("//")[0].strip().rstrip(";")
        if line:
            kind, names = re.fullmatch(r"((?:const )?(?:void|char|uint8_t|long long)\*|int|unsigned|long long) (.*)", line).groups()
            fields += [(name.strip(), ctypes.c_void_p if kind.endswith("*") else _TYPES[kind]) for name in names.split(",")]
    return type("ProductParams", (ctypes.Structure,), {"_fields_": fields})


def plan(direction, four_bits, rows, experts, k, n):
    """(form, chunks of depth of a whole sum, shares): k and n of the weights [experts][n][k], rows that are packed."""
    from paper_1610_06209_amd import binding

    rule = getattr(binding.lib, "_ZN7spinner12plan_productEibPNS_13ProductParamsE")
    rule.restype, rule.argtypes = None, [ctypes.c_int, ctypes.c_bool, ctypes.c_void_p]
    p = _params_class()(rows=rows, experts=experts)
    if direction == DW:
        p.height, p.width = n, k
    else:
        p.width, p.depth = (n, k) if direction == FORWARD else (k, n)
    rule(direction, four_bits, ctypes.addressof(p))
    form, depth = FORMS[p.tile], rows // experts if direction == DW else p.depth
    if not four_bits and form != "few rows" and (k % 8 or n % 8):
        form = "any 64" if form == "64" else "any 128"
    return form, -(-depth // (256 if four_bits else 64)), p.splits


# rows, experts, k, n: an odd number of chunks, the last one cut, more than twice as many as lie in LDS
SIXTEEN = [
    # forward: 256, 128, 128 deep, 64, and through registers 128, 64; one expert, then three
    (17685, 1, 296, 400), (17804, 1, 264, 152), (16455, 1, 648, 72), (20, 1, 544, 32), (20643, 1, 259, 65), (19, 1, 293, 35),
    (16700, 3, 312, 400), (18901, 3, 280, 144), (375, 3, 560, 4512), (60, 3, 560, 40), (16842, 3, 258, 71), (50, 3, 386, 32),
    # dx
    (18003, 1, 416, 264), (16973, 1, 152, 264), (16617, 1, 80, 648), (19, 1, 32, 520), (12849, 1, 129, 270), (16, 1, 35, 306),
    (10070, 3, 784, 280), (16326, 3, 136, 288), (16764, 3, 80, 568), (16, 3, 32, 520), (455, 3, 3951, 263), (19, 3, 35, 266),
    # dw, whole sums and in shares
    (260, 1, 1576, 5560), (268, 1, 664, 5424), (515, 1, 648, 2984), (554, 1, 32, 32), (276, 1, 3318, 582), (290, 1, 33, 33),
    (15509, 1, 952, 2504), (16644, 1, 80, 4464), (9992, 1, 72, 2680), (10402, 1, 40, 32), (5553, 1, 77, 4822), (5918, 1, 33, 40),
]
FOUR = [
    # 256, 128, 64
    (4659, 1, 1056, 1706), (20071, 1, 1056, 35), (19, 1, 2656, 37),
    (10952, 3, 1152, 664), (113, 3, 1152, 5237), (57, 3, 2784, 32),
    # longer sums
    (4659, 1, 2336, 1706), (1100, 3, 4384, 2051), (20071, 1, 2080, 35),
]


def runs_through(direction, four_bits, rows, experts, k, n):
    """(form, whether in shares) where the sizes send every workgroup through the form's whole round of chunks, more than twice, to an odd and cut last one."""
    form, chunks, shares = plan(direction, four_bits, rows, experts, k, n)
    depth = {FORWARD: k, DX: n, DW: rows}[direction]
    if form == "few rows" or chunks // shares <= 2 * STAGES[form] or chunks % 2 == 0 or depth % (256 if four_bits else 64) == 0:
        return None
    return form, shares > 1
