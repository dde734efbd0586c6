"""Routing and 8-bit layers on the host: what is refused before anything is launched, by the C ABI and by the binding, and whose memory a call takes."""
import ctypes

import pytest

from test_products_host import FAR, b  # noqa: F401
from test_streams_host import CURRENT, MINE, T, made  # noqa: F401

f, i32, i64, i8, u8, h = dict(dtype="float32"), dict(dtype="int32"), dict(dtype="int64"), dict(dtype="int8"), dict(dtype="uint8"), dict(dtype="bfloat16")
BIG = 0x7fff0000


def but(t, **changed):
    t.__dict__.update(changed)
    return t


def _refused(b, name, good, cases):
    """``good`` in the order of the C ABI; cases: position -> [(value, status)]."""
    call = getattr(b.lib._lib if hasattr(b.lib, "_lib") else b.lib, name)
    for at, values in cases.items():
        for value, status in values:
            args = list(good)
            args[at] = value
            assert call(*args) == status, (name, at, value)


def test_int_entry_points_refuse(b):
    N, S, A, B_, Y, W = (getattr(b, "SPINNER_ERR_" + n) for n in ("NULL_PTR", "BAD_SHAPE", "ALIGNMENT", "BAD_BATCH", "BAD_TYPE", "WORKSPACE"))
    # x, dtype, rows, k, stride, diag, block, places, top, codes, scales, stream
    _refused(b, "spinner_int_quantize", [64, 1, 4, 512, 512, 64, 256, 64, 2, 64, 64, None],
             {0: [(None, N), (72, A)], 1: [(3, Y), (-1, Y)], 2: [(-1, B_), (BIG, B_)], 3: [(0, S), ((1 << 17), S), (500, S)], 4: [(-1, S)], 5: [(72, A)],
              6: [(0, S), (16, S), (8192, S), (384, S)], 7: [(None, S), (66, A)], 8: [(0, S), (33, S)], 9: [(None, N), (72, A)], 10: [(None, N), (66, A)]})
    # codes, scales, rows, k, out, dtype, stride, stream
    _refused(b, "spinner_int_dequantize", [64, 64, 4, 40, 64, 1, 40, None],
             {0: [(None, N), (72, A)], 1: [(None, N), (66, A)], 2: [(-1, B_), (BIG + 1, B_)], 3: [(0, S), (1 << 17, S)], 4: [(None, N), (72, A)], 5: [(3, Y)], 6: [(39, S)]})
    # a, a_scales, rows, k, w, w_scales, n, experts, ends, out, dtype, stride, stream
    _refused(b, "spinner_int_matmul", [64, 64, 4, 40, 64, 64, 10, 3, 64, 64, 1, 10, None],
             {0: [(None, N), (72, A)], 1: [(None, N), (66, A)], 2: [(-1, B_), (BIG + 1, B_)], 3: [(0, S), (1 << 17, S)], 4: [(None, N), (72, A)], 5: [(None, N), (66, A)],
              6: [(0, S), ((1 << 24) + 1, S)], 7: [(0, S), (1025, S)], 8: [(None, N), (68, A)], 9: [(None, N), (72, A)], 10: [(3, Y)], 11: [(9, S)]})
    # x, dtype, rows, k, stride, diag, block, places, top, w, w_scales, n, experts, ends, out, stride, workspace, stream
    _refused(b, "spinner_int_linear", [64, 1, 4, 512, 512, 64, 256, 64, 2, 64, 64, 10, 3, 64, 64, 10, 64, None],
             {0: [(None, N), (72, A)], 1: [(3, Y)], 2: [(-1, B_), (BIG, B_)], 3: [(0, S), (1 << 17, S), (500, S)], 6: [(0, S), (8192, S)], 7: [(None, S)], 8: [(0, S), (33, S)],
              9: [(None, N), (72, A)], 10: [(None, N), (66, A)], 11: [(0, S)], 12: [(0, S), (1025, S)], 13: [(None, N), (68, A)], 14: [(None, N), (72, A)], 15: [(9, S)],
              16: [(None, W), (72, A)]})
    lib = b.lib._lib
    assert lib.spinner_int_quantize(None, 0, 0, 40, 40, None, 0, None, 1, None, None, None) == b.SPINNER_OK
    assert lib.spinner_int_linear(None, 0, 0, 40, 40, None, 0, None, 1, None, None, 5, 1, None, None, 5, None, None) == b.SPINNER_OK
    assert b.spinner_int_linear_workspace_bytes(3, 40) == 3 * 52 and b.spinner_int_linear_workspace_bytes(3, 1 << 17) == 0
    assert b.spinner_int_linear_workspace_bytes(1, FAR + 32) == 0


def test_routing_entry_points_refuse(b):
    N, S, A, B_, Y, W, E = (getattr(b, "SPINNER_ERR_" + n) for n in ("NULL_PTR", "BAD_SHAPE", "ALIGNMENT", "BAD_BATCH", "BAD_TYPE", "WORKSPACE", "BAD_EPILOGUE"))
    one = ctypes.c_float(1.0)
    # logits, dtype, rows, experts, stride, bias, mask, score, groups, top_groups, group_top, top, renormalise, scale, weights, chosen, stream
    _refused(b, "spinner_route", [64, 1, 4, 32, 32, 64, 64, 1, 4, 2, 2, 8, 1, one, 64, 64, None],
             {0: [(None, N), (72, A)], 1: [(3, Y)], 2: [(-1, B_), (BIG, B_)], 3: [(0, S), (1025, S), (30, S), (7, S)], 4: [(-1, S)], 5: [(66, A)], 7: [(2, E), (-1, E)],
              8: [(0, S), (3, S), (64, S), (16, S)], 9: [(0, S), (5, S)], 10: [(0, S), (3, S)], 11: [(0, S), (17, S), (33, S)], 14: [(None, N), (66, A)], 15: [(None, N), (66, A)]})
    _refused(b, "spinner_route", [64, 1, 4, 1024, 1024, None, None, 1, 128, 64, 2, 8, 1, one, 64, 64, None], {8: [(128, S)]})
    # dweights, logits, dtype, rows, experts, stride, chosen, score, top, renormalise, scale, dlogits, stride, stream
    _refused(b, "spinner_route_grad", [64, 64, 1, 4, 32, 32, 64, 1, 8, 1, one, 64, 32, None],
             {0: [(None, N), (66, A)], 1: [(None, N), (72, A)], 2: [(3, Y)], 3: [(-1, B_), (BIG, B_)], 4: [(0, S), (1025, S), (7, S), (33, S)], 5: [(-1, S)], 6: [(None, N), (66, A)],
              7: [(2, E)], 8: [(0, S), (33, S)], 11: [(None, N), (72, A)], 12: [(31, S)]})
    # chosen, count, experts, places, ends, workspace, stream
    _refused(b, "spinner_route_order", [64, 100000, 32, 64, 64, 64, None],
             {0: [(None, N), (66, A)], 1: [(-1, B_), (BIG + 1, B_)], 2: [(0, S), (1025, S)], 3: [(None, N), (66, A)], 4: [(None, N), (68, A)], 5: [(None, W), (66, A)]})
    assert b.spinner_route_order_workspace_bytes(100, 32) == 0 and b.spinner_route_order_workspace_bytes(100000, 32) % (33 * 4) == 0
    assert b.spinner_route_order_workspace_bytes(100000, 32) > 0 and b.spinner_route_order_workspace_bytes(100000, FAR + 32) == 0
    # x, dtype, rows, n, stride, places, top, out, stride, stream
    _refused(b, "spinner_dispatch", [64, 1, 4, 40, 40, 64, 2, 64, 40, None],
             {0: [(None, N), (72, A)], 1: [(3, Y)], 2: [(-1, B_), (BIG, B_)], 3: [(0, S), ((1 << 24) + 1, S), (41, S)], 4: [(-1, S)], 5: [(None, N), (66, A)], 6: [(0, S), (33, S)],
              7: [(None, N), (72, A)], 8: [(39, S)]})
    # y, dtype, rows, n, stride, places, weights, top, out, stride, stream
    _refused(b, "spinner_combine", [64, 1, 4, 40, 40, 64, 64, 2, 64, 40, None],
             {0: [(None, N), (72, A)], 1: [(3, Y)], 2: [(-1, B_), (BIG, B_)], 3: [(0, S), (41, S)], 4: [(-1, S)], 5: [(None, N), (66, A)], 6: [(66, A)], 7: [(0, S), (33, S)],
              8: [(None, N), (72, A)], 9: [(39, S)]})
    # dout, y, dtype, rows, n, dout_stride, y_stride, places, weights, top, dy, stride, dweights, stream
    _refused(b, "spinner_combine_grad", [64, 64, 1, 4, 40, 40, 40, 64, 64, 2, 64, 40, 64, None],
             {0: [(None, N), (72, A)], 1: [(None, N), (72, A)], 2: [(3, Y)], 3: [(-1, B_), (BIG, B_)], 4: [(0, S), (41, S)], 5: [(-1, S)], 6: [(-1, S)], 7: [(None, N), (66, A)],
              8: [(None, N), (66, A)], 9: [(0, S), (33, S)], 10: [(None, N), (72, A)], 11: [(39, S)], 12: [(None, N), (66, A)]})


GOOD = {
    "spinner_int_quantize": dict(x=T(5, 40, **h), diag=None, places=T(5, 2, **i32), codes=T(10, 48, **i8), scales=T(10)),
    "spinner_int_dequantize": dict(codes=T(5, 48, **i8), scales=T(5), k=40),
    "spinner_int_matmul": dict(a_codes=T(5, 48, **i8), a_scales=T(5), w_codes=T(3, 7, 48, **i8), w_scales=T(3, 7), ends=T(3, **i64)),
    "spinner_int_linear": dict(x=T(5, 40, **h), w_codes=T(3, 7, 48, **i8), w_scales=T(3, 7), ends=T(3, **i64), places=T(5, 2, **i32)),
    "spinner_route": dict(logits=T(5, 32, **h), top=4, bias=T(32), mask=T(5, dtype="bool"), weights=T(5, 4), experts=T(5, 4, **i32)),
    "spinner_route_grad": dict(dweights=T(5, 4), logits=T(5, 32, **h), experts=T(5, 4, **i32)),
    "spinner_route_order": dict(experts=T(5000, 4, **i32), count=32, places=T(5000, 4, **i32), ends=T(32, **i64)),
    "spinner_dispatch": dict(x=T(5, 40, **h), places=T(5, 2, **i32)),
    "spinner_combine": dict(y=T(10, 40, **h), places=T(5, 2, **i32), weights=T(5, 2)),
    "spinner_combine_grad": dict(dout=T(5, 40, **h), y=T(10, 40, **h), places=T(5, 2, **i32), weights=T(5, 2)),
}
BAD = {
    "spinner_int_quantize": dict(x=[but(T(5, 40), is_cuda=False)], places=[T(5, 2, **i64), T(4, 2, **i32), T(10, **i32), but(T(5, 2, **i32), whole=False)],
                                 codes=[T(10, 40, **i8), T(10, 48, **u8), T(9, 48, **i8), but(T(10, 48, **i8), whole=False), T(10, 64, **i8)], scales=[T(9), T(10, **h), T(10, 1)]),
    "spinner_int_dequantize": dict(codes=[T(5, 40, **i8), T(5, 48, **u8), but(T(5, 48, **i8), is_cuda=False)], scales=[T(4), T(5, **h)], k=[32, 49, 0], out=[T(5, 48), T(4, 40), T(5, 40, **h)]),
    "spinner_int_matmul": dict(a_codes=[T(5, 64, **i8), T(5, 48, **u8)], a_scales=[T(6), T(5, **h)], w_codes=[T(3, 7, 64, **i8), T(3, 7, 48, **u8), but(T(3, 7, 48, **i8), whole=False)],
                               w_scales=[T(3, 8), T(21), T(3, 7, **h)], ends=[None, T(4, **i64), T(3, **i32)], out=[T(5, 7), T(5, 8, **h)]),
    "spinner_int_linear": dict(w_codes=[T(3, 7, 64, **i8)], w_scales=[T(7, 3)], ends=[None, T(2, **i64)], places=[T(6, 2, **i32)], out=[T(5, 7, **h), T(10, 7)], workspace=[T(519, **u8), but(T(520, **u8), is_cuda=False)],
                               diag=[T(39), T(40, **h)]),
    "spinner_route": dict(bias=[T(31), T(32, **h)], mask=[T(4, dtype="bool"), T(5), but(T(5, dtype="bool"), is_cuda=False)], weights=[T(5, 5), T(5, 4, **h)], experts=[T(5, 4, **i64), T(4, 5, **i32)]),
    "spinner_route_grad": dict(dweights=[T(5, 5), T(5, 4, **h)], experts=[T(5, 4, **i64), T(4, 4, **i32)], dlogits=[T(5, 32), T(5, 31, **h)]),
    "spinner_route_order": dict(experts=[T(5000, 4, **i64), T(20000, **i32)], places=[T(5000, 3, **i32), T(5000, 4, **i64)], ends=[T(31, **i64), T(32, **i32)], workspace=[T(64, **u8)]),
    "spinner_dispatch": dict(places=[T(4, 2, **i32), T(5, 2, **i64), T(5, **i32)], out=[T(9, 40, **h), T(10, 40)]),
    "spinner_combine": dict(places=[T(6, 2, **i32), T(5, 2, **i64)], weights=[T(5, 3), T(5, 2, **h)], out=[T(5, 40), T(6, 40, **h)]),
    "spinner_combine_grad": dict(dout=[T(5, 41, **h), T(5, 40), T(6, 40, **h)], weights=[T(5, 3)], dy=[T(10, 40), T(9, 40, **h)], dweights=[T(5, 2, **h), T(10)]),
}


@pytest.mark.parametrize("name", list(GOOD))
def test_the_binding_refuses_what_a_kernel_would_reach_past(b, name):
    getattr(b, name)(**GOOD[name])
    assert b.lib.calls == [name]
    for arg, values in BAD[name].items():
        for v in values:
            b.lib.calls.clear()
            with pytest.raises(ValueError):
                getattr(b, name)(**{**GOOD[name], arg: v})
            assert b.lib.calls == [], (name, arg)


TOO_MANY = {
    "quantise, k": ("spinner_int_quantize", dict(x=T(1, FAR + 64))),
    "quantise, block": ("spinner_int_quantize", dict(x=T(1, 64), block=FAR + 64)),
    "quantise, top": ("spinner_int_quantize", dict(x=T(1, 64), places=T(1, FAR + 1, **i32))),
    "dequantise, k": ("spinner_int_dequantize", dict(codes=T(1, FAR + 16, **i8), scales=T(1))),
    "matmul, k": ("spinner_int_matmul", dict(a_codes=T(1, FAR + 16, **i8), a_scales=T(1), w_codes=T(2, FAR + 16, **i8), w_scales=T(2))),
    "linear, n": ("spinner_int_linear", dict(x=T(1, 32, **h), w_codes=T(FAR + 2, 32, **i8), w_scales=T(FAR + 2))),
    "route, experts": ("spinner_route", dict(logits=T(1, FAR + 8), top=1)),
    "route, top": ("spinner_route", dict(logits=T(1, 8), top=FAR + 1)),
    "route, groups": ("spinner_route", dict(logits=T(1, 8), top=1, groups=FAR + 1)),
    "grad, experts": ("spinner_route_grad", dict(dweights=T(1, 2), logits=T(1, FAR + 8), experts=T(1, 2, **i32))),
    "order, experts": ("spinner_route_order", dict(experts=T(1, 2, **i32), count=FAR + 2)),
    "dispatch, n": ("spinner_dispatch", dict(x=T(1, FAR + 8), places=T(1, 1, **i32))),
    "combine, n": ("spinner_combine", dict(y=T(1, FAR + 8), places=T(1, 1, **i32))),
    "combine's gradient, n": ("spinner_combine_grad", dict(dout=T(1, FAR + 8), y=T(1, FAR + 8), places=T(1, 1, **i32), weights=T(1, 1))),
}


@pytest.mark.parametrize("case", list(TOO_MANY))
def test_sizes_that_the_abi_would_cut_off_are_refused(b, case):
    name, args = TOO_MANY[case]
    with pytest.raises(b.SpinnerError) as e:
        getattr(b, name)(**args)
    assert e.value.status == b.SPINNER_ERR_BAD_SHAPE and b.lib.calls == []


CALLS = {name: {k: v for k, v in args.items() if k not in ("codes", "scales", "weights", "places", "ends") or name not in ("spinner_int_quantize", "spinner_route", "spinner_route_order")}
         for name, args in GOOD.items()}
CALLS["spinner_route"].pop("experts")
SCRATCH = {"spinner_int_linear": 1, "spinner_route_order": 1}


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_comes_from_the_stream_of_the_call(made, name):
    binding, tensors = made
    r = getattr(binding, name)(stream=MINE, **CALLS[name])
    results = r if isinstance(r, tuple) else (r,)
    assert len(tensors) == len(results) + SCRATCH.get(name, 0) and all(t.made_on is MINE for t in tensors)
    assert all(t.used_on == ([CURRENT] if any(t is q for q in results) else []) for t in tensors)
    tensors.clear()
    getattr(binding, name)(**CALLS[name])
    assert tensors and all(t.made_on is CURRENT and not t.used_on for t in tensors)


def test_sizes_of_the_products_take_every_form():
    """The sizes that the 8-bit products are tested at take all of their tiles, and the form for few rows with 16, 32 and 64 columns, by the library's rule."""
    import ctypes

    import product_forms
    from paper_1610_06209_amd import binding
    from test_gpu_int import PRODUCTS

    rule = getattr(binding.lib, "_ZN7spinner16plan_product_intEPNS_13ProductParamsE")
    columns = getattr(binding.lib, "_ZN7spinner15few_columns_intERKNS_13ProductParamsEPd")
    rule.restype, columns.restype = None, ctypes.c_int
    rule.argtypes, columns.argtypes = [ctypes.c_void_p], [ctypes.c_void_p, ctypes.c_void_p]
    forms = set()
    for rows, k, n, experts in PRODUCTS:
        p, us = product_forms._params_class()(rows=rows, experts=experts), ctypes.c_double()
        p.width, p.depth = n, -(-k // 16) * 16
        rule(ctypes.addressof(p))
        forms.add(product_forms.FORMS[p.tile] + (" %d" % columns(ctypes.addressof(p), ctypes.addressof(us)) if p.tile == 0 else ""))
    assert forms == {"256", "128", "128 deep", "64", "few rows 16", "few rows 32", "few rows 64"}
