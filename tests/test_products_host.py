"""The 4-bit and grouped products on the host: what is refused before anything is launched, and which form of the kernels sizes take."""
import glob
import os
import re

import pytest

import product_forms as forms
from test_abi_host import _NoLaunch
from test_streams_host import T, h, u8


class _Lib(_NoLaunch):
    def spinner_strerror(self, status):
        return self._lib.spinner_strerror(status)


@pytest.fixture
def b(monkeypatch):
    import torch

    from paper_1610_06209_amd import binding

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: T(*(shape if isinstance(shape, tuple) else (shape,)), dtype=str(dtype)[6:]))
    monkeypatch.setattr(binding, "_stream_handle", lambda stream: 0)
    monkeypatch.setattr(binding, "lib", _Lib(binding.lib))
    return binding


# sizes and runs that the C ABI's int does not hold, beside the small number that its low half is
FAR = 1 << 32
TOO_MANY = {
    "quantise, k": ("spinner_mx_quantize", dict(x=T(1, FAR + 64))),
    "quantise, block": ("spinner_mx_quantize", dict(x=T(1, 64), block=FAR + 64)),
    "dequantise, k": ("spinner_mx_dequantize", dict(codes=T(1, FAR // 2 + 16, **u8), scales=T(1, FAR // 32 + 1, **u8))),
    "matmul, k": ("spinner_mx_matmul", dict(a_codes=T(1, FAR // 2 + 16, **u8), a_scales=T(1, FAR // 32 + 1, **u8), w_codes=T(2, FAR // 2 + 16, **u8),
                                            w_scales=T(2, FAR // 32 + 1, **u8))),
    "matmul, n": ("spinner_mx_matmul", dict(a_codes=T(1, 16, **u8), a_scales=T(1, 1, **u8), w_codes=T(FAR + 2, 16, **u8), w_scales=T(FAR + 2, 1, **u8))),
    "linear, n": ("spinner_mx_linear", dict(x=T(1, 32, **h), w_codes=T(FAR + 2, 16, **u8), w_scales=T(FAR + 2, 1, **u8))),
    "linear, block": ("spinner_mx_linear", dict(x=T(1, 32, **h), w_codes=T(2, 16, **u8), w_scales=T(2, 1, **u8), block=FAR + 32)),
    "linear, experts": ("spinner_mx_linear", dict(x=T(1, 32, **h), w_codes=T(FAR + 1, 2, 16, **u8), w_scales=T(FAR + 1, 2, 1, **u8), ends=T(FAR + 1, dtype="int64"))),
    "grouped, n": ("spinner_grouped_matmul", dict(x=T(1, 8, **h), w=T(FAR + 8, 8, **h))),
    "dx, k": ("spinner_grouped_matmul_dx", dict(dy=T(1, 8, **h), w=T(8, FAR + 8, **h))),
    "dw, k": ("spinner_grouped_matmul_dw", dict(dy=T(1, 8, **h), x=T(1, FAR + 8, **h))),
}


@pytest.mark.parametrize("case", list(TOO_MANY))
def test_sizes_that_the_abi_would_cut_off_are_refused(b, case):
    name, args = TOO_MANY[case]
    with pytest.raises(b.SpinnerError) as e:
        getattr(b, name)(**args)
    assert e.value.status == b.SPINNER_ERR_BAD_SHAPE and b.lib.calls == []


def test_workspace_sizes_of_what_is_refused_are_none(b):
    assert b.spinner_mx_linear_workspace_bytes(1, FAR + 32) == 0 and b.spinner_mx_linear_workspace_bytes(1, 32) == 17
    assert b.spinner_grouped_matmul_dw_workspace_bytes(4100, FAR + 40, 264, 1) == 0
    assert b.spinner_grouped_matmul_dw_workspace_bytes(4100, 40, FAR + 264, 1) == 0
    assert b.spinner_grouped_matmul_dw_workspace_bytes(4100, 40, 264, FAR + 1) == 0
    assert b.spinner_grouped_matmul_dw_workspace_bytes(4100, 40, 264, 1) > 0


def test_inline_assembly_declares_the_m0_that_it_writes():
    """The compiler keeps values of its own in m0 (spills, indexing): a statement that writes it has to say so."""
    from paper_1610_06209_amd import build

    found = 0
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.h*"))):
        for statement in re.findall(r"\basm\b[^;]*?\((.*?)\);", open(path).read(), re.S):
            if re.search(r"\bm0\s*,", statement):
                found += 1
                assert re.search(r":[^:]*\"m0\"[^:]*$", statement), (path, statement)
    assert found


def test_the_rule_for_forms_is_read_aright():
    """The weight gradient's shares are those that its workspace is made for, by the public call."""
    from paper_1610_06209_amd import binding

    for rows, experts, k, n in forms.SIXTEEN + [(1, 1, 1, 1), (70000, 7, 40, 56)]:
        shares = forms.plan(forms.DW, False, rows, experts, k, n)[2]
        assert binding.spinner_grouped_matmul_dw_workspace_bytes(rows, n, k, experts) == (4 * shares * experts * k * n if shares > 1 else 0)
    assert forms.plan(forms.FORWARD, False, 16, 1, 512, 512)[0] == forms.plan(forms.FORWARD, True, 64, 32, 512, 512)[0] == "few rows"


@pytest.mark.parametrize("one", [True, False])
@pytest.mark.parametrize("direction", [forms.FORWARD, forms.DX])
def test_tested_sizes_run_through_each_form(direction, one):
    """Sizes of test_gpu_product_depth.py: for each form more chunks of depth than its buffers hold, by the library's rule as it stands."""
    found = {forms.runs_through(direction, False, *s) for s in forms.SIXTEEN if (s[1] == 1) == one} - {None}
    assert found == {(f, False) for f in forms.STAGES}


def test_tested_sizes_run_through_each_form_of_weight_gradients():
    found = {forms.runs_through(forms.DW, False, *s) for s in forms.SIXTEEN if s[1] == 1} - {None}
    assert found == {(f, shares) for f in forms.STAGES for shares in (False, True)}


@pytest.mark.parametrize("one", [True, False])
def test_tested_sizes_run_through_each_form_in_4_bits(one):
    found = {forms.runs_through(forms.FORWARD, True, *s) for s in forms.FOUR if (s[1] == 1) == one} - {None}
    assert found == {(f, False) for f in ("256", "128", "64")}
