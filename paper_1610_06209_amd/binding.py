"""Thin binding of ``libspinner.so`` (the C ABI in ``include/spinner.h``): ctypes, with the usual calls in native code.

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  PyTorch is used for device memory and streams, nothing else.  There
is no fallback: if the library has not been built, importing this module
raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspinner.so")

SPINNER_OK = 0
SPINNER_ERR_BAD_N = -1
SPINNER_ERR_BAD_M = -2
SPINNER_ERR_NULL_PTR = -3
SPINNER_ERR_BAD_EPILOGUE = -4
SPINNER_ERR_BAD_BATCH = -5
SPINNER_ERR_WORKSPACE = -6
SPINNER_ERR_HIP = -7
SPINNER_ERR_BAD_L = -8
SPINNER_ERR_ALIGNMENT = -9
SPINNER_ERR_UNSUPPORTED = -10
SPINNER_ERR_SCRATCH_LIMIT = -11
SPINNER_ERR_BAD_TYPE = -12
SPINNER_ERR_BAD_SHAPE = -13

SPINNER_EPI_NONE = 0
SPINNER_EPI_COSSIN = 1
EPILOGUES = {"none": SPINNER_EPI_NONE, "cossin": SPINNER_EPI_COSSIN}

EXPORTS = ["spinner_apply", "spinner_hash", "spinner_workspace_bytes", "spinner_strerror",
           "spinner_version", "spinner_stream_copy", "spinner_signs_bytes", "spinner_pack_signs",
           "spinner_apply_signs", "spinner_hash_signs", "spinner_hash_workspace_bytes", "spinner_hash_ws", "spinner_hash_signs_ws", "spinner_code_bytes", "spinner_codes_workspace_bytes",
           "spinner_code_position", "spinner_sign_codes", "spinner_sign_codes_signs", "spinner_angular_gram",
           "spinner_layer_saved_bytes", "spinner_layer_workspace_bytes", "spinner_layer_forward",
           "spinner_layer_backward", "spinner_sketch_workspace_bytes", "spinner_sketch", "spinner_sketch_gram",
           "spinner_sketch_gram_workspace_bytes", "spinner_sketch_gram_static", "spinner_sketch_gram_static_limit",
           "spinner_blocks_workspace_bytes", "spinner_apply_blocks",
           "spinner_struct_params", "spinner_struct_spectrum_bytes", "spinner_struct_prepare", "spinner_struct_apply",
           "spinner_struct_workspace_bytes", "spinner_struct_apply_ws",
           "spinner_mx_quantize", "spinner_mx_dequantize", "spinner_mx_matmul", "spinner_mx_linear_workspace_bytes",
           "spinner_mx_linear", "spinner_grouped_matmul", "spinner_grouped_matmul_dx", "spinner_grouped_matmul_dw",
           "spinner_grouped_matmul_dw_workspace_bytes"]

if not os.path.exists(LIB_PATH) or not os.path.exists(os.path.join(_HERE, "_native.so")):
    raise ImportError(
        "libspinner.so or _native.so is not built: run `python -m paper_1610_06209_amd.build` "
        "(or __graft_entry__.build()); there is no fallback path")

# PyTorch ships its own HIP runtime and loads it by path; the library must bind to that same copy (it owns
# the device memory and the streams handed in here), so torch is loaded first and the library's
# dependency on libamdhip64 then resolves to the runtime already in the process.
import torch  # noqa: E402

lib = ctypes.CDLL(LIB_PATH)
# The usual calls, checks and allocations included, in native code (csrc/binding_native.cpp); each answers None to a call
# that is out of the ordinary or that the library refuses, which then goes the long way below.
from . import _native  # noqa: E402

_vp = ctypes.c_void_p
lib.spinner_apply.restype = ctypes.c_int
lib.spinner_apply.argtypes = [_vp, ctypes.c_int, ctypes.c_long, _vp, _vp, _vp, ctypes.c_int, ctypes.c_int,
                              ctypes.c_float, _vp, _vp, _vp]
lib.spinner_hash.restype = ctypes.c_int
lib.spinner_hash.argtypes = [_vp, ctypes.c_int, ctypes.c_long, ctypes.c_int, _vp, _vp, _vp]
lib.spinner_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_long, ctypes.c_int, ctypes.c_int]
lib.spinner_strerror.restype = ctypes.c_char_p
lib.spinner_strerror.argtypes = [ctypes.c_int]
lib.spinner_version.restype = ctypes.c_int
lib.spinner_version.argtypes = []
lib.spinner_signs_bytes.restype = ctypes.c_size_t
lib.spinner_signs_bytes.argtypes = [ctypes.c_int, ctypes.c_int]
lib.spinner_pack_signs.restype = ctypes.c_int
lib.spinner_pack_signs.argtypes = [_vp, ctypes.c_int, ctypes.c_int, _vp, _vp]
lib.spinner_apply_signs.restype = ctypes.c_int
lib.spinner_apply_signs.argtypes = [_vp, ctypes.c_int, ctypes.c_long, _vp, ctypes.c_int, ctypes.c_int,
                                    ctypes.c_float, _vp, _vp, _vp]
lib.spinner_hash_signs.restype = ctypes.c_int
lib.spinner_hash_signs.argtypes = [_vp, ctypes.c_int, ctypes.c_long, ctypes.c_int, _vp, _vp, _vp]
lib.spinner_hash_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_hash_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_long]
lib.spinner_hash_ws.restype = ctypes.c_int
lib.spinner_hash_ws.argtypes = [_vp, ctypes.c_int, ctypes.c_long, ctypes.c_int, _vp, _vp, _vp, _vp]
lib.spinner_hash_signs_ws.restype = ctypes.c_int
lib.spinner_hash_signs_ws.argtypes = [_vp, ctypes.c_int, ctypes.c_long, ctypes.c_int, _vp, _vp, _vp, _vp]
lib.spinner_stream_copy.restype = ctypes.c_int
lib.spinner_stream_copy.argtypes = [_vp, _vp, ctypes.c_size_t, _vp]
lib.spinner_code_bytes.restype = ctypes.c_size_t
lib.spinner_code_bytes.argtypes = [ctypes.c_int]
lib.spinner_codes_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_codes_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_long]
lib.spinner_code_position.restype = ctypes.c_int
lib.spinner_code_position.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int)]
lib.spinner_sign_codes.restype = ctypes.c_int
lib.spinner_sign_codes.argtypes = [_vp, ctypes.c_int, ctypes.c_long, _vp, _vp, _vp, ctypes.c_int, _vp, _vp, _vp]
lib.spinner_sign_codes_signs.restype = ctypes.c_int
lib.spinner_sign_codes_signs.argtypes = [_vp, ctypes.c_int, ctypes.c_long, _vp, ctypes.c_int, _vp, _vp, _vp]
lib.spinner_angular_gram.restype = ctypes.c_int
lib.spinner_angular_gram.argtypes = [_vp, ctypes.c_long, _vp, ctypes.c_long, ctypes.c_int, _vp, _vp]
lib.spinner_layer_saved_bytes.restype = ctypes.c_size_t
lib.spinner_layer_saved_bytes.argtypes = [ctypes.c_int, ctypes.c_long]
lib.spinner_layer_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_layer_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_long]
lib.spinner_layer_forward.restype = ctypes.c_int
lib.spinner_layer_forward.argtypes = [_vp, ctypes.c_int, ctypes.c_long, _vp, _vp, _vp, ctypes.c_float, _vp, _vp, _vp]
lib.spinner_layer_backward.restype = ctypes.c_int
lib.spinner_layer_backward.argtypes = [_vp, _vp, _vp, ctypes.c_int, ctypes.c_long, _vp, _vp, _vp, ctypes.c_float, _vp, _vp,
                                       _vp, _vp]
lib.spinner_sketch_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_sketch_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int]
lib.spinner_sketch.restype = ctypes.c_int
lib.spinner_sketch.argtypes = [_vp, ctypes.c_int, ctypes.c_int, _vp, _vp, _vp, _vp, ctypes.c_int, ctypes.c_float, _vp, _vp, _vp]
lib.spinner_sketch_gram.restype = ctypes.c_int
lib.spinner_sketch_gram.argtypes = [_vp, ctypes.c_int, ctypes.c_int, _vp, _vp, _vp]
lib.spinner_sketch_gram_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_sketch_gram_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_int]
lib.spinner_sketch_gram_static.restype = ctypes.c_int
lib.spinner_sketch_gram_static.argtypes = [_vp, ctypes.c_int, ctypes.c_int, _vp, _vp]
lib.spinner_sketch_gram_static_limit.restype = ctypes.c_size_t
lib.spinner_sketch_gram_static_limit.argtypes = []
lib.spinner_blocks_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_blocks_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_long, ctypes.c_int, ctypes.c_int]
lib.spinner_apply_blocks.restype = ctypes.c_int
lib.spinner_apply_blocks.argtypes = [_vp, ctypes.c_int, ctypes.c_long, ctypes.c_int, _vp, ctypes.c_int, ctypes.c_int,
                                     ctypes.c_float, _vp, _vp, _vp]
lib.spinner_struct_params.restype = ctypes.c_size_t
lib.spinner_struct_params.argtypes = [ctypes.c_int, ctypes.c_int]
lib.spinner_struct_spectrum_bytes.restype = ctypes.c_size_t
lib.spinner_struct_spectrum_bytes.argtypes = [ctypes.c_int, ctypes.c_int]
lib.spinner_struct_prepare.restype = ctypes.c_int
lib.spinner_struct_prepare.argtypes = [ctypes.c_int, _vp, ctypes.c_int, _vp, _vp]
lib.spinner_struct_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_struct_workspace_bytes.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_long]
lib.spinner_struct_apply_ws.restype = ctypes.c_int
lib.spinner_struct_apply_ws.argtypes = [_vp, ctypes.c_int, ctypes.c_long, ctypes.c_int, _vp, _vp, _vp, ctypes.c_int, ctypes.c_float,
                                        _vp, _vp, _vp]
lib.spinner_struct_apply.restype = ctypes.c_int
lib.spinner_struct_apply.argtypes = [_vp, ctypes.c_int, ctypes.c_long, ctypes.c_int, _vp, _vp, _vp, ctypes.c_int, ctypes.c_float,
                                     _vp, _vp]
_int, _long = ctypes.c_int, ctypes.c_long
lib.spinner_mx_quantize.restype = _int
lib.spinner_mx_quantize.argtypes = [_vp, _int, _long, _int, _long, _vp, _int, _vp, _vp, _vp]
lib.spinner_mx_dequantize.restype = _int
lib.spinner_mx_dequantize.argtypes = [_vp, _vp, _long, _int, _vp, _int, _long, _vp]
lib.spinner_mx_matmul.restype = _int
lib.spinner_mx_matmul.argtypes = [_vp, _vp, _long, _int, _vp, _vp, _int, _int, _vp, _vp, _int, _long, _vp]
lib.spinner_mx_linear_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_mx_linear_workspace_bytes.argtypes = [_long, _int]
lib.spinner_mx_linear.restype = _int
lib.spinner_mx_linear.argtypes = [_vp, _int, _long, _int, _long, _vp, _int, _vp, _vp, _int, _int, _vp, _vp, _long, _vp, _vp]
lib.spinner_grouped_matmul.restype = _int
lib.spinner_grouped_matmul.argtypes = [_vp, _int, _long, _int, _long, _vp, _int, _int, _vp, _vp, _long, _vp]
lib.spinner_grouped_matmul_dx.restype = _int
lib.spinner_grouped_matmul_dx.argtypes = [_vp, _int, _long, _int, _long, _vp, _int, _int, _vp, _vp, _long, _vp]
lib.spinner_grouped_matmul_dw.restype = _int
lib.spinner_grouped_matmul_dw.argtypes = [_vp, _vp, _int, _long, _int, _int, _long, _long, _int, _vp, _vp, _int, _vp, _vp]
lib.spinner_grouped_matmul_dw_workspace_bytes.restype = ctypes.c_size_t
lib.spinner_grouped_matmul_dw_workspace_bytes.argtypes = [_long, _int, _int, _int]
STRUCT_KINDS = {"circulant": 0, "skew_circulant": 1, "toeplitz": 2, "hankel": 3}


class SpinnerError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__("spinner: %s (status %d)" % (spinner_strerror(status), status))


def spinner_strerror(status: int) -> str:
    return lib.spinner_strerror(int(status)).decode()


def spinner_version() -> int:
    return int(lib.spinner_version())


def spinner_workspace_bytes(n: int, batch: int, m: int, epilogue) -> int:
    return _workspace_bytes(int(n), int(batch), int(m), _epi(epilogue))


# The sizes that every call looks up are pure functions of whole numbers: the last ones asked for are remembered.
@functools.lru_cache(maxsize=256)
def _workspace_bytes(n, batch, m, epi):
    return int(lib.spinner_workspace_bytes(n, batch, m, epi))


@functools.lru_cache(maxsize=256)
def _signs_bytes(n, L):
    return int(lib.spinner_signs_bytes(n, L))


@functools.lru_cache(maxsize=256)
def _layer_workspace_bytes(n, batch):
    return int(lib.spinner_layer_workspace_bytes(n, batch))


def _epi(e) -> int:
    return EPILOGUES[e] if isinstance(e, str) else int(e)


# The handle of torch's current stream without the Stream object that torch.cuda.current_stream() makes of it on every
# call (1.2 us of the 10 us that a small call took); a torch without these two functions takes the long way.
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(stream):
    if stream is not None:
        return stream.cuda_stream
    if _current_raw_stream is not None and _current_device is not None:
        return _current_raw_stream(_current_device())
    return torch.cuda.current_stream().cuda_stream


_new_on = _native._new_on


def _new(shape, dtype, device, stream, scratch=False):
    """Memory for a result, or for scratch that is let go of on return, of a call on ``stream``.

    With an explicit stream it is memory of that stream: a block that the current stream has let go of may still be read or written by what
    is queued there.  A result is then used on the current stream too.
    """
    if stream is None or device.type != "cuda" or stream.cuda_stream == _stream_handle(None):
        return torch.empty(shape, dtype=dtype, device=device)
    return _new_on(shape if isinstance(shape, tuple) else (shape,), dtype, device.index, stream.cuda_stream, scratch)


def _check_tensor(t, name, dtype):
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s CUDA tensor" % (name, dtype))


# Nothing behind the C ABI knows how long a buffer is: a call that could reach past one, or into memory the GPU has no way to, is
# refused here.
def _check_device(t, name):
    if not t.is_cuda and not t.is_pinned():
        raise ValueError("%s must be in GPU memory" % name)


def _check_workspace(t, need):
    if t is None:
        return
    if t.numel() * t.element_size() < need or t.untyped_storage().nbytes() - t.storage_offset() * t.element_size() < need:
        raise ValueError("workspace too small")
    _check_device(t, "workspace")


def _check_signs(signs, n, triples, first=0):
    if first < 0 or signs.numel() < (first + triples) * spinner_signs_bytes(n, 1):
        raise ValueError("signs buffer too small for this n / triple")
    _check_device(signs, "signs")


def _check_diagonals(n, **diagonals):
    for name, d in diagonals.items():
        _check_tensor(d, name, torch.float32)
        if d.numel() < n:
            raise ValueError("%s is shorter than n" % name)


def _check_result(t, name, count):
    _check_device(t, name)
    if not t.is_contiguous() or t.numel() * t.element_size() < 4 * count:
        raise ValueError("%s must be contiguous and hold %d floats" % (name, count))


def spinner_apply(x, d1, d2, d3, m=None, epilogue="none", scale=1.0, out=None, workspace=None, stream=None):
    """out = epilogue(scale * first m coordinates of H D3 H D2 H D1 x) for each row of x.

    x: fp32 CUDA tensor [batch][n]; d1..d3: fp32 CUDA tensors [n].  Allocates
    ``out`` (and the workspace when one is needed) unless given.  Asynchronous
    on ``stream`` (default: torch's current stream).
    """
    r = _native.apply(x, d1, d2, d3, m, epilogue, scale, out, workspace, stream)
    if r is not None:
        return r
    _check_tensor(x, "x", torch.float32)
    for name, d in (("d1", d1), ("d2", d2), ("d3", d3)):
        _check_tensor(d, name, torch.float32)
    batch, n = x.shape
    for d in (d1, d2, d3):
        if d.numel() != n:
            raise ValueError("diagonal length must equal n")
    m = n if m is None else int(m)
    epi = _epi(epilogue)
    width = 2 * m if epi == SPINNER_EPI_COSSIN else m
    if out is None:
        out = _new((batch, width), torch.float32, x.device, stream)
    else:
        _check_tensor(out, "out", torch.float32)
        if out.numel() != batch * width:
            raise ValueError("out has the wrong size")
    need = spinner_workspace_bytes(n, batch, m, epi)
    if need and workspace is None:
        workspace = _new(need, torch.uint8, x.device, stream, scratch=True)
    _check_workspace(workspace, need)
    rc = lib.spinner_apply(x.data_ptr(), n, batch, d1.data_ptr(), d2.data_ptr(), d3.data_ptr(), m, epi,
                           ctypes.c_float(scale), out.data_ptr(),
                           workspace.data_ptr() if workspace is not None else None, _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out


def spinner_hash(x, diag_sets, out_idx=None, stream=None):
    """Cross-polytope buckets, int32 [batch][L], for L diagonal triples diag_sets fp32 [L][3][n]."""
    r = _native.hash(x, diag_sets, out_idx, stream)
    if r is not None:
        return r
    _check_tensor(x, "x", torch.float32)
    _check_tensor(diag_sets, "diag_sets", torch.float32)
    batch, n = x.shape
    if diag_sets.dim() != 3 or diag_sets.shape[1] != 3 or diag_sets.shape[2] != n:
        raise ValueError("diag_sets must be [L][3][n]")
    L = diag_sets.shape[0]
    if out_idx is None:
        out_idx = _new((batch, L), torch.int32, x.device, stream)
    else:
        _check_tensor(out_idx, "out_idx", torch.int32)
        if out_idx.numel() != batch * L:
            raise ValueError("out_idx has the wrong size")
    rc = lib.spinner_hash(x.data_ptr(), n, batch, L, diag_sets.data_ptr(), out_idx.data_ptr(), _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out_idx


def spinner_hash_workspace_bytes(n: int, batch: int) -> int:
    return int(lib.spinner_hash_workspace_bytes(int(n), int(batch)))


def _hash_workspace(x, n, batch, workspace, stream):
    need = spinner_hash_workspace_bytes(n, batch)
    if workspace is None and need:
        workspace = _new(need, torch.uint8, x.device, stream, scratch=True)
    _check_workspace(workspace, need)
    return workspace


def spinner_hash_ws(x, diag_sets, out_idx=None, workspace=None, stream=None):
    """spinner_hash for every n up to 2^24 (a workspace tensor is made when none is given and one is needed)."""
    _check_tensor(x, "x", torch.float32)
    _check_tensor(diag_sets, "diag_sets", torch.float32)
    batch, n = x.shape
    if diag_sets.dim() != 3 or diag_sets.shape[1] != 3 or diag_sets.shape[2] != n:
        raise ValueError("diag_sets must be [L][3][n]")
    L = diag_sets.shape[0]
    if out_idx is None:
        out_idx = _new((batch, L), torch.int32, x.device, stream)
    else:
        _check_tensor(out_idx, "out_idx", torch.int32)
        if out_idx.numel() != batch * L:
            raise ValueError("out_idx has the wrong size")
    workspace = _hash_workspace(x, n, batch, workspace, stream)
    rc = lib.spinner_hash_ws(x.data_ptr(), n, batch, L, diag_sets.data_ptr(), out_idx.data_ptr(),
                             workspace.data_ptr() if workspace is not None else None, _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out_idx


def spinner_hash_signs_ws(x, signs, L, out_idx=None, workspace=None, stream=None):
    """spinner_hash_signs for every n up to 2^24."""
    _check_tensor(x, "x", torch.float32)
    batch, n = x.shape
    _check_signs(signs, n, L)
    if out_idx is None:
        out_idx = _new((batch, L), torch.int32, x.device, stream)
    else:
        _check_tensor(out_idx, "out_idx", torch.int32)
        if out_idx.numel() != batch * L:
            raise ValueError("out_idx has the wrong size")
    workspace = _hash_workspace(x, n, batch, workspace, stream)
    rc = lib.spinner_hash_signs_ws(x.data_ptr(), n, batch, L, signs.data_ptr(), out_idx.data_ptr(),
                                   workspace.data_ptr() if workspace is not None else None, _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out_idx


def spinner_signs_bytes(n: int, L: int) -> int:
    return _signs_bytes(int(n), int(L))


def spinner_pack_signs(diag_sets, stream=None):
    """Pack fp32 +-1 diagonals [L][3][n] into the library's sign words (uint8 CUDA tensor, opaque)."""
    _check_tensor(diag_sets, "diag_sets", torch.float32)
    if diag_sets.dim() != 3 or diag_sets.shape[1] != 3:
        raise ValueError("diag_sets must be [L][3][n]")
    L, _, n = diag_sets.shape
    nbytes = spinner_signs_bytes(n, L)
    if nbytes == 0:
        raise SpinnerError(SPINNER_ERR_BAD_N)
    signs = _new(nbytes, torch.uint8, diag_sets.device, stream)
    rc = lib.spinner_pack_signs(diag_sets.data_ptr(), n, L, signs.data_ptr(), _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return signs


def spinner_apply_signs(x, signs, m=None, epilogue="none", scale=1.0, out=None, workspace=None, stream=None,
                        triple=0):
    """spinner_apply for +-1 diagonals given as packed sign words (see spinner_pack_signs)."""
    r = _native.apply_signs(x, signs, m, epilogue, scale, out, workspace, stream, triple)
    if r is not None:
        return r
    _check_tensor(x, "x", torch.float32)
    batch, n = x.shape
    m = n if m is None else int(m)
    epi = _epi(epilogue)
    width = 2 * m if epi == SPINNER_EPI_COSSIN else m
    if out is None:
        out = _new((batch, width), torch.float32, x.device, stream)
    else:
        _check_tensor(out, "out", torch.float32)
        if out.numel() != batch * width:
            raise ValueError("out has the wrong size")
    one = spinner_signs_bytes(n, 1)
    _check_signs(signs, n, 1, triple)
    need = spinner_workspace_bytes(n, batch, m, epi)
    if need and workspace is None:
        workspace = _new(need, torch.uint8, x.device, stream, scratch=True)
    _check_workspace(workspace, need)
    rc = lib.spinner_apply_signs(x.data_ptr(), n, batch, signs.data_ptr() + triple * one, m, epi,
                                 ctypes.c_float(scale), out.data_ptr(),
                                 workspace.data_ptr() if workspace is not None else None, _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out


def spinner_hash_signs(x, signs, L, out_idx=None, stream=None):
    """spinner_hash for +-1 diagonals given as packed sign words of L triples."""
    r = _native.hash_signs(x, signs, L, out_idx, stream)
    if r is not None:
        return r
    _check_tensor(x, "x", torch.float32)
    batch, n = x.shape
    _check_signs(signs, n, L)
    if out_idx is None:
        out_idx = _new((batch, L), torch.int32, x.device, stream)
    else:
        _check_tensor(out_idx, "out_idx", torch.int32)
        if out_idx.numel() != batch * L:
            raise ValueError("out_idx has the wrong size")
    rc = lib.spinner_hash_signs(x.data_ptr(), n, batch, L, signs.data_ptr(), out_idx.data_ptr(), _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out_idx


def spinner_stream_copy(src, dst, stream=None):
    """dst[:] = src with the library's plain copy kernel (measurement aid)."""
    _check_tensor(src, "src", torch.float32)
    _check_tensor(dst, "dst", torch.float32)
    if src.numel() != dst.numel():
        raise ValueError("size mismatch")
    rc = lib.spinner_stream_copy(src.data_ptr(), dst.data_ptr(), src.numel(), _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return dst


def spinner_code_bytes(m: int) -> int:
    return int(lib.spinner_code_bytes(int(m)))


def spinner_codes_workspace_bytes(n: int, batch: int) -> int:
    return int(lib.spinner_codes_workspace_bytes(int(n), int(batch)))


def spinner_code_position(coordinate: int):
    """(word, bit) of a coordinate inside a row of sign codes."""
    w, b = ctypes.c_int(), ctypes.c_int()
    rc = lib.spinner_code_position(int(coordinate), ctypes.byref(w), ctypes.byref(b))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return w.value, b.value


def _codes_out(x, m, codes, stream):
    batch = x.shape[0]
    nbytes = spinner_code_bytes(m)
    if nbytes == 0:
        raise SpinnerError(SPINNER_ERR_BAD_M)
    if codes is None:
        codes = _new((batch, nbytes // 8), torch.int64, x.device, stream)
    else:
        _check_tensor(codes, "codes", torch.int64)
        if codes.numel() != batch * (nbytes // 8):
            raise ValueError("codes has the wrong size")
    return codes


def _codes_workspace(x, workspace, stream):
    batch, n = x.shape
    need = spinner_codes_workspace_bytes(n, batch)
    if need and workspace is None:
        workspace = _new(need, torch.uint8, x.device, stream, scratch=True)
    _check_workspace(workspace, need)
    return workspace


def spinner_sign_codes(x, d1, d2, d3, m=None, codes=None, workspace=None, stream=None):
    """Sign bits of the first m coordinates of H D3 H D2 H D1 x, int64 CUDA tensor [batch][m/64]."""
    r = _native.sign_codes(x, d1, d2, d3, m, codes, workspace, stream)
    if r is not None:
        return r
    _check_tensor(x, "x", torch.float32)
    batch, n = x.shape
    _check_diagonals(n, d1=d1, d2=d2, d3=d3)
    m = n if m is None else int(m)
    codes = _codes_out(x, m, codes, stream)
    workspace = _codes_workspace(x, workspace, stream)
    rc = lib.spinner_sign_codes(x.data_ptr(), n, batch, d1.data_ptr(), d2.data_ptr(), d3.data_ptr(), m, codes.data_ptr(),
                                workspace.data_ptr() if workspace is not None else None, _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return codes


def spinner_sign_codes_signs(x, signs, m=None, codes=None, workspace=None, stream=None, triple=0):
    """spinner_sign_codes for +-1 diagonals given as packed sign words (see spinner_pack_signs)."""
    r = _native.sign_codes_signs(x, signs, m, codes, workspace, stream, triple)
    if r is not None:
        return r
    _check_tensor(x, "x", torch.float32)
    batch, n = x.shape
    m = n if m is None else int(m)
    codes = _codes_out(x, m, codes, stream)
    workspace = _codes_workspace(x, workspace, stream)
    one = spinner_signs_bytes(n, 1)
    _check_signs(signs, n, 1, triple)
    rc = lib.spinner_sign_codes_signs(x.data_ptr(), n, batch, signs.data_ptr() + triple * one, m, codes.data_ptr(),
                                      workspace.data_ptr() if workspace is not None else None, _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return codes


def spinner_angular_gram(codes_a, codes_b, m, out=None, stream=None):
    """out[i][j] = 1 - Hamming(codes_a[i], codes_b[j]) / m, fp32 CUDA tensor [na][nb]."""
    r = _native.angular_gram(codes_a, codes_b, m, out, stream)
    if r is not None:
        return r
    _check_tensor(codes_a, "codes_a", torch.int64)
    _check_tensor(codes_b, "codes_b", torch.int64)
    words = spinner_code_bytes(m) // 8
    if words == 0:
        raise SpinnerError(SPINNER_ERR_BAD_M)
    if codes_a.shape[-1] != words or codes_b.shape[-1] != words:
        raise ValueError("codes do not have m / 64 words per row")
    na, nb = codes_a.shape[0], codes_b.shape[0]
    if codes_a.numel() < na * words or codes_b.numel() < nb * words:
        raise ValueError("codes do not have m / 64 words per row")
    if out is None:
        out = _new((na, nb), torch.float32, codes_a.device, stream)
    else:
        _check_tensor(out, "out", torch.float32)
        if out.numel() != na * nb:
            raise ValueError("out has the wrong size")
    rc = lib.spinner_angular_gram(codes_a.data_ptr(), na, codes_b.data_ptr(), nb, int(m), out.data_ptr(),
                                  _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out


def spinner_layer_saved_bytes(n: int, batch: int) -> int:
    return int(lib.spinner_layer_saved_bytes(int(n), int(batch)))


def spinner_layer_workspace_bytes(n: int, batch: int) -> int:
    return _layer_workspace_bytes(int(n), int(batch))


def spinner_layer_forward(x, d1, d2, d3, scale=1.0, y=None, saved=None, stream=None):
    """y = scale * H D3 H D2 H D1 x and the opaque activations the backward pass needs: returns (y, saved)."""
    r = _native.layer_forward(x, d1, d2, d3, scale, y, saved, stream)
    if r is not None:
        return r
    _check_tensor(x, "x", torch.float32)
    batch, n = x.shape
    _check_diagonals(n, d1=d1, d2=d2, d3=d3)
    if y is None:
        y = _new(x.shape, torch.float32, x.device, stream)
    else:
        _check_tensor(y, "y", torch.float32)
        _check_result(y, "y", batch * n)
    if saved is None:
        saved = _new((2, batch, n), torch.float32, x.device, stream)
    else:
        _check_tensor(saved, "saved", torch.float32)
        if saved.numel() != 2 * batch * n:
            raise ValueError("saved has the wrong size")
    rc = lib.spinner_layer_forward(x.data_ptr(), n, batch, d1.data_ptr(), d2.data_ptr(), d3.data_ptr(),
                                   ctypes.c_float(scale), y.data_ptr(), saved.data_ptr(), _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return y, saved


def spinner_layer_backward(dy, x, saved, d1, d2, d3, scale=1.0, dx=None, dd=None, workspace=None, stream=None):
    """Gradients for x ([batch][n]) and for the three diagonals ([3][n], summed over the batch): returns (dx, dd)."""
    r = _native.layer_backward(dy, x, saved, d1, d2, d3, scale, dx, dd, workspace, stream)
    if r is not None:
        return r
    for name, t in (("dy", dy), ("x", x), ("saved", saved)):
        _check_tensor(t, name, torch.float32)
    batch, n = x.shape
    _check_diagonals(n, d1=d1, d2=d2, d3=d3)
    if dy.shape != x.shape or saved.numel() != 2 * batch * n:
        raise ValueError("dy / saved do not match x")
    if dx is None:
        dx = _new(x.shape, torch.float32, x.device, stream)
    else:
        _check_result(dx, "dx", batch * n)
    if dd is None:
        dd = _new((3, n), torch.float32, x.device, stream)
    else:
        _check_result(dd, "dd", 3 * n)
    need = spinner_layer_workspace_bytes(n, batch)
    if workspace is None:
        workspace = _new(max(need, 16), torch.uint8, x.device, stream, scratch=True)
    _check_workspace(workspace, need)
    rc = lib.spinner_layer_backward(dy.data_ptr(), x.data_ptr(), saved.data_ptr(), n, batch, d1.data_ptr(), d2.data_ptr(),
                                    d3.data_ptr(), ctypes.c_float(scale), dx.data_ptr(), dd.data_ptr(), workspace.data_ptr(),
                                    _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return dx, dd


def spinner_sketch_workspace_bytes(n: int, d: int, m: int) -> int:
    return int(lib.spinner_sketch_workspace_bytes(int(n), int(d), int(m)))


def spinner_sketch(A, w, d1, d2, d3, m, scale=1.0, out=None, workspace=None, stream=None):
    """B = scale * (first m rows of H D3 H D2 H D1) diag(w) A for A fp32 [n][d]; w may be None.  Returns B [m][d]."""
    r = _native.sketch(A, w, d1, d2, d3, m, scale, out, workspace, stream)
    if r is not None:
        return r
    _check_tensor(A, "A", torch.float32)
    n, d = A.shape
    _check_diagonals(n, d1=d1, d2=d2, d3=d3)
    if w is not None:
        _check_diagonals(n, w=w)
    if out is None:
        out = _new((int(m), d), torch.float32, A.device, stream)
    else:
        _check_tensor(out, "out", torch.float32)
        if out.numel() != int(m) * d:
            raise ValueError("out has the wrong size")
    need = spinner_sketch_workspace_bytes(n, d, m)
    if workspace is None:
        workspace = _new(max(need, 16), torch.uint8, A.device, stream, scratch=True)
    _check_workspace(workspace, need)
    rc = lib.spinner_sketch(A.data_ptr(), n, d, w.data_ptr() if w is not None else None, d1.data_ptr(), d2.data_ptr(),
                            d3.data_ptr(), int(m), ctypes.c_float(scale), out.data_ptr(), workspace.data_ptr(),
                            _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out


def spinner_sketch_gram_static_limit() -> int:
    return int(lib.spinner_sketch_gram_static_limit())


def spinner_sketch_gram_static(B, out, stream=None):
    """G = B^T B into the caller's `out` [d][d]; the call allocates nothing (the library's built-in scratch)."""
    _check_tensor(B, "B", torch.float32)
    _check_tensor(out, "out", torch.float32)
    m, d = B.shape
    if out.numel() != d * d:
        raise ValueError("out has the wrong size")
    rc = lib.spinner_sketch_gram_static(B.data_ptr(), m, d, out.data_ptr(), _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out


def spinner_sketch_gram_workspace_bytes(m: int, d: int) -> int:
    return int(lib.spinner_sketch_gram_workspace_bytes(int(m), int(d)))


def spinner_sketch_gram(B, out=None, workspace=None, stream=None):
    """G = B^T B, fp32 CUDA tensor [d][d]."""
    r = _native.sketch_gram(B, out, workspace, stream)
    if r is not None:
        return r
    _check_tensor(B, "B", torch.float32)
    m, d = B.shape
    if out is None:
        out = _new((d, d), torch.float32, B.device, stream)
    else:
        _check_tensor(out, "out", torch.float32)
        if out.numel() != d * d:
            raise ValueError("out has the wrong size")
    need = spinner_sketch_gram_workspace_bytes(m, d)
    if need and workspace is None:
        workspace = _new(need, torch.uint8, B.device, stream, scratch=True)
    _check_workspace(workspace, need)
    rc = lib.spinner_sketch_gram(B.data_ptr(), m, d, out.data_ptr(), workspace.data_ptr() if workspace is not None else None,
                                 _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out


def spinner_apply_blocks(x, diag_sets, m=None, epilogue="none", scale=1.0, out=None, workspace=None, stream=None):
    """L independent triples (diag_sets fp32 [L][3][n]) applied to the same x, their m-row blocks side by side:
    out [batch][L m] (epilogue none) or [batch][2 L m] (cos block | sin block)."""
    r = _native.apply_blocks(x, diag_sets, m, epilogue, scale, out, workspace, stream)
    if r is not None:
        return r
    _check_tensor(x, "x", torch.float32)
    _check_tensor(diag_sets, "diag_sets", torch.float32)
    batch, n = x.shape
    if diag_sets.dim() != 3 or diag_sets.shape[1] != 3 or diag_sets.shape[2] != n:
        raise ValueError("diag_sets must be [L][3][n]")
    L = diag_sets.shape[0]
    m = n if m is None else int(m)
    epi = _epi(epilogue)
    width = (2 * m if epi == SPINNER_EPI_COSSIN else m) * L
    if out is None:
        out = _new((batch, width), torch.float32, x.device, stream)
    else:
        _check_tensor(out, "out", torch.float32)
        if out.numel() != batch * width:
            raise ValueError("out has the wrong size")
    need = int(lib.spinner_blocks_workspace_bytes(n, batch, m, epi))
    if need and workspace is None:
        workspace = _new(need, torch.uint8, x.device, stream, scratch=True)
    _check_workspace(workspace, need)
    rc = lib.spinner_apply_blocks(x.data_ptr(), n, batch, L, diag_sets.data_ptr(), m, epi, ctypes.c_float(scale),
                                  out.data_ptr(), workspace.data_ptr() if workspace is not None else None,
                                  _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out


def spinner_struct_prepare(kind, params, n, stream=None):
    """Opaque spectrum (uint8 CUDA tensor) of a structured third block from its generating vector (fp32 CUDA tensor)."""
    k = STRUCT_KINDS[kind] if isinstance(kind, str) else int(kind)
    _check_tensor(params, "params", torch.float32)
    nbytes = int(lib.spinner_struct_spectrum_bytes(k, int(n)))
    if nbytes == 0:
        raise SpinnerError(SPINNER_ERR_UNSUPPORTED)
    if params.numel() != int(lib.spinner_struct_params(k, int(n))):
        raise ValueError("generating vector has the wrong length")
    spec = _new(nbytes, torch.uint8, params.device, stream)
    rc = lib.spinner_struct_prepare(k, params.data_ptr(), int(n), spec.data_ptr(), _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return spec


def _check_spectrum(spectrum, k, n):
    _check_device(spectrum, "spectrum")
    if spectrum.numel() * spectrum.element_size() < int(lib.spinner_struct_spectrum_bytes(k, n)):
        raise ValueError("spectrum of another kind or a smaller n")


def spinner_struct_apply(x, kind, spectrum, d1, d2, m=None, scale=1.0, out=None, stream=None):
    """out [batch][m] = scale * (first m rows of G_struct D2 H D1 x)."""
    k = STRUCT_KINDS[kind] if isinstance(kind, str) else int(kind)
    _check_tensor(x, "x", torch.float32)
    batch, n = x.shape
    _check_diagonals(n, d1=d1, d2=d2)
    _check_spectrum(spectrum, k, n)
    m = n if m is None else int(m)
    if out is None:
        out = _new((batch, m), torch.float32, x.device, stream)
    else:
        _check_tensor(out, "out", torch.float32)
        if out.numel() != batch * m:
            raise ValueError("out has the wrong size")
    rc = lib.spinner_struct_apply(x.data_ptr(), n, batch, k, spectrum.data_ptr(), d1.data_ptr(), d2.data_ptr(), m,
                                  ctypes.c_float(scale), out.data_ptr(), _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out


def spinner_struct_workspace_bytes(kind, n: int, batch: int) -> int:
    k = STRUCT_KINDS[kind] if isinstance(kind, str) else int(kind)
    return int(lib.spinner_struct_workspace_bytes(k, int(n), int(batch)))


def spinner_struct_apply_ws(x, kind, spectrum, d1, d2, m=None, scale=1.0, out=None, workspace=None, stream=None):
    """spinner_struct_apply for every supported n (a workspace tensor is made when none is given and one is needed)."""
    r = _native.struct_apply_ws(x, kind, spectrum, d1, d2, m, scale, out, workspace, stream)
    if r is not None:
        return r
    k = STRUCT_KINDS[kind] if isinstance(kind, str) else int(kind)
    _check_tensor(x, "x", torch.float32)
    batch, n = x.shape
    _check_diagonals(n, d1=d1, d2=d2)
    _check_spectrum(spectrum, k, n)
    m = n if m is None else int(m)
    if out is None:
        out = _new((batch, m), torch.float32, x.device, stream)
    else:
        _check_tensor(out, "out", torch.float32)
        if out.numel() != batch * m:
            raise ValueError("out has the wrong size")
    need = spinner_struct_workspace_bytes(k, n, batch)
    if workspace is None and need:
        workspace = _new(need, torch.uint8, x.device, stream, scratch=True)
    _check_workspace(workspace, need)
    rc = lib.spinner_struct_apply_ws(x.data_ptr(), n, batch, k, spectrum.data_ptr(), d1.data_ptr(), d2.data_ptr(), m,
                                     ctypes.c_float(scale), out.data_ptr(),
                                     workspace.data_ptr() if workspace is not None else None, _stream_handle(stream))
    if rc != SPINNER_OK:
        raise SpinnerError(rc)
    return out


# ------------------------------------------------------------------ 4-bit numbers and products of rows grouped by expert
_native_products = _native._products
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
MX4_BLOCK = 32


def _dtype_code(dtype):
    if dtype not in DTYPES:
        raise SpinnerError(SPINNER_ERR_BAD_TYPE)
    return DTYPES[dtype]


def _fits(*numbers):
    """Whether numbers are as many as the C ABI's int holds; ctypes would cut them off."""
    return all(-1 << 31 <= v < 1 << 31 for v in numbers)


def _check_sizes(*numbers):
    if not _fits(*numbers):
        raise SpinnerError(SPINNER_ERR_BAD_SHAPE)


def _check_here(t, name, dtype=None, dim=None):
    """A tensor of the expected type and number of dimensions on the GPU that the call runs on."""
    if not t.is_cuda or (dtype is not None and t.dtype != dtype) or (dim is not None and t.dim() != dim):
        raise ValueError("%s must be a %s%sCUDA tensor" % (name, "" if dim is None else "%d-dimensional " % dim,
                                                         "" if dtype is None else "%s " % dtype))
    if t.device.index != torch.cuda.current_device():
        raise ValueError("%s must be on the current GPU" % name)


def _check_bytes(t, name, shape):
    _check_here(t, name, torch.uint8)
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError("%s must be contiguous, of shape %s" % (name, tuple(shape)))


def _check_rows(t, name, dtype=None):
    """[rows][numbers], numbers side by side; returns the distance between rows."""
    _check_here(t, name, dtype, 2)
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError("the numbers of a row of %s must lie side by side" % name)
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _new_or_checked(out, name, shape, dtype, like, stream):
    """A result of rows (the caller's may have rows further apart) and the distance between them."""
    if out is None:
        out = _new(shape, dtype, like.device, stream)
    stride = _check_rows(out, name, dtype)
    if tuple(out.shape) != tuple(shape):
        raise ValueError("%s has the wrong size" % name)
    if stride < shape[1]:
        raise ValueError("rows of %s lie over one another" % name)
    return out, stride


def _check_ends(ends, experts, weights):
    """The ends of the experts' rows; None goes with a single weight matrix."""
    if ends is None:
        if experts != 1:
            raise ValueError("ends is needed: %s holds %d experts" % (weights, experts))
        return None
    _check_here(ends, "ends", torch.int64, 1)
    if ends.numel() != experts or not ends.is_contiguous():
        raise ValueError("ends must be contiguous, one number for each of %d experts" % experts)
    return ends.data_ptr()


def _check_weights(w, name):
    """[n][k] or [experts][n][k], contiguous; returns experts, n, k."""
    _check_here(w, name)
    if w.dim() not in (2, 3) or not w.is_contiguous():
        raise ValueError("%s must be a contiguous [n][k] or [experts][n][k] CUDA tensor" % name)
    return (1, *w.shape) if w.dim() == 2 else tuple(w.shape)


def _check_rotation(diag, block, k):
    if diag is None:
        return None
    _check_here(diag, "diag", torch.float32, 1)
    if diag.numel() != k or not diag.is_contiguous():
        raise ValueError("diag must be contiguous, one number for each of %d coordinates" % k)
    return diag.data_ptr()


def _done(rc):
    if rc != SPINNER_OK:
        raise SpinnerError(rc)


def spinner_mx_quantize(x, diag=None, block=0, codes=None, scales=None, stream=None):
    """Rotate runs of ``block`` coordinates (v = H D x, D = diag(diag); block = 0: v = x) and round to microscaled 4-bit numbers.

    x: fp32, bf16 or fp16 CUDA tensor [rows][k], rows any distance apart, k a multiple of 32.  diag: fp32 [k] or None (D = I).
    Returns (codes uint8 [rows][k / 2], scales uint8 [rows][k / 32]); see include/spinner.h for the format.
    """
    r = _native_products.mx_quantize(x, diag, block, codes, scales, stream)
    if r is not None:
        return r
    stride = _check_rows(x, "x")
    rows, k = x.shape
    _check_sizes(k, int(block))
    if codes is None:
        codes = _new((rows, k // 2), torch.uint8, x.device, stream)
    if scales is None:
        scales = _new((rows, k // MX4_BLOCK), torch.uint8, x.device, stream)
    _check_bytes(codes, "codes", (rows, k // 2))
    _check_bytes(scales, "scales", (rows, k // MX4_BLOCK))
    d = _check_rotation(diag, block, k)
    _done(lib.spinner_mx_quantize(x.data_ptr(), _dtype_code(x.dtype), rows, k, stride, d, int(block), codes.data_ptr(), scales.data_ptr(),
                                   _stream_handle(stream)))
    return codes, scales


def spinner_mx_dequantize(codes, scales, dtype=torch.float32, out=None, stream=None):
    """The numbers that 4-bit codes stand for: [rows][k] of ``dtype``."""
    r = _native_products.mx_dequantize(codes, scales, dtype, out, stream)
    if r is not None:
        return r
    _check_here(codes, "codes", torch.uint8, 2)
    rows, k = codes.shape[0], 2 * codes.shape[1]
    _check_sizes(k)
    _check_bytes(codes, "codes", (rows, k // 2))
    _check_bytes(scales, "scales", (rows, k // MX4_BLOCK))
    code = _dtype_code(dtype)
    out, stride = _new_or_checked(out, "out", (rows, k), dtype, codes, stream)
    _done(lib.spinner_mx_dequantize(codes.data_ptr(), scales.data_ptr(), rows, k, out.data_ptr(), code, stride, _stream_handle(stream)))
    return out


def spinner_mx_matmul(a_codes, a_scales, w_codes, w_scales, ends=None, dtype=torch.bfloat16, out=None, stream=None):
    """out = a w^T on 4-bit operands: a [rows][k], w [n][k], or [experts][n][k] with each expert's rows up to its entry of ``ends``.

    codes and scales as spinner_mx_quantize gives them (w's with the experts in front); ends: int64 CUDA tensor [experts],
    cumulative.  Rows from the last end on come out as 0.
    """
    r = _native_products.mx_matmul(a_codes, a_scales, w_codes, w_scales, ends, dtype, out, stream)
    if r is not None:
        return r
    _check_here(a_codes, "a_codes", torch.uint8, 2)
    rows, k = a_codes.shape[0], 2 * a_codes.shape[1]
    _check_bytes(a_codes, "a_codes", (rows, k // 2))
    _check_bytes(a_scales, "a_scales", (rows, k // MX4_BLOCK))
    experts, n, _ = _check_weights(w_codes, "w_codes")
    _check_sizes(k, n, experts)
    _check_bytes(w_codes, "w_codes", (*w_codes.shape[:-1], k // 2))
    _check_bytes(w_scales, "w_scales", (*w_codes.shape[:-1], k // MX4_BLOCK))
    e = _check_ends(ends, experts, "w_codes")
    code = _dtype_code(dtype)
    out, stride = _new_or_checked(out, "out", (rows, n), dtype, a_codes, stream)
    _done(lib.spinner_mx_matmul(a_codes.data_ptr(), a_scales.data_ptr(), rows, k, w_codes.data_ptr(), w_scales.data_ptr(), n, experts, e,
                                 out.data_ptr(), code, stride, _stream_handle(stream)))
    return out


def spinner_mx_linear_workspace_bytes(rows: int, k: int) -> int:
    return int(lib.spinner_mx_linear_workspace_bytes(int(rows), int(k))) if _fits(int(k)) else 0


def spinner_mx_linear(x, w_codes, w_scales, diag=None, block=0, ends=None, out=None, workspace=None, stream=None):
    """A layer with 4-bit weights on plain inputs: spinner_mx_quantize(x, diag, block), then spinner_mx_matmul; out of the type of x.

    The weights are quantised with the same diag and block, which then cancel in the product.  Results have no autograd history, and there is no gradient of this call.
    """
    r = _native_products.mx_linear(x, w_codes, w_scales, diag, block, ends, out, workspace, stream)
    if r is not None:
        return r
    x_stride = _check_rows(x, "x")
    code = _dtype_code(x.dtype)
    rows, k = x.shape
    experts, n, _ = _check_weights(w_codes, "w_codes")
    _check_sizes(k, n, experts, int(block))
    _check_bytes(w_codes, "w_codes", (*w_codes.shape[:-1], k // 2))
    _check_bytes(w_scales, "w_scales", (*w_codes.shape[:-1], k // MX4_BLOCK))
    d = _check_rotation(diag, block, k)
    e = _check_ends(ends, experts, "w_codes")
    out, stride = _new_or_checked(out, "out", (rows, n), x.dtype, x, stream)
    need = spinner_mx_linear_workspace_bytes(rows, k)
    if workspace is None:
        workspace = _new(need, torch.uint8, x.device, stream, scratch=True)
    _check_workspace(workspace, need)
    _done(lib.spinner_mx_linear(x.data_ptr(), code, rows, k, x_stride, d, int(block), w_codes.data_ptr(), w_scales.data_ptr(), n, experts, e,
                                 out.data_ptr(), stride, workspace.data_ptr(), _stream_handle(stream)))
    return out


def _grouped(call, a, w, ends, out, stream, across):
    a_stride = _check_rows(a, "x" if across else "dy")
    code = _dtype_code(a.dtype)
    experts, n, k = _check_weights(w, "w")
    _check_sizes(experts, n, k)
    if w.dtype != a.dtype or a.shape[1] != (k if across else n):
        raise ValueError("w must be of the type and width of the rows")
    e = _check_ends(ends, experts, "w")
    out, stride = _new_or_checked(out, "out" if across else "dx", (a.shape[0], n if across else k), a.dtype, a, stream)
    depth, width = (k, n) if across else (n, k)
    _done(call(a.data_ptr(), code, a.shape[0], depth, a_stride, w.data_ptr(), width, experts, e, out.data_ptr(), stride, _stream_handle(stream)))
    return out


def spinner_grouped_matmul(x, w, ends=None, out=None, stream=None):
    """out = x w^T of each expert's rows with its own weights: x bf16 or fp16 [rows][k], w [experts][n][k] (or [n][k] without ends).

    ends: int64 CUDA tensor [experts]; the rows of expert e are ends[e - 1] .. ends[e].  Rows from the last end on come out as 0.
    As everywhere here, results have no autograd history: the gradients are spinner_grouped_matmul_dx and spinner_grouped_matmul_dw.
    """
    r = _native_products.grouped_matmul(x, w, ends, out, stream)
    return r if r is not None else _grouped(lib.spinner_grouped_matmul, x, w, ends, out, stream, True)


def spinner_grouped_matmul_dx(dy, w, ends=None, dx=None, stream=None):
    """Gradient of spinner_grouped_matmul with respect to x: dx = dy w of each expert's rows."""
    r = _native_products.grouped_matmul_dx(dy, w, ends, dx, stream)
    return r if r is not None else _grouped(lib.spinner_grouped_matmul_dx, dy, w, ends, dx, stream, False)


def spinner_grouped_matmul_dw_workspace_bytes(rows: int, n: int, k: int, experts: int) -> int:
    return int(lib.spinner_grouped_matmul_dw_workspace_bytes(int(rows), int(n), int(k), int(experts))) if _fits(int(n), int(k), int(experts)) else 0


def spinner_grouped_matmul_dw(dy, x, ends=None, dtype=torch.float32, dw=None, workspace=None, stream=None):
    """Gradient with respect to w: dw = dy^T x over each expert's rows, [experts][n][k] ([n][k] without ends).

    dtype: fp32, or the type of dy and x.  Experts without rows get zeros.
    """
    r = _native_products.grouped_matmul_dw(dy, x, ends, dtype, dw, workspace, stream)
    if r is not None:
        return r
    dy_stride, x_stride = _check_rows(dy, "dy"), _check_rows(x, "x", dy.dtype)
    code, dw_code = _dtype_code(dy.dtype), _dtype_code(dtype)
    rows, n, k = dy.shape[0], dy.shape[1], x.shape[1]
    if x.shape[0] != rows:
        raise ValueError("dy and x must have as many rows")
    experts = 1 if ends is None else ends.numel()
    _check_sizes(n, k, experts)
    e = _check_ends(ends, experts, "dw")
    shape = (n, k) if ends is None else (experts, n, k)
    if dw is None:
        dw = _new(shape, dtype, dy.device, stream)
    _check_here(dw, "dw", dtype)
    if tuple(dw.shape) != shape or not dw.is_contiguous():
        raise ValueError("dw must be contiguous, of shape %s" % (shape,))
    need = spinner_grouped_matmul_dw_workspace_bytes(rows, n, k, experts)
    if need and workspace is None:
        workspace = _new(need, torch.uint8, dy.device, stream, scratch=True)
    _check_workspace(workspace, need)
    _done(lib.spinner_grouped_matmul_dw(dy.data_ptr(), x.data_ptr(), code, rows, n, k, dy_stride, x_stride, experts, e, dw.data_ptr(), dw_code,
                                        workspace.data_ptr() if workspace is not None else None, _stream_handle(stream)))
    return dw
