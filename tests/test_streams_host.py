"""Where the memory comes from that a call makes for itself when it is given a stream: from that stream, whatever the current one has queued
on blocks that it let go of.  On the host, with tensors that are only described and a library that launches nothing."""
import pytest

from test_abi_host import _NoLaunch, _Tensor

MINE = type("Stream", (), {"cuda_stream": 4096})()
CURRENT = type("Stream", (), {"cuda_stream": 0})()


class _OnGpu(_Tensor):
    def __init__(self, *shape, dtype="float32", made_on=None):
        import torch

        super().__init__(*shape, dtype=dtype)
        self.device, self.made_on, self.used_on = torch.device("cuda:0"), made_on, []

    def stride(self, i):
        return 1 if i else self.shape[1]

    def untyped_storage(self):
        return type("Storage", (), {"nbytes": lambda _, n=self.numel() * self.element_size(): n})()

    def record_stream(self, stream):
        self.used_on.append(stream)


@pytest.fixture
def made(monkeypatch):
    """Every tensor that is made, with the stream whose memory it is; the binding without launches."""
    import torch

    from paper_1610_06209_amd import binding as b

    tensors = []

    def empty(*shape, dtype=torch.float32, device=None):
        shape = shape[0] if len(shape) == 1 and not isinstance(shape[0], int) else shape
        tensors.append(_OnGpu(*shape, dtype=str(dtype)[6:], made_on=CURRENT))
        return tensors[-1]

    def new_on(shape, dtype, device, handle, scratch):
        assert device == 0 and handle == MINE.cuda_stream
        t = empty(shape, dtype=dtype)
        t.made_on = MINE
        if not scratch:
            t.record_stream(CURRENT)
        return t

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(b, "_new_on", new_on)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(b, "lib", _NoLaunch(b.lib))
    monkeypatch.setattr(b, "_stream_handle", lambda stream: (stream or CURRENT).cuda_stream)
    return b, tensors


T, u8, h = _OnGpu, dict(dtype="uint8"), dict(dtype="bfloat16")
CALLS = {
    "spinner_mx_quantize": dict(x=T(5, 128)),
    "spinner_mx_dequantize": dict(codes=T(5, 64, **u8), scales=T(5, 4, **u8)),
    "spinner_mx_matmul": dict(a_codes=T(5, 64, **u8), a_scales=T(5, 4, **u8), w_codes=T(7, 64, **u8), w_scales=T(7, 4, **u8)),
    "spinner_mx_linear": dict(x=T(5, 128, **h), w_codes=T(7, 64, **u8), w_scales=T(7, 4, **u8)),
    "spinner_grouped_matmul": dict(x=T(5, 128, **h), w=T(7, 128, **h)),
    "spinner_grouped_matmul_dx": dict(dy=T(5, 7, **h), w=T(7, 128, **h)),
    "spinner_grouped_matmul_dw": dict(dy=T(4100, 40, **h), x=T(4100, 264, **h)),           # (sums in shares: with a workspace)
}
# the other entry points, at sizes where they make scratch memory if they ever do
_n, _wide, _d3 = 1 << 15, 1 << 17, lambda n: dict(d1=T(n), d2=T(n), d3=T(n))              # noqa: E731
_signs = lambda n, L: T(1 << 20, **u8)                                                    # noqa: E731
CALLS.update({
    "spinner_apply": dict(x=T(3, _wide), m=100, **_d3(_wide)),
    "spinner_apply_signs": dict(x=T(3, _wide), signs=_signs(_wide, 1), m=100),
    "spinner_apply_blocks": dict(x=T(3, _wide), diag_sets=T(2, 3, _wide), m=100),
    "spinner_pack_signs": dict(diag_sets=T(2, 3, _n)),
    "spinner_hash": dict(x=T(3, _n), diag_sets=T(2, 3, _n)),
    "spinner_hash_signs": dict(x=T(3, _n), signs=_signs(_n, 2), L=2),
    "spinner_hash_ws": dict(x=T(3, _wide), diag_sets=T(2, 3, _wide)),
    "spinner_hash_signs_ws": dict(x=T(3, _wide), signs=_signs(_wide, 2), L=2),
    "spinner_sign_codes": dict(x=T(3, _wide), **_d3(_wide)),
    "spinner_sign_codes_signs": dict(x=T(3, _wide), signs=_signs(_wide, 1)),
    "spinner_angular_gram": dict(codes_a=T(5, 4, dtype="int64"), codes_b=T(3, 4, dtype="int64"), m=256),
    "spinner_layer_forward": dict(x=T(3, _n), **_d3(_n)),
    "spinner_layer_backward": dict(dy=T(3, _n), x=T(3, _n), saved=T(2, 3, _n), **_d3(_n)),
    "spinner_sketch": dict(A=T(_n, 20), w=None, m=64, **_d3(_n)),
    "spinner_sketch_gram": dict(B=T(4096, 200)),
    "spinner_struct_prepare": dict(kind="circulant", params=T(_n), n=_n),
    "spinner_struct_apply": dict(x=T(3, 1 << 12), kind="circulant", spectrum=_signs(0, 0), d1=T(1 << 12), d2=T(1 << 12)),
    "spinner_struct_apply_ws": dict(x=T(3, _n), kind="circulant", spectrum=_signs(0, 0), d1=T(_n), d2=T(_n)),
})
# tensors made and not returned
SCRATCH = {name: 1 for name in ("spinner_mx_linear", "spinner_grouped_matmul_dw", "spinner_apply", "spinner_apply_signs", "spinner_apply_blocks", "spinner_hash_ws",
                                "spinner_hash_signs_ws", "spinner_sign_codes", "spinner_sign_codes_signs", "spinner_layer_backward", "spinner_sketch", "spinner_sketch_gram",
                                "spinner_struct_apply_ws")}


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_comes_from_the_stream_of_the_call(made, name):
    b, tensors = made
    r = getattr(b, name)(stream=MINE, **CALLS[name])
    results = r if isinstance(r, tuple) else (r,)
    assert tensors and all(t.made_on is MINE for t in tensors)
    assert len(tensors) == len(results) + SCRATCH.get(name, 0)
    # results are used by the caller afterwards, on the stream that is current there
    assert all(t.used_on == ([CURRENT] if any(t is q for q in results) else []) for t in tensors)


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_of_other_calls_comes_from_the_current_stream(made, name):
    b, tensors = made
    getattr(b, name)(**CALLS[name])
    assert tensors and all(t.made_on is CURRENT and not t.used_on for t in tensors)


@pytest.mark.parametrize("name", list(CALLS))
def test_the_current_stream_given_is_the_current_stream(made, name):
    b, tensors = made
    getattr(b, name)(stream=type("Stream", (), {"cuda_stream": CURRENT.cuda_stream})(), **CALLS[name])
    assert tensors and all(t.made_on is CURRENT and not t.used_on for t in tensors)
