"""The native form of the 8-bit calls: what it takes gives what the Python form gives, bit for bit; what the Python form refuses it
leaves alone or refuses alike."""
import ctypes

import pytest
import torch

import int8_cases as ic
from test_gpu_native import PythonOnly, flat, others

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def layer(gpu_api):
    gpu_api._fast()
    T, d_in, d_out = 24, 256, 128
    gen = torch.Generator("cuda").manual_seed(4)
    rand = lambda *n: torch.randn(n, device="cuda", generator=gen)  # noqa: E731
    codes, scale = ic.drawn_weight(5, d_in, d_out)
    L = dict(w=(codes.cuda(), scale.cuda()), x=rand(T, d_in).to(BF16), dy=rand(T, d_out).to(BF16), gu=rand(T, 2 * d_out).to(BF16),
             bias=rand(d_out), mul=rand(T, d_out).to(BF16), res=rand(T, d_out), res_in=rand(T, d_in), factor=rand(d_in).abs())
    L["tokens8"] = gpu_api.quantize_tokens(L["x"])
    L["z8"], L["mul8"] = gpu_api.keep8(L["dy"]), gpu_api.keep8(L["mul"])
    L["kept"] = gpu_api.swiglu_forward_keep8(L["gu"], d_out)[1]
    return L


def calls(api, L):
    """name -> (function, its positional arguments, the place of `act`)"""
    w, N = L["w"], None
    return {
        "quantize_tokens": (api.quantize_tokens, (L["x"], L["factor"], N, N), N),
        "forward_int8": (api.forward_int8, (L["x"], *w, L["bias"], "silu", L["mul"], L["res"], True, F32, N, N, N), 4),
        "forward_int8 tokens": (api.forward_int8, (L["tokens8"], *w, N, "gelu", N, L["res"].to(BF16), False, BF16, N, N, N), 4),
        "backward_int8": (api.backward_int8, (L["dy"], *w, L["res_in"], F32, N, N), N),
        "backward_int8 bf16": (api.backward_int8, (L["dy"], *w, N, BF16, N, N), N),
        "keep8": (api.keep8, (L["x"], N), N),
        "swiglu_forward_keep8": (api.swiglu_forward_keep8, (L["gu"], 128, N, N), N),
        "swiglu_forward_int8": (api.swiglu_forward_int8, (L["gu"], 128, True, N, N, N, N), N),
        "swiglu_forward_int8 only": (api.swiglu_forward_int8, (L["gu"], 128, False, N, N, N, N), N),
        "swiglu_backward_kept8": (api.swiglu_backward_kept8, (L["dy"], L["kept"], 128, N), N),
        "epilogue_backward_kept8": (api.epilogue_backward_kept8, (L["dy"], L["z8"], "silu", L["mul8"], True, True, N, N, N, False, N), 2),
        "epilogue_backward_kept8 fp32": (api.epilogue_backward_kept8, (L["res"], L["z8"], "gelu", N, True, True, N, N, L["bias"].clone(),
                                                                       True, N), 2),
    }


CALLS = ["quantize_tokens", "forward_int8", "forward_int8 tokens", "backward_int8", "backward_int8 bf16", "keep8", "swiglu_forward_keep8",
         "swiglu_forward_int8", "swiglu_forward_int8 only", "swiglu_backward_kept8", "epilogue_backward_kept8",
         "epilogue_backward_kept8 fp32"]


def native(api, name, args, at):
    if at is not None:
        args = (*args[:at], api.ACTIVATIONS.get(args[at]) if isinstance(args[at], str) else args[at], *args[at + 1:])
    return getattr(api._native, name.split()[0])(*args)


def equal(a, b):
    a, b = flat(a), flat(b)
    assert len(a) == len(b) > 0
    for s, t in zip(a, b):
        assert s.dtype == t.dtype and s.shape == t.shape
        if s.dtype != torch.uint8:   # (kept bytes: some between the codes and the exponents, and the last, are nobody's)
            ic.same(s, t)            # (what was kept, read as of fewer rows, holds NaN)


@pytest.mark.parametrize("name", CALLS)
def test_same_results(gpu_api, layer, monkeypatch, name):
    fn, args, at = calls(gpu_api, layer)[name]
    got = native(gpu_api, name, args, at)
    assert got is not None
    fn, args, at = calls(gpu_api, layer)[name]
    monkeypatch.setattr(gpu_api, "_native", PythonOnly())
    equal(got, fn(*args))


def changed(v):
    if isinstance(v, tuple):   # (q, s)
        yield from ((), v[:1], v * 2, list(v), v[::-1], None)
        for k in range(2):
            for o in others(v[k]):
                yield (*v[:k], o, *v[k + 1:])
    else:
        yield from others(v)


@pytest.mark.parametrize("name", CALLS)
def test_the_same_calls_are_refused(gpu_api, layer, monkeypatch, name):
    def outcome(python, i, k):
        fn, args, at = calls(gpu_api, layer)[name]
        args = (*args[:i], list(changed(args[i]))[k], *args[i + 1:])
        with monkeypatch.context() as m:
            if python:
                m.setattr(gpu_api, "_native", PythonOnly())
            try:
                return fn(*args) if python else native(gpu_api, name, args, at)
            except gpu_api.QaloraError as e:
                return str(e)
            except (ValueError, TypeError, AttributeError, RuntimeError, IndexError, OverflowError, ctypes.ArgumentError) as e:
                return e
    _, args, at = calls(gpu_api, layer)[name]
    left = 0
    for i in range(len(args)):
        for k in range(len(list(changed(args[i])))):
            got, python = outcome(False, i, k), outcome(True, i, k)
            if got is None:
                left += 1
            elif isinstance(got, str):
                assert got == python, (i, k)
            else:
                assert not isinstance(got, Exception) and not isinstance(python, (str, Exception)), (i, k, got, python)
                equal(got, python)
    assert left > 0
    if at is not None:
        assert native(gpu_api, name, (*args[:at], "tanh", *args[at + 1:]), at) is None


def test_given_outputs_are_used_and_returned(gpu_api, layer):
    L, w = layer, layer["w"]
    q, s = torch.empty((24, 256), dtype=torch.int8, device="cuda"), torch.empty(24, device="cuda")
    out = gpu_api.quantize_tokens(L["x"], q=q, s=s)
    assert out[0] is q and out[1] is s
    y, z = torch.empty((24, 128), device="cuda"), torch.empty((24, 128), dtype=BF16, device="cuda")
    ws = torch.empty(gpu_api.int8_workspace_bytes(24, 256, 128, gpu_api.OP_FORWARD), dtype=torch.uint8, device="cuda")
    out = gpu_api.forward_int8((q, s), *w, keep_z=True, y=y, z=z, ws=ws)
    assert out[0] is y and out[1] is z
    dx = torch.empty((24, 256), dtype=BF16, device="cuda")
    assert gpu_api.backward_int8(z, *w, dx=dx) is dx
    kept = torch.empty(gpu_api.kept8_bytes(48, 128), dtype=torch.uint8, device="cuda")
    h = torch.empty((24, 128), dtype=BF16, device="cuda")
    out = gpu_api.swiglu_forward_keep8(L["gu"], 128, h=h, kept=kept)
    assert out[0] is h and out[1] is kept
    q, s = torch.empty((24, 128), dtype=torch.int8, device="cuda"), torch.empty(24, device="cuda")
    out = gpu_api.swiglu_forward_int8(L["gu"], 128, keep=True, q=q, s=s, kept=kept, h=h)
    assert out[0][0] is q and out[0][1] is s and out[1] is kept
    dgu = torch.empty((24, 256), dtype=BF16, device="cuda")
    assert gpu_api.swiglu_backward_kept8(h, kept, 128, dgu=dgu) is dgu
    with pytest.raises(ValueError, match="kept"):
        gpu_api.swiglu_forward_int8(L["gu"], 128, kept=kept)
    with pytest.raises(ValueError, match="z"):
        gpu_api.forward_int8(L["x"], *w, z=z)
    with pytest.raises(ValueError, match="act"):
        gpu_api.forward_int8(L["x"], *w, act="tanh")
