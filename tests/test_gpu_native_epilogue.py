"""The native form of the epilogue's calls and of the orthogonalised step: what it takes gives what the Python form gives, bit
for bit; what the Python form refuses it leaves alone or refuses alike."""
import ctypes

import pytest
import torch

from helpers import layer_on_gpu
from paper_2309_14717_amd import synth
from test_gpu_native import PythonOnly, others, same

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def layer(gpu_api):
    gpu_api._fast()
    L = layer_on_gpu(gpu_api, synth.LayerConfig("native_epi", 24, 512, 256, 4, 32, 8, 0.5, seed=102))
    L["w"] = (L["packed"], L["g_alpha"], L["g_beta"])
    L["deployed"] = gpu_api.deploy(L["desc"], *L["w"])
    gen = torch.Generator("cuda").manual_seed(4)
    rand = lambda *n: torch.randn(n, device="cuda", generator=gen)  # noqa: E731
    L["bias"], L["mul"], L["res"], L["z"] = rand(256), rand(24, 256).to(BF), rand(24, 256), rand(24, 256).to(BF)
    return L


def calls(api, L):
    """name -> (function, its positional arguments, the place of `act`)"""
    d, x, w, N = L["desc"], L["x"], L["w"], None
    return {
        "forward_epilogue": (api.forward_epilogue, (d, x, *w, L["A"], L["B"], L["bias"], "silu", L["mul"], L["res"], True, True,
                                                    torch.float32, N, N, N, N), 8),
        "forward_epilogue merged": (api.forward_epilogue, (d, x, *w, N, N, L["bias"], "gelu", N, L["res"].to(BF), False, False, BF,
                                                           N, N, N, N), 8),
        "forward_deployed_epilogue": (api.forward_deployed_epilogue, (d, x, L["deployed"], L["packed"], L["bias"], "relu",
                                                                      L["mul"], L["res"], torch.float32, N, N), 5),
        "epilogue_backward": (api.epilogue_backward, (L["dy"], L["z"], "gelu_tanh", L["mul"], True, True, N, N, N, False, N), 2),
        "epilogue_backward fp32": (api.epilogue_backward, (L["res"], L["z"], "silu", N, True, True, N, N, L["bias"].clone(), True,
                                                           N), 2),
    }


CALLS = ["forward_epilogue", "forward_epilogue merged", "forward_deployed_epilogue", "epilogue_backward", "epilogue_backward fp32"]


def native(api, name, args, at):
    args = (*args[:at], api.ACTIVATIONS.get(args[at]) if isinstance(args[at], str) else args[at], *args[at + 1:])
    return getattr(api._native, name.split()[0])(*args)


def compared(name, a, b):
    if name == "forward_epilogue":   # (the kept bytes are the library's own, and not all written)
        a, b = a[:2], b[:2]
    same("", a, b)


@pytest.mark.parametrize("name", CALLS)
def test_same_results(gpu_api, layer, monkeypatch, name):
    fn, args, at = calls(gpu_api, layer)[name]
    got = native(gpu_api, name, args, at)
    fn, args, at = calls(gpu_api, layer)[name]
    monkeypatch.setattr(gpu_api, "_native", PythonOnly())
    compared(name, got, fn(*args))


@pytest.mark.parametrize("name", CALLS)
def test_the_same_calls_are_refused(gpu_api, layer, monkeypatch, name):
    def outcome(python, i, k):
        fn, args, at = calls(gpu_api, layer)[name]
        args = (*args[:i], list(others(args[i]))[k], *args[i + 1:])
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
        for k in range(len(list(others(args[i])))):
            got, python = outcome(False, i, k), outcome(True, i, k)
            if got is None:
                left += 1
            elif isinstance(got, str):
                assert got == python, (i, k)
            else:
                assert not isinstance(got, Exception) and not isinstance(python, (str, Exception)), (i, k, got, python)
                compared(name, got, python)
    assert left > 0
    assert native(gpu_api, name, (*args[:at], "tanh", *args[at + 1:]), at) is None


def test_given_outputs_are_used_and_returned(gpu_api, layer):
    L = layer
    y, z = torch.empty(24, 256, device="cuda"), torch.empty(24, 256, device="cuda", dtype=BF)
    kept = torch.empty(gpu_api.kept_bytes(L["desc"], 24), dtype=torch.uint8, device="cuda")
    ws = torch.empty(gpu_api.workspace_bytes(L["desc"], 24, gpu_api.OP_FORWARD), dtype=torch.uint8, device="cuda")
    out = gpu_api.forward_epilogue(L["desc"], L["x"], *L["w"], L["A"], L["B"], keep_z=True, keep=True, y=y, z=z, kept=kept, ws=ws)
    assert out[0] is y and out[1] is z and out[2] is kept
    dz, dmul, dbias = torch.empty_like(z), torch.empty_like(z), torch.zeros(256, device="cuda")
    out = gpu_api.epilogue_backward(L["dy"], z, "silu", mul=L["mul"], dz=dz, dmul=dmul, dbias=dbias, ws=ws)
    assert out[0] is dz and out[1] is dmul and out[2] is dbias and dbias.abs().sum() > 0


def test_muon(gpu_api, monkeypatch):
    gen = torch.Generator("cuda").manual_seed(5)
    make = lambda: [[torch.randn(s, device="cuda", generator=gen) for s in ((32, 8), (8, 256), (5, 5))] for _ in range(3)]  # noqa: E731
    a = make()
    b = [[t.clone() for t in ts] for ts in a]
    hp = gpu_api.Muon(lr=1e-2, weight_decay=0.01)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    assert gpu_api._native.muon_step(hp, *a, True, ws) is True
    for wrong in ([a[0][:2], *a[1:]], [[a[0][0], a[0][2], a[0][1]], *a[1:]], [[t.double() for t in a[0]], *a[1:]],
                  [[t.view(-1) for t in ts] for ts in a], [iter(a[0]), *a[1:]], [[], [], []], [[t.cpu() for t in a[0]], *a[1:]]):
        assert gpu_api._native.muon_step(hp, *wrong, False, ws) is None
    assert gpu_api._native.muon_step(bytes(hp), *a, False, ws) is None
    monkeypatch.setattr(gpu_api, "_native", PythonOnly())
    gpu_api.muon_step(hp, *b, zero_grads=True, ws=ws)
    assert all(torch.equal(s, t) for p, q in zip(a, b) for s, t in zip(p, q))
