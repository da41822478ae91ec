"""Thin Python binding of the C-ABI library (include/qalora.h).

Argument marshalling only: every step of the layer runs in the HIP kernels behind the
C ABI.  PyTorch supplies device memory and the stream.  The calls of a training step or a serving
loop are marshalled in native code (csrc/binding.cpp) where their arguments are plainly valid.
There is no fallback: if the shared library has not been built, or a call returns an error
status, this raises.
"""
from __future__ import annotations

import array
import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqalora_hip.so")

OK, EINVAL, EALIGN, EWORKSPACE, EUNSUPPORTED, EHIP = 0, -1, -2, -3, -4, -5
F32, BF16 = 0, 1
OP_QUANTIZE, OP_FORWARD, OP_BACKWARD, OP_MERGE, OP_FORWARD_FACTORS16, OP_QUANTIZE_COMPENSATED = 0, 1, 2, 3, 4, 5

EXPORTS = (
    "qalora_status_string", "qalora_check_desc", "qalora_packed_bytes", "qalora_workspace_bytes",
    "qalora_quantize", "qalora_unpack", "qalora_pack", "qalora_forward", "qalora_backward",
    "qalora_merge", "qalora_profile_arm", "qalora_profile_event_create",
    "qalora_profile_event_elapsed_ms", "qalora_profile_event_destroy", "qalora_profile_copy",
    "qalora_swiglu_forward", "qalora_swiglu_backward",
    "qalora_profile_arm_clock", "qalora_profile_arm_blocks", "qalora_profile_wall_clock_khz",
    "qalora_profile_mid_blocks",
    "qalora_beta_from_zero_point", "qalora_zero_point_from_beta",
    "qalora_pack_factors16", "qalora_forward_factors16",
    "qalora_adamw_workspace_bytes", "qalora_adamw_step",
    "qalora_kept_bytes", "qalora_forward_keep", "qalora_backward_kept",
    "qalora_forward_noalloc", "qalora_profile_mfma_probe",
    "qalora_deployed_bytes", "qalora_deploy", "qalora_forward_deployed",
    "qalora_shared_kept_bytes", "qalora_shared_workspace_bytes", "qalora_forward_shared",
    "qalora_quantize_compensated",
    "qalora_backward_shared", "qalora_swiglu_forward_wide", "qalora_swiglu_backward_wide",
    "qalora_muon_workspace_bytes", "qalora_muon_step",
    "qalora_forward_epilogue", "qalora_forward_deployed_epilogue",
    "qalora_epilogue_backward_workspace_bytes", "qalora_epilogue_backward",
    "qalora_quantize_int8", "qalora_deploy_int8", "qalora_quantize_tokens", "qalora_int8_workspace_bytes",
    "qalora_forward_int8", "qalora_backward_int8",
    "qalora_kept8_bytes", "qalora_keep8", "qalora_restore8", "qalora_swiglu_forward8", "qalora_swiglu_backward_kept8",
    "qalora_epilogue_backward_kept8",
)


class Desc(ctypes.Structure):
    """Mirror of ``qalora_desc``."""
    _fields_ = [("d_in", ctypes.c_int32), ("d_out", ctypes.c_int32), ("bits", ctypes.c_int32),
                ("group", ctypes.c_int32), ("rank", ctypes.c_int32), ("s", ctypes.c_float)]


class QaloraError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


def _c_int(value):
    """``value``, which ctypes would take modulo 2^32."""
    if isinstance(value, int) and not -2 ** 31 <= value < 2 ** 31:
        raise ValueError(f"{value} is no C int")
    return value


class _Int(ctypes.c_int):
    """A C int in a call."""

    @classmethod
    def from_param(cls, value):
        return ctypes.c_int.from_param(_c_int(value))


_lib = None


def load() -> ctypes.CDLL:
    """Load the in-tree shared library; fail loudly when it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} not found: build the HIP library first "
            "(python -m paper_2309_14717_amd.build); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, cp, i, sz = ctypes.c_void_p, ctypes.POINTER(Desc), _Int, ctypes.c_size_t
    lib.qalora_status_string.restype = ctypes.c_char_p
    lib.qalora_status_string.argtypes = [i]
    lib.qalora_check_desc.argtypes = [cp]
    lib.qalora_packed_bytes.restype = sz
    lib.qalora_packed_bytes.argtypes = [cp]
    lib.qalora_workspace_bytes.restype = sz
    lib.qalora_workspace_bytes.argtypes = [cp, i, i]
    lib.qalora_quantize.argtypes = [cp, vp, vp, vp, vp, vp, sz, vp]
    lib.qalora_quantize_compensated.argtypes = [cp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.qalora_unpack.argtypes = [cp, vp, vp, vp]
    lib.qalora_pack.argtypes = [cp, vp, vp, vp]
    lib.qalora_forward.argtypes = [cp, i, vp, vp, vp, vp, vp, vp, vp, i, vp, sz, vp]
    lib.qalora_backward.argtypes = [cp, i, vp, vp, vp, vp, vp, vp, vp, vp, i, vp, vp, i, vp, sz, vp]
    lib.qalora_merge.argtypes = [cp, vp, vp, vp, vp, vp]
    lib.qalora_shared_kept_bytes.restype = sz
    lib.qalora_shared_kept_bytes.argtypes = [cp, i, i, vp]
    lib.qalora_shared_workspace_bytes.restype = sz
    lib.qalora_shared_workspace_bytes.argtypes = [cp, i, i, i, vp]
    lib.qalora_forward_shared.argtypes = [cp, i, vp, vp, vp, vp, i, vp, vp, i, vp, vp, sz, vp]
    lib.qalora_backward_shared.argtypes = [cp, i, vp, vp, vp, vp, vp, vp, i, vp, vp, i, i, vp, sz, vp]
    lib.qalora_swiglu_forward_wide.argtypes = [vp, vp, sz, sz, vp]
    lib.qalora_swiglu_backward_wide.argtypes = [vp, vp, vp, sz, sz, vp]
    lib.qalora_deployed_bytes.restype = sz
    lib.qalora_deployed_bytes.argtypes = [cp]
    lib.qalora_deploy.argtypes = [cp, vp, vp, vp, vp, vp]
    lib.qalora_forward_deployed.argtypes = [cp, i, vp, vp, vp, vp, i, vp, sz, vp]
    lib.qalora_profile_mfma_probe.argtypes = [i, i, i, i, i, vp, vp, vp]
    lib.qalora_forward_noalloc.argtypes = [cp, i, vp, vp, vp, vp, vp, i, vp]
    lib.qalora_kept_bytes.restype = sz
    lib.qalora_kept_bytes.argtypes = [cp, i]
    lib.qalora_forward_keep.argtypes = [cp, i, vp, vp, vp, vp, vp, vp, vp, i, vp, vp, sz, vp]
    lib.qalora_backward_kept.argtypes = [cp, i, vp, vp, vp, vp, vp, vp, vp, vp, i, vp, vp, i, vp, sz, vp]
    lib.qalora_profile_arm.argtypes = [i, vp, vp]
    lib.qalora_profile_event_create.argtypes = [ctypes.POINTER(vp)]
    lib.qalora_profile_event_elapsed_ms.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_float)]
    lib.qalora_profile_event_destroy.argtypes = [vp]
    lib.qalora_profile_copy.argtypes = [vp, vp, sz, vp]
    lib.qalora_swiglu_forward.argtypes = [vp, vp, vp, sz, vp]
    lib.qalora_profile_arm_clock.argtypes = [i, vp]
    lib.qalora_profile_arm_blocks.argtypes = [i, vp, i]
    lib.qalora_profile_mid_blocks.argtypes = [cp, i, ctypes.POINTER(ctypes.c_int)]
    lib.qalora_profile_wall_clock_khz.argtypes = [ctypes.POINTER(ctypes.c_int)]
    lib.qalora_swiglu_backward.argtypes = [vp, vp, vp, vp, vp, sz, vp]
    lib.qalora_pack_factors16.argtypes = [cp, vp, vp, vp, vp]
    lib.qalora_forward_factors16.argtypes = [cp, i, vp, vp, vp, vp, i, vp, sz, vp]
    lib.qalora_adamw_workspace_bytes.restype = sz
    lib.qalora_adamw_workspace_bytes.argtypes = [i, vp]
    lib.qalora_adamw_step.argtypes = [vp, i, i, vp, vp, vp, vp, vp, i, vp, vp, sz, vp]
    lib.qalora_forward_epilogue.argtypes = [cp, i, vp, vp, vp, vp, vp, vp, vp, vp, i, vp, vp, sz, vp]
    lib.qalora_forward_deployed_epilogue.argtypes = [cp, i, vp, vp, vp, vp, vp, i, vp, sz, vp]
    lib.qalora_epilogue_backward_workspace_bytes.restype = sz
    lib.qalora_epilogue_backward_workspace_bytes.argtypes = [i, i]
    lib.qalora_epilogue_backward.argtypes = [i, i, i, vp, i, vp, vp, vp, vp, vp, i, vp, sz, vp]
    lib.qalora_quantize_int8.argtypes = [i, i, vp, vp, vp, vp]
    lib.qalora_deploy_int8.argtypes = [cp, vp, vp, vp, vp, vp, vp]
    lib.qalora_quantize_tokens.argtypes = [i, i, vp, vp, vp, vp, vp]
    lib.qalora_int8_workspace_bytes.restype = sz
    lib.qalora_int8_workspace_bytes.argtypes = [i, i, i, i]
    lib.qalora_forward_int8.argtypes = [i, i, i, vp, vp, vp, vp, vp, vp, i, vp, sz, vp]
    lib.qalora_backward_int8.argtypes = [i, i, i, vp, vp, vp, vp, vp, i, vp, sz, vp]
    lib.qalora_kept8_bytes.restype = sz
    lib.qalora_kept8_bytes.argtypes = [i, i]
    lib.qalora_keep8.argtypes = [i, i, vp, vp, vp]
    lib.qalora_restore8.argtypes = [i, i, vp, vp, vp]
    lib.qalora_swiglu_forward8.argtypes = [i, i, vp, vp, vp, vp, vp, vp]
    lib.qalora_swiglu_backward_kept8.argtypes = [i, i, vp, vp, vp, vp]
    lib.qalora_epilogue_backward_kept8.argtypes = [i, i, i, vp, i, vp, vp, vp, vp, vp, i, vp, sz, vp]
    lib.qalora_muon_workspace_bytes.restype = sz
    lib.qalora_muon_workspace_bytes.argtypes = [i, vp, vp]
    lib.qalora_muon_step.argtypes = [vp, i, vp, vp, vp, vp, vp, i, vp, sz, vp]
    lib.qalora_beta_from_zero_point.argtypes = [cp, vp, vp, vp, vp]
    lib.qalora_zero_point_from_beta.argtypes = [cp, vp, vp, vp, vp]
    _lib = lib
    return lib


_native = None
_NATIVE_ENTRIES = (
    "qalora_check_desc", "qalora_packed_bytes", "qalora_workspace_bytes", "qalora_quantize", "qalora_forward",
    "qalora_kept_bytes", "qalora_forward_keep", "qalora_backward", "qalora_backward_kept", "qalora_deployed_bytes",
    "qalora_forward_deployed", "qalora_forward_factors16", "qalora_adamw_step", "qalora_shared_kept_bytes",
    "qalora_shared_workspace_bytes", "qalora_forward_shared", "qalora_backward_shared", "qalora_swiglu_forward_wide",
    "qalora_swiglu_backward_wide", "qalora_forward_epilogue", "qalora_forward_deployed_epilogue",
    "qalora_epilogue_backward", "qalora_epilogue_backward_workspace_bytes", "qalora_muon_step",
    "qalora_muon_workspace_bytes", "qalora_quantize_tokens", "qalora_int8_workspace_bytes", "qalora_forward_int8",
    "qalora_backward_int8", "qalora_kept8_bytes", "qalora_keep8", "qalora_swiglu_forward8", "qalora_swiglu_backward_kept8",
    "qalora_epilogue_backward_kept8")


def _bind_native():
    """Hand the library's entry points to the native form of the calls below (csrc/binding.cpp).  Each function
    asks it first: it takes the calls whose arguments are plainly valid and returns None for all others, which
    the checks here then look at one by one.  (Host-side queries need the library alone.)"""
    global _native
    lib = load()
    path = os.path.join(_HERE, "_native.so")
    if not os.path.exists(path):
        raise RuntimeError(f"{path} not found: build it first (python -m paper_2309_14717_amd.build)")
    from . import _native as native
    native.bind({name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _NATIVE_ENTRIES}, _check,
                Desc, AdamW, Muon)
    _native = native


def _fast():
    if _native is None:
        _bind_native()
    return _native


def status_string(status: int) -> str:
    return load().qalora_status_string(int(status)).decode()


def make_desc(d_in, d_out, bits=4, group=32, rank=0, s=0.0) -> Desc:
    return Desc(*(_c_int(int(v)) for v in (d_in, d_out, bits, group, rank)), float(s))


def check_desc(desc: Desc) -> int:
    return int(load().qalora_check_desc(ctypes.byref(desc)))


def packed_bytes(desc: Desc) -> int:
    return int(load().qalora_packed_bytes(ctypes.byref(desc)))


def workspace_bytes(desc: Desc, tokens: int, op: int) -> int:
    return int(load().qalora_workspace_bytes(ctypes.byref(desc), int(tokens), int(op)))


def _p(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _on(dev):
    """The device of a call's tensors as the current one, whose stream the call then takes."""
    return torch.cuda.device(dev)


def _check(rc, where):
    if rc != OK:
        raise QaloraError(int(rc), where)


def _workspace(desc, tokens, op, ws, device="cuda"):
    # a caller-provided workspace is passed through as it is (the library checks its size)
    if ws is None:
        ws = torch.empty(max(workspace_bytes(desc, tokens, op), 16), dtype=torch.uint8, device=device)
    else:
        _need(ws, "ws", device=device)
    return ws, ws.numel() * ws.element_size()


def _need(t, name, dtype=None, shape=None, nbytes=None, device=None, optional=False):
    """The C ABI sees raw pointers only: a tensor of the wrong size, type or device would become
    an out-of-bounds device access there, so every operand is checked here first."""
    if t is None:
        if optional:
            return
        raise ValueError(f"{name}: missing")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: must be a device tensor")
    if device is not None and t.device != torch.device(device):
        raise ValueError(f"{name}: on {t.device}, expected {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if nbytes is not None and t.numel() * t.element_size() < nbytes:
        raise ValueError(f"{name}: {t.numel() * t.element_size()} bytes, needs at least {nbytes}")


def _need_layer(desc, x, in_features, packed, alpha, beta, A, B, x_name="x"):
    """Checks shared by every forward / backward entry; returns (tokens, device)."""
    _need(x, x_name, torch.bfloat16)
    dev = x.device
    if check_desc(desc) != OK:  # the library rejects the call with its own status
        return x.shape[0], dev
    if x.dim() != 2 or x.shape[1] != in_features:
        raise ValueError(f"{x_name}: shape {tuple(x.shape)}, expected [tokens, {in_features}]")
    L = desc.d_in // max(desc.group, 1)
    _need(packed, "packed", nbytes=packed_bytes(desc), device=dev)
    _need(alpha, "alpha", torch.float32, (L, desc.d_out), device=dev)
    if beta is not None:
        _need(beta, "beta", torch.float32, (L, desc.d_out), device=dev)
    if (A is None) != (B is None):
        raise ValueError("A and B must be given together")
    if A is not None:
        _need(A, "A", torch.float32, (L, desc.rank), device=dev)
        _need(B, "B", torch.float32, (desc.rank, desc.d_out), device=dev)
    return x.shape[0], dev


def _need_factor_pair(desc, alpha, other, other_name):
    _need(alpha, "alpha", torch.float32)
    shape = (desc.d_in // desc.group, desc.d_out) if check_desc(desc) == OK else tuple(alpha.shape)
    _need(alpha, "alpha", shape=shape)
    _need(other, other_name, torch.float32, shape, device=alpha.device)


def _need_out(t, name, rows, cols, dev):
    _need(t, name, shape=(rows, cols), device=dev)
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"{name}: dtype {t.dtype}, expected float32 or bfloat16")


def quantize(desc: Desc, W: torch.Tensor):
    """W fp32 [d_in, d_out] (device) -> (packed uint8, alpha fp32 [L, d_out], beta fp32 [L, d_out])."""
    out = _fast().quantize(desc, W)
    if out is not None:
        return out
    _need(W, "W", torch.float32)
    if check_desc(desc) == OK:
        _need(W, "W", shape=(desc.d_in, desc.d_out))
    L = desc.d_in // max(desc.group, 1)
    packed = torch.empty(packed_bytes(desc), dtype=torch.uint8, device=W.device)
    alpha = torch.empty((L, desc.d_out), dtype=torch.float32, device=W.device)
    beta = torch.empty_like(alpha)
    rc = load().qalora_quantize(ctypes.byref(desc), _p(W), _p(packed), _p(alpha), _p(beta), None, 0,
                                _stream())
    _check(rc, "qalora_quantize")
    return packed, alpha, beta


def quantize_compensated(desc: Desc, W: torch.Tensor, hinv_chol: torch.Tensor):
    """Error-compensated code selection under an inverse-Hessian Cholesky factor U [d_in, d_in]
    (upper triangular, H^-1 = U^T U).  Returns (packed, alpha, beta) like quantize()."""
    _need(W, "W", torch.float32)
    if check_desc(desc) == OK:
        _need(W, "W", shape=(desc.d_in, desc.d_out))
        _need(hinv_chol, "hinv_chol", torch.float32, (desc.d_in, desc.d_in), device=W.device)
    L = desc.d_in // max(desc.group, 1)
    packed = torch.empty(packed_bytes(desc), dtype=torch.uint8, device=W.device)
    alpha = torch.empty((L, desc.d_out), dtype=torch.float32, device=W.device)
    beta = torch.empty_like(alpha)
    ws = torch.empty(max(workspace_bytes(desc, 1, OP_QUANTIZE_COMPENSATED), 16), dtype=torch.uint8, device=W.device)
    rc = load().qalora_quantize_compensated(ctypes.byref(desc), _p(W), _p(hinv_chol), _p(packed), _p(alpha),
                                            _p(beta), _p(ws), ws.numel(), _stream())
    _check(rc, "qalora_quantize_compensated")
    return packed, alpha, beta


def unpack(desc: Desc, packed: torch.Tensor) -> torch.Tensor:
    _need(packed, "packed", nbytes=packed_bytes(desc))
    codes = torch.empty((desc.d_in, desc.d_out), dtype=torch.uint8, device=packed.device)
    _check(load().qalora_unpack(ctypes.byref(desc), _p(packed), _p(codes), _stream()), "qalora_unpack")
    return codes


def pack(desc: Desc, codes: torch.Tensor) -> torch.Tensor:
    _need(codes, "codes", torch.uint8)
    if check_desc(desc) == OK:
        _need(codes, "codes", shape=(desc.d_in, desc.d_out))
    packed = torch.empty(packed_bytes(desc), dtype=torch.uint8, device=codes.device)
    _check(load().qalora_pack(ctypes.byref(desc), _p(codes), _p(packed), _stream()), "qalora_pack")
    return packed


def forward(desc: Desc, x, packed, alpha, beta, A=None, B=None, out_dtype=torch.float32, ws=None,
            y=None):
    """y = x W~ + s (pool(x) A) B.  x bf16 [T, d_in]; returns y [T, d_out]."""
    out = _fast().forward(desc, x, packed, alpha, beta, A, B, out_dtype, ws, y)
    if out is not None:
        return out
    T, dev = _need_layer(desc, x, desc.d_in, packed, alpha, beta, A, B)
    if y is None:
        y = torch.empty((T, desc.d_out), dtype=out_dtype, device=dev)
    _need_out(y, "y", T, desc.d_out, dev)
    ws, ws_bytes = _workspace(desc, T, OP_FORWARD, ws, dev)
    rc = load().qalora_forward(ctypes.byref(desc), T, _p(x), _p(packed), _p(alpha), _p(beta), _p(A),
                               _p(B), _p(y), BF16 if y.dtype == torch.bfloat16 else F32, _p(ws),
                               ws_bytes, _stream())
    _check(rc, "qalora_forward")
    return y


def forward_noalloc(desc: Desc, x, packed, alpha, beta, out_dtype=torch.float32, y=None):
    """Adapter-free few-token forward on the library's built-in scratch (no workspace)."""
    T, dev = _need_layer(desc, x, desc.d_in, packed, alpha, beta, None, None)
    if y is None:
        y = torch.empty((T, desc.d_out), dtype=out_dtype, device=dev)
    _need_out(y, "y", T, desc.d_out, dev)
    rc = load().qalora_forward_noalloc(ctypes.byref(desc), T, _p(x), _p(packed), _p(alpha), _p(beta), _p(y),
                                       BF16 if y.dtype == torch.bfloat16 else F32, _stream())
    _check(rc, "qalora_forward_noalloc")
    return y


ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


class Epilogue(ctypes.Structure):
    """Mirror of ``qalora_epilogue``."""
    _fields_ = [("act", ctypes.c_int32), ("bias", ctypes.c_void_p), ("mul", ctypes.c_void_p),
                ("residual", ctypes.c_void_p), ("z", ctypes.c_void_p)]


def _act(act):
    if act not in ACTIVATIONS:
        raise ValueError(f"act: {act!r}, expected one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[act]


def _epilogue(T, d_out, dev, y, bias, act, mul, residual, z):
    _need(bias, "bias", torch.float32, (d_out,), device=dev, optional=True)
    _need(mul, "mul", torch.bfloat16, (T, d_out), device=dev, optional=True)
    _need(residual, "residual", y.dtype, (T, d_out), device=dev, optional=True)
    _need(z, "z", torch.bfloat16, (T, d_out), device=dev, optional=True)
    address = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    return Epilogue(_act(act), address(bias), address(mul), address(residual), address(z))


def forward_epilogue(desc: Desc, x, packed, alpha, beta, A=None, B=None, bias=None, act="none", mul=None,
                     residual=None, keep_z=False, keep=False, out_dtype=torch.float32, ws=None, y=None, z=None, kept=None):
    """forward() with y = act(x W~ + ... + bias) * mul + residual (see qalora_forward_epilogue).  ``act`` is one of
    ACTIVATIONS; ``residual`` has y's type and may be the ``y`` that is passed, as may a ``mul`` where y is bfloat16; other
    outputs over operands are refused.  Returns y; or (y, z, kept) with
    ``keep_z`` (z in bf16, for epilogue_backward) or ``keep`` (the pooled activations, for backward_kept), None in the place
    of the one not asked for."""
    out = _fast().forward_epilogue(desc, x, packed, alpha, beta, A, B, bias, ACTIVATIONS.get(act), mul, residual, keep_z, keep,
                                   out_dtype, ws, y, z, kept)
    if out is not None:
        return out
    T, dev = _need_layer(desc, x, desc.d_in, packed, alpha, beta, A, B)
    if y is None:
        y = torch.empty((T, desc.d_out), dtype=out_dtype, device=dev)
    _need_out(y, "y", T, desc.d_out, dev)
    for t, wanted, name, flag in ((z, keep_z, "z", "keep_z"), (kept, keep, "kept", "keep")):
        if t is not None and not wanted:
            raise ValueError(f"{name}: given without {flag}")
    if keep_z and z is None:
        z = torch.empty((T, desc.d_out), dtype=torch.bfloat16, device=dev)
    if keep:
        if kept is None:
            kept = torch.empty(max(kept_bytes(desc, T), 16), dtype=torch.uint8, device=dev)
        _need(kept, "kept", nbytes=kept_bytes(desc, T), device=dev)
    epi = _epilogue(T, desc.d_out, dev, y, bias, act, mul, residual, z if keep_z else None)
    ws, ws_bytes = _workspace(desc, T, OP_FORWARD, ws, dev)
    with _on(dev):
        rc = load().qalora_forward_epilogue(ctypes.byref(desc), T, _p(x), _p(packed), _p(alpha), _p(beta), _p(A), _p(B),
                                            ctypes.byref(epi), _p(y), BF16 if y.dtype == torch.bfloat16 else F32,
                                            _p(kept) if keep else None, _p(ws), ws_bytes, _stream())
    _check(rc, "qalora_forward_epilogue")
    return (y, z if keep_z else None, kept if keep else None) if keep or keep_z else y


def epilogue_backward(dy, z=None, act="none", mul=None, want_dz=True, want_dbias=False, dz=None, dmul=None, dbias=None,
                      accumulate=False, ws=None):
    """Backward of the epilogue at the kept z (see qalora_epilogue_backward): (dz, dmul, dbias), None in the place of what
    is not there: dmul without ``mul``, dbias unless wanted or given.  ``dz`` or ``dmul`` may be z, mul or a bfloat16 dy; other
    overlaps are refused.  dz is the dy of backward(); the gradient of the
    residual is dy itself."""
    out = _fast().epilogue_backward(dy, z, ACTIVATIONS.get(act), mul, want_dz, want_dbias, dz, dmul, dbias, accumulate, ws)
    if out is not None:
        return out
    _need(dy, "dy")
    if dy.dim() != 2 or dy.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"dy: {dy.dtype} {tuple(dy.shape)}, expected a float32 or bfloat16 matrix")
    (T, cols), dev = dy.shape, dy.device
    _need(z, "z", torch.bfloat16, (T, cols), device=dev, optional=True)
    _need(mul, "mul", torch.bfloat16, (T, cols), device=dev, optional=True)
    if dmul is not None and mul is None:
        raise ValueError("dmul: given without mul")
    if want_dz and dz is None:
        dz = torch.empty((T, cols), dtype=torch.bfloat16, device=dev)
    if mul is not None and dmul is None:
        dmul = torch.empty((T, cols), dtype=torch.bfloat16, device=dev)
    if want_dbias and dbias is None:
        dbias = torch.zeros(cols, dtype=torch.float32, device=dev)
    _need(dz, "dz", torch.bfloat16, (T, cols), device=dev, optional=True)
    _need(dmul, "dmul", torch.bfloat16, (T, cols), device=dev, optional=True)
    _need(dbias, "dbias", torch.float32, (cols,), device=dev, optional=True)
    if ws is None and dbias is not None:
        n = int(load().qalora_epilogue_backward_workspace_bytes(T, cols))
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
    _need(ws, "ws", device=dev, optional=True)
    act = _act(act)
    with _on(dev):
        rc = load().qalora_epilogue_backward(act, T, cols, _p(dy), BF16 if dy.dtype == torch.bfloat16 else F32, _p(z),
                                             _p(mul), _p(dz), _p(dmul), _p(dbias), 1 if accumulate else 0, _p(ws),
                                             0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(rc, "qalora_epilogue_backward")
    return dz, dmul, dbias


class Part(ctypes.Structure):
    """Mirror of ``qalora_part``."""
    _fields_ = [("d_out", ctypes.c_int32), ("rank", ctypes.c_int32), ("s", ctypes.c_float),
                ("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("dA", ctypes.c_void_p), ("dB", ctypes.c_void_p)]


def _parts(desc, adapters, dev, grads=None):
    """adapters: list of (A [L, rank], B [rank, d_out_p], s); grads: list of (dA, dB) or None."""
    L = desc.d_in // max(desc.group, 1)
    arr = (Part * len(adapters))()
    for q, (A, B, s) in enumerate(adapters):
        _need(A, f"A[{q}]", torch.float32, device=dev)
        _need(B, f"B[{q}]", torch.float32, device=dev)
        if A.dim() != 2 or B.dim() != 2 or A.shape[0] != L or A.shape[1] != B.shape[0]:
            raise ValueError(f"part {q}: A {tuple(A.shape)}, B {tuple(B.shape)}, expected [{L}, r] and [r, d_out]")
        arr[q].d_out, arr[q].rank, arr[q].s = int(B.shape[1]), int(A.shape[1]), float(s)
        arr[q].A, arr[q].B = A.data_ptr(), B.data_ptr()
        if grads is not None:
            dA, dB = grads[q]
            _need(dA, f"dA[{q}]", torch.float32, tuple(A.shape), device=dev)
            _need(dB, f"dB[{q}]", torch.float32, tuple(B.shape), device=dev)
            arr[q].dA, arr[q].dB = dA.data_ptr(), dB.data_ptr()
    if sum(int(B.shape[1]) for _, B, _ in adapters) != desc.d_out:
        raise ValueError("the parts' widths must add up to d_out")
    return arr


def forward_shared(desc: Desc, x, packed, alpha, beta, adapters, keep=False, out_dtype=torch.float32,
                   ws=None, y=None, kept=None):
    """Linears that share x as one wide layer (see qalora_forward_shared).  ``adapters`` is a
    list of (A, B, s), one per part in column order.  Returns y, or (y, kept) with ``keep``."""
    out = _fast().forward_shared(desc, x, packed, alpha, beta, adapters, keep, out_dtype, ws, y, kept)
    if out is not None:
        return out
    T, dev = _need_layer(desc, x, desc.d_in, packed, alpha, beta, None, None)
    arr = _parts(desc, adapters, dev)
    n = len(adapters)
    if y is None:
        y = torch.empty((T, desc.d_out), dtype=out_dtype, device=dev)
    _need_out(y, "y", T, desc.d_out, dev)
    if keep:
        kb = int(load().qalora_shared_kept_bytes(ctypes.byref(desc), T, n, arr))
        if kept is None:
            kept = torch.empty(max(kb, 16), dtype=torch.uint8, device=dev)
        _need(kept, "kept", nbytes=kb, device=dev)
    if ws is None:
        ws = torch.empty(max(int(load().qalora_shared_workspace_bytes(ctypes.byref(desc), T, OP_FORWARD, n, arr)), 16),
                         dtype=torch.uint8, device=dev)
    _need(ws, "ws", device=dev)
    rc = load().qalora_forward_shared(ctypes.byref(desc), T, _p(x), _p(packed), _p(alpha), _p(beta), n, arr,
                                      _p(y), BF16 if y.dtype == torch.bfloat16 else F32,
                                      _p(kept) if keep else None, _p(ws), ws.numel() * ws.element_size(), _stream())
    _check(rc, "qalora_forward_shared")
    return (y, kept) if keep else y


def backward_shared(desc: Desc, dy, x, kept, packed, alpha, beta, adapters, want_dx=True,
                    dx_dtype=torch.float32, grads=None, accumulate=False, ws=None, dx=None):
    """Backward of forward_shared: one dx over all parts, (dA, dB) per part.  Pass ``kept`` (from
    forward_shared(keep=True)) or ``x``.  Returns (dx, [(dA, dB), ...])."""
    out = _fast().backward_shared(desc, dy, x, kept, packed, alpha, beta, adapters, want_dx, dx_dtype, grads, accumulate,
                                  ws, dx)
    if out is not None:
        return out
    T, dev = _need_layer(desc, dy, desc.d_out, packed, alpha, beta, None, None, x_name="dy")
    if kept is None:
        _need(x, "x", torch.bfloat16, (T, desc.d_in), device=dev)
    if grads is None:
        grads = [(torch.zeros_like(A), torch.zeros_like(B)) for A, B, _ in adapters]
    arr = _parts(desc, adapters, dev, grads)
    n = len(adapters)
    if kept is not None:
        _need(kept, "kept", nbytes=int(load().qalora_shared_kept_bytes(ctypes.byref(desc), T, n, arr)), device=dev)
    if want_dx and dx is None:
        dx = torch.empty((T, desc.d_in), dtype=dx_dtype, device=dev)
    if dx is not None:
        _need_out(dx, "dx", T, desc.d_in, dev)
    if ws is None:
        ws = torch.empty(max(int(load().qalora_shared_workspace_bytes(ctypes.byref(desc), T, OP_BACKWARD, n, arr)), 16),
                         dtype=torch.uint8, device=dev)
    _need(ws, "ws", device=dev)
    dxd = BF16 if (dx is not None and dx.dtype == torch.bfloat16) else F32
    rc = load().qalora_backward_shared(ctypes.byref(desc), T, _p(dy), _p(x) if kept is None else None, _p(kept),
                                       _p(packed), _p(alpha), _p(beta), n, arr, _p(dx), dxd,
                                       1 if accumulate else 0, _p(ws), ws.numel() * ws.element_size(), _stream())
    _check(rc, "qalora_backward_shared")
    return dx, grads


def deploy(desc: Desc, packed, alpha, beta):
    """One-time repack of a (merged) 4-bit layer into the decode kernel's stream."""
    n = int(load().qalora_deployed_bytes(ctypes.byref(desc)))
    if n == 0:
        raise QaloraError(EUNSUPPORTED, "qalora_deployed_bytes")
    L = desc.d_in // desc.group
    _need(packed, "packed", nbytes=packed_bytes(desc))
    _need(alpha, "alpha", torch.float32, (L, desc.d_out), device=packed.device)
    _need(beta, "beta", torch.float32, (L, desc.d_out), device=packed.device)
    out = torch.empty(n, dtype=torch.uint8, device=packed.device)
    _check(load().qalora_deploy(ctypes.byref(desc), _p(packed), _p(alpha), _p(beta), _p(out), _stream()),
           "qalora_deploy")
    return out


def forward_deployed(desc: Desc, x, deployed, packed=None, out_dtype=torch.float32, ws=None, y=None):
    """Adapter-free forward of a deployed layer: the decode stream up to four tokens; beyond that
    ``packed`` is required: the mid-token kernel up to 64 tokens, the dense kernel with the prepared factor
    words above (see mid_blocks)."""
    out = _fast().forward_deployed(desc, x, deployed, packed, out_dtype, ws, y)
    if out is not None:
        return out
    _need(x, "x", torch.bfloat16)
    T, dev = x.shape[0], x.device
    if check_desc(desc) == OK:
        _need(x, "x", shape=(T, desc.d_in))
        _need(deployed, "deployed", nbytes=int(load().qalora_deployed_bytes(ctypes.byref(desc))), device=dev)
        if T > 4:
            _need(packed, "packed", nbytes=packed_bytes(desc), device=dev)
    if y is None:
        y = torch.empty((T, desc.d_out), dtype=out_dtype, device=dev)
    _need_out(y, "y", T, desc.d_out, dev)
    ws, ws_bytes = _workspace(desc, T, OP_FORWARD, ws, dev)
    rc = load().qalora_forward_deployed(ctypes.byref(desc), T, _p(x), _p(packed), _p(deployed), _p(y),
                                        BF16 if y.dtype == torch.bfloat16 else F32, _p(ws), ws_bytes, _stream())
    _check(rc, "qalora_forward_deployed")
    return y


def forward_deployed_epilogue(desc: Desc, x, deployed, packed=None, bias=None, act="none", mul=None, residual=None,
                              out_dtype=torch.float32, ws=None, y=None):
    """forward_deployed() with the epilogue of forward_epilogue()."""
    out = _fast().forward_deployed_epilogue(desc, x, deployed, packed, bias, ACTIVATIONS.get(act), mul, residual, out_dtype, ws,
                                            y)
    if out is not None:
        return out
    _need(x, "x", torch.bfloat16)
    T, dev = x.shape[0], x.device
    if check_desc(desc) == OK:
        _need(x, "x", shape=(T, desc.d_in))
        _need(deployed, "deployed", nbytes=int(load().qalora_deployed_bytes(ctypes.byref(desc))), device=dev)
        if T > 4:
            _need(packed, "packed", nbytes=packed_bytes(desc), device=dev)
    if y is None:
        y = torch.empty((T, desc.d_out), dtype=out_dtype, device=dev)
    _need_out(y, "y", T, desc.d_out, dev)
    epi = _epilogue(T, desc.d_out, dev, y, bias, act, mul, residual, None)
    ws, ws_bytes = _workspace(desc, T, OP_FORWARD, ws, dev)
    with _on(dev):
        rc = load().qalora_forward_deployed_epilogue(ctypes.byref(desc), T, _p(x), _p(packed), _p(deployed),
                                                     ctypes.byref(epi), _p(y), BF16 if y.dtype == torch.bfloat16 else F32,
                                                     _p(ws), ws_bytes, _stream())
    _check(rc, "qalora_forward_deployed_epilogue")
    return y


WS_STATUS_OFFSET = 2048


def streaming_status(ws) -> int:
    """The status word the kernels for up to 64 tokens set in a forward workspace when a bounded wait ran
    out (0 = never, provided the caller zeroed it first).  Synchronises."""
    _need(ws, "ws", nbytes=WS_STATUS_OFFSET + 8)
    return int(ws.view(torch.uint8)[WS_STATUS_OFFSET:WS_STATUS_OFFSET + 8].cpu().view(torch.int64).item())


def mid_blocks(desc: Desc, tokens: int) -> int:
    """Blocks the kernel for up to 64 tokens launches for the adapter-free forward, 0: the dense kernel."""
    n = ctypes.c_int()
    _check(load().qalora_profile_mid_blocks(ctypes.byref(desc), int(tokens), ctypes.byref(n)), "qalora_profile_mid_blocks")
    return n.value


def pack_factors16(desc: Desc, alpha, beta, out=None):
    """One int32 word per (group, column): fp16(alpha) | fp16(beta) << 16."""
    L = desc.d_in // max(desc.group, 1)
    _need(alpha, "alpha", torch.float32, (L, desc.d_out))
    _need(beta, "beta", torch.float32, (L, desc.d_out), device=alpha.device)
    if out is None:
        out = torch.empty(alpha.shape, dtype=torch.int32, device=alpha.device)
    _need(out, "out", nbytes=4 * L * desc.d_out, device=alpha.device)
    _check(load().qalora_pack_factors16(ctypes.byref(desc), _p(alpha), _p(beta), _p(out), _stream()),
           "qalora_pack_factors16")
    return out


def forward_factors16(desc: Desc, x, packed, factors16, out_dtype=torch.float32, ws=None, y=None):
    """Adapter-free y = x W~ with the factors stored in 16 bits (see pack_factors16)."""
    out = _fast().forward_factors16(desc, x, packed, factors16, out_dtype, ws, y)
    if out is not None:
        return out
    _need(x, "x", torch.bfloat16)
    T, dev = x.shape[0], x.device
    if check_desc(desc) == OK:
        _need(x, "x", shape=(T, desc.d_in))
        _need(packed, "packed", nbytes=packed_bytes(desc), device=dev)
        _need(factors16, "factors16", nbytes=4 * (desc.d_in // desc.group) * desc.d_out, device=dev)
    if y is None:
        y = torch.empty((T, desc.d_out), dtype=out_dtype, device=dev)
    _need_out(y, "y", T, desc.d_out, dev)
    ws, ws_bytes = _workspace(desc, T, OP_FORWARD_FACTORS16, ws, dev)
    rc = load().qalora_forward_factors16(ctypes.byref(desc), T, _p(x), _p(packed), _p(factors16), _p(y),
                                         BF16 if y.dtype == torch.bfloat16 else F32, _p(ws), ws_bytes,
                                         _stream())
    _check(rc, "qalora_forward_factors16")
    return y


def backward(desc: Desc, dy, x, packed, alpha, beta, A=None, B=None, want_dx=True,
             dx_dtype=torch.float32, dA=None, dB=None, accumulate=False, ws=None, dx=None):
    """Returns (dx, dA, dB).  dy bf16 [T, d_out], x bf16 [T, d_in]."""
    out = _fast().backward(desc, dy, x, packed, alpha, beta, A, B, want_dx, dx_dtype, dA, dB, accumulate, ws, dx)
    if out is not None:
        return out
    T, dev = _need_layer(desc, dy, desc.d_out, packed, alpha, beta, A, B, x_name="dy")
    if A is not None or x is not None:
        _need(x, "x", torch.bfloat16, (T, desc.d_in), device=dev)
    if want_dx and dx is None:
        dx = torch.empty((T, desc.d_in), dtype=dx_dtype, device=dev)
    if dx is not None:
        _need_out(dx, "dx", T, desc.d_in, dev)
    if A is not None:
        if dA is None:
            dA = torch.zeros_like(A)
        if dB is None:
            dB = torch.zeros_like(B)
        _need(dA, "dA", torch.float32, tuple(A.shape), device=dev)
        _need(dB, "dB", torch.float32, tuple(B.shape), device=dev)
    ws, ws_bytes = _workspace(desc, T, OP_BACKWARD, ws, dev)
    dxd = BF16 if (dx is not None and dx.dtype == torch.bfloat16) else F32
    rc = load().qalora_backward(ctypes.byref(desc), T, _p(dy), _p(x), _p(packed), _p(alpha),
                                _p(beta), _p(A), _p(B), _p(dx), dxd, _p(dA), _p(dB),
                                1 if accumulate else 0, _p(ws), ws_bytes, _stream())
    _check(rc, "qalora_backward")
    return dx, dA, dB


def kept_bytes(desc: Desc, tokens: int) -> int:
    return int(load().qalora_kept_bytes(ctypes.byref(desc), tokens))


def forward_keep(desc: Desc, x, packed, alpha, beta, A, B, out_dtype=torch.float32, ws=None, y=None,
                 kept=None):
    """forward() that also leaves the pooled activations the backward needs.  Returns (y, kept)."""
    out = _fast().forward_keep(desc, x, packed, alpha, beta, A, B, out_dtype, ws, y, kept)
    if out is not None:
        return out
    T, dev = _need_layer(desc, x, desc.d_in, packed, alpha, beta, A, B)
    if y is None:
        y = torch.empty((T, desc.d_out), dtype=out_dtype, device=dev)
    _need_out(y, "y", T, desc.d_out, dev)
    if kept is None:
        kept = torch.empty(max(kept_bytes(desc, T), 16), dtype=torch.uint8, device=dev)
    _need(kept, "kept", nbytes=kept_bytes(desc, T), device=dev)
    ws, ws_bytes = _workspace(desc, T, OP_FORWARD, ws, dev)
    rc = load().qalora_forward_keep(ctypes.byref(desc), T, _p(x), _p(packed), _p(alpha), _p(beta), _p(A),
                                    _p(B), _p(y), BF16 if y.dtype == torch.bfloat16 else F32, _p(kept),
                                    _p(ws), ws_bytes, _stream())
    _check(rc, "qalora_forward_keep")
    return y, kept


def backward_kept(desc: Desc, dy, kept, packed, alpha, beta, A, B, want_dx=True,
                  dx_dtype=torch.float32, dA=None, dB=None, accumulate=False, ws=None, dx=None):
    """backward() from what forward_keep() left instead of x.  Returns (dx, dA, dB)."""
    out = _fast().backward_kept(desc, dy, kept, packed, alpha, beta, A, B, want_dx, dx_dtype, dA, dB, accumulate, ws, dx)
    if out is not None:
        return out
    T, dev = _need_layer(desc, dy, desc.d_out, packed, alpha, beta, A, B, x_name="dy")
    _need(kept, "kept", nbytes=kept_bytes(desc, T), device=dev)
    if want_dx and dx is None:
        dx = torch.empty((T, desc.d_in), dtype=dx_dtype, device=dev)
    if dx is not None:
        _need_out(dx, "dx", T, desc.d_in, dev)
    if dA is None:
        dA = torch.zeros_like(A)
    if dB is None:
        dB = torch.zeros_like(B)
    _need(dA, "dA", torch.float32, tuple(A.shape), device=dev)
    _need(dB, "dB", torch.float32, tuple(B.shape), device=dev)
    ws, ws_bytes = _workspace(desc, T, OP_BACKWARD, ws, dev)
    dxd = BF16 if (dx is not None and dx.dtype == torch.bfloat16) else F32
    rc = load().qalora_backward_kept(ctypes.byref(desc), T, _p(dy), _p(kept), _p(packed), _p(alpha),
                                     _p(beta), _p(A), _p(B), _p(dx), dxd, _p(dA), _p(dB),
                                     1 if accumulate else 0, _p(ws), ws_bytes, _stream())
    _check(rc, "qalora_backward_kept")
    return dx, dA, dB


def merge(desc: Desc, beta, A, B, out=None):
    """beta' = beta + (s/g) A B; ``out`` may be ``beta`` itself."""
    _need(beta, "beta", torch.float32)
    if check_desc(desc) == OK:
        L = desc.d_in // desc.group
        _need(beta, "beta", shape=(L, desc.d_out))
        _need(A, "A", torch.float32, (L, desc.rank), device=beta.device)
        _need(B, "B", torch.float32, (desc.rank, desc.d_out), device=beta.device)
    if out is None:
        out = torch.empty_like(beta)
    _need(out, "out", torch.float32, tuple(beta.shape), device=beta.device)
    _check(load().qalora_merge(ctypes.byref(desc), _p(beta), _p(A), _p(B), _p(out), _stream()),
           "qalora_merge")
    return out


def beta_from_zero_point(desc: Desc, alpha, z, out=None):
    """beta = -(alpha z): import a zero point (code units) as the zero factor of Eq. 1."""
    _need_factor_pair(desc, alpha, z, "z")
    if out is None:
        out = torch.empty_like(alpha)
    _need(out, "out", torch.float32, tuple(alpha.shape), device=alpha.device)
    _check(load().qalora_beta_from_zero_point(ctypes.byref(desc), _p(alpha), _p(z), _p(out), _stream()),
           "qalora_beta_from_zero_point")
    return out


def zero_point_from_beta(desc: Desc, alpha, beta, out=None):
    """z = -(beta / alpha): export the zero factor as a zero point in code units."""
    _need_factor_pair(desc, alpha, beta, "beta")
    if out is None:
        out = torch.empty_like(alpha)
    _need(out, "out", torch.float32, tuple(alpha.shape), device=alpha.device)
    _check(load().qalora_zero_point_from_beta(ctypes.byref(desc), _p(alpha), _p(beta), _p(out), _stream()),
           "qalora_zero_point_from_beta")
    return out


class AdamW(ctypes.Structure):
    """Mirror of ``qalora_adamw``."""
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float), ("max_grad_norm", ctypes.c_float)]


def adamw_step(hp: AdamW, step: int, params, grads, exp_avg, exp_avg_sq, zero_grads=False, grad_norm=None,
               ws=None):
    """One fused AdamW step with a joint gradient-norm clip over lists of fp32 device tensors
    (updated in place).  ``grad_norm``: optional one-element fp32 device tensor for the norm."""
    if _fast().adamw_step(hp, step, params, grads, exp_avg, exp_avg_sq, zero_grads, grad_norm, ws):
        return
    n = len(params)
    lists = ((params, "params"), (grads, "grads"), (exp_avg, "exp_avg"), (exp_avg_sq, "exp_avg_sq"))
    tensors = [t for ts, _ in lists for t in ts]
    for ts, nm in lists:
        if len(ts) != n:
            raise ValueError(f"{nm}: {len(ts)} tensors, expected {n}")
        for t, p0 in zip(ts, params):
            _need(t, nm, torch.float32, tuple(p0.shape), device=params[0].device)
    _need(grad_norm, "grad_norm", torch.float32, nbytes=4, optional=True)
    table = array.array("Q", map(torch.Tensor.data_ptr, tensors))  # n addresses of each list
    sizes = array.array("Q", map(torch.Tensor.numel, params))
    ptrs = [table.buffer_info()[0] + 8 * n * i for i in range(4)]
    numel = sizes.buffer_info()[0]
    if ws is None:
        ws = torch.empty(max(load().qalora_adamw_workspace_bytes(n, numel), 16), dtype=torch.uint8, device="cuda")
    rc = load().qalora_adamw_step(ctypes.byref(hp), int(step), n, ptrs[0], ptrs[1], ptrs[2], ptrs[3], numel,
                                  1 if zero_grads else 0, _p(grad_norm), _p(ws), ws.numel(), _stream())
    _check(rc, "qalora_adamw_step")


# 1; sqrt(max(1, rows / cols)), the published factor of weights stored [out, in] (A and B are [in, out]: see qalora_muon_step);
# 0.2 sqrt(max(rows, cols))
MUON_SCALE_NONE, MUON_SCALE_SHAPE, MUON_SCALE_RMS = 0, 1, 2


class Muon(ctypes.Structure):
    """Mirror of ``qalora_muon``; a, b, c, steps and eps default to the published ones."""
    _fields_ = [("lr", ctypes.c_float), ("momentum", ctypes.c_float), ("weight_decay", ctypes.c_float),
                ("eps", ctypes.c_float), ("a", ctypes.c_float), ("b", ctypes.c_float), ("c", ctypes.c_float),
                ("steps", ctypes.c_int32), ("nesterov", ctypes.c_int32), ("scale_mode", ctypes.c_int32)]

    def __init__(self, lr=0.0, momentum=0.95, weight_decay=0.0, eps=1e-7, a=3.4445, b=-4.7750, c=2.0315, steps=5,
                 nesterov=True, scale_mode=MUON_SCALE_RMS):
        super().__init__(lr, momentum, weight_decay, eps, a, b, c, steps, 1 if nesterov else 0, scale_mode)


def _sides(tensors):
    rows, cols = (array.array("i", (int(t.shape[k]) for t in tensors)) for k in (0, 1))
    return rows, cols


def muon_workspace_bytes(tensors) -> int:
    """Workspace of muon_step() over matrices of these shapes; 0 where they are not acceptable."""
    rows, cols = _sides(tensors)
    return int(load().qalora_muon_workspace_bytes(len(rows), rows.buffer_info()[0], cols.buffer_info()[0]))


def muon_step(hp: Muon, params, grads, momentum, zero_grads=False, ws=None):
    """One orthogonalised step (see qalora_muon_step) over lists of fp32 device matrices, one side of each at most
    128; ``params`` and ``momentum`` are updated in place."""
    if _fast().muon_step(hp, params, grads, momentum, zero_grads, ws):
        return
    n = len(params)
    if n == 0:
        raise ValueError("params: no tensors")
    for ts, nm in ((params, "params"), (grads, "grads"), (momentum, "momentum")):
        if len(ts) != n:
            raise ValueError(f"{nm}: {len(ts)} tensors, expected {n}")
        for t, p0 in zip(ts, params):
            _need(t, nm, torch.float32, tuple(p0.shape), device=params[0].device)
            if t.dim() != 2:
                raise ValueError(f"{nm}: shape {tuple(t.shape)}, expected a matrix")
    rows, cols = _sides(params)
    table = array.array("Q", (t.data_ptr() for ts in (params, grads, momentum) for t in ts))
    ptrs = [table.buffer_info()[0] + 8 * n * i for i in range(3)]
    if ws is None:
        ws = torch.empty(max(muon_workspace_bytes(params), 16), dtype=torch.uint8, device=params[0].device)
    _need(ws, "ws", device=params[0].device)
    with _on(params[0].device):
        rc = load().qalora_muon_step(ctypes.byref(hp), n, ptrs[0], ptrs[1], ptrs[2], rows.buffer_info()[0],
                                     cols.buffer_info()[0], 1 if zero_grads else 0, _p(ws), ws.numel() * ws.element_size(),
                                     _stream())
    _check(rc, "qalora_muon_step")


def profile_copy(dst: torch.Tensor, src: torch.Tensor):
    """Plain copy kernel of known size (yardstick for the HBM traffic counters)."""
    _need(src, "src")
    n = src.numel() * src.element_size()
    _need(dst, "dst", nbytes=n, device=src.device)
    _check(load().qalora_profile_copy(_p(dst), _p(src), n, _stream()), "qalora_profile_copy")


def mfma_probe(shape: int, lds_reads: bool, valu_per_mfma: int, iters: int = 500, blocks: int = 256):
    """Issue-rate probe of the matrix cores (measurement aid).  Returns (cycles per matrix
    instruction per SIMD, shader clock in GHz, TFLOP/s) over all blocks of the launch."""
    sink = torch.empty(blocks * 512, dtype=torch.float32, device="cuda")
    counts = torch.zeros((blocks, 2), dtype=torch.int64, device="cuda")
    for _ in range(2):  # the second launch runs at the clock the mix settles to
        _check(load().qalora_profile_mfma_probe(int(shape), 1 if lds_reads else 0, int(valu_per_mfma), int(iters),
                                                int(blocks), _p(sink), _p(counts), _stream()), "qalora_profile_mfma_probe")
        torch.cuda.synchronize()
    khz = ctypes.c_int()
    _check(load().qalora_profile_wall_clock_khz(ctypes.byref(khz)), "wall_clock_khz")
    c = counts.cpu().double()
    cycles, ticks = c[:, 0].mean().item(), c[:, 1].mean().item()
    per_simd = iters * 64.0  # matrix instructions per SIMD: 32 per K step per wavefront, 2 wavefronts (or 64, 1)
    seconds = ticks / (khz.value * 1e3)
    flops = blocks * 4 * per_simd * 2.0 * 32 * 32 * 16
    return cycles / per_simd, cycles / ticks * khz.value * 1e3 / 1e9, flops / seconds / 1e12


def swiglu_forward(gate, up, out=None):
    """Harness glue: h = silu(gate) * up, bf16 tensors of equal shape."""
    _need(gate, "gate", torch.bfloat16)
    _need(up, "up", torch.bfloat16, tuple(gate.shape), device=gate.device)
    if out is None:
        out = torch.empty_like(gate)
    _need(out, "out", torch.bfloat16, tuple(gate.shape), device=gate.device)
    _check(load().qalora_swiglu_forward(_p(gate), _p(up), _p(out), gate.numel(), _stream()),
           "qalora_swiglu_forward")
    return out


def swiglu_backward(dh, gate, up, dgate=None, dup=None):
    """Harness glue: gradients of h = silu(gate) * up with respect to gate and up (bf16)."""
    _need(gate, "gate", torch.bfloat16)
    _need(up, "up", torch.bfloat16, tuple(gate.shape), device=gate.device)
    _need(dh, "dh", torch.bfloat16, tuple(gate.shape), device=gate.device)
    if dgate is None:
        dgate = torch.empty_like(gate)
    if dup is None:
        dup = torch.empty_like(up)
    _need(dgate, "dgate", torch.bfloat16, tuple(gate.shape), device=gate.device)
    _need(dup, "dup", torch.bfloat16, tuple(gate.shape), device=gate.device)
    _check(load().qalora_swiglu_backward(_p(dh), _p(gate), _p(up), _p(dgate), _p(dup), gate.numel(),
                                         _stream()), "qalora_swiglu_backward")
    return dgate, dup


def swiglu_forward_strided(gu, cols, out=None):
    """Harness glue on gu = [gate | up] ([rows, 2 cols] bf16): h = silu(gate) * up."""
    h = _fast().swiglu_forward_wide(gu, cols, out)
    if h is not None:
        return h
    _need(gu, "gu", torch.bfloat16)
    rows = gu.shape[0]
    _need(gu, "gu", shape=(rows, 2 * cols))
    if out is None:
        out = torch.empty((rows, cols), dtype=torch.bfloat16, device=gu.device)
    _need(out, "out", torch.bfloat16, (rows, cols), device=gu.device)
    _check(load().qalora_swiglu_forward_wide(_p(gu), _p(out), rows, cols, _stream()), "qalora_swiglu_forward_wide")
    return out


def swiglu_backward_strided(dh, gu, cols, out=None):
    """Harness glue: dgu = [dgate | dup] of h = silu(gate) * up on gu = [gate | up]."""
    dgu = _fast().swiglu_backward_wide(dh, gu, cols, out)
    if dgu is not None:
        return dgu
    _need(gu, "gu", torch.bfloat16)
    rows = gu.shape[0]
    _need(gu, "gu", shape=(rows, 2 * cols))
    _need(dh, "dh", torch.bfloat16, (rows, cols), device=gu.device)
    if out is None:
        out = torch.empty_like(gu)
    _need(out, "out", torch.bfloat16, (rows, 2 * cols), device=gu.device)
    _check(load().qalora_swiglu_backward_wide(_p(dh), _p(gu), _p(out), rows, cols, _stream()),
           "qalora_swiglu_backward_wide")
    return out


def quantize_int8(W):
    """W fp32 [d_in, d_out] -> (codes int8 [d_out, d_in], scale fp32 [d_out]): a frozen weight for forward_int8 and backward_int8."""
    _need(W, "W", torch.float32)
    if W.dim() != 2:
        raise ValueError(f"W: shape {tuple(W.shape)}, expected [d_in, d_out]")
    (d_in, d_out), dev = W.shape, W.device
    codes = torch.empty((d_out, d_in), dtype=torch.int8, device=dev)
    scale = torch.empty(d_out, dtype=torch.float32, device=dev)
    with _on(dev):
        rc = load().qalora_quantize_int8(d_in, d_out, _p(W), _p(codes), _p(scale), _stream())
    _check(rc, "qalora_quantize_int8")
    return codes, scale


def deploy_int8(desc: Desc, packed, alpha, beta):
    """The 8-bit form (codes, scale) of a merged layer, or of one without an adapter (see qalora_deploy_int8)."""
    _need(packed, "packed", nbytes=packed_bytes(desc))
    dev = packed.device
    L = desc.d_in // max(desc.group, 1)
    if check_desc(desc) == OK:
        _need(alpha, "alpha", torch.float32, (L, desc.d_out), device=dev)
        _need(beta, "beta", torch.float32, (L, desc.d_out), device=dev)
    codes = torch.empty((max(desc.d_out, 0), max(desc.d_in, 0)), dtype=torch.int8, device=dev)
    scale = torch.empty(max(desc.d_out, 0), dtype=torch.float32, device=dev)
    with _on(dev):
        rc = load().qalora_deploy_int8(ctypes.byref(desc), _p(packed), _p(alpha), _p(beta), _p(codes), _p(scale), _stream())
    _check(rc, "qalora_deploy_int8")
    return codes, scale


def _matrix(t, name, dtype):
    _need(t, name, dtype)
    if t.dim() != 2:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected a matrix")
    return t.shape[0], t.shape[1], t.device


def _given(t, name, dtype, shape, dev):
    """An output: the caller's, or a new one."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    _need(t, name, dtype, shape, device=dev)
    return t


def quantize_tokens(x, factor=None, q=None, s=None):
    """x bf16 [tokens, cols], each row in 8 bits with a scale of its own: (q int8 [tokens, cols], s fp32 [tokens]), what
    forward_int8 takes in place of x.  ``factor`` fp32 [cols] multiplies the columns first."""
    out = _fast().quantize_tokens(x, factor, q, s)
    if out is not None:
        return out
    T, cols, dev = _matrix(x, "x", torch.bfloat16)
    _need(factor, "factor", torch.float32, (cols,), device=dev, optional=True)
    q, s = _given(q, "q", torch.int8, (T, cols), dev), _given(s, "s", torch.float32, (T,), dev)
    with _on(dev):
        rc = load().qalora_quantize_tokens(T, cols, _p(x), _p(factor), _p(q), _p(s), _stream())
    _check(rc, "qalora_quantize_tokens")
    return q, s


def int8_workspace_bytes(tokens: int, d_in: int, d_out: int, op: int) -> int:
    """Workspace of forward_int8 (OP_FORWARD) and backward_int8 (OP_BACKWARD) for up to so many tokens."""
    return int(load().qalora_int8_workspace_bytes(int(tokens), int(d_in), int(d_out), int(op)))


def _int8_workspace(T, d_in, d_out, op, ws, dev):
    if ws is None:
        ws = torch.empty(max(int8_workspace_bytes(T, d_in, d_out, op), 16), dtype=torch.uint8, device=dev)
    _need(ws, "ws", device=dev)
    return ws, ws.numel() * ws.element_size()


def forward_int8(x, codes, scale, bias=None, act="none", mul=None, residual=None, keep_z=False, out_dtype=torch.float32, ws=None,
                 y=None, z=None):
    """y = act(s (q codes^T) scale + bias) * mul + residual in 8-bit integers (see qalora_forward_int8).  ``x`` is bf16
    [tokens, d_in], or what quantize_tokens or swiglu_forward_int8 made of one: (q, s).  The epilogue is forward_epilogue's.
    Returns y, or with ``keep_z`` (y, z)."""
    out = _fast().forward_int8(x, codes, scale, bias, ACTIVATIONS.get(act), mul, residual, keep_z, out_dtype, ws, y, z)
    if out is not None:
        return out
    d_out, d_in, dev = _matrix(codes, "codes", torch.int8)
    _need(scale, "scale", torch.float32, (d_out,), device=dev)
    s = None
    if isinstance(x, (tuple, list)):
        x, s = x
        _need(x, "x", torch.int8, device=dev)
    else:
        _need(x, "x", torch.bfloat16, device=dev)
    if x.dim() != 2 or x.shape[1] != d_in:
        raise ValueError(f"x: shape {tuple(x.shape)}, expected [tokens, {d_in}]")
    if x.dtype == torch.int8:
        _need(s, "x's scales", torch.float32, (x.shape[0],), device=dev)
    T = x.shape[0]
    if y is None:
        y = torch.empty((T, d_out), dtype=out_dtype, device=dev)
    _need_out(y, "y", T, d_out, dev)
    if z is not None and not keep_z:
        raise ValueError("z: given without keep_z")
    if keep_z and z is None:
        z = torch.empty((T, d_out), dtype=torch.bfloat16, device=dev)
    epi = _epilogue(T, d_out, dev, y, bias, act, mul, residual, z)
    ws, ws_bytes = _int8_workspace(T, d_in, d_out, OP_FORWARD, ws, dev)
    with _on(dev):
        rc = load().qalora_forward_int8(T, d_in, d_out, _p(x), _p(s), _p(codes), _p(scale), ctypes.byref(epi), _p(y),
                                        BF16 if y.dtype == torch.bfloat16 else F32, _p(ws), ws_bytes, _stream())
    _check(rc, "qalora_forward_int8")
    return (y, z) if keep_z else y


def backward_int8(dy, codes, scale, residual=None, dx_dtype=torch.float32, ws=None, dx=None):
    """dx of forward_int8's product with the weight frozen (see qalora_backward_int8): dy bf16 [tokens, d_out] -> dx [tokens, d_in],
    plus ``residual`` (dx's type; it may be the ``dx`` that is passed: gradients of several linears then add up in place)."""
    out = _fast().backward_int8(dy, codes, scale, residual, dx_dtype, ws, dx)
    if out is not None:
        return out
    d_out, d_in, dev = _matrix(codes, "codes", torch.int8)
    _need(scale, "scale", torch.float32, (d_out,), device=dev)
    _need(dy, "dy", torch.bfloat16, device=dev)
    if dy.dim() != 2 or dy.shape[1] != d_out:
        raise ValueError(f"dy: shape {tuple(dy.shape)}, expected [tokens, {d_out}]")
    T = dy.shape[0]
    if dx is None:
        dx = torch.empty((T, d_in), dtype=dx_dtype, device=dev)
    _need_out(dx, "dx", T, d_in, dev)
    _need(residual, "residual", dx.dtype, (T, d_in), device=dev, optional=True)
    ws, ws_bytes = _int8_workspace(T, d_in, d_out, OP_BACKWARD, ws, dev)
    with _on(dev):
        rc = load().qalora_backward_int8(T, d_in, d_out, _p(dy), _p(codes), _p(scale), _p(residual), _p(dx),
                                         BF16 if dx.dtype == torch.bfloat16 else F32, _p(ws), ws_bytes, _stream())
    _check(rc, "qalora_backward_int8")
    return dx


def kept8_bytes(tokens: int, cols: int) -> int:
    return int(load().qalora_kept8_bytes(int(tokens), int(cols)))


def _kept8(kept, name, tokens, cols, dev, new=False):
    n = kept8_bytes(tokens, cols)
    if kept is None and new:
        return torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
    _need(kept, name, torch.uint8, nbytes=n, device=dev)
    return kept


def keep8(x, kept=None):
    """x bf16 [tokens, cols] kept in 8 bits for a backward (see qalora_keep8): an opaque uint8 tensor."""
    out = _fast().keep8(x, kept)
    if out is not None:
        return out
    T, cols, dev = _matrix(x, "x", torch.bfloat16)
    kept = _kept8(kept, "kept", T, cols, dev, new=True)
    with _on(dev):
        rc = load().qalora_keep8(T, cols, _p(x), _p(kept), _stream())
    _check(rc, "qalora_keep8")
    return kept


def restore8(kept, tokens, cols, x=None):
    """What keep8 (or, with twice the tokens, swiglu_forward_keep8) kept, as bf16 [tokens, cols]."""
    _need(kept, "kept", torch.uint8, nbytes=kept8_bytes(tokens, cols))
    x = _given(x, "x", torch.bfloat16, (tokens, cols), kept.device)
    with _on(kept.device):
        rc = load().qalora_restore8(tokens, cols, _p(kept), _p(x), _stream())
    _check(rc, "qalora_restore8")
    return x


def _swiglu_input(gu, cols):
    T, width, dev = _matrix(gu, "gu", torch.bfloat16)
    if width != 2 * cols:
        raise ValueError(f"gu: shape {tuple(gu.shape)}, expected [tokens, {2 * cols}]")
    return T, dev


def swiglu_forward_keep8(gu, cols, h=None, kept=None):
    """h = silu(gate) * up of gu = [gate | up] (bf16 [tokens, 2 cols]), and gate and up kept in 8 bits: (h, kept)."""
    out = _fast().swiglu_forward_keep8(gu, cols, h, kept)
    if out is not None:
        return out
    T, dev = _swiglu_input(gu, cols)
    h = _given(h, "h", torch.bfloat16, (T, cols), dev)
    kept = _kept8(kept, "kept", 2 * T, cols, dev, new=True)
    with _on(dev):
        rc = load().qalora_swiglu_forward8(T, cols, _p(gu), _p(h), None, None, _p(kept), _stream())
    _check(rc, "qalora_swiglu_forward8")
    return h, kept


def swiglu_forward_int8(gu, cols, keep=False, q=None, s=None, kept=None, h=None):
    """silu(gate) * up of gu = [gate | up] as 8-bit tokens (q, s), what forward_int8 of the down projection takes; with
    ``keep`` ((q, s), kept), gate and up kept in 8 bits as by swiglu_forward_keep8.  A given ``h`` receives the hidden activations."""
    out = _fast().swiglu_forward_int8(gu, cols, keep, q, s, kept, h)
    if out is not None:
        return out
    T, dev = _swiglu_input(gu, cols)
    q, s = _given(q, "q", torch.int8, (T, cols), dev), _given(s, "s", torch.float32, (T,), dev)
    _need(h, "h", torch.bfloat16, (T, cols), device=dev, optional=True)
    if kept is not None and not keep:
        raise ValueError("kept: given without keep")
    if keep:
        kept = _kept8(kept, "kept", 2 * T, cols, dev, new=True)
    with _on(dev):
        rc = load().qalora_swiglu_forward8(T, cols, _p(gu), _p(h), _p(q), _p(s), _p(kept), _stream())
    _check(rc, "qalora_swiglu_forward8")
    return ((q, s), kept) if keep else (q, s)


def swiglu_backward_kept8(dh, kept, cols, dgu=None):
    """dgu = [dgate | dup] from dh (bf16 [tokens, cols]) and the gate and up that were kept in 8 bits."""
    out = _fast().swiglu_backward_kept8(dh, kept, cols, dgu)
    if out is not None:
        return out
    T, width, dev = _matrix(dh, "dh", torch.bfloat16)
    if width != cols:
        raise ValueError(f"dh: shape {tuple(dh.shape)}, expected [tokens, {cols}]")
    _kept8(kept, "kept", 2 * T, cols, dev)
    dgu = _given(dgu, "dgu", torch.bfloat16, (T, 2 * cols), dev)
    with _on(dev):
        rc = load().qalora_swiglu_backward_kept8(T, cols, _p(dh), _p(kept), _p(dgu), _stream())
    _check(rc, "qalora_swiglu_backward_kept8")
    return dgu


def epilogue_backward_kept8(dy, z8=None, act="none", mul8=None, want_dz=True, want_dbias=False, dz=None, dmul=None, dbias=None,
                            accumulate=False, ws=None):
    """epilogue_backward with z and mul as keep8 kept them: (dz, dmul, dbias), None in the place of what is not there."""
    out = _fast().epilogue_backward_kept8(dy, z8, ACTIVATIONS.get(act), mul8, want_dz, want_dbias, dz, dmul, dbias, accumulate, ws)
    if out is not None:
        return out
    _need(dy, "dy")
    if dy.dim() != 2 or dy.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"dy: {dy.dtype} {tuple(dy.shape)}, expected a float32 or bfloat16 matrix")
    (T, cols), dev = dy.shape, dy.device
    if z8 is not None:
        _kept8(z8, "z8", T, cols, dev)
    if mul8 is not None:
        _kept8(mul8, "mul8", T, cols, dev)
    if dmul is not None and mul8 is None:
        raise ValueError("dmul: given without mul8")
    if want_dz or dz is not None:
        dz = _given(dz, "dz", torch.bfloat16, (T, cols), dev)
    if mul8 is not None:
        dmul = _given(dmul, "dmul", torch.bfloat16, (T, cols), dev)
    if want_dbias and dbias is None:
        dbias = torch.zeros(cols, dtype=torch.float32, device=dev)
    _need(dbias, "dbias", torch.float32, (cols,), device=dev, optional=True)
    if ws is None and dbias is not None:
        n = int(load().qalora_epilogue_backward_workspace_bytes(T, cols))
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
    _need(ws, "ws", device=dev, optional=True)
    act = _act(act)
    with _on(dev):
        rc = load().qalora_epilogue_backward_kept8(act, T, cols, _p(dy), BF16 if dy.dtype == torch.bfloat16 else F32, _p(z8),
                                                   _p(mul8), _p(dz), _p(dmul), _p(dbias), 1 if accumulate else 0, _p(ws),
                                                   0 if ws is None else ws.numel() * ws.element_size(), _stream())
    _check(rc, "qalora_epilogue_backward_kept8")
    return dz, dmul, dbias


class KernelTimer:
    """HIP-event pairs recorded by the library around its dense-contraction kernel
    (measurement aid of the C ABI); ``direction`` 0 = forward kernel, 1 = backward kernel."""

    def __init__(self, direction: int, n: int):
        self.direction = direction
        self.pairs = []
        for _ in range(n):
            a, b = ctypes.c_void_p(), ctypes.c_void_p()
            _check(load().qalora_profile_event_create(ctypes.byref(a)), "event_create")
            _check(load().qalora_profile_event_create(ctypes.byref(b)), "event_create")
            self.pairs.append((a, b))
        self.used = 0
        # per launch: shader cycles and wall-clock ticks at the first block's start and end
        self.counts = torch.zeros((n, 4), dtype=torch.int64, device="cuda")

    def arm(self):
        a, b = self.pairs[self.used]
        _check(load().qalora_profile_arm(self.direction, a, b), "profile_arm")
        _check(load().qalora_profile_arm_clock(self.direction, _p(self.counts[self.used])),
               "profile_arm_clock")
        self.used += 1

    def arm_blocks(self, capacity=4096):
        """Call right after arm(): the armed kernel's blocks also report their time line."""
        self.block_times = torch.zeros((capacity, 4), dtype=torch.int64, device="cuda")
        _check(load().qalora_profile_arm_blocks(self.direction, _p(self.block_times), capacity),
               "profile_arm_blocks")

    def block_timeline(self):
        """Summary of the last arm_blocks() launch, in microseconds from the first block's start."""
        khz = ctypes.c_int()
        _check(load().qalora_profile_wall_clock_khz(ctypes.byref(khz)), "wall_clock_khz")
        c = self.block_times.cpu().numpy()
        c = c[c[:, 0] > 0]
        if len(c) == 0:
            return None
        import numpy as np
        us = lambda v: (v - c[:, 0].min()) / khz.value * 1e3
        st, kend, en, xcd = us(c[:, 0]), us(c[:, 1]), us(c[:, 2]), c[:, 3]
        q = lambda v: [round(float(x), 1) for x in (v.min(), np.median(v), v.max())]
        return {"blocks": int(len(c)), "start_us_min_med_max": q(st), "k_loop_end_us_min_med_max": q(kend),
                "end_us_min_med_max": q(en), "epilogue_us_median": round(float(np.median(en - kend)), 1),
                "end_us_median_by_xcd": {int(x): round(float(np.median(en[xcd == x])), 1) for x in sorted(set(xcd.tolist()))}}

    def shader_clock_ghz(self):
        """Average shader clock over the life of the armed kernels' first blocks (None when the
        armed kernel was one that does not report)."""
        khz = ctypes.c_int()
        _check(load().qalora_profile_wall_clock_khz(ctypes.byref(khz)), "wall_clock_khz")
        c = self.counts[: self.used].cpu().double()
        cycles, ticks = c[:, 2] - c[:, 0], c[:, 3] - c[:, 1]
        ok = ticks > 0
        if not bool(ok.any()):
            return None
        return float((cycles[ok] / ticks[ok]).mean()) * khz.value * 1e3 / 1e9

    def block_cycles(self):
        """Mean shader cycles the armed kernels' first blocks lived for (None if not reported)."""
        c = self.counts[: self.used].cpu().double()
        cycles = c[:, 2] - c[:, 0]
        ok = (c[:, 3] - c[:, 1]) > 0
        return float(cycles[ok].mean()) if bool(ok.any()) else None

    def elapsed_ms(self):
        out = []
        for a, b in self.pairs[: self.used]:
            ms = ctypes.c_float()
            _check(load().qalora_profile_event_elapsed_ms(a, b, ctypes.byref(ms)), "event_elapsed")
            out.append(ms.value)
        return out

    def close(self):
        for a, b in self.pairs:
            load().qalora_profile_event_destroy(a)
            load().qalora_profile_event_destroy(b)
        self.pairs = []
