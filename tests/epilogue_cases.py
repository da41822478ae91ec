"""Shapes that reach every kernel an epilogue is applied in, and the epilogue in 64 bits."""
import math

import numpy as np
import torch

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")

# tokens, d_in, d_out, bits, group -> (tile rows, K split, fast addressing) of the dense product
DENSE = {
    (65, 64, 264, 4, 32): (64, False, True),
    (77, 128, 520, 2, 64): (64, False, True),
    (65, 1024, 264, 3, 32): (64, True, True),
    (129, 512, 22016, 4, 32): (128, False, True),
    (129, 512, 22016, 2, 32): (128, False, True),
    (65, 2048, 16392, 4, 32): (128, True, True),
    (450, 256, 16392, 4, 32): (192, False, True),
    (450, 256, 16392, 2, 128): (192, False, True),
    (1025, 512, 12296, 4, 32): (256, False, True),
    (65, 96, 264, 4, 48): (64, False, False),
    (100, 480, 520, 3, 96): (64, True, False),
    (65, 992, 264, 4, 32): (64, True, False),
    (129, 480, 22016, 4, 48): (128, False, False),
}
# tokens, d_in, d_out, bits, group of the adapter-free layer
STREAMED = [(1, 1024, 520, 4, 32), (3, 2176, 5128, 4, 64), (4, 256, 264, 4, 128), (2, 1024, 520, 3, 32), (16, 1152, 1032, 3, 64),
            (7, 1024, 2056, 2, 128), (13, 384, 520, 2, 32),                       # a column per lane
            (5, 1024, 520, 4, 32), (16, 4096, 5128, 4, 64), (32, 2176, 1032, 4, 128), (17, 128, 264, 4, 32)]  # sixteen-token tiles
MID = [(33, 4096, 2056, 4, 32), (64, 2176, 5128, 4, 64), (40, 4096, 4104, 3, 32), (20, 4096, 2056, 2, 128), (61, 5120, 4104, 2, 64)]


def phi(z):
    return 0.5 * torch.erfc(-z * math.sqrt(0.5))


def tanh_arg(z):
    return math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)


def act64(z, act):
    """act(z), its slope, and the magnitude of the exponent that fp32 takes exp of (its rounding is the relative error)."""
    if act == "relu":
        return z.clamp(min=0), (z > 0).double(), torch.zeros_like(z)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s), z.abs()
    if act == "gelu":
        return z * phi(z), phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), z * z
    if act == "gelu_tanh":
        a = tanh_arg(z)
        s = torch.sigmoid(2 * a)
        return z * s, s + z * s * (1 - s) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z), 2 * a.abs()
    return z, torch.ones_like(z), torch.zeros_like(z)


def drawn_layer(seed, tokens, d_in, d_out, bits, group, rank=0):
    """A layer around zero, x of unit size: codes, alpha, beta, x, A, B as CPU tensors."""
    g = torch.Generator().manual_seed(seed)
    L, top = d_in // group, 2 ** bits - 1
    codes = torch.randint(0, top + 1, (d_in, d_out), generator=g, dtype=torch.uint8)
    alpha = (0.1 + 0.05 * torch.rand((L, d_out), generator=g)) / top / math.sqrt(d_in / 256)
    beta = -0.5 * top * alpha + 0.01 * torch.randn((L, d_out), generator=g) / math.sqrt(d_in)
    x = torch.randn((tokens, d_in), generator=g).to(torch.bfloat16)
    A = 0.1 * torch.randn((L, rank), generator=g) if rank else None
    B = 0.1 * torch.randn((rank, d_out), generator=g) if rank else None
    return codes, alpha, beta, x, A, B


def extras(seed, tokens, d_out, out_dtype):
    g = torch.Generator().manual_seed(seed)
    draw = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    return 0.5 * draw(d_out), draw(tokens, d_out).to(torch.bfloat16), draw(tokens, d_out).to(out_dtype)


def linear64(codes, alpha, beta, x, group, A=None, B=None, s=0.0):
    rows = lambda t: t.double().repeat_interleave(group, 0)  # noqa: E731
    x = x.double()
    z = x @ (codes.double() * rows(alpha) + rows(beta))
    if A is not None:
        z = z + s * (x.view(x.shape[0], -1, group).mean(2) @ A.double()) @ B.double()
    return z


def after(z, act, mul=None, residual=None):
    """y from z (64 bits), and what fp32 may be off it by: the exponent's rounding and up to eight half steps more for act,
    a half step each for the product and the sum."""
    value, _, exponent = act64(z, act)
    m = mul.double() if mul is not None else 1.0
    y = value * m
    tol = 2.0 ** -24 * (8 + 4 * exponent) * (value * m).abs()
    if residual is not None:
        y = y + residual.double()
        tol = tol + 2.0 ** -24 * residual.double().abs()
    return y, tol + 2.0 ** -24 * (2 * y.abs()) + 1e-36


def numpy_of(t):
    return np.asarray(t.cpu().double())
