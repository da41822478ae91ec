"""Activations kept in 8 bits, and the backwards from them, against the definitions."""
import ctypes

import pytest
import torch

import epilogue_cases as ec
import int8_cases as ic
from int8_cases import BF16, F32, same

pytestmark = pytest.mark.gpu

SHAPES = [(1, 8), (3, 24), (5, 32), (2, 40), (64, 1024), (7, 1000), (33, 5128), (1, 22016), (300, 264), (1531, 72), (9, 65544)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_keep_and_restore(gpu_api, shape):
    T, C = shape
    x = ic.drawn_tokens(1, T, C)
    kept = gpu_api.keep8(x.cuda())
    assert kept.numel() == gpu_api.kept8_bytes(T, C) >= T * C
    same(gpu_api.restore8(kept, T, C), ic.restored8(x))


def test_keep_at_the_ends_of_the_range(gpu_api):
    """Zeros, the smallest and largest numbers, ties, codes that would be 128, infinities and NaN (which stay in their group)."""
    x = torch.zeros((6, 72))
    x[0, :32] = torch.arange(32) * 2.0 ** -133           # subnormal
    x[0, 32:64] = -(2.0 ** -126) * (1 + torch.arange(32) / 128)
    x[0, 64:] = 2.0 ** -127
    x[1] = 3.3895313892515355e38                          # the largest bf16: 127.5 steps
    x[2] = 255.0 / 128 * (1 - 2 * (torch.arange(72) % 2))
    x[3] = (torch.arange(72) % 32 + 0.5)                  # ties once 63.5 is there: a step is 1/2 then, and 1 with 64
    x[3, 31], x[3, 63] = 64.0, 127.0
    x[4, 5], x[4, 40] = float("inf"), float("nan")
    x[4, 70] = 1.0
    x[5, :32] = 1.0
    x[5, 64:] = float("-inf")
    x = x.to(BF16)
    got = gpu_api.restore8(gpu_api.keep8(x.cuda()), 6, 72).cpu()
    same(got, ic.restored8(x))
    assert torch.isnan(got[4, :64]).all() and (got[4, 64:] == x[4, 64:]).all() and torch.isfinite(got[5, :64]).all()
    fine = torch.isfinite(got)
    groups = torch.nn.functional.pad(x.double().abs(), (0, 24)).view(6, 3, 32).amax(2).repeat_interleave(32, 1)[:, :72]
    assert ((got.double() - x.double()).abs() <= 2.0 ** -7 * groups.clamp(min=2.0 ** -126))[fine].all()


def swiglu64(gu, dh, C):
    g, u, d = gu[:, :C].double(), gu[:, C:].double(), dh.double()
    s = torch.sigmoid(g)
    # fp32: the exponential's argument and its own rounding, the sum and the division: (|g| + 4) half steps on s; those on
    # 1 - s and on the products after it, of numbers up to 1 + |g|
    dup, dgate = d * g * s, d * u * s * (1 + g * (1 - s))
    tol_g = (d * u).abs() * s * (1 + g.abs()) * (g.abs() + 12) * 2.0 ** -24
    tol_u = dup.abs() * (g.abs() + 8) * 2.0 ** -24
    both, tol = torch.cat([dgate, dup], 1), torch.cat([tol_g, tol_u], 1)
    return both, tol + 2.0 ** -8 * (both.abs() + tol) + 1e-36


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_swiglu(gpu_api, shape):
    T, C = shape
    gu = ic.drawn_tokens(2, T, 2 * C)
    dh = ic.drawn_tokens(3, T, C)
    h, kept = gpu_api.swiglu_forward_keep8(gu.cuda(), C)
    g64 = gu[:, :C].double()
    h64 = g64 * torch.sigmoid(g64) * gu[:, C:].double()
    tol = (8 + 4 * g64.abs()) * 2.0 ** -24 * h64.abs() + 1e-38
    assert ((h.cpu().double() - h64).abs() <= tol + 2.0 ** -8 * (h64.abs() + tol)).all()
    same(gpu_api.restore8(kept, 2 * T, C), ic.restored8(gu.view(2 * T, C)))
    (q, s), kept2 = gpu_api.swiglu_forward_int8(gu.cuda(), C, keep=True)
    same(gpu_api.restore8(kept2, 2 * T, C), ic.restored8(gu.view(2 * T, C)))
    for got, ref in zip((q, s), ic.rows8(h.float().cpu())):
        same(got, ref.to(got.dtype))
    h3 = torch.empty_like(h)
    for got, ref in zip(gpu_api.swiglu_forward_int8(gu.cuda(), C, h=h3), (q, s)):
        same(got, ref)
    same(h3, h)
    lib, P = gpu_api.load(), lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    for with_h in (True, False):                          # one output alone
        h4, k4 = torch.empty_like(h), torch.empty_like(kept)
        g = gu.cuda()
        rc = lib.qalora_swiglu_forward8(T, C, P(g), P(h4) if with_h else None, None, None, None if with_h else P(k4), None)
        torch.cuda.synchronize()
        assert rc == gpu_api.OK
        if with_h:
            same(h4, h)
        else:
            same(gpu_api.restore8(k4, 2 * T, C), gpu_api.restore8(kept, 2 * T, C))
    dgu = gpu_api.swiglu_backward_kept8(dh.cuda(), kept, C).cpu()
    ref, tol = swiglu64(ic.restored8(gu.view(2 * T, C)).view(T, 2 * C), dh, C)
    bad = ((dgu.double() - ref).abs() > tol) | ~torch.isfinite(dgu)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[0].tolist())


@pytest.mark.parametrize("C", [40, 1024, 5128, 22016])
def test_swiglu_of_infinities_and_nan(gpu_api, C):
    """A row whose hidden activations are not all finite has a NaN scale and codes of zero; its kept groups that are finite stay."""
    gu = ic.drawn_tokens(6, 7, 2 * C)
    gu[1, 3], gu[2, C + 5], gu[4, C - 1], gu[5, 2 * C - 1] = float("inf"), float("nan"), float("-inf"), float("-inf")
    (q, s), kept = gpu_api.swiglu_forward_int8(gu.cuda(), C, keep=True)
    h = gpu_api.swiglu_forward_keep8(gu.cuda(), C)[0].cpu()
    assert (torch.isfinite(h).all(1) == torch.tensor([True, False, False, True, False, False, True])).all()
    for got, ref in zip((q, s), ic.rows8(h.float())):
        same(got, ref.to(got.dtype))
    same(gpu_api.restore8(kept, 14, C), ic.restored8(gu.view(14, C)))


def test_swiglu_gradient_against_differences(gpu_api):
    """Gate and up on the kept grid; differences of the definition in 64 bits."""
    T, C = 6, 96
    gu = ic.restored8(ic.drawn_tokens(4, 2 * T, C)).view(T, 2 * C)
    dh = ic.drawn_tokens(5, T, C)
    same(gpu_api.restore8(gpu_api.keep8(gu.view(2 * T, C).cuda()), 2 * T, C), gu.view(2 * T, C))
    dgu = gpu_api.swiglu_backward_kept8(dh.cuda(), gpu_api.swiglu_forward_keep8(gu.cuda(), C)[1], C).cpu().double()
    f = lambda v: dh.double() * v[:, :C] * torch.sigmoid(v[:, :C]) * v[:, C:]  # noqa: E731
    e = 1e-5
    for half in (0, 1):
        step = torch.zeros(2 * C, dtype=torch.float64)
        step[half * C:(half + 1) * C] = e
        slope = (f(gu.double() + step) - f(gu.double() - step)) / (2 * e)
        got = dgu[:, half * C:(half + 1) * C]
        size = (dh.double() * gu[:, C:].double()).abs() if half == 0 else torch.zeros_like(slope)
        # half a step of bf16; fp32's share and e^2 / 6 of a third derivative (below 2 |dh up|) are under 1e-5 of |dh up|
        assert ((got - slope).abs() <= (2.0 ** -8 + 1e-6) * slope.abs() + 1e-5 * size + 1e-9).all()


@pytest.mark.parametrize("shape", [(1, 8), (3, 40), (64, 1024), (300, 264), (1531, 72), (700, 5128)], ids=str)
@pytest.mark.parametrize("dy_dtype", [F32, BF16])
def test_epilogue_backward(gpu_api, shape, dy_dtype):
    """What epilogue_backward makes of the restored z and mul, bit for bit."""
    T, C = shape
    z, mul = (ic.drawn_tokens(k, T, C).cuda() for k in (6, 7))
    dy = ic.drawn_tokens(8, T, C).to(dy_dtype).cuda()
    z8, mul8 = gpu_api.keep8(z), gpu_api.keep8(mul)
    zr, mr = gpu_api.restore8(z8, T, C), gpu_api.restore8(mul8, T, C)
    for act in ec.ACTS:
        for with_mul in (False, True):
            if act == "none" and not with_mul:
                continue
            b0 = torch.randn(C, device="cuda")
            got = gpu_api.epilogue_backward_kept8(dy, z8, act, mul8=mul8 if with_mul else None, want_dbias=True)
            ref = gpu_api.epilogue_backward(dy, zr, act, mul=mr if with_mul else None, want_dbias=True)
            for a, b in zip(got, ref):
                assert (a is None) == (b is None)
                if a is not None:
                    same(a, b)
            acc = [f(dy, zz, act, mm, dbias=b0.clone(), accumulate=True)[2] for f, zz, mm in
                   ((gpu_api.epilogue_backward_kept8, z8, mul8 if with_mul else None),
                    (gpu_api.epilogue_backward, zr, mr if with_mul else None))]
            same(*acc)
    if dy_dtype == BF16:  # in place of dy
        d = dy.clone()
        dz, _, _ = gpu_api.epilogue_backward_kept8(d, z8, "silu", dz=d)
        assert dz is d
        same(d, gpu_api.epilogue_backward(dy, zr, "silu")[0])
