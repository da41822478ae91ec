"""Results of the 8-bit linear to the last bit, the sign of a zero among them: from the definition's own steps where these fix them (sums,
z, what a bias or a residual is added to), and as those of a smaller batch where an activation comes in."""
import pytest
import torch

import epilogue_cases as ec
import int8_cases as ic
from int8_cases import BF16, F32

pytestmark = pytest.mark.gpu

# all kernels: one launch for few tokens; the smaller tiles, with and without slices of K; the larger; two widths of them
SIZES = [(1, 1024, 264), (5, 64, 72), (16, 1024, 1024), (4, 11008, 520), (17, 5120, 520), (33, 4096, 264), (64, 1024, 1024), (100, 2064, 520),
         (129, 4112, 1544), (257, 1024, 328)] + ic.LARGE + ic.MIXED


def bits(t):
    return t.view({2: torch.int16, 4: torch.int32}[t.element_size()])


def alike(got, ref):
    assert got.dtype == ref.dtype and got.shape == ref.shape and not torch.isnan(ref).any()
    bad = bits(got) != bits(ref)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[0].tolist(), got[bad][:4], ref[bad][:4])


def drawn(T, K, N):
    """Tokens of which one is zeros, and channels of which some have a negative scale: products that are -0."""
    x = ic.drawn_tokens(2, T, K)
    x[T // 2] = 0
    codes, scale = ic.drawn_weight(1, K, N)
    scale[::3] *= -1
    return x.cuda(), codes.cuda(), scale.cuda()


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_is_its_definition(gpu_api, size):
    T, K, N = size
    x, codes, scale = drawn(*size)
    q, s = gpu_api.quantize_tokens(x)
    prod = (q.double() @ codes.double().T.contiguous()).to(F32) * s[:, None] * scale   # whole numbers below 2^53, then two roundings
    assert (bits(prod[T // 2]) == -2 ** 31).any()
    for tokens in (x, (q, s)):
        for dtype in (F32, BF16):
            bias, _, residual = (t.cuda() for t in ec.extras(3, T, N, dtype))
            bias[1::4] = -0.0
            residual[:, ::5] = -0.0
            for use in range(4):
                b, r = bias if use & 1 else None, residual if use & 2 else None
                z = prod + b if use & 1 else prod
                y = z + r.to(F32) if use & 2 else z
                got, got_z = gpu_api.forward_int8(tokens, codes, scale, bias=b, residual=r, keep_z=True, out_dtype=dtype)
                alike(got_z, z.to(BF16))
                alike(got, y.to(dtype))


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward_is_its_definition(gpu_api, size):
    T, K, N = size                                         # of the product: d_out, d_in
    K, N = K // 8 * 8, -(-N // 16) * 16
    dy, codes, scale = drawn(T, K, N)[0], *(t.cuda() for t in ic.drawn_weight(5, N, K))
    scale[::3] *= -1
    q, s = gpu_api.quantize_tokens(dy, scale)
    prod = (q.double() @ codes.double()).to(F32) * s[:, None]
    alike(gpu_api.backward_int8(dy, codes, scale), prod)
    for dtype in (F32, BF16):
        r = torch.randn((T, N), generator=torch.Generator("cuda").manual_seed(9), device="cuda").to(dtype)
        r[:, ::5] = -0.0
        alike(gpu_api.backward_int8(dy, codes, scale, residual=r, dx_dtype=dtype), (prod + r.to(F32)).to(dtype))


@pytest.mark.parametrize("size", ic.LARGE + ic.MIXED, ids=str)
def test_a_large_batch_is_its_parts(gpu_api, size):
    """With every operand of the epilogue: rows of the largest tiles' launches as in batches of few, which other kernels take."""
    T, K, N = size
    x, codes, scale = drawn(*size)
    tokens = gpu_api.quantize_tokens(x)
    some = [slice(0, 1), slice(T // 2 - 1, T // 2 + 2), slice(100, 117), slice(T - 66, T)]
    for dtype in (F32, BF16):
        bias, mul, residual = (t.cuda() for t in ec.extras(3, T, N, dtype))
        for act in ec.ACTS:
            for use in range(8):
                call = lambda at: gpu_api.forward_int8(  # noqa: E731
                    tuple(t[at].clone() for t in tokens), codes, scale, bias=bias if use & 1 else None, act=act, mul=mul[at] if use & 2 else None,
                    residual=residual[at] if use & 4 else None, keep_z=True, out_dtype=dtype)
                whole = call(slice(0, T))
                for at in some:
                    for part, all_rows in zip(call(at), whole):
                        alike(part, all_rows[at])


@pytest.mark.parametrize("up", [1.0, -3.0, 1e30])
def test_hidden_activations_of_very_negative_gates(gpu_api, up):
    """As documented: (8 + 4 |gate|) 2^-24 of themselves, and half a step of bf16, down to gates of -87.33; zero below, where a silu
    is less than 2^-119.  (Half a step of a subnormal bf16 number is 2^-134.)"""
    gate = torch.cat([torch.arange(-110, -79.75, 0.25), torch.arange(-87.5, -86.5, 2.0 ** -4)]).to(BF16)
    C = gate.numel() // 8 * 8
    gate = gate[:C]
    gu = torch.cat([gate, torch.full((C,), up, dtype=BF16)])[None].cuda()
    h, _ = gpu_api.swiglu_forward_keep8(gu, C)
    h2 = torch.empty_like(h)
    gpu_api.swiglu_forward_int8(gu, C, h=h2)
    alike(h2, h)
    g = gate.double()
    ref = g * torch.sigmoid(g) * float(torch.tensor(up).to(BF16))
    tol = (8 + 4 * g.abs()) * 2.0 ** -24 * ref.abs()
    off = (h[0].cpu().double() - ref).abs()
    near = off <= tol + 2.0 ** -8 * (ref.abs() + tol) + 2.0 ** -134
    assert near[g > -87.33].all()
    assert (h[0].cpu()[g < -87.34] == 0).all() and (ref.abs()[g < -87.34] < 2.0 ** -119 * abs(up) * (1 + 2.0 ** -8)).all()
