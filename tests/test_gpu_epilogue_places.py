"""Outputs of the calls with an epilogue that take the place of an operand, where that is allowed."""
import pytest
import torch

import epilogue_cases as ec

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dy_dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(5, 64), (700, 264)], ids=str)
def test_backward_in_the_place_of_its_operands(gpu_api, shape, dy_dtype):
    g = torch.Generator().manual_seed(5)
    host = [torch.randn(shape, generator=g).to(t) for t in (dy_dtype, BF16, BF16)]
    dz, dmul, db = gpu_api.epilogue_backward(*(t.cuda() for t in host[:2]), "gelu", mul=host[2].cuda(), want_dbias=True)
    for a, b in ((0, 1), (1, 0), (2, 1), (1, 2), (0, 2), (2, 0)):   # dz and dmul at dy (0), z (1) or mul (2)
        if dy_dtype == F32 and 0 in (a, b):
            continue
        at = [t.cuda() for t in host]
        got = gpu_api.epilogue_backward(at[0], at[1], "gelu", mul=at[2], dz=at[a], dmul=at[b], want_dbias=True)
        assert got[0] is at[a] and got[1] is at[b]
        assert torch.equal(got[0], dz) and torch.equal(got[1], dmul) and torch.equal(got[2], db)
    if dy_dtype == F32:
        dy = host[0].cuda()
        over = dy.view(BF16).view(-1)[: dz.numel()].view(shape)
        with pytest.raises(gpu_api.QaloraError) as e:
            gpu_api.epilogue_backward(dy, host[1].cuda(), "gelu", dz=over)
        assert e.value.status == gpu_api.EINVAL and torch.equal(dy.cpu(), host[0])


@pytest.mark.parametrize("rank", [0, 24])
@pytest.mark.parametrize("shape", [(1, 1024, 1024, 4, 32), (13, 512, 512, 2, 32), (20, 1024, 1024, 4, 32), (40, 4096, 2056, 4, 32),
                                   (65, 1024, 264, 3, 32), (300, 512, 1032, 4, 32)], ids=str)
def test_forward_in_the_place_of_mul_or_residual(gpu_api, shape, rank):
    """y at a bf16 mul, at the residual, and at both at once, for each kernel that has an epilogue; refused over x and shifted."""
    T, d_in, d_out, bits, group = shape
    codes, alpha, beta, x, A, B = (None if t is None else t.cuda() for t in ec.drawn_layer(3, *shape, rank))
    desc = gpu_api.make_desc(d_in, d_out, bits, group, rank, 0.25 if rank else 0.0)
    packed = gpu_api.pack(desc, codes)
    bias, mul, residual = (t.cuda() for t in ec.extras(4, T, d_out, BF16))

    def call(mul, residual, **kw):
        return gpu_api.forward_epilogue(desc, x, packed, alpha, beta, A, B, bias=bias, act="silu", mul=mul, residual=residual,
                                        out_dtype=BF16, **kw)

    ref, both = call(mul, residual), call(mul, mul)
    place = mul.clone()
    assert call(place, residual, y=place) is place and torch.equal(place, ref)
    place = residual.clone()
    assert call(mul, place, y=place) is place and torch.equal(place, ref)
    place = mul.clone()
    assert call(place, place, y=place) is place and torch.equal(place, both)
    if d_in == d_out:
        with pytest.raises(gpu_api.QaloraError) as e:
            call(mul, x, y=x)
        assert e.value.status == gpu_api.EINVAL
    room = torch.zeros((T + 1, d_out), dtype=BF16, device="cuda")
    for kw in (dict(mul=room[1:], residual=residual), dict(mul=mul, residual=room[1:])) if T > 1 else ():   # by a row
        with pytest.raises(gpu_api.QaloraError) as e:
            call(y=room[:-1], **kw)
        assert e.value.status == gpu_api.EINVAL
    assert not room.any()


@pytest.mark.parametrize("shape", [(3, 1024, 520, 4, 32), (2, 1024, 520, 3, 32), (13, 512, 520, 2, 32), (20, 1024, 1032, 4, 32), (40, 4096, 2056, 4, 32),
                                   (65, 1024, 264, 3, 32), (130, 512, 1032, 4, 32)], ids=str)
def test_a_row_that_is_nan_stays_nan(gpu_api, shape):
    """NaN sums, as a kernel leaves them where a wait ran out (no call can bring that about; here by a NaN in x), come through
    every activation, a mul of zeros, a residual in place and z; the other rows are those of the same call without the NaN."""
    T, d_in, d_out, bits, group = shape
    codes, alpha, beta, x, _, _ = (None if t is None else t.cuda() for t in ec.drawn_layer(5, *shape))
    desc = gpu_api.make_desc(d_in, d_out, bits, group)
    packed = gpu_api.pack(desc, codes)
    bias, mul, residual = (t.cuda() for t in ec.extras(6, T, d_out, BF16))
    mul[:, ::2] = 0
    at = T // 2
    sick = x.clone()
    sick[at, 5] = float("nan")
    others = [t for t in range(T) if t != at]
    for act in ec.ACTS:
        def call(x):
            stream = residual.clone()
            return gpu_api.forward_epilogue(desc, x, packed, alpha, beta, bias=bias, act=act, mul=mul, residual=stream, keep_z=True,
                                            out_dtype=BF16, y=stream)[:2]
        for got, clean in zip(call(sick), call(x)):
            assert torch.isnan(got[at]).all() and torch.equal(got[others], clean[others]), act


@pytest.mark.parametrize("act", ec.ACTS)
def test_activations_in_fp32(gpu_api, act):
    """act(z) in an fp32 y to the documented (8 + 4 e) 2^-24 of itself: v log2(e) rounded and its constant (2 half steps of e and 1 of the
    exponent's conversion, below 4 e in all), the exponential, the sum, the reciprocal and the products (2 + 1 + 2 + 2, below 8)."""
    n, g = 1 << 16, torch.Generator().manual_seed(9)
    packed = gpu_api.pack(gpu_api.make_desc(64, n, 4, 32), torch.zeros((64, n), dtype=torch.uint8, device="cuda"))
    zero, x = torch.zeros((2, n), device="cuda"), torch.zeros((1, 64), dtype=BF16, device="cuda")
    for low, high in ((-70, -30), (-30, -8), (-8, -1), (-1, 1), (1, 8), (8, 70)):
        z = low + (high - low) * torch.rand(n, generator=g)
        y = gpu_api.forward_epilogue(gpu_api.make_desc(64, n, 4, 32), x, packed, zero, zero, bias=z.cuda(), act=act)[0].cpu().double()
        ref, _, e = ec.act64(z.double(), act)
        assert ((y - ref).abs() <= (8 + 4 * e) * 2.0 ** -24 * ref.abs() + 1e-30).all(), (low, high)
