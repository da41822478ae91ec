"""Tokens and weights in 8 bits, and their products forward and backward, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import epilogue_cases as ec
import int8_cases as ic
from int8_cases import BACK_SHAPES, BF16, F32, SHAPES, same

pytestmark = pytest.mark.gpu

@pytest.mark.parametrize("cols", [8, 24, 264, 1000, 1024, 1032, 2048, 4096, 5000, 8192, 8200, 11008, 22016, 32768, 40000, 65536, 131072])
@pytest.mark.parametrize("scaled", [False, True])
@pytest.mark.parametrize("many", [False, True])  # the launch has another shape for more than 512 rows
def test_tokens(gpu_api, cols, scaled, many):
    T = 7 if cols < 30000 else 3
    if many:
        T = 515 if cols < 30000 else 513
    x = ic.drawn_tokens(cols, T, cols)
    x[1] = 0
    x[2, :] = 0
    x[2, cols // 2] = -3.0
    factor = torch.rand(cols, generator=torch.Generator().manual_seed(1)) + 0.01 if scaled else None
    v = x.float() * factor if scaled else x.float()
    q, s = gpu_api.quantize_tokens(x.cuda(), factor.cuda() if scaled else None)
    ref_q, ref_s = ic.rows8(v)
    same(s, ref_s)
    same(q, ref_q.to(torch.int8))


def test_tokens_on_the_border(gpu_api):
    """Ties (to even), and values that lie a last place beside one."""
    cols = 2048
    k = torch.arange(cols) % 254 - 127 + 0.5
    x = torch.stack([k.clamp(-127, 127) * 2.0 ** e for e in (-140 + 20, -100, -60, -3, 0, 40, 100, 120)])
    x[:, 0] = 127.0 * torch.tensor([2.0 ** e for e in (-140 + 20, -100, -60, -3, 0, 40, 100, 120)])
    assert torch.equal(x.to(BF16).float(), x)
    q, s = gpu_api.quantize_tokens(x.to(BF16).cuda())
    ref_q, ref_s = ic.rows8(x)
    same(s, ref_s)
    same(q, ref_q.to(torch.int8))
    assert int((ref_q % 2 == 0).sum()) > 0.9 * x.numel()  # (ties)
    # by the factors: v = (k + 1/2) s and its neighbours, for scales of all kinds of last places
    rng = np.random.default_rng(3)
    for top in (1.0, 0.37, 3e-20, 7e-37, 2.1e-38, 5e-42, 8e30):
        top = np.float32(top * (1 + rng.random()))
        s = top * np.float32(1 / 127)
        v = ((rng.integers(-127, 127, cols) + 0.5) * np.float64(s)).astype(np.float32)
        for shift in (-1, 0, 1):
            f = v if shift == 0 else np.nextafter(v, np.float32(shift * np.inf))
            f[0] = top
            f = torch.from_numpy(np.clip(f, -top, top))
            q, got_s = gpu_api.quantize_tokens(torch.ones((1, cols), dtype=BF16, device="cuda"), f.cuda())
            ref_q, ref_s = ic.rows8(f[None])
            same(got_s, ref_s)
            same(q, ref_q.to(torch.int8))


def test_tokens_without_a_scale(gpu_api):
    """Rows of zeros, of subnormal numbers, and with an infinity or a NaN; the others do not see them."""
    x = ic.drawn_tokens(5, 9, 520)
    x[0], x[2, 7], x[4, 519], x[5, 0] = 0, float("inf"), float("nan"), float("-inf")
    x[7] = torch.arange(520).float() * 2.0 ** -133
    x[8] = torch.where(torch.arange(520) % 2 == 0, 3.3e38, -1e38)
    q, s = gpu_api.quantize_tokens(x.cuda())
    ref_q, ref_s = ic.rows8(x.float())
    same(s, ref_s)
    same(q, ref_q.to(torch.int8))
    codes, scale = ic.drawn_weight(1, 528, 40)
    x = torch.nn.functional.pad(x, (0, 8))
    y = gpu_api.forward_int8(x.cuda(), codes.cuda(), scale.cuda()).cpu()
    assert torch.isnan(y[[2, 4, 5]]).all() and torch.isfinite(y[[0, 1, 3, 6, 7]]).all() and (y[0] == 0).all()
    same(y, ic.scaled(ic.products(*(ic.rows8(x.float())[0], codes)), ic.rows8(x.float())[1], scale))


@pytest.mark.parametrize("shape", [(16, 8), (1024, 264), (272, 1000), (4096, 72), (80, 8200)], ids=str)
def test_weights(gpu_api, shape):
    W = 0.02 * torch.randn(shape, generator=torch.Generator().manual_seed(2))
    W[:, 3] = 0
    codes, scale = gpu_api.quantize_int8(W.cuda())
    ref, ref_s = ic.weight8(W)
    same(scale, ref_s)
    same(codes, ref)


@pytest.mark.parametrize("layer", [(1024, 264, 4, 32), (256, 72, 2, 64), (512, 136, 3, 32), (96, 520, 4, 48)], ids=str)
def test_deployed_layer(gpu_api, layer):
    d_in, d_out, bits, group = layer
    triple = ec.drawn_layer(4, 1, d_in, d_out, bits, group)[:3]
    desc = gpu_api.make_desc(d_in, d_out, bits, group)
    codes, alpha, beta = triple
    got, scale = gpu_api.deploy_int8(desc, gpu_api.pack(desc, codes.cuda()), alpha.cuda(), beta.cuda())
    rows = lambda t: t.double().repeat_interleave(group, 0)  # noqa: E731
    # (alpha code and the sum with beta need 24 + 4 + 24 bits at most where their exponents are near: 64 bits hold them)
    ref, ref_s = ic.weight8((codes.double() * rows(alpha) + rows(beta)).to(F32))
    same(scale, ref_s)
    same(got, ref)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(gpu_api, shape):
    T, d_in, d_out = shape
    codes, scale = ic.drawn_weight(1, d_in, d_out)
    x = ic.drawn_tokens(2, T, d_in)
    q, s = ic.rows8(x.float())
    acc = ic.products(q, codes)
    ref = ic.scaled(acc, s, scale)
    w = (codes.cuda(), scale.cuda())
    same(gpu_api.forward_int8(x.cuda(), *w), ref)
    same(gpu_api.forward_int8(x.cuda(), *w, out_dtype=BF16), ref.to(BF16))
    tokens8 = gpu_api.quantize_tokens(x.cuda())
    same(gpu_api.forward_int8(tokens8, *w), ref)
    for out_dtype in (F32, BF16):
        bias, mul, residual = ec.extras(3, T, d_out, out_dtype)
        for k, act in enumerate(ec.ACTS):
            use = [True] * 3 if k % 2 else [(k + j) % 2 == 0 for j in range(3)]
            kw = dict(bias=bias.cuda() if use[0] else None, mul=mul.cuda() if use[1] else None, residual=residual.cuda() if use[2] else None)
            y, z = gpu_api.forward_int8(tokens8, *w, act=act, keep_z=True, out_dtype=out_dtype, **kw)
            z64 = acc.to(F32).mul(s[:, None]).double() * scale.double()
            off = 2.0 ** -24 * z64.abs()                        # a product's rounding, or none where the sum follows in one step
            if use[0]:
                z64 = z64 + bias.double()
                off = off + 2.0 ** -24 * z64.abs()
            bad = (z.cpu().double() - z64).abs() > off + 2.0 ** -8 * (z64.abs() + off)
            assert not bad.any()
            y64, tol = ec.after(z64, act, mul if use[1] else None, residual if use[2] else None)
            tol = tol + 1.2 * off * (mul.double().abs() if use[1] else 1.0)   # (no slope is above 1.13)
            if out_dtype == BF16:
                tol = tol + 2.0 ** -8 * (y64.abs() + tol)
            bad = ((y.cpu().double() - y64).abs() > tol) | ~torch.isfinite(y.cpu())
            assert not bad.any(), (act, int(bad.sum()), bad.nonzero()[0].tolist())
        stream = residual.cuda().clone()                        # the residual stream in place, with the sums' exact product
        y = gpu_api.forward_int8(tokens8, *w, residual=stream, y=stream)
        assert y is stream
        same(stream, gpu_api.forward_int8(tokens8, *w, residual=residual.cuda(), out_dtype=out_dtype))


@pytest.mark.parametrize("shape", SHAPES + BACK_SHAPES, ids=str)
def test_backward(gpu_api, shape):
    T, d_in, d_out = shape
    codes, scale = ic.drawn_weight(3, d_in, d_out)
    dy = ic.drawn_tokens(4, T, d_out)
    v = dy.float() * scale
    q, s = ic.rows8(v)
    acc = ic.products(q, codes.T.contiguous())
    ref = ic.scaled(acc, s)
    w = (codes.cuda(), scale.cuda())
    dx = gpu_api.backward_int8(dy.cuda(), *w)
    same(dx, ref)
    same(gpu_api.backward_int8(dy.cuda(), *w, dx_dtype=BF16), ref.to(BF16))
    # the formula without dy's rounding: half a scale an element of v, times the codes
    exact = v.double() @ codes.double()
    bound = 0.5 * s[:, None].double() * codes.double().abs().sum(0) * (1 + 1e-6) + 2.0 ** -22 * ref.double().abs()
    assert ((dx.cpu().double() - exact).abs() <= bound).all()
    for dtype in (F32, BF16):
        r = torch.randn((T, d_in), generator=torch.Generator().manual_seed(9)).to(dtype)
        got = gpu_api.backward_int8(dy.cuda(), *w, residual=r.cuda(), dx_dtype=dtype)
        # one rounding of product and sum, or two (2^-24 of the product more)
        ref64 = acc * s[:, None].double() + r.double()
        tol = 2.0 ** -24 * (2 * ref.double().abs() + ref64.abs())
        if dtype == BF16:
            tol = tol + 2.0 ** -8 * (ref64.abs() + tol)
        assert ((got.cpu().double() - ref64).abs() <= tol).all()
        stream = r.cuda().clone()
        same(gpu_api.backward_int8(dy.cuda(), *w, residual=stream, dx=stream), got)


@pytest.mark.parametrize("shape", [(4, 48, 24), (40, 528, 72), (300, 272, 264)], ids=str)
def test_gradient_is_the_forwards_difference(gpu_api, shape):
    """On whole numbers whose rows' largest magnitude is 127, nothing rounds: L(x + d) - L(x - d) = 2 <dx, d> for L = <dy, y(x)>."""
    T, d_in, d_out = shape
    g = torch.Generator().manual_seed(6)
    whole = lambda *n, top: torch.randint(-top, top + 1, n, generator=g).float()  # noqa: E731
    codes = whole(d_out, d_in, top=127).to(torch.int8).cuda()
    scale = torch.full((d_out,), 2.0 ** -9, device="cuda")
    x, d, dy = whole(T, d_in, top=60), whole(T, d_in, top=60), whole(T, d_out, top=126)
    x[:, 0], d[:, 0], dy[:, 0] = 127, 0, -127
    y = lambda v: gpu_api.forward_int8(v.to(BF16).cuda(), codes, scale).double().cpu()  # noqa: E731
    dx = gpu_api.backward_int8(dy.to(BF16).cuda(), codes, scale).double().cpu()
    assert float((dy.double() * (y(x + d) - y(x - d))).sum()) == 2 * float((dx * d.double()).sum())


@pytest.mark.parametrize("size", ic.LARGE + ic.MIXED, ids=str)
def test_large_tiles(gpu_api, size):
    """Both directions of a product, with an epilogue, against 64 bits on the GPU."""
    T, depth, width = size
    codes, scale = (t.cuda() for t in ic.drawn_weight(7, depth, width))
    q, s = gpu_api.quantize_tokens(ic.drawn_tokens(8, T, depth).cuda())
    acc = q.double() @ codes.double().T
    ref = acc.to(F32) * s[:, None] * scale
    same(gpu_api.forward_int8((q, s), codes, scale), ref)
    bias, mul, residual = (t.cuda() for t in ec.extras(3, T, width, BF16))
    y, z = gpu_api.forward_int8((q, s), codes, scale, bias=bias, act="silu", mul=mul, residual=residual, keep_z=True, out_dtype=BF16)
    z64 = (acc.to(F32) * s[:, None]).double() * scale.double() + bias.double()
    off = 2.0 ** -24 * (ref.double().abs() + z64.abs())
    assert ((z.double() - z64).abs() <= off + 2.0 ** -8 * (z64.abs() + off)).all()
    y64, tol = ec.after(z64, "silu", mul, residual)
    tol = tol + 1.2 * off * mul.double().abs()
    assert ((y.double() - y64).abs() <= tol + 2.0 ** -8 * (y64.abs() + tol)).all()
    dy = ic.drawn_tokens(9, T, depth).cuda()                    # [tokens, d_out], d_out = depth here
    w, ws = codes.T.contiguous(), torch.rand(depth, device="cuda") + 0.5
    q, s = gpu_api.quantize_tokens(dy, ws)
    acc = q.double() @ w.double()
    same(gpu_api.backward_int8(dy, w, ws), acc.to(F32) * s[:, None])
    r = torch.randn((T, width), device="cuda").to(BF16)
    ref64 = acc * s[:, None].double() + r.double()
    tol = 2.0 ** -24 * (2 * (acc * s[:, None].double()).abs() + ref64.abs())
    got = gpu_api.backward_int8(dy, w, ws, residual=r, dx_dtype=BF16)
    assert ((got.double() - ref64).abs() <= tol + 2.0 ** -8 * (ref64.abs() + tol)).all()


def test_largest_sums(gpu_api):
    """The longest rows of the largest codes: the sums reach 127^2 131072, a 32-bit number."""
    n = 131072
    x = torch.ones((2, n), dtype=BF16, device="cuda")
    x[1] = -1
    codes = torch.full((8, n), 127, dtype=torch.int8, device="cuda")
    scale = torch.ones(8, device="cuda")
    s = torch.full((2,), np.float32(1 / 127))
    acc = torch.tensor([[127.0 * 127 * n], [-127.0 * 127 * n]]).expand(2, 8)
    same(gpu_api.forward_int8(x, codes, scale), ic.scaled(acc.double(), s, scale.cpu()))
    back = gpu_api.backward_int8(x, codes.T.contiguous()[:, :8].contiguous().repeat(1, 2), torch.ones(n, device="cuda"))
    same(back, ic.scaled(torch.tensor([[127.0 * 127 * n], [-127.0 * 127 * n]]).expand(2, 16).double(), s))


def test_one_workspace_for_every_shorter_batch(gpu_api):
    codes, scale = ic.drawn_weight(1, 1040, 264)
    w = (codes.cuda(), scale.cuda())
    n = gpu_api.int8_workspace_bytes(700, 1040, 264, gpu_api.OP_FORWARD)
    m = gpu_api.int8_workspace_bytes(700, 1040, 264, gpu_api.OP_BACKWARD)
    ws = torch.full((max(n, m),), 255, dtype=torch.uint8, device="cuda")
    x, dy = ic.drawn_tokens(2, 700, 1040).cuda(), ic.drawn_tokens(3, 700, 264).cuda()
    y, dx = gpu_api.forward_int8(x, *w), gpu_api.backward_int8(dy, *w)
    for T in (700, 1, 5, 16, 17, 64, 100, 300, 513):
        assert n >= gpu_api.int8_workspace_bytes(T, 1040, 264, gpu_api.OP_FORWARD)
        assert m >= gpu_api.int8_workspace_bytes(T, 1040, 264, gpu_api.OP_BACKWARD)
        same(gpu_api.forward_int8(x[:T], *w, ws=ws[:n]), y[:T])
        same(gpu_api.backward_int8(dy[:T], *w, ws=ws[:m]), dx[:T])
