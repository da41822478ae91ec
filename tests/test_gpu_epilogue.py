"""The linear with an epilogue and the epilogue's backward on the GPU, in 64 bits from the definition and, for the epilogue
itself, from the sums that the plain call returns in fp32 (the same kernels', so the same sums)."""
import math

import numpy as np
import pytest
import torch

import epilogue_cases as ec
from helpers import TOL, record

pytestmark = pytest.mark.gpu

S = 0.25
BF16, F32 = torch.bfloat16, torch.float32


class Layer:
    def __init__(self, api, seed, T, d_in, d_out, bits, group, rank=0):
        self.api, self.group = api, group
        self.host = ec.drawn_layer(seed, T, d_in, d_out, bits, group, rank)
        codes, alpha, beta, x, A, B = (None if t is None else t.cuda() for t in self.host)
        self.desc = api.make_desc(d_in, d_out, bits, group, rank, S if rank else 0.0)
        self.triple = (api.pack(self.desc, codes), alpha, beta)
        self.x, self.A, self.B = x, A, B

    def z64(self):
        codes, alpha, beta, x, A, B = self.host
        return ec.linear64(codes, alpha, beta, x, self.group, A, B, S)

    def plain(self):
        return self.api.forward(self.desc, self.x, *self.triple, self.A, self.B)

    def call(self, **kw):
        return self.api.forward_epilogue(self.desc, self.x, *self.triple, self.A, self.B, **kw)


def within(got, ref, tol, out_dtype):
    """|got - ref| <= tol, and half a step of y's type more."""
    tol = tol + (2.0 ** -8 * (ref.abs() + tol) if out_dtype == BF16 else 0)
    bad = ((got.cpu().double() - ref).abs() > tol) | ~torch.isfinite(got.cpu())
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[0].tolist())


def check_all(layer, T, d_out, tol, seed=1):
    """Every activation and combination's y, from the plain call's sums; and y from the definition."""
    base = layer.plain().cpu()
    z64 = layer.z64()
    err = float((base.double() - z64).abs().max() / z64.abs().max())
    assert err <= tol
    for out_dtype in (F32, BF16):
        bias, mul, residual = ec.extras(seed, T, d_out, out_dtype)
        b, m, r = bias.cuda(), mul.cuda(), residual.cuda()
        for k, act in enumerate(ec.ACTS):
            z = (base + bias).double()                      # fp32, as the kernel has it
            y, zk, kept = layer.call(bias=b, act=act, mul=m, residual=r, keep_z=True, out_dtype=out_dtype)
            assert kept is None and torch.equal(zk.cpu(), (base + bias).to(BF16))
            within(y, *ec.after(z, act, mul, residual), out_dtype)
            use = [(k + j) % 2 for j in range(3)]           # some of them
            y = layer.call(bias=b if use[0] else None, act=act, mul=m if use[1] else None, residual=r if use[2] else None,
                           out_dtype=out_dtype)
            within(y, *ec.after((base + bias).double() if use[0] else base.double(), act, mul if use[1] else None,
                                residual if use[2] else None), out_dtype)
        # the residual stream in place
        stream = r.clone()
        y = layer.call(act="silu", residual=stream, y=stream)
        assert y is stream and torch.equal(stream, layer.call(act="silu", residual=r, out_dtype=out_dtype))
        assert torch.equal(layer.call(out_dtype=out_dtype), base.to(out_dtype).cuda())  # nothing to apply: the plain call
        assert torch.equal(b.cpu(), bias) and torch.equal(m.cpu(), mul) and torch.equal(r.cpu(), residual)
    return err


@pytest.mark.parametrize("shape", ec.STREAMED, ids=str)
def test_few_tokens(gpu_api, shape):
    T, d_in, d_out, bits, group = shape
    record(f"epilogue {shape}", z=check_all(Layer(gpu_api, 3, *shape), T, d_out, 1e-5))


@pytest.mark.parametrize("shape", ec.MID, ids=str)
def test_mid_tokens(gpu_api, shape):
    record(f"epilogue {shape}", z=check_all(Layer(gpu_api, 4, *shape), shape[0], shape[2], TOL))


@pytest.mark.parametrize("shape", sorted(ec.DENSE), ids=str)
def test_dense(gpu_api, shape):
    record(f"epilogue {shape}", z=check_all(Layer(gpu_api, 5, *shape), shape[0], shape[2], TOL))


@pytest.mark.parametrize("shape", [(1, 1024, 520, 4, 32), (16, 1024, 520, 2, 32), (64, 1024, 264, 4, 32), (300, 512, 1032, 3, 64)], ids=str)
def test_adapted_and_kept(gpu_api, shape):
    """With an adapter (any number of tokens on the dense product), and what the forward keeps for the backward."""
    layer = Layer(gpu_api, 6, *shape, rank=24)
    record(f"epilogue {shape} rank 24", z=check_all(layer, shape[0], shape[2], TOL))
    y0, kept0 = gpu_api.forward_keep(layer.desc, layer.x, *layer.triple, layer.A, layer.B)
    y, z, kept = layer.call(act="relu", keep=True)
    assert z is None and torch.equal(y, y0.clamp(min=0))
    dy = torch.randn((shape[0], shape[2]), device="cuda").to(BF16)
    got, ref = (gpu_api.backward_kept(layer.desc, dy, k, *layer.triple, layer.A, layer.B) for k in (kept, kept0))
    assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("T", [1, 4, 5, 24, 64, 200])
def test_deployed(gpu_api, T):
    layer = Layer(gpu_api, 7, T, 1024, 1032, 4, 64)
    dep = gpu_api.deploy(layer.desc, *layer.triple)
    packed = layer.triple[0] if T > 4 else None
    base = gpu_api.forward_deployed(layer.desc, layer.x, dep, packed).cpu()
    for out_dtype in (F32, BF16):
        bias, mul, residual = ec.extras(2, T, 1032, out_dtype)
        for act in ec.ACTS:
            y = gpu_api.forward_deployed_epilogue(layer.desc, layer.x, dep, packed, bias=bias.cuda(), act=act, mul=mul.cuda(),
                                                  residual=residual.cuda(), out_dtype=out_dtype)
            within(y, *ec.after((base + bias).double(), act, mul, residual), out_dtype)
        assert torch.equal(gpu_api.forward_deployed_epilogue(layer.desc, layer.x, dep, packed), base.cuda())


def test_extreme_activations(gpu_api):
    """Values at which an exponential overflows or a product of zero and infinity lurks, by way of the bias; a NaN stays."""
    layer = Layer(gpu_api, 8, 3, 256, 64, 4, 32)
    layer.x.zero_()
    special = [0.0, -0.0, 1e-30, -1e-30, 20.0, -20.0, 88.0, -88.0, 89.5, -89.5, 104.0, -104.0, 1e4, -1e4, 1e19, -1e19, 3e38, -3e38,
               math.inf, math.nan]
    bias = torch.tensor((special * 4)[:64])
    for act in ec.ACTS:
        y, z, _ = layer.call(bias=bias.cuda(), act=act, keep_z=True)
        ref, tol = ec.after(bias.double().expand(3, 64), act)
        y = y.cpu().double()
        nan = torch.isnan(bias).expand(3, 64)
        assert torch.equal(torch.isnan(y), nan), act
        inf = torch.isinf(bias).expand(3, 64)
        assert (y[inf] == math.inf).all()
        ok = ~nan & ~inf
        # (below 1e-30 fp32's exponential has run out: the reference's remainder is smaller than any use)
        assert ((y - ref)[ok].abs() <= torch.where(torch.isfinite(tol[ok]), tol[ok], torch.zeros_like(tol[ok])) + 1e-30).all(), act
        dy = torch.ones((3, 64), device="cuda")
        dz, _, db = gpu_api.epilogue_backward(dy, z, act, want_dbias=True)
        zz = z.cpu().double()
        slope = ec.act64(zz.clamp(-1e3, 1e3), act)[1].float()
        live = ~torch.isnan(zz)
        assert torch.isfinite(dz.cpu()[live]).all(), act
        assert ((dz.cpu().double() - slope.double())[live].abs() <= 2.0 ** -8 * slope.double()[live].abs() + 1e-6).all(), act


BACK = [(1, 8), (1, 520), (3, 64), (7, 1032), (64, 1024), (100, 24), (257, 136), (1531, 2056), (40000, 8)]


@pytest.mark.parametrize("dy_dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("act", ec.ACTS)
@pytest.mark.parametrize("shape", BACK, ids=str)
def test_backward(gpu_api, shape, act, dy_dtype):
    """dz, dmul and dbias from the formula in 64 bits.  fp32's share: the exponent's rounding (as in the forward) and a few half
    steps; where the slope is a difference its terms set the scale (all slopes here are below 1.2, their terms below 1.2 +
    |z| s (1 - s) ...: 4 in all).  dbias adds rows / blocks values in a row: 2^-24 sqrt(rows) of their squares' root, times 8."""
    T, cols = shape
    g = torch.Generator().manual_seed(T * 31 + cols)
    dy = torch.randn((T, cols), generator=g).to(dy_dtype)
    z = (2.0 * torch.randn((T, cols), generator=g)).to(BF16)
    mul = torch.randn((T, cols), generator=g).to(BF16)
    z[0, :4] = torch.tensor([0.0, -0.0, 30.0, -30.0])
    value, slope, exponent = ec.act64(z.double(), act)
    part = 2.0 ** -24 * (16 + 4 * exponent.clamp(max=90)) * 4
    for m, acc in ((mul, True), (None, False)):
        factor = dy.double() * (1.0 if m is None else m.double())
        start = torch.randn(cols, generator=g)
        db = start.cuda() if acc else None
        dz, dmul, dbias = gpu_api.epilogue_backward(dy.cuda(), z.cuda(), act, mul=None if m is None else m.cuda(), want_dbias=True,
                                                    dbias=db, accumulate=acc)
        ref = factor * slope
        within(dz, ref, part * factor.abs() + 1e-36, BF16)
        if m is None:
            assert dmul is None
        else:
            within(dmul, dy.double() * value, part * (dy.double() * value).abs() + 1e-36, BF16)
        total = ref.sum(0) + (start.double() if acc else 0)
        tol = (part * factor.abs()).sum(0) + 8 * 2.0 ** -24 * math.sqrt(T) * ref.square().sum(0).sqrt() + 2.0 ** -24 * total.abs() + 1e-36
        assert ((dbias.cpu().double() - total).abs() <= tol).all()
        assert not acc or dbias is db
        again = gpu_api.epilogue_backward(dy.cuda(), z.cuda(), act, mul=None if m is None else m.cuda(), want_dbias=True,
                                          dbias=start.cuda() if acc else None, accumulate=acc)
        assert torch.equal(again[0], dz) and torch.equal(again[2], dbias)


def test_backward_forms(gpu_api):
    """Outputs alone, in place, and without z."""
    g = torch.Generator(device="cuda").manual_seed(3)
    dy, z, mul = (torch.randn((37, 264), generator=g, device="cuda").to(BF16) for _ in range(3))
    dz, dmul, db = gpu_api.epilogue_backward(dy, z, "silu", mul=mul, want_dbias=True)
    only, dmul1, db1 = gpu_api.epilogue_backward(dy, z, "silu", mul=mul, want_dz=False, want_dbias=True)
    assert only is None and torch.equal(dmul1, dmul) and torch.equal(db1, db)
    inplace = dy.clone()
    assert gpu_api.epilogue_backward(inplace, z, "silu", mul=mul, dz=inplace)[0] is inplace and torch.equal(inplace, dz)
    copy, _, db = gpu_api.epilogue_backward(dy, want_dbias=True)   # a bias alone: dz is dy
    assert torch.equal(copy, dy)
    assert ((db.double() - dy.double().sum(0)).abs() <= 37 * 2.0 ** -24 * dy.double().abs().sum(0)).all()
    assert torch.equal(gpu_api.epilogue_backward(dy, mul=mul, z=z)[1], (dy.float() * z.float()).to(BF16))


def test_backward_of_one_row_of_many_columns(gpu_api):
    """As many columns as are taken, 2^29: the launch has 2^31 threads."""
    cols = 2 ** 29
    dy = torch.randn(1 << 20, device="cuda").to(BF16).repeat(512).view(1, cols)
    dz, none, db = gpu_api.epilogue_backward(dy, want_dbias=True)
    assert none is None and torch.equal(dz, dy) and torch.equal(db.to(BF16), dy[0])


@pytest.mark.parametrize("act", ec.ACTS)
def test_gradients_against_differences(gpu_api, act):
    """dbias and the bias's differences in sum(dy * y), on a layer whose sums are exact.  A difference over +-h is off by h^2 / 6 of
    the third derivative (below 2 for these; relu's corner: skipped where z is within h of it); the slope is taken at z
    rounded to bf16 (2^-8 |z| of the second derivative, below 1.2); y's fp32 rounding is over 2 h."""
    T, d_out, h = 6, 72, 2.0 ** -5
    layer = Layer(gpu_api, 9, T, 256, d_out, 4, 32)
    bias, mul, residual = ec.extras(4, T, d_out, F32)
    dy = torch.randn((T, d_out), generator=torch.Generator().manual_seed(5)).to(BF16)
    call = lambda b: layer.call(bias=b.cuda(), act=act, mul=mul.cuda(), residual=residual.cuda()).cpu().double()  # noqa: E731
    y0, z, _ = layer.call(bias=bias.cuda(), act=act, mul=mul.cuda(), residual=residual.cuda(), keep_z=True)
    _, dmul, dbias = gpu_api.epilogue_backward(dy.cuda(), z, act, mul=mul.cuda(), want_dbias=True)
    diff = (dy.double() * (call(bias + h) - call(bias - h)) / (2 * h)).sum(0)
    z = z.cpu().double()
    weight = (dy.double() * mul.double()).abs()
    tol = (weight * (h * h / 3 + 2.0 ** -8 * z.abs() * 1.2)).sum(0) + (dy.double().abs() * y0.cpu().double().abs() * 2.0 ** -20 / h).sum(0)
    skip = (z.abs() <= 2 * h).any(0) if act == "relu" else torch.zeros(d_out, dtype=torch.bool)
    assert skip.sum() < d_out / 2
    assert ((dbias.cpu().double() - diff).abs() <= tol)[~skip].all()
    # y is linear in mul: its difference over one is exact up to the roundings
    one = layer.call(bias=bias.cuda(), act=act, mul=(0 * mul + 1).cuda()).cpu().double()
    within(dmul, dy.double() * one, dy.double().abs() * (2.0 ** -8 * z.abs() * 1.3 + 1e-5 * one.abs()), BF16)


def test_streams_and_captured_replays(gpu_api):
    """On another stream, and captured: forward (split and streamed forms) and backward replayed with eager calls between."""
    for shape, rank in (((3, 1024, 520, 4, 32), 0), ((40, 4096, 2056, 4, 32), 0), ((65, 1024, 264, 3, 32), 8), ((300, 512, 1032, 4, 32), 8)):
        T, _, d_out, _, _ = shape
        layer = Layer(gpu_api, 10, *shape, rank=rank)
        bias, mul, residual = (t.cuda() for t in ec.extras(6, T, d_out, BF16))
        ws = torch.zeros(gpu_api.workspace_bytes(layer.desc, T, gpu_api.OP_FORWARD), dtype=torch.uint8, device="cuda")
        bws = torch.empty(gpu_api.load().qalora_epilogue_backward_workspace_bytes(T, d_out), dtype=torch.uint8, device="cuda")
        y, z, dz, dm = (torch.empty((T, d_out), dtype=BF16, device="cuda") for _ in range(4))
        db = torch.zeros(d_out, device="cuda")

        def step(out):
            y, z, dz, dm, db = out
            layer.call(bias=bias, act="silu", mul=mul, residual=residual, keep_z=True, y=y, z=z, ws=ws)
            gpu_api.epilogue_backward(y, z, "silu", mul=mul, dz=dz, dmul=dm, dbias=db, accumulate=False, ws=bws)

        eager = [torch.empty_like(t) for t in (y, z, dz, dm, db)]
        step(eager)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step([y, z, dz, dm, db])
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, z, dz, dm, db), eager))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step([y, z, dz, dm, db])
        for k in range(4):
            layer.x.copy_(torch.randn(layer.x.shape, device="cuda").to(BF16))   # new inputs in the captured buffers
            for t in (y, z, dz, dm, db):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            step(eager)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((y, z, dz, dm, db), eager))
        assert gpu_api.streaming_status(ws) == 0 if rank == 0 else True


def test_a_timed_out_wait_stays_loud(gpu_api):
    """The NaN that a few-token kernel leaves where its wait ran out must come through every epilogue: by a NaN in x."""
    layer = Layer(gpu_api, 11, 3, 1024, 520, 4, 32)
    layer.x[1, 5] = math.nan
    for act in ec.ACTS:
        y = layer.call(act=act, out_dtype=BF16)
        assert torch.isnan(y[1]).all() and not torch.isnan(y[0]).any() and not torch.isnan(y[2]).any()


def test_refusals(gpu_api):
    layer = Layer(gpu_api, 12, 5, 256, 64, 4, 32)
    T, n = 5, 64
    ok = dict(bias=torch.zeros(n), mul=torch.zeros((T, n), dtype=BF16), residual=torch.zeros((T, n)))
    for name, bad in (("bias", torch.zeros(n + 1)), ("bias", torch.zeros(n, dtype=BF16)), ("mul", torch.zeros((T, n))),
                      ("mul", torch.zeros((T + 1, n), dtype=BF16)), ("residual", torch.zeros((T, n), dtype=BF16)),
                      ("residual", torch.zeros((n, T)).T), ("residual", torch.zeros((1, n)))):
        with pytest.raises(ValueError, match=name):
            layer.call(**{name: bad.cuda()})
        with pytest.raises(ValueError, match=name):
            layer.call(**{name: ok[name]})   # on the host
    with pytest.raises(ValueError, match="act"):
        layer.call(act="tanh")
    with pytest.raises(ValueError, match="z: dtype"):
        layer.call(z=torch.zeros((T, n), device="cuda"), keep_z=True)
    with pytest.raises(ValueError, match="z: given"):
        layer.call(z=torch.zeros((T, n), device="cuda", dtype=BF16))
    with pytest.raises(ValueError, match="kept: given"):
        layer.call(kept=torch.zeros(4096, device="cuda", dtype=torch.uint8))
    with pytest.raises(gpu_api.QaloraError):
        layer.call(keep=True)                # nothing to keep without an adapter
    dy = torch.zeros((T, n), device="cuda", dtype=BF16)
    z = torch.zeros((T, n), device="cuda", dtype=BF16)
    with pytest.raises(gpu_api.QaloraError):
        gpu_api.epilogue_backward(dy, None, "silu")
    with pytest.raises(gpu_api.QaloraError):
        gpu_api.epilogue_backward(dy[:, :60].contiguous(), z[:, :60].contiguous(), "silu")
    with pytest.raises(ValueError, match="dmul"):
        gpu_api.epilogue_backward(dy, z, "silu", dmul=dy)
    with pytest.raises(ValueError, match="z"):
        gpu_api.epilogue_backward(dy, z.float(), "silu")
    with pytest.raises(ValueError, match="dy"):
        gpu_api.epilogue_backward(dy.half(), z, "silu")
    with pytest.raises(ValueError, match="dy"):
        gpu_api.epilogue_backward(dy.T, z, "silu")
