"""The 8-bit operators as they are used: a frozen MLP block forward and backward with what the backward needs kept in 8 bits, then its
serving of single tokens; captured into graphs and replayed; on several streams; with bytes on each side of every output; far operands."""
import ctypes

import pytest
import torch

import epilogue_cases as ec
import int8_cases as ic
from int8_cases import BF16, F32, same

pytestmark = pytest.mark.gpu


class Block:
    """x + down(silu(gate x) * (up x)), gate and up as one weight; frozen, in 8 bits."""

    def __init__(self, api, d, ff, seed=1):
        self.api, self.d, self.ff = api, d, ff
        self.host_gu, self.host_down = ic.drawn_weight(seed, d, 2 * ff), ic.drawn_weight(seed + 1, ff, d)
        self.gu = [t.cuda() for t in self.host_gu]
        self.down = [t.cuda() for t in self.host_down]

    def forward(self, x, out_dtype=BF16):
        api = self.api
        gu = api.forward_int8(api.quantize_tokens(x), *self.gu, out_dtype=BF16)
        tokens8, kept = api.swiglu_forward_int8(gu, self.ff, keep=True)
        y = api.forward_int8(tokens8, *self.down, residual=x if out_dtype == BF16 else x.float(), out_dtype=out_dtype)
        return y, gu, tokens8, kept

    def backward(self, dy, kept):
        api = self.api
        dh = api.backward_int8(dy, *self.down, dx_dtype=BF16)
        dgu = api.swiglu_backward_kept8(dh, kept, self.ff)
        return dh, dgu, api.backward_int8(dgu, *self.gu, residual=dy, dx_dtype=BF16)


def bf16_near(got, ref, tol):
    """One rounding to bf16 of something within tol of ref."""
    bad = ~((got.cpu().double() - ref).abs() <= tol + 2.0 ** -8 * (ref.abs() + tol))
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[0].tolist())


def linear(x, codes, scale):
    """Forward of the definition at x, bf16 on the CPU, in fp32 steps."""
    q, s = ic.rows8(x.float())
    return ic.scaled(ic.products(q, codes), s, scale)


def back(dy, codes, scale):
    q, s = ic.rows8(dy.float() * scale)
    return ic.scaled(ic.products(q, codes.T.contiguous()), s)


def sigmoid_parts(v, ff):
    g, u = v[:, :ff].double(), v[:, ff:].double()
    return g, u, torch.sigmoid(g)


@pytest.mark.parametrize("T", [1, 5, 33, 300])
def test_mlp_step(gpu_api, T):
    """Every stage in 64 bits at the tensors that the stage before it left on the GPU."""
    b = Block(gpu_api, 256, 528)
    x, dy = ic.drawn_tokens(3, T, b.d), ic.drawn_tokens(4, T, b.d)
    y, gu, tokens8, kept = b.forward(x.cuda())
    same(gu, linear(x, *b.host_gu).to(BF16))
    g, u, s = sigmoid_parts(gu.cpu(), b.ff)
    q, scale = tokens8
    restored = q.double().cpu() * scale.double().cpu()[:, None]
    h = g * s * u
    # h's rounding to bf16 (and fp32's before it), then half a step of the row's scale
    assert ((restored - h).abs() <= 2.0 ** -8 * h.abs() * 1.01 + 1e-37 + 0.5 * scale.double().cpu()[:, None] * (1 + 2.0 ** -20)).all()
    acc = ic.products(q.cpu().double(), b.host_down[0])
    prod = ic.scaled(acc, scale.cpu(), b.host_down[1]).double()
    ref = prod + x.double()
    bf16_near(y, ref, 2.0 ** -24 * (prod.abs() * 2 + ref.abs()))
    dh, dgu, dx = b.backward(dy.cuda(), kept)
    same(dh, back(dy, *b.host_down).to(BF16))
    gur = ic.restored8(gu.cpu().view(2 * T, b.ff)).view(T, 2 * b.ff)
    g, u, s = sigmoid_parts(gur, b.ff)
    d = dh.cpu().double()
    dgate, dup = d * u * s * (1 + g * (1 - s)), d * g * s
    tol = torch.cat([(d * u).abs() * s * (1 + g.abs()) * (g.abs() + 12), dup.abs() * (g.abs() + 8)], 1) * 2.0 ** -24 + 1e-36
    bf16_near(dgu, torch.cat([dgate, dup], 1), tol)
    prod = back(dgu.cpu(), *b.host_gu).double()
    ref = prod + dy.double()
    bf16_near(dx, ref, 2.0 ** -24 * (prod.abs() * 2 + ref.abs()))
    # serving: a token alone is what it was in the batch (whole sums, and the same steps after them)
    for t in (0, T - 1):
        alone = b.forward(x[t:t + 1].cuda())
        same(alone[1], gu[t:t + 1])
        for a, c in zip(alone[2], tokens8):
            same(a, c[t:t + 1])


def test_mlp_gradient_against_differences(gpu_api):
    """The block's gradient along itself against differences of the block in 64 bits on its weights' values.  Six roundings to 8 bits
    lie on the path (x, h, dy, dgu, gate, up), each off by at most half a step, 5/254 = 0.02 of a row's root mean square where no element
    is above five of it (a kept group's step is no larger); a product with random codes at most doubles a relative error: 6 * 2 * 0.02 =
    0.24 of the gradient's length in all.  The signs are the elements' own: of 40 * 256 of them six deviations are 6 * 0.24 / sqrt(10240)
    = 0.015 of the slope, and what is left are squares, 0.24^2 = 0.058; bf16 between the stages has 2^-8 each.  Together below 0.09."""
    T, b = 40, Block(gpu_api, 256, 528)
    gen = torch.Generator().manual_seed(3)
    x, dy = (torch.randn((T, b.d), generator=gen).to(BF16) for _ in range(2))
    for v in (x, dy):
        assert (v.double().abs().amax(1) <= 5 * v.double().square().mean(1).sqrt()).all()
    _, _, _, kept = b.forward(x.cuda())
    dx = b.backward(dy.cuda(), kept)[2].cpu().double()
    W = [w.double() * s.double()[:, None] for w, s in (b.host_gu, b.host_down)]

    def loss(v):
        gu = v @ W[0].T
        g, u = gu[:, :b.ff], gu[:, b.ff:]
        return float(((v + (g * torch.sigmoid(g) * u) @ W[1].T) * dy.double()).sum())

    e = 1e-4 / float(dx.square().mean().sqrt())
    slope = (loss(x.double() + e * dx) - loss(x.double() - e * dx)) / (2 * e)
    assert abs(float((dx * dx).sum()) - slope) <= 0.09 * abs(slope)


@pytest.mark.parametrize("T", [1, 16, 40, 300])
def test_block_captured(gpu_api, T):
    """Forward and backward in one graph, the eager block beside it, several replays with new inputs."""
    b, other = Block(gpu_api, 1024, 1040), Block(gpu_api, 1024, 1040, seed=9)
    draw = lambda k: ic.drawn_tokens(k, T, b.d).cuda()  # noqa: E731
    x, dy = draw(1), draw(2)
    both = lambda: (*(f := b.forward(x))[:3], *b.backward(dy, f[3]))  # noqa: E731
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for k in range(4):
        x.copy_(draw(10 + k))
        dy.copy_(draw(20 + k))
        for t in (out[0], out[1], out[2][0], out[3], out[4], out[5]):
            t.fill_(77)
        other.forward(dy)
        torch.cuda.synchronize()
        graph.replay()
        other.forward(x)
        torch.cuda.synchronize()
        got = [t.clone() for t in (out[0], out[1], *out[2], *out[3:])]
        want = both()
        for a, c in zip(got, (want[0], want[1], *want[2], *want[3:])):
            same(a, c)


@pytest.mark.parametrize("shape", [(4, 11008, 520), (128, 4096, 264), (4090, 144, 6704)], ids=str)
def test_products_and_the_kept_captured(gpu_api, shape):
    """The split and the mixed products, and the epilogue's forward, its kept tensors and its backward, replayed four times."""
    T, d_in, d_out = shape
    w = [t.cuda() for t in ic.drawn_weight(1, d_in, d_out)]
    x, dy = ic.drawn_tokens(2, T, d_in).cuda(), ic.drawn_tokens(3, T, d_out).cuda()
    bias, mul, _ = (t.cuda() for t in ec.extras(3, T, d_out, BF16))

    def step():
        y, z = gpu_api.forward_int8(x, *w, bias=bias, act="silu", mul=mul, keep_z=True, out_dtype=BF16)
        dz, dmul, db = gpu_api.epilogue_backward_kept8(dy, gpu_api.keep8(z), "silu", mul8=gpu_api.keep8(mul), want_dbias=True)
        return y, z, dz, dmul, db, gpu_api.backward_int8(dz, *w)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(ic.drawn_tokens(10 + k, T, d_in))
        dy.copy_(ic.drawn_tokens(20 + k, T, d_out))
        for t in out:
            t.fill_(77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, c in zip(got, step()):
            same(a, c)


def test_two_graphs_with_one_workspace(gpu_api):
    """A forward and a backward, both with K in slices, captured apart on one workspace and replayed in turn, eager calls on it between."""
    T, d_in, d_out = 40, 4096, 520
    w = [t.cuda() for t in ic.drawn_weight(1, d_in, d_out)]
    x, dy = ic.drawn_tokens(2, T, d_in).cuda(), ic.drawn_tokens(3, T, d_out).cuda()
    n = max(gpu_api.int8_workspace_bytes(T, d_in, d_out, op) for op in (gpu_api.OP_FORWARD, gpu_api.OP_BACKWARD))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    y, dx = torch.empty((T, d_out), device="cuda"), torch.empty((T, d_in), device="cuda")
    calls = (lambda: gpu_api.forward_int8(x, *w, ws=ws, y=y), lambda: gpu_api.backward_int8(dy, *w, ws=ws, dx=dx))
    graphs = []
    for call in calls:
        call()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    for k in range(4):
        x.copy_(ic.drawn_tokens(10 + k, T, d_in))
        dy.copy_(ic.drawn_tokens(20 + k, T, d_out))
        y.fill_(77), dx.fill_(77), ws.fill_(0x7f)
        graphs[k % 2].replay()
        graphs[1 - k % 2].replay()
        torch.cuda.synchronize()
        same(y, gpu_api.forward_int8(x, *w)), same(dx, gpu_api.backward_int8(dy, *w))
        calls[k % 2]()


def test_streams_at_once(gpu_api):
    """The same weights on four streams, each call with outputs and workspaces of its own."""
    blocks = [Block(gpu_api, 1024, 1040), Block(gpu_api, 256, 528)]
    jobs = [(blocks[k % 2], ic.drawn_tokens(k, (1, 16, 64, 700)[k], blocks[k % 2].d).cuda()) for k in range(4)]
    want = [(f := b.forward(x), b.backward(x, f[3])) for b, x in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(3):
        got = []
        for (b, x), st in zip(jobs, streams):
            with torch.cuda.stream(st):
                f = b.forward(x)
                got.append((f, b.backward(x, f[3])))
        torch.cuda.synchronize()
        for (f, r), (f0, r0) in zip(got, want):
            for a, c in zip((f[0], f[1], *f[2], *r), (f0[0], f0[1], *f0[2], *r0)):
                same(a, c)


class Guarded:
    """Tensors between bytes that have to stay; a call sees nothing but its own."""
    ROOM = 4096

    def __init__(self):
        self.all = []

    def __call__(self, shape, dtype):
        n = torch.empty(shape, dtype=dtype, device="meta").numel() * torch.empty((), dtype=dtype).element_size()
        raw = torch.full((n + 2 * self.ROOM,), 0xa5, dtype=torch.uint8, device="cuda")
        self.all.append((raw, n))
        return raw[self.ROOM:self.ROOM + n].view(dtype).view(shape)

    def check(self):
        torch.cuda.synchronize()
        for raw, n in self.all:
            assert (raw[:self.ROOM] == 0xa5).all() and (raw[self.ROOM + n:] == 0xa5).all()


@pytest.mark.parametrize("shape", [(1, 16, 8), (3, 4096, 72), (16, 1024, 520), (17, 272, 136), (33, 4096, 264), (65, 528, 1032), (257, 1024, 328),
                                   (700, 144, 16400), (4090, 144, 6704)], ids=str)
def test_nothing_beside_the_outputs(gpu_api, shape):
    """Nothing before or behind an output or a workspace of exactly its size is written, and what is behind the operands (0xa5a5, small
    numbers as bf16; other rows of a larger batch) has no part in the results."""
    T, d_in, d_out = shape
    api, g = gpu_api, Guarded()
    w = [t.cuda() for t in ic.drawn_weight(1, d_in, d_out)]
    gw = [g(t.shape, t.dtype).copy_(t) for t in w]
    x, dy = ic.drawn_tokens(2, T, d_in).cuda(), ic.drawn_tokens(3, T, d_out).cuda()
    gx, gdy = g(x.shape, BF16).copy_(x), g(dy.shape, BF16).copy_(dy)
    n, m = (api.int8_workspace_bytes(T, d_in, d_out, op) for op in (api.OP_FORWARD, api.OP_BACKWARD))
    bias, mul, residual = (t.cuda() for t in ec.extras(3, T, d_out, BF16))
    gb, gm, gr = (g(t.shape, t.dtype).copy_(t) for t in (bias, mul, residual))
    y, z = api.forward_int8(x, *w, bias=bias, act="gelu", mul=mul, residual=residual, keep_z=True, out_dtype=BF16)
    gy, gz = api.forward_int8(gx, *gw, bias=gb, act="gelu", mul=gm, residual=gr, keep_z=True, y=g((T, d_out), BF16), z=g((T, d_out), BF16),
                              ws=g((n,), torch.uint8))
    same(gy, y), same(gz, z)
    y32 = api.forward_int8(gx, *gw, y=g((T, d_out), F32), ws=g((n,), torch.uint8))
    same(y32, api.forward_int8(x, *w))
    dx = api.backward_int8(dy, *w)
    same(api.backward_int8(gdy, *gw, dx=g((T, d_in), F32), ws=g((m,), torch.uint8)), dx)
    same(api.backward_int8(gdy, *gw, dx=g((T, d_in), BF16), ws=g((m,), torch.uint8)), dx.to(BF16))
    q, s = api.quantize_tokens(gx, q=g((T, d_in), torch.int8), s=g((T,), F32))
    for a, c in zip((q, s), api.quantize_tokens(x)):
        same(a, c)
    kept = api.keep8(gdy, kept=g((api.kept8_bytes(T, d_out),), torch.uint8))
    same(api.restore8(kept, T, d_out, x=g((T, d_out), BF16)), api.restore8(api.keep8(dy), T, d_out))
    gu = torch.cat([dy, mul], 1)
    ggu = g((T, 2 * d_out), BF16).copy_(gu)
    k2 = g((api.kept8_bytes(2 * T, d_out),), torch.uint8)
    (q, s), _ = api.swiglu_forward_int8(ggu, d_out, keep=True, q=g((T, d_out), torch.int8), s=g((T,), F32), kept=k2, h=g((T, d_out), BF16))
    for a, c in zip((q, s), api.swiglu_forward_int8(gu, d_out)):
        same(a, c)
    k3 = api.swiglu_forward_keep8(ggu, d_out, h=g((T, d_out), BF16), kept=g((api.kept8_bytes(2 * T, d_out),), torch.uint8))[1]
    back = api.swiglu_backward_kept8(dy, api.swiglu_forward_keep8(gu, d_out)[1], d_out)
    for k in (k2, k3):
        same(api.swiglu_backward_kept8(gdy, k, d_out, dgu=g((T, 2 * d_out), BF16)), back)
    ref = api.epilogue_backward_kept8(dy, api.keep8(z), "silu", mul8=api.keep8(mul), want_dbias=True)
    ws = g((int(api.load().qalora_epilogue_backward_workspace_bytes(T, d_out)),), torch.uint8)
    got = api.epilogue_backward_kept8(gdy, api.keep8(z), "silu", mul8=api.keep8(gm), dz=g((T, d_out), BF16), dmul=g((T, d_out), BF16),
                                      dbias=g((d_out,), F32), ws=ws if ws.numel() else None)
    for a, c in zip(got, ref):
        same(a, c)
    g.check()


@pytest.mark.parametrize("T", [2, 5, 16, 40, 130, 300])
def test_a_row_that_is_nan_stays_alone(gpu_api, T):
    """A NaN or an infinity in a row makes that row NaN through every activation, a mul of zeros and z, and no other."""
    d_in, d_out = 1024, 264
    w = [t.cuda() for t in ic.drawn_weight(1, d_in, d_out)]
    x = ic.drawn_tokens(2, T, d_in).cuda()
    sick = x.clone()
    sick[T // 2, 5], sick[0, 1023] = float("nan"), float("inf")
    mul, residual = torch.zeros((T, d_out), dtype=BF16, device="cuda"), torch.ones((T, d_out), device="cuda")
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[T // 2] = rows[0] = False
    for act in ec.ACTS:
        y, z = gpu_api.forward_int8(sick, *w, act=act, mul=mul, residual=residual, keep_z=True)
        yr, zr = gpu_api.forward_int8(x, *w, act=act, mul=mul, residual=residual, keep_z=True)
        assert torch.isnan(y[~rows]).all() and torch.isnan(z[~rows]).all()
        same(y[rows], yr[rows]), same(z[rows], zr[rows])
    dy = ic.drawn_tokens(3, T, d_out).cuda()
    sick = dy.clone()
    sick[T // 2, 5], sick[0, 263] = float("-inf"), float("nan")
    dx = gpu_api.backward_int8(sick, *w)
    assert torch.isnan(dx[~rows]).all()
    same(dx[rows], gpu_api.backward_int8(dy, *w)[rows])


@pytest.mark.parametrize("size", [(1024, 1032), (11008, 520), (64, 16400), (272, 8200)], ids=str)
def test_a_token_is_the_same_in_every_batch(gpu_api, size):
    """Whatever kernel, tile and split of K the number of tokens brings: bit for bit, with every operand of the epilogue, and backward."""
    K, N = size
    most = 4096 if N < 2000 else 700
    w = [t.cuda() for t in ic.drawn_weight(1, K, N)]
    x = ic.drawn_tokens(2, most, K).cuda()
    back = [t.cuda() for t in ic.drawn_weight(3, N // 16 * 16, K)]
    residual_in = torch.randn((most, N // 16 * 16), device="cuda")
    counts = [T for T in (1, 2, 5, 16, 17, 31, 40, 64, 65, 100, 130, 200, 260, 300, 520, 700, 1031, 2500, 4096) if T <= most]
    for out_dtype in (F32, BF16):
        bias, mul, residual = (t.cuda() for t in ec.extras(3, most, N, out_dtype))
        for k, act in enumerate(ec.ACTS):
            for use in (1, 2 + k % 2, 4 + k % 2, 7):
                call = lambda T: gpu_api.forward_int8(  # noqa: E731
                    x[:T], *w, bias=bias if use & 1 else None, act=act, mul=mul[:T] if use & 2 else None,
                    residual=residual[:T] if use & 4 else None, keep_z=True, out_dtype=out_dtype)
                whole = call(most)
                for T in counts:
                    for a, b in zip(call(T), whole):
                        assert torch.equal(a, b[:T]), (out_dtype, act, use, T)
        r = residual_in.to(out_dtype)
        whole = gpu_api.backward_int8(x, *back, residual=r, dx_dtype=out_dtype)
        for T in counts:
            assert torch.equal(gpu_api.backward_int8(x[:T], *back, residual=r[:T], dx_dtype=out_dtype), whole[:T]), (out_dtype, T)


def test_very_many_tokens(gpu_api):
    """More rows than a launch that brings them to 8 bits takes (2^21)."""
    T, K, N = 2 ** 21 + 3, 16, 8
    x = ic.drawn_tokens(5, T, K)
    codes, scale = ic.drawn_weight(1, K, N)
    q, s = gpu_api.quantize_tokens(x.cuda())
    rq, rs = ic.rows8(x.float())
    same(s, rs), same(q, rq.to(torch.int8))
    same(gpu_api.forward_int8(x.cuda(), codes.cuda(), scale.cuda()), ic.scaled(ic.products(rq, codes), rs, scale))
    gu = x.cuda()
    (q, s), kept = gpu_api.swiglu_forward_int8(gu, 8, keep=True)
    h, kept2 = gpu_api.swiglu_forward_keep8(gu, 8)
    for a, b in zip((q, s), gpu_api.quantize_tokens(h)):
        same(a, b)
    for k in (kept, kept2):
        same(gpu_api.restore8(k, 2 * T, 8), ic.restored8(x.view(2 * T, 8)))


def test_the_place_of_an_operand(gpu_api):
    """y and z in the place of a bf16 mul or residual of exactly their elements; refused a row further on."""
    for T, d_in, d_out in ((1, 256, 264), (16, 1024, 520), (3, 11008, 264), (100, 2064, 520), (300, 512, 1032), (4090, 144, 6704)):
        w = [t.cuda() for t in ic.drawn_weight(1, d_in, d_out)]
        x = gpu_api.quantize_tokens(ic.drawn_tokens(2, T, d_in).cuda())
        _, mul, residual = (t.cuda() for t in ec.extras(4, T, d_out, BF16))
        call = lambda m, r, **kw: gpu_api.forward_int8(x, *w, act="silu", mul=m, residual=r, out_dtype=BF16, **kw)  # noqa: E731
        ref, both = call(mul, residual), call(mul, mul)
        for at, args in ((m := mul.clone(), (m, residual)), (r := residual.clone(), (mul, r))):
            assert call(*args, y=at) is at
            same(at, ref)
        m = mul.clone()
        same(call(m, m, y=m), both)
        if T > 1:
            room = torch.zeros((T + 1, d_out), dtype=BF16, device="cuda")
            for m, r in ((room[1:], residual), (mul, room[1:])):
                with pytest.raises(gpu_api.QaloraError) as e:
                    call(m, r, y=room[:-1])
                assert e.value.status == gpu_api.EINVAL
            assert not room.any()


def test_the_c_entries_with_their_own_stream(gpu_api):
    """The C entry itself on a stream of the caller's."""
    lib, P = gpu_api.load(), lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    T, d_in, d_out = 33, 1024, 264
    w = [t.cuda() for t in ic.drawn_weight(1, d_in, d_out)]
    x = ic.drawn_tokens(2, T, d_in).cuda()
    want = gpu_api.forward_int8(x, *w)
    y = torch.empty_like(want)
    n = gpu_api.int8_workspace_bytes(T, d_in, d_out, gpu_api.OP_FORWARD)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    rc = lib.qalora_forward_int8(T, d_in, d_out, P(x), None, P(w[0]), P(w[1]), None, P(y), 0, P(ws), n, ctypes.c_void_p(st.cuda_stream))
    st.synchronize()
    assert rc == gpu_api.OK
    same(y, want)
