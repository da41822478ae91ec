"""Operands of more than 4 GB: offsets past 32 bits in the orthogonalised update, the epilogue's backward and the linear's epilogue."""
import math

import pytest
import torch

import epilogue_cases as ec

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def room():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("tall", [False, True])
def test_update_of_a_long_matrix(gpu_api, tall):
    """66 x 2^24 (4.4 GB), a matrix of 40 x 50 behind it in the list.  X in 64 bits on the GPU; tolerance as in test_gpu_muon_forms.py,
    16384 columns in a row."""
    short, long = 66, 2 ** 24
    gen = torch.Generator("cuda").manual_seed(3)
    shapes = [(long, short) if tall else (short, long), (40, 50)]
    g = [torch.randn(s, generator=gen, device="cuda") for s in shapes]
    view = g[0] if tall else g[0].T              # [long, short]
    view[:, 0] += 4.0 * view[:, 1]               # not all singular values alike
    before = [t.clone() for t in g[1:]]
    p, m = ([torch.zeros_like(t) for t in g] for _ in range(2))
    hp = gpu_api.Muon(lr=1.0, momentum=0.0, nesterov=False, scale_mode=gpu_api.MUON_SCALE_NONE)
    gpu_api.muon_step(hp, p, g, m)
    assert torch.equal(m[0], g[0]) and torch.equal(g[1], before[0])
    a, b, c = hp.a, hp.b, hp.c
    for grad, got in zip(g, p):
        X = (grad if grad.shape[0] >= grad.shape[1] else grad.T).double()
        X = X / (X.square().sum().sqrt() + hp.eps)
        bound, eye = 0.0, torch.eye(X.shape[1], dtype=torch.float64, device="cuda")
        for k in range(hp.steps):
            bound += a ** (hp.steps - k) * float(X.square().sum().sqrt())
            G = sum(part.T.contiguous() @ part for part in X.split(1 << 20))
            P = a * eye + b * G + c * (G @ G)
            for part in X.split(1 << 20):
                part.copy_(part @ P)
        bound += float(X.square().sum().sqrt())
        got = got if got.shape[0] >= got.shape[1] else got.T
        off = math.sqrt(sum(float((x + q.double()).square().sum()) for x, q in zip(X.split(1 << 20), got.split(1 << 20))))
        assert off <= 3 * (8 + math.sqrt(16384) / 2) * 2.0 ** -24 * bound, (tuple(grad.shape), off, bound)


@pytest.mark.parametrize("dy_dtype", [BF16, torch.float32], ids=["bf16", "fp32"])
def test_epilogue_backward_of_many_rows(gpu_api, dy_dtype):
    """270001 rows of 8192: 4.4 GB in bf16.  relu and a mul: dz, dmul exact; dbias to its sums (test_gpu_epilogue.py's bound)."""
    T, cols = 270001, 8192
    gen = torch.Generator("cuda").manual_seed(4)
    draw = lambda dtype: torch.randn((T, cols), generator=gen, device="cuda", dtype=dtype)  # noqa: E731
    dy, z, mul = draw(dy_dtype), draw(BF16), draw(BF16)
    dz, dmul, db = gpu_api.epilogue_backward(dy, z, "relu", mul=mul, want_dbias=True)
    total = torch.zeros(cols, dtype=torch.float64, device="cuda")
    squares = torch.zeros_like(total)
    for r in range(0, T, 20000):
        s = slice(r, r + 20000)
        d = torch.where(z[s] > 0, dy[s].float(), torch.zeros((), device="cuda")) * mul[s].float()
        assert torch.equal(dz[s], d.to(BF16)) and torch.equal(dmul[s], (dy[s].float() * z[s].float().clamp(min=0)).to(BF16))
        total += d.double().sum(0)
        squares += d.double().square().sum(0)
    assert ((db.double() - total).abs() <= 8 * 2.0 ** -24 * math.sqrt(T) * squares.sqrt() + 2.0 ** -24 * total.abs()).all()


def test_forward_of_many_tokens(gpu_api):
    """60000 tokens of 1024 -> 20000, y and its residual in fp32 (4.8 GB each), in place: from the plain call's sums, bit for bit."""
    T, d_in, d_out = 60000, 1024, 20000
    codes, alpha, beta, _, _, _ = ec.drawn_layer(3, 1, d_in, d_out, 4, 64)
    desc = gpu_api.make_desc(d_in, d_out, 4, 64)
    layer = (gpu_api.pack(desc, codes.cuda()), alpha.cuda(), beta.cuda())
    gen = torch.Generator("cuda").manual_seed(5)
    x = torch.randn((T, d_in), generator=gen, device="cuda").to(BF16)
    residual = torch.randn((T, d_out), generator=gen, device="cuda")
    bias = torch.randn(d_out, generator=gen, device="cuda")
    base = gpu_api.forward(desc, x, *layer)
    stream = residual.clone()
    y, z, _ = gpu_api.forward_epilogue(desc, x, *layer, bias=bias, act="relu", residual=stream, keep_z=True, y=stream)
    assert y is stream
    for r in range(0, T, 10000):
        s = slice(r, r + 10000)
        sums = base[s] + bias
        assert torch.equal(z[s], sums.to(BF16)) and torch.equal(y[s], sums.clamp(min=0) + residual[s])
