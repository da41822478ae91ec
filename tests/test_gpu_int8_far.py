"""The 8-bit operators on operands of more than 4 GB: offsets past 32 bits.  The whole against calls on parts of it (rows are
independent), and a few rows against the definition."""
import pytest
import torch

import int8_cases as ic
from int8_cases import BF16, F32

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    yield
    torch.cuda.empty_cache()


def draw(shape, seed, dtype=BF16):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda", dtype=dtype)


def parts(T, n=3):
    step = -(-T // n)
    return [slice(a, min(T, a + step)) for a in range(0, T, step)]


def alike(a, b):
    assert a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, b)


def test_many_tokens(gpu_api):
    """270001 tokens of 16400: 8.9 GB, 4.4 GB of codes; a product with 24 channels."""
    T, K, N = 270001, 16400, 24
    x = draw((T, K), 1)
    codes, scale = (t.cuda() for t in ic.drawn_weight(2, K, N))
    q, s = gpu_api.quantize_tokens(x)
    y, y8 = gpu_api.forward_int8(x, codes, scale), gpu_api.forward_int8((q, s), codes, scale)
    alike(y, y8)
    for p in parts(T):
        for a, b in zip((q[p], s[p]), gpu_api.quantize_tokens(x[p])):
            alike(a, b)
        alike(y[p], gpu_api.forward_int8(x[p], codes, scale))
    rows = [0, 1, 130943, 130944, 261888, T - 1]   # (at 2^31 and 2^32 bytes)
    rq, rs = ic.rows8(x[rows].float().cpu())
    ic.same(y[rows], ic.scaled(ic.products(rq, codes.cpu()), rs, scale.cpu()))
    dy = draw((T, N), 3)                           # dx: 270001 x 16400
    dx = gpu_api.backward_int8(dy, codes, scale, residual=x, dx_dtype=BF16)
    for p in parts(T):
        alike(dx[p], gpu_api.backward_int8(dy[p], codes, scale, residual=x[p], dx_dtype=BF16))
    v = dy[rows].float().cpu() * scale.cpu()
    rq, rs = ic.rows8(v)
    ref = ic.products(rq, codes.cpu().T.contiguous()) * rs[:, None].double() + x[rows].cpu().double()
    assert ((dx[rows].cpu().double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -22) * ref.abs() + 2.0 ** -22 * x[rows].cpu().double().abs() + 1e-30).all()


def test_a_large_result(gpu_api):
    """270001 x 8192: y of 8.8 GB, z and mul of 4.4 GB."""
    T, K, N = 270001, 16, 8192
    x, mul = draw((T, K), 1), draw((T, N), 2)
    codes, scale = (t.cuda() for t in ic.drawn_weight(2, K, N))
    y, z = gpu_api.forward_int8(x, codes, scale, act="silu", mul=mul, keep_z=True)
    for p in parts(T):
        for a, b in zip((y[p], z[p]), gpu_api.forward_int8(x[p], codes, scale, act="silu", mul=mul[p], keep_z=True)):
            alike(a, b)
    rows = [0, 131071, 131072, 262143, 262144, T - 1]
    rq, rs = ic.rows8(x[rows].float().cpu())
    ic.same(z[rows], ic.scaled(ic.products(rq, codes.cpu()), rs, scale.cpu()).to(BF16))


@pytest.mark.parametrize("T", [3, 300])
def test_a_large_weight(gpu_api, T):
    """131072 channels of 40000: 5.2 GB; both directions in 64 bits, some channels at a time."""
    K, N = 40000, 131072
    codes = torch.randint(-127, 128, (N, K), generator=torch.Generator("cuda").manual_seed(5), device="cuda", dtype=torch.int8)
    scale = torch.rand(N, generator=torch.Generator("cuda").manual_seed(6), device="cuda") + 0.5
    x, dy = draw((T, K), 7), draw((T, N), 8)
    q, s = gpu_api.quantize_tokens(x)
    v, t = gpu_api.quantize_tokens(dy, scale)
    y, acc = gpu_api.forward_int8(x, codes, scale), torch.zeros((T, K), dtype=torch.float64, device="cuda")
    for a in range(0, N, 16384):
        w = codes[a:a + 16384].double()
        alike(y[:, a:a + 16384].contiguous(), (q.double() @ w.T.contiguous()).to(F32) * s[:, None] * scale[a:a + 16384])
        acc += v[:, a:a + 16384].double() @ w
    alike(gpu_api.backward_int8(dy, codes, scale), acc.to(F32) * t[:, None])


def test_one_token_of_a_large_weight(gpu_api):
    """131072 x 16384, 2 GiB, in one launch."""
    K, N = 16384, 131072
    codes = torch.randint(-127, 128, (N, K), generator=torch.Generator("cuda").manual_seed(5), device="cuda", dtype=torch.int8)
    scale = torch.ones(N, device="cuda")
    x = draw((1, K), 7)
    q, s = gpu_api.quantize_tokens(x)
    y = gpu_api.forward_int8(x, codes, scale)
    for a in range(0, N, 16384):
        alike(y[:, a:a + 16384].contiguous(), (q.double() @ codes[a:a + 16384].double().T.contiguous()).to(F32) * s[:, None])


def test_many_kept_rows(gpu_api):
    """270001 rows of gate and up of 8192: 8.8 GB, 4.6 GB kept."""
    T, C = 270001, 8192
    gu, dh = draw((T, 2 * C), 1), draw((T, C), 2)
    h, kept = gpu_api.swiglu_forward_keep8(gu, C)
    (q, s), kept2 = gpu_api.swiglu_forward_int8(gu, C, keep=True)
    dgu = gpu_api.swiglu_backward_kept8(dh, kept, C)
    alike(gpu_api.swiglu_backward_kept8(dh, kept2, C), dgu)
    restored = gpu_api.restore8(kept, 2 * T, C).view(T, 2 * C)
    rows = [0, 131071, 131072, 262143, 262144, T - 1]
    ic.same(restored[rows].view(-1, C), ic.restored8(gu[rows].cpu().view(-1, C)))
    for p in parts(T):
        h1, kept1 = gpu_api.swiglu_forward_keep8(gu[p], C)
        alike(h[p], h1)
        for a, b in zip((q[p], s[p]), gpu_api.swiglu_forward_int8(gu[p], C)):
            alike(a, b)
        n = h1.shape[0]
        alike(restored[p], gpu_api.restore8(kept1, 2 * n, C).view(n, 2 * C))
        alike(dgu[p], gpu_api.swiglu_backward_kept8(dh[p], kept1, C))


def test_the_epilogues_backward_of_many_kept_rows(gpu_api):
    """540001 rows of 8192: 4.6 GB kept, dy and dz 8.8 GB each."""
    T, C = 540001, 8192
    z, dy = draw((T, C), 1), draw((T, C), 2)
    z8 = gpu_api.keep8(z)
    dz = gpu_api.epilogue_backward_kept8(dy, z8, "relu")[0]
    z = gpu_api.restore8(z8, T, C, x=z)
    for p in parts(T, 5):
        alike(dz[p], gpu_api.epilogue_backward(dy[p], z[p], "relu")[0])
