"""The 8-bit operators in 64 bits, from their definitions."""
import numpy as np
import torch

BF16, F32 = torch.bfloat16, torch.float32

# tokens, d_in, d_out: one token to long batches, widths that end inside every tile, every tile and K split (a test without a GPU
# looks at that)
SHAPES = [(1, 16, 8), (1, 4096, 1032), (3, 1024, 264), (4, 11008, 520), (7, 48, 24), (16, 1024, 1024), (16, 272, 136), (17, 5120, 520),
          (31, 144, 72), (33, 4096, 264), (61, 1040, 776), (64, 1024, 1024), (65, 256, 72), (100, 2064, 520), (128, 512, 512),
          (129, 4112, 1544), (200, 208, 2056), (257, 1024, 328), (511, 96, 40), (700, 1536, 1288), (1031, 784, 600)]
BACK_SHAPES = [(5, 64, 11008), (300, 16, 4104)]
# tokens, depth and width of the product, for the larger tiles
LARGE = [(700, 64, 16400), (500, 144, 16400), (380, 64, 11024), (380, 272, 8208), (250, 144, 4112), (140, 272, 16400), (513, 80, 8208)]
# the same, of more than a round of 256 x 256 tiles: the last columns in tiles of 256 x 128 and 256 x 192
MIXED = [(65000, 16, 272), (64800, 144, 336), (2040, 144, 19408), (4090, 144, 6704), (8200, 144, 3024), (700, 80, 32784)]


def rows8(v):
    """Codes (float64) and scales (float32) of the rows of v, an fp32 tensor on the CPU.  The quotient of two fp32 numbers differs from
    a middle between whole numbers up to 128 by nothing or by at least 2^-26: rounding the 64-bit quotient is rounding the exact one."""
    v = np.asarray(v, dtype=np.float32)
    with np.errstate(all="ignore"):
        s = np.abs(v).max(1) * np.float32(1 / 127)
        good = np.isfinite(v).all(1)
        d = np.where((s > 0) & good, s, 1).astype(np.float64)
        q = np.clip(np.rint(v.astype(np.float64) / d[:, None]), -127, 127)
    q[~((s > 0) & good)] = 0
    s[~good] = np.nan
    return torch.from_numpy(q), torch.from_numpy(s)


def weight8(W):
    """Codes [d_out, d_in] and scales [d_out] of W [d_in, d_out] (fp32)."""
    q, s = rows8(W.T.contiguous())
    return q.to(torch.int8), s


def drawn_weight(seed, d_in, d_out):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(-127, 128, (d_out, d_in), generator=g, dtype=torch.int8)
    return codes, (0.5 + torch.rand(d_out, generator=g)) / (73 * d_in ** 0.5)


def drawn_tokens(seed, T, cols):
    """Unit size, some columns larger."""
    x = torch.randn((T, cols), generator=torch.Generator().manual_seed(seed))
    x[:, ::97] *= 20
    return x.to(BF16)


def products(q, w):
    """q [T, K] . w [N, K], whole numbers: exact."""
    return q.double() @ w.double().T


def scaled(acc, s, sw=None):
    """(acc s) sw with an fp32 rounding after each step, as the kernels have it."""
    v = acc.to(F32) * s[:, None]
    return v if sw is None else v * sw


def kept8(x):
    """(codes, biased exponents for each element) of x, bf16 on the CPU."""
    T, C = x.shape
    bits = np.zeros((T, -(-C // 32) * 32), np.int64)
    bits[:, :C] = x.contiguous().view(torch.int16).numpy().astype(np.int64) & 0x7fff
    E = np.maximum(bits.reshape(T, -1, 32).max(2) >> 7, 1).repeat(32, 1)[:, :C]
    with np.errstate(all="ignore"):
        q = np.clip(np.rint(np.ldexp(x.double().numpy(), 133 - E)), -127, 127)
    q[E == 255] = 0
    return q, E


def restored8(x):
    q, E = kept8(x)
    v = np.ldexp(q, E - 133)
    v[E == 255] = np.nan
    return torch.from_numpy(v).to(BF16)


def same(got, ref):
    """Equal, NaN with NaN."""
    got, ref = got.cpu(), ref.cpu()
    assert got.dtype == ref.dtype and got.shape == ref.shape
    bad = ~((got == ref) | (torch.isnan(got) & torch.isnan(ref))) if got.is_floating_point() else got != ref
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[0].tolist(), got[bad][:4], ref[bad][:4])
