"""The 8-bit operators without a GPU: their refusals, sizes and launch shapes, and the gradients' formulas against differences."""
import ctypes
import random

import pytest
import torch

import int8_cases as ic
from host_code import host_library
from paper_2309_14717_amd import api

SOURCE = r"""
#include "gemm_i8_plan.hpp"
#include "int8.hpp"
#include "tokens8_plan.hpp"
using namespace qalora;
extern "C" void tokens(int rows, int cols, int* o) {
  const Tokens8Plan p = tokens8_plan(rows, cols);
  o[0] = p.lanes; o[1] = p.pieces; o[2] = p.rows;
}
extern "C" void product(int M, int N, int K, int back, int* o) {
  const Int8Plan p = int8_plan(M, N, K, back);
  o[0] = p.tile; o[1] = p.slices; o[2] = kInt8Tiles[p.tile].rows; o[3] = kInt8Tiles[p.tile].cols; o[4] = kInt8Tiles[p.tile].threads;
}
extern "C" void mixed(int M, int N, int slices, int back, int* o) {
  const Int8Mixed m = int8_mixed(M, N, slices, back);
  o[0] = m.narrow; o[1] = m.wide_n;
  if (m.narrow) {
    const int tiles_m = (M + 255) / 256, narrow = tiles_m * ((N - m.wide_n * 256 + m.narrow - 1) / m.narrow);
    o[2] = tiles_m * m.wide_n; o[3] = narrow; o[4] = int8_narrow_first(narrow);
  }
}
extern "C" long long partials(int M, int N) { return (long long)int8_partials(M, N); }
extern "C" long long kept(long long rows, long long cols) { return (long long)keep8_bytes(rows, cols); }
extern "C" long long exponents_at(long long rows, long long cols) { return (long long)keep8_exponents_at(rows, cols); }
"""
P = ctypes.c_void_p
GOOD, ODD = 0x10000, 0x10004


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    lib = host_library(tmp_path_factory.mktemp("int8"), "int8_plan", SOURCE)
    lib.kept.restype = lib.exponents_at.restype = lib.partials.restype = ctypes.c_longlong
    lib.kept.argtypes = lib.exponents_at.argtypes = [ctypes.c_longlong] * 2
    return lib


def test_rows_are_covered(host):
    o = (ctypes.c_int * 3)()
    for cols in list(range(8, 20000, 8)) + list(range(20000, 131073, 24)) + [131072]:
        for rows_in in (1, 512, 513, 100000):
            host.tokens(rows_in, cols, o)
            lanes, pieces, rows = o
            assert lanes * pieces * 8 >= cols and (lanes, pieces) in {(64, 1), (64, 2), (256, 1), (256, 2), (512, 2), (512, 3), (512, 4), (1024, 1),
                                                                      (1024, 2), (1024, 4), (1024, 8), (1024, 16)}
            assert rows == (4 if lanes == 64 else 1)


def test_product_plans(host):
    """Slices that are all there and fit their room, launches that the device takes; and the GPU tests reach every tile and a split."""
    o = (ctypes.c_int * 5)()
    rng = random.Random(3)
    sizes = [(1, 8, 16), (2 ** 29, 8, 16), (2 ** 29, 256, 16), (2 ** 27, 1032, 16), (1, 131072, 131072), (4096, 11008, 4096), (1, 8, 131072)]
    sizes += [(rng.randint(1, 10 ** rng.randint(1, 6)), 8 * rng.randint(1, 4000), 16 * rng.randint(1, 2000)) for _ in range(2000)]
    for M, N, K in sizes:
        for back in (0, 1):
            host.product(M, N, K, back, o)
            _, slices, rows, cols, threads = o
            steps = -(-K // 128)
            per = -(-steps // slices)
            assert per * (slices - 1) < steps <= per * slices and slices <= 32
            assert slices == 1 or slices * M * N * 4 <= host.partials(M, N)
            assert -(-M // rows) * -(-N // cols) * threads < 2 ** 32
    for shapes, back in ((ic.SHAPES, 0), (ic.SHAPES + ic.BACK_SHAPES, 1)):
        got = set()
        for T, d_in, d_out in shapes:
            host.product(T, d_in if back else d_out, d_out if back else d_in, back, o)
            got.add((o[0], o[1] > 1))
        assert {s for _, s in got} == {False, True}
        for T, depth, width in ic.LARGE:
            host.product(T, width, depth, back, o)
            got.add((o[0], o[1] > 1))
        assert {t for t, _ in got} == set(range(11)) - ({4, 6, 8, 10} if back else {7, 9}), (back, sorted(got))


def test_mixed_plans(host):
    """Whole rounds of wide tiles, the rest in one round of narrow ones, every column in one of them; the GPU tests reach each kind."""
    o, m = (ctypes.c_int * 5)(), (ctypes.c_int * 5)()
    rng = random.Random(4)
    seen = set()
    for M, N in [(1, 131072), (65536, 8), (65537, 8), (2 ** 29, 131072), (65536, 256), (65536, 264), (4096, 4096), (4096, 4104)] + \
                [(rng.randint(1, 10 ** rng.randint(3, 6)), 8 * rng.randint(1, 16384)) for _ in range(4000)]:
        for back in (0, 1):
            host.mixed(M, N, 2, back, m)
            assert m[0] == 0
            host.mixed(M, N, 1, back, m)
            narrow, wide_n, wide, narrows, first = m
            seen.add((back, narrow))
            tiles = -(-M // 256) * -(-N // 256)
            if narrow:
                assert wide_n > 0 and 0 < N - 256 * wide_n and 256 * (tiles // 256) - -(-M // 256) < wide <= 256 * (tiles // 256)
                assert 0 <= first <= narrows <= 256 and first % 8 == 0 and (wide + narrows) * 512 < 2 ** 32
    assert seen == {(0, 0), (0, 128), (0, 192), (1, 0), (1, 128)}
    for back in (0, 1):
        got = set()
        for T, depth, width in ic.MIXED:
            host.product(T, width, depth, back, o)
            host.mixed(T, width, o[1], back, m)
            got.add((o[0], m[0]))
        assert got == ({(0, 0), (0, 128)} if back else {(0, 128), (0, 192)})


def test_kept_sizes(host):
    for rows, cols in ((1, 8), (3, 40), (7, 1000), (2 ** 31 - 1, 8), (5, 2 ** 29), (4096, 22016)):
        n, at = host.kept(rows, cols), host.exponents_at(rows, cols)
        assert at >= rows * cols and at % 16 == 0 and n >= at + rows * -(-cols // 32) and n < rows * cols * 1.2 + 64 + rows
        assert api.kept8_bytes(rows, cols) == n
    for rows, cols in ((0, 8), (-1, 8), (4, 0), (4, 12), (4, 2 ** 29 + 8)):
        assert api.kept8_bytes(rows, cols) == 0


def test_workspace_sizes():
    size = api.int8_workspace_bytes
    for T in (1, 5, 64, 4096):
        assert size(T, 1024, 264, api.OP_FORWARD) >= T * (1024 + 4) and size(T, 1024, 264, api.OP_BACKWARD) >= T * (264 + 4)
    for bad in ((0, 1024, 264, 1), (4, 1000, 264, 1), (4, 1024, 260, 1), (4, 131088, 8, 1), (4, 16, 131080, 1), (4, 1024, 264, 0),
                (4, 1024, 264, 3)):
        assert size(*bad) == 0, bad


def test_argument_errors_are_caught_before_launch():
    """Fake (never dereferenced) device addresses: every call must return on the host."""
    lib = api.load()
    far = lambda k: P(0x100000000 * k)  # noqa: E731  (far enough from each other)

    def forward(T=8, d_in=64, d_out=32, x=far(1), xs=None, codes=far(2), scale=far(3), epi=None, y=far(4), dt=0, ws=far(5), n=1 << 30):
        return lib.qalora_forward_int8(T, d_in, d_out, x, xs, codes, scale, ctypes.byref(epi) if epi else None, y, dt, ws, n, None)

    for bad in (dict(T=0), dict(T=-3), dict(x=None), dict(codes=None), dict(scale=None), dict(y=None), dict(dt=2), dict(d_in=0),
                dict(d_out=-8), dict(epi=api.Epilogue(5)), dict(epi=api.Epilogue(-1)), dict(y=far(1)), dict(y=far(2)), dict(y=far(3)),
                dict(xs=far(4)), dict(y=P(far(1).value + 16)), dict(epi=api.Epilogue(1, z=far(2).value)),
                dict(epi=api.Epilogue(1, z=far(4).value)), dict(epi=api.Epilogue(1, z=far(1).value)),
                dict(epi=api.Epilogue(0, bias=far(4).value)), dict(epi=api.Epilogue(0, mul=far(4).value)),   # (fp32 y over bf16 mul)
                dict(epi=api.Epilogue(0, residual=far(4).value + 16))):
        assert forward(**bad) == api.EINVAL, bad
    for bad in (dict(d_in=72), dict(d_out=36), dict(d_in=131088), dict(d_out=131080), dict(T=2 ** 29 + 1)):
        assert forward(**bad) == api.EUNSUPPORTED, bad
    for name in ("x", "xs", "codes", "scale", "y", "ws"):
        assert forward(**{name: P(ODD)}) == api.EALIGN, name
    assert forward(epi=api.Epilogue(1, bias=ODD)) == api.EALIGN
    assert forward(ws=None) == forward(n=8 * 64) == api.EWORKSPACE

    def backward(T=8, d_in=64, d_out=32, dy=far(1), codes=far(2), scale=far(3), r=None, dx=far(4), dt=0, ws=far(5), n=1 << 30):
        return lib.qalora_backward_int8(T, d_in, d_out, dy, codes, scale, r, dx, dt, ws, n, None)

    for bad in (dict(T=0), dict(dy=None), dict(codes=None), dict(scale=None), dict(dx=None), dict(dt=-1), dict(d_in=0), dict(dx=far(1)),
                dict(dx=far(2)), dict(dx=far(3)), dict(r=P(far(4).value + 32))):
        assert backward(**bad) == api.EINVAL, bad
    for bad in (dict(d_in=72), dict(d_out=36), dict(d_in=131088), dict(d_out=131080), dict(T=2 ** 29 + 1)):
        assert backward(**bad) == api.EUNSUPPORTED, bad
    for name in ("dy", "codes", "scale", "r", "dx", "ws"):
        assert backward(**{name: P(ODD)}) == api.EALIGN, name
    assert backward(ws=None) == backward(n=8 * 32) == api.EWORKSPACE

    def tokens(T=4, cols=64, x=far(1), f=None, q=far(2), s=far(3)):
        return lib.qalora_quantize_tokens(T, cols, x, f, q, s, None)

    for bad in (dict(T=0), dict(cols=0), dict(x=None), dict(q=None), dict(s=None), dict(q=far(1)), dict(s=far(2)), dict(f=far(2)),
                dict(f=far(3))):
        assert tokens(**bad) == api.EINVAL, bad
    assert tokens(cols=60) == tokens(cols=131080) == api.EUNSUPPORTED
    for name in ("x", "f", "q", "s"):
        assert tokens(**{name: P(ODD)}) == api.EALIGN, name

    def weights(d_in=64, d_out=32, W=far(1), codes=far(2), scale=far(3)):
        return lib.qalora_quantize_int8(d_in, d_out, W, codes, scale, None)

    for bad in (dict(d_in=0), dict(W=None), dict(codes=None), dict(scale=None), dict(codes=far(1)), dict(scale=far(1)), dict(scale=far(2))):
        assert weights(**bad) == api.EINVAL, bad
    assert weights(d_in=72) == weights(d_out=36) == api.EUNSUPPORTED
    for name in ("W", "codes", "scale"):
        assert weights(**{name: P(ODD)}) == api.EALIGN, name

    d = api.make_desc(64, 32, 4, 32)

    def deploy(desc=d, packed=far(1), alpha=far(2), beta=far(3), codes=far(4), scale=far(5)):
        return lib.qalora_deploy_int8(ctypes.byref(desc), packed, alpha, beta, codes, scale, None)

    for bad in (dict(packed=None), dict(alpha=None), dict(beta=None), dict(codes=None), dict(scale=None), dict(codes=far(1)),
                dict(codes=far(2)), dict(scale=far(3)), dict(scale=far(4)), dict(desc=api.make_desc(64, 32, 5, 32))):
        assert deploy(**bad) == api.EINVAL, bad
    assert deploy(desc=api.make_desc(24, 32, 4, 8)) == deploy(desc=api.make_desc(64, 36, 4, 32)) == api.EUNSUPPORTED
    for name in ("packed", "alpha", "beta", "codes", "scale"):
        assert deploy(**{name: P(ODD)}) == api.EALIGN, name

    for call in (lib.qalora_keep8, lib.qalora_restore8):
        for T, cols, a, b in ((0, 64, far(1), far(2)), (4, 0, far(1), far(2)), (4, 64, None, far(2)), (4, 64, far(1), None),
                              (4, 64, far(1), far(1))):
            assert call(T, cols, a, b, None) == api.EINVAL
        assert call(4, 60, far(1), far(2), None) == call(4, 2 ** 29 + 8, far(1), far(2), None) == api.EUNSUPPORTED
        assert call(4, 64, P(ODD), far(2), None) == call(4, 64, far(1), P(ODD), None) == api.EALIGN

    def swiglu(T=4, cols=64, gu=far(1), h=far(2), q=far(3), s=far(4), kept=far(5)):
        return lib.qalora_swiglu_forward8(T, cols, gu, h, q, s, kept, None)

    for bad in (dict(T=0), dict(cols=0), dict(gu=None), dict(q=None), dict(s=None), dict(h=None, q=None, s=None, kept=None), dict(h=far(1)),
                dict(q=far(2)), dict(s=far(3)), dict(kept=far(2)), dict(kept=far(1))):
        assert swiglu(**bad) == api.EINVAL, bad
    assert swiglu(cols=60) == swiglu(cols=131080) == swiglu(T=1 << 30) == api.EUNSUPPORTED
    for name in ("gu", "h", "q", "s", "kept"):
        assert swiglu(**{name: P(ODD)}) == api.EALIGN, name

    def swiglu_back(T=4, cols=64, dh=far(1), kept=far(2), dgu=far(3)):
        return lib.qalora_swiglu_backward_kept8(T, cols, dh, kept, dgu, None)

    for bad in (dict(T=0), dict(cols=0), dict(dh=None), dict(kept=None), dict(dgu=None), dict(dgu=far(1)), dict(dgu=far(2))):
        assert swiglu_back(**bad) == api.EINVAL, bad
    assert swiglu_back(cols=60) == swiglu_back(T=1 << 30) == api.EUNSUPPORTED
    for name in ("dh", "kept", "dgu"):
        assert swiglu_back(**{name: P(ODD)}) == api.EALIGN, name

    def back(act=2, T=5, cols=64, dy=far(1), dt=1, z=far(2), mul=None, dz=far(3), dmul=None, dbias=None, acc=0, ws=None, n=0):
        return lib.qalora_epilogue_backward_kept8(act, T, cols, dy, dt, z, mul, dz, dmul, dbias, acc, ws, n, None)

    for bad in (dict(act=-1), dict(act=5), dict(T=0), dict(cols=0), dict(dy=None), dict(dt=2), dict(dz=None), dict(z=None),
                dict(acc=2), dict(dmul=far(4)), dict(z=None, mul=far(4)), dict(dz=far(2)), dict(mul=far(4), dz=far(4)),
                dict(mul=far(4), dmul=far(4)), dict(mul=far(4), dmul=far(3)), dict(dbias=far(3), T=1), dict(dt=0, dz=far(1))):
        assert back(**bad) == api.EINVAL, bad
    for name in ("dy", "z", "mul", "dz", "dbias", "ws"):
        assert back(**{name: P(ODD)}) == api.EALIGN, name
    assert back(cols=60) == back(cols=2 ** 29 + 8) == api.EUNSUPPORTED
    assert back(T=300, dbias=far(4)) == back(T=300, dbias=far(4), ws=far(5), n=64) == api.EWORKSPACE


def test_kept_values_are_near():
    """The definition itself: half a step off at most, which is 2^-7 of the group's largest magnitude; seven bits restore as bf16."""
    x = ic.drawn_tokens(1, 50, 1000)
    back = ic.restored8(x).double()
    groups = torch.nn.functional.pad(x.double().abs(), (0, 24)).view(50, -1, 32).amax(2).repeat_interleave(32, 1)[:, :1000]
    assert ((back - x.double()).abs() <= 2.0 ** -7 * groups).all()
    q, E = ic.kept8(x)
    assert abs(q).max() <= 127 and (back == torch.from_numpy(q * 2.0 ** (E - 133.0))).all()


def test_rows_are_near():
    v = ic.drawn_tokens(2, 20, 500).float()
    q, s = ic.rows8(v)
    assert ((q * s[:, None].double() - v.double()).abs() <= 0.5 * s[:, None].double() * (1 + 2.0 ** -22)).all()
    assert (q.abs().amax(1) == 127).all()


def test_binding_refusals():
    """What the binding looks at before the C entries see an address: host tensors are refused by name."""
    x, codes = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((32, 64), dtype=torch.int8)
    for call in (lambda: api.forward_int8(x, codes, None), lambda: api.backward_int8(x, codes, None), lambda: api.quantize_tokens(x),
                 lambda: api.keep8(x), lambda: api.quantize_int8(x), lambda: api.swiglu_forward_keep8(x, 32),
                 lambda: api.swiglu_forward_int8(x, 32), lambda: api.swiglu_backward_kept8(x, None, 64),
                 lambda: api.epilogue_backward_kept8(x), lambda: api.restore8(x, 4, 64)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
