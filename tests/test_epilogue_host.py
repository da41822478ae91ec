"""The epilogue without a GPU: which kernels the GPU tests' shapes reach, the backward's launch shape, the slopes against
differences, and the refusals of the C entries."""
import ctypes
import random

import pytest
import torch

import epilogue_cases as ec
from host_code import host_library
from paper_2309_14717_amd import api

SOURCE = r"""
#include "epilogue_plan.hpp"
#include "gemm_plan.hpp"
using namespace qalora;
extern "C" void gemm(int bits, int M, int N, int K, int g, int* o) {
  const GemmPlan p = gemm_dq_plan(bits, M, N, K, g, false);
  o[0] = p.tile_rows; o[1] = p.ksplit; o[2] = gemm_fast_shape(K, g);
}
extern "C" void back(int rows, int cols, int* o) {
  const EpilogueBackPlan p = epilogue_back_plan(rows, cols);
  o[0] = p.lanes; o[1] = p.col_blocks; o[2] = p.row_blocks; o[3] = p.rows_per;
}
extern "C" long long floats(int rows, int cols) { return (long long)epilogue_back_floats(rows, cols); }
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    lib = host_library(tmp_path_factory.mktemp("epilogue"), "epilogue_plan", SOURCE)
    lib.floats.restype = ctypes.c_longlong
    return lib


def test_shapes_reach_every_dense_form(host):
    o = (ctypes.c_int * 3)()
    for (T, d_in, d_out, bits, group), (rows, split, fast) in ec.DENSE.items():
        host.gemm(bits, T, d_out, d_in, group, o)
        assert (o[0], o[1] > 1, bool(o[2])) == (rows, split, fast), (T, d_in, d_out, bits, group, list(o))
        assert api.mid_blocks(api.make_desc(d_in, d_out, bits, group), T) == 0
    for T, d_in, d_out, bits, group in ec.MID:
        assert api.mid_blocks(api.make_desc(d_in, d_out, bits, group), T) > 0 and T > (32 if bits == 4 else 16)


def test_backward_blocks_cover_the_matrix(host):
    rng = random.Random(5)
    sizes = [(1, 8), (2 ** 31 - 1, 8), (1, 2 ** 31 - 8), (4096, 11008), (300000, 8), (7, 520)]
    sizes += [(rng.randint(1, 10 ** rng.randint(1, 6)), 8 * rng.randint(1, 10 ** rng.randint(1, 4))) for _ in range(500)]
    o = (ctypes.c_int * 4)()
    for rows, cols in sizes:
        host.back(rows, cols, o)
        lanes, cb, rb, per = o
        assert lanes in (8, 16, 32, 64) and 256 % lanes == 0 and per % (256 // lanes) == 0 and per > 0
        assert lanes * 8 * (cb - 1) < cols <= lanes * 8 * cb
        assert per * (rb - 1) < rows <= per * rb and rb <= 65535
        assert host.floats(rows, cols) == (rb * cols if rb > 1 else 0)
        assert api.load().qalora_epilogue_backward_workspace_bytes(rows, cols) >= (4 * rb * cols if rb > 1 else 0)
        assert rows > 256 or rb == 1


@pytest.mark.parametrize("act", ec.ACTS)
def test_slopes_are_the_differences_of_the_values(act):
    z = torch.linspace(-9, 9, 4001, dtype=torch.float64) + 1e-3   # (not at relu's corner)
    h = 1e-5
    slope = (ec.act64(z + h, act)[0] - ec.act64(z - h, act)[0]) / (2 * h)
    assert (ec.act64(z, act)[1] - slope).abs().max() <= 1e-9


def test_argument_errors_are_caught_before_launch():
    """Fake (never dereferenced) device addresses: every call must return on the host."""
    lib = api.load()
    P = ctypes.c_void_p
    good, odd = P(0x10000), P(0x10004)
    d = api.make_desc(1024, 1024, 4, 32, 16, 2.0)

    def forward(desc=d, T=64, x=good, packed=good, alpha=good, beta=good, A=None, B=None, epi=api.Epilogue(), y=good, dt=0,
                kept=None, ws=good, n=1 << 30):
        return lib.qalora_forward_epilogue(ctypes.byref(desc), T, x, packed, alpha, beta, A, B,
                                           ctypes.byref(epi) if epi else None, y, dt, kept, ws, n, None)

    for bad in (dict(x=None), dict(packed=None), dict(alpha=None), dict(y=None), dict(T=0), dict(dt=2), dict(A=good),
                dict(kept=good), dict(epi=api.Epilogue(-1)), dict(epi=api.Epilogue(5))):
        assert forward(**bad) == api.EINVAL, bad
    for k, name in enumerate(("bias", "mul", "residual", "z")):
        assert forward(epi=api.Epilogue(1, **{name: 0x10008})) == api.EALIGN, name
    for name in ("mul", "residual"):
        assert forward(epi=api.Epilogue(1, z=0x20000, **{name: 0x20000})) == api.EINVAL, name
    assert forward(epi=api.Epilogue(0, z=0x10000)) == api.EINVAL       # y
    assert forward(x=odd) == forward(y=odd) == api.EALIGN
    for epi in (None, api.Epilogue(2, bias=0x10000)):
        assert forward(epi=epi, n=64) == forward(epi=epi, ws=None) == api.EWORKSPACE
    assert forward(desc=api.make_desc(64, 60, 4, 32)) == api.EUNSUPPORTED

    def deployed(T=2, x=good, packed=None, dep=good, epi=api.Epilogue(1), y=good, dt=0, ws=good, n=64):
        return lib.qalora_forward_deployed_epilogue(ctypes.byref(d), T, x, packed, dep, ctypes.byref(epi), y, dt, ws, n, None)

    assert deployed(x=None) == deployed(dep=None) == deployed(T=5) == deployed(epi=api.Epilogue(9)) == api.EINVAL
    assert deployed(epi=api.Epilogue(1, mul=0x10002)) == api.EALIGN
    assert deployed() == deployed(T=100, packed=good) == api.EWORKSPACE

    def back(act=2, T=5, cols=64, dy=good, dt=1, z=good, mul=None, dz=good, dmul=None, dbias=None, acc=0, ws=None, n=0):
        return lib.qalora_epilogue_backward(act, T, cols, dy, dt, z, mul, dz, dmul, dbias, acc, ws, n, None)

    for bad in (dict(act=-1), dict(act=5), dict(T=0), dict(cols=0), dict(dy=None), dict(dt=2), dict(dz=None), dict(z=None),
                dict(acc=2), dict(dmul=good), dict(mul=good, dmul=good), dict(act=0, z=None, mul=good, dmul=good)):
        assert back(**bad) == api.EINVAL, bad
    for name in ("dy", "z", "mul", "dz", "dbias", "ws"):
        assert back(**{name: odd}) == api.EALIGN, name
    assert back(cols=60) == back(cols=2 ** 29 + 8) == api.EUNSUPPORTED
    assert back(T=300, dbias=good) == back(T=300, dbias=good, ws=good, n=64) == api.EWORKSPACE
    assert lib.qalora_epilogue_backward_workspace_bytes(0, 64) == lib.qalora_epilogue_backward_workspace_bytes(4, 60) == 0
    assert lib.qalora_epilogue_backward_workspace_bytes(4, 2 ** 29 + 8) == 0
