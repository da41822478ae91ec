"""The orthogonalised update without a GPU: its launch table and workspace, and the refusals of its C entries."""
import ctypes
import random

import pytest

from host_code import host_library
from paper_2309_14717_amd import api

SOURCE = r"""
#include "muon_plan.hpp"
using namespace qalora;
static MuonTable table;
extern "C" long long plan(int n, const int* rows, const int* cols, int* unsupported) {
  bool u;
  const size_t floats = muon_table(n, rows, cols, table, u);
  *unsupported = u;
  return (long long)floats;
}
extern "C" void totals(long long* out) {
  out[0] = table.blocks; out[1] = table.reduce_blocks; out[2] = table.per_block; out[3] = table.tiles; out[4] = table.alone; out[5] = table.direct;
}
extern "C" void tensor(int i, long long* out) {
  const MuonTensor& t = table.t[i];
  out[0] = table.tiles; out[1] = t.chunks; out[2] = table.block0[i]; out[3] = table.reduce0[i];
  out[4] = (long long)t.x; out[5] = (long long)t.gram; out[6] = (long long)t.partial;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    lib = host_library(tmp_path_factory.mktemp("muon"), "muon_plan", SOURCE)
    lib.plan.restype = ctypes.c_longlong

    def of(shapes):
        n = len(shapes)
        arr = ctypes.c_int * max(n, 1)
        u = ctypes.c_int()
        floats = lib.plan(n, arr(*(r for r, _ in shapes)), arr(*(c for _, c in shapes)), ctypes.byref(u))
        tot, ts = (ctypes.c_longlong * 6)(), []
        lib.totals(tot)
        for i in range(n if floats else 0):
            t = (ctypes.c_longlong * 7)()
            lib.tensor(i, t)
            ts.append(list(t))
        return floats, bool(u.value), list(tot), ts

    return of


def test_table_covers_every_matrix_once(plan):
    rng = random.Random(3)
    lists = [[(rng.randint(1, 128), rng.randint(1, 30000)) for _ in range(rng.randint(1, 32))] for _ in range(200)]
    lists += [[(rng.randint(1, 64), rng.randint(1, 1200)) for _ in range(rng.randint(1, 4))] for _ in range(100)]
    lists += [[(1, 1)], [(128, 2 ** 27)], [(2 ** 27, 1)], [(128, 128)] * 32, [(64, 1000000)] * 32]
    for shapes in lists:
        shapes = [s if rng.random() < 0.5 else s[::-1] for s in shapes]
        floats, unsupported, (blocks, reduce_blocks, per_block, tiles, alone, direct), ts = plan(shapes)
        assert floats > 0 and not unsupported
        end = block = reduce = 0
        for (rows, cols), (_, chunks, block0, reduce0, x, gram, partial) in zip(shapes, ts):
            short, long = min(rows, cols), max(rows, cols)
            assert tiles in (1, 2, 4) and short <= 32 * tiles and 32 * (chunks - 1) < long <= 32 * chunks
            slices, upper = -(-chunks // per_block), tiles * (tiles + 1) // 2
            assert (block0, reduce0, x) == (block, reduce, end)           # regions follow each other without a gap
            assert gram == x + chunks * tiles * 32 * 32 and partial == gram + tiles * tiles * 1024
            end, block, reduce = partial + slices * upper * 1024 * (1 + direct), block + slices, reduce + 8 * upper
            assert x % 4 == gram % 4 == partial % 4 == 0                  # 16-byte accesses
        assert direct == (tiles < 4 and -(-max(t[1] for t in ts) // per_block) * tiles * (tiles + 1) // 2 <= 48)
        assert alone == (tiles < 4 and max(max(s) for s in shapes) <= 768 // tiles)
        assert max(min(s) for s in shapes) > (32 * tiles // 2 if tiles > 1 else 0)
        assert (floats, blocks, reduce_blocks) == (end, block, reduce) and blocks < 2 ** 31


def test_unacceptable_lists(plan):
    assert plan([(129, 129)])[:2] == (0, True)
    assert plan([(8, 8), (300, 129)])[:2] == (0, True)
    assert plan([(8, 2 ** 27 + 1)])[:2] == (0, True) and plan([(2 ** 31 - 1, 8)])[:2] == (0, True)
    for shapes in ([], [(0, 4)], [(4, 0)], [(-1, 4)], [(4, 4)] * 33):
        assert plan(shapes)[:2] == (0, False)


def test_argument_errors_are_caught_before_launch():
    """Fake (never dereferenced) device addresses: every call must return on the host."""
    lib = api.load()
    I2, P2 = ctypes.c_int32 * 2, ctypes.c_void_p * 2
    rows, cols = I2(16, 64), I2(400, 8)
    size = lib.qalora_muon_workspace_bytes(2, rows, cols)
    assert size > 4 * (16 * 400 + 64 * 8)
    assert lib.qalora_muon_workspace_bytes(2, I2(16, 129), I2(400, 129)) == 0
    assert lib.qalora_muon_workspace_bytes(0, rows, cols) == lib.qalora_muon_workspace_bytes(2, None, cols) == 0
    good, odd, none = P2(0x10000, 0x20000), P2(0x10000, 0x20004), P2(0x10000, None)
    G, M = P2(0x30000, 0x40000), P2(0x50000, 0x60000)
    W = ctypes.c_void_p(0x100000)

    def call(hp=api.Muon(lr=0.1), n=2, p=good, g=G, m=M, r=rows, c=cols, ws=W, nbytes=size):
        return lib.qalora_muon_step(ctypes.byref(hp) if hp else None, n, p, g, m, r, c, 0, ws, nbytes, None)

    for bad in (dict(hp=None), dict(p=None), dict(g=None), dict(m=None), dict(r=None), dict(c=None), dict(n=0), dict(n=33),
                dict(p=none), dict(g=none), dict(m=none), dict(r=I2(0, 8))):
        assert call(**bad) == api.EINVAL, bad
    end = 0x10000 + 4 * 16 * 400
    for bad in (dict(p=P2(0x10000, 0x10000)), dict(g=good), dict(m=good), dict(m=G), dict(p=P2(0x10000, 0x10010)),
                dict(g=P2(0x30000, end - 16)), dict(m=P2(0x20000 + 4 * 64 * 8 - 16, 0x70000))):
        assert call(**bad) == api.EINVAL, bad        # matrices that overlap
    assert call(p=P2(0x10000, end), ws=None) == api.EWORKSPACE   # neighbours do not
    nan, inf = float("nan"), float("inf")
    for hp in (dict(lr=-1.0), dict(lr=nan), dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=nan), dict(eps=0.0),
               dict(eps=nan), dict(weight_decay=-1.0), dict(steps=0), dict(steps=17), dict(scale_mode=3), dict(scale_mode=-1),
               dict(a=nan), dict(b=inf), dict(c=-inf)):
        assert call(hp=api.Muon(**{"lr": 0.1, **hp})) == api.EINVAL, hp
    for bad in (dict(p=odd), dict(g=odd), dict(m=odd), dict(ws=ctypes.c_void_p(0x100008))):
        assert call(**bad) == api.EALIGN, bad
    assert call(r=I2(129, 8), c=I2(129, 8)) == api.EUNSUPPORTED
    assert call(ws=None) == call(nbytes=size - 256) == call(nbytes=0) == api.EWORKSPACE
