"""Operands that lie over each other in the calls with an epilogue: refused on the host, before anything is launched."""
import ctypes
import itertools

from paper_2309_14717_amd import api

P = ctypes.c_void_p
M = 1 << 20  # distance between the operands, more than any of them takes


def test_backward_refuses_outputs_over_what_is_still_read():
    """Fake (never dereferenced) device addresses.  T = 300 rows of 64: dz and dmul 38400 bytes, dy twice that in fp32."""
    lib, T, cols = api.load(), 300, 64
    two = 2 * T * cols
    where = dict(dy=P(1 * M), z=P(2 * M), mul=P(3 * M), dz=P(4 * M), dmul=P(5 * M), dbias=P(6 * M))

    def back(dt=api.BF16, **at):
        a = {**where, **at}
        return lib.qalora_epilogue_backward(2, T, cols, a["dy"], dt, a["z"], a["mul"], a["dz"], a["dmul"], a["dbias"], 0, P(7 * M),
                                            1 << 19, None)

    for out in ("dz", "dmul"):
        # rows of an fp32 dy that other blocks have yet to read: over its start, its second half, its last 16 bytes
        for off in (0, two, 2 * two - 16):
            assert back(dt=api.F32, **{out: P(1 * M + off)}) == api.EINVAL, (out, off)
        # shifted by a row either way, against each input
        for k, off in itertools.product((1, 2, 3), (-2 * cols, 2 * cols, two - 16, 16 - two)):
            assert back(**{out: P(k * M + off)}) == api.EINVAL, (out, k, off)
    for off in (-2 * cols, 0, 2 * cols, two - 16, 16 - two):
        assert back(dmul=P(4 * M + off)) == api.EINVAL, off
    for k in (1, 2, 3, 4, 5):
        for off in (0, 16 - 4 * cols, two - 16):
            assert back(dbias=P(k * M + off)) == api.EINVAL, (k, off)
