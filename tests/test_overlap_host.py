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


def test_forwards_refuse_outputs_over_what_is_still_read():
    """Every form: few tokens, mid tokens and dense, with an adapter and what it keeps, deployed.  Operands of 2 MB at most."""
    lib = api.load()
    d_in = d_out = 1024

    def spans(T, dt):
        n = T * d_out
        y = n * (2 if dt == api.BF16 else 4)
        return dict(x=2 * T * d_in, bias=4 * d_out, mul=2 * n, residual=y, y=y, z=2 * n)

    for form, T, dt in itertools.product(("merged", "kept", "deployed"), (1, 3, 7, 40, 300), (api.F32, api.BF16)):
        d = api.make_desc(d_in, d_out, 4, 32, 16 if form == "kept" else 0, 0.5 if form == "kept" else 0.0)
        size = spans(T, dt)
        if form == "kept":
            size["kept"] = int(lib.qalora_kept_bytes(ctypes.byref(d), T))
        base = {name: (k + 1) * 4 * M for k, name in enumerate(size)}
        far = P(100 * M)

        def call(**at):
            a = {**base, **at}
            epi = api.Epilogue(2, a["bias"], a["mul"], a["residual"], a["z"])
            A = far if form == "kept" else None
            if form == "deployed":
                return lib.qalora_forward_deployed_epilogue(ctypes.byref(d), T, P(a["x"]), far, far, ctypes.byref(epi), P(a["y"]), dt,
                                                            P(200 * M), 1 << 28, None)
            return lib.qalora_forward_epilogue(ctypes.byref(d), T, P(a["x"]), far, far, far, A, A, ctypes.byref(epi), P(a["y"]), dt,
                                               P(a["kept"]) if form == "kept" else None, P(200 * M), 1 << 28, None)

        outs = [name for name in ("y", "z", "kept") if name in size]
        for out, other in itertools.product(outs, size):
            if out == other:
                continue
            for off in (0, 16, 16 - size[out], size[other] - 16):    # from one start on, and by any amount
                may = off == 0 and out == "y" and (other == "residual" or (other == "mul" and dt == api.BF16))
                if not may and (off == 0 or (off < size[other] and -off < size[out])):
                    assert call(**{out: base[other] + off}) == api.EINVAL, (form, T, dt, out, other, off)
