"""Whole numbers that a C int does not hold are refused by the binding: taken modulo 2^32, a matrix of 2^32 + 4 rows would be one of four."""
import ctypes

import pytest

from paper_2309_14717_amd import api

FAR = [ctypes.c_void_p(0x100000000 * k) for k in range(1, 6)]   # (never dereferenced)
PAST = [2 ** 31, 2 ** 32 + 8, -2 ** 31 - 1, -2 ** 32 + 8]


@pytest.mark.parametrize("n", PAST)
def test_sizes(n):
    desc = api.make_desc(64, 32, 4, 32)
    for call in (lambda: api.kept8_bytes(n, 8), lambda: api.kept8_bytes(8, n), lambda: api.int8_workspace_bytes(n, 64, 32, api.OP_FORWARD),
                 lambda: api.int8_workspace_bytes(8, n, 32, api.OP_FORWARD), lambda: api.int8_workspace_bytes(8, 64, n, api.OP_BACKWARD),
                 lambda: api.workspace_bytes(desc, n, api.OP_FORWARD)):
        with pytest.raises(ctypes.ArgumentError, match="C int"):
            call()


@pytest.mark.parametrize("n", PAST)
def test_rows_and_columns(n):
    """As the Python forms call the library: what the native forms leave to them comes here."""
    lib = api.load()
    a, b, c, d, e = FAR
    for call, args in ((lib.qalora_quantize_tokens, (n, 64, a, None, b, c, None)), (lib.qalora_quantize_tokens, (4, n, a, None, b, c, None)),
                       (lib.qalora_keep8, (n, 64, a, b, None)), (lib.qalora_restore8, (4, n, a, b, None)),
                       (lib.qalora_swiglu_forward8, (n, 64, a, b, None, None, c, None)), (lib.qalora_swiglu_backward_kept8, (n, 64, a, b, c, None)),
                       (lib.qalora_quantize_int8, (64, n, a, b, c, None)),
                       (lib.qalora_epilogue_backward_kept8, (2, n, 64, a, 1, b, None, c, None, None, 0, None, 0, None)),
                       (lib.qalora_epilogue_backward, (2, n, 64, a, 1, b, None, c, None, None, 0, None, 0, None)),
                       (lib.qalora_forward_int8, (n, 64, 32, a, None, b, c, None, d, 0, e, 1 << 30, None)),
                       (lib.qalora_backward_int8, (n, 64, 32, a, b, c, None, d, 0, e, 1 << 30, None))):
        with pytest.raises(ctypes.ArgumentError, match="C int"):
            call(*args)


def test_ints_at_the_ends_are_taken():
    assert api.kept8_bytes(2 ** 31 - 1, 8) > 2 ** 31 and api.kept8_bytes(-2 ** 31, 8) == 0


@pytest.mark.parametrize("n", PAST)
def test_a_layers_sizes(n):
    for sizes in ((n, 32, 4, 32), (64, n, 4, 32), (64, 32, n, 32), (64, 32, 4, n), (64, 32, 4, 32, n)):
        with pytest.raises(ValueError, match="C int"):
            api.make_desc(*sizes)
