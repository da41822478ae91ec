"""Which few-token products of 8-bit integers go in one launch: never more tokens than its LDS holds, and not where the blocks of a
compute unit would bring them to 8 bits over and over."""
import ctypes
import random

import pytest

from host_code import host_library

SOURCE = r"""
#include "stream_i8_plan.hpp"
extern "C" int takes(int tokens, int K, int N) { return qalora::stream8_takes(tokens, K, N); }
"""


@pytest.fixture(scope="module")
def takes(tmp_path_factory):
    return host_library(tmp_path_factory.mktemp("stream8"), "stream8", SOURCE).takes


def test_room(takes):
    rng = random.Random(1)
    for _ in range(20000):
        T, K, N = rng.randint(1, 40), 16 * rng.randint(1, 8192), 8 * rng.randint(1, 16384)
        assert not takes(T, K, N) or (T <= 16 and T * K <= 16384)


@pytest.mark.parametrize("size", [(1, 16, 8), (16, 1024, 1024), (16, 1024, 4096), (8, 1024, 8192), (16, 1024, 8192), (8, 1024, 12288), (1, 1024, 13824), (4, 4096, 4096), (1, 4096, 11008), (2, 8192, 8192),
                                  (1, 8192, 22016), (1, 11008, 4096), (1, 16384, 131072)], ids=str)
def test_one_launch(takes, size):
    assert takes(*size)


@pytest.mark.parametrize("size", [(17, 16, 8), (16, 1040, 8), (16, 1024, 9216), (16, 1024, 22016), (8, 2048, 22016), (16, 256, 131072),
                                  (1, 1024, 65536), (2, 8192, 22016), (1, 16400, 8)], ids=str)
def test_two_launches(takes, size):
    assert not takes(*size)


def test_a_wider_weight_is_not_taken_where_a_narrower_is_not(takes):
    for T in range(1, 17):
        for K in (64, 512, 1024, 2048, 4096, 8192, 16384):
            got = [takes(T, K, N) for N in range(1024, 131073, 1024)]
            assert got == sorted(got, reverse=True), (T, K)
