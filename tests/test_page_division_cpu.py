"""Positions divided by a page's size with a product, against the division (page_division.hip: the kernels' own function, built for the host)."""
import ctypes
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("division") / "page_division.so")
    subprocess.check_call(["hipcc", "--offload-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC", "-shared", "-fsanitize=signed-integer-overflow",
                           "-fsanitize-trap=signed-integer-overflow", "-o", so, os.path.join(HERE, "page_division.hip")], stderr=subprocess.DEVNULL)
    lib = ctypes.CDLL(so)
    lib.t_divided.restype, lib.t_divided.argtypes = ctypes.c_uint32, (ctypes.c_uint32, ctypes.c_uint32)
    lib.t_first_wrong.restype, lib.t_first_wrong.argtypes = ctypes.c_int64, (ctypes.c_uint32, ctypes.c_uint32)
    return lib


@pytest.mark.parametrize("size", [1, 2, 3, 5, 7, 16, 17, 20, 64, 100, 127, 128, 129, 255, 256, 257, 1000, 65535, 65536, 65537, 2 ** 20 - 1, 2 ** 29, 2 ** 29 + 1,
                                  2 ** 30 - 1, 2 ** 30])
def test_beside_every_multiple(lib, size):
    assert lib.t_first_wrong(size, max(1, 200 // size)) == -1


def test_any_size_and_number(lib):
    rng = random.Random(3)
    for _ in range(50000):
        size, x = rng.randrange(1, 2 ** rng.randrange(1, 31) + 1), rng.randrange(2 ** rng.randrange(1, 32))
        assert lib.t_divided(x, size) == x // size, (x, size)
