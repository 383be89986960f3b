"""The attention's units of work at sizes that no test can run: the arithmetic of the kernel's own source, compiled for the
host."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2608_25431_amd import build, gift
from test_kv_refusals import attention, lib  # noqa: F401

SOURCE = """
#include "gift_kv_units.hpp"
extern "C" {
uint32_t small(uint32_t a, uint32_t b) { return gift::quotient(a, b); }
uint64_t large(uint64_t a, uint64_t b) { return gift::quotient(a, b, 1.0 / (double)b); }
uint64_t unit(uint64_t at, uint32_t rounds) {
  const gift::Unit u = gift::unit_of(at, rounds);
  return (uint64_t)u.column << 32 | u.round;
}
}
"""


@pytest.fixture(scope="module")
def units(tmp_path_factory):
    d = tmp_path_factory.mktemp("units")
    (d / "units.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I", build.CSRC, "-I",
                    "/opt/rocm/include", str(d / "units.cpp"), "-o", str(d / "units.so")], check=True, timeout=120)
    so = ctypes.CDLL(os.path.join(d, "units.so"))
    so.small.argtypes, so.small.restype = [ctypes.c_uint32, ctypes.c_uint32], ctypes.c_uint32
    so.large.argtypes, so.large.restype = [ctypes.c_uint64, ctypes.c_uint64], ctypes.c_uint64
    so.unit.argtypes, so.unit.restype = [ctypes.c_uint64, ctypes.c_uint32], ctypes.c_uint64
    return so


@pytest.mark.parametrize("columns,rounds", [(1, 1), (7, 3), (1 << 18, 1 << 14), ((1 << 18) + 5, (1 << 14) + 1), (70000001, 3),
                                            (70000001, 67108863), (1 << 26, (1 << 26) - 1)])
def test_a_unit_of_any_request(units, columns, rounds):
    r = random.Random(columns)
    n = columns * rounds
    some = [0, n - 1, n // 2, rounds - 1, rounds % n, (1 << 32) % n, ((1 << 32) - 1) % n, (columns - 1) * rounds]
    for at in some + [r.randrange(n) for _ in range(2000)] + [c * rounds for c in (r.randrange(columns) for _ in range(500))]:
        u = units.unit(at, rounds)
        assert (u >> 32, u & 0xFFFFFFFF) == divmod(at, rounds), at


def test_quotients(units):
    r = random.Random(1)
    for _ in range(20000):
        a, b = r.getrandbits(r.randint(1, 32)), r.getrandbits(r.randint(1, 32)) or 1
        assert units.small(a, b) == a // b, (a, b)
        a, b = r.getrandbits(r.randint(1, 63)), r.getrandbits(r.randint(1, 40)) or 1
        if a // b < 1 << 56:
            assert units.large(a, b) == a // b, (a, b)
    for b in (1, 2, 3, 255, 256, 512, 65535, 8388607):
        for a in (k * b + d for k in (1, 2, 1000, (1 << 23) // b, (1 << 54) // b) for d in (-1, 0, 1) if k):
            assert units.large(a, b) == a // b, (a, b)
            if a < 1 << 32:
                assert units.small(a, b) == a // b, (a, b)


def test_rows_that_no_memory_holds(lib):  # noqa: F811
    assert attention(lib, n_rows=1 << 27) == gift.E_TOO_LARGE and "n_heads" in gift.last_error()
