"""What a stage of a product's loads may reach of an operand (csrc/gemm_stage.h, compiled here for the host): all that is its own, and of what lies behind a row's end or
behind the last row nothing that counts, whether a load's bounds go by its first byte or by that byte's word."""
import ctypes as C
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
STAGE = 64


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("stage") / "stage.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "csrc", "gemm_stage_host.cpp"), "-o", so], check=True)
    lib = C.CDLL(so)
    lib.bytes_of_stage.argtypes, lib.bytes_of_stage.restype = [C.c_int] + [C.c_uint32] * 3, C.c_uint32
    lib.ld_of.argtypes, lib.ld_of.restype = [C.c_uint64] * 3, C.c_uint64
    return lib


def lds(rows, cols):
    """The distances of rows that are read as they lie: multiples of 8, but any for a row alone."""
    up = (cols + 7) // 8 * 8
    return range(cols, cols + 9) if rows == 1 else (up, up + 8, 4096)


@pytest.mark.parametrize("edge", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 2, 3, 63, 64])
def test_across(lib, rows, edge):
    """Rows of K; a lane reads 16 bytes of each of a stage's 64, also where there are fewer."""
    for cols in list(range(1, 300)) + [511, 513, 1001]:
        for ld in lds(rows, cols):
            at = lib.ld_of(rows, cols, ld)
            assert at >= cols and (rows == 1 or at == ld)
            for first in range(0, cols, edge):
                count = min(edge, cols - first)
                end = lib.bytes_of_stage(1, rows, count, 2 * at)
                assert 2 * ((rows - 1) * at + count) <= end <= (2 * ((rows - 1) * at + count) + 3) // 4 * 4
                beyond = rows * 2 * at                                   # the first load of the row behind the last one
                assert beyond // 4 * 4 >= end, (rows, cols, ld, first)


@pytest.mark.parametrize("edge", [64, 128, 256])
def test_along(lib, edge):
    """Rows of M or N, whose parts of K are multiples of 8 elements."""
    for rows in (1, 2, edge - 1, edge):
        for cols in range(8, 264, 8):
            for ld in lds(rows, cols):
                at = lib.ld_of(rows, cols, ld)
                for k0 in range(0, cols, STAGE):
                    count = min(STAGE, cols - k0)
                    end = lib.bytes_of_stage(0, rows, count, 2 * at)
                    assert end == 2 * ((rows - 1) * at + count)
                    if rows < edge:
                        assert rows * 2 * at // 4 * 4 >= end, (rows, cols, ld, k0)


def test_nothing(lib):
    for across in (0, 1):
        assert lib.bytes_of_stage(across, 0, 8, 64) == 0 and lib.bytes_of_stage(across, 8, 0, 64) == 0
