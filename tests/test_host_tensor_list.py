"""Host arithmetic behind the calls on lists of tensors (csrc/tensor_list.hpp), compiled for the host, no GPU: arrays that share memory are
found whatever their order, and the units that a list is cut into cover every scalar of every array once."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2201_05989_amd.build import CSRC, INCLUDE, hipcc

HERE = os.path.dirname(os.path.abspath(__file__))
P, U32, U64 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("tensor_list") / "libtensorlist.so")
    subprocess.run([hipcc(), "--cuda-host-only", "-O2", "-std=c++17", "-fPIC", "-shared", f"-I{INCLUDE}", f"-I{CSRC}",
                    os.path.join(HERE, "tensor_list_check.hip"), "-o", out], check=True, capture_output=True)
    so = ctypes.CDLL(out)
    for f in (so.clash2, so.clash5):
        f.argtypes, f.restype = [U32, P, P, P], ctypes.c_int32
    so.places.argtypes, so.places.restype = [U32, P, U32, P, P], U32
    for f in (so.unit_for, so.step_unit_for):
        f.argtypes, f.restype = [U64], U32
    return so


def brute(begin, end, written):
    real = end > begin
    b, e, w = begin[real], end[real], written[real]
    meet = (b[:, None] < e[None, :]) & (b[None, :] < e[:, None]) & (w[:, None] | w[None, :])
    np.fill_diagonal(meet, False)
    return bool(meet.any())


@pytest.mark.parametrize("kinds", [2, 5])
def test_clashes_against_every_pair(lib, kinds):
    rng = np.random.default_rng(kinds)
    seen = set()
    for trial in range(4000):
        n = int(rng.integers(1, 7))
        # few arrays in little memory, or more room: both answers come up often
        room = int(rng.choice([30, 100, 1000]))
        begin = rng.integers(1, room, (kinds, n)).astype(np.uint64)
        size = rng.integers(0, 6, (kinds, n)).astype(np.uint64)
        written = rng.random((kinds, n)) < rng.choice([0.1, 0.5, 1.0])
        if trial % 3 == 0:
            begin.sort(axis=1)
        end, w8 = begin + size, written.astype(np.uint8)
        got = (lib.clash2 if kinds == 2 else lib.clash5)(n, begin.ctypes.data, end.ctypes.data, w8.ctypes.data)
        assert bool(got) == brute(begin.ravel(), end.ravel(), written.ravel()), (begin, size, written)
        seen.add(bool(got))
    assert seen == {True, False}


def test_a_thousand_arrays_in_any_order(lib):
    rng = np.random.default_rng(1)
    n = 1024
    begin = (rng.permutation(5 * n).reshape(5, n) * 64 + (1 << 40)).astype(np.uint64)
    end, written = begin + np.uint64(64), np.ones((5, n), dtype=np.uint8)  # side by side, nothing shared
    call = lambda: lib.clash5(n, begin.ctypes.data, end.ctypes.data, written.ctypes.data)
    assert call() == 0
    end[3, 700] += np.uint64(1)
    assert call() == (1 if int(end[3, 700]) - 1 < (1 << 40) + 5 * n * 64 else 0)


@pytest.mark.parametrize("unit", [1024, 2048, 4096, 8192])
def test_units_cover_every_scalar_once(lib, unit):
    rng = np.random.default_rng(unit)  # (units of 1024 are for short lists)
    for sizes in ([1], [unit], [unit + 1], [unit - 1, 1, unit, 2 * unit], [(1 << 42 if unit > 1024 else 1 << 14) - 3], rng.integers(1, 5 * unit, 240).tolist()):
        n = np.array(sizes, dtype=np.uint64)
        first, last = np.zeros(len(n), dtype=np.uint32), np.zeros(len(n), dtype=np.uint32)
        units = lib.places(len(n), n.ctypes.data, unit, first.ctypes.data, last.ctypes.data)
        ends = np.append(first[1:], units).astype(np.int64)
        of = ends - first
        assert first[0] == 0 and (of >= 1).all() and ((last >= 1) & (last <= unit)).all()
        assert ((of - 1) * unit + last == n.astype(np.int64)).all()


def test_rules_for_units(lib):
    for rule in (lib.unit_for, lib.step_unit_for):
        units = [rule(1 << k) for k in range(43)]
        assert units == sorted(units) and units[0] == 2048 and units[-1] == 8192
        assert (1 << 42) // units[-1] + 1024 + 1024 < 1 << 32   # numbers of units, and one turn beyond the last, fit 32 bits
    assert lib.unit_for(4 << 20) == 2048 and lib.unit_for((4 << 20) + 1) == 4096 and lib.unit_for((8 << 20) + 1) == 8192
    assert lib.step_unit_for(8 << 20) == 2048 and lib.step_unit_for((8 << 20) + 1) == 8192
