"""Attention over 8-bit stores and lists of blocks: workgroups and their work.  A launch has a workgroup for every tile of
columns of every (sequence, kv head, split); the dies take them round-robin by linear index.  No GPU."""
import ctypes
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DIES = 8


@pytest.fixture(scope="module")
def work(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("host") / "host_units_work.so")
    subprocess.check_call(
        ["g++", "-std=c++17", "-O1", "-w", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-x", "c++", os.path.join(ROOT, "tests", "host_units_work.cpp"),
         "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2501_05408_amd", "csrc"), "-o", path])
    fn = ctypes.CDLL(path).units_work_of
    fn.argtypes = [ctypes.c_uint32] * 6 + [ctypes.c_int, ctypes.POINTER(ctypes.c_int32)]
    out = (ctypes.c_int32 * 4)()

    def call(*args):
        fn(*args, out)
        return tuple(out)

    return call


@pytest.mark.parametrize("Hkv", [1, 2, 3, 4, 6, 8, 12])
def test_all_work_is_taken_once_and_a_units_tiles_on_one_die(work, Hkv):
    for tiles, B, splits in itertools.product((1, 2, 3, 4, 8), (1, 2, 5, 16), (1, 2, 3, 7)):
        nx, units = Hkv * tiles, Hkv * B * splits
        dies, seen = {}, set()
        for z, y, x in itertools.product(range(splits), range(B), range(nx)):
            hkv, tile, b, split = got = work(x, y, z, nx, B, splits, Hkv)
            assert 0 <= hkv < Hkv and 0 <= tile < tiles and 0 <= b < B and 0 <= split < splits
            seen.add(got)
            dies.setdefault((split, b, hkv), set()).add((x + nx * (y + B * z)) % DIES)
        assert len(seen) == units * tiles
        whole = sorted(dies)[:units // DIES * DIES]            # splits in turn, as launched; the rest is fewer than the dies
        assert all(len(dies[unit]) == 1 for unit in whole)


def test_far_indexes(work):
    nx, ny, nz, Hkv = 2000, 20000, 50, 500                      # 2e9 workgroups
    assert work(0, 0, 0, nx, ny, nz, Hkv) == (0, 0, 0, 0)
    assert work(nx - 1, ny - 1, nz - 1, nx, ny, nz, Hkv) == (Hkv - 1, 3, ny - 1, nz - 1)
