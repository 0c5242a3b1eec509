"""Attention over the paged cache in as many launches as its workgroups need: the plan's threads, compiled for the host, and the source that launches."""
import ctypes
import pathlib
import re
import shutil
import subprocess

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2210_15748_amd" / "csrc"
SOURCE = """
#include "cache_plans.hpp"
extern "C" uint64_t launches(uint64_t seqs, uint64_t tokens, uint32_t heads, uint32_t group, uint32_t dim, uint64_t length, int lists, uint64_t* out, int room) {
    const dessert::AttendPlan p = dessert::attend_plan(seqs, tokens, heads, group, dim, length, lists);
    int at = 0;
    dessert::attend_launches(p, [&](uint32_t first, uint32_t workgroups) {
        if (at < room) { out[3 + 2 * at] = first; out[4 + 2 * at] = workgroups; }
        ++at;
    });
    out[0] = p.rows; out[1] = p.few; out[2] = p.waves;
    return (uint64_t)at << 32 | p.groups * p.parts;
}
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    d = tmp_path_factory.mktemp("launches")
    (d / "rule.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-O1", "-shared", "-fPIC", "-I", str(CSRC), str(d / "rule.cpp"), "-o", str(d / "rule.so")],
                   check=True)
    lib = ctypes.CDLL(str(d / "rule.so"))
    lib.launches.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int,
                             ctypes.POINTER(ctypes.c_uint64), ctypes.c_int]
    lib.launches.restype = ctypes.c_uint64

    def of(*sizes):
        out = (ctypes.c_uint64 * 2003)()
        n = lib.launches(*sizes, out, 1000)
        return n & 0xFFFFFFFF, out[0], bool(out[1]), out[2], [tuple(out[3 + 2 * i:5 + 2 * i]) for i in range(n >> 32)]
    return of


@pytest.mark.parametrize("sizes", [(1024, 65536, 8, 4, 128, 9000, 0), (1100, 65536, 8, 4, 160, 9000, 0), (3000, 65536, 8, 4, 192, 9000, 0),
                                   (70000, 32768, 1, 1, 128, 48, 0), (60000, 100000, 4, 8, 64, 100, 0), (2000000, 1, 8, 4, 128, 500, 0), (1, 1, 1, 1, 32, 1, 0),
                                   (1, 1, 8, 4, 128, 100000, 0), (16, 1, 8, 4, 96, 900, 0), (16000000, 1, 1, 4, 256, 900, 1), (7, 500, 3, 5, 160, 700, 0)])
def test_every_workgroup_in_one_launch_that_can_be_made(launches, sizes):
    total, rows, few, waves, parts = launches(*sizes)
    assert waves == (rows // 32 if not few else waves) and waves in (4, 8)
    at = 0
    for first, workgroups in parts:
        assert first == at and workgroups > 0
        assert workgroups * 64 * waves < 1 << 32
        at += workgroups
    assert at == total


def test_attention_is_launched_that_way():
    """Each launch takes its number of workgroups from a slice, and as many threads as the plan's waves say; a workgroup counts from the slice's first."""
    text = (CSRC / "attention_kernels.hip").read_text()
    found = re.findall(r"attend_(few|many)_kernel<ND, (\d), \w+><<<(\w+), dim3\((\d+)\)", text)
    assert len(found) == 8
    assert all(grid == "grid" and int(threads) == 64 * int(waves) for _, waves, grid, threads in found)
    assert "const dim3 grid(workgroups);" in text and text.count("attend_launches(p, ") == 1
    assert text.count("uint32_t id = a.first + blockIdx.x;") == 2
