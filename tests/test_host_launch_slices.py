"""Calls with more workgroups than a launch may have go in several launches: the rule of csrc/launch_slices.hpp, compiled for the host."""
import ctypes
import pathlib
import re
import shutil
import subprocess

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2210_15748_amd" / "csrc"
SOURCE = """
#include "launch_slices.hpp"
extern "C" int slices(uint64_t n, uint64_t per, uint32_t threads, uint64_t* out, int room) {
    int at = 0;
    dessert::in_launches(n, per, threads, [&](uint64_t first, uint64_t count, uint32_t workgroups) {
        if (at < room) { out[3 * at] = first; out[3 * at + 1] = count; out[3 * at + 2] = workgroups; }
        ++at;
    });
    return at;
}
"""


@pytest.fixture(scope="module")
def slices(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    d = tmp_path_factory.mktemp("slices")
    (d / "rule.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-O1", "-shared", "-fPIC", "-I", str(CSRC), str(d / "rule.cpp"), "-o", str(d / "rule.so")],
                   check=True)
    lib = ctypes.CDLL(str(d / "rule.so"))
    lib.slices.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint32, ctypes.POINTER(ctypes.c_uint64), ctypes.c_int]

    def of(n, per, threads):
        out = (ctypes.c_uint64 * 3000)()
        return [tuple(out[3 * i:3 * i + 3]) for i in range(lib.slices(n, per, threads, out, 1000))]
    return of


# (items to a workgroup, threads): rows of int8 in their five shapes and the long ones, a row of logits, channels of few tokens
@pytest.mark.parametrize("per,threads", [(64, 256), (32, 256), (16, 256), (8, 256), (4, 256), (1, 256), (1, 1024), (128, 512), (64, 512), (16, 512)])
def test_slices_cover_every_item_once_and_fit_a_launch(slices, per, threads):
    edge = 0xFFFFFFFF // threads * per
    for n in (1, per, per + 1, edge - 1, edge, edge + 1, 2 * edge, 2 * edge + 7, (1 << 31) - 1):
        at = 0
        for first, count, workgroups in slices(n, per, threads):
            assert first == at and count > 0
            assert workgroups * threads < 1 << 32
            assert (workgroups - 1) * per < count <= workgroups * per
            at += count
        assert at == n
        assert len(slices(n, per, threads)) == -(-n // edge)
    assert slices(0, per, threads) == []


@pytest.mark.parametrize("source,kernels", [("quantize_kernels", {"quantize_rows_kernel", "quantize_long_rows_kernel"}),
                                            ("matmul_kernels", {"scaled_matmul_few_kernel"})])
def test_what_a_call_sizes_freely_is_launched_in_slices(source, kernels):
    """Every launch of these kernels takes its number of workgroups from a slice."""
    text = (CSRC / (source + ".hip")).read_text()
    launches = re.findall(r"(\w+)(?:<[^<>]*>)?<<<(\w+\([^()]*(?:\([^()]*\)[^()]*)*\))", text)
    seen = {name: grid for name, grid in launches if name in kernels}
    assert seen.keys() == kernels
    assert all(grid == "dim3(workgroups)" for name, grid in launches if name in kernels), launches
