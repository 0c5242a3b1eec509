"""Scratch memory of the row operators by sizes: the rules of csrc/row_plans.hpp, compiled for the host.  What a caller is told for a number of rows
serves every call of as many rows or fewer."""
import ctypes as C
import importlib.util
import pathlib
import random
import shutil
import subprocess

import pytest

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2210_15748_amd" / "csrc"
SOURCE = """
#include "row_plans.hpp"
using namespace dessert;
extern "C" {
size_t matmul_needs(uint64_t m, uint64_t n, uint32_t k, uint32_t) { return scaled_matmul_workspace(m, n, k); }
size_t matmul_told(uint64_t m, uint64_t n, uint32_t k, uint32_t) { return scaled_matmul_workspace_upto(m, n, k); }
size_t token_needs(uint64_t rows, uint64_t vocab, uint32_t, uint32_t n_top) { return logprob_plan(rows, (uint32_t)vocab, n_top).bytes; }
size_t token_told(uint64_t rows, uint64_t vocab, uint32_t, uint32_t n_top) { return logprob_workspace_upto(rows, (uint32_t)vocab, n_top); }
size_t head_needs(uint64_t rows, uint64_t vocab, uint32_t k, uint32_t n_top) {
    return std::max(head_plan(rows, (uint32_t)vocab, k, n_top).bytes, group_plan(rows, (uint32_t)vocab, k, n_top).bytes);
}
int by_groups(uint64_t rows, uint32_t vocab, uint32_t k, uint32_t n_top) { return groups_pay(rows, vocab, k, n_top); }
uint64_t group_turn(uint64_t rows, uint32_t vocab, uint32_t k, uint32_t n_top) { return group_plan(rows, vocab, k, n_top).rows; }
size_t head_told(uint64_t rows, uint64_t vocab, uint32_t k, uint32_t n_top) { return head_workspace_upto(rows, (uint32_t)vocab, k, n_top); }
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    d = tmp_path_factory.mktemp("plans")
    (d / "rule.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-O1", "-shared", "-fPIC", "-I", str(CSRC), str(d / "rule.cpp"), "-o", str(d / "rule.so")],
                   check=True)
    lib = C.CDLL(str(d / "rule.so"))
    for call in ("matmul", "token", "head"):
        for what in ("needs", "told"):
            f = getattr(lib, f"{call}_{what}")
            f.argtypes = [C.c_uint64, C.c_uint64, C.c_uint32, C.c_uint32]
            f.restype = C.c_size_t
    lib.by_groups.argtypes = lib.group_turn.argtypes = [C.c_uint64, C.c_uint32, C.c_uint32, C.c_uint32]
    lib.group_turn.restype = C.c_uint64
    return lib


ROWS = sorted({1, 2, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 512, 700, 1000, 1023, 1024, 1025, 1400, 2048, 4096, 8191, 33000,
               1 << 20, (1 << 31) - 1} | set(range(40, 2000, 97)))
SHAPES = {
    "matmul": [(n, k, 0) for n in (1, 64, 130, 1000, 4096, 8192, 50021) for k in (16, 77, 1029, 2047, 2048, 2304, 4096, 4099, 8192, 8193, 9000, 16384, 131071)],
    "token": [(V, 0, top) for V in (1, 2048, 2049, 9600, 32000, 50257, 128000, 1 << 20) for top in (0, 1, 10, 64)],
    "head": [(V, k, top) for V in (5, 600, 3000, 20000, 32000, 50021, 128000) for k in (16, 776, 2304, 4099, 8192) for top in (0, 5, 64)],
}


@pytest.mark.parametrize("call", SHAPES)
def test_memory_for_a_number_of_rows_serves_fewer(rule, call):
    needs, told = getattr(rule, call + "_needs"), getattr(rule, call + "_told")
    for n, k, top in SHAPES[call]:
        largest = last = 0
        for m in ROWS:
            largest = max(largest, needs(m, n, k, top))
            here = told(m, n, k, top)
            assert here >= largest, (call, m, n, k, top)
            assert here >= last, (call, m, n, k, top)
            last = here


@pytest.mark.parametrize("call", SHAPES)
def test_every_number_of_rows_of_some_sizes(rule, call):
    rng = random.Random(5)
    needs, told = getattr(rule, call + "_needs"), getattr(rule, call + "_told")
    for _ in range(40):
        n, k, top = int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(4, 16.9)) // 4 * 4 or 4, rng.randint(0, 64)
        k += rng.choice((0, 0, 1))
        largest = 0
        for m in range(1, 1300):
            largest = max(largest, needs(m, n, k, top))
            assert told(m, n, k, top) >= largest, (call, m, n, k, top)


def test_it_is_not_more_than_it_has_to_be(rule):
    """The largest need of any fewer rows, up to the rounding of a row's parts."""
    for call in ("matmul", "token"):
        needs, told = getattr(rule, call + "_needs"), getattr(rule, call + "_told")
        for n, k, top in SHAPES[call]:
            for m in (1, 8, 64, 300, 1100):
                largest = max(needs(i, n, k, top) for i in range(1, m + 1))
                assert told(m, n, k, top) <= 2 * largest + (1 << 17), (call, m, n, k, top)
    assert rule.matmul_told(0, 100, 9000, 0) == 0


# rows, vocabulary, columns, alternatives, us by logits, us by groups: calls on both sides (300 x 128000 x 1024 with 64, 155 / 168, is one that the rule misses)
@pytest.mark.parametrize("n,V,k,top,logits,groups", [
    (4096, 32000, 2048, 5, 423, 308), (4096, 32000, 2048, 10, 418, 354), (4096, 32000, 2048, 33, 434, 528), (4096, 32000, 2048, 64, 448, 764),
    (4096, 32000, 128, 20, 233, 183), (4096, 32000, 128, 64, 268, 383), (1024, 32000, 1024, 0, 77, 46), (1024, 32000, 1024, 10, 80, 76),
    (1024, 32000, 1024, 20, 87, 95), (300, 128000, 1024, 5, 130, 114), (16384, 4000, 512, 0, 131, 82),
    (16384, 4000, 512, 5, 139, 207), (128, 50000, 1024, 0, 38, 27), (128, 50000, 1024, 1, 41, 45), (4096, 4000, 1024, 5, 49, 78),
    (512, 4000, 2048, 0, 19, 34), (64, 32000, 1024, 0, 23, 25)])
def test_groups_where_they_were_measured_to_pay(rule, n, V, k, top, logits, groups):
    assert bool(rule.by_groups(n, V, k, top)) == (groups < logits)


def test_the_calls_that_are_tested_by_groups_go_that_way(rule):
    spec = importlib.util.spec_from_file_location("head_groups", pathlib.Path(__file__).resolve().parent / "test_gpu_head_groups.py")
    gpu = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(gpu)
    for shape in [*gpu.SHAPES, gpu.VALUES, gpu.TURNS, gpu.PARTS, gpu.GRAPH, *((*gpu.SWITCH, top) for top in (1, 8, 20))]:
        assert rule.by_groups(*shape), shape
    assert not rule.by_groups(*gpu.SWITCH, 64)
    assert rule.group_turn(*gpu.TURNS) == 46848 < gpu.TURNS[0]
