"""The row operators' host code under AddressSanitizer and UndefinedBehaviorSanitizer: the C entry points' checks and plans, in a library whose
api.hip has the sanitizers on its host pass only, and the plans themselves over sizes up to the largest."""
import os
import pathlib
import shutil
import subprocess

import pytest

ROOT = pathlib.Path(__file__).resolve().parent.parent
PKG = ROOT / "paper_2210_15748_amd"
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]


def ran(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300, **kw)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    return r.stdout


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_entry_points(tmp_path):
    from paper_2210_15748_amd import build as hip_build
    objs = [hip_build.OBJ / (s.rsplit(".", 1)[0] + ".o") for s in hip_build.SOURCES if s != "api.hip"]
    if not all(o.exists() for o in objs):
        hip_build.build(force=True)
    ran(["hipcc", *hip_build.FLAGS, *SAN, "-g", "-fno-omit-frame-pointer", "-c", str(PKG / "csrc" / "api.hip"), "-o", str(tmp_path / "api.o")])
    ran(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *SAN, "-shared-libsan", str(tmp_path / "api.o"), *map(str, objs),
         "-o", str(tmp_path / "libdessert_hip_san.so")])
    ran(["hipcc", "-x", "c", str(ROOT / "tests" / "sanitize" / "row_operators_driver.c"), "-x", "none", *SAN, "-shared-libsan", "-g", "-L", str(tmp_path),
         "-ldessert_hip_san", "-Wl,-rpath," + str(tmp_path), "-o", str(tmp_path / "driver")])
    rt = subprocess.run(["hipcc", "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True).stdout.strip()
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    if rt and os.path.exists(rt):
        env["LD_LIBRARY_PATH"] = os.path.dirname(rt) + ":" + env.get("LD_LIBRARY_PATH", "")
    assert "row operators host sanitizer run: ok" in ran([str(tmp_path / "driver")], env=env)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plans(tmp_path):
    ran(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
         "-I", str(PKG / "csrc"), str(ROOT / "tests" / "sanitize" / "row_plans_driver.cpp"), "-o", str(tmp_path / "plans")])
    assert "row plans sanitizer run: ok" in ran([str(tmp_path / "plans")], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
