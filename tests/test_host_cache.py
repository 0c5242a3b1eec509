"""The paged cache's calls without a GPU: refusals of the C ABI and of the binding, plans and host code under the sanitizers, barriers and
registers of the compiled kernels, the plain forms' own check."""
import ctypes as C
import importlib.util
import os
import pathlib
import re
import shutil
import subprocess

import pytest
import torch

import paper_2210_15748_amd as dz

import cache_plain as plain

HERE = pathlib.Path(__file__).resolve().parent
ROOT = HERE.parent
PKG = ROOT / "paper_2210_15748_amd"
SOURCES = ["attention_kernels", "cache_kernels", "cache_pages_kernels"]
P = 4096            # an address that no refused call touches
ALL_OK = "index is NULL"


def refused(status, match):
    assert status == dz.EINVAL
    assert match in dz.last_error(), dz.last_error()


def cache_struct(k=P, v=P, ks=P, vs=P, bounds=P, pages=20, heads=2, page=16, dim=64):
    return dz._CacheStruct(k, v, ks, vs, bounds, pages, heads, page, dim)


def batch_struct(tables=P, lengths=P, starts=P, seqs=3, width=5, tokens=7, most=4, length=80):
    return dz._BatchStruct(tables, lengths, starts, seqs, width, tokens, most, length)


def split(kw):
    c = {k[2:]: kw.pop(k) for k in list(kw) if k.startswith("c_")}
    b = {k[2:]: kw.pop(k) for k in list(kw) if k.startswith("b_")}
    return C.byref(cache_struct(**c)), C.byref(batch_struct(**b)), kw


def append(**kw):
    c, b, o = split(kw)
    a = dict(k=P, k_stride=128, v=P, v_stride=128, dtype=dz.F16) | o
    return dz.lib().dessert_cache_append(None, c, b, a["k"], a["k_stride"], a["v"], a["v_stride"], a["dtype"])


def attention(**kw):
    c, b, o = split(kw)
    a = dict(q=P, dtype=dz.F16, stride=256, heads=4, scale=0.1, window=0, pages=None, n=0, ws=None, wsn=0, out=P, lse=P) | o
    return dz.lib().dessert_cache_attention(None, c, b, a["q"], a["dtype"], a["stride"], a["heads"], a["scale"], a["window"], a["pages"], a["n"],
                                            a["ws"], a["wsn"], a["out"], a["lse"])


def select(**kw):
    c, b, o = split(kw)
    a = dict(q=P, scales=P, heads=4, n=3, first=1, last=1, ws=P, wsn=1 << 30, out=P) | o
    return dz.lib().dessert_cache_select(None, c, b, a["q"], a["scales"], a["heads"], a["n"], a["first"], a["last"], a["ws"], a["wsn"], a["out"])


def advance(layers=None, **kw):
    c, _, o = split(kw)
    a = dict(n_layers=1, refs=P, tables=P, width=5, lengths=P, seqs=3, parents=P, add=P, new=4, ws=P, wsn=1 << 30, t=8 * P, l=9 * P, s=P) | o
    return dz.lib().dessert_cache_advance(None, c if layers is None else layers, a["n_layers"], a["refs"], a["tables"], a["width"], a["lengths"], a["seqs"],
                                          a["parents"], a["add"], a["new"], a["ws"], a["wsn"], a["t"], a["l"], a["s"])


def compact(**kw):
    c, _, o = split(kw)
    a = dict(n_layers=1, refs=P, tables=P, width=5, lengths=P, seqs=3, ws=P, wsn=1 << 30, numbers=P, live=P) | o
    return dz.lib().dessert_cache_compact(None, c, a["n_layers"], a["refs"], a["tables"], a["width"], a["lengths"], a["seqs"], a["ws"], a["wsn"], a["numbers"],
                                          a["live"])


def test_a_call_that_is_right_but_for_its_handle_is_refused_for_that():
    for call in (append, attention, select, advance, compact):
        refused(call(), ALL_OK)
    for call in (append, attention, select):
        refused(call(b_seqs=0, b_tables=None, b_lengths=None), ALL_OK)
    refused(append(b_tokens=0, b_most=0, k=None, v=None), ALL_OK)
    refused(attention(b_tokens=0, q=None, out=None), ALL_OK)
    refused(attention(lse=None, pages=P, n=5), ALL_OK)
    refused(attention(b_starts=None, b_tokens=3, b_most=1), ALL_OK)
    refused(advance(new=0, parents=None, add=None, t=None, l=None), ALL_OK)
    refused(advance(new=3, parents=None), ALL_OK)
    refused(compact(seqs=0, tables=None, lengths=None), ALL_OK)


@pytest.mark.parametrize("call", [append, attention, select, advance, compact])
def test_refusals_of_caches_and_tables(call):
    for page in (0, 8, 24, 512):
        refused(call(c_page=page), "page_tokens")
    for dim in (0, 16, 48, 288):
        refused(call(c_dim=dim), "dim must")
    for heads in (0, 65536):
        refused(call(c_heads=heads), "n_heads")
    for pages in (0, 0x7FFFFF01):
        refused(call(c_pages=pages), "n_pages")
    for name in ("k", "v", "ks", "vs"):
        refused(call(**{"c_" + name: None}), "NULL")
    for name in ("k", "v", "bounds"):
        refused(call(**{"c_" + name: P + 8}), "16-byte")
    for name in ("ks", "vs"):
        refused(call(**{"c_" + name: P + 2}), "4-byte")
    pre = "" if call in (advance, compact) else "b_"
    for name in ("tables", "lengths"):
        refused(call(**{pre + name: None}), "NULL")
        refused(call(**{pre + name: P + 1}), "4-byte")
    for width in (0, 0x7FFFFF00 // 16 + 1):
        refused(call(**{pre + "width": width}), "table_pages")
    refused(call(**{pre + "seqs": 0x7FFFFF01}), "sequences")


@pytest.mark.parametrize("call", [append, attention, select])
def test_refusals_of_batches(call):
    refused(call(b_starts=P + 2), "starts_dev")
    refused(call(b_starts=None), "without starts_dev")
    refused(call(b_starts=None, b_tokens=3), "without starts_dev")
    refused(call(b_most=0), "max_tokens")
    refused(call(b_most=8), "max_tokens")
    refused(call(b_tokens=0x7FFFFF01), "tokens")
    refused(call(b_seqs=1 << 26, b_tokens=1 << 30, b_most=1 << 30), "too many")


def test_refusals_of_each_call():
    for dtype in (dz.I8, 4):
        refused(append(dtype=dtype), "dtype")
    for dtype in (dz.I8, dz.F32, 4):
        refused(attention(dtype=dtype), "dtype")
    for name in ("k", "v"):
        refused(append(**{name: None}), "NULL")
        refused(append(**{name: P + 1}), "aligned")
        refused(append(**{name: P + 2}, dtype=dz.F32), "aligned")
        for stride in (127, 1 << 31):
            refused(append(**{name + "_stride": stride}), "stride")
    for call in (attention, select):
        for heads in (0, 3, 1 << 21):
            refused(call(heads=heads), "n_q_heads")
    for name in ("q", "out"):
        refused(attention(**{name: None}), "NULL")
        refused(attention(**{name: P + 1}), "aligned")
    refused(attention(stride=255), "stride")
    refused(attention(lse=P + 2), "aligned")
    refused(attention(pages=P + 2, n=3), "aligned")
    refused(attention(pages=P), "go together")
    refused(attention(n=2), "go together")
    refused(attention(pages=P, n=0x7FFFFF00 // 16 + 1), "n_select")
    refused(attention(b_length=5000, b_width=400), "workspace_dev is NULL")
    refused(attention(b_length=5000, b_width=400, ws=P, wsn=256), "workspace too small")
    refused(attention(b_length=5000, b_width=400, ws=P + 4, wsn=1 << 30), "256-byte")
    refused(attention(b_length=5000, b_width=400, ws=P, wsn=1 << 30), ALL_OK)
    refused(select(c_bounds=None), "bounds")
    refused(attention(c_bounds=None), ALL_OK)
    refused(append(c_bounds=None), ALL_OK)
    for n, first, last in ((0, 0, 0), (3, 2, 2), (3, 0xFFFFFFFF, 4), (0x7FFFFF01, 0, 0)):
        refused(select(n=n, first=first, last=last), "n_select")
    for name in ("q", "scales", "out"):
        refused(select(**{name: None}), "NULL")
    for name in ("scales", "out"):
        refused(select(**{name: P + 2}), "4-byte")
    refused(select(ws=None), "workspace_dev is NULL")
    refused(select(wsn=0), "too small")
    for name in ("refs", "add", "t", "l", "s"):
        refused(advance(**{name: None}), "NULL")
        refused(advance(**{name: 64 * P + 2}), "4-byte")
    refused(advance(parents=P + 2), "4-byte")
    refused(advance(parents=None), "n_new = n_seqs")
    refused(advance(t=P), "apart")
    refused(advance(t=P - 4 * 4 * 5 + 4), "apart")
    refused(advance(l=P + 8), "apart")
    refused(advance(ws=None), "workspace_dev is NULL")
    refused(advance(wsn=100), "too small")
    refused(advance(new=1 << 28, width=100), "too many")
    for name in ("refs", "numbers", "live"):
        refused(compact(**{name: None}), "NULL")
        refused(compact(**{name: P + 2}), "4-byte")
    refused(compact(wsn=100), "too small")
    for call in (advance, compact):
        refused(call(n_layers=0), "layers")
        refused(call(n_layers=65536), "layers")
    for change in (dict(pages=21), dict(heads=3), dict(page=32), dict(dim=32)):
        layers = (dz._CacheStruct * 2)(cache_struct(), cache_struct(**change))
        refused(advance(layers=layers, n_layers=2), "same sizes")


def cpu_index():
    return dz.Index(None, dz.Config(stream=None), torch.device("cpu"))


def test_refusals_of_the_binding():
    ix = cpu_index()
    z = lambda *s: torch.zeros(*s, dtype=torch.int8)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    good = (z(5, 2, 16, 64), z(5, 2, 64, 16), torch.zeros(5, 2), torch.zeros(5, 2), z(5, 2, 2, 64))
    c = dz.cache(ix, *good)
    assert (c.n_pages, c.n_heads, c.page_tokens, c.dim) == (5, 2, 16, 64)
    for at, bad in ((0, z(5, 2, 16, 64).transpose(0, 1)), (0, good[0].int()), (1, z(5, 2, 16, 64)), (2, torch.zeros(5, 3)), (3, torch.zeros(5, 2).double()),
                    (4, z(5, 2, 64, 2))):
        with pytest.raises(ValueError, match="must be a contiguous"):
            dz.cache(ix, *good[:at], bad, *good[at + 1:])
    b = dz.cache_batch(ix, i(3, 4), i(3))
    assert b.n_tokens == 3
    with pytest.raises(ValueError, match="n_tokens is needed"):
        dz.cache_batch(ix, i(3, 4), i(3), i(4))
    for args in ((i(3, 4).long(), i(3)), (i(3, 4), i(4)), (i(4, 3).t(), i(3)), (i(3, 4), i(3), i(3))):
        with pytest.raises(ValueError, match="must be a contiguous"):
            dz.cache_batch(ix, *args, n_tokens=3)
    with pytest.raises(ValueError, match="n_tokens"):
        dz.cache_batch(ix, i(3, 4), i(3), i(4), n_tokens=-1)
    h = lambda *s: torch.zeros(*s, dtype=torch.float16)  # noqa: E731
    for k, v, match in ((h(3, 2, 64), h(3, 2, 32), "v must"), (h(2, 2, 64), h(3, 2, 64), "k must"), (h(3, 2, 64), torch.zeros(3, 2, 64), "one dtype"),
                        (h(3, 4, 64), h(3, 2, 64), "k must")):
        with pytest.raises(ValueError, match=match):
            dz.cache_append(ix, c, b, k, v)
    for q, kw, match in ((torch.zeros(3, 4, 64), {}, "q must"), (h(3, 4, 32), {}, "q must"), (h(3, 4, 64), dict(pages=i(3, 2, 0)), "no places"),
                         (h(3, 4, 64), dict(pages=i(3, 4, 2)), "pages must"), (h(3, 4, 64), dict(out=h(3, 64, 4)), "out must"),
                         (h(3, 4, 64), dict(out_lse=h(3, 4)), "out_lse must"), (h(3, 4, 64), dict(workspace=torch.zeros(8, 2).t()), "workspace"),
                         (h(3, 4, 64), dict(window=-1, workspace=torch.zeros(8)), "window")):
        with pytest.raises(ValueError, match=match):
            dz.cache_attention(ix, c, b, q, **kw)
    with pytest.raises(ValueError, match="rows for 3 tokens"):
        dz.cache_select(ix, c, b, z(4, 64), torch.zeros(4), 2)
    with pytest.raises(ValueError, match="q_scales"):
        dz.cache_select(ix, c, b, z(6, 64), torch.zeros(5), 2)
    with pytest.raises(ValueError, match="no layers"):
        dz.cache_advance(ix, [], i(5), i(3, 4), i(3), i(3))
    for args, kw, match in (((i(4), i(3, 4), i(3), i(3)), {}, "refs"), ((i(5), i(3, 4), i(2), i(3)), {}, "lengths"), ((i(5), i(3), i(3), i(3)), {}, "tables"),
                            ((i(5), i(3, 4), i(3), i(3)), dict(parents=i(2)), "parents"), ((i(5), i(3, 4), i(3), i(3)), dict(outs=(i(3, 5), None, None)), "outs")):
        with pytest.raises(ValueError, match=match):
            dz.cache_advance(ix, c, *args, **kw)
    with pytest.raises(ValueError, match="outs"):
        dz.cache_compact(ix, c, i(5), i(3, 4), i(3), outs=(i(4), None))


def test_plain_forms_against_values_worked_out_by_hand():
    c = dict(k=torch.zeros(2, 1, 16, 32, dtype=torch.int8), v=torch.zeros(2, 1, 32, 16, dtype=torch.int8), ks=torch.ones(2, 1), vs=torch.ones(2, 1),
             bounds=torch.zeros(2, 1, 2, 32, dtype=torch.int8))
    tables = torch.tensor([[1]], dtype=torch.int32)
    x = torch.zeros(2, 1, 32)
    x[0, 0, 0], x[1, 0, 0], x[1, 0, 1] = 127.0, -63.5, 2.5
    plain.append(c, tables, [2], [2], x, x)
    assert c["k"][1, 0, :2, :2].tolist() == [[127, 0], [-64, 2]] and c["bounds"][1, 0, :, :2].tolist() == [[-64, 0], [127, 2]]
    plain.append(c, tables, [3], [1], x[:1] * 2, x[:1] * 2)
    assert float(c["ks"][1]) == 2.0 and c["k"][1, 0, :3, 0].tolist() == [64, -32, 127] and c["v"][1, 0, 0, :3].tolist() == [64, -32, 127]
    q = torch.zeros(1, 1, 32)
    out, lse, _, _ = plain.attend(c, tables, [3], [1], q, 1.0)
    assert abs(float(out[0, 0, 0]) - 2 * (64 - 32 + 127) / 3) < 1e-12 and abs(float(lse) - 1.0986122886681098) < 1e-12
    assert plain.attend(c, tables, [3], [1], q, 1.0, window=1)[0][0, 0, 0] == 254
    chosen = plain.select(c, torch.tensor([[1, 0]], dtype=torch.int32), [20], [1], torch.ones(1, 32, dtype=torch.int8), torch.ones(1), 1, 0, 0)
    assert chosen.tolist() == [[[0]]]


def tool(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300, **kw)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    return r.stdout


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plans(tmp_path):
    tool(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
          "-I", str(PKG / "csrc"), str(HERE / "sanitize" / "cache_plans_driver.cpp"), "-o", str(tmp_path / "plans")])
    assert "cache plans sanitizer run: ok" in tool([str(tmp_path / "plans")], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_entry_points_under_the_sanitizers(tmp_path):
    from paper_2210_15748_amd import build as hip_build
    objs = [hip_build.OBJ / (s.rsplit(".", 1)[0] + ".o") for s in hip_build.SOURCES if s != "api.hip"]
    if not all(o.exists() for o in objs):
        hip_build.build(force=True)
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
    tool(["hipcc", *hip_build.FLAGS, *san, "-g", "-fno-omit-frame-pointer", "-c", str(PKG / "csrc" / "api.hip"), "-o", str(tmp_path / "api.o")])
    tool(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *san, "-shared-libsan", str(tmp_path / "api.o"), *map(str, objs),
          "-o", str(tmp_path / "libdessert_hip_san.so")])
    tool(["hipcc", "-x", "c", str(HERE / "sanitize" / "cache_driver.c"), "-x", "none", *san, "-shared-libsan", "-g", "-L", str(tmp_path),
          "-ldessert_hip_san", "-Wl,-rpath," + str(tmp_path), "-o", str(tmp_path / "driver")])
    rt = subprocess.run(["hipcc", "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True).stdout.strip()
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    if rt and os.path.exists(rt):
        env["LD_LIBRARY_PATH"] = os.path.dirname(rt) + ":" + env.get("LD_LIBRARY_PATH", "")
    assert "paged cache host sanitizer run: ok" in tool([str(tmp_path / "driver")], env=env)


@pytest.fixture(scope="module")
def barriers():
    spec = importlib.util.spec_from_file_location("host_barriers", HERE / "test_host_barriers.py")
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source", SOURCES)
def test_no_barrier_leaves_lds_operations_behind(source, tmp_path, barriers):
    from paper_2210_15748_amd import build as hip_build
    obj = hip_build.OBJ / (source + ".o")
    if not obj.exists() or hip_build.stale():
        hip_build.build(force=True)
    # (ds_bpermute moves registers between lanes and touches no LDS memory)
    kernels = {k: [(at, "s_nop 0" if text.startswith("ds_bpermute") else text, to) for at, text, to in v]
               for k, v in barriers.kernels_of(barriers.disassembled(obj, tmp_path)).items()}
    assert kernels
    assert not {k: n for k, v in kernels.items() if (n := barriers.unwaited_barriers(v))}


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source", SOURCES)
def test_what_goes_to_scratch_memory(source, tmp_path):
    """Nothing but a few registers of the form for many rows at 160 and 192 channels, whose eight waves pay all the same."""
    from paper_2210_15748_amd import build as hip_build
    obj = hip_build.OBJ / (source + ".o")
    if not obj.exists() or hip_build.stale():
        hip_build.build(force=True)
    llvm = "/opt/rocm/llvm/bin"
    tool([f"{llvm}/llvm-objcopy", "--dump-section", f".hip_fatbin={tmp_path}/fatbin", str(obj), f"{tmp_path}/host.o"])
    tool([f"{llvm}/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={tmp_path}/fatbin",
          f"--output={tmp_path}/device.co"])
    most = {}
    for block in tool([f"{llvm}/llvm-readobj", "--notes", f"{tmp_path}/device.co"]).split("- .agpr_count")[1:]:
        name = re.search(r"\.name:\s+(\S+)", block).group(1)
        most[name] = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", block).group(1))
    assert most
    allowed = lambda k: 256 if re.search(r"attend_many_kernelILi[56]ELi8E", k) else 32  # noqa: E731
    assert {k: v for k, v in most.items() if v > allowed(k)} == {}
