"""The row operators without a GPU: refusals of the C ABI and of the binding, the plain forms' own check, barriers and registers of the
compiled kernels."""
import ctypes as C
import importlib.util
import pathlib
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2210_15748_amd as dz

import row_operators_plain as plain

HERE = pathlib.Path(__file__).resolve().parent
P = 4096            # an address that no refused call touches
ALL_OK = "index is NULL"


def refused(status, match):
    assert status == dz.EINVAL
    assert match in dz.last_error(), dz.last_error()


def quantize(x=P, dtype=dz.F16, rows=4, cols=8, stride=8, scaling=0, codes=P, scales=P):
    return dz.lib().dessert_quantize_rows(None, x, dtype, rows, cols, stride, scaling, codes, scales)


def matmul(a=P, lda=8, sa=P, m=4, b=P, ldb=8, sb=P, bias=None, n=4, k=8, dtype=dz.F16, out=P, ldo=4, ws=P, wsn=1 << 40):
    return dz.lib().dessert_scaled_matmul(None, a, lda, sa, m, b, ldb, sb, bias, n, k, dtype, out, ldo, ws, wsn)


def token(x=P, dtype=dz.F32, rows=4, V=100, stride=100, tokens=P, top=3, ws=P, wsn=1 << 40, lp=P, ent=P, ids=P, tlp=P):
    return dz.lib().dessert_token_logprobs(None, x, dtype, rows, V, stride, tokens, top, ws, wsn, lp, ent, ids, tlp)


def head(a=P, lda=8, sa=P, rows=4, b=P, ldb=8, sb=P, V=100, k=8, tokens=P, top=3, ws=P, wsn=1 << 40, lp=P, ent=P, ids=P, tlp=P):
    return dz.lib().dessert_head_logprobs(None, a, lda, sa, rows, b, ldb, sb, V, k, tokens, top, ws, wsn, lp, ent, ids, tlp)


def test_a_call_that_is_right_but_for_its_handle_is_refused_for_that():
    for call in (quantize, matmul, token, head):
        refused(call(), ALL_OK)
    refused(quantize(rows=0, x=None, codes=None, scales=None), ALL_OK)
    refused(matmul(m=0, a=None, sa=None, out=None), ALL_OK)
    refused(matmul(n=0, b=None, sb=None, out=None), ALL_OK)
    refused(token(rows=0, x=None, tokens=None, lp=None, ws=None), ALL_OK)
    refused(head(rows=0, a=None, sa=None, ws=None), ALL_OK)


def test_quantize_refusals():
    for dtype in (dz.I8, 4, 77):
        refused(quantize(dtype=dtype), "dtype must be")
    for scaling in (-1, 2):
        refused(quantize(scaling=scaling), "unknown scaling")
    refused(quantize(cols=0, stride=0), "n_cols")
    refused(quantize(cols=(1 << 30) + 1, stride=1 << 31), "n_cols")
    refused(quantize(stride=7), "stride")
    refused(quantize(stride=1 << 31), "stride")
    refused(quantize(rows=1 << 31), "rows")
    for name in ("x", "codes", "scales"):
        refused(quantize(**{name: None}), "NULL")
    refused(quantize(x=P + 1), "aligned")
    refused(quantize(x=P + 2, dtype=dz.F32), "aligned")
    refused(quantize(scales=P + 2), "aligned")
    refused(quantize(codes=P + 1), ALL_OK)          # codes go to any address


def test_matmul_refusals():
    for dtype in (dz.I8, 4):
        refused(matmul(dtype=dtype), "out_dtype")
    refused(matmul(k=0), "n_cols")
    refused(matmul(k=131072, lda=131072, ldb=131072), "n_cols")
    refused(matmul(k=131071, lda=131071, ldb=131071), ALL_OK)
    for name in ("a", "sa", "b", "sb", "out"):
        refused(matmul(**{name: None}), "NULL")
    refused(matmul(lda=7), "stride")
    refused(matmul(ldb=7), "stride")
    refused(matmul(lda=1 << 31), "stride")
    refused(matmul(ldo=3), "out_stride")
    refused(matmul(m=1 << 31), "rows")
    refused(matmul(n=1 << 31, ldo=1 << 31), "rows")
    refused(matmul(m=(1 << 31) - 1, n=(1 << 31) - 1, ldo=(1 << 31) - 1), "too large")
    refused(matmul(out=P + 1), "aligned")
    refused(matmul(sa=P + 2), "aligned")
    refused(matmul(bias=P + 2), "aligned")
    refused(matmul(a=P + 1, b=P + 3), ALL_OK)
    big = dict(m=64, n=64, k=8192, lda=8192, ldb=8192, ldo=64)
    refused(matmul(**big), ALL_OK)
    refused(matmul(**big, ws=None), "workspace_dev is NULL")
    refused(matmul(**big, ws=P + 64), "256-byte")
    refused(matmul(**big, wsn=1000), "workspace too small")
    refused(matmul(ws=None, wsn=0), ALL_OK)              # none needed


def test_logprob_refusals():
    for dtype in (dz.I8, 4):
        refused(token(dtype=dtype), "dtype must be")
    refused(token(x=None), "NULL")
    refused(token(x=P + 2), "aligned")
    refused(token(stride=99), "row_stride")
    refused(head(k=0), "n_cols")
    refused(head(a=None), "NULL")
    refused(head(sb=None), "NULL")
    refused(head(ldb=7), "stride")
    for call in (token, head):
        refused(call(V=0), "n_vocab")
        refused(call(rows=1 << 31), "rows")
        refused(call(top=65), "n_top")
        refused(call(tokens=None), "go together")
        refused(call(lp=None), "go together")
        refused(call(tokens=None, lp=None), ALL_OK)
        refused(call(ids=None), "NULL")
        refused(call(tlp=None), "NULL")
        refused(call(top=0, ids=None, tlp=None), ALL_OK)
        refused(call(ent=None), ALL_OK)
        refused(call(tokens=P + 1), "aligned")
    refused(token(rows=2, V=100000, stride=100000, ws=None), "workspace_dev is NULL")
    refused(token(rows=2, V=100000, stride=100000, ws=P + 128), "256-byte")
    refused(token(rows=2, V=100000, stride=100000, wsn=8), "workspace too small")
    refused(head(ws=None), "workspace_dev is NULL")
    refused(head(ws=P + 128), "256-byte")
    refused(head(wsn=100), "workspace too small")


def test_workspace_sizes_without_a_handle_are_zero():
    l = dz.lib()
    assert l.dessert_scaled_matmul_workspace_bytes(None, 4, 4, 4) == 0
    assert l.dessert_token_logprobs_workspace_bytes(None, 4, 4, 4) == 0
    assert l.dessert_head_logprobs_workspace_bytes(None, 4, 4, 4, 4) == 0


def cpu_index():
    """A handle-less index on the CPU: the binding's own checks pass or raise before the library sees the call."""
    return dz.Index(None, dz.Config(d=128, L=32, C=7), torch.device("cpu"))


def test_the_binding_refuses_shapes_types_and_devices():
    ix = cpu_index()
    i8, f = torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4)
    x = torch.zeros(4, 8)
    with pytest.raises(dz.DessertError, match=ALL_OK):
        dz.quantize_rows(ix, x, out=i8, out_scales=f)
    with pytest.raises(dz.DessertError, match=ALL_OK):
        dz.scaled_matmul(ix, i8, f, i8, f, out=torch.zeros(4, 6)[:, :4])
    for bad in (x[0], x.double(), x.to("meta")):
        with pytest.raises(ValueError, match="x must be"):
            dz.quantize_rows(ix, bad)
    with pytest.raises(ValueError, match="out must be"):
        dz.quantize_rows(ix, x, out=torch.zeros(4, 16, dtype=torch.int8)[:, :8])
    with pytest.raises(ValueError, match="out_scales must be"):
        dz.quantize_rows(ix, x, out_scales=torch.zeros(5))
    with pytest.raises(ValueError, match="columns"):
        dz.scaled_matmul(ix, i8, f, torch.zeros(4, 9, dtype=torch.int8), f)
    with pytest.raises(ValueError, match="a_scales"):
        dz.scaled_matmul(ix, i8, torch.zeros(3), i8, f)
    with pytest.raises(ValueError, match="b_scales"):
        dz.scaled_matmul(ix, i8, f, i8, f.double())
    with pytest.raises(ValueError, match="bias"):
        dz.scaled_matmul(ix, i8, f, i8, f, bias=torch.zeros(4, 1))
    with pytest.raises(ValueError, match="out_dtype"):
        dz.scaled_matmul(ix, i8, f, i8, f, out_dtype=torch.float64)
    for out in (torch.zeros(4, 5), torch.zeros(4, 4).t(), torch.zeros(1, 4).expand(4, 4)):
        with pytest.raises(ValueError, match="out must be"):
            dz.scaled_matmul(ix, i8, f, i8, f, out=out)
    with pytest.raises(ValueError, match="tokens"):
        dz.token_logprobs(ix, x, torch.zeros(4))
    with pytest.raises(ValueError, match="tokens"):
        dz.token_logprobs(ix, x, torch.zeros(5, dtype=torch.int32))
    with pytest.raises(ValueError, match="outs"):
        dz.token_logprobs(ix, x, None, 2, outs=(None, None, torch.zeros(4, 2, dtype=torch.int64), None))
    with pytest.raises(ValueError, match="columns"):
        dz.head_logprobs(ix, i8, f, torch.zeros(9, 7, dtype=torch.int8), torch.zeros(9))
    with pytest.raises(ValueError, match="vocab_scales"):
        dz.head_logprobs(ix, i8, f, torch.zeros(9, 8, dtype=torch.int8), torch.zeros(8))


def test_the_binding_keeps_what_it_converts_until_the_call(monkeypatch):
    """Copies that the binding makes (ids of 64 bits, columns that lie apart) are alive, and right, when the library is called."""
    seen = {}

    class Library:
        @staticmethod
        def dessert_head_logprobs(handle, a, a_apart, sa, n, b, b_apart, sb, V, k, tokens, *rest):
            junk = [torch.full((n,), 7, dtype=torch.int32) for _ in range(64)]        # what freed memory would be used for
            seen["tokens"] = list((C.c_int32 * n).from_address(tokens))
            seen["a"] = np.ctypeslib.as_array((C.c_int8 * (n * k)).from_address(a)).reshape(n, k).copy()
            seen["scales"] = list((C.c_float * n).from_address(sa))
            return len(junk) - 64

    monkeypatch.setattr(dz, "lib", lambda: Library)
    monkeypatch.setattr(dz, "_lend", lambda ix, made: seen.update(lent=len(made)))
    wide = torch.arange(600, dtype=torch.int32).to(torch.int8).view(100, 6)
    tokens = torch.arange(100) - 1
    tokens[5], tokens[6] = 1 << 40, -2
    dz.head_logprobs(cpu_index(), wide[:, ::2], torch.arange(200.0)[::2], torch.zeros(9, 3, dtype=torch.int8), torch.zeros(9), tokens, 2,
                     workspace=torch.zeros(256, dtype=torch.uint8))
    assert seen["tokens"] == [-1, 0, 1, 2, 3, 0x7FFFFFFF, 0x7FFFFFFF] + list(range(6, 99))
    assert np.array_equal(seen["a"], wide[:, ::2].numpy()) and seen["scales"] == list(range(0, 200, 2))
    assert seen["lent"] == 3 + 4                          # the copies and the outputs


def test_plain_forms_against_values_worked_out_by_hand():
    c, s = plain.quantize(torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -3.5]]), False)
    assert s[0] == 1.0 and c.tolist() == [[127, 0, 2, 2, 0, -4]]
    c, s = plain.quantize(torch.tensor([[253.0, 22, 4, 2, 1, -1, 1]]), True)       # norm 254
    assert s[0] == 2.0 and c.tolist() == [[126, 11, 2, 1, 0, 0, 0]]
    c, s = plain.quantize(torch.tensor([[0.0, 0.0], [1.0, float("inf")]]), False)
    assert s[0] == 0 and np.isnan(s[1]) and not c.any()
    lp, ent, ids, top, _, _ = plain.logprobs(torch.tensor([[0.0, 0.0, -np.inf], [1.0, 1.0, 1.0]]), np.array([1, -1]), 3)
    assert np.allclose(lp, [-np.log(2), 0]) and np.allclose(ent, [np.log(2), np.log(3)])
    assert ids.tolist() == [[0, 1, plain.NONE], [0, 1, 2]] and np.isneginf(top[0, 2])


@pytest.mark.parametrize("source", ["quantize_kernels", "matmul_kernels", "logprob_kernels"])
def test_no_barrier_of_the_row_operators_leaves_lds_operations_behind(source, tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("needs hipcc")
    spec = importlib.util.spec_from_file_location("host_barriers", HERE / "test_host_barriers.py")
    barriers = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(barriers)
    from paper_2210_15748_amd import build as hip_build
    obj = hip_build.OBJ / (source + ".o")
    if not obj.exists() or hip_build.stale():
        hip_build.build(force=True)
    kernels = barriers.kernels_of(barriers.disassembled(obj, tmp_path))
    assert kernels
    assert not {k: n for k, v in kernels.items() if (n := barriers.unwaited_barriers(v))}


@pytest.mark.parametrize("source", ["quantize_kernels", "matmul_kernels", "logprob_kernels"])
def test_the_row_operators_keep_nothing_in_scratch_memory(source, tmp_path):
    """What the compiler recorded per lane: accumulators and rows stay in registers (a second copy of a tile's accumulators would not)."""
    if shutil.which("hipcc") is None:
        pytest.skip("needs hipcc")
    from paper_2210_15748_amd import build as hip_build
    obj = hip_build.OBJ / (source + ".o")
    if not obj.exists() or hip_build.stale():
        hip_build.build(force=True)
    llvm = "/opt/rocm/llvm/bin"
    subprocess.run([f"{llvm}/llvm-objcopy", "--dump-section", f".hip_fatbin={tmp_path}/fatbin", str(obj), f"{tmp_path}/host.o"], check=True)
    subprocess.run([f"{llvm}/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                    f"--input={tmp_path}/fatbin", f"--output={tmp_path}/device.co"], check=True)
    notes = subprocess.run([f"{llvm}/llvm-readobj", "--notes", f"{tmp_path}/device.co"], check=True, capture_output=True, text=True).stdout
    scratch = {}
    for block in notes.split("- .agpr_count")[1:]:
        scratch[re.search(r"\.name:\s+(\S+)", block).group(1)] = int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", block).group(1))
    assert scratch and {k: v for k, v in scratch.items() if v} == {}
