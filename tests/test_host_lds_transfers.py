"""Transfers from memory to LDS are waited for before a barrier, behind which other waves read them, and before a wave ends.  The product's
tiles are read by all waves of a workgroup; each wave has to know its own transfers landed when it comes to the barrier.  The built objects
are disassembled and the transfers that may be under way followed through each kernel's flow.  (The hashing and filter kernels fetch a next
step only where there is one, which the flow of their instructions does not show; their waits are instructions of their source.)"""
import importlib.util
import pathlib
import re
import shutil

import pytest

HERE = pathlib.Path(__file__).resolve().parent
CSRC = HERE.parent / "paper_2210_15748_amd" / "csrc"
spec = importlib.util.spec_from_file_location("host_barriers", HERE / "test_host_barriers.py")
barriers = importlib.util.module_from_spec(spec)
spec.loader.exec_module(barriers)

LOAD = re.compile(r"(buffer|global|flat|scratch)_load")
TRANSFER = re.compile(r"(buffer_load_\S+ .*\blds$|buffer_load_\S+ .*\blds |global_load_lds_)")


def walk(state, instructions, found=None):
    """state: loads issued since the last transfer that may be under way, or None.  Loads end in order; stores are not counted, as they may end
    before a load that was issued first."""
    for text in instructions:
        if text.startswith("s_waitcnt"):
            m = re.search(r"vmcnt\((\d+)\)", text)
            if m and state is not None and state >= int(m.group(1)):
                state = None
        elif TRANSFER.match(text):
            state = 0
        elif state is not None and LOAD.match(text):
            state += 1
        elif text.startswith(("s_barrier", "s_endpgm")) and found is not None and state is not None:
            found.append(text)
    return state


def unwaited_transfers(listing):
    blocks = barriers.blocks_of(listing)
    entry = [("unseen",)] * len(blocks)
    entry[0], work = None, [0]
    while work:
        b = work.pop()
        end = walk(entry[b], blocks[b][0])
        for s in blocks[b][1]:
            joined = end if entry[s] == ("unseen",) else min((x for x in (entry[s], end) if x is not None), default=None)
            if joined != entry[s]:
                entry[s] = joined
                work.append(s)
    found = []
    for b, (instructions, _) in enumerate(blocks):
        if entry[b] != ("unseen",):
            walk(entry[b], instructions, found)
    return len(found)


def test_the_check_itself():
    transfer = "buffer_load_dwordx4 v1, s[0:3], s8 offen lds"
    loop = [(0, transfer, None), (4, "s_waitcnt vmcnt(0)", None), (8, "s_barrier", None), (12, transfer, None),
            (16, "v_mfma_i32_16x16x64_i8 a[0:3], v[0:3], v[4:7], a[0:3]", None), (20, "s_cbranch_scc1 65530", 4),
            (24, "s_waitcnt vmcnt(0)", None), (28, "s_endpgm", None)]
    assert unwaited_transfers(loop) == 0
    assert unwaited_transfers([x for x in loop if x[0] != 24]) == 1                   # the last ones still under way at the end
    late = [(a, t, 8 if g is not None else None) for a, t, g in loop]                 # back to the barrier, behind the wait
    assert unwaited_transfers(late) == 1
    assert unwaited_transfers([x if x[0] != 4 else (4, "s_waitcnt lgkmcnt(0)", None) for x in loop]) == 1
    # a load behind the transfer lets the wait leave one under way; a store does not
    between = loop[:1] + [(1, "global_load_dword v9, v[2:3], off", None), (4, "s_waitcnt vmcnt(1)", None)] + loop[2:3] + loop[6:]
    assert unwaited_transfers(between) == 0
    assert unwaited_transfers([x if x[0] != 1 else (1, "global_store_dword v[2:3], v9, off", None) for x in between]) == 1
    assert unwaited_transfers([(0, "global_load_lds_dwordx4 v[2:3], off", None), (4, "s_barrier", None), (8, "s_endpgm", None)]) == 2


@pytest.mark.parametrize("source", ["matmul_kernels"])
def test_transfers_to_lds_have_landed_at_barriers_and_at_the_end(source, tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("needs hipcc")
    from paper_2210_15748_amd import build as hip_build
    obj = hip_build.OBJ / (source + ".o")
    if not obj.exists() or hip_build.stale():
        hip_build.build(force=True)
    kernels = {k: v for k, v in barriers.kernels_of(barriers.disassembled(obj, tmp_path)).items() if any(TRANSFER.match(t) for _, t, _ in v)}
    assert kernels
    assert not {k: n for k, v in kernels.items() if (n := unwaited_transfers(v))}


def test_the_tiles_wait_is_written_out():
    """The wait before the barrier that publishes a step stands in the source; it is not left to what the compiler puts there."""
    text = (CSRC / "matmul_kernels.hip").read_text()
    body = text[text.index("void scaled_matmul_kernel("):text.index("// ---- few tokens")]
    loop = body[body.index("for (;;)"):]
    assert loop.count("__syncthreads();") == 2
    assert len(re.findall(r"src\.arrived\(\);\s+__syncthreads\(\);", loop)) == 2
