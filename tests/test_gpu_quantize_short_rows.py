"""Many short rows to int8: the kernels in which a group of lanes has several rows, each lane one row's root and quotients."""
import sys

import numpy as np
import pytest
import torch

import paper_2210_15748_amd as dz

import row_operators_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ix():
    return dz.create(128, 32, 7, seed=3, device=torch.device(DEV))


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


def rows_of(n, cols, dtype, seed):
    """Ordinary rows, and in every group of neighbours others: zeros, -0, infinities, NaN, the smallest numbers, the largest, ties."""
    g = torch.Generator()
    g.manual_seed(seed)
    x = torch.randn(n, cols, generator=g) * torch.exp(torch.randn(n, 1, generator=g))
    info = torch.finfo(dtype)
    at = torch.randint(0, cols, (n,), generator=g)
    for i, (step, first) in enumerate([(29, 3), (31, 5), (37, 7), (41, 11), (43, 13), (47, 17), (53, 19), (59, 23)]):
        r = torch.arange(first, n, step)
        if i < 2:
            x[r] = (0.0, -0.0)[i]
        elif i < 5:
            x[r, at[r]] = (float("inf"), float("-inf"), float("nan"))[i - 2]
        elif i == 5:
            x[r] = info.tiny * info.eps * torch.randint(-3, 4, (len(r), cols), generator=g)
        elif i == 6:
            x[r] = info.max * torch.sign(x[r])
        else:   # halves of the scale: ties where the largest magnitude is 127 (cols > 1), 254 in norm elsewhere
            x[r] = torch.randint(-40, 41, (len(r), cols), generator=g) / 2
            x[r, at[r]] = 127.0
    x[-1] = float("nan")                                 # behind the last whole group of rows
    x[-2, 0] = 1.0
    return x.to(dtype)


@pytest.mark.parametrize("unit", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [1, 7, 127, 128, 129, 512])
def test_short_rows_by_several_to_a_group_of_lanes(ix, cols, dtype, unit):
    # rows behind the last whole workgroup (64, 32, 16 or 8 rows) and behind the last whole run of a group of lanes (4 or 2)
    for n, pad, at in [(65536 + 37, 3, 1), (65536 + 9, 8, 0)] if cols < 512 else [(65536 + 3, 1, 1)]:
        say("short rows", n, cols, dtype, unit, pad, at)
        x = rows_of(n, cols, dtype, cols)
        buf = torch.full((at + n * (cols + pad),), float("nan"), dtype=dtype, device=DEV)
        view = buf[at:].view(n, cols + pad)[:, :cols]
        view.copy_(x)
        codes, scales = torch.full((n + 2, cols), 55, dtype=torch.int8, device=DEV), torch.full((n + 2,), 7.0, device=DEV)
        dz.quantize_rows(ix, view, dz.SCALE_UNIT if unit else dz.SCALE_MAXABS, out=codes[1:-1], out_scales=scales[1:-1])
        assert (codes[0] == 55).all() and (codes[-1] == 55).all() and scales[0] == 7 and scales[-1] == 7
        want, want_s = plain.quantize(x, unit)
        assert np.array_equal(codes[1:-1].cpu().numpy(), want)
        if unit:   # the 64-bit norm / 127, rounded once
            plain.close(scales[1:-1].cpu().numpy(), want_s, 1.001 * plain.U32 * np.nan_to_num(np.abs(want_s)) + 2.0 ** -149)
        else:
            assert np.array_equal(scales[1:-1].cpu().numpy(), want_s.astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("unit", [False, True])
@pytest.mark.parametrize("cols", [5, 300])
def test_short_rows_are_the_same_bits_however_many_there_are(ix, cols, unit):
    """Several rows to a group of lanes from 65536 rows on, one below."""
    x = rows_of(65536 + 5, cols, torch.float16, 1).to(DEV)
    scaling = dz.SCALE_UNIT if unit else dz.SCALE_MAXABS
    codes, scales = dz.quantize_rows(ix, x, scaling)
    for lo in (0, 30000):
        c, s = dz.quantize_rows(ix, x[lo:lo + 35541], scaling)
        assert torch.equal(c, codes[lo:lo + 35541]) and torch.equal(s.view(torch.int32), scales[lo:lo + 35541].view(torch.int32))


def test_scales_that_underflow(ix):
    """The smallest 32-bit numbers: by the largest magnitude there is no scale to divide by; to unit norm the direction is there all the same."""
    x = torch.zeros(3, 4)
    x[0, 1], x[1, 1] = 2.0 ** -149, -63 * 2.0 ** -149               # 63 / 127 of the smallest number is below half of it
    x[2] = torch.tensor([3.0, 0.0, -4.0, 0.0]) * 2.0 ** -147        # norm 5 * 2^-147
    codes, scales = dz.quantize_rows(ix, x.to(DEV))
    assert not codes[:2].any() and not scales.any()
    codes, scales = dz.quantize_rows(ix, x.to(DEV), dz.SCALE_UNIT)
    assert codes.tolist() == [[0, 127, 0, 0], [0, -127, 0, 0], [76, 0, -102, 0]] and not scales.any()
