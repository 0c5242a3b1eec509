"""The row operators on more rows or channels than one launch takes."""
import sys

import pytest
import torch

import paper_2210_15748_amd as dz

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ix():
    return dz.create(128, 32, 7, seed=3, device=torch.device(DEV))


@pytest.fixture(autouse=True)
def room():
    """The tensors here take up to 60 GB: none of it is kept from test to test."""
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


def around(*borders, n, reach=70):
    """Rows on both sides of the borders, the first and the last ones."""
    at = torch.cat([torch.arange(max(0, b - reach), min(n, b + reach)) for b in (0, *borders, n)])
    return torch.unique(at).to(DEV)


def test_quantize_a_column_of_more_numbers_than_a_launch_takes(ix):
    n = (1 << 30) + 37                                   # 64 rows a workgroup of 256
    say("quantize", n, 1)
    x = torch.empty(n, 1, dtype=torch.float16, device=DEV)
    for part in x.split(1 << 26):
        part.normal_()
    codes, scales = torch.full((n, 1), 55, dtype=torch.int8, device=DEV), torch.full((n,), -1.0, device=DEV)
    dz.quantize_rows(ix, x, out=codes, out_scales=scales)
    for v, c, s in zip(x.split(1 << 26), codes.split(1 << 26), scales.split(1 << 26)):
        v = v[:, 0].float()
        assert torch.equal(s, v.abs() * torch.tensor(1 / 127, dtype=torch.float32, device=DEV))
        assert torch.equal(c[:, 0], (127 * v.sign()).to(torch.int8))


def test_quantize_more_rows_of_a_workgroup_each_than_a_launch_takes(ix):
    n, cols = (1 << 24) + 3, 1025
    say("quantize", n, cols)
    x = torch.empty(n, cols, dtype=torch.bfloat16, device=DEV)
    for part in x.split(1 << 20):
        part.normal_()
    codes, scales = torch.empty(n, cols, dtype=torch.int8, device=DEV), torch.full((n,), -1.0, device=DEV)
    dz.quantize_rows(ix, x, out=codes, out_scales=scales)
    for v, s in zip(x.split(1 << 20), scales.split(1 << 20)):
        assert torch.equal(s, v.abs().amax(1).float() * torch.tensor(1 / 127, dtype=torch.float32, device=DEV))
    pick = around((1 << 24) - 1, n=n)
    few, few_scales = dz.quantize_rows(ix, x[pick].contiguous())
    assert torch.equal(codes[pick], few) and torch.equal(scales[pick], few_scales)
