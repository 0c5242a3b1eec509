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


@pytest.mark.parametrize("with_tokens", [True, False])
def test_logprobs_of_more_rows_than_a_launch_takes(ix, with_tokens):
    """Pairs of logits: p and 1 - p by the logistic function; every 11th row has one entry."""
    n = (1 << 24) + 5
    say("logprobs", n, 2, with_tokens)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = 3 * torch.randn(n, 2, generator=g, device=DEV)
    x[::11, 1] = -float("inf")
    tokens = torch.randint(0, 2, (n,), generator=g, device=DEV, dtype=torch.int32)
    tokens[::7] = -1
    outs = (torch.full((n,), 5.0, device=DEV), torch.full((n,), 5.0, device=DEV), torch.zeros(n, 1, dtype=torch.int32, device=DEV).view(torch.uint32),
            torch.full((n, 1), 5.0, device=DEV))
    lp, entropy, ids, top = dz.token_logprobs(ix, x, tokens if with_tokens else None, 1, outs=outs)
    l = torch.log_softmax(x.double(), 1)
    p = l.exp()
    # 32-bit steps: |l - m| <= 26 (6 standard deviations of 4.25) rounds twice, as a difference and with the logarithm; the sum of at most 2 is
    # off by at most (3 |d| + 4) e^d, below 6, and its logarithm by 1 more
    tol = 64 * 2.0 ** -24
    want = l.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0]
    want[tokens == -1] = 0.0
    if with_tokens:
        masked = want.isinf()
        assert torch.equal(lp.isinf(), masked) and (lp[~masked].double() - want[~masked]).abs().max() <= tol
    else:
        assert lp is None
    assert (entropy.double() + torch.special.xlogy(p, p).sum(1)).abs().max() <= tol
    assert torch.equal(ids.view(torch.int32)[:, 0], (x[:, 1] > x[:, 0]).to(torch.int32))
    assert (top[:, 0].double() - l.amax(1)).abs().max() <= tol


@pytest.mark.parametrize("at", [0, 1])
def test_matmul_of_a_token_with_more_channels_than_a_launch_takes(ix, at):
    """at: rows at whole 16 bytes, or anywhere."""
    n, k = (1 << 30) + 100, 16                           # 128 channels a workgroup of 512
    say("matmul", 1, n, k, at)
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    a = torch.randint(-128, 128, (1, k), generator=g, device=DEV, dtype=torch.int8)
    b = torch.empty(n * k + at, dtype=torch.int8, device=DEV)[at:].view(n, k)
    for part in b.split(1 << 26):
        part.random_(-128, 128, generator=g)
    sb = torch.rand(n, generator=g, device=DEV) + 0.5
    bias = torch.rand(n, generator=g, device=DEV)
    sa = torch.tensor([0.01], device=DEV)
    out = torch.full((1, n), 5.0, dtype=torch.float16, device=DEV)
    dz.scaled_matmul(ix, a, sa, b, sb, bias, out=out)
    step = 1 << 23
    for lo in range(0, n, step):
        hi = min(n, lo + step)
        p = (b[lo:hi].float() * a.float()).sum(1).double() * sa.double() * sb[lo:hi].double()     # whole numbers below 2^24: exact sums
        want = p + bias[lo:hi].double()
        tol = 3.01 * 2.0 ** -24 * p.abs() + (1.01 * 2.0 ** -24 + 1.01 * 2.0 ** -11) * want.abs() + 2.0 ** -25
        assert ((out[0, lo:hi].double() - want).abs() <= tol).all()
