"""The row operators on the GPU (int8 rows with scales, scaled int8 products, log probabilities from logits and from int8 states) against
their 64-bit forms, at the sizes, strides, masks and values where they can go wrong, and together with the search."""
import sys

import numpy as np
import pytest
import torch

import paper_2210_15748_amd as dz

import row_operators_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FLOATS = [torch.float16, torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def ix():
    return dz.create(128, 32, 7, seed=3, device=torch.device(DEV))


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def apart(t, pad, at=0):
    """The same rows on the GPU, `pad` elements apart, the first one `at` elements into its buffer; what is between them is loud."""
    rows, cols = t.shape
    fill = 101 if t.dtype == torch.int8 else float("nan")
    buf = torch.full((at + rows * (cols + pad),), fill, dtype=t.dtype, device=DEV)
    view = buf[at:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


# ---- int8 rows ------------------------------------------------------------------------------------------------------------
def check_quantize(ix, x, unit, pad=0, at=0):
    codes, scales = dz.quantize_rows(ix, apart(x, pad, at), dz.SCALE_UNIT if unit else dz.SCALE_MAXABS)
    want, want_s = plain.quantize(x, unit)
    assert np.array_equal(codes.cpu().numpy(), want)
    if unit:   # the 64-bit norm / 127, rounded once
        plain.close(scales.cpu().numpy(), want_s, 1.001 * plain.U32 * np.nan_to_num(np.abs(want_s)) + 2.0 ** -149)
    else:
        assert np.array_equal(scales.cpu().numpy(), want_s.astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("unit", [False, True])
@pytest.mark.parametrize("dtype", FLOATS)
def test_quantize_sizes(ix, dtype, unit):
    g = gen(1)
    for rows, cols in [(1, 1), (1, 2), (3, 7), (17, 8), (5, 63), (33, 127), (16, 128), (15, 129), (9, 500), (4, 1023), (6, 1024), (3, 1025), (2, 2047),
                       (3, 4096), (2, 8192), (2, 8200), (3, 16384), (2, 16385), (1, 40000)]:
        x = (torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(dtype)
        for pad, at in [(0, 0), (1, 0), (8, 3)]:
            say("quantize", dtype, unit, rows, cols, pad, at)
            check_quantize(ix, x, unit, pad, at)


@pytest.mark.parametrize("dtype", FLOATS)
def test_quantize_ties_zeros_and_numbers_that_are_not_finite(ix, dtype):
    x = torch.zeros(9, 40)
    x[0, :7] = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -3.5, 126.5])              # scale 1: ties to even
    x[1, :7] = torch.tensor([253.0, 22, 4, 2, 1, -1, 1]) if dtype != torch.bfloat16 else torch.tensor([6.0, 0, 0, 0, 0, 0, 8])
    x[3, 5] = float("inf")
    x[4, 39] = float("nan")
    x[5, 0], x[5, 1] = float("-inf"), 1.0
    x[6, 2] = torch.finfo(dtype).tiny * torch.finfo(dtype).eps                      # the smallest number there is
    x[7] = torch.finfo(dtype).max
    x[8] = -0.0
    for unit in (False, True):
        say("quantize values", dtype, unit)
        check_quantize(ix, x.to(dtype), unit)
    codes, scales = dz.quantize_rows(ix, x.to(dtype).to(DEV), dz.SCALE_UNIT)
    assert torch.isnan(scales[3:6]).all() and not codes[3:6].any()


def test_quantize_takes_rows_behind_each_other_without_writing_between(ix):
    x = torch.randn(50, 37, generator=gen(2)).to(DEV)
    codes = torch.full((52, 37), 55, dtype=torch.int8, device=DEV)
    scales = torch.full((52,), 7.0, device=DEV)
    dz.quantize_rows(ix, x, out=codes[1:51], out_scales=scales[1:51])
    assert (codes[0] == 55).all() and (codes[51] == 55).all() and scales[0] == 7 and scales[51] == 7
    assert np.array_equal(codes[1:51].cpu().numpy(), plain.quantize(x.cpu(), False)[0])
    e, s = dz.quantize_rows(ix, x[:0])
    assert e.shape == (0, 37) and s.shape == (0,)


# ---- scaled int8 products -------------------------------------------------------------------------------------------------
def product_inputs(m, n, k, seed, extreme=False):
    g = gen(seed)
    if extreme:
        a, b = torch.full((m, k), -128, dtype=torch.int8), torch.full((n, k), -128, dtype=torch.int8)
    else:
        a = torch.randint(-128, 128, (m, k), generator=g, dtype=torch.int8)
        b = torch.randint(-128, 128, (n, k), generator=g, dtype=torch.int8)
    return a, torch.rand(m, generator=g) * 0.01 + 1e-4, b, torch.rand(n, generator=g) * 0.01 + 1e-4, torch.randn(n, generator=g)


def check_matmul(ix, m, n, k, out_dtype, bias, pads=(0, 0, 0), at=0, seed=0, extreme=False):
    say("matmul", m, n, k, out_dtype, bias, pads, at)
    a, sa, b, sb, c = product_inputs(m, n, k, seed, extreme)
    buf = torch.full((m, n + pads[2]), 55.0, dtype=out_dtype, device=DEV)
    out = buf[:, :n]
    got = dz.scaled_matmul(ix, apart(a, pads[0], at), sa.to(DEV), apart(b, pads[1], at), sb.to(DEV), c.to(DEV) if bias else None, out=out)
    assert got is out
    assert (buf[:, n:] == 55).all()
    want, tol = plain.matmul(a, sa, b, sb, c if bias else None, out_dtype)
    plain.close(out.cpu().double().numpy(), want.numpy(), tol.numpy())


SIZES = [(1, 1, 1), (1, 16, 64), (2, 15, 63), (3, 17, 65), (16, 64, 128), (17, 65, 129), (15, 130, 127), (1, 200, 1024), (5, 1000, 272), (33, 100, 640),
         (63, 257, 144), (64, 64, 2048), (65, 70, 256), (127, 129, 112), (128, 128, 128), (129, 127, 384), (200, 260, 528), (255, 513, 192),
         (256, 256, 256), (257, 255, 1040), (300, 1, 320), (1, 1, 70000), (700, 40, 96), (513, 770, 160), (64, 130, 4096), (33, 1000, 4112), (100, 66, 8192),
         (200, 500, 5008), (18, 100, 3000), (65, 64, 20000), (31, 70, 9216), (16, 64, 4099), (2, 600, 5001), (1, 300, 8197),
         (100, 250, 2047), (100, 250, 2051), (3000, 4100, 196), (1700, 1900, 332), (130, 70, 4), (40, 100, 12), (1, 5, 20), (30, 4000, 1028)]


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_matmul_sizes(ix, size):
    for i, out_dtype in enumerate(FLOATS):
        check_matmul(ix, *size, out_dtype, bias=i != 1, seed=i)
    check_matmul(ix, *size, torch.float32, True, pads=(16, 32, 5), seed=4)
    check_matmul(ix, *size, torch.float16, True, pads=(3, 1, 1), at=5, seed=5)
    check_matmul(ix, *size, torch.bfloat16, False, pads=(16 - size[2] % 16, 32 - size[2] % 16, 8), at=16, seed=6)


def test_matmul_sums_up_to_the_last_bit(ix):
    """The largest sums there are, 131071 products of -128 and -128, and sums whose 32-bit float is a rounding."""
    check_matmul(ix, 3, 5, 131071, torch.float32, False, extreme=True)
    check_matmul(ix, 70, 66, 131071, torch.float32, False, extreme=True)
    check_matmul(ix, 130, 140, 9999, torch.float32, True, extreme=True)


def test_matmul_rows_without_values(ix):
    """Scales that are NaN, infinite or zero go through to their rows and channels only."""
    a, sa, b, sb, c = product_inputs(40, 70, 96, 1)
    sa[3], sa[7], sb[5] = float("nan"), 0.0, float("inf")
    out = dz.scaled_matmul(ix, a.to(DEV), sa.to(DEV), b.to(DEV), sb.to(DEV)).cpu()
    want = plain.sums(a, b).float() * (sa[:, None] * sb[None])
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.isinf(out), torch.isinf(want))
    assert (out[7, 6:] == 0).all()
    assert dz.scaled_matmul(ix, a[:0].to(DEV), sa[:0].to(DEV), b.to(DEV), sb.to(DEV)).shape == (0, 70)
    assert dz.scaled_matmul(ix, a.to(DEV), sa.to(DEV), b[:0].to(DEV), sb[:0].to(DEV)).shape == (40, 0)


def test_matmul_is_the_same_bits_however_its_rows_are_grouped(ix):
    a, sa, b, sb, c = (t.to(DEV) for t in product_inputs(700, 300, 520, 2))
    whole = dz.scaled_matmul(ix, a, sa, b, sb, c)
    for lo, hi in [(0, 1), (1, 17), (17, 81), (81, 300), (300, 700)]:
        assert torch.equal(dz.scaled_matmul(ix, a[lo:hi], sa[lo:hi], b, sb, c), whole[lo:hi])
    assert torch.equal(dz.scaled_matmul(ix, a, sa, b[:33], sb[:33], c[:33]), whole[:, :33])


def test_matmul_over_parts_of_the_columns(ix):
    """Few tiles and many columns: the parts' sums lie in the workspace, which nothing is written behind; rows at odd bytes, which go in other
    parts, give the same bits, and so do calls of some of the rows."""
    for m, n, k in [(70, 200, 4096), (128, 1000, 8192), (64, 2000, 4864), (20, 64, 16384), (33, 130, 2049), (512, 1030, 4099), (5, 66, 4109), (1, 64, 9000)]:
        a, sa, b, sb, c = (t.to(DEV) for t in product_inputs(m, n, k, m))
        nbytes = dz.scaled_matmul_workspace_bytes(ix, m, n, k)
        assert nbytes >= 4 * 4 * m * n
        ws = torch.full((nbytes + 256,), 77, dtype=torch.uint8, device=DEV)
        for out_dtype in FLOATS:
            got = dz.scaled_matmul(ix, a, sa, b, sb, c, out_dtype=out_dtype, workspace=ws[:nbytes])
            odd = dz.scaled_matmul(ix, apart(a, 1, 3), sa, apart(b, 3, 1), sb, c, out_dtype=out_dtype, workspace=ws[:nbytes])
            assert torch.equal(got, odd)
            few = dz.scaled_matmul(ix, a[m // 2:], sa[m // 2:], b, sb, c, out_dtype=out_dtype)
            assert torch.equal(got[m // 2:], few)
        assert (ws[nbytes:] == 77).all()
        with pytest.raises(dz.DessertError, match="workspace too small"):
            dz.scaled_matmul(ix, a, sa, b, sb, c, workspace=ws[:nbytes - 256])


def test_matmul_over_more_than_32_bits_of_output_and_rows_far_apart(ix):
    """Element offsets past 2^31 and 2^32: rows of a 4 MB apart, an output of 2^32 elements' span."""
    m, n, k, far = 1100, 64, 128, 1 << 22
    a, sa, b, sb, _ = product_inputs(m, n, k, 3)
    buf = torch.zeros(m * far, dtype=torch.int8, device=DEV)
    view = buf.view(m, far)[:, :k]
    view.copy_(a)
    obuf = torch.zeros(m * far, dtype=torch.float16, device=DEV)
    out = obuf.view(m, far)[:, :n]
    dz.scaled_matmul(ix, view, sa.to(DEV), b.to(DEV), sb.to(DEV), out=out)
    want, tol = plain.matmul(a, sa, b, sb, None, torch.float16)
    plain.close(out.cpu().double().numpy(), want.numpy(), tol.numpy())


# ---- log probabilities ----------------------------------------------------------------------------------------------------
def tokens_for(n, V, g):
    t = torch.randint(0, V, (n,), generator=g)
    t[::7] = -1                                       # padded positions
    if n > 3:
        t[3] = V                                      # no such id
    return t


def check_token(ix, x, tokens, n_top, pad=0, at=0):
    got = dz.token_logprobs(ix, apart(x, pad, at), None if tokens is None else tokens.to(DEV), n_top)
    plain.check_logprobs(got, x, None if tokens is None else tokens.numpy(), n_top)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("shape", [(1, 1), (1, 2), (2, 7), (3, 64), (5, 255), (4, 257), (9, 2048), (7, 2049), (3, 8191), (2, 8200), (5, 30001), (1, 131071),
                                   (1030, 513), (1025, 8300), (100, 9600), (100, 9601), (24, 2300), (200, 20000)], ids=str)
def test_logprob_sizes(ix, shape, dtype):
    g = gen(shape[1])
    x = (3 * torch.randn(*shape, generator=g)).to(dtype)
    t = tokens_for(*shape, g)
    say("logprobs", shape, dtype)
    check_token(ix, x, t, min(5, shape[1]))
    check_token(ix, x, t.to(torch.int32), 20, pad=3, at=1)
    check_token(ix, x[:40], None, 0)
    check_token(ix, x[:40], t[:40], 64, pad=8)


@pytest.mark.parametrize("rows", [6, 1200])
@pytest.mark.parametrize("V", [50, 9000])
@pytest.mark.parametrize("dtype", FLOATS)
def test_logprob_masks_ties_and_numbers_that_are_not_finite(ix, dtype, V, rows):
    g = gen(V + rows)
    base = torch.randn(12, V, generator=g)
    inf, low = float("inf"), torch.finfo(dtype).min
    base[0] = -inf                                     # nothing left
    base[1] = low                                      # masked with the lowest value: even
    base[2, V // 2:] = -inf
    base[3] = -inf
    base[3, V - 1] = 2.0                               # one entry left
    base[4, 10] = inf
    base[5, V - 3] = float("nan")
    base[6] = 1.5                                      # all the same
    base[7] = torch.arange(V) / V                      # rising: every entry beats the ones before it
    base[8] = torch.where(torch.arange(V) % 3 == 0, low, 0.25)
    base[9, :] = 0.0
    base[9, 1::2] = -0.0                               # the two zeros tie
    base[10] = torch.finfo(dtype).max / 2
    base[10, 0] = low
    base[11] = -torch.arange(V) / 8.0                  # falling, into nothing
    x = base.to(dtype).repeat((rows + 11) // 12, 1)[:rows] if rows > 12 else base.to(dtype)
    t = torch.randint(0, V, (x.shape[0],), generator=g)
    t[4:6] = -1                                        # padded positions of rows without values
    say("logprob values", dtype, V, rows)
    for n_top in (1, 8, 64):
        check_token(ix, x, t, n_top)


def test_logprob_leaves_the_rows_behind_alone(ix):
    x = torch.randn(9, 3000, generator=gen(5)).to(DEV)
    lp, ent = torch.full((12,), 5.0, device=DEV), torch.full((12,), 5.0, device=DEV)
    ids = torch.full((12, 4), 9, dtype=torch.int32, device=DEV).view(torch.uint32)
    top = torch.full((12, 4), 5.0, device=DEV)
    t = torch.zeros(9, dtype=torch.int32, device=DEV)
    got = dz.token_logprobs(ix, x, t, 4, outs=(lp[:9], ent[:9], ids[:9], top[:9]))
    plain.check_logprobs(got, x.cpu(), t.cpu().numpy(), 4)
    assert (lp[9:] == 5).all() and (ent[9:] == 5).all() and (top[9:] == 5).all() and (ids.view(torch.int32)[9:] == 9).all()
    empty = dz.token_logprobs(ix, x[:0], t[:0], 4)
    assert [tuple(o.shape) for o in empty] == [(0,), (0,), (0, 4), (0, 4)]


def head_inputs(n, V, k, seed):
    g = gen(seed)
    a = torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8)
    b = torch.randint(-127, 128, (V, k), generator=g, dtype=torch.int8)
    scale = 3.0 / (73.3 * 73.3 * k ** 0.5)            # logits of about 3
    return a, torch.exp(0.3 * torch.randn(n, generator=g)), b, scale * torch.exp(0.1 * torch.randn(V, generator=g)), tokens_for(n, V, g)


@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 5, 16), (1, 1000, 64), (3, 130, 77), (1, 33000, 128), (16, 5000, 256), (17, 2049, 96), (70, 6001, 200),
                                   (130, 3000, 512), (300, 8500, 80), (1100, 600, 144), (40, 3000, 4096), (70, 1000, 8208), (50, 1000, 2301)], ids=str)
def test_head_sizes(ix, shape):
    n, V, k = shape
    a, sa, b, sb, t = head_inputs(n, V, k, V)
    l = plain.head_logits(a, sa, b, sb)
    for pad, at, n_top in [(0, 0, min(5, V)), (16, 16, 20), (5, 3, 64), (0, 0, 0)]:
        say("head", shape, pad, at, n_top)
        tokens = t if n_top != 20 else None
        got = dz.head_logprobs(ix, apart(a, pad, at), sa.to(DEV), apart(b, pad, at), sb.to(DEV), None if tokens is None else tokens.to(DEV), n_top)
        plain.check_logprobs(got, l, None if tokens is None else tokens.numpy(), n_top)


def test_head_in_turns_over_the_rows(ix):
    """More rows than one turn's logits take, the last turn a short one: the rows of all turns as one turn has them."""
    n, V, k = 1300, 60000, 64
    a, sa, b, sb, t = head_inputs(n, V, k, 8)
    ws = dz.head_logprobs_workspace_bytes(ix, n, V, k, 6)
    assert ws < n * V * 4
    args = [v.to(DEV) for v in (a, sa, b, sb, t.to(torch.int32))]
    whole = dz.head_logprobs(ix, *args, 6)
    for lo in (0, 255, 256, 1023, 1024, 1279, 1299):
        part = dz.head_logprobs(ix, args[0][lo:lo + 1], args[1][lo:lo + 1], args[2], args[3], args[4][lo:lo + 1], 6)
        plain.check_logprobs(part, plain.head_logits(a[lo:lo + 1], sa[lo:lo + 1], b, sb), t[lo:lo + 1].numpy(), 6)
        assert torch.equal(part[2].view(torch.int32)[0], whole[2].view(torch.int32)[lo])
    pick = torch.tensor([0, 254, 255, 256, 511, 512, 1000, 1279, 1280, 1299])
    got = [o[pick.to(DEV)] if o.dtype != torch.uint32 else o.view(torch.int32)[pick.to(DEV)].view(torch.uint32) for o in whole]
    plain.check_logprobs(got, plain.head_logits(a[pick], sa[pick], b, sb), t[pick].numpy(), 6)


def test_head_ties_and_scales_that_are_not_finite(ix):
    n, V, k = 40, 700, 64
    a, sa, b, sb, t = head_inputs(n, V, k, 9)
    b[100:400] = b[50]                                  # equal columns
    sb[100:400] = sb[50]
    a[1] = 0                                            # every logit 0
    sa[2], sa[3] = float("nan"), 0.0
    got = dz.head_logprobs(ix, *(v.to(DEV) for v in (a, sa, b, sb, t)), 30)
    plain.check_logprobs(got, plain.head_logits(a, sa, b, sb), t.numpy(), 30)


# rows and vocabularies from which on the logits do not go through memory
GROUPS = [(300, 20000, 128, 5), (256, 20129, 272, 33), (513, 20001, 64, 0), (1100, 7000, 96, 13), (33000, 200, 16, 0), (700, 11111, 1040, 21)]


@pytest.mark.parametrize("shape", GROUPS, ids=str)
def test_head_by_groups(ix, shape):
    n, V, k, n_top = shape
    say("head by groups", shape)
    a, sa, b, sb, t = head_inputs(n, V, k, V)
    pick = torch.unique(torch.cat([torch.arange(min(n, 40)), torch.randint(0, n, (60,), generator=gen(1)), torch.tensor([n - 1])]))
    l = plain.head_logits(a[pick], sa[pick], b, sb)
    for pad, tokens in [(0, t), (16, None), (32, t)]:
        got = dz.head_logprobs(ix, apart(a, pad), sa.to(DEV), apart(b, 2 * pad), sb.to(DEV), None if tokens is None else tokens.to(DEV), n_top)
        got = [None if o is None else o.view(torch.int32)[pick.to(DEV)].view(o.dtype) for o in got]
        plain.check_logprobs(got, l, None if tokens is None else tokens[pick].numpy(), n_top)
    # rows at odd bytes take the other way: the same alternatives, and sums that differ by their order only
    other = dz.head_logprobs(ix, apart(a, 3, 1), sa.to(DEV), apart(b, 5, 7), sb.to(DEV), t.to(DEV), n_top)
    other = [o.view(torch.int32)[pick.to(DEV)].view(o.dtype) for o in other]
    plain.check_logprobs(other, l, t[pick].numpy(), n_top)
    assert torch.equal(got[2].view(torch.int32), other[2].view(torch.int32))


def test_head_by_groups_ties_and_numbers_that_are_not_finite(ix):
    n, V, k, n_top = 300, 20100, 64, 30
    a, sa, b, sb, t = head_inputs(n, V, k, 12)
    b[300:9000] = b[50]                                 # equal columns, over many groups
    sb[300:9000] = sb[50]
    b[20050:] = b[20040]
    sb[20050:] = sb[20040]
    a[1] = 0                                            # every logit 0: the first ids
    sa[2], sa[3], sa[4] = float("nan"), 0.0, float("inf")
    a[5:200] = a[5]                                     # every row wants the same groups
    sa[5:200] = sa[5]
    a[10], sa[11] = b[50], 3.0                          # best entries are the equal ones
    got = dz.head_logprobs(ix, *(v.to(DEV) for v in (a, sa, b, sb, t)), n_top)
    pick = torch.arange(0, 60)
    with np.errstate(invalid="ignore"):
        l = plain.head_logits(a[pick], sa[pick], b, sb)
    plain.check_logprobs([o.view(torch.int32)[pick.to(DEV)].view(o.dtype) for o in got], l, t[pick].numpy(), n_top)
    # masked entries: scales of -inf make logits of -inf (or +inf, or NaN), whole groups of them
    sb[128:2048] = float("-inf")
    b[128:2048] = 1
    a[:60] = a[:60].abs().clamp(min=1)                  # positive sums there
    got = dz.head_logprobs(ix, *(v.to(DEV) for v in (a, sa, b, sb, t)), n_top)
    with np.errstate(invalid="ignore"):
        l = plain.head_logits(a[pick], sa[pick], b, sb)
    plain.check_logprobs([o.view(torch.int32)[pick.to(DEV)].view(o.dtype) for o in got], l, t[pick].numpy(), n_top)


def test_head_by_groups_in_turns_and_again(ix):
    """More rows than a turn takes, twice with one workspace: the same bits, though lists are filled in no fixed order."""
    n, V, k, n_top = 13000, 20000, 32, 39
    a, sa, b, sb, t = head_inputs(n, V, k, 14)
    args = [v.to(DEV) for v in (a, sa, b, sb, t.to(torch.int32))]
    ws = torch.empty(dz.head_logprobs_workspace_bytes(ix, n, V, k, n_top), dtype=torch.uint8, device=DEV)
    assert ws.numel() < 300 << 20
    first = [o.clone() for o in dz.head_logprobs(ix, *args, n_top, workspace=ws)]
    again = dz.head_logprobs(ix, *args, n_top, workspace=ws)
    for u, v in zip(first, again):
        assert torch.equal(u.view(torch.int32), v.view(torch.int32))
    pick = torch.cat([torch.arange(0, 13000, 311), torch.arange(11200, 11800, 40), torch.tensor([12999])])
    got = [o.view(torch.int32)[pick.to(DEV)].view(o.dtype) for o in first]
    plain.check_logprobs(got, plain.head_logits(a[pick], sa[pick], b, sb), t[pick].numpy(), n_top)


@pytest.mark.parametrize("n, V", [(9, 5000), (300, 20000)])
def test_outputs_that_nobody_asked_for(ix, n, V):
    """The C entry points without entropy, without tokens, and with nothing but alternatives."""
    k, n_top = 64, 6
    a, sa, b, sb, t = head_inputs(n, V, k, 17)
    l = plain.head_logits(a[:9], sa[:9], b, sb)
    d = [v.to(DEV) for v in (a, sa, b, sb, t.to(torch.int32))]
    logits = dz.scaled_matmul(ix, *d[:4])
    ws = torch.empty(max(dz.head_logprobs_workspace_bytes(ix, n, V, k, n_top), dz.token_logprobs_workspace_bytes(ix, n, V, n_top)),
                     dtype=torch.uint8, device=DEV)
    lp, ids, top = torch.empty(n, device=DEV), torch.empty(n, n_top, dtype=torch.int32, device=DEV), torch.empty(n, n_top, device=DEV)
    want = plain.logprobs(l, t[:9].numpy(), n_top)
    for with_tokens in (True, False):
        for call in ("head", "token"):
            lp.fill_(5.0)
            ids.zero_()
            tok = d[4].data_ptr() if with_tokens else None
            out = lp.data_ptr() if with_tokens else None
            if call == "head":
                st = dz.lib().dessert_head_logprobs(ix.handle, d[0].data_ptr(), k, d[1].data_ptr(), n, d[2].data_ptr(), k, d[3].data_ptr(), V, k, tok, n_top,
                                                    ws.data_ptr(), ws.numel(), out, None, ids.data_ptr(), top.data_ptr())
            else:
                st = dz.lib().dessert_token_logprobs(ix.handle, logits.data_ptr(), dz.F32, n, V, V, tok, n_top, ws.data_ptr(), ws.numel(), out, None,
                                                     ids.data_ptr(), top.data_ptr())
            assert st == dz.OK, dz.last_error()
            assert np.array_equal(ids[:9].cpu().numpy().view(np.uint32), want[2])
            if with_tokens:
                plain.close(lp[:9].cpu().numpy(), want[0], want[4] + 4 * plain.U32 * np.where(np.isfinite(want[0]), np.abs(want[0]), 0))
            else:
                assert (lp == 5).all()


# ---- as they are used -------------------------------------------------------------------------------------------------------
def test_from_states_to_the_index_and_from_candidates_to_likelihoods():
    """Encoder states -> int8 -> last layer -> unit vectors -> index and search, then the candidates' likelihoods: every step's outputs are
    the next one's inputs, and the search finds what it finds with vectors made in 64 bits."""
    g = gen(11)
    docs, m, hidden, d = 300, 20, 192, 128
    ix = dz.create(d, 32, 7, seed=3, device=torch.device(DEV))
    w = torch.randn(d, hidden, generator=g).to(DEV)
    states = torch.randn(docs * m, hidden, generator=g).to(torch.bfloat16).to(DEV)
    q = (states[7 * m:7 * m + 8].float() + 0.05 * torch.randn(8, hidden, generator=g).to(DEV)).to(torch.bfloat16)
    wc, ws = dz.quantize_rows(ix, w)

    def vectors(x):
        c, s = dz.quantize_rows(ix, x)
        y = dz.scaled_matmul(ix, c, s, wc, ws, out_dtype=torch.float16)
        v, _ = dz.quantize_rows(ix, y, dz.SCALE_UNIT)
        pc, ps = plain.quantize(x.cpu(), False)
        want, tol = plain.matmul(torch.from_numpy(pc), torch.from_numpy(ps), wc.cpu(), ws.cpu(), None, torch.float16)
        plain.close(y.cpu().double().numpy(), want.numpy(), tol.numpy())
        assert np.array_equal(v.cpu().numpy(), plain.quantize(y.cpu(), True)[0])
        return v

    X, Q = vectors(states), vectors(q)
    dz.build_index(ix, X, np.full(docs, m))
    ids, scores = dz.search(ix, Q, [8], 5)
    assert ids.view(torch.int32)[0, 0] == 7
    # likelihood of a query of 8 tokens under each candidate: states of the 5 candidates' continuations, padded to 10 positions
    V = 3001
    head, heads = dz.quantize_rows(ix, torch.randn(V, hidden, generator=g).to(DEV) / hidden ** 0.5)
    cont = torch.randn(5 * 10, hidden, generator=g).to(DEV)
    t = torch.randint(0, V, (5, 10), generator=g)
    t[:, 8:] = -1
    c, s = dz.quantize_rows(ix, cont)
    lp, ent, tid, tlp = dz.head_logprobs(ix, c, s, head, heads, t.reshape(-1).to(DEV), 4)
    l = plain.head_logits(c.cpu(), s.cpu(), head.cpu(), heads.cpu())
    plain.check_logprobs((lp, ent, tid, tlp), l, t.reshape(-1).numpy(), 4)
    logits = dz.scaled_matmul(ix, c, s, head, heads)    # the two forms agree
    again = dz.token_logprobs(ix, logits, t.reshape(-1).to(DEV), 4)
    plain.check_logprobs(again, logits.cpu(), t.reshape(-1).numpy(), 4)
    assert torch.equal(again[2].view(torch.int32), tid.view(torch.int32))
    assert (lp.view(5, 10)[:, 8:] == 0).all()
    likelihood = lp.view(5, 10).sum(1)
    assert torch.isfinite(likelihood).all()


@pytest.mark.parametrize("n", [37, 1024])
def test_captured_into_a_graph_and_replayed_with_new_inputs(n):
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ix = dz.create(128, 32, 7, seed=3)
        V, k = 9001, 208
        x = torch.empty(n, k, device=DEV)
        b = torch.empty(V, k, dtype=torch.int8, device=DEV)
        sb = torch.empty(V, device=DEV)
        t = torch.zeros(n, dtype=torch.int32, device=DEV)
        codes, scales = torch.empty(n, k, dtype=torch.int8, device=DEV), torch.empty(n, device=DEV)
        outs = (torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, 7, dtype=torch.uint32, device=DEV),
                torch.empty(n, 7, device=DEV))
        logits = torch.empty(n, V, device=DEV)
        outs2 = tuple(torch.empty_like(o) for o in outs)
        wsp = torch.empty(dz.head_logprobs_workspace_bytes(ix, n, V, k, 7), dtype=torch.uint8, device=DEV)
        wsp2 = torch.empty(max(256, dz.token_logprobs_workspace_bytes(ix, n, V, 7)), dtype=torch.uint8, device=DEV)
        wsp3 = torch.empty(max(256, dz.scaled_matmul_workspace_bytes(ix, n, V, k)), dtype=torch.uint8, device=DEV)

        def fill(seed):
            g = gen(seed)
            x.copy_(torch.randn(n, k, generator=g))
            a, sa, bb, s, tt = head_inputs(n, V, k, seed)
            b.copy_(bb)
            sb.copy_(s * 40)
            t.copy_(tt)

        def go():
            dz.quantize_rows(ix, x, out=codes, out_scales=scales)
            dz.head_logprobs(ix, codes, scales, b, sb, t, 7, workspace=wsp, outs=outs)
            dz.scaled_matmul(ix, codes, scales, b, sb, out=logits, workspace=wsp3)
            dz.token_logprobs(ix, logits, t, 7, workspace=wsp2, outs=outs2)

        fill(0)
        go()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            go()
        for seed in range(1, 5):
            fill(seed)
            for o in (*outs, *outs2):
                o.view(torch.int32).zero_()
            graph.replay()
            side.synchronize()
            pc, ps = plain.quantize(x.cpu(), False)
            pick = torch.arange(0, n, max(1, n // 37))
            l = plain.head_logits(torch.from_numpy(pc)[pick], torch.from_numpy(ps)[pick], b.cpu(), sb.cpu())
            replayed = [o.clone() for o in (*outs, *outs2)]
            picked = [o.view(torch.int32)[pick.to(DEV)].view(o.dtype) for o in replayed]
            plain.check_logprobs(picked[:4], l, t.cpu()[pick].numpy(), 7)
            plain.check_logprobs(picked[4:], logits.cpu()[pick], t.cpu()[pick].numpy(), 7)
            go()
            side.synchronize()
            for u, v in zip(replayed, (*outs, *outs2)):
                assert torch.equal(u.view(torch.int32), v.view(torch.int32))


@pytest.mark.parametrize("m,n,k", [(64, 1024, 4096), (20, 130, 4101), (100, 300, 8196)])
def test_parts_of_the_columns_captured_and_replayed(m, n, k):
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ix = dz.create(128, 32, 7, seed=3)
        a, sa, b, sb, c = (t.to(DEV) for t in product_inputs(m, n, k, 1))
        out = torch.empty(m, n, device=DEV)
        ws = torch.empty(dz.scaled_matmul_workspace_bytes(ix, m, n, k), dtype=torch.uint8, device=DEV)
        assert ws.numel()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            dz.scaled_matmul(ix, a, sa, b, sb, c, out=out, workspace=ws)
        for seed in range(2, 6):
            for t, new in zip((a, sa, b, sb, c), product_inputs(m, n, k, seed)):
                t.copy_(new)
            ws.fill_(seed)
            out.zero_()
            graph.replay()
            replayed = out.clone()
            side.synchronize()
            assert torch.equal(replayed, dz.scaled_matmul(ix, a, sa, b, sb, c))
            assert torch.equal(replayed, torch.cat([dz.scaled_matmul(ix, a[i:i + 16], sa[i:i + 16], b, sb, c) for i in range(0, m, 16)]))


def test_workspaces_of_sizes_that_are_refused(ix):
    for m, n, k in [(2 ** 40, 5, 9000), (5, 2 ** 63, 9000), (5, 5, 131072), (0, 5, 9000)]:
        assert dz.scaled_matmul_workspace_bytes(ix, m, n, k) == 0
    assert dz.head_logprobs_workspace_bytes(ix, 5, 1000, 131072, 3) == 0


def test_a_handle_on_another_stream_takes_tensors_made_here():
    """Copies, outputs and workspaces that the binding makes on the current stream go to work on the handle's."""
    side = torch.cuda.Stream()
    ix = dz.create(128, 32, 7, seed=3, device=torch.device(DEV), stream=side)
    for i in range(3):
        n, V, k = 260, 4001, 512
        a, sa, b, sb, t = head_inputs(n, V, k, 20 + i)
        wide = torch.empty(n, 2 * k, dtype=torch.int8, device=DEV)
        wide[:, ::2] = a.to(DEV)
        args = [wide[:, ::2], sa.to(DEV), b.to(DEV), sb.to(DEV), t.to(DEV)]        # every other column: copied by the binding
        got = dz.head_logprobs(ix, *args, 6)
        y = dz.scaled_matmul(ix, *args[:4], out_dtype=torch.float32)
        torch.cuda.current_stream().wait_stream(side)
        l = plain.head_logits(a, sa, b, sb)
        plain.check_logprobs(got, l, t.numpy(), 6)
        assert torch.equal(y.cpu(), l)


def test_two_handles_on_two_streams_at_once():
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    jobs = []
    for i, s in enumerate(streams):
        ix = dz.create(128, 32, 7, seed=3, device=torch.device(DEV), stream=s)
        n, V, k = 90, 20011, 320
        a, sa, b, sb, t = head_inputs(n, V, k, 30 + i)
        jobs.append((ix, [v.to(DEV) for v in (a, sa, b, sb, t.to(torch.int32))], plain.head_logits(a, sa, b, sb), t))
    torch.cuda.synchronize()
    got = [[dz.head_logprobs(ix, *args, 9) for ix, args, _, _ in jobs] for _ in range(4)]
    torch.cuda.synchronize()
    for turn in got:
        for out, (_, _, l, t) in zip(turn, jobs):
            plain.check_logprobs(out, l, t.numpy(), 9)
