"""Attention over the paged cache with scales of every size: outputs that bfloat16 holds come out right whatever the scales are."""
import math

import pytest
import torch

import paper_2210_15748_amd as dz

import cache_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAMES = ("k", "v", "ks", "vs", "bounds")


@pytest.fixture(scope="module")
def ix():
    return dz.create(128, 32, 7, seed=1)


# (lengths, new tokens, query heads of a key head): one workgroup of eight waves; split and joined, by a wave a row; split far, joined by a workgroup
# a row; many rows in one part; many rows split
FORMS = {"few": ([700, 333], [1, 1], 2), "few split": ([3000, 90], [1, 3], 2), "few split far": ([9000], [1], 1), "many": ([250, 200], [90, 60], 2),
         "many split": ([1500, 300], [70, 70], 2)}


def check(ix, c, lengths, new, group, page, scale=0.125, q=None, window=0):
    P, H, _, D = c["k"].shape
    tables = plain.make_tables(lengths, page, P, 3)
    if q is None:
        q = torch.randn(sum(new), H * group, D, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    want = plain.attend(c, tables, lengths, new, q, scale, window)
    b = dz.cache_batch(ix, tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), plain.starts_of(new).to(DEV), n_tokens=sum(new),
                       max_tokens=max(new), max_length=max(lengths))
    g = {k: v.to(DEV) for k, v in c.items()}
    out, lse = dz.cache_attention(ix, dz.cache(ix, *(g[n] for n in NAMES)), b, q.to(DEV), scale, window=window)
    t_out, t_lse = plain.attend_tolerance(*want, torch.bfloat16, max(lengths), D)
    t_out = t_out + 2.0 ** -134      # half the step of bfloat16's subnormal numbers (32-bit ones': 2^-150 an addition)
    out, lse = out.cpu().double(), lse.cpu().double()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    assert bool(((out - want[0]).abs() <= t_out).all()), float(((out - want[0]).abs() / t_out).max())
    assert bool(((lse - want[1]).abs() <= t_lse).all()), float(((lse - want[1]).abs() / t_lse).max())
    return want[0]


def pool(lengths, page, dim, seed=4):
    return plain.make_cache(sum(-(-n // page) for n in lengths), 1, page, dim, seed)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("power", [-104, -108, -110, -113, -118, -126, -133])
def test_small_value_scales(ix, form, page, power):
    lengths, new, group = FORMS[form]
    c = pool(lengths, page, 64)
    c["vs"] = torch.ldexp(c["vs"] / 0.022, torch.tensor(power))
    assert float(c["vs"].max()) < 2.0 ** power and bool((c["vs"] > 0).all())
    want = check(ix, c, lengths, new, group, page)
    assert float(want.abs().max()) > 2.0 ** power


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("power", [100, 112, 120])
def test_large_value_scales(ix, form, page, power):
    """Values near the largest that bfloat16 holds: their mean is one of them, though their sum is none."""
    lengths, new, group = FORMS[form]
    c = pool(lengths, page, 64)
    c["vs"] = torch.ldexp(c["vs"] / 0.022, torch.tensor(power))
    c["v"] = c["v"].abs()
    q = torch.zeros(sum(new), group, 64, dtype=torch.bfloat16)
    check(ix, c, lengths, new, group, page, q=q)


# Powers of two of two kinds of pages' value scales, and of e^s on the second kind's keys (1 on the first's)
APART = [(-20, 20, -30), (-63, 63, -120), (-100, 20, -115), (0, 119, -124), (-75, 75, -145), (-110, 100, -205)]


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("small,large,depth", APART)
def test_value_scales_far_apart_that_scores_make_up_for(ix, form, page, small, large, depth):
    """Keys with next to no weight and values so large that they count all the same, among keys with all the weight and small values."""
    lengths, new, group = FORMS[form]
    c = pool(lengths, page, 64)
    g = torch.Generator().manual_seed(depth)
    P = c["k"].shape[0]
    second = torch.rand(P, generator=g) < 0.4
    c["k"][:] = 0
    c["k"][second] = -127
    c["ks"][:] = -depth * math.log(2.0) / (127 * 64 * 0.125)
    c["vs"] = torch.ldexp(c["vs"] / 0.022, torch.where(second, large, small)[:, None])
    q = torch.ones(sum(new), group, 64, dtype=torch.bfloat16)
    check(ix, c, lengths, new, group, page, q=q)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("q_power,k_power", [(-110, 104), (-120, 114), (-122, 116), (-126, 119), (120, -127), (124, -131), (125, -133)])
def test_queries_and_key_scales_of_opposite_sizes(ix, form, page, q_power, k_power):
    """Scores of an ordinary size, of tiny queries and huge keys or the other way round."""
    lengths, new, group = FORMS[form]
    c = pool(lengths, page, 64)
    c["ks"] = torch.ldexp(c["ks"] / 0.022, torch.tensor(k_power))
    q = torch.ldexp(torch.randn(sum(new), group, 64, generator=torch.Generator().manual_seed(5)), torch.tensor(q_power)).to(torch.bfloat16)
    assert torch.isfinite(q).all()
    check(ix, c, lengths, new, group, page, q=q)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("depth", [-20, -60])
def test_few_keys_of_all_the_weight_among_many_large_values(ix, form, page, depth):
    """One page with the weight of a row; parts of the other keys' axis whose sums are many times its, and whose values are near the largest number."""
    lengths, new, group = FORMS[form]
    c = pool(lengths, page, 64)
    tables = plain.make_tables(lengths, page, c["k"].shape[0], 3)
    first = tables[:, 0].long()
    c["k"][:] = -127
    c["k"][first] = 0
    c["ks"][:] = -depth * math.log(2.0) / (127 * 64 * 0.125)
    c["vs"] = torch.ldexp(c["vs"] / 0.022, torch.tensor(120))
    c["vs"][first] *= 2.0 ** -110
    c["v"] = torch.full_like(c["v"], 127)
    q = torch.ones(sum(new), group, 64, dtype=torch.bfloat16)
    check(ix, c, lengths, new, group, page, q=q)
