"""The paged int8 cache on the GPU against its definitions: attention over one token and many, pages given and chosen, appending, sequences
that go on, compaction, and a run of them together."""
import math

import numpy as np
import pytest
import torch

import paper_2210_15748_amd as dz

import cache_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ix():
    return dz.create(128, 32, 7, seed=1)


def on_gpu(c):
    return {k: v.to(DEV) for k, v in c.items()}


def taken(ix, c):
    return dz.cache(ix, c["k"], c["v"], c["ks"], c["vs"], c["bounds"])


def batch_of(ix, tables, lengths, new, rows=None, **kw):
    return dz.cache_batch(ix, tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), plain.starts_of(new).to(DEV),
                          n_tokens=sum(new) if rows is None else rows, max_tokens=max(max(new), 1), max_length=max(lengths), **kw)


def check_attention(ix, c, tables, lengths, new, heads, dtype, window=0, pages=None, seed=0, scale=None, q=None, one_each=False):
    D = c["k"].shape[3]
    g = torch.Generator().manual_seed(seed + 77)
    if q is None:
        q = torch.randn(sum(new), heads, D, generator=g).to(dtype)
    scale = 1 / math.sqrt(D) if scale is None else scale
    want = plain.attend(c, tables, lengths, new, q, scale, window, pages)
    gc = on_gpu(c)
    b = batch_of(ix, tables, lengths, new)
    if one_each:
        b = dz.cache_batch(ix, tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), max_length=max(lengths))
    out, lse = dz.cache_attention(ix, taken(ix, gc), b, q.to(DEV), scale, window=window, pages=None if pages is None else pages.to(DEV))
    torch.cuda.synchronize()
    close(out, lse, want, dtype, max(lengths), D)
    return out, lse


def close(out, lse, want, dtype, keys, D):
    t_out, t_lse = plain.attend_tolerance(*want, dtype, keys, D)
    out, lse = out.cpu().double(), lse.cpu().double()
    w_out, w_lse = want[0], want[1]
    assert torch.equal(out.isnan(), w_out.isnan()) and torch.equal(lse.isnan(), w_lse.isnan())
    assert torch.equal(torch.isneginf(lse), torch.isneginf(w_lse))
    f = torch.isfinite(w_out)
    assert bool(((out - w_out).abs()[f] <= t_out[f]).all()), float(((out - w_out).abs() / t_out)[f].max())
    f = torch.isfinite(w_lse)
    assert bool(((lse - w_lse).abs()[f] <= t_lse[f]).all()), float(((lse - w_lse).abs() / t_lse)[f].max())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("lengths,new,group", [
    ([1, 70, 333], [1, 1, 1], 4),          # one token each
    ([5, 64, 129], [5, 3, 1], 1),          # a few
    ([40, 65, 300], [40, 33, 17], 3),      # many rows, a first token of a sequence among them
])
def test_attention_over_dims(ix, dim, dtype, lengths, new, group):
    c = plain.make_cache(48, 2, 16, dim, dim)
    check_attention(ix, c, plain.make_tables(lengths, 16, 48, dim + 1), lengths, new, 2 * group, dtype)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window", [0, 1, 50, 1000])
@pytest.mark.parametrize("new", [1, 7, 150])
def test_attention_over_pages_and_windows(ix, page, window, new):
    lengths = [new, 511, 900, page + 1 if page + 1 >= new else new]
    pages = sum(-(-n // page) for n in lengths) + 3
    c = plain.make_cache(pages, 2, page, 64, page)
    check_attention(ix, c, plain.make_tables(lengths, page, pages, page), lengths, [new, new, new // 2 + 1, new], 4, torch.float16, window=window)


@pytest.mark.parametrize("group", [1, 2, 5, 16, 17, 40])
@pytest.mark.parametrize("new", [1, 3])
def test_attention_over_groups(ix, group, new):
    lengths = [new, 200, 77]
    c = plain.make_cache(12, 3, 32, 64, group)
    check_attention(ix, c, plain.make_tables(lengths, 32, 12, 4), lengths, [new] * 3, 3 * group, torch.bfloat16)


@pytest.mark.parametrize("length,new", [(9000, 1), (20000, 1), (9000, 40), (9000, 300)])
def test_attention_split_along_the_keys(ix, length, new):
    lengths = [length, max(new, length // 7 + 3), new]
    pages = sum(-(-n // 64) for n in lengths)
    c = plain.make_cache(pages, 1, 64, 64, 5)
    check_attention(ix, c, plain.make_tables(lengths, 64, pages, 6), lengths, [new, new, new], 2, torch.float16)
    check_attention(ix, c, plain.make_tables(lengths, 64, pages, 6), lengths, [new, new, new], 2, torch.bfloat16, window=5000)


def test_one_token_each_without_starts(ix):
    lengths = [1, 90, 256, 300]
    c = plain.make_cache(50, 2, 16, 128, 1)
    check_attention(ix, c, plain.make_tables(lengths, 16, 50, 1), lengths, [1] * 4, 8, torch.float16, one_each=True)


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [0, 3, 2, 0], [60, 0, 70, 5]])
def test_rows_that_see_nothing(ix, new):
    """A length of 0, tokens before a sequence's beginning, pages that are missing: zeros and -inf, or what the other pages hold."""
    lengths = [0, 100, 64, 3]
    c = plain.make_cache(20, 2, 32, 64, 2)
    tables = plain.make_tables(lengths, 32, 20, 3)
    tables[1, 1] = -1
    tables[1, 2] = 20              # not in the pool
    tables[2, :] = 0x7FFFFFFF
    check_attention(ix, c, tables, lengths, new, 4, torch.float16)
    check_attention(ix, c, tables, lengths, new, 4, torch.float16, window=30)


@pytest.mark.parametrize("new", [1, 50])
def test_what_no_row_sees_does_not_matter(ix, new):
    """Scales that are no numbers on pages behind a row's position or before its window; codes behind a sequence's end."""
    lengths = [150, 170]
    c = plain.make_cache(30, 1, 16, 64, 2)
    tables = plain.make_tables(lengths, 16, 30, 3, width=14)
    free = sorted(set(range(30)) - set(tables.flatten().tolist()))
    tables[0, 10:14] = torch.tensor(free[:4])
    for bad in (math.nan, math.inf):
        d = {k: v.clone() for k, v in c.items()}
        for b, first in ((0, 0), (1, 1)):
            d["ks"][tables[b, first]] = bad        # before the window of every row
            d["vs"][tables[b, first]] = bad
        for p in free:
            d["ks"][p] = bad
            d["vs"][p] = bad
        check_attention(ix, d, tables, lengths, [new] * 2, 2, torch.float16, window=60)
    # a page of later tokens that only the last rows see
    if new > 1:
        d = {k: v.clone() for k, v in c.items()}
        d["vs"][tables[0, 9]] = math.nan
        want = plain.attend(c, tables, lengths, [new] * 2, torch.zeros(2 * new, 2, 64), 1.0)
        q = torch.zeros(2 * new, 2, 64, dtype=torch.float16)
        gd = on_gpu(d)
        out, _ = dz.cache_attention(ix, taken(ix, gd), batch_of(ix, tables, lengths, [new] * 2), q.to(DEV), 1.0)
        out = out.cpu().double()
        hit = torch.zeros(2 * new, dtype=torch.bool)
        hit[new - 6:new] = True                    # positions 144 .. 149
        assert out[hit].isnan().all() and not out[~hit].isnan().any()
        assert float((out - want[0])[~hit].abs().max()) < 0.01


def test_scales_far_apart(ix):
    """Pages whose scales differ by many powers of two, zeros among them: the small ones still count where they are what a row sees."""
    lengths = [400, 333]
    c = plain.make_cache(64, 1, 16, 64, 8)
    c["vs"] *= torch.exp2(torch.randint(-30, 30, c["vs"].shape, generator=torch.Generator().manual_seed(1)).float())
    c["vs"][3] = 0
    c["ks"][5] = 0
    tables = plain.make_tables(lengths, 16, 64, 8)
    for new in (1, 40):
        check_attention(ix, c, tables, lengths, [new] * 2, 2, torch.bfloat16)
        check_attention(ix, c, tables, lengths, [new] * 2, 2, torch.bfloat16, window=5)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("new", [1, 30])
def test_queries_of_every_size(ix, dtype, new):
    """Large and small rows, rows of zeros, infinities and NaN; a negative scale."""
    lengths = [100, 64]
    c = plain.make_cache(16, 2, 16, 64, 4)
    q = torch.randn(2 * new, 4, 64, generator=torch.Generator().manual_seed(4))
    q[:, 0] *= 60.0
    q[:, 1] *= 1e-4
    q[0, 2] = 0
    q[-1, 3, 5] = math.inf
    q[0, 3, 5] = math.nan
    if dtype == torch.bfloat16:
        q[:, 1] *= 1e-30
    check_attention(ix, c, plain.make_tables(lengths, 16, 16, 4), lengths, [new] * 2, 4, dtype, q=q.to(dtype))
    check_attention(ix, c, plain.make_tables(lengths, 16, 16, 4), lengths, [new] * 2, 4, dtype, q=q.to(dtype), scale=-0.07)
    if dtype == torch.bfloat16:
        big = torch.randn(2 * new, 4, 64, generator=torch.Generator().manual_seed(4)) * 1e30
        check_attention(ix, c, plain.make_tables(lengths, 16, 16, 4), lengths, [new] * 2, 4, dtype, q=big.to(dtype), scale=1e-31)


def test_queries_out_of_a_wider_array_and_rows_behind_the_last(ix):
    lengths, new = [100, 64, 30], [2, 0, 1]
    c = plain.make_cache(16, 2, 16, 64, 4)
    tables = plain.make_tables(lengths, 16, 16, 4)
    wide = torch.randn(6, 10, 64, generator=torch.Generator().manual_seed(9)).to(torch.float16)
    want = plain.attend(c, tables, lengths, new, wide[:3, 3:7], 0.125)
    out, lse = torch.full((6, 4, 64), 7.0, dtype=torch.float16, device=DEV), torch.full((6, 4), 7.0, device=DEV)
    g = on_gpu(c)
    dz.cache_attention(ix, taken(ix, g), batch_of(ix, tables, lengths, new, rows=6), wide.to(DEV)[:, 3:7], 0.125, out=out, out_lse=lse)
    torch.cuda.synchronize()
    close(out[:3], lse[:3], want, torch.float16, 100, 64)
    assert bool((out[3:] == 7).all()) and bool((lse[3:] == 7).all())


@pytest.mark.parametrize("group", [1, 4, 20])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("new", [1, 3])
def test_attention_over_listed_pages(ix, group, page, new):
    lengths = [new, 700, 1500]
    pages = sum(-(-n // page) for n in lengths)
    c = plain.make_cache(pages, 2, page, 64, page)
    tables = plain.make_tables(lengths, page, pages, 6)
    g = torch.Generator().manual_seed(3)
    width = tables.shape[1]
    ids = torch.stack([torch.randperm(width + 3, generator=g)[:6] for _ in range(3 * new * 2)]).view(3 * new, 2, 6).to(torch.int32)
    ids[1, 1] = -1                    # a token that looks at nothing
    ids[:, 0, 5] = -1
    check_attention(ix, c, tables, lengths, [new] * 3, 2 * group, torch.float16, pages=ids)
    check_attention(ix, c, tables, lengths, [new] * 3, 2 * group, torch.float16, pages=ids, window=300)


# ---- appending -----------------------------------------------------------------------------------------------------------------
def same_cache(got, want):
    for name in want:
        a, b = got[name].cpu(), want[name]
        if a.dtype.is_floating_point:
            a, b = a.view(torch.int32), b.view(torch.int32)
            a, b = torch.where(got[name].cpu().isnan(), 0, a), torch.where(want[name].isnan(), 0, b)
            assert torch.equal(got[name].cpu().isnan(), want[name].isnan())
        assert torch.equal(a, b), name


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dim", [32, 96, 128, 256])
def test_append(ix, dtype, page, dim):
    """Chunks of unequal lengths one after the other, single tokens among them, in pages that hold something else before."""
    c = plain.make_cache(24 if page >= 64 else 90, 2, page, dim, 3)
    g = torch.Generator().manual_seed(dim + page)
    steps = [[70, 0, 1], [1, 130, 1], [1, 1, 1], [5, 40, 16], [1, 1, 31], [200, 1, 0]]
    total = [sum(s[b] for s in steps) for b in range(3)]
    tables = plain.make_tables(total, page, c["k"].shape[0], 5)
    gc = on_gpu(c)
    length = [0, 0, 0]
    for i, new in enumerate(steps):
        length = [a + b for a, b in zip(length, new)]
        x = torch.randn(sum(new), 5, dim, generator=g) * (1 + i) * torch.exp(torch.randn(sum(new), 1, 1, generator=g))
        x = x.to(dtype)
        plain.append(c, tables, length, new, x[:, :2], x[:, 3:])
        dz.cache_append(ix, taken(ix, gc), batch_of(ix, tables, length, new), x.to(DEV)[:, :2], x.to(DEV)[:, 3:])
        same_cache(gc, c)


def test_append_of_odd_values(ix):
    """Halves between codes, zeros, subnormal and huge numbers, infinities and NaN and what comes after them; pages that are missing."""
    page, dim = 16, 32
    c = plain.make_cache(12, 1, page, dim, 3)
    tables = plain.make_tables([16, 16, 16, 16, 16, 48], page, 12, 5)
    tables[5, 1] = -1
    gc = on_gpu(c)
    x = torch.zeros(6 * 16, 1, dim)
    half = torch.arange(dim) - 15.5
    x[0:16, 0] = half * torch.arange(1, 17)[:, None]
    x[0:16, 0, 0] = 127
    x[16:32, 0] = 1e-44 * torch.arange(dim)
    x[32:48, 0] = 3e38
    x[48:64, 0, 3] = math.inf
    x[64:80, 0, 3] = math.nan
    x[80:] = torch.randn(16, 1, dim, generator=torch.Generator().manual_seed(1))
    for lengths, new in (([8, 8, 8, 8, 8, 40], [8, 8, 8, 8, 8, 40]), ([9, 9, 9, 9, 9, 41], [1] * 6), ([16, 16, 16, 16, 16, 48], [7] * 6)):
        y = torch.cat([x[16 * min(b, 5):16 * min(b, 5) + 16].repeat(3, 1, 1)[:n] * (1 + (n == 7)) for b, n in enumerate(new)])
        if new[0] == 1:
            y[:] = 1.0
        plain.append(c, tables, lengths, new, y, -y)
        dz.cache_append(ix, taken(ix, gc), batch_of(ix, tables, lengths, new), y.to(DEV), -y.to(DEV))
        same_cache(gc, c)
    assert c["ks"].isnan().any()


def test_append_begins_pages_anew_and_leaves_the_rest(ix):
    c = plain.make_cache(8, 2, 32, 64, 3)
    before = {k: v.clone() for k, v in c.items()}
    tables = torch.tensor([[2, 5], [7, 0]], dtype=torch.int32)
    gc = on_gpu(c)
    gc["ks"][2] = math.nan                        # of the page's last use
    c["ks"][2] = math.nan
    x = torch.randn(8, 2, 64, generator=torch.Generator().manual_seed(2))
    plain.append(c, tables, [3, 34], [3, 2], x[:5], x[:5])
    dz.cache_append(ix, taken(ix, gc), batch_of(ix, tables, [3, 34], [3, 2], rows=8), x.to(DEV), x.to(DEV))
    same_cache(gc, c)
    for name in before:
        for p in (1, 3, 4, 5, 6, 7):
            assert torch.equal(gc[name][p].cpu(), before[name][p])
    assert torch.equal(gc["k"][2, :, 3:].cpu(), before["k"][2, :, 3:]) and torch.equal(gc["v"][2, :, :, 3:].cpu(), before["v"][2, :, :, 3:])


def test_append_without_bounds(ix):
    c = plain.make_cache(8, 2, 32, 64, 3)
    gc = on_gpu(c)
    tables = torch.tensor([[2, 5]], dtype=torch.int32)
    x = torch.randn(40, 2, 64, generator=torch.Generator().manual_seed(2)).to(torch.float16)
    kept = c["bounds"].clone()
    plain.append(c, tables, [40], [40], x, x)
    dz.cache_append(ix, dz.cache(ix, gc["k"], gc["v"], gc["ks"], gc["vs"]), batch_of(ix, tables, [40], [40]), x.to(DEV), x.to(DEV))
    c["bounds"] = kept
    same_cache(gc, c)


# ---- choosing pages --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("group", [1, 5, 16, 19])
def test_select(ix, dim, group):
    page, lengths, new = 16, [1, 900, 5000, 0, 37], [1, 2, 1, 1, 3]
    pages = sum(-(-n // page) for n in lengths)
    c = plain.make_cache(pages, 2, page, dim, dim)
    tables = plain.make_tables(lengths, page, pages, 1)
    g = torch.Generator().manual_seed(2)
    n, heads = sum(new), 2 * group
    codes = torch.randint(-127, 128, (n * heads, dim), generator=g, dtype=torch.int8)
    scales = torch.rand(n * heads, generator=g)
    gc = on_gpu(c)
    for n_select, first, last in ((1, 0, 0), (1, 0, 1), (7, 1, 2), (40, 0, 0), (64, 3, 5), (400, 1, 1)):
        want = plain.select(c, tables, lengths, new, codes, scales, n_select, first, last)
        out = torch.full((n, 2, n_select), 5, dtype=torch.int32, device=DEV).view(torch.uint32)
        got = dz.cache_select(ix, taken(ix, gc), batch_of(ix, tables, lengths, new), codes.to(DEV), scales.to(DEV), n_select, first, last, out=out)
        assert np.array_equal(got.cpu().numpy(), want)


def test_select_ties_and_numbers_that_are_none(ix):
    """Equal scores go to the lower place; NaN and infinities are the highest; missing pages are none."""
    page, lengths, new = 16, [4000], [1]
    c = plain.make_cache(250, 1, page, 32, 1)
    c["bounds"][:] = c["bounds"][0]
    c["ks"][:] = 0.5
    tables = plain.make_tables(lengths, page, 250, 1)
    codes = torch.randint(-127, 128, (2, 32), generator=torch.Generator().manual_seed(1), dtype=torch.int8)
    scales = torch.tensor([1.0, 0.25])
    b = batch_of(ix, tables, lengths, new)
    for change in ("", "nan", "inf", "missing", "zero"):
        if change == "nan":
            c["ks"][tables[0, 77]] = math.nan
        elif change == "inf":
            c["ks"][tables[0, 99]] = math.inf
        elif change == "missing":
            tables[0, 3] = -1
            tables[0, 249] = 9999
            b = batch_of(ix, tables, lengths, new)
        elif change == "zero":
            codes.zero_()
        gc = on_gpu(c)
        for n_select, first, last in ((20, 0, 0), (20, 2, 3), (300, 0, 0)):
            want = plain.select(c, tables, lengths, new, codes, scales, n_select, first, last)
            got = dz.cache_select(ix, taken(ix, gc), b, codes.to(DEV), scales.to(DEV), n_select, first, last)
            assert np.array_equal(got.cpu().numpy(), want), change


# ---- sequences going on, compaction ---------------------------------------------------------------------------------------------
def check_advance(ix, c, refs, tables, lengths, add, parents):
    gc = on_gpu(c)
    g_refs, g_tables, g_lengths = refs.to(DEV), tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV)
    caches = [dz.cache(ix, *(gc[k][i] for k in ("k", "v", "ks", "vs", "bounds"))) for i in range(c["k"].shape[0])]
    got = dz.cache_advance(ix, caches, g_refs, g_tables, g_lengths, torch.tensor(add, dtype=torch.int32, device=DEV),
                           parents=None if parents is None else torch.tensor(parents, dtype=torch.int32, device=DEV))
    t, l, status = plain.advance(c, refs, tables, lengths, add, parents)
    assert torch.equal(got[0].cpu(), t) and torch.equal(got[1].cpu(), l) and got[2].tolist() == status
    assert torch.equal(g_refs.cpu(), refs)
    same_cache(gc, c)
    return t, l.tolist(), status


def held(tables, lengths, page, pages):
    refs = torch.zeros(pages, dtype=torch.int32)
    for b, n in enumerate(lengths):
        for j in range(-(-n // page)):
            refs[tables[b, j]] += 1
    return refs


@pytest.mark.parametrize("page,heads,dim", [(16, 1, 32), (64, 2, 96)])
def test_advance_step_by_step(ix, page, heads, dim):
    """Forks, beams that go on from one another, ended ones, new ones, a run out of pages, one after the other from an empty pool."""
    pages, width = 30, 9
    c = plain.make_cache(pages, heads, page, dim, 1, layers=2)
    refs, tables, lengths = torch.zeros(pages, dtype=torch.int32), torch.full((1, width), -1, dtype=torch.int32), [0]
    rng = np.random.default_rng(page)
    refused = 0
    steps = [([-1, -1, -1], [page * 2 + 3, page, 1]), ([0, 0, 0, 1, 1, 2], [1] * 6), ([0, 1, 2, 3, 4, 5], [1, 0, 1, 0, 1, 0]),
             ([0, 0, 1, 1, 2, 2], [0, 1, 1, 1, page, 1]), (None, [1] * 6), ([5, 4, 3, 2, 1, 0, 0, 0], [1] * 8)]
    for i in range(12):
        n = 8 if i == 0 else int(rng.integers(1, 11))
        steps.append(([int(x) for x in rng.integers(-1, n if i else 8, int(rng.integers(1, 11)))], None))
    for parents, add in steps:
        if add is None:
            parents = [p if p < len(lengths) else -1 for p in parents]
            add = [int(x) for x in rng.choice([0, 1, 1, 1, 2, page, 3 * page], len(parents))]
        tables, lengths, status = check_advance(ix, c, refs, tables, lengths, add, parents)
        refused += status[1]
        assert torch.equal(refs, held(tables, lengths, page, pages))
        tables = tables.contiguous()
    _, _, status = check_advance(ix, c, refs, tables, lengths, [page * 5] * 8, [0] * 8)
    assert refused + status[1] > 0


def test_advance_of_many_sequences(ix):
    """More sequences and pages than one pass of a workgroup."""
    page, pages, n = 16, 9000, 1500
    g = np.random.default_rng(1)
    lengths = [int(x) for x in g.integers(1, 60, n)]
    c = plain.make_cache(pages, 1, page, 32, 1, layers=1)
    tables = plain.make_tables(lengths, page, pages, 2, width=5)
    refs = held(tables, lengths, page, pages)
    parents = [int(x) for x in g.integers(0, n, n)]
    tables, lengths, _ = check_advance(ix, c, refs, tables, lengths, [1] * n, parents)
    tables, lengths, _ = check_advance(ix, c, refs, tables, lengths, [int(x) for x in g.integers(0, 30, n)], None)
    refs[refs == 0] = torch.from_numpy((g.random(int((refs == 0).sum())) < 0.97).astype(np.int32))
    _, _, status = check_advance(ix, c, refs, tables, lengths, [int(x) for x in g.integers(0, 30, n)], [int(x) for x in g.integers(0, n, n)])
    assert status[1] > 0


def test_advance_of_many_layers(ix):
    page, pages = 16, 12
    c = plain.make_cache(pages, 1, page, 32, 1, layers=35)
    tables = torch.tensor([[4, 2, -1]], dtype=torch.int32)
    check_advance(ix, c, held(tables, [20], page, pages), tables, [20], [1, 1, 1], [0, 0, 0])


def test_advance_to_nothing_and_from_nothing(ix):
    c = plain.make_cache(6, 1, 16, 32, 1, layers=1)
    tables = torch.tensor([[4, 2, -1]], dtype=torch.int32)
    refs = held(tables, [20], 16, 6)
    check_advance(ix, c, refs, tables, [20], [], [])
    assert not refs.any()
    check_advance(ix, c, refs, torch.zeros(0, 3, dtype=torch.int32), [], [5, 40, 100], [-1, 7, -1])


@pytest.mark.parametrize("pages,part", [(1, 1.0), (5, 0.0), (40, 0.5), (3000, 0.3), (3000, 0.99)])
def test_compact(ix, pages, part):
    page, layers = 16, 2
    g = np.random.default_rng(pages)
    c = plain.make_cache(pages, 1, page, 32, 1, layers=layers)
    used = g.permutation(pages)[:int(pages * part)]
    width = 4
    rows = [used[i:i + width] for i in range(0, len(used), width)]
    tables = torch.full((len(rows) + 1, width), -1, dtype=torch.int32)
    lengths = [0] * (len(rows) + 1)
    for b, r in enumerate(rows):
        tables[b, :len(r)] = torch.from_numpy(r.astype(np.int32))
        lengths[b] = len(r) * page - b % page
    if rows:
        tables[-1], lengths[-1] = tables[0], lengths[0]        # shared pages
        tables[0, len(rows[0]):] = 12345                       # behind a sequence's pages: stays
    refs = held(tables, lengths, page, pages)
    gc, g_refs, g_tables = on_gpu(c), refs.to(DEV), tables.to(DEV)
    caches = [dz.cache(ix, *(gc[k][i] for k in ("k", "v", "ks", "vs", "bounds"))) for i in range(layers)]
    before = {k: v.clone() for k, v in c.items()}
    numbers, live = dz.cache_compact(ix, caches, g_refs, g_tables, torch.tensor(lengths, dtype=torch.int32, device=DEV))
    w_numbers, n = plain.compact(c, refs, tables, lengths)
    assert live.tolist() == [n] and torch.equal(numbers.cpu(), w_numbers)
    assert torch.equal(g_tables.cpu(), tables) and torch.equal(g_refs.cpu(), refs)
    same_cache(gc, c)
    assert torch.equal(gc["k"][:, n:].cpu(), before["k"][:, n:])
