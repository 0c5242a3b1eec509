"""Calls on the paged cache at the edges of their forms: workgroups of 256 rows, pages of a whole step with scales far apart or that are no numbers, any
address, more tokens than were announced, tables of thousands of pages, hundreds of sequences that ask for thousands of pages."""
import math

import numpy as np
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


def taken(ix, c):
    return dz.cache(ix, *(c[n] for n in NAMES))


def on_gpu(c):
    return {k: v.to(DEV) for k, v in c.items()}


def batch_of(ix, tables, lengths, new, rows=None, most=None):
    return dz.cache_batch(ix, tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), plain.starts_of(new).to(DEV),
                          n_tokens=sum(new) if rows is None else rows, max_tokens=most or max(new), max_length=max(lengths))


def close(out, lse, want, dtype, keys, D):
    t_out, t_lse = plain.attend_tolerance(*want, dtype, keys, D)
    out, lse = out.cpu().double(), lse.cpu().double()
    assert torch.equal(out.isnan(), want[0].isnan()) and torch.equal(lse.isnan(), want[1].isnan())
    assert torch.equal(torch.isneginf(lse), torch.isneginf(want[1]))
    f, g = torch.isfinite(want[0]), torch.isfinite(want[1])
    assert bool(((out - want[0]).abs()[f] <= t_out[f]).all()), float(((out - want[0]).abs() / t_out)[f].max())
    assert bool(((lse - want[1]).abs()[g] <= t_lse[g]).all()), float(((lse - want[1]).abs() / t_lse)[g].max())


def check(ix, c, tables, lengths, new, heads, dtype, window=0, seed=0, q=None):
    D = c["k"].shape[3]
    if q is None:
        q = torch.randn(sum(new), heads, D, generator=torch.Generator().manual_seed(seed)).to(dtype)
    want = plain.attend(c, tables, lengths, new, q, D ** -0.5, window)
    g = on_gpu(c)
    out, lse = dz.cache_attention(ix, taken(ix, g), batch_of(ix, tables, lengths, new), q.to(DEV), window=window)
    close(out, lse, want, dtype, max(lengths), D)


@pytest.mark.parametrize("dim", [128, 160, 192])
@pytest.mark.parametrize("page", [32, 64])
@pytest.mark.parametrize("window", [0, 45])
def test_workgroups_of_256_rows(ix, dim, page, window):
    """16 sequences x 16 heads with more than 64 rows each; pages missing, sequences without new tokens."""
    n, H, G = 16, 16, 4
    lengths = [20 + 13 * b for b in range(n)]
    new = [17 + b % 4 for b in range(n)]
    new[5] = 0
    pages = sum(-(-m // page) for m in lengths)
    c = plain.make_cache(pages, H, page, dim, dim)
    tables = plain.make_tables(lengths, page, pages, 2)
    tables[9, 0] = -1
    check(ix, c, tables, lengths, new, H * G, torch.float16 if page == 32 else torch.bfloat16, window=window)


@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("page", [64, 128])
def test_a_step_on_one_page_with_any_scale(ix, new, page):
    lengths = [700, 333]
    pages = 32
    c = plain.make_cache(pages, 1, page, 64, 8)
    c["vs"] *= torch.exp2(torch.randint(-45, 45, c["vs"].shape, generator=torch.Generator().manual_seed(1)).float())
    tables = plain.make_tables(lengths, page, pages, 8)
    c["vs"][tables[0, 1]] = 0
    c["ks"][tables[1, 1]] = 0
    check(ix, c, tables, lengths, [new] * 2, 2, torch.bfloat16)
    check(ix, c, tables, lengths, [new] * 2, 2, torch.bfloat16, window=150)
    # scales that are no numbers where no row sees them: before all windows
    for bad in (math.nan, math.inf):
        d = {k: v.clone() for k, v in c.items()}
        d["vs"][:] = c["vs"].clamp(1e-3, 1.0)
        d["vs"][tables[0, 0]], d["ks"][tables[1, 0]] = bad, bad
        check(ix, d, tables, lengths, [new] * 2, 2, torch.float16, window=80)
    # and on the last page, which the earlier of many rows do not see
    if new > 1:
        last = (lengths[0] - 1) // page
        first_hit = new - (lengths[0] - last * page)
        for name in ("ks", "vs"):
            d = {k: v.clone() for k, v in c.items()}
            d["vs"][:] = c["vs"].clamp(1e-3, 1.0)
            good = plain.attend(d, tables, lengths, [new] * 2, torch.ones(2 * new, 2, 64), 0.125)
            d[name][tables[0, last]] = math.nan
            g = on_gpu(d)
            out, lse = dz.cache_attention(ix, taken(ix, g), batch_of(ix, tables, lengths, [new] * 2), torch.ones(2 * new, 2, 64, dtype=torch.float16, device=DEV))
            hit = torch.zeros(2 * new, dtype=torch.bool)
            hit[first_hit:new] = True
            out = out.cpu().double()
            assert out[hit].isnan().all() and not out[~hit].isnan().any()
            close(out[~hit], lse[~hit.to(DEV)], tuple(x[~hit] for x in good), torch.float16, 700, 64)


@pytest.mark.parametrize("new", [1, 40])
def test_tokens_at_any_address(ix, new):
    """Queries, keys, values and outputs that begin at odd elements, tokens apart by odd strides."""
    page, H, G, D, lengths = 16, 2, 2, 96, [100, 77]
    c = plain.make_cache(16, H, page, D, 3)
    tables = plain.make_tables(lengths, page, 16, 3)
    gc = on_gpu(c)
    n = 2 * new
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        heads = G * H + 2 * H
        flat = torch.randn(n * (heads * D + 5) + 3, generator=torch.Generator().manual_seed(4)).to(dtype)
        x = flat[3:].view(n, heads * D + 5)[:, :heads * D].view(n, heads, D)
        gx = flat.to(DEV)[3:].view(n, heads * D + 5)[:, :heads * D].view(n, heads, D)
        assert gx.data_ptr() % 4 == (2 if dtype != torch.float32 else 0) and gx.stride(0) % 2 == 1
        plain.append(c, tables, lengths, [new] * 2, x[:, :H], x[:, H:2 * H])
        b = batch_of(ix, tables, lengths, [new] * 2)
        dz.cache_append(ix, taken(ix, gc), b, gx[:, :H], gx[:, H:2 * H])
        for name in NAMES:
            assert torch.equal(gc[name].cpu(), c[name]), name
        if dtype == torch.float32:
            continue
        room = torch.empty(n * G * H * D + 1, dtype=dtype, device=DEV)
        out, lse = dz.cache_attention(ix, taken(ix, gc), b, gx[:, 2 * H:], 0.1, out=room[1:].view(n, G * H, D))
        close(out, lse, plain.attend(c, tables, lengths, [new] * 2, x[:, 2 * H:], 0.1), dtype, 100, D)


def test_more_new_tokens_than_announced(ix):
    """The first max_tokens of a sequence keep their positions; what is behind them is neither written nor attended for."""
    page, H, D, lengths, new, most = 16, 1, 64, [60, 33], [30, 9], 12
    c = plain.make_cache(12, H, page, D, 3)
    tables = plain.make_tables(lengths, page, 12, 3)
    gc = on_gpu(c)
    x = torch.randn(39, 3, D, generator=torch.Generator().manual_seed(4)).to(torch.float16)
    b = batch_of(ix, tables, lengths, new, most=most)
    kept = list(range(12)) + list(range(30, 39))
    dz.cache_append(ix, taken(ix, gc), b, x.to(DEV)[:, :1], x.to(DEV)[:, 1:2])
    plain.append(c, tables, [42, 33], [12, 9], x[kept, :1], x[kept, 1:2])
    for name in NAMES:
        assert torch.equal(gc[name].cpu(), c[name]), name
    out, lse = torch.full((39, 1, D), 7.0, dtype=torch.float16, device=DEV), torch.full((39, 1), 7.0, device=DEV)
    dz.cache_attention(ix, taken(ix, gc), b, x.to(DEV)[:, 2:], 0.125, out=out, out_lse=lse)
    want = plain.attend(c, tables, [42, 33], [12, 9], x[kept, 2:], 0.125)
    close(out[kept], lse[kept], want, torch.float16, 60, D)
    assert bool((out[12:30] == 7).all()) and bool((lse[12:30] == 7).all())


@pytest.mark.parametrize("places", [600, 2048, 2500, 16384, 17001])
def test_select_from_many_pages(ix, places):
    page, H = 16, 1
    lengths = [places * page, places * page // 3]
    c = plain.make_cache(64, H, page, 32, places)
    g = torch.Generator().manual_seed(places)
    c["ks"] = torch.rand(64, H, generator=g).clamp_min(0.1)
    tables = torch.randint(0, 64, (2, places), generator=g, dtype=torch.int32)     # pages may stand in several places
    tables[0, 5] = -1
    codes, scales = torch.randint(-127, 128, (2 * 3, 32), generator=g, dtype=torch.int8), torch.rand(6, generator=g)
    gc = on_gpu(c)
    b = batch_of(ix, tables, lengths, [1, 1])
    for n_select, first, last in ((1, 0, 0), (37, 0, 0), (37, 4, 4), (places - 2, 1, 1), (places + 3, 0, 2)):
        want = plain.select(c, tables, lengths, [1, 1], codes, scales, n_select, first, last)
        got = dz.cache_select(ix, taken(ix, gc), b, codes.to(DEV), scales.to(DEV), n_select, first, last)
        assert np.array_equal(got.cpu().numpy(), want), n_select


@pytest.mark.parametrize("n,width,most", [(600, 12, 110), (1024, 3, 20), (40, 60, 500), (1, 300, 4000)])
def test_advance_that_asks_for_many_pages(ix, n, width, most):
    page = 16
    g = np.random.default_rng(n)
    lengths = [int(x) for x in g.integers(1, 30, n)]
    for part in (1.0, 0.4):
        add = [int(x) for x in g.integers(0, most, n)]
        pages = sum(-(-m // page) for m in lengths) + int(part * sum(-(-a // page) for a in add)) + 5
        c = plain.make_cache(pages, 1, page, 32, 1, layers=1)
        tables = plain.make_tables(lengths, page, pages, 2, width=width)
        parents = [int(x) for x in g.integers(0, n, n)]
        for p in (None, parents):
            d = {k: v.clone() for k, v in c.items()}
            refs = torch.zeros(pages, dtype=torch.int32)
            refs[tables[tables >= 0].long()] = 1
            gc, g_refs = on_gpu(d), refs.to(DEV)
            got = dz.cache_advance(ix, dz.cache(ix, *(gc[k][0] for k in NAMES)), g_refs, tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV),
                                   torch.tensor(add, dtype=torch.int32, device=DEV), parents=None if p is None else torch.tensor(p, dtype=torch.int32, device=DEV))
            t, l, status = plain.advance(d, refs, tables, lengths, add, p)
            assert torch.equal(got[0].cpu(), t) and torch.equal(got[1].cpu(), l) and got[2].tolist() == status
            assert torch.equal(g_refs.cpu(), refs)
            for name in NAMES:
                assert torch.equal(gc[name].cpu(), d[name]), name


@pytest.mark.parametrize("told", [1, 700, 100000])
@pytest.mark.parametrize("new", [1, 12, 80])
def test_whatever_length_is_told(ix, told, new):
    """max_length divides the work; sequences may be longer or shorter."""
    lengths, page = [3000, 90, 1500], 32
    pages = sum(-(-m // page) for m in lengths)
    c = plain.make_cache(pages, 1, page, 64, 4)
    tables = plain.make_tables(lengths, page, pages, 4)
    q = torch.randn(3 * new, 2, 64, generator=torch.Generator().manual_seed(4)).to(torch.float16)
    g = on_gpu(c)
    b = dz.cache_batch(ix, tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), plain.starts_of([new] * 3).to(DEV), n_tokens=3 * new,
                       max_tokens=new, max_length=told)
    out, lse = dz.cache_attention(ix, taken(ix, g), b, q.to(DEV))
    close(out, lse, plain.attend(c, tables, lengths, [new] * 3, q, 0.125), torch.float16, 3000, 64)
    # a workspace for more serves this call
    more = dz.cache_batch(ix, tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), plain.starts_of([new] * 3).to(DEV), n_tokens=3 * new + 50,
                          max_tokens=new + 50, max_length=told + 1000)
    room = torch.empty(dz.cache_attention_workspace_bytes(ix, taken(ix, g), more, 2), dtype=torch.uint8, device=DEV)
    again = dz.cache_attention(ix, taken(ix, g), b, q.to(DEV), workspace=room)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("scale", [0.125, -0.07, 0.0])
def test_many_queries_of_every_size(ix, dtype, page, scale):
    """More than 64 rows a head: large and small rows, rows of zeros, infinities and NaN, scales of either sign."""
    lengths, new = [100, 164], [90, 77]
    pages = sum(-(-m // page) for m in lengths)
    c = plain.make_cache(pages, 2, page, 64, 4)
    tables = plain.make_tables(lengths, page, pages, 4)
    q = torch.randn(167, 4, 64, generator=torch.Generator().manual_seed(4))
    q[:, 0] *= 60.0
    q[:, 1] *= 1e-30 if dtype == torch.bfloat16 else 1e-4
    q[0, 2] = 0
    q[-1, 3, 5] = math.inf
    q[0, 3, 5] = math.nan
    q = q.to(dtype)
    g = on_gpu(c)
    for window in (0, 20):
        out, lse = dz.cache_attention(ix, taken(ix, g), batch_of(ix, tables, lengths, new), q.to(DEV), scale, window=window)
        close(out, lse, plain.attend(c, tables, lengths, new, q, scale, window), dtype, 164, 64)
    if dtype == torch.bfloat16 and scale:
        big = (q.float().nan_to_num(0, 0, 0) * 1e30).to(dtype)
        out, lse = dz.cache_attention(ix, taken(ix, g), batch_of(ix, tables, lengths, new), big.to(DEV), scale * 1e-31)
        close(out, lse, plain.attend(c, tables, lengths, new, big, scale * 1e-31), dtype, 164, 64)
