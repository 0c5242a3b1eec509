"""The paged cache's calls together, as a program that generates with beams makes them: prompts taken in, steps of decoding in which beams go on
from one another, pages chosen, compaction; in a graph that is replayed; on a stream of their own; in a cache past 32-bit offsets."""
import math

import numpy as np
import pytest
import torch

import paper_2210_15748_amd as dz

import cache_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAMES = ("k", "v", "ks", "vs", "bounds")


def close(out, lse, want, dtype, keys, D):
    t_out, t_lse = plain.attend_tolerance(*want, dtype, keys, D)
    assert bool(((out.cpu().double() - want[0]).abs() <= t_out).all())
    assert bool(((lse.cpu().double() - want[1]).abs() <= t_lse).all())


def same(got, want):
    for name in NAMES:
        assert torch.equal(got[name].cpu(), want[name]), name


def layer(c, i):
    return {n: c[n][i] for n in NAMES}


@pytest.mark.parametrize("page,dtype", [(16, torch.float16), (64, torch.bfloat16)])
def test_prompts_then_steps_of_beams_then_compaction(page, dtype):
    ix = dz.create(128, 32, 7, seed=1)
    L, H, G, D, pages, width = 2, 2, 3, 64, 90 if page == 16 else 40, 24 if page == 16 else 8
    g = torch.Generator().manual_seed(page)
    c = plain.make_cache(pages, H, page, D, 1, layers=L)
    gc = {n: c[n].to(DEV) for n in NAMES}
    caches = [dz.cache(ix, *(gc[n][i] for n in NAMES)) for i in range(L)]
    refs, tables, lengths = torch.zeros(pages, dtype=torch.int32), torch.full((2, width), -1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    g_refs, g_tables, g_lengths = refs.to(DEV), tables.to(DEV), lengths.to(DEV)
    new = [70, 37]
    parents, add = [-1, -1], new
    for step in range(9):
        got = dz.cache_advance(ix, caches, g_refs, g_tables, g_lengths, torch.tensor(add, dtype=torch.int32, device=DEV),
                               parents=torch.tensor(parents, dtype=torch.int32, device=DEV))
        tables, lengths, status = plain.advance(c, refs, tables, lengths, add, parents)
        g_tables, g_lengths = got[0], got[1]
        assert torch.equal(g_tables.cpu(), tables) and torch.equal(g_lengths.cpu(), lengths) and got[2].tolist() == status and status[1] == 0
        n = sum(add)
        b = dz.cache_batch(ix, g_tables, g_lengths, plain.starts_of(add).to(DEV) if step == 0 else None, n_tokens=n, max_tokens=max(add), max_length=200)
        for i in range(L):
            x = torch.randn(n, H * (G + 2), D, generator=g).to(dtype)
            gx = x.to(DEV)
            q, k, v = x[:, :H * G], x[:, H * G:H * (G + 1)], x[:, H * (G + 1):]
            plain.append(layer(c, i), tables, lengths.tolist(), add, k, v)
            dz.cache_append(ix, caches[i], b, gx[:, H * G:H * (G + 1)], gx[:, H * (G + 1):])
            out, lse = dz.cache_attention(ix, caches[i], b, gx[:, :H * G], 0.125)
            close(out, lse, plain.attend(layer(c, i), tables, lengths.tolist(), add, q, 0.125), dtype, 200, D)
            codes, scales = dz.quantize_rows(ix, gx[:, :H * G].reshape(-1, D))
            ids = dz.cache_select(ix, caches[i], b, codes, scales, 3, n_first=1, n_last=1)
            want_ids = plain.select(layer(c, i), tables, lengths.tolist(), add, codes.cpu(), scales.cpu(), 3, 1, 1)
            assert np.array_equal(ids.cpu().numpy(), want_ids)
            out, lse = dz.cache_attention(ix, caches[i], b, gx[:, :H * G], 0.125, pages=ids)
            close(out, lse, plain.attend(layer(c, i), tables, lengths.tolist(), add, q, 0.125, pages=torch.from_numpy(want_ids.astype(np.int64))),
                  dtype, 200, D)
        same(gc, c)
        beams = len(add)
        parents = [0, 0, 1, 1] if step == 0 else [int(p) for p in torch.randint(0, beams, (4,), generator=g)]
        add = [1] * 4
        if step == 5:
            numbers, live = dz.cache_compact(ix, caches, g_refs, g_tables, g_lengths)
            want_numbers, n_live = plain.compact(c, refs, tables, lengths)
            assert torch.equal(numbers.cpu(), want_numbers) and live.tolist() == [n_live]
            assert torch.equal(g_tables.cpu(), tables) and torch.equal(g_refs.cpu(), refs)
            same(gc, c)


def step_state(seed):
    """A decoding step's inputs on the GPU, and the same on the CPU."""
    page, H, G, D, n = 16, 2, 4, 64, 6
    lengths = [700 + 40 * b for b in range(n)]
    pages = sum(-(-m // page) for m in lengths) + 2 * n
    c = plain.make_cache(pages, H, page, D, seed, layers=1)
    tables = plain.make_tables(lengths, page, pages, seed, width=70)
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[tables[tables >= 0].long()] = 1
    x = torch.randn(n, H * (G + 2), D, generator=torch.Generator().manual_seed(seed)).to(torch.float16)
    return c, tables, lengths, refs, x, page, H, G, D, n


def run_step(ix, gc, refs, tables, lengths, add, x, outs, ws):
    H, G = 2, 4
    cache = dz.cache(ix, *(gc[n][0] for n in NAMES))
    dz.cache_advance(ix, cache, refs, tables, lengths, add, outs=outs[:3], workspace=ws[0])
    b = dz.cache_batch(ix, outs[0], outs[1], max_length=1000)
    dz.cache_append(ix, cache, b, x[:, H * G:H * (G + 1)], x[:, H * (G + 1):])
    codes, scales = dz.quantize_rows(ix, outs[5].copy_(x[:, :H * G]).view(-1, 64), out=outs[3], out_scales=outs[4])
    ids = dz.cache_select(ix, cache, b, codes, scales, 9, 1, 2, out=outs[6], workspace=ws[1])
    dz.cache_attention(ix, cache, b, x[:, :H * G], 0.125, out=outs[7], out_lse=outs[8], workspace=ws[2])
    dz.cache_attention(ix, cache, b, x[:, :H * G], 0.125, pages=ids, out=outs[9], out_lse=outs[10], workspace=ws[2])


def step_buffers(n, H, G, D, width, pages, ix, seed):
    i32 = dict(dtype=torch.int32, device=DEV)
    outs = [torch.empty(n, width, **i32), torch.empty(n, **i32), torch.empty(2, **i32), torch.empty(n * H * G, D, dtype=torch.int8, device=DEV),
            torch.empty(n * H * G, device=DEV), torch.empty(n, H * G, D, dtype=torch.float16, device=DEV),
            torch.empty(n, H, 9, dtype=torch.uint32, device=DEV), torch.empty(n, H * G, D, dtype=torch.float16, device=DEV),
            torch.empty(n, H * G, device=DEV), torch.empty(n, H * G, D, dtype=torch.float16, device=DEV), torch.empty(n, H * G, device=DEV)]
    ws = [torch.full((1 << 24,), seed, dtype=torch.uint8, device=DEV) for _ in range(3)]
    return outs, ws


def test_a_captured_step_replays_as_it_ran():
    """Two graphs with workspaces of their own, replayed by turns with eager work between, against eager calls on the same inputs."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ix = dz.create(128, 32, 7, seed=1, stream=stream)
        made = []
        for seed in (1, 2):
            c, tables, lengths, refs, x, page, H, G, D, n = step_state(seed)
            src = ({k: v.to(DEV) for k, v in c.items()}, refs.to(DEV), tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV),
                   torch.ones(n, dtype=torch.int32, device=DEV), x.to(DEV))
            outs, ws = step_buffers(n, H, G, D, 70, refs.shape[0], ix, seed)
            gc = {k: v.clone() for k, v in src[0].items()}
            r = src[1].clone()
            run_step(ix, gc, r, *src[2:], outs, ws)
            stream.synchronize()
            eager = [o.clone() for o in outs] + [v.clone() for v in gc.values()] + [r.clone()]
            for k in gc:
                gc[k].copy_(src[0][k])
            r.copy_(src[1])
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                run_step(ix, gc, r, *src[2:], outs, ws)
            # a graph's replay reads and writes all of these: the workspaces have to live as long as it does, too
            made.append((graph, src, gc, r, outs, ws, eager, (c, tables, lengths, refs, x, H, G, D, n)))
        for turn in range(4):
            for graph, src, gc, r, outs, _, eager, _ in made:
                for k in gc:
                    gc[k].copy_(src[0][k])
                r.copy_(src[1])
                for o in outs:
                    o.view(torch.uint8).fill_(turn)
                graph.replay()
                stream.synchronize()
                for a, b in zip(outs + list(gc.values()) + [r], eager):
                    assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), turn
                (torch.randn(1000, 1000, device=DEV) @ torch.randn(1000, 1000, device=DEV)).sum().item()
    # and what they give is right
    _, _, _, _, outs, _, _, (c, tables, lengths, refs, x, H, G, D, n) = made[1]
    t, l, _ = plain.advance(c, refs, tables, lengths, [1] * n, None)
    plain.append(layer(c, 0), t, l.tolist(), [1] * n, x[:, H * G:H * (G + 1)], x[:, H * (G + 1):])
    close(outs[7], outs[8], plain.attend(layer(c, 0), t, l.tolist(), [1] * n, x[:, :H * G], 0.125), torch.float16, 1000, D)


def test_calls_on_a_stream_of_their_own_keep_what_they_convert():
    """Inputs in another layout are copied by the binding on the caller's stream; the calls run on the index's."""
    stream = torch.cuda.Stream()
    ix = dz.create(128, 32, 7, seed=1, stream=stream)
    c, tables, lengths, refs, x, page, H, G, D, n = step_state(3)
    gc = {k: v.to(DEV) for k, v in c.items()}
    gt, gl = tables.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV)
    q = x[:, :H * G]
    torch.cuda.synchronize()
    cache, b = dz.cache(ix, *(gc[k][0] for k in NAMES)), dz.cache_batch(ix, gt, gl, max_length=1000)
    for _ in range(5):
        turned = q.to(DEV).permute(2, 0, 1).contiguous().permute(1, 2, 0)      # a channel's tokens side by side
        out, lse = dz.cache_attention(ix, cache, b, turned, 0.125)
        del turned
        junk = [torch.full((n, H * G, D), 9.0, dtype=torch.float16, device=DEV) for _ in range(20)]
    torch.cuda.synchronize()
    assert len(junk) == 20
    close(out, lse, plain.attend(layer(c, 0), tables, lengths, [1] * n, q, 0.125), torch.float16, 1000, D)


def test_a_cache_past_32_bit_offsets():
    """Pages whose codes lie 2^32 bytes and more into the pool: written, read, chosen, copied and moved."""
    ix = dz.create(128, 32, 7, seed=1)
    page, H, D = 256, 8, 256
    pages = (1 << 33) // (page * H * D) // 2 + 40        # 4 GiB and some of keys
    torch.cuda.empty_cache()
    big = dict(k=torch.zeros(pages, H, page, D, dtype=torch.int8, device=DEV), v=torch.zeros(pages, H, D, page, dtype=torch.int8, device=DEV),
               ks=torch.zeros(pages, H, device=DEV), vs=torch.zeros(pages, H, device=DEV), bounds=torch.zeros(pages, H, 2, D, dtype=torch.int8, device=DEV))
    assert big["k"].numel() > 1 << 32
    last = pages - 1
    order = [last, 3, last - 7]
    tables = torch.tensor([order + [-1]], dtype=torch.int32)
    small = plain.make_cache(4, H, page, D, 1)           # pages 0, 1, 2 stand for those
    st = torch.tensor([[0, 1, 2, -1]], dtype=torch.int32)
    for s, p in enumerate(order):
        for n in NAMES:
            big[n][p] = small[n][s].to(DEV)
    cache = dz.cache(ix, *(big[n] for n in NAMES))
    gt = tables.to(DEV)
    x = torch.randn(5, 3 * H, D, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    b = dz.cache_batch(ix, gt, torch.tensor([700], dtype=torch.int32, device=DEV), plain.starts_of([5]).to(DEV), n_tokens=5, max_tokens=5, max_length=700)
    gx = x.to(DEV)
    dz.cache_append(ix, cache, b, gx[:, H:2 * H], gx[:, 2 * H:])
    plain.append(small, st, [700], [5], x[:, H:2 * H], x[:, 2 * H:])
    out, lse = dz.cache_attention(ix, cache, b, gx[:, :H], 0.0625)
    close(out, lse, plain.attend(small, st, [700], [5], x[:, :H], 0.0625), torch.bfloat16, 700, D)
    many = torch.randn(200, H, D, generator=torch.Generator().manual_seed(6)).to(torch.float16)
    mb = dz.cache_batch(ix, gt, torch.tensor([700], dtype=torch.int32, device=DEV), plain.starts_of([200]).to(DEV), n_tokens=200, max_tokens=200, max_length=700)
    out, lse = dz.cache_attention(ix, cache, mb, many.to(DEV), 0.0625)
    close(out, lse, plain.attend(small, st, [700], [200], many, 0.0625), torch.float16, 700, D)
    codes = torch.randint(-127, 128, (5 * H, D), generator=torch.Generator().manual_seed(7), dtype=torch.int8)
    scales = torch.rand(5 * H, generator=torch.Generator().manual_seed(8))
    ids = dz.cache_select(ix, cache, b, codes.to(DEV), scales.to(DEV), 1)
    assert np.array_equal(ids.cpu().numpy(), plain.select(small, st, [700], [5], codes, scales, 1, 0, 0))
    refs = torch.ones(pages, dtype=torch.int32, device=DEV)
    refs[[1, last - 2]] = 0
    refs[last - 7] = 2
    t, l, status = dz.cache_advance(ix, cache, refs, gt, torch.tensor([700], dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV))
    assert t.tolist() == [[last, 3, 1, -1]] and l.tolist() == [701] and status.tolist() == [1, 0]
    for n in NAMES:
        assert torch.equal(big[n][1], big[n][last - 7])
    moved = {n: big[n][last].clone() for n in NAMES}
    refs.fill_(0)
    refs[[1, 3, last]] = 1
    numbers, live = dz.cache_compact(ix, cache, refs, t, l)
    assert live.tolist() == [3] and t.tolist() == [[2, 0, 1, -1]] or t.tolist() == [[0, 2, 1, -1]]
    for n in NAMES:
        assert torch.equal(big[n][int(numbers[last].item())], moved[n])
