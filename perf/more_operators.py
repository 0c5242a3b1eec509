"""The operators on a paged int8 cache, as measurable cases: what a language model that reads found documents keeps of their tokens.

  append   new tokens' keys and values into the pages: int8 codes with one scale for each page and head, and the keys' bounds
  attend   attention of new tokens over the cache, one token a sequence (decoding) or many (a prompt)
  sparse   one token over a few pages: its int8 codes, the pages that their bounds score highest, attention over those
  advance  sequences go on from parents (beams, forks, ended ones) with room for new tokens: pages shared, copied, taken, freed
  compact  the pages in use moved to the front of the pool

The cache of one layer: k codes [pages][kv heads][page tokens][dim], v codes [pages][kv heads][dim][page tokens], scales
[pages][kv heads], bounds [pages][kv heads][2][dim] (smallest and largest k code of a page).  A sequence's page numbers are a row of
`tables`, its length counts the new tokens.  Codes are whole numbers by definition (an exact rounding), and returned as such.

`own` chooses between the plain form, in elementary torch operations, and the library's entry points.
"""
import math

import torch

own = False

NONE = -1            # as uint32 the library's empty value: no page, no parent
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
INV127 = 1.0 / 127.0


# ---- the cases ----------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decoded token of each of 8 sequences: the smallest call, all latency
        dict(name="append_step", kind="append", seqs=8, new=1, max_len=900, kv=8, dim=128, page=64, dtype="f16"),
        # a few long documents read in, two of them on from where an earlier chunk ended
        dict(name="append_prompt", kind="append", seqs=4, new=6000, max_len=6500, kv=8, dim=128, page=16, dtype="bf16"),
        # a few short sequences being decoded: latency
        dict(name="attend_step", kind="attend", seqs=4, new=1, max_len=500, kv=8, group=4, dim=64, page=16, dtype="f16", window=0),
        # the decoding step of a busy server: ragged lengths, small pages
        dict(name="attend_batch", kind="attend", seqs=64, new=1, max_len=4096, kv=8, group=4, dim=128, page=16, dtype="bf16", window=0),
        # one answer from a long context: few rows, a long axis
        dict(name="attend_long", kind="attend", seqs=1, new=1, max_len=131072, kv=8, group=4, dim=128, page=64, dtype="f16", window=0),
        # a few drafted tokens at once, every head with keys of its own, a width that is no power of two, a window
        dict(name="attend_odd", kind="attend", seqs=7, new=5, max_len=3001, kv=12, group=1, dim=96, page=32, dtype="f16", window=1000),
        # a chunk of two prompts over what has been read: the matrix cores' rate
        dict(name="attend_prompt", kind="attend", seqs=2, new=2048, max_len=8192, kv=8, group=4, dim=128, page=64, dtype="bf16", window=0),
        # one answer from a long context, a thirtieth of it looked at
        dict(name="sparse_long", kind="sparse", seqs=1, max_len=131072, kv=8, group=4, dim=128, page=64, dtype="f16", n_select=64),
        # a batch over middling contexts, small pages
        dict(name="sparse_batch", kind="sparse", seqs=32, max_len=16384, kv=4, group=8, dim=128, page=32, dtype="bf16", n_select=48),
        # room for one more token of a few sequences
        dict(name="advance_step", kind="advance", prompts=16, beams=1, max_len=700, kv=8, dim=64, page=16, layers=2, tight=False),
        # a step of 32 beam searches: pages shared with the parents, the last ones copied, ended beams' freed
        dict(name="advance_beams", kind="advance", prompts=32, beams=4, max_len=2000, kv=8, dim=128, page=64, layers=4, tight=False),
        # a pool two thirds empty brought together
        dict(name="compact_pool", kind="compact", seqs=24, max_len=2048, kv=8, dim=128, page=64, layers=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "sparse", "advance", "compact"])
    kv, dim, page = rng.choice([1, 2, 4, 8, 12]), rng.choice([32, 64, 96, 128, 128, 160, 256]), rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["f16", "bf16"])
    if kind == "append":
        new, seqs = (1, _log(rng, 1, 64)) if rng.random() < 0.5 else (_log(rng, 2, 6000), _log(rng, 1, 8))
        while seqs * new * kv * dim > 24000 * 1024:
            new = new * 2 // 3
        return dict(kind=kind, seqs=seqs, new=new, max_len=new + _log(rng, 1, 1000), kv=kv, dim=dim, page=page, dtype=rng.choice(list(DTYPES)))
    if kind == "attend":
        group, seqs = rng.choice([1, 2, 3, 4, 8, 16]), _log(rng, 1, 64)
        new = rng.choice([1, 1, 1, rng.randint(2, 16), _log(rng, 17, 2048)])
        max_len = max(new, _log(rng, 1, 131072))
        while seqs > 1 and seqs * max_len * kv * dim > 131072 * 1024:
            seqs = seqs * 2 // 3
        while max_len > new and seqs * max_len * kv * max(dim, group * new) > 131072 * 1024:
            max_len = max(new, max_len * 2 // 3)
        while seqs * max_len * kv * group * new > 131072 * 1024:
            new = max(1, new * 2 // 3)
        return dict(kind=kind, seqs=seqs, new=new, max_len=max_len, kv=kv, group=group, dim=dim, page=page, dtype=dtype,
                    window=rng.choice([0, 0, 0, _log(rng, 1, 4096)]))
    if kind == "sparse":
        group, seqs, max_len = rng.choice([1, 2, 4, 8, 16]), _log(rng, 1, 64), _log(rng, 100, 131072)
        while seqs * max_len * kv * dim > 131072 * 1024:
            seqs, max_len = (seqs * 2 // 3, max_len) if seqs > 1 else (1, max_len * 2 // 3)
        return dict(kind=kind, seqs=seqs, max_len=max_len, kv=kv, group=group, dim=dim, page=page, dtype=dtype, n_select=_log(rng, 4, 128))
    if kind == "advance":
        prompts, beams, max_len = _log(rng, 1, 64), rng.choice([1, 2, 4, 5]), _log(rng, 20, 4000)
        while prompts > 1 and prompts * beams * max_len * kv * dim > 65536 * 1024:
            prompts = prompts * 2 // 3
        while prompts * beams * max_len * kv * dim > 65536 * 1024:
            max_len = max_len * 2 // 3
        return dict(kind=kind, prompts=prompts, beams=beams, max_len=max_len, kv=kv, dim=dim, page=page, layers=rng.randint(1, 3),
                    tight=rng.random() < 0.3)
    seqs, max_len = _log(rng, 1, 64), _log(rng, 20, 8192)
    while seqs * max_len * kv * dim > 32768 * 1024:
        seqs, max_len = (seqs * 2 // 3, max_len) if seqs > 1 else (1, max_len * 2 // 3)
    return dict(kind=kind, seqs=seqs, max_len=max_len, kv=kv, dim=dim, page=page, layers=rng.randint(1, 3))


def _lengths(case):
    """Lengths of the sequences, and how many tokens of each are new: unequal, and odd for the most part."""
    n, top = case["seqs"], case["max_len"]
    new = [max(1, case.get("new", 1) - b * case.get("new", 1) // (2 * n)) for b in range(n)]
    return [max(new[b], top - b * (3 * top // (4 * n))) for b in range(n)], new


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _dev():
    return torch.device("cuda", torch.cuda.current_device())


def _generator(seed):
    g = torch.Generator(device=_dev())
    g.manual_seed(seed)
    return g


def _tables(used, pool, g):
    """Page numbers in no order: [sequences][most pages] int32, NONE behind a sequence's last."""
    dev = _dev()
    used = torch.tensor(used, device=dev)
    numbers = torch.randperm(pool, generator=g, device=dev).to(torch.int32)
    at = torch.arange(int(used.max()), device=dev)
    first = used.cumsum(0) - used
    place = first[:, None] + at
    return torch.where(at < used[:, None], numbers[place.clamp_max(pool - 1)], NONE).contiguous()


def _codes(x, dims):
    """int8 codes with one scale for each of what is left when `dims` are taken together"""
    s = x.abs().amax(dim=dims, keepdim=True) * INV127
    return (x / s).round_().clamp_(-127, 127).to(torch.int8), s


def _filled(case, pages, g):
    """A pool whose pages hold tokens that are alike: a direction for each page and head beside the noise, some channels large."""
    dev, H, T, D = _dev(), case["kv"], case["page"], case["dim"]
    k = torch.empty(pages, H, T, D, dtype=torch.int8, device=dev)
    v = torch.empty(pages, H, D, T, dtype=torch.int8, device=dev)
    ks, vs = torch.empty(pages, H, device=dev), torch.empty(pages, H, device=dev)
    wide = torch.exp(0.5 * torch.randn(H, 1, D, generator=g, device=dev))
    step = max(1, (1 << 26) // (H * T * D))
    for lo in range(0, pages, step):
        n = min(step, pages - lo)
        x = torch.randn(n, H, 1, D, generator=g, device=dev) * 0.7 + torch.randn(n, H, T, D, generator=g, device=dev)
        c, s = _codes(x * wide, (2, 3))
        k[lo:lo + n], ks[lo:lo + n] = c, s[:, :, 0, 0]
        c, s = _codes(torch.randn(n, H, D, T, generator=g, device=dev), (2, 3))
        v[lo:lo + n], vs[lo:lo + n] = c, s[:, :, 0, 0]
    return dict(k=k, v=v, ks=ks, vs=vs)


def _states(case, n, g):
    """q, k, v of n tokens, as one product of a layer leaves them: side by side in rows; a few rows larger than the others."""
    dev, D = _dev(), case["dim"]
    heads = case["kv"] * (case.get("group", 1) + 2)
    x = torch.randn(n, heads * D, generator=g, device=dev) * torch.exp(0.3 * torch.randn(n, 1, generator=g, device=dev))
    x = x.to(DTYPES[case["dtype"]]).view(n, heads, D)
    at = heads - 2 * case["kv"]
    return x[:, :at], x[:, at:at + case["kv"]], x[:, at + case["kv"]:]


def _inputs(case, seed):
    dev, g, kind = _dev(), _generator(seed), case["kind"]
    T, H, D = case["page"], case["kv"], case["dim"]
    if kind in ("append", "attend", "sparse"):
        lengths, new = _lengths(case)
        used = [-(-n // T) for n in lengths]
        pool = sum(used) + 3
        s = dict(tables=_tables(used, pool, g), lengths=torch.tensor(lengths, dtype=torch.int32, device=dev), n_tokens=sum(new), max_new=max(new),
                 starts=torch.tensor([0] + new, dtype=torch.int32, device=dev).cumsum(0).to(torch.int32))
        s["q"], s["new_k"], s["new_v"] = _states(case, s["n_tokens"], g)
        s |= _filled(case, pool, g)
        if kind != "attend":
            s["bounds"] = torch.stack([s["k"].amin(dim=2), s["k"].amax(dim=2)], dim=2)
        return s
    layers = case["layers"]
    if kind == "advance":
        # beams of a prompt share its pages and have the later ones to themselves; the next ones go on from some of them
        P, B = case["prompts"], case["beams"]
        n = P * B
        lengths = [max(2, case["max_len"] - i * (case["max_len"] // (2 * P))) for i in range(P) for _ in range(B)]
        used = [-(-m // T) for m in lengths]
        pool = sum(used) + 2 * n + 3
        tables = torch.nn.functional.pad(_tables(used, pool, g), (0, 1), value=NONE)
        shared = torch.tensor([m // (2 * T) for m in lengths], device=dev)
        first = torch.arange(n, device=dev) // B * B
        at = torch.arange(tables.shape[1], device=dev)
        tables = torch.where(at < shared[:, None], tables[first], tables).contiguous()
        parents = first + torch.randint(0, B, (n,), generator=g, device=dev)
        ended = (torch.rand(n, generator=g, device=dev) < 0.05) & (torch.arange(n, device=dev) > 0)
        parents = torch.where(ended, NONE, parents).to(torch.int32)
        s = dict(tables=tables, lengths=torch.tensor(lengths, dtype=torch.int32, device=dev), parents=parents if B > 1 else None,
                 add=torch.where(ended, 0, 1).to(torch.int32) if B > 1 else torch.ones(n, dtype=torch.int32, device=dev))
    else:
        lengths, _ = _lengths(case)
        used = [-(-m // T) for m in lengths]
        pool = 3 * sum(used) + 1
        s = dict(tables=_tables(used, pool, g), lengths=torch.tensor(lengths, dtype=torch.int32, device=dev))
    held = s["tables"][s["tables"] >= 0].long()
    s["refs"] = torch.zeros(pool, dtype=torch.int32, device=dev).index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
    if case.get("tight"):     # most of the other pages are held by somebody else
        empty = s["refs"] == 0
        s["refs"][empty & (empty.cumsum(0) > max(1, n // 6))] = 1
    s["k"] = torch.randint(-127, 128, (layers, pool, H, T, D), generator=g, device=dev, dtype=torch.int8)
    s["v"] = torch.randint(-127, 128, (layers, pool, H, D, T), generator=g, device=dev, dtype=torch.int8)
    s["ks"] = torch.rand(layers, pool, H, generator=g, device=dev)
    s["vs"] = torch.rand(layers, pool, H, generator=g, device=dev)
    s["bounds"] = torch.randint(-127, 128, (layers, pool, H, 2, D), generator=g, device=dev, dtype=torch.int8)
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case, kind=case["kind"], scale=1.0 / math.sqrt(case["dim"]))
    if s["kind"] in ("advance", "compact"):     # what the call changes in place is set back before each pass
        s["held"] = s["refs"].clone(), s["tables"].clone()
    if not own:
        return s
    # what a serving program keeps from call to call: a handle, the cache and the batch as the calls take them, outputs, workspaces
    import paper_2210_15748_amd as dz
    dev = _dev()
    ix = s["ix"] = dz.create(128, 32, 7, seed=1)
    if s["kind"] in ("advance", "compact"):
        s["cache"] = [dz.cache(ix, s["k"][i], s["v"][i], s["ks"][i], s["vs"][i], s["bounds"][i]) for i in range(case["layers"])]
        n, pool = s["lengths"].shape[0], s["refs"].shape[0]
        if s["kind"] == "advance":
            nbytes = dz.cache_advance_workspace_bytes(ix, pool, n)
            s["outs"] = (torch.empty_like(s["tables"]), torch.empty_like(s["lengths"]), torch.empty(2, dtype=torch.int32, device=dev))
        else:
            nbytes = dz.cache_compact_workspace_bytes(ix, pool)
            s["outs"] = (torch.empty(pool, dtype=torch.int32, device=dev), torch.empty(1, dtype=torch.int32, device=dev))
        s["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
        return s
    s["cache"] = dz.cache(ix, s["k"], s["v"], s["ks"], s["vs"], s.get("bounds"))
    s["batch"] = dz.cache_batch(ix, s["tables"], s["lengths"], None if s["max_new"] == 1 else s["starts"], n_tokens=s["n_tokens"],
                                max_tokens=s["max_new"], max_length=case["max_len"])
    if s["kind"] == "append":
        return s
    n, heads = s["q"].shape[:2]
    chosen = case.get("n_select", 0)
    s["out"] = torch.empty(n, heads, case["dim"], dtype=s["q"].dtype, device=dev)
    s["lse"] = torch.empty(n, heads, device=dev)
    nbytes = dz.cache_attention_workspace_bytes(ix, s["cache"], s["batch"], heads, n_select=chosen)
    if chosen:
        s["codes"] = torch.empty(n * heads, case["dim"], dtype=torch.int8, device=dev)
        s["code_scales"] = torch.empty(n * heads, device=dev)
        s["pages"] = torch.empty(n, case["kv"], chosen, dtype=torch.uint32, device=dev)
        nbytes = max(nbytes, dz.cache_select_workspace_bytes(ix, s["cache"], s["batch"]))
    s["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2210_15748_amd as dz
    case, kind, ix = s["case"], s["kind"], s["ix"]
    if kind == "append":
        dz.cache_append(ix, s["cache"], s["batch"], s["new_k"], s["new_v"])
        return s["k"], s["v"], s["ks"], s["vs"], s["bounds"]
    if kind == "attend":
        return dz.cache_attention(ix, s["cache"], s["batch"], s["q"], s["scale"], window=case["window"], out=s["out"], out_lse=s["lse"],
                                  workspace=s["ws"])
    if kind == "sparse":
        n, heads, D = s["q"].shape
        codes, scales = dz.quantize_rows(ix, s["q"].reshape(n * heads, D), out=s["codes"], out_scales=s["code_scales"])
        pages = dz.cache_select(ix, s["cache"], s["batch"], codes, scales, case["n_select"], n_first=1, n_last=2, out=s["pages"], workspace=s["ws"])
        out, lse = dz.cache_attention(ix, s["cache"], s["batch"], s["q"], s["scale"], pages=pages, out=s["out"], out_lse=s["lse"],
                                      workspace=s["ws"])
        return out, lse, pages.view(torch.int32)
    s["refs"].copy_(s["held"][0])
    if kind == "advance":
        out = dz.cache_advance(ix, s["cache"], s["refs"], s["tables"], s["lengths"], s["add"], parents=s["parents"], outs=s["outs"],
                               workspace=s["ws"])
        return *out, s["refs"], s["k"], s["v"], s["ks"], s["vs"], s["bounds"]
    s["tables"].copy_(s["held"][1])
    out = dz.cache_compact(ix, s["cache"], s["refs"], s["tables"], s["lengths"], outs=s["outs"], workspace=s["ws"])
    return *out, s["tables"], s["refs"], s["k"], s["v"], s["ks"], s["vs"], s["bounds"]


def _places(s):
    """For each new token: its sequence, its position."""
    at = torch.arange(s["n_tokens"], device=s["starts"].device)
    seq = torch.searchsorted(s["starts"].long(), at, right=True) - 1
    return seq, s["lengths"].long()[seq] - s["starts"].long()[seq + 1] + at


def _plain_append(s):
    T = s["case"]["page"]
    seq, pos = _places(s)
    tables = s["tables"].long()
    page, slot = tables[seq, pos // T], pos % T
    # pages that a sequence's earlier tokens share with its first new one: [sequences], where there is such a page
    begin = s["lengths"].long() - (s["starts"][1:] - s["starts"][:-1]).long()
    old = tables.gather(1, (begin // T).clamp_max(tables.shape[1] - 1)[:, None])[:, 0]
    partly = begin % T > 0
    old = old[partly]
    fresh = torch.ones(s["k"].shape[0], dtype=torch.bool, device=page.device)
    fresh[old] = False
    touched = torch.zeros_like(fresh)
    touched[page] = True
    starts_new = (touched & fresh)[:, None]
    earlier = (torch.arange(T, device=page.device) < (begin % T)[partly][:, None])[:, None]     # [pages][1][slots]
    for codes, scales, x, keys in ((s["k"], s["ks"], s["new_k"], True), (s["v"], s["vs"], s["new_v"], False)):
        x = x.float()
        before = scales.clone()
        most = torch.zeros_like(scales).scatter_reduce_(0, page[:, None].expand(-1, scales.shape[1]), x.abs().amax(dim=2), "amax")
        scales.copy_(torch.where(touched[:, None], torch.maximum(torch.where(starts_new, 0.0, before), most * INV127), before))
        # codes of tokens that were there, in the new scale
        ratio = [t[old].double()[:, :, None, None] for t in (before, scales)]
        again = lambda c: torch.where(ratio[1] > ratio[0], torch.round(c.double() * ratio[0] / ratio[1]), c.double()).to(torch.int8)  # noqa: E731
        codes[old] = torch.where(earlier[..., None] if keys else earlier[:, :, None], again(codes[old]), codes[old])
        per = scales[page].double()[:, :, None]
        new = torch.round(x.double() / torch.where(per == 0, 1.0, per)).clamp(-127, 127).to(torch.int8)
        if keys:
            s["bounds"][old] = again(s["bounds"][old])
            codes[page, :, slot] = new
            wide = s["bounds"].int()
            wide = torch.where(starts_new[:, :, None, None], torch.tensor([127, -127], device=page.device, dtype=torch.int32)[:, None], wide)
            to = page[:, None, None].expand(new.shape)
            wide[:, :, 0].scatter_reduce_(0, to, new.int(), "amin")
            wide[:, :, 1].scatter_reduce_(0, to, new.int(), "amax")
            s["bounds"].copy_(wide)
        else:
            codes[page, :, :, slot] = new
    return s["k"], s["v"], s["ks"], s["vs"], s["bounds"]


def _softmax(scores, seen):
    """exp(scores - largest), their sums and the logarithm of the whole; rows that see nothing: zeros, -inf."""
    scores = torch.where(seen, scores, -math.inf)
    peak = scores.amax(dim=-1, keepdim=True)
    base = torch.where(peak == -math.inf, 0.0, peak)
    e = (scores - base).exp_()
    total = e.sum(dim=-1, keepdim=True)
    return e, total, (base + total.log())[..., 0]


def _plain_attend(s):
    case = s["case"]
    T, H, D, G, top = case["page"], case["kv"], case["dim"], case["group"], s["max_new"]
    seq, pos = _places(s)
    B, M = s["tables"].shape
    pages = s["tables"].long().clamp_min(0)
    k = (s["k"][pages].float() * s["ks"][pages][..., None, None]).transpose(1, 2).reshape(B, H, M * T, D)
    v = (s["v"][pages].float() * s["vs"][pages][..., None, None]).permute(0, 2, 1, 4, 3).reshape(B, H, M * T, D)
    # rows of a sequence side by side, as many for each
    row = torch.arange(s["n_tokens"], device=seq.device) - s["starts"].long()[seq]
    q = torch.zeros(B, top, H * G, D, device=seq.device)
    q[seq, row] = s["q"].float()
    q = q.view(B, top, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, top * G, D)
    at = torch.zeros(B, top, dtype=torch.long, device=seq.device)
    at[seq, row] = pos
    j = torch.arange(M * T, device=seq.device)
    seen = j <= at[:, :, None]
    if case["window"]:
        seen &= j > at[:, :, None] - case["window"]
    seen = seen[:, None, :, None].expand(B, 1, top, G, M * T).reshape(B, 1, top * G, M * T)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    e, total, lse = _softmax(scores, seen)
    out = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
    out = out.view(B, H, top, G, D).permute(0, 2, 1, 3, 4).reshape(B, top, H * G, D)[seq, row]
    lse = lse.view(B, H, top, G).permute(0, 2, 1, 3).reshape(B, top, H * G)[seq, row]
    return out.to(s["q"].dtype), lse


def _plain_sparse(s):
    case = s["case"]
    T, H, D, G, chosen = case["page"], case["kv"], case["dim"], case["group"], case["n_select"]
    n = s["n_tokens"]
    pos = s["lengths"].long() - 1
    M = s["tables"].shape[1]
    pages = s["tables"].long().clamp_min(0)
    q = s["q"].float()
    # the score of a page: what its keys can come to at most, in whole numbers, the largest over the heads that share it
    q_scale = q.abs().amax(dim=2) * INV127
    codes = torch.round(q.double() / torch.where(q_scale == 0, 1.0, q_scale).double()[..., None]).float().view(n, H, G, D)
    bounds = s["bounds"][pages].float().permute(0, 2, 3, 4, 1)      # [n][H][2][D][M]
    sums = torch.matmul(codes.clamp_min(0), bounds[:, :, 1].contiguous()) + torch.matmul(codes.clamp_max(0), bounds[:, :, 0].contiguous())
    score = (sums * (q_scale.view(n, H, G, 1) * s["ks"][pages].transpose(1, 2)[:, :, None])).amax(dim=2)
    j, last = torch.arange(M, device=pos.device), (pos // T)[:, None]
    score = torch.where(((j < 1) | (j > last - 2))[:, None], math.inf, score)
    score = torch.where((j <= last)[:, None], score, -math.inf)
    best = torch.sort(score, dim=2, descending=True, stable=True)
    ids = torch.where(best.values == -math.inf, M, best.indices)[:, :, :chosen].sort(dim=2).values
    ids = torch.cat([ids, ids.new_full((n, H, max(0, chosen - M)), M)], dim=2)
    # attention over those
    there = ids < M
    number = pages.gather(1, ids.clamp_max(M - 1).view(n, -1)).view(n, H, chosen)
    head = torch.arange(H, device=pos.device)[None, :, None]
    k = (s["k"][number, head].float() * s["ks"][number, head][..., None, None]).view(n, H, chosen * T, D)
    v = (s["v"][number, head].float() * s["vs"][number, head][..., None, None]).transpose(3, 4).reshape(n, H, chosen * T, D)
    at = ids[..., None] * T + torch.arange(T, device=pos.device)
    seen = (there[..., None] & (at <= pos[:, None, None, None])).view(n, H, 1, chosen * T)
    scores = torch.matmul(q.view(n, H, G, D), k.transpose(2, 3).contiguous()) * s["scale"]
    e, total, lse = _softmax(scores, seen)
    out = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
    return out.view(n, H * G, D).to(s["q"].dtype), lse.view(n, H * G), torch.where(there, ids, NONE).to(torch.int32)


def _plain_advance(s):
    T, refs, tables = s["case"]["page"], s["refs"], s["tables"].long()
    stride = tables.shape[1]
    refs.copy_(s["held"][0])
    lengths, add, j = s["lengths"].long(), s["add"].long(), torch.arange(stride, device=refs.device)
    parent = torch.arange(lengths.shape[0], device=refs.device) if s["parents"] is None else s["parents"].long()
    length = torch.where(parent >= 0, lengths[parent.clamp_min(0)], 0)
    have = (length + T - 1) // T
    table = torch.where(j < have[:, None], tables[parent.clamp_min(0)], NONE)
    # who holds a page: the old sequences no more, the new ones
    count = torch.zeros(refs.shape[0] + 1, dtype=torch.int32, device=refs.device)
    count.index_add_(0, table.view(-1) % count.shape[0], torch.ones(table.numel(), dtype=torch.int32, device=refs.device))
    held = torch.where(j < ((lengths + T - 1) // T)[:, None], tables, NONE)
    count.index_add_(0, held.view(-1) % count.shape[0], torch.full((held.numel(),), -1, dtype=torch.int32, device=refs.device))
    refs += count[:-1]
    # a last page that has room and is shared is copied before it is written; where all who share it write, the first one keeps it
    total = (length + add + T - 1) // T
    fits = total <= stride
    last = table.gather(1, (have - 1).clamp_min(0)[:, None])[:, 0].clamp_min(0)
    writes = fits & (add > 0) & (length % T > 0)
    at = torch.arange(lengths.shape[0], device=refs.device)
    writers = torch.zeros_like(refs).index_add_(0, last, writes.to(torch.int32))
    lowest = torch.full_like(refs, at.shape[0]).long().scatter_reduce_(0, last, torch.where(writes, at, at.shape[0]), "amin")
    keeps = writes & (refs[last] > 1) & (writers[last] == refs[last]) & (lowest[last] == at)
    copied = writes & (refs[last] > 1) & ~keeps
    need = torch.where(fits, total - have + copied, 0)
    free = (refs == 0).nonzero()[:, 0]
    upto = need.cumsum(0)
    granted = fits & ((need == 0) | (upto <= free.shape[0]))
    stays = torch.zeros_like(refs).index_add_(0, last, (copied & ~granted).to(torch.int32)) > 0
    granted &= ~(keeps & stays[last])
    copied &= granted
    first = torch.where(granted, upto - need, 0)
    number = (first + copied)[:, None] + j - have[:, None]
    number = torch.where(copied[:, None] & (j == have[:, None] - 1), first[:, None], number)
    takes = granted[:, None] & (j >= (have - copied.long())[:, None]) & (j < total[:, None])
    refs.index_add_(0, last[copied], torch.full_like(last[copied], -1, dtype=torch.int32))
    table = torch.where(takes, free[number.clamp(0, free.shape[0] - 1)], table)
    refs[table[takes]] = 1
    to = table.gather(1, (have - 1).clamp_min(0)[:, None])[:, 0][copied]
    for pool in (s["k"], s["v"], s["ks"], s["vs"], s["bounds"]):
        pool[:, to] = pool[:, last[copied]]
    status = torch.stack([(refs == 0).sum(), (~granted).sum()]).to(torch.int32)
    return (table.to(torch.int32), torch.where(granted, length + add, length).to(torch.int32), status, refs,
            s["k"], s["v"], s["ks"], s["vs"], s["bounds"])


def _plain_compact(s):
    T, refs, tables = s["case"]["page"], s["refs"], s["tables"]
    refs.copy_(s["held"][0])
    tables.copy_(s["held"][1])
    live = refs > 0
    n = live.sum()
    at = torch.arange(refs.shape[0], device=refs.device)
    moved, to = (live & (at >= n)).nonzero()[:, 0], (~live & (at < n)).nonzero()[:, 0]
    number = torch.where(live, at, NONE)
    number[moved] = to
    for pool in (s["k"], s["v"], s["ks"], s["vs"], s["bounds"]):
        pool[:, to] = pool[:, moved]
    refs[to] = refs[moved]
    refs[moved] = 0
    inside = torch.arange(tables.shape[1], device=refs.device) < ((s["lengths"].long() + T - 1) // T)[:, None]
    tables.copy_(torch.where(inside, number[tables.long().clamp_min(0)].to(torch.int32), tables))
    return number.to(torch.int32), n.to(torch.int32).view(1), tables, refs, s["k"], s["v"], s["ks"], s["vs"], s["bounds"]


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "attend": _plain_attend, "sparse": _plain_sparse, "advance": _plain_advance,
            "compact": _plain_compact}[state["kind"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def _seen(case):
    """Tokens that the new tokens see, summed over them, and tokens that some new token of a sequence sees, summed over the sequences."""
    each = both = 0
    for length, new in zip(*_lengths(case)):
        w = case.get("window", 0) or length
        each += sum(min(p + 1, w) for p in range(length - new, length))
        both += min(length, w + new - 1)
    return each, both


def work(case):
    kind, T, H, D = case["kind"], case["page"], case["kv"], case["dim"]
    page = H * (2 * T * D + 8 + 2 * D)
    if kind == "advance":
        n = case["prompts"] * case["beams"]
        copies = 0 if case["beams"] == 1 else n // 3      # sequences whose last page another one shares: some
        return {"bytes": 2 * copies * page * case["layers"] + n * (case["max_len"] * 3 // 4 // T) * 8 + n * 16, "flops": 0}
    lengths, new = _lengths(case)
    if kind == "compact":
        used = sum(-(-n // T) for n in lengths)
        return {"bytes": 2 * (used * 2 // 3) * page * case["layers"] + used * 16 + (3 * used + 1) * 12, "flops": 0}
    n, size = sum(new), DTYPES[case["dtype"]].itemsize
    if kind == "append":
        touched = sum(-(-m // T) for m in new)
        return {"bytes": 2 * n * H * D * (size + 1) + touched * H * (8 + 2 * D), "flops": 4 * n * H * D}
    rows = n * H * case["group"]
    ends = rows * (2 * D * size + 4)
    if kind == "attend":
        each, both = _seen(case)
        return {"bytes": both * H * (2 * D + 8 / T) + ends, "flops": 4 * each * H * case["group"] * D}
    held = sum(-(-m // T) for m in lengths)
    looked = sum(min(m, case["n_select"] * T) for m in lengths)
    return {"bytes": held * H * (2 * D + 4) + looked * H * (2 * D + 8 / T) + ends + 4 * n * H * case["n_select"],
            "flops": 4 * held * H * case["group"] * D + 4 * looked * H * case["group"] * D}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------
def _exact_append(case, s):
    """The scales: the largest magnitude among a page's new tokens / 127, or what the page had; codes, bounds: no 64-bit value."""
    T, scales = case["page"], []
    for x, before in ((s["new_k"], s["ks"]), (s["new_v"], s["vs"])):
        most = x.to(torch.float64).abs().max(dim=2).values / 127.0
        out = before.to(torch.float64)
        at = 0
        for b, (length, new) in enumerate(zip(*_lengths(case))):
            first = length - new
            for j in range(first // T, (length - 1) // T + 1):
                lo, hi = max(first, j * T), min(length, (j + 1) * T)
                p = int(s["tables"][b, j])
                largest = most[at + lo - first:at + hi - first].max(dim=0).values
                out[p] = largest if j * T >= first else torch.maximum(out[p], largest)
            at += new
        scales.append(out)
    return None, None, scales[0], scales[1], None


def _exact_rows(q, k, v, seen, scale):
    l = torch.mm(q, k.t().contiguous()) * scale
    l = l.masked_fill(~seen, -math.inf)
    return torch.mm(torch.softmax(l, dim=1), v), torch.logsumexp(l, dim=1)


def _exact_attention(case, s):
    T, D, G, sparse = case["page"], case["dim"], case["group"], case["kind"] == "sparse"
    dev, out, lse = s["q"].device, [], []
    scale, at = 1.0 / math.sqrt(D), 0
    for b, (length, new) in enumerate(zip(*_lengths(case))):
        number = s["tables"][b, :-(-length // T)].long()
        pos = torch.arange(length - new, length, device=dev)
        rows_o, rows_l = [], []
        for h in range(case["kv"]):
            q = s["q"][at:at + new, h * G:(h + 1) * G].to(torch.float64).reshape(new * G, D)
            j = torch.arange(number.shape[0], device=dev)
            if sparse:      # the scores are 32-bit numbers by definition
                q32 = s["q"][at, h * G:(h + 1) * G].to(torch.float32)
                sq = q32.abs().max(dim=1).values * torch.tensor(1.0 / 127.0, dtype=torch.float32, device=dev)
                c = torch.round(q32.to(torch.float64) / sq[:, None].to(torch.float64))
                lo, hi = (s["bounds"][number, h, i].to(torch.float64) for i in (0, 1))
                bound = torch.stack([torch.maximum(lo * r, hi * r).sum(dim=1) for r in c]).to(torch.float32)
                bound = (bound * (sq[:, None] * s["ks"][number, h])).max(dim=0).values
                bound[0] = math.inf
                bound[-2:] = math.inf
                j = torch.sort(bound, descending=True, stable=True).indices[:case["n_select"]]
            p = number[j]
            k = (s["k"][p, h].to(torch.float64) * s["ks"][p, h].to(torch.float64)[:, None, None]).reshape(-1, D)
            v = (s["v"][p, h].to(torch.float64) * s["vs"][p, h].to(torch.float64)[:, None, None]).transpose(1, 2).reshape(-1, D)
            place = (j[:, None] * T + torch.arange(T, device=dev)).reshape(-1)
            seen = place[None] <= pos[:, None]
            if case.get("window"):
                seen &= place[None] > pos[:, None] - case["window"]
            o, l = _exact_rows(q, k, v, seen.repeat_interleave(G, dim=0), scale)
            rows_o.append(o.view(new, G, D))
            rows_l.append(l.view(new, G))
        out.append(torch.cat(rows_o, dim=1))
        lse.append(torch.cat(rows_l, dim=1))
        at += new
    return torch.cat(out), torch.cat(lse)


def exact(case, seed):
    if case["kind"] in ("advance", "compact"):      # nothing is computed: numbers of pages, and pages as they were
        return None
    s = _inputs(case, seed)
    if case["kind"] == "append":
        return _exact_append(case, s)
    out, lse = _exact_attention(case, s)
    return (out, lse, None) if case["kind"] == "sparse" else (out, lse)
