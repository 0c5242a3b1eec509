"""The operators on a paged int8 cache, written from their definitions on the CPU: attention and quotients in 64 bits, page bookkeeping one
sequence after the other.  With them the inputs that the tests share."""
import math

import numpy as np
import torch

NONE = 0xFFFFFFFF
INV127 = np.float32(1.0) / np.float32(127.0)


def make_cache(pages, heads, page, dim, seed, layers=None):
    g = torch.Generator().manual_seed(seed)
    lead = (pages,) if layers is None else (layers, pages)
    return dict(k=torch.randint(-127, 128, (*lead, heads, page, dim), generator=g, dtype=torch.int8),
                v=torch.randint(-127, 128, (*lead, heads, dim, page), generator=g, dtype=torch.int8),
                ks=torch.rand(*lead, heads, generator=g) * 0.02 + 0.002, vs=torch.rand(*lead, heads, generator=g) * 0.02 + 0.002,
                bounds=torch.randint(-127, 128, (*lead, heads, 2, dim), generator=g, dtype=torch.int8))


def make_tables(lengths, page, pages, seed, width=None):
    """Tables of unequal sequences, page numbers in no order; 0xFFFFFFFF (as -1) behind a sequence's last."""
    g = torch.Generator().manual_seed(seed)
    used = [-(-n // page) for n in lengths]
    numbers = torch.randperm(pages, generator=g).to(torch.int32)
    assert sum(used) <= pages
    t = torch.full((len(lengths), max(1, width or max(used))), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        t[b, :n] = numbers[at:at + n]
        at += n
    return t


def starts_of(new):
    return torch.tensor([0] + list(new), dtype=torch.int32).cumsum(0).to(torch.int32)


def attend(c, tables, lengths, new, q, scale, window=0, pages=None):
    """(out, lse, and how much of each output a relative error of one term can move: sum p |v| / sum p, the largest sum |q| |k| behind a score)"""
    P, H, T, D = c["k"].shape
    n, heads, _ = q.shape
    G = heads // H
    out, lse = torch.zeros(n, heads, D, dtype=torch.float64), torch.full((n, heads), -math.inf, dtype=torch.float64)
    mass, reach = torch.zeros(n, heads, D, dtype=torch.float64), torch.zeros(n, heads, dtype=torch.float64)
    row = 0
    width = tables.shape[1]
    for b, (length, m) in enumerate(zip(lengths, new)):
        number = (tables[b].long() & NONE)
        k = c["k"][number.clamp_max(P - 1)].double() * c["ks"][number.clamp_max(P - 1)].double()[..., None, None]
        v = c["v"][number.clamp_max(P - 1)].double() * c["vs"][number.clamp_max(P - 1)].double()[..., None, None]
        k, v = k.transpose(0, 1).reshape(H, width * T, D), v.permute(1, 0, 3, 2).reshape(H, width * T, D)
        there = (number < P).repeat_interleave(T)
        j = torch.arange(width * T)
        for t in range(m):
            p = length - m + t
            seen = there & (j <= p)
            if window:
                seen &= j > p - window
            for h in range(H):
                s = seen
                if pages is not None:
                    listed = torch.zeros(width, dtype=torch.bool)
                    ids = pages[row, h].long() & NONE
                    listed[ids[ids < width]] = True
                    s = seen & listed.repeat_interleave(T)
                if not s.any():
                    continue
                kk, vv = k[h, s], v[h, s]
                x = q[row, h * G:(h + 1) * G].double()
                l = x @ kk.t() * scale
                w = torch.softmax(l, dim=1)
                out[row, h * G:(h + 1) * G] = w @ vv
                lse[row, h * G:(h + 1) * G] = torch.logsumexp(l, dim=1)
                mass[row, h * G:(h + 1) * G] = w @ vv.abs()
                reach[row, h * G:(h + 1) * G] = (x.abs() @ kk.abs().t() * abs(scale)).amax(dim=1)
                bad = ~torch.isfinite(x).all(dim=1)
                out[row, h * G:(h + 1) * G][bad] = math.nan
                lse[row, h * G:(h + 1) * G][bad] = math.nan
            row += 1
    return out, lse, mass, reach


def attend_tolerance(out, lse, mass, reach, dtype, keys, dim):
    """How far 32-bit sums and fp16 weights may be off, term by term:
    a score's error d: dim + 8 roundings (products, the scales, the power of two, the largest) of at most reach each, and 2 more of the
    score itself in the exponential's argument; a weight e^(s - m) then is off by 2 d (its own and the largest's), the exponential's 2^-22,
    the factor's roundings and the rounding to fp16, 2^-11; sums of `keys` terms lose keys * 2^-24 at most; what is below the normal numbers
    of fp16 is off by 2^-37 of the largest weight times scale a key, of which 127 times at most come to an output (a channel of the largest mass holds
    a code of 1 at least where it is); the result's rounding: half a step of its type."""
    d = (dim + 12) * 2.0 ** -24 * reach
    rel = 2.0 ** -11 + 2 * d + 2.0 ** -21 + (keys + 64) * 2.0 ** -24
    least = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}[dtype]      # half the smallest step of fp16's subnormal numbers
    t_out = out.abs() * torch.finfo(dtype).eps / 2 + 2 * rel[..., None] * mass + keys * 2.0 ** -30 * mass.amax(dim=-1, keepdim=True) + least
    t_lse = d + (keys + 64) * 2.0 ** -24 + 2.0 ** -21 + lse.abs().nan_to_num(0, 0, 0) * 2.0 ** -22
    return t_out, t_lse


def rounded(num, den):
    """The integer nearest to num / den, ties to even, of 64-bit arrays whose values are 32-bit ones or products of such with codes"""
    return np.clip(np.rint(num / den), -127, 127).astype(np.int8)


def append(c, tables, lengths, new, k, v):
    """In place, token by token of a page."""
    P, H, T, D = c["k"].shape
    row = 0
    for b, (length, m) in enumerate(zip(lengths, new)):
        begin = length - m
        for place in range(max(begin, 0) // T, -(-length // T) if m else 0):
            lo, hi = max(begin, place * T, 0), min(length, (place + 1) * T)
            page = int(tables[b, place]) & NONE if place < tables.shape[1] else NONE
            if page >= P or lo >= hi:
                continue
            s0, s1 = lo % T, lo % T + hi - lo
            for h in range(H):
                for x, codes, scales, keys in ((k, c["k"], c["ks"], True), (v, c["v"], c["vs"], False)):
                    x = x[row + lo - begin:row + hi - begin, h].float().numpy()
                    had = np.float32(scales[page, h]) if s0 else np.float32(0)
                    most = np.abs(x).max()
                    now = np.float32(np.nan) if not np.isfinite(x).all() or np.isnan(had) else max(had, np.float32(most) * INV127)
                    old = codes[page, h].numpy() if keys else codes[page, h].numpy().T     # [T][D], a view
                    bounds = c["bounds"][page, h].numpy()
                    if now > had:
                        old[:s0] = rounded(old[:s0].astype(np.float64) * np.float64(had), np.float64(now))
                        if keys:
                            bounds[:] = rounded(bounds.astype(np.float64) * np.float64(had), np.float64(now))
                    fresh = rounded(x.astype(np.float64), np.float64(now)) if now > 0 else np.zeros(x.shape, np.int8)
                    old[s0:s1] = fresh
                    if keys:
                        least, most_code = fresh.min(axis=0), fresh.max(axis=0)
                        bounds[:] = np.stack([least, most_code] if s0 == 0 else [np.minimum(bounds[0], least), np.maximum(bounds[1], most_code)])
                    scales[page, h] = float(now)
        row += m


def select(c, tables, lengths, new, codes, scales, n_select, n_first, n_last):
    P, H, T, D = c["k"].shape
    n = sum(new)
    heads = codes.shape[0] // n
    G = heads // H
    out = np.full((n, H, n_select), NONE, dtype=np.uint32)
    row = 0
    for b, (length, m) in enumerate(zip(lengths, new)):
        for t in range(m):
            p = length - m + t
            if p >= 0:
                places = min(p // T + 1, tables.shape[1])
                number = np.array([int(x) & NONE for x in tables[b, :places]])
                there = number < P
                safe = np.minimum(number, P - 1)
                for h in range(H):
                    lo, hi = (c["bounds"][safe, h, i].numpy().astype(np.int64) for i in (0, 1))
                    best = np.full(places, -np.inf, dtype=np.float32)
                    nan = np.zeros(places, dtype=bool)
                    for i in range(row * heads + h * G, row * heads + (h + 1) * G):
                        cq = codes[i].numpy().astype(np.int64)
                        sums = np.where(cq < 0, cq * lo, cq * hi).sum(axis=1).astype(np.float32)
                        with np.errstate(invalid="ignore"):
                            s = sums * (np.float32(scales[i]) * c["ks"][safe, h].numpy())
                        nan |= np.isnan(s)
                        best = np.fmax(best, s)
                    best[nan] = np.inf
                    always = (np.arange(places) < n_first) | (np.arange(places) + n_last > p // T)
                    order = sorted((i for i in range(places) if there[i]), key=lambda i: (not always[i], -best[i], i))
                    chosen = sorted(order[:n_select])
                    out[row, h, :len(chosen)] = chosen
            row += 1
    return out


def advance(c, refs, tables, lengths, add, parents):
    """(tables, lengths, status); c [layers, pages, ...] and refs in place.  Lists of ints throughout."""
    P, T = c["k"].shape[1], c["k"].shape[3]
    width = tables.shape[1]
    old = [[int(x) & NONE for x in r] for r in tables]
    length = [int(x) for x in lengths]
    add = [int(x) for x in add]
    gives = parents is not None
    parents = list(range(len(old))) if parents is None else [int(x) & NONE for x in parents]
    r = [int(x) for x in refs]
    if gives:
        for b, n in enumerate(length):
            for j in range(-(-n // T)):
                r[old[b][j]] -= 1
    new, size = [], []
    for b, p in enumerate(parents):
        n = length[p] if p < len(old) else 0
        size.append(n)
        new.append([old[p][j] for j in range(-(-n // T))] if n else [])
        if gives:
            for page in new[-1]:
                r[page] += 1
    total = [-(-(n + a) // T) for n, a in zip(size, add)]
    fits = [t <= width for t in total]
    writes = [fits[b] and add[b] > 0 and size[b] % T > 0 for b in range(len(new))]
    role = [None] * len(new)
    for b in range(len(new)):
        if writes[b] and r[new[b][-1]] > 1:
            page = new[b][-1]
            writers = [x for x in range(len(new)) if writes[x] and new[x][-1] == page]
            role[b] = "keeps" if len(writers) == r[page] and writers[0] == b else "copies"
    need = [total[b] - len(new[b]) + (role[b] == "copies") if fits[b] else 0 for b in range(len(new))]
    free = [p for p in range(P) if r[p] == 0]
    before, granted = 0, []
    for b in range(len(new)):
        granted.append(fits[b] and (need[b] == 0 or before + need[b] <= len(free)))
        before += need[b]
    for b in range(len(new)):
        if role[b] == "keeps" and any(role[x] == "copies" and not granted[x] and new[x][-1] == new[b][-1] for x in range(len(new))):
            granted[b] = False
    before, moves, taken = 0, [], 0
    for b in range(len(new)):
        mine = free[before:before + need[b]]
        before += need[b]
        if not granted[b]:
            continue
        taken += need[b]
        if role[b] == "copies":
            moves.append((new[b][-1], mine[0]))
            r[new[b][-1]] -= 1
            new[b][-1] = mine[0]
            new[b] += mine[1:]
        else:
            new[b] += mine
        for p in mine:
            r[p] = 1
    for x in c.values():
        for a, b in moves:
            x[:, b] = x[:, a]
    refs[:] = torch.tensor(r, dtype=refs.dtype)
    table = torch.full((len(new), width), -1, dtype=torch.int32)
    for b, pages in enumerate(new):
        table[b, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
    sizes = [n + a if g else n for n, a, g in zip(size, add, granted)]
    return table, torch.tensor(sizes, dtype=torch.int32), [len(free) - taken, len(new) - sum(granted)]


def compact(c, refs, tables, lengths):
    """(numbers, pages in use); c, refs and tables in place"""
    P, T = c["k"].shape[1], c["k"].shape[3]
    used = [p for p in range(P) if int(refs[p])]
    n = len(used)
    number = {p: p for p in used if p < n}
    holes = [p for p in range(n) if not int(refs[p])]
    for a, b in zip([p for p in used if p >= n], holes):
        number[a] = b
        for x in c.values():
            x[:, b] = x[:, a]
        refs[b], refs[a] = refs[a].clone(), 0
    for b, length in enumerate(lengths):
        for j in range(-(-int(length) // T)):
            tables[b, j] = number[int(tables[b, j])]
    return torch.tensor([number.get(p, -1) for p in range(P)], dtype=torch.int32), n
