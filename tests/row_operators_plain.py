"""The row operators (int8 rows with scales, scaled int8 products, log probabilities) in 64 bits on the CPU, and how far 32-bit
arithmetic may be off them.  Written from the formulas; shares nothing with the package."""
import numpy as np
import torch

U32 = 2.0 ** -24                                     # half a step of a 32-bit float, relative
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SMALLEST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half the smallest step
NONE = 0xFFFFFFFF


def quantize(x, unit):
    """codes int8, scales float32 (largest magnitude: a product of 32-bit floats) or float64 (unit norm), of a CPU tensor"""
    x = x.to(torch.float64).numpy().astype(np.longdouble)
    ok = np.isfinite(x).all(axis=1)
    x = np.where(ok[:, None], x, 0)
    if unit:
        norm = np.sqrt((x * x).sum(axis=1))
        with np.errstate(divide="ignore", invalid="ignore"):
            codes = np.where(norm[:, None] > 0, np.rint(127 * x / norm[:, None]), 0)
        scales = (norm / 127).astype(np.float64)
    else:
        scales = np.abs(x).max(axis=1).astype(np.float32) * (np.float32(1) / np.float32(127))
        with np.errstate(divide="ignore", invalid="ignore"):
            codes = np.where(scales[:, None] > 0, np.rint(x / scales[:, None].astype(np.longdouble)), 0)
    return np.clip(codes, -127, 127).astype(np.int8), np.where(ok, scales, np.nan)


def sums(a, b):
    """Exact products of int8 matrices (torch, CPU) as int64."""
    return (a.double() @ b.double().t()).to(torch.int64)     # |sum| < 2^31: exact in 64-bit floats


def matmul(a, sa, b, sb, bias, out_dtype):
    """64-bit result and the largest error of the 32-bit form: the sum's conversion, the product of the scales and the product with
    it each round once, then the bias and the result's type."""
    p = sums(a, b).double() * sa.double()[:, None] * sb.double()
    y = p if bias is None else p + bias.double()
    tol = 3.01 * U32 * p.abs() + U32 * y.abs() * 1.01 + HALF_STEP[out_dtype] * 1.01 * y.abs() + SMALLEST[out_dtype]
    return y, tol


def head_logits(a, sa, b, sb):
    """The logits of the head form: 32-bit floats by definition."""
    s = sums(a, b).numpy().astype(np.float32)
    return torch.from_numpy(s * (sa.numpy()[:, None] * sb.numpy()[None, :]))


def logprobs(x, tokens, n_top):
    """x: CPU tensor of logits, tokens: int64 numpy or None.  (logprobs, entropy, ids, top logprobs, tolerance of the log
    probabilities [n], of the entropy [n]); rows as documented for masks, infinities and NaN.

    The 32-bit form: a lane adds its entries one after the other, at most V / 256 + 64 of them and of partial sums, each addition
    off by U32 relative (all terms are positive).  A term e^d, d = l - m <= 0, is off by U32 (|d| for the difference, 2 |d| for the
    multiplication with log2 e and that constant, 4 for the exponential), and every move to a larger maximum does the same once
    more for a d of its own, which adds to at most the same |d| (the d of the moves add up to the whole).  So log s is off by
    U32 (V / 256 + 64 + 6 E|d|) with E|d| = sum p |d| = |t / s|, plus its own rounding, and t / s by that much relative."""
    l = x.double().numpy()
    n, V = l.shape
    lp, ent, tol, tol_ent = np.zeros(n), np.zeros(n), np.zeros(n), np.zeros(n)
    ids, top = np.full((n, n_top), NONE, np.uint32), np.full((n, n_top), -np.inf)
    for i in range(n):
        r = l[i]
        token = None if tokens is None else int(tokens[i]) & 0xFFFFFFFF
        if np.isnan(r).any() or np.isposinf(r).any():
            lp[i] = ent[i] = np.nan
            top[i] = np.nan
        elif np.isneginf(r).all():
            lp[i] = -np.inf
        else:
            m = r.max()
            d = r - m
            e = np.exp(d)
            s = e.sum()
            mean_d = np.where(e > 0, e * np.where(e > 0, d, 0), 0).sum() / s
            ent[i] = np.log(s) - mean_d
            if token is not None:
                lp[i] = d[token] - np.log(s) if token < V else -np.inf
            order = np.lexsort((np.arange(V), -r))[:n_top]
            order = order[~np.isneginf(r[order])]
            ids[i, :len(order)] = order
            top[i, :len(order)] = d[order] - np.log(s)
            rel = V / 256 + 64 + 6 * abs(mean_d)
            tol[i] = U32 * (rel + 3 * np.log(s))
            tol_ent[i] = U32 * (rel * (1 + abs(mean_d)) * 2 + 3 * np.log(s) + 2 * ent[i])
        if token == NONE:
            lp[i] = 0.0
    return lp, ent, ids, top, tol, tol_ent


def close(got, want, tol):
    """Equal infinities and NaN, and finite values within tol."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    tol = np.broadcast_to(tol, want.shape)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)     # past the largest 32-bit float
    fin = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fin)
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True)
    off = np.abs(got[fin] - want[fin]) - tol[fin]
    assert (off <= 0).all(), f"off by {np.abs(got[fin] - want[fin])[off.argmax()]:.3g}, allowed {tol[fin][off.argmax()]:.3g}"


def check_logprobs(got, x, tokens, n_top):
    lp, ent, ids, top, tol, tol_ent = logprobs(x, tokens, n_top)
    g_lp, g_ent, g_ids, g_top = (None if t is None else t.cpu().view(torch.int32).numpy().view(np.uint32) if t.dtype == torch.uint32
                                 else t.cpu().numpy() for t in got)
    # the difference l - m of the token and the last subtraction round too: 2 U32 of the log probability and its parts
    def of(v):
        return tol + 4 * U32 * np.where(np.isfinite(v), np.abs(v), 0)
    if tokens is None:
        assert g_lp is None
    else:
        close(g_lp, lp, of(lp))
    close(g_ent, ent, tol_ent)
    assert np.array_equal(g_ids, ids)
    if n_top:
        close(g_top, top, tol[:, None] + 4 * U32 * np.where(np.isfinite(top), np.abs(top), 0))
