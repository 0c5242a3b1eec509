"""The operators on either side of the search, as measurable cases: int8 rows with scales, int8 products with a scale for each
token and channel, and log probabilities of given tokens with the entropy and the best alternatives.

  quantize  rows to int8 with one scale a row: by the largest magnitude (states on their way into an int8 product) or to unit
            norm x 127 (token vectors as the index takes them)
  matmul    int8 x int8 products, scaled per row of the left operand (token) and per row of the right one (output channel)
  logprobs  from logits that the caller has
  head      from int8 states and an int8 vocabulary matrix, without the logits in the caller's hands

`own` chooses between the plain form, in elementary torch operations, and the library's entry points.
"""
import math

import torch

own = False

TOKEN_NONE = -1      # as uint32 the library's empty-slot value: a padded position, whose log probability is 0
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases ----------------------------------------------------------------------------------------------------------
def listed():
    return [
        # states of a few tokens that are being decoded: the smallest call, all latency
        dict(name="quantize_step", kind="quantize", rows=4, cols=1024, dtype="f16", unit=False, pad=0),
        # the hidden states of a batch of passages on their way into an int8 layer
        dict(name="quantize_batch", kind="quantize", rows=16384, cols=4096, dtype="bf16", unit=False, pad=0),
        # token vectors of 8192 documents of 70 into the format that an index of 128 dimensions takes, out of a wider buffer
        dict(name="quantize_vectors", kind="quantize", rows=573440, cols=128, dtype="f16", unit=True, pad=8),
        # one token through a layer: reading the weights is all there is
        dict(name="matmul_token", kind="matmul", m=1, n=4096, k=4096, out="f16", bias=False, pad=0),
        # 256 query sets of 32 tokens through an encoder's last layer, to the 128 dimensions of the index
        dict(name="matmul_vectors", kind="matmul", m=8192, n=128, k=768, out="f16", bias=False, pad=0),
        # odd everything: rows that begin at any byte, a last k-step and last tiles in pieces
        dict(name="matmul_ragged", kind="matmul", m=1111, n=1003, k=1029, out="f32", bias=True, pad=2),
        # a large layer over a long prompt: the matrix cores' rate
        dict(name="matmul_large", kind="matmul", m=8192, n=8192, k=8192, out="bf16", bias=False, pad=0),
        # logits of a few sequences that are being decoded, best alternatives reported
        dict(name="logprobs_step", kind="logprobs", rows=8, V=50257, dtype="f32", top=5),
        # logits of the tokens of 64 queries of 32, each scored under its candidate document
        dict(name="logprobs_batch", kind="logprobs", rows=2048, V=32000, dtype="bf16", top=10),
        # one decoded token from the states: reading the vocabulary matrix
        dict(name="head_token", kind="head", rows=1, V=32000, k=1024, top=8),
        # a middling batch, a vocabulary and a width that fill no tile
        dict(name="head_ragged", kind="head", rows=203, V=50021, k=776, top=5),
        # likelihood of 128 queries of 32 tokens, each under its candidate document
        dict(name="head_batch", kind="head", rows=4096, V=32000, k=2048, top=5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "matmul", "logprobs", "head"])
    if kind == "quantize":
        rows, cols = _log(rng, 1, 573440), _log(rng, 32, 8192)
        while rows * cols > 16384 * 4096:
            rows = rows * 2 // 3
        return dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(list(DTYPES)), unit=rng.random() < 0.5,
                    pad=rng.choice([0, 0, 1, 8]))
    if kind == "matmul":
        m, n, k = _log(rng, 1, 8192), _log(rng, 16, 8192), _log(rng, 16, 8192)
        if rng.random() < 0.5:
            n, k = (n + 15) // 16 * 16, (k + 15) // 16 * 16
        return dict(kind=kind, m=m, n=n, k=k, out=rng.choice(list(DTYPES)), bias=rng.random() < 0.5,
                    pad=rng.choice([0, 0, 0, 16, 3]))
    if kind == "logprobs":
        rows, V = _log(rng, 1, 4096), _log(rng, 1000, 131072)
        while rows * V > 4096 * 32000:
            rows = rows * 2 // 3
        return dict(kind=kind, rows=rows, V=V, dtype=rng.choice(list(DTYPES)), top=rng.randint(0, 20))
    rows, V, k = _log(rng, 1, 4096), _log(rng, 1000, 131072), _log(rng, 64, 4096)
    while rows * V * k > 4096 * 32000 * 2048 or rows * V > 4096 * 32000:
        rows = rows * 2 // 3
    if rng.random() < 0.5:
        k = (k + 15) // 16 * 16
    return dict(kind=kind, rows=rows, V=V, k=k, top=rng.randint(0, 20))


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _codes(rows, cols, g, dev, pad=0):
    """Rows of int8 as rounding to 127 / largest magnitude leaves them, and their scales; pad: unused columns behind each row."""
    buf = torch.empty(rows, cols + pad, dtype=torch.int8, device=dev)
    scales = torch.empty(rows, device=dev)
    step = max(1, (1 << 26) // (cols + pad))
    for lo in range(0, rows, step):
        x = torch.randn(min(step, rows - lo), cols + pad, generator=g, device=dev)
        s = x[:, :cols].abs().amax(dim=1) / 127.0
        buf[lo:lo + x.shape[0]] = (x / s[:, None]).round_().clamp_(-128, 127).to(torch.int8)
        scales[lo:lo + x.shape[0]] = s
    return buf[:, :cols], scales


def _tokens(rows, V, g, dev):
    t = torch.randint(0, V, (rows,), generator=g, device=dev, dtype=torch.int32)
    t[torch.rand(rows, generator=g, device=dev) < 0.05] = TOKEN_NONE     # padded positions
    return t


def _inputs(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    kind = case["kind"]
    if kind == "quantize":
        # activations: rows of unequal size, a few columns far larger than the others
        x = torch.empty(case["rows"], case["cols"] + case["pad"], dtype=DTYPES[case["dtype"]], device=dev)
        wide = torch.ones(x.shape[1], device=dev)
        wide[torch.randint(0, x.shape[1], (max(1, x.shape[1] // 256),), generator=g, device=dev)] = 8.0
        step = max(1, (1 << 26) // x.shape[1])
        for lo in range(0, x.shape[0], step):
            rows = min(step, x.shape[0] - lo)
            size = torch.exp(0.5 * torch.randn(rows, 1, generator=g, device=dev))
            x[lo:lo + rows] = (size * wide * torch.randn(rows, x.shape[1], generator=g, device=dev)).to(x.dtype)
        return dict(x=x[:, :case["cols"]])
    if kind == "matmul":
        a, sa = _codes(case["m"], case["k"], g, dev, case["pad"])
        b, sb = _codes(case["n"], case["k"], g, dev, case["pad"])
        sb = sb / math.sqrt(case["k"])
        return dict(a=a, sa=sa, b=b, sb=sb, bias=torch.randn(case["n"], generator=g, device=dev) if case["bias"] else None)
    if kind == "logprobs":
        # the vocabulary ends in a few unused entries, masked out
        x = (3.0 * torch.randn(case["rows"], case["V"], generator=g, device=dev)).to(DTYPES[case["dtype"]])
        x[:, case["V"] - 7:] = -math.inf
        return dict(x=x, tokens=_tokens(case["rows"], case["V"], g, dev))
    a, sa = _codes(case["rows"], case["k"], g, dev)
    b, sb = _codes(case["V"], case["k"], g, dev)
    return dict(a=a, sa=sa, b=b, sb=sb * (3.0 / math.sqrt(case["k"])), tokens=_tokens(case["rows"], case["V"], g, dev))


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case, kind=case["kind"])
    if not own:
        return s
    # what a serving program keeps from call to call: a handle, the output buffers, the workspace
    import paper_2210_15748_amd as dz
    dev = torch.device("cuda", torch.cuda.current_device())
    ix = s["ix"] = dz.create(128, 32, 7, seed=1)
    if s["kind"] == "quantize":
        s["codes"] = torch.empty(case["rows"], case["cols"], dtype=torch.int8, device=dev)
        s["scales"] = torch.empty(case["rows"], device=dev)
    elif s["kind"] == "matmul":
        s["out"] = torch.empty(case["m"], case["n"], dtype=DTYPES[case["out"]], device=dev)
        nbytes = dz.scaled_matmul_workspace_bytes(ix, case["m"], case["n"], case["k"])
    else:
        rows, top = case["rows"], case["top"]
        s["outs"] = (torch.empty(rows, device=dev), torch.empty(rows, device=dev),
                     torch.empty(rows, top, dtype=torch.uint32, device=dev), torch.empty(rows, top, device=dev))
        if s["kind"] == "logprobs":
            nbytes = dz.token_logprobs_workspace_bytes(ix, rows, case["V"], top)
        else:
            nbytes = dz.head_logprobs_workspace_bytes(ix, rows, case["V"], case["k"], top)
    if s["kind"] != "quantize":
        s["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------
def _plain_quantize(x, unit):
    x = x.double()          # the rounding of a quotient next to a half needs more than 32 bits
    if unit:
        size = (x * x).sum(dim=1).sqrt()
        ratio = 127.0 * x / size.clamp_min(1e-300)[:, None]
        return ratio.round().to(torch.int8), (size / 127.0).float()
    scale = x.abs().amax(dim=1).float() / 127.0
    ratio = x / torch.where(scale == 0, 1.0, scale).double()[:, None]
    return ratio.round().clamp(-127, 127).to(torch.int8), scale


def _plain_logprobs(x, tokens, top):
    x = x.float()
    peak = x.amax(dim=1, keepdim=True)
    d = x - peak
    e = d.exp()
    total = e.sum(dim=1)
    log_total = total.log()
    at = tokens.long().clamp_min(0)
    given = d.gather(1, at[:, None])[:, 0] - log_total
    given = torch.where(tokens == TOKEN_NONE, 0.0, given)
    entropy = log_total - torch.where(e > 0, e * d, 0.0).sum(dim=1) / total
    ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    return given, entropy, ids, d.gather(1, ids) - log_total[:, None]


def _products(a, b):
    # whole numbers below 2^24 in the cases' data: 32-bit floats hold every partial sum
    return a.float() @ b.float().t()


def run(state):
    kind, case = state["kind"], state["case"]
    if own:
        import paper_2210_15748_amd as dz
        ix = state["ix"]
        if kind == "quantize":
            return dz.quantize_rows(ix, state["x"], dz.SCALE_UNIT if case["unit"] else dz.SCALE_MAXABS,
                                    out=state["codes"], out_scales=state["scales"])
        if kind == "matmul":
            return dz.scaled_matmul(ix, state["a"], state["sa"], state["b"], state["sb"], state["bias"], out=state["out"],
                                    workspace=state["ws"])
        if kind == "logprobs":
            out = dz.token_logprobs(ix, state["x"], state["tokens"], case["top"], workspace=state["ws"], outs=state["outs"])
        else:
            out = dz.head_logprobs(ix, state["a"], state["sa"], state["b"], state["sb"], state["tokens"], case["top"],
                                   workspace=state["ws"], outs=state["outs"])
        return out[0], out[1], out[2].view(torch.int32), out[3]
    if kind == "quantize":
        return _plain_quantize(state["x"], case["unit"])
    if kind == "matmul":
        y = _products(state["a"], state["b"]) * (state["sa"][:, None] * state["sb"])
        if state["bias"] is not None:
            y = y + state["bias"]
        return y.to(DTYPES[case["out"]])
    x = state["x"] if kind == "logprobs" else _products(state["a"], state["b"]) * (state["sa"][:, None] * state["sb"])
    given, entropy, ids, best = _plain_logprobs(x, state["tokens"], case["top"])
    return given, entropy, ids.to(torch.int32), best


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        size = DTYPES[case["dtype"]].itemsize
        return {"bytes": case["rows"] * (case["cols"] * (size + 1) + 4), "flops": 2 * case["rows"] * case["cols"]}
    if kind == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k + n * k + 4 * (m + n) + (4 * n if case["bias"] else 0) + m * n * DTYPES[case["out"]].itemsize,
                "flops": 2 * m * n * k}
    out = case["rows"] * (4 + 8 + 8 * case["top"])
    if kind == "logprobs":
        return {"bytes": case["rows"] * case["V"] * DTYPES[case["dtype"]].itemsize + out, "flops": 5 * case["rows"] * case["V"]}
    return {"bytes": (case["rows"] + case["V"]) * (case["k"] + 4) + out, "flops": 2 * case["rows"] * case["V"] * case["k"]}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------
def _exact_rows(l, tokens, top):
    """Rows of logits as 64-bit numbers: log softmax at the tokens, the entropy, the best entries."""
    lse = torch.logsumexp(l, dim=1)
    p = torch.exp(l - lse[:, None])
    lp = l - lse[:, None]
    entropy = -torch.special.xlogy(p, p).sum(dim=1)
    rows = torch.arange(l.shape[0], device=l.device)
    given = torch.where(tokens < 0, 0.0, lp[rows, tokens.clamp_min(0).long()])
    best, ids = torch.topk(lp, top, dim=1)
    # equal entries in the order of their ids
    for _ in range(2):
        ids, by_id = ids.sort(dim=1)
        best = best.gather(1, by_id)
        best, by_value = best.sort(dim=1, descending=True, stable=True)
        ids = ids.gather(1, by_value)
    return given, entropy, best


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        codes, scales = [], []
        for x in s["x"].split(max(1, (1 << 26) // case["cols"])):
            x = x.to(torch.float64)
            if case["unit"]:
                norm = torch.linalg.vector_norm(x, dim=1, keepdim=True)
                codes.append(torch.round(x * 127.0 / norm).to(torch.int8))
                scales.append(norm[:, 0] / 127.0)
            else:
                # the scale is a 32-bit number by definition, and the codes are those of that scale
                scale = (x.abs().max(dim=1).values / 127.0).to(torch.float32)
                codes.append(torch.round(x / scale[:, None].to(torch.float64)).to(torch.int8))
                scales.append(x.abs().max(dim=1).values / 127.0)
        return torch.cat(codes), torch.cat(scales)
    if kind == "matmul":
        out = []
        b = s["b"].to(torch.float64).t().contiguous()
        for a, sa in zip(s["a"].split(2048), s["sa"].split(2048)):
            y = torch.mm(a.to(torch.float64), b) * sa[:, None].to(torch.float64) * s["sb"].to(torch.float64)
            out.append(y if s["bias"] is None else y + s["bias"].to(torch.float64))
        return torch.cat(out)
    parts = []
    per = max(1, (1 << 26) // case["V"])
    b = None if kind == "logprobs" else s["b"].to(torch.float64).t().contiguous()
    for lo in range(0, case["rows"], per):
        hi = min(case["rows"], lo + per)
        if kind == "logprobs":
            l = s["x"][lo:hi].to(torch.float64)
        else:
            l = torch.mm(s["a"][lo:hi].to(torch.float64), b) * s["sa"][lo:hi, None].to(torch.float64) * s["sb"].to(torch.float64)
        parts.append(_exact_rows(l, s["tokens"][lo:hi], case["top"]))
    given, entropy, best = (torch.cat(p) for p in zip(*parts))
    # the ids have no value in 64 bits: which of two logits is the larger one is decided on 32-bit logits, by definition
    return given, entropy, None, best
