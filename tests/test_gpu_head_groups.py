"""Log probabilities from int8 states where the logits do not go through memory: by groups of the vocabulary (tests/test_host_row_plans.py holds that
these calls go that way)."""
import sys

import numpy as np
import pytest
import torch

import paper_2210_15748_amd as dz

import row_operators_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# rows, vocabulary, columns, alternatives
SHAPES = [(1100, 20129, 272, 3), (513, 20001, 64, 0), (33000, 200, 16, 0), (2100, 20001, 1040, 4), (1000, 131000, 96, 64), (700, 70001, 1040, 21),
          (9000, 9001, 48, 8), (1500, 48011, 64, 33), (97, 102473, 128, 1)]
VALUES = (1000, 50100, 64, 30)
TURNS = (50000, 20000, 32, 5)
PARTS = (1000, 40000, 64, 6)
GRAPH = (3000, 9001, 208, 3)
SWITCH = (4096, 32000, 80)                               # rows, vocabulary, columns: few alternatives by groups, many by logits


@pytest.fixture(scope="module")
def ix():
    return dz.create(128, 32, 7, seed=3, device=torch.device(DEV))


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


def inputs(n, V, k, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    a = torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8)
    b = torch.randint(-127, 128, (V, k), generator=g, dtype=torch.int8)
    scale = 3.0 / (73.3 * 73.3 * k ** 0.5)               # logits of about 3
    t = torch.randint(0, V, (n,), generator=g)
    t[::7] = -1                                          # padded positions
    t[3] = V                                             # no such id
    return a, torch.exp(0.3 * torch.randn(n, generator=g)), b, scale * torch.exp(0.1 * torch.randn(V, generator=g)), t


def apart(t, pad):
    buf = torch.full((t.shape[0], t.shape[1] + pad), 101, dtype=t.dtype, device=DEV)
    return buf[:, :t.shape[1]].copy_(t)


def check(got, inp, n_top, pick, with_tokens=True):
    a, sa, b, sb, t = inp
    with np.errstate(invalid="ignore"):
        l = plain.head_logits(a[pick], sa[pick], b, sb)
    at = pick.to(DEV)
    got = [None if o is None else o.view(torch.int32)[at].view(o.dtype) for o in got]
    plain.check_logprobs(got, l, t[pick].numpy() if with_tokens else None, n_top)


def some_rows(n, *more):
    g = torch.Generator()
    g.manual_seed(n)
    return torch.unique(torch.cat([torch.arange(min(n, 20)), torch.randint(0, n, (30,), generator=g), torch.tensor([n - 1, *more])]))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_sizes(ix, shape):
    n, V, k, n_top = shape
    inp = inputs(n, V, k, V)
    a, sa, b, sb, t = inp
    for pad, with_tokens in [(0, True), (16, False)]:
        say("head by groups", shape, pad)
        got = dz.head_logprobs(ix, apart(a, pad), sa.to(DEV), apart(b, 2 * pad), sb.to(DEV), t.to(DEV) if with_tokens else None, n_top)
        check(got, inp, n_top, some_rows(n), with_tokens)
    # rows at odd bytes take the other way: the same alternatives in every row
    other = dz.head_logprobs(ix, apart(a, 3), sa.to(DEV), apart(b, 5), sb.to(DEV), None, n_top)
    assert torch.equal(got[2].view(torch.int32), other[2].view(torch.int32))


def test_ties_and_numbers_that_are_not_finite(ix):
    n, V, k, n_top = VALUES
    a, sa, b, sb, t = inputs(n, V, k, 12)
    b[300:9000] = b[50]                                  # equal columns, over many groups
    sb[300:9000] = sb[50]
    b[50050:] = b[50040]
    sb[50050:] = sb[50040]
    a[1] = 0                                             # every logit 0: the first ids
    sa[2], sa[3], sa[4] = float("nan"), 0.0, float("inf")
    a[5:600] = a[5]                                      # these rows want the same groups
    sa[5:600] = sa[5]
    a[10], sa[11] = b[50], 3.0                           # best entries are the equal ones
    pick = torch.arange(0, 40)
    got = dz.head_logprobs(ix, *(v.to(DEV) for v in (a, sa, b, sb, t)), n_top)
    check(got, (a, sa, b, sb, t), n_top, pick)
    # scales of -inf make logits of -inf (or +inf, or NaN): whole groups of masked entries
    sb[128:2048] = float("-inf")
    b[128:2048] = 1
    a[:40] = a[:40].abs().clamp(min=1)                   # positive sums there
    got = dz.head_logprobs(ix, *(v.to(DEV) for v in (a, sa, b, sb, t)), n_top)
    check(got, (a, sa, b, sb, t), n_top, pick)
    # fewer entries left than alternatives asked for, in one group, and none at all
    sb[:] = float("-inf")
    b[:] = 1
    sb[777:777 + n_top // 2] = 0.01
    a[:] = a.abs().clamp(min=1)
    for left in (n_top // 2, 0):
        sb[777 + left:777 + n_top // 2] = float("-inf")
        got = dz.head_logprobs(ix, *(v.to(DEV) for v in (a, sa, b, sb, t)), n_top)
        check(got, (a, sa, b, sb, t), n_top, pick)


def test_in_turns_and_again(ix):
    """More rows than a turn takes, twice with one workspace: the same bits, though lists are filled in no fixed order."""
    n, V, k, n_top = TURNS
    inp = inputs(n, V, k, 14)
    args = [v.to(DEV) for v in inp[:4]] + [inp[4].to(torch.int32).to(DEV)]
    ws = torch.empty(dz.head_logprobs_workspace_bytes(ix, n, V, k, n_top), dtype=torch.uint8, device=DEV)
    assert ws.numel() < 300 << 20
    first = [o.clone() for o in dz.head_logprobs(ix, *args, n_top, workspace=ws)]
    ws.random_(0, 256)
    again = dz.head_logprobs(ix, *args, n_top, workspace=ws)
    for u, v in zip(first, again):
        assert torch.equal(u.view(torch.int32), v.view(torch.int32))
    check(first, inp, n_top, some_rows(n, *range(46800, 46900, 9)))


def test_outputs_that_nobody_asked_for(ix):
    n, V, k, n_top = PARTS
    a, sa, b, sb, t = inputs(n, V, k, 17)
    want = plain.logprobs(plain.head_logits(a[:9], sa[:9], b, sb), t[:9].numpy(), n_top)
    d = [v.to(DEV) for v in (a, sa, b, sb, t.to(torch.int32))]
    ws = torch.empty(dz.head_logprobs_workspace_bytes(ix, n, V, k, n_top), dtype=torch.uint8, device=DEV)
    lp, ids, top = torch.empty(n, device=DEV), torch.empty(n, n_top, dtype=torch.int32, device=DEV), torch.empty(n, n_top, device=DEV)
    for with_tokens in (True, False):
        lp.fill_(5.0)
        ids.zero_()
        st = dz.lib().dessert_head_logprobs(ix.handle, d[0].data_ptr(), k, d[1].data_ptr(), n, d[2].data_ptr(), k, d[3].data_ptr(), V, k,
                                            d[4].data_ptr() if with_tokens else None, n_top, ws.data_ptr(), ws.numel(),
                                            lp.data_ptr() if with_tokens else None, None, ids.data_ptr(), top.data_ptr())
        assert st == dz.OK, dz.last_error()
        assert np.array_equal(ids[:9].cpu().numpy().view(np.uint32), want[2])
        if with_tokens:
            plain.close(lp[:9].cpu().numpy(), want[0], want[4] + 4 * plain.U32 * np.where(np.isfinite(want[0]), np.abs(want[0]), 0))
        else:
            assert (lp == 5).all()


def test_captured_into_a_graph_and_replayed_with_new_inputs():
    n, V, k, n_top = GRAPH
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ix = dz.create(128, 32, 7, seed=3)
        held = [v.to(DEV) for v in inputs(n, V, k, 0)]
        held[4] = held[4].to(torch.int32)
        ws = torch.empty(dz.head_logprobs_workspace_bytes(ix, n, V, k, n_top), dtype=torch.uint8, device=DEV)
        outs = (torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, n_top, dtype=torch.uint32, device=DEV), torch.empty(n, n_top, device=DEV))

        def go():
            dz.head_logprobs(ix, *held, n_top, workspace=ws, outs=outs)

        go()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            go()
        for seed in range(1, 5):
            inp = inputs(n, V, k, seed)
            for h, v in zip(held, inp):
                h.copy_(v)
            for o in outs:
                o.view(torch.int32).zero_()
            graph.replay()
            side.synchronize()
            replayed = [o.clone() for o in outs]
            check(replayed, inp, n_top, some_rows(n))
            go()
            side.synchronize()
            for u, v in zip(replayed, outs):
                assert torch.equal(u.view(torch.int32), v.view(torch.int32))


def test_more_alternatives_go_the_other_way_to_the_same_ones(ix):
    n, V, k = SWITCH
    args = [v.to(DEV) for v in inputs(n, V, k, 21)]
    many = dz.head_logprobs(ix, *args, 64)
    for n_top in (1, 8, 20):
        few = dz.head_logprobs(ix, *args, n_top)
        assert torch.equal(few[2].view(torch.int32), many[2].view(torch.int32)[:, :n_top])
        # both are within the sums' error of the formula: V / 256 additions one after the other at most, and exponentials of differences of some 20
        tol = 2 * plain.U32 * (V / 256 + 64 + 6 * 20 + 3 * np.log(V) + 4 * 20)
        assert (few[3] - many[3][:, :n_top]).abs().max() <= tol
        assert (few[0] - many[0]).nan_to_num(0.0, 0.0, 0.0).abs().max() <= tol and torch.equal(few[0].isinf(), many[0].isinf())
