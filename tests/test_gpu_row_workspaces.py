"""One workspace, sized for the largest batch, serves the smaller ones (the column parts of a product and the parts of a row of logits are more where
rows are few)."""
import pytest
import torch

import paper_2210_15748_amd as dz

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ix():
    return dz.create(128, 32, 7, seed=3, device=torch.device(DEV))


def guarded(nbytes):
    buf = torch.full((nbytes + 512,), 77, dtype=torch.uint8, device=DEV)
    return buf[:nbytes], buf[nbytes:]


@pytest.mark.parametrize("n,k", [(1000, 8192), (1000, 8193), (4096, 4100), (130, 2049)])
def test_products_of_smaller_batches(ix, n, k):
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    most = 1100
    a = torch.randint(-128, 128, (most, k), generator=g, device=DEV, dtype=torch.int8)
    b = torch.randint(-128, 128, (n, k), generator=g, device=DEV, dtype=torch.int8)
    sa, sb = torch.rand(most, generator=g, device=DEV), torch.rand(n, generator=g, device=DEV)
    ws, behind = guarded(dz.scaled_matmul_workspace_bytes(ix, most, n, k))
    whole = dz.scaled_matmul(ix, a, sa, b, sb, workspace=ws)
    for m in (1, 5, 16, 17, 33, 64, 65, 128, 200, 320, 512, 900):
        print("[case]", m, n, k, flush=True)
        assert torch.equal(dz.scaled_matmul(ix, a[:m], sa[:m], b, sb, workspace=ws), whole[:m])
    assert (behind == 77).all()


@pytest.mark.parametrize("most", [300, 1024, 2000])
def test_log_probabilities_of_smaller_batches(ix, most):
    V, k, n_top = 40000, 64, 7
    g = torch.Generator(device=DEV)
    g.manual_seed(most)
    x = 3 * torch.randn(most, V, generator=g, device=DEV)
    t = torch.randint(0, V, (most,), generator=g, device=DEV, dtype=torch.int32)
    a = torch.randint(-127, 128, (most, k), generator=g, device=DEV, dtype=torch.int8)
    b = torch.randint(-127, 128, (V, k), generator=g, device=DEV, dtype=torch.int8)
    sa, sb = torch.rand(most, generator=g, device=DEV), torch.rand(V, generator=g, device=DEV) * 1e-3
    ws, behind = guarded(max(256, dz.token_logprobs_workspace_bytes(ix, most, V, n_top)))
    hws, hbehind = guarded(dz.head_logprobs_workspace_bytes(ix, most, V, k, n_top))
    odd = torch.zeros(most, k + 1, dtype=torch.int8, device=DEV)[:, :k].copy_(a)     # rows at odd bytes go the other way
    for m in (1, 2, 9, 60, 129, 256, 300, 416, 417, 700, 1000, 1023, 1024):
        if m > most:
            continue
        print("[case]", m, most, flush=True)
        given = dz.token_logprobs(ix, x[:m], t[:m], n_top, workspace=ws)
        own = dz.token_logprobs(ix, x[:m], t[:m], n_top)
        for u, v in zip(given, own):
            assert torch.equal(u.view(torch.int32), v.view(torch.int32))
        for rows in (a, odd):
            given = dz.head_logprobs(ix, rows[:m], sa[:m], b, sb, t[:m], n_top, workspace=hws)
            own = dz.head_logprobs(ix, rows[:m], sa[:m], b, sb, t[:m], n_top)
            for u, v in zip(given, own):
                assert torch.equal(u.view(torch.int32), v.view(torch.int32))
    assert (behind == 77).all() and (hbehind == 77).all()
