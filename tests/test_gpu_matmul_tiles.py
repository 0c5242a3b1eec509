"""Scaled products on both sides of the numbers of tiles at which their shape changes: 64^2, 128^2, 256^2."""
import sys

import pytest
import torch

import paper_2210_15748_amd as dz

import row_operators_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ix():
    return dz.create(128, 32, 7, seed=3, device=torch.device(DEV))


def apart(t, pad, at):
    rows, cols = t.shape
    buf = torch.full((at + rows * (cols + pad),), 101, dtype=torch.int8, device=DEV)
    return buf[at:].view(rows, cols + pad)[:, :cols].copy_(t)


# 128^2 tiles: 191, 192, 512, 516, 544, 792
@pytest.mark.parametrize("m,n,k", [(100, 24400, 80), (1500, 2000, 144), (2048, 4096, 144), (130, 33000, 80), (2049, 4090, 272), (3000, 4100, 208)])
def test_sizes_around_the_borders(ix, m, n, k):
    g = torch.Generator()
    g.manual_seed(m)
    a = torch.randint(-128, 128, (m, k), generator=g, dtype=torch.int8)
    b = torch.randint(-128, 128, (n, k), generator=g, dtype=torch.int8)
    sa, sb, c = torch.rand(m, generator=g) * 0.01 + 1e-4, torch.rand(n, generator=g) * 0.01 + 1e-4, torch.randn(n, generator=g)
    exact = {t: plain.matmul(a, sa, b, sb, c, t) for t in (torch.float16, torch.bfloat16, torch.float32)}
    # rows at whole 16 bytes, at 4, anywhere; a result whose rows lie apart
    for pad, at, gap in [(0, 0, 0), (16, 32, 3), (4, 8, 0), (1, 3, 1)]:
        x, y = apart(a, pad, at), apart(b, pad, at)
        for dtype, (want, tol) in exact.items():
            print("[case]", m, n, k, pad, at, gap, dtype, flush=True)
            sys.stdout.flush()
            buf = torch.full((m, n + gap), 55.0, dtype=dtype, device=DEV)
            out = dz.scaled_matmul(ix, x, sa.to(DEV), y, sb.to(DEV), c.to(DEV), out=buf[:, :n])
            assert ((out.double() - want.to(DEV)).abs() <= tol.to(DEV)).all()
            assert (buf[:, n:] == 55).all()
