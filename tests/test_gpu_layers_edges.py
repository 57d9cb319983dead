"""The layers at the edges of what their definitions allow, against their plain 64-bit definitions.  U = 2^-24 as in test_gpu_layers.py."""
import math

import pytest
import torch

from oracle import layers_oracle as lo
from paper_2406_11257_b200 import binding
from test_gpu_layers import DEV, DT, U, make, near, vector

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(workspace_numel=4096, device=0)
    yield handle
    handle.score_status()
    handle.close()


# ---- norms -------------------------------------------------------------------------
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols,slack", [(1000, 0), (1000, 3), (4096, 0), (300, 1), (8, 0), (17000, 0), (17001, 0)])
@pytest.mark.parametrize("rows", [5, 2000])
def test_gradient_of_equal_values_is_finite(h, rows, cols, slack, dtype, weighted):
    """Rows of one large value (which 8 bits hold exactly) with a small eps: xh is 0 in every column, so dx = rstd (g - mean g).  The mean
    times rstd, 2^91 * 2^49, is past fp32's numbers, and may not be formed where there is no column.  The mean of g is off by u of the mean
    magnitude for each of at most cols / 8 / 32 + 40 additions in a row and a product; four roundings are left."""
    x = torch.full((rows, cols + slack), 127 * 2.0 ** 84, device=DEV).to(DT[dtype])[:, :cols]
    dy = make(rows, cols, dtype, 3, slack)
    w = vector(cols, dtype, 4, 0.2, 1.0) if weighted else None
    r = h.layer_norm(x, w, eps=1e-30, keep=True)
    want, _, db = lo.norm_grad(dy, x, w, r.row_stats[:, 0], r.row_stats[:, 1])
    gg = dy.double().abs() * (1.0 if w is None else w.double().abs())
    tol = r.row_stats[:, 1:].double() * U * (4 * gg + (cols / 256 + 44) * gg.mean(1, keepdim=True))
    for v in (x, r.kept):
        for vectors in (True, False):
            g = h.layer_norm_grad(dy, v, w, r, vectors=vectors)
            near(g.dx, want, tol, "dx")
        g = h.layer_norm_grad(dy, v, w, r)
        assert not g.dweight.any()
        near(g.dbias, db, dy.double().abs().sum(0) * (rows + 40) * U, "dbias")


@pytest.mark.parametrize("rows", [3000, 200])
@pytest.mark.parametrize("cols", [256, 320, 4096, 16384, 20000])
def test_rstd_is_rounded_once(h, rows, cols):
    """Whole numbers, whose squares add up exactly (at most 64 * 20000 < 2^24): what is left is the rounding of the sum over cols (u, which the root
    halves) and of 1 / root (u).  With a power of two for cols the division is exact too."""
    g = torch.Generator().manual_seed(cols + rows)
    x = torch.randint(-8, 9, (rows, cols), generator=g).float().to(DEV)
    r = h.layer_norm(x, eps=0.0, rms=True)
    want = 1.0 / torch.sqrt((x.double() ** 2).mean(1))
    units = 1.0 if cols & (cols - 1) == 0 else 1.5
    assert bool(((r.row_stats[:, 1].double() - want).abs() <= units * U * 1.0001 * want).all())


# ---- products ------------------------------------------------------------------------
@pytest.mark.parametrize("rows,k,n", [(4, 512, 300), (64, 4096, 1024), (1, 11008, 4096)])
def test_waits_that_some_ctas_give_up(rows, k, n):
    """Limits at which some CTAs of a cluster give up and others do not: the product says so or is right, and the next one is right."""
    other = binding.Handle(workspace_numel=4096, device=0)
    x, w = make(rows, k, "bf16", 1), make(n, k, "bf16", 2)
    want = other.linear(x, w)
    other.score_status()
    for limit in (1, 500, 2000, 5000, 10000):
        for _ in range(3):
            other.set_wait_limit(limit)
            got = other.linear(x, w)
            try:
                other.score_status()
            except binding.ExcpError as e:
                assert e.status == -7
            else:
                assert torch.equal(got, want)
            other.set_wait_limit(2_000_000_000)
            assert torch.equal(other.linear(x, w), want)
            other.score_status()
    other.close()
