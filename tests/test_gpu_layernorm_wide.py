"""Layer norm of rows far wider than the registers of a workgroup hold."""
import pytest
import torch

from ops_common import HALF, TYPES, U, f64, within

pytestmark = pytest.mark.gpu


def test_more_columns_than_a_grid_of_the_sums_has_along_x():
    """2^25 + 6 columns: the sums of d_weight and d_bias over partial rows are a launch of more than 2^32 threads.  With two rows of +1 and -1
    in turn, the second one negated, xh is +-1 / sqrt(1 + eps) and every sum has two terms."""
    from paper_2307_07649_amd import tgnn
    c, eps = (1 << 25) + 6, 1.0
    x = torch.ones(2, c, dtype=torch.bfloat16, device="cuda")
    x[0, 1::2] = -1
    x[1, ::2] = -1
    y, mean, rstd = tgnn.tgnn_layer_norm_fwd(x, eps=eps)
    assert (mean == 0).all() and (rstd - 0.5 ** 0.5).abs().max() <= 4 * U     # (sums of whole numbers below 2^24: exact)
    dy = torch.full((2, c), 0.5, dtype=torch.bfloat16, device="cuda")
    dy[1] = 2
    dx, dw, db = tgnn.tgnn_layer_norm_bwd(dy, x, mean, rstd)
    assert dw.shape == db.shape == (c,)
    want = (f64(rstd)[0] * (0.5 - 2)).item()          # dy xh: 0.5 rstd and -2 rstd in the even columns, the other signs in the odd ones
    for part, sign in ((dw[::2], 1), (dw[1::2], -1)):
        assert (part - sign * want).abs().max() <= 4 * U * 2
    assert (db == 2.5).all()
    # g - mean(g) is zero, and so is the mean of g xh
    assert dx.abs().max() <= 4 * U
    assert (y[0, 0] - 0.5 ** 0.5).abs() <= HALF[torch.bfloat16]


@pytest.mark.parametrize("kind,rows,c", [("f32", 70, 9001), ("bf16", 3, 70_003), ("f32", 2, (1 << 22) + 1), ("bf16", 1, (1 << 25) + 3)])
def test_errors_do_not_grow_with_the_columns(kind, rows, c):
    """Rows far from zero.  What is left of the errors when sums are taken in double: a rounding of mean and of rstd (`within` counts it), so
    that xh is off by e_xh; a rounding of every factor and term, and of one partial sum per 64 rows of the weights' gradients."""
    from paper_2307_07649_amd import tgnn
    T, eps = TYPES[kind], 2.0 ** -16
    g = torch.Generator(device="cuda").manual_seed(c)
    x = (torch.randn(rows, c, device="cuda", generator=g) + 100).to(T)
    dy = (torch.randn(rows, c, device="cuda", generator=g) + 1).to(T)
    w, b = (torch.rand(c, device="cuda", generator=g) + 0.5 for _ in range(2))
    y, mean, rstd = tgnn.tgnn_layer_norm_fwd(x, w, b, eps)
    dx, dw, db = tgnn.tgnn_layer_norm_bwd(dy, x, mean, rstd, w)
    X, DY, W = x.double(), dy.double(), w.double()
    m = X.mean(1, keepdim=True)
    r = 1 / torch.sqrt(((X - m) ** 2).mean(1, keepdim=True) + eps)
    xh, gw = (X - m) * r, DY * W
    s1, s2 = gw.mean(1, keepdim=True), (gw * xh).mean(1, keepdim=True)
    within(mean, m[:, 0].cpu(), 0.1 * U * m[:, 0].abs().cpu(), "mean")
    within(rstd, r[:, 0].cpu(), 0.1 * U * r[:, 0].cpu(), "rstd")
    e_xh = 2 * U * m.abs() * r + 4 * U * xh.abs()
    within(y, (xh * W + b.double()).cpu(), (e_xh * W + 4 * U * ((xh * W).abs() + b)).cpu(), "y")
    e1 = 2 * U * gw.abs().mean(1, keepdim=True)
    e2 = (gw.abs() * (e_xh + 4 * U * xh.abs())).mean(1, keepdim=True)
    e_dx = r * (e1 + xh.abs() * e2 + e_xh * s2.abs() + 6 * U * (gw.abs() + s1.abs() + (xh * s2).abs()))
    within(dx, (r * (gw - s1 - xh * s2)).cpu(), e_dx.cpu(), "dx")
    within(dw, (DY * xh).sum(0).cpu(), (DY.abs() * (e_xh + 4 * U * xh.abs())).sum(0).cpu(), "dw")
    within(db, DY.sum(0).cpu(), (U * DY.abs().sum(0)).cpu(), "db")
