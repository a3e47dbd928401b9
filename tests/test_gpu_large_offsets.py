"""Offsets that 32 bits do not hold: rows far apart, states far into their table, a tensor of more than 2^31 elements.  What is near and what
is far goes through the same kernels, so that the results are the same bits."""
import pytest
import torch

from ops_common import dev, rng

pytestmark = pytest.mark.gpu

LD, ROWS = 1 << 26, 70      # 70 rows of 2^26 values: the last one begins 4.6e9 values in


class Far:
    """Columns of one large buffer, next to each other."""

    def __init__(self, dtype):
        self.buf, self.at = torch.empty(ROWS * LD, dtype=dtype, device="cuda").view(ROWS, LD), 0

    def __call__(self, near):
        d = near.shape[1]
        v = self.buf[:, self.at:self.at + d]
        self.at += (d + 7) // 8 * 8
        v.copy_(near)
        return v


def values(g, d, dtype):
    return dev(g.standard_normal((ROWS, d)), dtype)


def same(a, b):
    assert torch.equal(a, b)


@pytest.mark.parametrize("n", [5, 20])
def test_scan(n):
    from paper_2307_07649_amd import tgnn
    T, g, d = torch.bfloat16, rng(1), 70
    t = {k: values(g, w, T) for k, w in (("x", d), ("dt", d), ("B", n), ("C", n), ("z", d))}
    w = dict(A=dev(-g.uniform(0.2, 2.0, (d, n)), torch.float32), D=dev(g.standard_normal(d), torch.float32))
    dy, far = values(g, d, T), Far(T)
    big = {k: far(v) for k, v in t.items()}
    for indptr in ([0, 3, 3, ROWS], [0, ROWS]):
        q = tgnn.Seqs(ROWS, len(indptr) - 1, ROWS, indptr=torch.tensor(indptr, device="cuda"))
        y, y_far = tgnn.tgnn_selective_scan_fwd(q, **t, **w), far(torch.zeros_like(dy))
        tgnn.tgnn_selective_scan_fwd(q, **big, **w, out=y_far)
        same(y, y_far)
        near = tgnn.tgnn_selective_scan_bwd(q, dy, **t, **w)
        out = {"d" + k: far(torch.zeros_like(v)) for k, v in t.items()}
        got = tgnn.tgnn_selective_scan_bwd(q, far(dy), **big, **w, out=out)
        for k in near:
            same(near[k], got[k])
    y_far = far(torch.zeros_like(dy))
    tgnn.tgnn_selective_scan_step(**big, **w, out=y_far)
    same(tgnn.tgnn_selective_scan_step(**t, **w), y_far)


def test_conv_and_norm():
    from paper_2307_07649_amd import tgnn
    T, g, d = torch.float16, rng(2), 72
    x, dy, far = values(g, d, T), values(g, d, T), Far(torch.float16)
    fx, fdy = far(x), far(dy)
    w, b = dev(g.standard_normal((d, 4)), torch.float32), dev(g.standard_normal(d), torch.float32)
    q = tgnn.Seqs(ROWS, 2, ROWS, indptr=torch.tensor([0, 9, ROWS], device="cuda"))
    out = [far(torch.zeros_like(x)) for _ in range(5)]
    tgnn.tgnn_causal_conv_fwd(q, fx, w, b, out=out[0])
    same(tgnn.tgnn_causal_conv_fwd(q, x, w, b), out[0])
    near, got = tgnn.tgnn_causal_conv_bwd(q, dy, x, w, b), tgnn.tgnn_causal_conv_bwd(q, fdy, fx, w, b, out=out[1])
    for a, c in zip(near, got):
        same(a, c)
    tgnn.tgnn_causal_conv_step(fx, w, b, out=out[2])
    same(tgnn.tgnn_causal_conv_step(x, w, b), out[2])
    y, mean, rstd = tgnn.tgnn_layer_norm_fwd(x, b, b)
    _, fm, fr = tgnn.tgnn_layer_norm_fwd(fx, b, b, out=out[3])
    for a, c in ((y, out[3]), (mean, fm), (rstd, fr)):
        same(a, c)
    near, got = tgnn.tgnn_layer_norm_bwd(dy, x, mean, rstd, b), tgnn.tgnn_layer_norm_bwd(fdy, fx, mean, rstd, b, out=out[4])
    for a, c in zip(near, got):
        same(a, c)


def test_states_far_into_their_table():
    from paper_2307_07649_amd import tgnn
    g, d, n, n_states = rng(3), 512, 64, 70_000       # 2.3e9 values
    table = torch.empty(n_states, d, n, device="cuda")
    idx = [69_999, 0, 65_536, 40_000]
    small = dev(g.standard_normal((4, d, n)), torch.float32)
    at = torch.tensor(idx, dtype=torch.int32, device="cuda")
    t = {k: dev(g.standard_normal((4, w)), torch.float32) for k, w in (("x", d), ("dt", d), ("B", n), ("C", n))}
    A = dev(-g.uniform(0.2, 2.0, (d, n)), torch.float32)
    for k, i in enumerate(idx):
        table[i] = small[k]
    ends = torch.empty_like(small)
    y = tgnn.tgnn_selective_scan_fwd(tgnn.Seqs(4, 4, 1), **t, A=A, state_in=small, state_out=ends)
    same(y, tgnn.tgnn_selective_scan_fwd(tgnn.Seqs(4, 4, 1), **t, A=A, state_in=table, state_idx=at))
    near, own = tgnn.tgnn_selective_scan_step(**t, A=A, state_in=small, state_out=ends), table
    same(near, tgnn.tgnn_selective_scan_step(**t, A=A, state_in=table, state_out=own, state_idx=at))
    for k, i in enumerate(idx):
        same(own[i], ends[k])


def test_clip_more_than_two_to_the_31_elements():
    from paper_2307_07649_amd import tgnn
    n = (1 << 31) + 5
    ones = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    norm = float(tgnn.tgnn_clip_grads([ones], 0.25 * n ** 0.5))
    assert abs(norm - n ** 0.5) <= 2.0 ** -24 * n ** 0.5        # the sum of the squares is exact
    # 0.25 but for the roundings of max_norm and of the factor: one step of a bfloat16 at most
    assert (ones[:1000] - 0.25).abs().max() <= 2.0 ** -9 and (ones[-1000:] == ones[0]).all() and (ones[n // 2: n // 2 + 1000] == ones[0]).all()
