"""The sequence operators together, as a layer over a root's most recent events is trained and then served: norm, convolution,
selective scan with gate, norm, gradients of everything, clipping, update; and single events that go on where a sequence
ended."""
import numpy as np
import pytest
import torch

from gpu_common import custom_problem
from ops_common import dev, f64, rng

pytestmark = pytest.mark.gpu
EPS = 1e-5
K, D, N, W = 6, 20, 8, 4


def weights(seed):
    g = rng(seed)
    t = lambda *s, scale=1.0: dev(g.standard_normal(s) * scale, torch.float32)  # noqa: E731
    return dict(n1_w=t(D) * 0.2 + 1, n1_b=t(D, scale=0.1), conv_w=t(D, W, scale=0.5), conv_b=t(D, scale=0.1), w_dt=t(D, D, scale=0.2),
                w_bc=t(D, 2 * N, scale=0.3), w_z=t(D, D, scale=0.3), A=-torch.rand(D, N, device="cuda") * 2 - 0.1, skip=t(D), dt_bias=t(D) - 2,
                n2_w=t(D) * 0.2 + 1, n2_b=t(D, scale=0.1))


def layer(tgnn, seqs, x, p, conv_state=None, scan_state=None, conv_out=None, scan_out=None, saved=None):
    u, m1, r1 = tgnn.tgnn_layer_norm_fwd(x, p["n1_w"], p["n1_b"], EPS)
    v = tgnn.tgnn_causal_conv_fwd(seqs, u, p["conv_w"], p["conv_b"], state_in=conv_state, state_out=conv_out)
    dt, bc, z = v @ p["w_dt"], v @ p["w_bc"], u @ p["w_z"]
    y = tgnn.tgnn_selective_scan_fwd(seqs, v, dt, p["A"], bc[:, :N], bc[:, N:], D=p["skip"], z=z, dt_bias=p["dt_bias"],
                                     state_in=scan_state, state_out=scan_out, saved=saved)
    out, m2, r2 = tgnn.tgnn_layer_norm_fwd(y, p["n2_w"], p["n2_b"], EPS)
    return out, (x, u, m1, r1, v, dt, bc, z, y, m2, r2)


def layer_backward(tgnn, seqs, dout, kept, p, saved=None):
    x, u, m1, r1, v, dt, bc, z, y, m2, r2 = kept
    g = {}
    dy, g["n2_w"], g["n2_b"] = tgnn.tgnn_layer_norm_bwd(dout, y, m2, r2, p["n2_w"])
    s = tgnn.tgnn_selective_scan_bwd(seqs, dy, v, dt, p["A"], bc[:, :N], bc[:, N:], D=p["skip"], z=z, dt_bias=p["dt_bias"], saved=saved)
    g["A"], g["skip"], g["dt_bias"] = s["dA"], s["dD"], s["ddt_bias"]
    dbc = torch.cat([s["dB"], s["dC"]], 1)
    g["w_dt"], g["w_bc"], g["w_z"] = v.t() @ s["ddt"], v.t() @ dbc, u.t() @ s["dz"]
    dv = s["dx"] + s["ddt"] @ p["w_dt"].t() + dbc @ p["w_bc"].t()
    du, g["conv_w"], g["conv_b"] = tgnn.tgnn_causal_conv_bwd(seqs, dv, u, p["conv_w"], p["conv_b"])
    dx, g["n1_w"], g["n1_b"] = tgnn.tgnn_layer_norm_bwd(du + s["dz"] @ p["w_z"].t(), x, m1, r1, p["n1_w"])
    return dx, g


def reference(x, orders, p):
    """The layer in 64 bits, for autograd: rows of sequences, in rows' order."""
    def norm(v, w, b):
        return (v - v.mean(-1, keepdim=True)) / torch.sqrt(v.var(-1, unbiased=False, keepdim=True) + EPS) * w + b
    out = []
    for order in orders:
        if not order:
            continue
        u = norm(x[order], p["n1_w"], p["n1_b"])
        pad = torch.cat([torch.zeros(W - 1, D, dtype=torch.float64), u])
        pre = sum(pad[j:j + len(order)] * p["conv_w"][:, j] for j in range(W)) + p["conv_b"]
        v = torch.nn.functional.silu(pre)
        dt = torch.nn.functional.softplus(v @ p["w_dt"] + p["dt_bias"])
        bc, z = v @ p["w_bc"], u @ p["w_z"]
        h = torch.zeros(D, N, dtype=torch.float64)
        ys = []
        for i in range(len(order)):
            h = torch.exp(dt[i][:, None] * p["A"]) * h + (dt[i] * v[i])[:, None] * bc[i, :N]
            ys.append((h * bc[i, N:]).sum(1) + p["skip"] * v[i])
        y = torch.stack(ys) * torch.nn.functional.silu(z)
        out.append((order, norm(y, p["n2_w"], p["n2_b"])))
    return out


def sampled(tgnn):
    """A root's most recent events, as the sampler hands them out, and their features."""
    P = custom_problem(n_nodes=40, E=300, d_mem=8, d_time=4, d_edge=D, d_static=0, n_heads=1, k=K, batch=30)
    d = P["d"]
    ctx = tgnn.Context(d.n_nodes, d.d_mem, d.d_time, d.d_edge, d.d_static, d.n_heads, d.k, d.batch)
    graph = tgnn.Graph(P["src"], P["dst"], P["ts"], d.n_nodes, P["efeat"])
    roots = torch.arange(40, dtype=torch.int32, device="cuda")
    when = torch.from_numpy(np.linspace(P["ts"][0], P["ts"][-1], 40)).cuda()      # the first ones have no events yet
    nbr, eid, ts, cnt = ctx.tgnn_sample_recent(graph, roots, when)
    x = graph.efeat[eid.clamp(min=0).long().view(-1)] * 3
    x[(eid < 0).view(-1)] = float("nan")       # padding is never read
    seqs = tgnn.Seqs(40 * K, 40, K, cnt=cnt, newest_first=True)
    counts = cnt.cpu().tolist()
    assert 0 in counts and K in counts and len(set(counts)) > 2
    return ctx, seqs, x, [[s * K + c - 1 - i for i in range(c)] for s, c in enumerate(counts)]


@pytest.mark.parametrize("keep", [True, False])
def test_a_training_step(keep):
    from paper_2307_07649_amd import tgnn
    ctx, seqs, x, orders = sampled(tgnn)
    p = weights(1)
    valid = torch.zeros(len(x), dtype=torch.bool)
    valid[[r for o in orders for r in o]] = True
    dout = dev(rng(2).standard_normal(x.shape), torch.float32)
    dout[~valid.cuda()] = 0
    # the norm takes row by row what it is given; rows that are nobody's have to be numbers for the products around it
    x[~valid.cuda()] = 0
    saved = tgnn.selective_scan_saved(seqs, p["A"]) if keep else None
    out, kept = layer(tgnn, seqs, x, p, saved=saved)
    dx, g = layer_backward(tgnn, seqs, dout, kept, p, saved)
    X = f64(x).requires_grad_()
    R = {k: f64(v).requires_grad_() for k, v in p.items()}
    loss = 0.0
    for order, ref in reference(X, orders, R):
        # 1e-4 of the largest value, as every result of the library is held to
        assert (f64(out)[order] - ref).abs().max() <= 1e-4 * ref.abs().max()
        loss = loss + (ref * f64(dout)[order]).sum()
    loss.backward()
    for k, v in g.items():
        # (rows of no sequence: the second norm's bias there meets a gradient of zero)
        assert (f64(v) - R[k].grad).abs().max() <= 1e-4 * R[k].grad.abs().max(), k
    assert (f64(dx) - X.grad).abs().max() <= 1e-4 * X.grad.abs().max() and (dx[~valid.cuda()] == 0).all()
    # clipped and taken
    names = sorted(g)
    total = float(torch.sqrt(sum((f64(g[k]) ** 2).sum() for k in names)))
    want = {k: f64(p[k]) - 0.1 * f64(g[k]) * (0.5 * total / total) for k in names}
    norm = tgnn.tgnn_clip_grads([g[k] for k in names], 0.5 * total)
    assert abs(float(norm) - total) <= 1e-6 * total
    for k in names:
        p[k] -= 0.1 * g[k]
        assert (f64(p[k]) - want[k]).abs().max() <= 1e-6 * (1 + want[k].abs().max())


def test_single_events_go_on_where_sequences_ended():
    """A prompt of some events and single ones behind it: the same outputs as all of them as one sequence."""
    from paper_2307_07649_amd import tgnn
    p = weights(3)
    S, first, more = 5, [7, 0, 40, 1, 3], 4
    g = rng(4)
    hist = [dev(g.standard_normal((n + more, D)), torch.float32) for n in first]
    whole = torch.cat(hist)
    ends = np.concatenate([[0], np.cumsum([n + more for n in first])])
    seqs = tgnn.Seqs(len(whole), S, max(first) + more, indptr=torch.from_numpy(ends.astype(np.int64)).cuda())
    ref, _ = layer(tgnn, seqs, whole, p)
    slots = torch.tensor([4, 9, 0, 2, 7], dtype=torch.int32, device="cuda")
    conv, scan = torch.zeros(10, W - 1, D, device="cuda"), torch.zeros(10, D, N, device="cuda")
    prompt = torch.cat([h[:n] for h, n in zip(hist, first)])
    ends = np.concatenate([[0], np.cumsum(first)])
    seqs = tgnn.Seqs(len(prompt), S, max(first), indptr=torch.from_numpy(ends.astype(np.int64)).cuda())
    u, _, _ = tgnn.tgnn_layer_norm_fwd(prompt, p["n1_w"], p["n1_b"], EPS)
    v = tgnn.tgnn_causal_conv_fwd(seqs, u, p["conv_w"], p["conv_b"], state_out=conv, state_idx=slots)
    bc = v @ p["w_bc"]
    tgnn.tgnn_selective_scan_fwd(seqs, v, v @ p["w_dt"], p["A"], bc[:, :N], bc[:, N:], D=p["skip"], z=u @ p["w_z"], dt_bias=p["dt_bias"],
                                 state_out=scan, state_idx=slots)
    starts = np.cumsum([0] + [n + more for n in first])[:-1] + np.array(first)
    for i in range(more):
        x = torch.stack([h[n + i] for h, n in zip(hist, first)])
        u, _, _ = tgnn.tgnn_layer_norm_fwd(x, p["n1_w"], p["n1_b"], EPS)
        v = tgnn.tgnn_causal_conv_step(u, p["conv_w"], p["conv_b"], state_in=conv, state_out=conv, state_idx=slots)
        bc = v @ p["w_bc"]
        y = tgnn.tgnn_selective_scan_step(v, v @ p["w_dt"], p["A"], bc[:, :N], bc[:, N:], D=p["skip"], z=u @ p["w_z"], dt_bias=p["dt_bias"],
                                          state_in=scan, state_out=scan, state_idx=slots)
        out, _, _ = tgnn.tgnn_layer_norm_fwd(y, p["n2_w"], p["n2_b"], EPS)
        want = ref[torch.from_numpy(starts + i).cuda()]
        assert (out - want).abs().max() <= 1e-4 * want.abs().max(), i


def test_two_calls_at_once_and_a_captured_step():
    """Two streams work on different sequences at the same time; a captured training step gives the eager one's bits on every
    replay, with other work in between."""
    from paper_2307_07649_amd import tgnn
    ctx, seqs, x, orders = sampled(tgnn)
    x = torch.nan_to_num(x)
    p = weights(5)
    dout = dev(rng(6).standard_normal(x.shape), torch.float32)
    x2 = x.flip(0).contiguous()

    def step(x):
        saved = tgnn.selective_scan_saved(seqs, p["A"])
        out, kept = layer(tgnn, seqs, x, p, saved=saved)
        dx, g = layer_backward(tgnn, seqs, dout, kept, p, saved)
        norm = tgnn.tgnn_clip_grads([g[k] for k in sorted(g)], 1e-2)
        return [out, dx, norm] + [g[k] for k in sorted(g)]
    first, second = [t.clone() for t in step(x)], [t.clone() for t in step(x2)]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(a):
            ra = step(x)
        with torch.cuda.stream(b):
            rb = step(x2)
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(ra, first)) and all(torch.equal(u, v) for u, v in zip(rb, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x)
    for _ in range(3):
        for t in out:
            t.fill_(3)
        graph.replay()
        assert all(torch.equal(u, v) for u, v in zip(out, first))
        assert all(torch.equal(u, v) for u, v in zip(step(x2), second))
        torch.cuda.synchronize()
