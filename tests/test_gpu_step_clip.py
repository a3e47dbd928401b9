"""Clipping of the in-step update (tgnn_set_grad_clip): the norm of the step's own gradients, and the update that the scaled
gradients give, for every kind of step, both optimisers, with and without a captured graph."""
import ctypes as C

import numpy as np
import pytest
import torch

from gpu_common import GpuSide, batch_np, custom_problem, rel_err
from oracle import tgnn_oracle as O

pytestmark = pytest.mark.gpu
LR = 0.05
FROZEN = ("time_w", "time_b")


def sides(G, kind, s, J=3):
    """One step of that kind on batch s -> its outputs."""
    P, d = G.P, G.d
    b = batch_np(P, s * d.batch, (s + 1) * d.batch)
    if kind == "classes":
        b["labels"] = (np.random.default_rng(s).random((d.batch, d.n_classes)) < 0.3).astype(np.float32)
        return lambda lr: G.step([b], lr=lr)
    if kind == "sets":
        b["neg"] = np.random.default_rng(s).integers(0, d.n_nodes, (J, d.batch)).astype(np.int32)
        return lambda lr: G.step([b], lr=lr, n_neg_sets=J)
    return lambda lr: G.step([b], lr=lr)


@pytest.mark.parametrize("kind,own_stream,adam", [("train", True, False), ("train", False, False), ("train", True, True), ("sets", True, False),
                                                  ("classes", True, True)])
def test_clipped_update(kind, own_stream, adam):
    from paper_2307_07649_amd import tgnn
    P = custom_problem(n_nodes=80, E=900, d_mem=24, d_time=10, d_edge=6, d_static=0, n_heads=2, k=5, batch=60,
                       **(dict(n_classes=7) if kind == "classes" else {}))
    G = GpuSide(P, own_stream=own_stream, flags=tgnn.FLAG_OVERWRITE_GRADS, max_neg_sets=3)
    m = tgnn.Params.zeros_like(G.params); v = tgnn.Params.zeros_like(G.params)
    b1, b2, eps = (float(np.float32(x)) for x in (0.9, 0.999, 1e-8))
    if adam:
        G.ctx.tgnn_set_optimizer(1, m, v, b1, b2, eps)
    norm = torch.full((1,), -1.0, device="cuda")
    for s, bound in enumerate([0.0, 1e-3, 1e-3, 1e6, 0.02, float("inf"), 0.0]):
        if s in (1, 3, 4, 5, 6):
            G.ctx.tgnn_set_grad_clip(bound, norm)
        norm.fill_(-1.0)
        before = [{n: x.astype(np.float64) for n, x in q.numpy().items()} for q in (G.params, m, v)]
        g = sides(G, kind, s)(LR)
        grads = {n: x.astype(np.float64) for n, x in g["grads"].items()}
        ref = np.sqrt(sum((grads[n] ** 2).sum() for n in grads if n not in FROZEN))
        if bound:
            assert abs(float(norm) - ref) <= 2 ** -23 * ref, (s, float(norm), ref)
        else:
            assert float(norm) == -1.0
        scale = bound / ref if bound and ref > bound else 1.0
        start = {n: x.copy() for n, x in before[0].items()}
        assert (scale < 1) == (bound in (1e-3, 0.02)), (s, ref)
        if adam:
            st = dict(m=before[1], v=before[2], t=s)
            O.adam(before[0], {n: x * scale for n, x in grads.items()}, st, LR, b1, b2, eps)
            for n in grads:
                if n not in FROZEN:
                    assert rel_err(m.numpy()[n], st["m"][n]) <= 1e-6 and rel_err(v.numpy()[n], st["v"][n]) <= 1e-6, (s, n)
        else:
            for n in grads:
                if n not in FROZEN:
                    before[0][n] -= LR * scale * grads[n]
        for n, x in G.params.numpy().items():
            # p - update is rounded once, by at most 2^-24 of p or of the update, whichever is larger before they cancel (dec_b2 has
            # one element, which a step of Adam takes from 0.05 to 0.0006); the update itself has a dozen roundings
            assert np.abs(x - before[0][n]).max() <= 1e-6 * (np.abs(start[n]).max() + np.abs(before[0][n] - start[n]).max()), (s, n)


def test_several_steps_per_call():
    """tgnn_train_steps clips every one of its steps: the same parameters as one call a step (whose sums may be in another order)."""
    from paper_2307_07649_amd import tgnn
    P = custom_problem(n_nodes=80, E=900, d_mem=24, d_time=10, d_edge=6, d_static=0, n_heads=2, k=5, batch=60)
    a, b = (GpuSide(P, flags=tgnn.FLAG_OVERWRITE_GRADS) for _ in range(2))
    for G in (a, b):
        G.ctx.tgnn_set_grad_clip(0.01)
    batches = [batch_np(P, s * 60, (s + 1) * 60) for s in range(4)]
    for x in batches:
        a.step([x], lr=LR)
    bl = [[tgnn.Batch(x["src"], x["dst"], x["neg"], x["eid"], x["t"])] for x in batches]
    loss = torch.empty(4, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(b.stream):
        b.ctx.tgnn_train_steps(b.graph, b.state, b.params, b.grads, bl, lr=LR, out_loss=loss)
    torch.cuda.synchronize()
    start = P["params"]
    for n, x in a.params.numpy().items():
        # (the four steps' moves together are at most 4 lr 0.01 in norm, their difference a few roundings of them and of the parameters)
        assert np.abs(x - b.params.numpy()[n]).max() <= 1e-5 * 4 * LR * 0.01 + 2 ** -22 * np.abs(start[n]).max(), n
    moved = np.sqrt(sum(((x.astype(np.float64) - start[n]) ** 2).sum() for n, x in a.params.numpy().items()))
    # (of all tensors together: the key bias has a gradient of zero.  Every element rounded four times: 2^-24 of at most |start| each)
    slack = 4 * 2 ** -24 * np.sqrt(sum((start[n].astype(np.float64) ** 2).sum() for n in start))
    assert slack < moved <= 4 * LR * 0.01 * (1 + 1e-5) + slack


def test_refusals():
    from paper_2307_07649_amd import tgnn
    P = custom_problem(n_nodes=20, E=100, d_mem=8, d_time=4, d_edge=2, d_static=0, n_heads=1, k=3, batch=10)
    G = GpuSide(P)
    for bad in (-1.0, float("nan")):
        with pytest.raises(tgnn.TgnnError) as e:
            G.ctx.tgnn_set_grad_clip(bad)
        assert e.value.code == -1
    assert tgnn._lib.tgnn_set_grad_clip(None, 1.0, None) == -2
    assert tgnn._lib.tgnn_set_grad_clip(G.ctx.h, 1.0, C.c_void_p(G.loss.data_ptr() + 2)) == -3
