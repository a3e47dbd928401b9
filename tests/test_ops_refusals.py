"""What the sequence-layer operators refuse, before anything is launched (no GPU is touched): the C entry points' codes and
the binding's checks."""
import ctypes as C

import pytest
import torch

INVALID, NULL, MISALIGNED, RANGE, DIM, WORKSPACE = -1, -2, -3, -4, -6, -7
P, Q, R, S = 1 << 20, 2 << 20, 3 << 20, 4 << 20      # addresses that are never followed


@pytest.fixture(scope="module")
def tgnn():
    from paper_2307_07649_amd import tgnn as t
    return t


def call(tgnn, name, args, names, **over):
    unknown = set(over) - set(names)
    assert not unknown, unknown
    rc = getattr(tgnn._lib, name)(*[over.get(n, a) for n, a in zip(names, args)])
    return rc, tgnn._lib.tgnn_last_error().decode()


FWD = (["dtype", "rows", "cols", "x", "ld_x", "weight", "bias", "eps", "y", "ld_y", "mean", "rstd", "stream"],
       [0, 4, 8, P, 8, Q, Q, 1e-5, R, 8, S, S, None])
BWD = (["dtype", "rows", "cols", "dy", "ld_dy", "x", "ld_x", "mean", "rstd", "weight", "dx", "ld_dx", "dw", "db", "acc", "ws", "ws_bytes", "stream"],
       [0, 4, 8, P, 8, Q, 8, S, S, S, R, 8, S, S, 0, S, 1 << 19, None])


@pytest.mark.parametrize("over,code,word", [
    (dict(dtype=3), INVALID, "dtype"), (dict(cols=0), DIM, "n_cols"), (dict(rows=-1), RANGE, "n_rows"), (dict(rows=1 << 31), RANGE, "n_rows"),
    (dict(x=None), NULL, "x"), (dict(y=None), NULL, "y"), (dict(x=P + 2), MISALIGNED, "x"), (dict(dtype=1, y=R + 1), MISALIGNED, "y"),
    (dict(weight=Q + 2), MISALIGNED, "weight"), (dict(ld_x=7), INVALID, "rows of x"), (dict(ld_y=7), INVALID, "rows of y"),
    (dict(eps=-1e-3), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"), (dict(y=P + 4), INVALID, "overlaps"),
    (dict(y=P, ld_y=9), INVALID, "overlaps"), (dict(mean=S + 1), MISALIGNED, "out_mean")])
def test_layer_norm_fwd(tgnn, over, code, word):
    rc, msg = call(tgnn, "tgnn_layer_norm_fwd", FWD[1], FWD[0], **over)
    assert rc == code and word in msg, (rc, msg)


@pytest.mark.parametrize("over,code,word", [
    (dict(dtype=-1), INVALID, "dtype"), (dict(dy=None), NULL, "dy"), (dict(mean=None), NULL, "mean"), (dict(rstd=None), NULL, "rstd"),
    (dict(dx=Q), INVALID, "overlaps x"), (dict(dx=P + 4), INVALID, "overlaps dy"), (dict(ws=None), NULL, "workspace"),
    (dict(ws=S + 8), MISALIGNED, "workspace"), (dict(ws_bytes=100), WORKSPACE, "needed"), (dict(db=S + 3), MISALIGNED, "d_bias"),
    (dict(ld_dx=3), INVALID, "rows of dx")])
def test_layer_norm_bwd(tgnn, over, code, word):
    rc, msg = call(tgnn, "tgnn_layer_norm_bwd", BWD[1], BWD[0], **over)
    assert rc == code and word in msg, (rc, msg)


def clip_args(ptrs, numel, dtypes, max_norm=1.0, out=None, norm=S, ws=S, ws_bytes=1 << 16):
    n = len(ptrs)
    return [n, (C.c_void_p * n)(*ptrs), (C.c_int64 * n)(*numel), (C.c_int32 * n)(*dtypes), max_norm,
            (C.c_void_p * n)(*out) if out else None, norm, ws, ws_bytes, None]


@pytest.mark.parametrize("args,code,word", [
    (([P], [-1], [0]), RANGE, "numel"), (([P], [1 << 43], [0]), RANGE, "numel"), (([P], [4], [7]), INVALID, "dtype"), (([None], [4], [0]), NULL, "tensor 0"),
    (([P, Q + 1], [4, 4], [0, 1]), MISALIGNED, "tensor 1"), (([P], [4], [0], 0.0), INVALID, "max_norm"), (([P], [4], [0], -1.0), INVALID, "max_norm"),
    (([P], [4], [0], float("nan")), INVALID, "max_norm"), (([P], [4], [0], 1.0, [None]), NULL, "out[0]"), (([P], [4], [0], 1.0, [Q + 2]), MISALIGNED, "out[0]"),
    (([P, P], [4, 4], [0, 0]), INVALID, "shares"), (([P, P + 8], [4, 4], [0, 0]), INVALID, "shares"), (([P], [4], [0], 1.0, [P + 4]), INVALID, "shares"),
    (([P, Q], [4, 4], [0, 0], 1.0, [R, R]), INVALID, "shares"), (([P, Q], [4, 4], [0, 0], 1.0, [Q, R]), INVALID, "shares"),
    (([P], [4], [0], 1.0, None, None), NULL, "out_norm"), (([P], [4], [0], 1.0, None, S, None), NULL, "workspace"),
    (([P], [4], [0], 1.0, None, S, S, 8), WORKSPACE, "needed")])
def test_clip(tgnn, args, code, word):
    rc = tgnn._lib.tgnn_clip_grads(*clip_args(*args))
    msg = tgnn._lib.tgnn_last_error().decode()
    assert rc == code and word in msg, (rc, msg)


def test_norm(tgnn):
    a = clip_args([P], [4], [0])
    assert tgnn._lib.tgnn_grad_norm(a[0], None, a[2], a[3], S, S, 1 << 16, None) == NULL
    assert tgnn._lib.tgnn_grad_norm(-1, a[1], a[2], a[3], S, S, 1 << 16, None) == INVALID
    assert tgnn._lib.tgnn_grad_norm(1, a[1], a[2], a[3], S + 2, S, 1 << 16, None) == MISALIGNED
    assert tgnn._lib.tgnn_grad_norm(1, a[1], a[2], a[3], S, S, 8, None) == WORKSPACE
    assert tgnn._lib.tgnn_clip_workspace_bytes(129) == 2 * tgnn._lib.tgnn_clip_workspace_bytes(128) > 0


def test_the_binding_refuses_what_it_cannot_hand_over(tgnn):
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="current GPU"):
        tgnn.tgnn_layer_norm_fwd(x)
    with pytest.raises(ValueError, match="two-dimensional"):
        tgnn.tgnn_layer_norm_fwd(torch.zeros(8))
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        tgnn.tgnn_layer_norm_fwd(x.double())
    with pytest.raises(ValueError, match="contiguous"):
        tgnn.tgnn_layer_norm_fwd(torch.zeros(8, 4).t())
    with pytest.raises(ValueError, match="contiguous"):
        tgnn.tgnn_grad_norm([torch.zeros(8, 4).t()])
    with pytest.raises(ValueError, match="current GPU"):
        tgnn.tgnn_clip_grads([x], 1.0)
