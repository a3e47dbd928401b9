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


def make_seqs(tgnn, n_rows=40, n_seqs=4, max_len=10, indptr=None, cnt=None, newest_first=0):
    return tgnn.tgnn_seqs(indptr, cnt, n_rows, n_seqs, max_len, newest_first)


CONV = (["seqs", "dtype", "d", "width", "x", "ld_x", "weight", "bias", "silu", "state_in", "state_out", "state_idx", "n_states", "y", "ld_y", "stream"],
        [None, 0, 8, 4, P, 8, S, S, 1, Q, R, None, 4, S + 4096, 8, None])
STEP = (["dtype", "rows"] + CONV[0][2:], [0, 4] + CONV[1][2:])
CONV_BWD = (["seqs", "dtype", "d", "width", "dy", "ld_dy", "x", "ld_x", "weight", "bias", "silu", "state_in", "state_idx", "n_states", "dx", "ld_dx", "dw",
             "db", "acc", "ws", "ws_bytes", "stream"],
            [None, 0, 8, 4, P, 8, Q, 8, S, S, 1, S + 8192, None, 4, R, 8, S, S, 0, S, 1 << 20, None])

SEQS_BAD = [(dict(n_seqs=-1), INVALID, "negative"), (dict(max_len=-1), INVALID, "negative"), (dict(n_rows=-1), INVALID, "negative"),
            (dict(newest_first=2), INVALID, "newest_first"), (dict(indptr=P + 4), MISALIGNED, "indptr"), (dict(cnt=P + 2), MISALIGNED, "cnt"),
            (dict(max_len=11), RANGE, "do not fit"), (dict(n_rows=1 << 33, indptr=P), RANGE, "rows"),
            (dict(n_rows=(1 << 33) - 1, n_seqs=(1 << 31) - 1, indptr=P), RANGE, "sequences")]


@pytest.mark.parametrize("seqs,code,word", SEQS_BAD)
def test_sequences(tgnn, seqs, code, word):
    for name, (names, args) in (("tgnn_causal_conv_fwd", CONV), ("tgnn_causal_conv_bwd", CONV_BWD)):
        rc, msg = call(tgnn, name, args, names, seqs=make_seqs(tgnn, **seqs))
        assert rc == code and word in msg, (name, rc, msg)
    q = make_seqs(tgnn, **seqs)
    p = make_scan(tgnn)
    assert tgnn._lib.tgnn_selective_scan_fwd(q, p, R, 8, None, None, 0, S, 1 << 20, None) == code
    assert tgnn._lib.tgnn_selective_scan_bwd(q, p, P, 8, None, 0, make_grads(tgnn), 0, S, 1 << 20, None) == code
    assert tgnn._lib.tgnn_selective_scan_saved_bytes(q, 8, 4) == code
    assert tgnn._lib.tgnn_selective_scan_workspace_bytes(q, 8, 4, 1, 0, 0) == code


CONV_BAD = [(dict(dtype=9), INVALID, "dtype"), (dict(d=0), DIM, "d = 0"), (dict(d=65537), DIM, "d ="), (dict(width=0), DIM, "width"), (dict(width=9), DIM, "width"),
            (dict(weight=None), NULL, "weight"), (dict(weight=S + 2), MISALIGNED, "weight"), (dict(x=None), NULL, "x"), (dict(ld_x=7), INVALID, "rows of x"),
            (dict(n_states=-1), INVALID, "n_states"), (dict(state_in=Q + 2), MISALIGNED, "state"), (dict(state_idx=P + 1), MISALIGNED, "state_idx")]


@pytest.mark.parametrize("over,code,word", CONV_BAD + [
    (dict(y=None), NULL, "y"), (dict(ld_y=2), INVALID, "rows of y"), (dict(y=P), INVALID, "y overlaps x"), (dict(state_out=Q), INVALID, "state_out overlaps"),
    (dict(state_out=Q + 4 * 3 * 8 * 4 - 4), INVALID, "state_out overlaps")])
def test_conv_fwd(tgnn, over, code, word):
    rc, msg = call(tgnn, "tgnn_causal_conv_fwd", CONV[1], CONV[0], **{"seqs": make_seqs(tgnn), **over})
    assert rc == code and word in msg, (rc, msg)
    assert call(tgnn, "tgnn_causal_conv_fwd", CONV[1], CONV[0], seqs=None)[0] == NULL


@pytest.mark.parametrize("over,code,word", CONV_BAD + [
    (dict(rows=-1), RANGE, "n_rows"), (dict(rows=1 << 31), RANGE, "n_rows"), (dict(y=P + 4), INVALID, "without being it"), (dict(y=P, ld_y=9), INVALID, "without being it"),
    (dict(state_out=Q + 4), INVALID, "without being it")])
def test_conv_step(tgnn, over, code, word):
    rc, msg = call(tgnn, "tgnn_causal_conv_step", STEP[1], STEP[0], **over)
    assert rc == code and word in msg, (rc, msg)


@pytest.mark.parametrize("over,code,word", CONV_BAD + [
    (dict(dy=None), NULL, "dy"), (dict(dx=None), NULL, "dx"), (dict(dx=Q), INVALID, "overlaps"), (dict(dx=P), INVALID, "overlaps"), (dict(ws=None), NULL, "workspace"),
    (dict(ws=S + 4), MISALIGNED, "workspace"), (dict(ws_bytes=8), WORKSPACE, "needed"), (dict(dw=S + 1), MISALIGNED, "d_weight")])
def test_conv_bwd(tgnn, over, code, word):
    rc, msg = call(tgnn, "tgnn_causal_conv_bwd", CONV_BWD[1], CONV_BWD[0], **{"seqs": make_seqs(tgnn), **over})
    assert rc == code and word in msg, (rc, msg)


def make_scan(tgnn, **over):
    v = dict(dtype=0, d=8, n_state=4, n_groups=2, softplus=1, n_states=4, x=P, dt=P, B=P, C=P, z=P, ld_x=8, ld_dt=8, ld_b=8, ld_c=8, ld_z=8, A=Q, D=Q, dt_bias=Q,
             state_in=Q, state_idx=None)
    assert not set(over) - set(v)
    return tgnn.tgnn_scan(**{**v, **over})


def make_grads(tgnn, **over):
    v = dict(dx=R, ddt=R, dB=R, dC=R, dz=R, ld_dx=8, ld_ddt=8, ld_db=8, ld_dc=8, ld_dz=8, dA=S, dD=S, ddt_bias=S)
    return tgnn.tgnn_scan_grads(**{**v, **over})


@pytest.mark.parametrize("over,code,word", [
    (dict(dtype=-1), INVALID, "dtype"), (dict(d=0), DIM, "d = 0"), (dict(d=65538), DIM, "d ="), (dict(n_state=0), DIM, "n_state"), (dict(n_state=65), DIM, "n_state"),
    (dict(n_groups=3), DIM, "groups"), (dict(n_groups=0), DIM, "groups"), (dict(x=None), NULL, "x"), (dict(dt=None), NULL, "dt"), (dict(B=None), NULL, "B"),
    (dict(C=None), NULL, "C"), (dict(A=None), NULL, "A"), (dict(A=Q + 1), MISALIGNED, "A"), (dict(z=P + 2), MISALIGNED, "z"), (dict(ld_b=7), INVALID, "rows of B"),
    (dict(ld_x=1), INVALID, "rows of x"), (dict(state_in=Q + 2), MISALIGNED, "state_in"), (dict(n_states=-2), INVALID, "n_states")])
def test_scan_inputs(tgnn, over, code, word):
    q, p = make_seqs(tgnn), make_scan(tgnn, **over)
    lib = tgnn._lib
    for rc in (lib.tgnn_selective_scan_fwd(q, p, R, 8, None, None, 0, S, 1 << 20, None), lib.tgnn_selective_scan_step(p, 4, R, 8, None, None),
               lib.tgnn_selective_scan_bwd(q, p, P, 8, None, 0, make_grads(tgnn), 0, S, 1 << 20, None)):
        assert rc == code and word in lib.tgnn_last_error().decode(), (rc, lib.tgnn_last_error())


def test_scan_outputs_and_workspaces(tgnn):
    lib, q, p, g = tgnn._lib, make_seqs(tgnn), make_scan(tgnn), make_grads(tgnn)

    def fwd(y=R, ld=8, so=None, sv=None, svb=0, ws=S, wsb=1 << 20, q=q, p=p):
        return lib.tgnn_selective_scan_fwd(q, p, y, ld, so, sv, svb, ws, wsb, None)
    assert fwd(y=None) == NULL and fwd(y=R + 2) == MISALIGNED and fwd(ld=7) == INVALID and fwd(y=P) == INVALID
    assert fwd(so=Q) == INVALID and fwd(so=Q + 4 * 8 * 4 * 4 - 4) == INVALID and fwd(so=S + 1) == MISALIGNED
    assert fwd(sv=S + 4) == MISALIGNED and fwd(sv=S, svb=100) == WORKSPACE and fwd(p=None) == NULL and fwd(q=None) == NULL
    long = make_seqs(tgnn, n_rows=4000, n_seqs=1, max_len=4000)
    need = lib.tgnn_selective_scan_workspace_bytes(long, 8, 4, 2, 0, 0)
    assert need > 0 and fwd(q=long, ws=None) == NULL and fwd(q=long, y=R + (1 << 19), ws=S, wsb=need - 1) == WORKSPACE and fwd(q=long, ws=S + 8, wsb=need) == MISALIGNED

    def step(rows=4, y=R, so=None, p=p):
        return lib.tgnn_selective_scan_step(p, rows, y, 8, so, None)
    assert step(rows=-1) == RANGE and step(rows=1 << 31) == RANGE and step(y=None) == NULL and step(y=P) == INVALID and step(so=Q + 4) == INVALID

    def bwd(dy=P, sv=None, svb=0, g=g, ws=S, wsb=1 << 20, p=p):
        return lib.tgnn_selective_scan_bwd(q, p, dy, 8, sv, svb, g, 0, ws, wsb, None)
    assert bwd(dy=None) == NULL and bwd(g=None) == NULL and bwd(ws=None) == NULL and bwd(ws=S + 4) == MISALIGNED and bwd(wsb=64) == WORKSPACE
    assert bwd(sv=S + 4) == MISALIGNED and bwd(sv=S, svb=4) == WORKSPACE
    for k in ("dx", "ddt", "dB", "dC", "dz"):
        assert bwd(g=make_grads(tgnn, **{k: None})) == NULL and bwd(g=make_grads(tgnn, **{k: P})) == INVALID, k
    assert bwd(g=make_grads(tgnn, ld_db=3)) == INVALID and bwd(g=make_grads(tgnn, dA=S + 2)) == MISALIGNED
    assert lib.tgnn_selective_scan_saved_bytes(q, 8, 65) == DIM and lib.tgnn_selective_scan_workspace_bytes(q, 8, 4, 3, 0, 0) == DIM


@pytest.mark.parametrize("cols", [(1 << 28) + 1, (1 << 31) - 1])
def test_layer_norm_columns(tgnn, cols):
    for name, (names, args) in (("tgnn_layer_norm_fwd", FWD), ("tgnn_layer_norm_bwd", BWD)):
        rc, msg = call(tgnn, name, args, names, rows=1, cols=cols)
        assert rc == DIM and "n_cols" in msg


def test_scan_gradients_apart(tgnn):
    """Gradients of one call share no memory (40 rows of 8 columns)."""
    lib, q, p = tgnn._lib, make_seqs(tgnn), make_scan(tgnn)
    at = {k: R + i * 4096 for i, k in enumerate(("dx", "ddt", "dB", "dC", "dz"))}
    for a, b in (("ddt", "dx"), ("dC", "dB"), ("dz", "ddt")):
        pitch = {"ld_" + a.lower(): 16, "ld_" + b.lower(): 16}
        # the same place; its first column is the other's last; its last column is the other's first of the next row
        for over in ({a: at[b]}, {a: at[b] + 28, **pitch}, {a: at[b] + 36, **pitch}):
            rc = lib.tgnn_selective_scan_bwd(q, p, P, 8, None, 0, make_grads(tgnn, **{**at, **over}), 0, S, 1 << 20, None)
            assert rc == INVALID and f"{a} overlaps {b}" in lib.tgnn_last_error().decode(), (a, over)


def test_outputs_beside_inputs(tgnn):
    """An output in other columns of an input's buffer does not overlap it; one column further it does."""
    lib, q = tgnn._lib, make_seqs(tgnn, n_rows=4000, n_seqs=1, max_len=4000)
    p = make_scan(tgnn, ld_x=16, dt=Q, B=Q, C=Q, z=Q, A=S, D=S, dt_bias=S, state_in=None)
    for off in (28, 36, -28, 64 * 7 + 20):
        assert lib.tgnn_selective_scan_fwd(q, p, P + off, 16, None, None, 0, None, 0, None) == INVALID, off
        assert "y overlaps" in lib.tgnn_last_error().decode()
    for off in (32, -32, 64 * 7 + 32):      # (what is refused is the workspace that is not there)
        assert lib.tgnn_selective_scan_fwd(q, p, P + off, 16, None, None, 0, None, 0, None) == NULL, off
        assert "workspace" in lib.tgnn_last_error().decode()


def test_struct_sizes(tgnn):
    assert C.sizeof(tgnn.tgnn_seqs) == 40 and C.sizeof(tgnn.tgnn_scan) == 24 + 15 * 8 and C.sizeof(tgnn.tgnn_scan_grads) == 13 * 8


def test_the_binding_refuses_sequences_and_states_that_do_not_fit(tgnn):
    with pytest.raises(ValueError, match="indptr"):
        tgnn.Seqs(10, 2, 5, indptr=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="cnt"):
        tgnn.Seqs(10, 2, 5, cnt=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="current GPU"):
        tgnn.Seqs(10, 2, 5, cnt=torch.zeros(2, dtype=torch.int32))
    x, A = torch.zeros(10, 8), torch.zeros(8, 4)
    q = tgnn.Seqs(10, 2, 5)
    for bad in (torch.zeros(2, 8, 5), torch.zeros(2, 8, 4, dtype=torch.float64), torch.zeros(2, 4, 8).transpose(1, 2)):
        with pytest.raises(ValueError, match="state_in"):
            tgnn.tgnn_selective_scan_fwd(q, x, x, A, x, x, state_in=bad)
    with pytest.raises(ValueError, match="rows"):
        tgnn.tgnn_selective_scan_fwd(q, torch.zeros(9, 8), x, A, x, x)
    with pytest.raises(ValueError, match="rows"):
        tgnn.tgnn_causal_conv_fwd(q, torch.zeros(9, 8), torch.zeros(8, 4))
