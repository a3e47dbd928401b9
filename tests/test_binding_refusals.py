"""What the binding refuses before it hands anything to the library: no GPU is touched."""
import types

import pytest
import torch

BIG = (1 << 32) + 100        # 100 in its low 32 bits


@pytest.fixture(scope="module")
def tgnn():
    from paper_2307_07649_amd import tgnn as t
    return t


def meta(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="meta")       # a shape without memory


@pytest.mark.parametrize("over", [dict(n_seqs=BIG), dict(max_len=BIG), dict(n_seqs=1 << 31), dict(max_len=-(1 << 31) - 1)])
def test_sequences_that_32_bits_do_not_count(tgnn, over):
    with pytest.raises(ValueError, match="32 bits"):
        tgnn.Seqs(**{**dict(n_rows=BIG, n_seqs=1, max_len=1), **over})
    q = tgnn.Seqs(BIG, (1 << 31) - 1, (1 << 31) - 1)
    assert (q.c.n_rows, q.c.n_seqs, q.c.max_len) == (BIG, (1 << 31) - 1, (1 << 31) - 1)


def test_columns_that_32_bits_do_not_count(tgnn):
    x, q = meta(1, BIG), tgnn.Seqs(1, 1, 1)
    for call in (lambda: tgnn.tgnn_layer_norm_fwd(x), lambda: tgnn.tgnn_layer_norm_bwd(x, x, meta(1), meta(1)),
                 lambda: tgnn.tgnn_causal_conv_fwd(q, x, meta(BIG, 4)), lambda: tgnn.tgnn_causal_conv_step(x, meta(BIG, 4)),
                 lambda: tgnn.tgnn_causal_conv_bwd(q, x, x, meta(BIG, 4)),
                 lambda: tgnn.tgnn_selective_scan_fwd(q, x, x, meta(BIG, 4), meta(1, 4), meta(1, 4)),
                 lambda: tgnn.tgnn_selective_scan_step(x, x, meta(BIG, 4), meta(1, 4), meta(1, 4)),
                 lambda: tgnn.tgnn_selective_scan_bwd(q, x, x, x, meta(BIG, 4), meta(1, 4), meta(1, 4)),
                 lambda: tgnn.selective_scan_saved(q, meta(BIG, 4)), lambda: tgnn.selective_scan_saved(q, meta(4, BIG))):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_states_that_32_bits_do_not_count(tgnn):
    x, q = meta(1, 8), tgnn.Seqs(1, 1, 1)
    idx = torch.zeros(1, dtype=torch.int32)
    for k in ("state_in", "state_out"):
        st = types.SimpleNamespace(shape=(BIG, 8, 4), dtype=torch.float32, is_contiguous=lambda: True, get_device=lambda: None, data_ptr=lambda: 0)
        with pytest.raises(ValueError, match="n_states"):
            tgnn.tgnn_selective_scan_fwd(q, x, x, meta(8, 4), meta(1, 4), meta(1, 4), state_idx=idx, **{k: st})


def test_where_the_steps_norm_goes(tgnn):
    """Every step writes to it: a tensor in host memory, of another type or of no element is none that it can write to."""
    ctx = types.SimpleNamespace(h=None, _clip_norm=None)
    for bad, word in ((torch.zeros(1), "current GPU"), (torch.zeros(1, dtype=torch.float64), "float32"), (torch.zeros(0), "float32"),
                      (torch.zeros(1, 1), "current GPU"), (torch.zeros(4)[::2], "contiguous")):
        with pytest.raises(ValueError, match=word):
            tgnn.Context.tgnn_set_grad_clip(ctx, 1.0, bad)
    assert ctx._clip_norm is None
    with pytest.raises(tgnn.TgnnError, match="ctx"):       # what is refused here is the context that is not there
        tgnn.Context.tgnn_set_grad_clip(ctx, 1.0, None)


def test_sequences_of_another_device(tgnn, monkeypatch):
    """Row ranges that were made on one GPU, and tensors on the one that is current now."""
    def on(dev, *shape, dtype=torch.float32):
        t = torch.empty(*shape, dtype=dtype)
        t.get_device = lambda: dev
        return t
    monkeypatch.setattr(tgnn, "_device_of", lambda t: t.get_device())
    for q in (tgnn.Seqs(4, 2, 4, indptr=on(1, 3, dtype=torch.int64)), tgnn.Seqs(4, 2, 2, cnt=on(1, 2, dtype=torch.int32))):
        x, A, B = on(0, 4, 8), on(0, 8, 4), on(0, 4, 4)
        for call in (lambda: tgnn.tgnn_causal_conv_fwd(q, x, A), lambda: tgnn.tgnn_causal_conv_bwd(q, x, x, A),
                     lambda: tgnn.tgnn_selective_scan_fwd(q, x, x, A, B, B), lambda: tgnn.tgnn_selective_scan_bwd(q, x, x, x, A, B, B)):
            with pytest.raises(ValueError, match="the sequences on cuda:1"):
                call()
