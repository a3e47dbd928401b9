"""Causal convolution: forward, backward and single events against the formula in 64 bits, with error bounds carried along."""
import pytest
import torch

from ops_common import TYPES, dev, f64, rng, wide_rows, within
from seq_common import conv_reference, lists, on_gpu, packed, places, poison

pytestmark = pytest.mark.gpu


def inputs(q, d, width, kind, seed, bias=True, state=True, n_states=None):
    g = rng(seed)
    T = TYPES[kind]
    t = dict(x=dev(g.standard_normal((q["n_rows"], d)), T), weight=dev(g.standard_normal((d, width)), torch.float32))
    if bias:
        t["bias"] = dev(g.standard_normal(d), torch.float32)
    if state:
        t["state_in"] = dev(g.standard_normal((n_states or q["n_seqs"], width - 1, d)), T)
    return t, dev(g.standard_normal((q["n_rows"], d)), T)


def ref_of(q, t, dy, silu=True, idx=None):
    p = {k: f64(v) for k, v in t.items() if k != "state_in"}
    if "state_in" in t:
        st = f64(t["state_in"])
        p["state"] = st if idx is None else torch.stack([st[i] if 0 <= i < len(st) else torch.zeros_like(st[0]) for i in idx])
    return conv_reference(places(**q), {**p, "silu": silu}, None if dy is None else f64(dy))


def run(tgnn, q, t, dy, silu=True, idx=None, **grads):
    seqs = on_gpu(tgnn, q)
    t = {**t, "x": poison(t["x"].clone(), q)}
    dy = poison(dy.clone(), q)
    so = torch.full_like(t["state_in"], 5.0) if "state_in" in t else None
    kw = dict(silu=silu, state_idx=idx)
    y = tgnn.tgnn_causal_conv_fwd(seqs, **t, **kw, state_out=so, out=torch.full_like(t["x"], 7.0))
    dx, dw, db = tgnn.tgnn_causal_conv_bwd(seqs, dy, **t, **kw, **grads, out=torch.full_like(t["x"], 7.0))
    return dict(y=y, dx=dx, d_weight=dw, d_bias=db, state=so)


def check(q, got, ref, label, states=True):
    for k in ("y", "dx", "d_weight", "d_bias"):
        v = ref[k].v.clone()
        if k in ("y", "dx"):
            outside = torch.ones(q["n_rows"], dtype=torch.bool)
            for order, rest in places(**q):
                outside[order] = False; outside[rest] = False
            v[outside] = 7.0
        within(got[k], v, ref[k].e, f"{label} {k}")
    if states and got["state"] is not None:
        assert torch.equal(f64(got["state"]), torch.stack(ref["state"]))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,width", [(1, 2), (7, 4), (8, 1), (16, 3), (33, 5), (64, 4), (100, 4), (100, 2), (260, 8), (1028, 4), (1030, 3)])
def test_lists_and_histories(kind, d, width):
    from paper_2307_07649_amd import tgnn
    for q in (lists([10, 0, 1, 2, 3, 10, 7], 10), packed([130, 0, 1, 2, 64, 65, 63, 3], behind=4), lists([4, 0, 5], 5, newest_first=False)):
        t, dy = inputs(q, d, width, kind, d + width)
        check(q, run(tgnn, q, t, dy), ref_of(q, t, dy), f"{kind} {d} {width}")


@pytest.mark.parametrize("bias,state,silu", [(0, 0, 0), (1, 0, 1), (0, 1, 1), (1, 1, 0)])
def test_optional_parts(bias, state, silu):
    from paper_2307_07649_amd import tgnn
    q = packed([70, 0, 5])
    for width in (4, 6):
        t, dy = inputs(q, 12, width, "f32", 3, bias=bias, state=state)
        check(q, run(tgnn, q, t, dy, silu=bool(silu)), ref_of(q, t, dy, silu=bool(silu)), "optional")


def test_states_by_index_bad_ranges_and_added_gradients():
    from paper_2307_07649_amd import tgnn
    q = packed([3, 80, 0, 7, 1])
    idx = [11, 0, 5, -1, 99]
    t, dy = inputs(q, 10, 4, "f32", 2, n_states=12)
    start = (dev(rng(1).standard_normal((10, 4)), torch.float32), dev(rng(2).standard_normal(10), torch.float32))
    dw, db = (v.clone() for v in start)
    got = run(tgnn, q, t, dy, idx=torch.tensor(idx, dtype=torch.int32, device="cuda"), d_weight=dw, d_bias=db)
    ref = ref_of(q, t, dy, idx=idx)
    assert got["d_weight"] is dw and got["d_bias"] is db
    ref["d_weight"].v += f64(start[0]); ref["d_bias"].v += f64(start[1])
    check(q, got, ref, "idx", states=False)
    for s, i in enumerate(idx):
        if 0 <= i < 12:
            assert torch.equal(f64(got["state"][i]), ref["state"][s])
    assert (got["state"][[1, 2, 3, 4, 6, 7, 8, 9, 10]] == 5.0).all()
    q = dict(n_rows=30, n_seqs=4, max_len=12, indptr=torch.tensor([-5, 8, 20, 27, 44]), cnt=torch.tensor([3, 12, -1, 2], dtype=torch.int32))
    t, dy = inputs(q, 8, 4, "f32", 6)
    check(q, run(tgnn, q, t, dy), ref_of(q, t, dy), "bad")


def test_nothing_at_all():
    from paper_2307_07649_amd import tgnn
    for q in (lists([], 10), packed([0, 0, 0]), lists([0, 0], 4), packed([0], behind=3)):
        t, dy = inputs(q, 8, 4, "f32", 6)
        got = run(tgnn, q, t, dy)
        check(q, got, ref_of(q, t, dy), "nothing", states=False)
        assert torch.equal(got["state"], t["state_in"])


def test_many_short_lists_and_one_long():
    from paper_2307_07649_amd import tgnn
    g = rng(3)
    q = lists(list(g.integers(0, 4, 9000)), 3)
    t, dy = inputs(q, 3, 3, "f32", 4)
    # (the reference of 9,000 lists at once: their events are few, the sums over them long)
    got = run(tgnn, q, t, dy)
    assert torch.equal(run(tgnn, q, t, dy)["d_weight"], got["d_weight"])
    few = dict(n_rows=q["n_rows"], n_seqs=9000, max_len=3, cnt=q["cnt"], newest_first=True)
    ref = ref_of(few, t, dy)
    check(q, got, ref, "many")
    q = packed([5000])
    t, dy = inputs(q, 5, 4, "bf16", 5)
    check(q, run(tgnn, q, t, dy), ref_of(q, t, dy), "long")


@pytest.mark.parametrize("kind,d", [("f32", 32), ("bf16", 33), ("bf16", 24)])
def test_strided_rows_and_odd_addresses(kind, d):
    from paper_2307_07649_amd import tgnn
    q = packed([40, 2, 90])
    t, dy = inputs(q, d, 4, kind, 11)
    ref = ref_of(q, t, dy)
    seqs = on_gpu(tgnn, q)
    w = {**t, "x": wide_rows(t["x"], 3, 1)}
    y = tgnn.tgnn_causal_conv_fwd(seqs, **w, out=wide_rows(torch.zeros_like(t["x"]), 5, 3, fill=7.0))
    dx, dw, db = tgnn.tgnn_causal_conv_bwd(seqs, wide_rows(dy, 4, 4), **w, out=wide_rows(torch.zeros_like(t["x"]), 5, 3, fill=7.0))
    check(q, dict(y=y, dx=dx, d_weight=dw, d_bias=db, state=None), ref, "strided")
    for v in (y, dx):
        assert (v.as_strided((v.shape[0] - 1, 5), (v.stride(0), 1), v.storage_offset() + d) == 7.0).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d,width", [(1, 1, 2), (3, 7, 4), (200, 32, 4), (5, 100, 1), (9, 30, 8), (1030, 12, 3)])
def test_single_events(kind, rows, d, width):
    from paper_2307_07649_amd import tgnn
    q = lists([1] * rows, 1, newest_first=False)
    t, _ = inputs(q, d, width, kind, rows + d)
    ref = ref_of(q, t, None)
    so = torch.empty_like(t["state_in"])
    y = tgnn.tgnn_causal_conv_step(**t, state_out=so)
    within(y, ref["y"].v, ref["y"].e, "step")
    assert torch.equal(f64(so), torch.stack(ref["state"]))
    own, x = t["state_in"].clone(), t["x"].clone()          # both in place
    y2 = tgnn.tgnn_causal_conv_step(**{**t, "state_in": own, "x": x}, state_out=own, out=x)
    assert y2 is x and torch.equal(y, y2) and torch.equal(own, so)


def test_single_events_by_index():
    from paper_2307_07649_amd import tgnn
    q = lists([1] * 6, 1, newest_first=False)
    idx = [3, 40, 0, -7, 8, 5]
    t, _ = inputs(q, 9, 4, "f32", 1, n_states=9)
    ref = ref_of(q, t, None, idx=idx)
    so = torch.full_like(t["state_in"], 5.0)
    y = tgnn.tgnn_causal_conv_step(**t, state_out=so, state_idx=torch.tensor(idx, dtype=torch.int32, device="cuda"))
    within(y, ref["y"].v, ref["y"].e, "idx")
    for s, i in enumerate(idx):
        if 0 <= i < 9:
            assert torch.equal(f64(so[i]), ref["state"][s])
    assert (so[[1, 2, 4, 6, 7]] == 5.0).all()
    e = torch.empty(0, 9, device="cuda")
    assert tgnn.tgnn_causal_conv_step(e, t["weight"]).shape == (0, 9)


def test_gradients_against_differences():
    from paper_2307_07649_amd import tgnn
    q = lists([5, 3], 6)
    t, dy = inputs(q, 4, 3, "f32", 21)
    got = run(tgnn, q, t, dy)

    def loss(name, i, step):
        p = {k: f64(v) for k, v in t.items()}
        p["state"] = p.pop("state_in")
        p[name].view(-1)[i] += step
        return float((conv_reference(places(**q), p)["y"].v * f64(dy)).sum())
    for name, grad in (("x", "dx"), ("weight", "d_weight"), ("bias", "d_bias")):
        for i in (0, 3):
            want = (loss(name, i, 1e-5) - loss(name, i, -1e-5)) / 2e-5
            assert abs(float(got[grad].view(-1)[i]) - want) < 2e-4 * (1 + abs(want)), name


def test_infinities_stay_in_reach_of_the_taps():
    from paper_2307_07649_amd import tgnn
    for width in (3, 5):        # a kernel of its own, and the one for any width
        q = packed([30, 30])
        t, dy = inputs(q, 4, width, "f32", 2, state=False)
        clean = run(tgnn, q, t, dy, silu=False)
        t["x"][10, 1] = float("inf")
        got = run(tgnn, q, t, dy, silu=False)
        keep = [r for r in range(60) if not 10 <= r < 10 + width]
        assert torch.equal(got["y"][keep], clean["y"][keep]) and not torch.isfinite(got["y"][10:10 + width, 1]).any()
        assert torch.equal(got["dx"], clean["dx"])


def test_same_result_every_time_and_in_a_graph():
    from paper_2307_07649_amd import tgnn
    q = packed([300, 20, 0, 141])
    t, dy = inputs(q, 70, 4, "bf16", 5)
    seqs = on_gpu(tgnn, q)
    so = torch.empty_like(t["state_in"])

    def both():
        y = tgnn.tgnn_causal_conv_fwd(seqs, **t, state_out=so)
        return (y, so) + tgnn.tgnn_causal_conv_bwd(seqs, dy, **t)
    first = [v.clone() for v in both()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for _ in range(3):
        for v in out:
            v.fill_(3)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, first))
        assert all(torch.equal(a, b) for a, b in zip(both(), first))
        torch.cuda.synchronize()
