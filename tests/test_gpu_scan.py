"""Selective scan: forward, backward and single events against the recurrence in 64 bits, with error bounds carried along."""
import numpy as np
import pytest
import torch

from ops_common import TYPES, U, dev, f64, rng, wide_rows, within
from seq_common import lists, on_gpu, packed, places, poison, scan_reference

pytestmark = pytest.mark.gpu


def inputs(q, d, n, groups, kind, seed, z=True, D=True, bias=True, softplus=True, state=True, n_states=None, idx=None):
    g = rng(seed)
    rows, T = q["n_rows"], TYPES[kind]
    t = dict(x=dev(g.standard_normal((rows, d)), T), dt=dev(g.standard_normal((rows, d)) * 0.7 - (0 if softplus else 0.0), T),
             B=dev(g.standard_normal((rows, groups * n)), T), C=dev(g.standard_normal((rows, groups * n)), T),
             A=dev(-g.uniform(0.2, 3.0, (d, n)) * np.arange(1, n + 1) ** 0.5, torch.float32))
    if not softplus:
        t["dt"] = dev(g.uniform(0.01, 0.4, (rows, d)), T)
    if z:
        t["z"] = dev(g.standard_normal((rows, d)), T)
    if D:
        t["D"] = dev(g.standard_normal(d), torch.float32)
    if bias:
        t["dt_bias"] = dev(g.uniform(-4, 0, d) if softplus else g.uniform(0, 0.1, d), torch.float32)
    if state:
        t["state_in"] = dev(g.standard_normal((n_states or q["n_seqs"], d, n)), torch.float32)
    dy = dev(g.standard_normal((rows, d)), T)
    return t, dy


def ref_of(q, t, dy, groups, softplus=True, idx=None, **kw):
    p = {k: f64(v) for k, v in t.items() if k != "state_in"}
    p.update(groups=groups, softplus=softplus)
    if "state_in" in t:
        st = f64(t["state_in"])
        if idx is not None:
            st = torch.stack([st[i] if 0 <= i < len(st) else torch.zeros_like(st[0]) for i in idx])
        p["state"] = st
    return scan_reference(places(**q), p, f64(dy) if dy is not None else None, **kw)


def compare(got, ref, names, label, q=None):
    """q: rows outside its slots are looked at elsewhere (check_rows_outside)."""
    for k in names:
        keep = slice(None)
        if q is not None and k not in ("dA", "dD", "ddt_bias"):
            keep = sorted(r for order, rest in places(**q) for r in order + rest)
        within(got[k][keep], ref[k].v[keep], ref[k].e[keep], f"{label} {k}")


def run(tgnn, q, t, dy, softplus=True, saved=True, idx=None, seqs=None, **grads):
    """Forward with the final states, backward; rows of no sequence are NaN in the inputs and 7 in the outputs' buffers."""
    seqs = seqs or on_gpu(tgnn, q)
    rows = [k for k in ("x", "dt", "B", "C", "z") if k in t]
    t = {**t, **{k: poison(t[k].clone(), q) for k in rows}}
    dy = poison(dy.clone(), q)
    so = torch.full_like(t["state_in"], 5.0) if "state_in" in t else None
    sv = tgnn.selective_scan_saved(seqs, t["A"]) if saved else None
    kw = dict(softplus=softplus, state_idx=idx, saved=sv)
    y = tgnn.tgnn_selective_scan_fwd(seqs, **t, **kw, state_out=so, out=torch.full_like(t["x"], 7.0))
    out = {"d" + k: torch.full_like(t[k], 7.0) for k in rows}
    g = tgnn.tgnn_selective_scan_bwd(seqs, dy, **t, **kw, **grads, out=out)
    return dict(g, y=y, state=so)


def names_of(t):
    return (["y", "dx", "ddt", "dB", "dC", "dA"] + ["dz"] * ("z" in t) + ["dD"] * ("D" in t) + ["ddt_bias"] * ("dt_bias" in t))


def check_rows_outside(q, got, names):
    """Padding rows are zero, rows behind the last slot as they were."""
    slots = torch.zeros(q["n_rows"], dtype=torch.bool)
    pad = torch.zeros(q["n_rows"], dtype=torch.bool)
    for order, rest in places(**q):
        slots[order] = True; slots[rest] = True; pad[rest] = True
    for k in names:
        if got[k].shape[0] == q["n_rows"] and k not in ("dA", "dD", "ddt_bias"):
            assert (got[k].cpu()[pad] == 0).all() and (got[k].cpu()[~slots] == 7).all(), k


SHAPES = [  # d, states, groups
    (1, 1, 1), (7, 3, 1), (16, 4, 1), (65, 5, 1), (64, 8, 2), (100, 16, 1), (130, 16, 1), (96, 16, 3), (33, 17, 1), (24, 32, 1), (70, 40, 2), (20, 64, 1)]


@pytest.mark.parametrize("d,n,groups", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_recent_events(kind, d, n, groups):
    """Lists as the sampler hands them out, newest first: full, empty, of one event."""
    from paper_2307_07649_amd import tgnn
    q = lists([10, 0, 1, 3, 10, 7, 4, 5, 8], 10)
    t, dy = inputs(q, d, n, groups, kind, d * 131 + n)
    got = run(tgnn, q, t, dy)
    ref = ref_of(q, t, dy, groups)
    compare(got, ref, names_of(t), f"{kind} {d} {n} {groups}", q)
    for s in range(q["n_seqs"]):
        within(got["state"][s], ref["state"][s].v, ref["state"][s].e, f"state {s}")
    check_rows_outside(q, got, names_of(t))


@pytest.mark.parametrize("d,n,groups", [(7, 3, 1), (65, 16, 1), (130, 16, 2), (34, 20, 2), (18, 64, 1)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_histories_in_segments(kind, d, n, groups):
    """Few long sequences: cut into segments; lengths around the segment and the saved states' distance; rows behind the last."""
    from paper_2307_07649_amd import tgnn
    q = packed([150, 0, 1, 32, 33, 31, 64, 65, 2, 97], behind=5)
    t, dy = inputs(q, d, n, groups, kind, d + n)
    assert tgnn._lib.tgnn_selective_scan_workspace_bytes(on_gpu(tgnn, q).c, d, n, groups, 0, 0) > 0      # in segments
    got = run(tgnn, q, t, dy)
    ref = ref_of(q, t, dy, groups)
    compare(got, ref, names_of(t), f"{kind} {d} {n}", q)
    for s in range(q["n_seqs"]):
        within(got["state"][s], ref["state"][s].v, ref["state"][s].e, f"state {s}")
    check_rows_outside(q, got, names_of(t))


@pytest.mark.parametrize("d,n", [(65, 16), (9, 33)])
def test_histories_whole(d, n):
    """The same in one walk (a call that says its sequences are short), and with the states formed again."""
    from paper_2307_07649_amd import tgnn
    q = packed([150, 0, 1, 32, 33, 31, 64, 65, 2, 97], behind=5)
    t, dy = inputs(q, d, n, 1, "f32", d + n)
    seqs = on_gpu(tgnn, q, max_len=8)
    assert tgnn._lib.tgnn_selective_scan_workspace_bytes(seqs.c, d, n, 1, 0, 0) == 0
    ref = ref_of(q, t, dy, 1)
    for saved in (True, False):
        got = run(tgnn, q, t, dy, seqs=seqs, saved=saved)
        compare(got, ref, names_of(t), "whole", q)
        check_rows_outside(q, got, names_of(t))
    got = run(tgnn, q, t, dy, saved=False)     # in segments, without saved states
    compare(got, ref, names_of(t), "segments", q)


@pytest.mark.parametrize("z,D,bias,softplus,state", [(0, 1, 1, 1, 1), (1, 0, 1, 1, 0), (0, 0, 0, 0, 0), (1, 1, 0, 1, 1), (1, 1, 1, 0, 1)])
def test_optional_parts(z, D, bias, softplus, state):
    from paper_2307_07649_amd import tgnn
    for q in (lists([5, 0, 6, 1], 6, newest_first=False), packed([90, 3, 0, 40])):
        t, dy = inputs(q, 20, 6, 2, "f32", 3, z=z, D=D, bias=bias, softplus=bool(softplus), state=state)
        got = run(tgnn, q, t, dy, softplus=bool(softplus))
        ref = ref_of(q, t, dy, 2, softplus=bool(softplus))
        assert set(names_of(t)) == set(got) - {"state"}
        compare(got, ref, names_of(t), "optional", q)


@pytest.mark.parametrize("z,D,bias,softplus,state", [(0, 1, 1, 1, 1), (1, 0, 0, 1, 0), (0, 0, 0, 0, 1), (1, 1, 1, 0, 0)])
@pytest.mark.parametrize("n", [17, 47, 64])
def test_many_states(n, z, D, bias, softplus, state):
    """More states than a workgroup of the backward pass takes at once: their sums are joined; several column tiles, padding."""
    from paper_2307_07649_amd import tgnn
    for q in (lists([5, 0, 6, 1, 3], 6), packed([90, 3, 0, 40], behind=3)):
        t, dy = inputs(q, 142, n, 2, "f32", n, z=z, D=D, bias=bias, softplus=bool(softplus), state=state)
        got = run(tgnn, q, t, dy, softplus=bool(softplus))
        compare(got, ref_of(q, t, dy, 2, softplus=bool(softplus)), names_of(t), f"{n} states", q)
        check_rows_outside(q, got, ["y", "dx", "ddt", "dB", "dC"] + ["dz"] * z)


def test_many_short_lists():
    """More pieces than workgroups, several column tiles: every one of the partial sums is used."""
    from paper_2307_07649_amd import tgnn
    g = rng(9)
    q = lists(list(g.integers(0, 3, 1300)), 2)
    t, dy = inputs(q, 70, 2, 1, "f32", 4, state=False)
    got = run(tgnn, q, t, dy)
    compare(got, ref_of(q, t, dy, 1), names_of(t), "many", q)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_strided_rows_and_odd_addresses(kind):
    from paper_2307_07649_amd import tgnn
    q = packed([40, 2, 90])
    t, dy = inputs(q, 33, 5, 1, kind, 11)
    ref = ref_of(q, t, dy, 1)
    seqs = on_gpu(tgnn, q)
    rows = ("x", "dt", "B", "C", "z")
    w = {**t, **{k: wide_rows(t[k], 3, 1) for k in rows}}
    y = tgnn.tgnn_selective_scan_fwd(seqs, **w, out=wide_rows(torch.zeros_like(t["x"]), 5, 3, fill=7.0))
    out = {"d" + k: wide_rows(torch.zeros_like(t[k]), 5, 3, fill=7.0) for k in rows}
    g = tgnn.tgnn_selective_scan_bwd(seqs, wide_rows(dy, 3, 1), **w, out=out)
    compare(dict(g, y=y), ref, names_of(t), "strided", q)
    for v in [y] + list(out.values()):
        assert (v.as_strided((v.shape[0] - 1, 5), (v.stride(0), 1), v.storage_offset() + v.shape[1]) == 7.0).all()


def test_gradients_in_columns_of_one_buffer():
    """y beside z, dB beside dC and dx beside ddt, as one product reads them."""
    from paper_2307_07649_amd import tgnn
    q = packed([40, 2, 90])
    t, dy = inputs(q, 33, 20, 1, "f32", 12)
    ref = ref_of(q, t, dy, 1)
    seqs, (rows, d), n = on_gpu(tgnn, q), t["x"].shape, t["B"].shape[1]
    zy = torch.full((rows, 2 * d), 7.0, device="cuda")
    zy[:, :d] = t["z"]
    y = tgnn.tgnn_selective_scan_fwd(seqs, **{**t, "z": zy[:, :d]}, out=zy[:, d:])
    bc, xdt = torch.full((rows, 2 * n), 7.0, device="cuda"), torch.full((rows, 2 * d), 7.0, device="cuda")
    out = dict(dB=bc[:, :n], dC=bc[:, n:], ddt=xdt[:, :d], dx=xdt[:, d:], dz=torch.empty_like(t["z"]))
    g = tgnn.tgnn_selective_scan_bwd(seqs, dy, **t, out=out)
    compare(dict(g, y=y), ref, names_of(t), "columns", q)
    assert (zy[:, :d] == t["z"]).all()


def test_more_wavefronts_than_a_grid_has_threads_along_x():
    """2^32 threads and more: 2^26 + 5 lists of one event, one column, one state (y = C delta x B), over sequences and as single events."""
    from paper_2307_07649_amd import tgnn
    n = (1 << 26) + 5
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dt, B, C = (torch.rand(n, 1, device="cuda", generator=g) + 0.5 for _ in range(4))
    A = torch.full((1, 1), -1.0, device="cuda")
    ref = dt * x * B * C
    for y in (tgnn.tgnn_selective_scan_fwd(tgnn.Seqs(n, n, 1), x, dt, A, B, C, softplus=False),
              tgnn.tgnn_selective_scan_step(x, dt, A, B, C, softplus=False)):
        # three roundings each, and those of three more fused steps that add zero
        assert ((y - ref).abs() <= 9 * U * ref.abs()).all()
        del y


def test_states_by_index():
    """Sequences on the states of nodes: any order, none for an index outside; states that nobody refers to stay."""
    from paper_2307_07649_amd import tgnn
    q = packed([3, 80, 0, 7, 5])
    idx = [11, 0, 5, -1, 99]
    t, dy = inputs(q, 10, 4, 1, "f32", 2, n_states=12)
    dev_idx = torch.tensor(idx, dtype=torch.int32, device="cuda")
    got = run(tgnn, q, t, dy, idx=dev_idx)
    ref = ref_of(q, t, dy, 1, idx=idx)
    compare(got, ref, names_of(t), "idx", q)
    for s, i in enumerate(idx):
        if 0 <= i < 12:
            within(got["state"][i], ref["state"][s].v, ref["state"][s].e, f"state {i}")
    rest = [i for i in range(12) if i not in idx]
    assert (got["state"][rest] == 5.0).all()
    assert torch.equal(got["state"][5], t["state_in"][5])        # an empty sequence hands its state on


def test_bad_ranges_and_counts_are_empty():
    """Slots outside the rows and counts outside the slot: nothing is read or written for them."""
    from paper_2307_07649_amd import tgnn
    q = dict(n_rows=30, n_seqs=4, max_len=12, indptr=torch.tensor([-5, 8, 20, 27, 44]), cnt=torch.tensor([3, 12, -1, 2], dtype=torch.int32))
    t, dy = inputs(q, 8, 4, 1, "f32", 6)
    got = run(tgnn, q, t, dy)
    compare(got, ref_of(q, t, dy, 1), names_of(t), "bad", q)
    check_rows_outside(q, got, names_of(t))
    q = lists([3, 11, -2, 10], 10)      # 11 is more than the slot has
    t, dy = inputs(q, 8, 4, 1, "f32", 6)
    got = run(tgnn, q, t, dy)
    compare(got, ref_of(q, t, dy, 1), names_of(t), "bad counts", q)
    check_rows_outside(q, got, names_of(t))


def test_nothing_at_all():
    from paper_2307_07649_amd import tgnn
    for q in (lists([], 10), packed([0, 0, 0]), lists([0, 0], 4), packed([0], behind=3)):
        t, dy = inputs(q, 8, 4, 1, "f32", 6)
        got = run(tgnn, q, t, dy)
        assert all((got[k] == 0).all() for k in ("dA", "dD", "ddt_bias"))
        assert torch.equal(got["state"], t["state_in"])
        check_rows_outside(q, got, names_of(t))


def test_gradients_are_added():
    from paper_2307_07649_amd import tgnn
    q = lists([4, 2, 0, 6], 6)
    t, dy = inputs(q, 12, 5, 1, "f32", 8)
    ref = ref_of(q, t, dy, 1)
    start = {k: dev(rng(5).standard_normal(s), torch.float32) for k, s in (("dA", (12, 5)), ("dD", 12), ("ddt_bias", 12))}
    given = {k: v.clone() for k, v in start.items()}
    got = run(tgnn, q, t, dy, **given)
    for k in given:
        assert got[k] is given[k]
        within(got[k], ref[k].v + f64(start[k]), ref[k].e + 2.0 ** -24 * (ref[k].v.abs() + f64(start[k]).abs()), k)


def test_gradients_against_differences():
    """Of the 64-bit recurrence, by central differences in single inputs and weights."""
    from paper_2307_07649_amd import tgnn
    q = lists([5, 3], 6)
    t, dy = inputs(q, 4, 3, 2, "f32", 21)
    got = run(tgnn, q, t, dy)

    def loss(name, i, step):
        p = {k: f64(v) for k, v in t.items()}
        p["state"] = p.pop("state_in")
        p[name].view(-1)[i] += step
        p.update(groups=2)
        return float((scan_reference(places(**q), p)["y"].v * f64(dy))[[0, 1, 2, 3, 4, 6, 7, 8]].sum())
    for name, grad in (("x", "dx"), ("dt", "ddt"), ("B", "dB"), ("C", "dC"), ("z", "dz"), ("A", "dA"), ("D", "dD"), ("dt_bias", "ddt_bias")):
        for i in (0, 3):
            want = (loss(name, i, 1e-5) - loss(name, i, -1e-5)) / 2e-5
            assert abs(float(got[grad].view(-1)[i]) - want) < 2e-4 * (1 + abs(want)), name


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d,n,groups", [(1, 1, 1, 1), (3, 7, 3, 1), (200, 32, 16, 1), (5, 100, 16, 2), (9, 30, 5, 3), (4, 66, 17, 1), (2, 20, 64, 2),
                                             (1030, 12, 2, 1)])
def test_single_events(kind, rows, d, n, groups):
    from paper_2307_07649_amd import tgnn
    q = lists([1] * rows, 1, newest_first=False)
    t, _ = inputs(q, d, n, groups, kind, rows + d)
    ref = ref_of(q, t, None, groups)
    so = torch.empty_like(t["state_in"])
    y = tgnn.tgnn_selective_scan_step(**t, state_out=so)
    within(y, ref["y"].v, ref["y"].e, "step")
    want = torch.stack([s.v for s in ref["state"]])
    within(so, want, torch.stack([s.e for s in ref["state"]]), "state")
    own = t["state_in"].clone()          # in place
    y2 = tgnn.tgnn_selective_scan_step(**{**t, "state_in": own}, state_out=own)
    assert torch.equal(y, y2) and torch.equal(own, so)


def test_single_events_by_index_without_gate_and_state():
    from paper_2307_07649_amd import tgnn
    q = lists([1] * 6, 1, newest_first=False)
    idx = [3, 40, 0, -7, 8, 5]
    t, _ = inputs(q, 9, 6, 1, "f32", 1, z=False, D=False, n_states=9)
    ref = ref_of(q, t, None, 1, idx=idx)
    so = torch.full_like(t["state_in"], 5.0)
    y = tgnn.tgnn_selective_scan_step(**t, state_out=so, state_idx=torch.tensor(idx, dtype=torch.int32, device="cuda"))
    within(y, ref["y"].v, ref["y"].e, "idx")
    for s, i in enumerate(idx):
        if 0 <= i < 9:
            within(so[i], ref["state"][s].v, ref["state"][s].e, f"state {i}")
    assert (so[[1, 2, 4, 6, 7]] == 5.0).all()
    t.pop("state_in")
    y = tgnn.tgnn_selective_scan_step(**t)
    within(y, ref_of(q, t, None, 1)["y"].v, ref_of(q, t, None, 1)["y"].e, "no state")
    e = torch.empty(0, 9, device="cuda")
    assert tgnn.tgnn_selective_scan_step(e, e, t["A"], torch.empty(0, 6, device="cuda"), torch.empty(0, 6, device="cuda")).shape == (0, 9)


def test_infinite_and_missing_numbers_stay_in_their_sequence():
    from paper_2307_07649_amd import tgnn
    q = packed([5, 6, 7])
    t, dy = inputs(q, 6, 4, 1, "f32", 14)
    clean = run(tgnn, q, t, dy)
    for value in (float("nan"), float("inf")):
        t2 = {**t, "x": t["x"].clone()}
        t2["x"][7, 2] = value
        got = run(tgnn, q, t2, dy)
        for k in ("y", "dx", "ddt", "dz", "dB", "dC"):
            keep = torch.tensor([0, 1, 2, 3, 4] + list(range(11, 18)))
            assert torch.equal(got[k][keep], clean[k][keep])
        assert not torch.isfinite(got["y"][7, 2]) and torch.equal(got["y"][5:11, [0, 1, 3, 4, 5]], clean["y"][5:11, [0, 1, 3, 4, 5]])


def test_same_result_every_time_streams_and_graphs():
    from paper_2307_07649_amd import tgnn
    q = packed([300, 20, 0, 141])
    t, dy = inputs(q, 70, 16, 1, "bf16", 5)
    seqs = on_gpu(tgnn, q)
    so = torch.empty_like(t["state_in"])

    def both():
        sv = tgnn.selective_scan_saved(seqs, t["A"])
        y = tgnn.tgnn_selective_scan_fwd(seqs, **t, saved=sv, state_out=so)
        g = tgnn.tgnn_selective_scan_bwd(seqs, dy, **t, saved=sv)
        return [y, so] + [g[k] for k in sorted(g)]
    first = [v.clone() for v in both()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = [v.clone() for v in both()]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
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


@pytest.mark.parametrize("n,saved", [(16, False), (40, True), (64, False)])
def test_two_captured_calls_of_their_own_workspaces(n, saved):
    """Two graphs of different calls, replayed in turn and on two streams at once: neither finds the other's scratch memory."""
    from paper_2307_07649_amd import tgnn
    calls = []
    for seed, q in ((1, packed([210, 0, 33])), (2, packed([9, 120, 77, 1]))):
        t, dy = inputs(q, 70, n, 1, "f32", seed)
        calls.append((on_gpu(tgnn, q), t, dy))

    def run_one(seqs, t, dy):
        sv = tgnn.selective_scan_saved(seqs, t["A"]) if saved else None
        y = tgnn.tgnn_selective_scan_fwd(seqs, **t, saved=sv)
        g = tgnn.tgnn_selective_scan_bwd(seqs, dy, **t, saved=sv)
        return [y] + [g[k] for k in sorted(g)]
    first = [[v.clone() for v in run_one(*c)] for c in calls]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(run_one(*c))
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for o in outs:
            for v in o:
                v.fill_(3)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, f in zip(outs, first):
            assert all(torch.equal(a, b) for a, b in zip(o, f))
        again = run_one(*calls[0])
        assert all(torch.equal(a, b) for a, b in zip(again, first[0]))
