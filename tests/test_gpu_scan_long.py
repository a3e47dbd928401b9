"""The scan over sequences long enough for every way of cutting them: segments longer than the distance of saved states, and the walk between
segments in runs."""
import pytest
import torch

from ops_common import within
from seq_common import lists, on_gpu, packed
from test_gpu_scan import SHAPES, check_rows_outside, compare, inputs, names_of, ref_of, run

pytestmark = pytest.mark.gpu


def segment_bits(rows, longest, units, spread, fill):
    """How a call cuts its sequences (None: not at all): segments of the power of two nearest to what leaves `fill` units of work for
    each of `spread` places, if the whole walks take longer than everything nearly twice."""
    work, bits = rows * units // spread, 5
    while bits < 12 and (3 << bits) // 2 <= work // fill:
        bits += 1
    return bits if max(min(longest, rows), work) > work + work * 4 // 5 + 40 + (1 << bits) else None


def plan(q, d, n, groups):
    """(bits forward, bits backward), of which the sizes of the library's workspaces have to be what they lead to."""
    dg = d // groups
    slices, tiles = -(-n // 16), -(-dg // 64)
    up = lambda floats: -(-4 * floats // 256) * 256  # noqa: E731
    segments = lambda bits: (q["n_rows"] >> bits) + q["n_seqs"]  # noqa: E731
    fwd = segment_bits(q["n_rows"], q["max_len"], groups * -(-dg // 64), 1024, 6)
    units = groups * tiles * slices
    bwd = segment_bits(q["n_rows"], q["max_len"], units, 256, 5)
    need_fwd = 0 if fwd is None else up(segments(fwd) * d * n) + up(segments(fwd) * d)
    items = q["n_seqs"] if bwd is None else segments(bwd)
    workers = max(1, min(items, 1024, 2560 // units))
    need_bwd = 0 if bwd is None else up(segments(bwd) * d * n) + up(segments(bwd) * d)
    need_bwd += up(workers * (d * n + 2 * d))
    assert slices == 1 and tiles == 1
    from paper_2307_07649_amd import tgnn
    c = on_gpu(tgnn, q).c
    assert tgnn._lib.tgnn_selective_scan_workspace_bytes(c, d, n, groups, 0, 0) == need_fwd
    assert tgnn._lib.tgnn_selective_scan_workspace_bytes(c, d, n, groups, 1, 1) == need_bwd
    return fwd, bwd


def check(q, d, n, groups, kind, seed, segment, saved=(True, False), **kw):
    """`segment`: events whose step sizes are summed up in float before an exponential of the sum."""
    from paper_2307_07649_amd import tgnn
    t, dy = inputs(q, d, n, groups, kind, seed, **kw)
    ref = ref_of(q, t, dy, groups, segment=segment)
    for s in saved:
        got = run(tgnn, q, t, dy, saved=s)
        compare(got, ref, names_of(t), f"{kind} saved {s}", q)
        if "state_in" in t:
            for i in range(q["n_seqs"]):
                within(got["state"][i], ref["state"][i].v, ref["state"][i].e, f"state {i}")
        check_rows_outside(q, got, names_of(t))


@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("newest_first", [False, True])
def test_walk_between_segments_in_runs(state, newest_first):
    """More than 64 segments of 32 events in the longest sequence: eight threads share a column's walk, with 79 segments, 65 (one of a single
    event), one and none.  32 step sizes are summed up in a segment, and ten of those sums in a thread's run."""
    q = dict(packed([2500, 0, 1, 2049], behind=3), newest_first=newest_first)
    assert plan(q, 3, 2, 1) == (5, 5) and q["max_len"] > 64 << 5
    check(q, 3, 2, 1, "f32", 5, 64, state=state)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_segments_longer_than_the_distance_of_saved_states(kind):
    """100 groups of one column each are work enough for segments of 128 events forward and 512 backward; lengths off both."""
    q = packed([5300, 0, 333, 1, 400], behind=2)
    assert plan(q, 100, 2, 100) == (7, 9)
    check(q, 100, 2, 100, kind, 6, 512, saved=(True,) if kind == "bf16" else (True, False))


def test_long_segments_in_runs():
    """Both: 70 segments of 64 events backward, and 140 of 32 forward."""
    q = packed([4470, 31])
    assert plan(q, 14, 1, 14) == (5, 6) and q["max_len"] > 64 << 6
    check(q, 14, 1, 14, "f32", 7, 96)


@pytest.mark.parametrize("d,n,groups", SHAPES)
def test_recent_events_in_float16(d, n, groups):
    from paper_2307_07649_amd import tgnn
    q = lists([10, 0, 1, 3, 10, 7, 4, 5, 8], 10)
    t, dy = inputs(q, d, n, groups, "f16", d * 131 + n)
    got = run(tgnn, q, t, dy)
    compare(got, ref_of(q, t, dy, groups), names_of(t), f"{d} {n} {groups}", q)
    check_rows_outside(q, got, names_of(t))
