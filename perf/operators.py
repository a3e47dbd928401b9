"""Timed calls of the sequence-layer operators, taken through the public binding (paper_2307_07649_amd.tgnn): the selective
state space scan and its short causal convolution over lists of a root's most recent events, over whole event histories and
for single events, layer norm with its backward pass, and the global gradient norm with clipping.

A case is a dict of plain values.  `prepare` draws what a program holds before the call, `run` is one call (a training case:
forward and backward), in the framework's kernels where `own` is set and otherwise in elementary torch operations in 32 bits,
rounded once at the end; `exact` is the definition in 64 bits, one event after the other.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def listed():
    return [
        # the newest event of a few nodes, the smallest memory width of the benchmark: launches and latency
        dict(name="scan-step-live", path="scan-step", dtype="f32", rows=200, width=32, states=16, groups=1, table=0),
        # a large batch's events, one per node, on the states of all nodes of the dense graph
        dict(name="scan-step-table", path="scan-step", dtype="bf16", rows=4000, width=256, states=16, groups=1, table=16_682),
        # every root of a 4,000-event batch over its ten most recent events, as the sampler hands them out
        dict(name="scan-recent", path="scan", dtype="f32", layout="recent", seqs=12_000, longest=10, width=100, states=16, groups=1),
        # whole histories of the busiest nodes, of very different lengths
        dict(name="scan-histories", path="scan", dtype="bf16", layout="packed", seqs=32, longest=4001, width=1024, states=16,
             groups=1),
        # training over recent events at the usual batch size of 600 events
        dict(name="scan-train-recent", path="scan-train", dtype="f32", layout="recent", seqs=1800, longest=10, width=100,
             states=16, groups=1),
        # training over a few long histories
        dict(name="scan-train-long", path="scan-train", dtype="bf16", layout="packed", seqs=3, longest=8191, width=512, states=16,
             groups=2),
        # single events through the convolution
        dict(name="conv-step-table", path="conv-step", dtype="f16", rows=4000, width=1024, taps=4, table=16_682),
        # the convolution in front of the scan, trained
        dict(name="conv-train-histories", path="conv-train", dtype="bf16", layout="packed", seqs=32, longest=4001, width=1024,
             taps=4),
        # norm of every slot's row of a 4,000-event batch (roots and ten neighbours each), forward and backward
        dict(name="norm-train-slots", path="norm-train", dtype="f32", rows=132_000, width=100),
        # wide rows, in 16 bits
        dict(name="norm-train-wide", path="norm-train", dtype="bf16", rows=8191, width=4096),
        # gradients of one model with the usual widths: nineteen small tensors
        dict(name="clip-model", path="clip", dtype="f32", tensors=0, elements=0),
        # gradients of several hundred tensors, some of them in 16 bits
        dict(name="clip-many", path="clip", dtype="mixed", tensors=300, elements=200_000_000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: lists of up to 32 recent events and histories of up to 8,191, widths 8 to 1,024, 1 to 64
    states, 2 to 8 taps, rows of 1 to 8,192 values, 1 to 400 gradient tensors."""
    path = rng.choice(["scan-step", "scan", "scan", "scan-train", "scan-train", "conv-step", "conv-train", "norm-train", "clip"])
    c = dict(path=path, dtype=rng.choice(["f32", "bf16", "f16"]))
    if path == "clip":
        c["dtype"] = rng.choice(["f32", "mixed"])
        c["tensors"] = _log_int(rng, 1, 400)
        c["elements"] = max(c["tensors"], _log_int(rng, 1000, 200_000_000))
        return c
    if path == "norm-train":
        c["width"] = _log_int(rng, 1, 8192)
        c["rows"] = _log_int(rng, 1, min(200_000, 33_000_000 // c["width"]))
        return c
    scan = path.startswith("scan")
    c["width"] = _log_int(rng, 8, 1024)
    if scan:
        c["states"] = rng.choice([16, 16, 16, rng.randint(1, 64)])
        c["groups"] = rng.choice([g for g in (1, 1, 2, 4) if c["width"] % g == 0])
    else:
        c["taps"] = rng.choice([4, 4, 3, 2, rng.randint(2, 8)])
    per_row = c["width"] * (c["states"] if scan else 4)
    if path.endswith("step"):
        c["rows"] = _log_int(rng, 1, max(2, min(8000, 16_000_000 // per_row)))
        c["table"] = rng.choice([0, c["rows"] + _log_int(rng, 1, 8000)])
        return c
    most = {"scan": 500_000_000, "scan-train": 64_000_000, "conv-train": 120_000_000}[path] // per_row
    c["layout"] = rng.choice(["recent", "packed"])
    if c["layout"] == "recent":
        c["longest"] = rng.randint(1, 32)
        c["seqs"] = _log_int(rng, 1, max(2, min(14_400, most // c["longest"])))
    else:
        c["longest"] = _log_int(rng, 1, max(2, min(8191, most // 2)))
        c["seqs"] = _log_int(rng, 1, max(2, min(2000, most // c["longest"])))
    return c


def _lengths(case):
    """Lengths of a case's sequences, the same for every seed up to their order: most lists of recent events are full; the
    histories' lengths are far apart, with one as long as named, and an empty one and one of a single event among them."""
    n, longest = case["seqs"], case["longest"]
    rng = np.random.RandomState((n * 8191 + longest) % (1 << 31))
    u = rng.random_sample(n)
    if case["layout"] == "recent":
        return np.where(u < 0.75, longest, rng.randint(0, longest + 1, n)).astype(np.int32)
    lens = np.floor((longest + 1) * u ** 3).astype(np.int64)
    lens[0] = longest
    if n > 2:
        lens[1:3] = 0, 1
    return lens


def _tensor_sizes(case):
    if case["tensors"] == 0:   # memory, time-encoding and edge-feature widths 100, 100, 172
        m, t, e = 100, 100, 172
        g, q, kv = 2 * m + t + e, m + t, m + e + t
        return [t, t, 3 * m * g, 3 * m * m, 3 * m, 3 * m, m * q, m, m * kv, m, m * kv, m, m * 2 * m, m, m * m, m * m, m, m, 1]
    rng = np.random.RandomState(case["tensors"] + case["elements"] % 99_991)
    share = np.exp(rng.uniform(0, math.log(1e4), case["tensors"]))
    return [max(1, int(v)) for v in share / share.sum() * case["elements"]]


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 31))

    def normal(*shape, scale=1.0, to=None):
        v = torch.randn(*shape, generator=g, device="cuda")
        return (v * scale).to(to or dtype)

    def uniform(*shape, lo, hi):
        return torch.rand(*shape, generator=g, device="cuda") * (hi - lo) + lo

    path, f32 = case["path"], torch.float32
    s = {"path": path}
    if path == "clip":
        sizes = _tensor_sizes(case)
        kinds = [torch.bfloat16 if case["dtype"] == "mixed" and i % 3 == 1 else f32 for i in range(len(sizes))]
        # a trainer's flat buffers, one of each type, and the tensors in them, at multiples of 16 bytes
        at, ends = [], {f32: 0, torch.bfloat16: 0}
        for n, k in zip(sizes, kinds):
            at.append(ends[k])
            ends[k] += (n + 7) // 8 * 8
        flat = {k: torch.zeros(n, dtype=k, device="cuda") for k, n in ends.items() if n}
        for k, buf in flat.items():
            buf.copy_(torch.randn(buf.numel(), generator=g, device="cuda") * 0.01)
        s["grads"] = [flat[k][a:a + n] for a, n, k in zip(at, sizes, kinds)]
        s["flat"] = list(flat.values())
        outs = {k: torch.zeros_like(v) for k, v in flat.items()}
        s["out"], s["out_flat"] = [outs[k][a:a + n] for a, n, k in zip(at, sizes, kinds)], list(outs.values())
        for k, buf in flat.items():   # nothing between the tensors
            keep = torch.zeros(buf.numel(), dtype=torch.bool, device="cuda")
            for a, n, kind in zip(at, sizes, kinds):
                if kind == k:
                    keep[a:a + n] = True
            buf.mul_(keep)
        s["max_norm"] = 1.0 if sum(sizes) > 20_000 else 0.1
        return s
    dtype = DTYPES[case["dtype"]]
    d = case["width"]
    if path == "norm-train":
        s["x"] = (torch.randn(case["rows"], d, generator=g, device="cuda") * 1.5 + uniform(case["rows"], 1, lo=-2, hi=2)).to(dtype)
        s["dy"] = normal(case["rows"], d)
        s["weight"], s["bias"] = uniform(d, lo=0.5, hi=1.5), normal(d, scale=0.1, to=f32)
        return s
    if path.endswith("step"):
        rows = case["rows"]
        slots = case["table"] or rows
        s["idx"] = torch.from_numpy(rng.permutation(slots)[:rows].astype(np.int32)).cuda() if case["table"] else None
    else:
        lens = rng.permutation(_lengths(case))
        s["seqs"], s["longest"], s["newest_first"] = case["seqs"], case["longest"], case["layout"] == "recent"
        if s["newest_first"]:
            rows, s["indptr"], s["cnt"] = case["seqs"] * case["longest"], None, torch.from_numpy(lens).cuda()
        else:
            rows = max(1, int(lens.sum()))
            s["indptr"], s["cnt"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)).cuda(), None
        slots = case["seqs"]
    if path.startswith("conv"):
        taps = case["taps"]
        s["x"] = normal(rows, d)
        s["weight"], s["bias"] = normal(d, taps, scale=taps ** -0.5, to=f32), normal(d, scale=0.1, to=f32)
        s["state"] = normal(slots, taps - 1, d)
        s["state_out"] = torch.zeros_like(s["state"])
        if path == "conv-train":
            s["dy"] = normal(rows, d)
        return s
    n, grp = case["states"], case["groups"]
    # x and its gate are the two halves of one projection's rows, dt a product of its own, B and C two parts of another's
    xz, bc = normal(rows, 2 * d), normal(rows, 2 * grp * n)
    s["x"], s["z"], s["B"], s["C"] = xz[:, :d], xz[:, d:], bc[:, :grp * n], bc[:, grp * n:]
    s["dt"] = normal(rows, d, scale=0.5)
    s["A"] = -(torch.arange(1, n + 1, device="cuda") * uniform(d, n, lo=0.8, hi=1.25)).contiguous()
    step = torch.exp(uniform(d, lo=math.log(1e-3), hi=math.log(0.1)))
    s["dt_bias"] = torch.log(torch.expm1(step))
    s["D"] = normal(d, to=f32)
    s["state"] = normal(slots, d, n, scale=0.5, to=f32)
    s["state_out"] = torch.zeros_like(s["state"])
    s["groups"] = grp
    if path == "scan-train":
        s["dy"] = normal(rows, d)
    return s


# ---- the operators' plain forms ----
def _spans(s):
    """First row and length of every sequence."""
    if s["indptr"] is None:
        return torch.arange(s["seqs"], device="cuda") * s["longest"], s["cnt"].long()
    return s["indptr"][:-1], s["indptr"][1:] - s["indptr"][:-1]


def _rows_of(s):
    """Of every row: its sequence, its place in time there, and whether it belongs to one."""
    r = torch.arange(s["x"].shape[0], device="cuda")
    begin, length = _spans(s)
    if s["indptr"] is None:
        seq = r // s["longest"]
    else:
        seq = (torch.searchsorted(s["indptr"], r, right=True) - 1).clamp(max=s["seqs"] - 1)
    off, length = r - begin[seq], length[seq]
    return seq, length - 1 - off if s["newest_first"] else off, off < length


def _recur(a, b, longest):
    """h[r] = a[r] h[r - 1] + b[r] over the rows, by doubling; a is zero where a sequence begins."""
    for i in range(max(0, (longest - 1).bit_length())):
        k = 1 << i
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
    return b


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def _plain_scan(s, train):
    to, longest, grp = s["x"].dtype, s["longest"], s["groups"]
    d, n = s["A"].shape
    seq, t, valid = _rows_of(s)
    flip = (lambda v: v.flip(0)) if s["newest_first"] else (lambda v: v)   # rows in time order
    seq, t, valid = flip(seq), flip(t), flip(valid)
    first, on = valid & (t == 0), valid[:, None]

    def rows(name):
        return torch.where(on, flip(s[name]).float(), 0.0)

    def spread(v):   # a group's values for each of its columns
        return v.view(-1, grp, 1, n).expand(-1, grp, d // grp, n).reshape(-1, d, n)

    x, z, raw, Bs, Cs = rows("x"), rows("z"), rows("dt") + s["dt_bias"], spread(rows("B")), spread(rows("C"))
    delta = torch.where(on, _softplus(raw), 0.0)
    a = torch.exp(delta[:, :, None] * s["A"])
    h0 = s["state"][seq]
    b = (delta * x)[:, :, None] * Bs
    go = torch.where(first[:, None, None], b + a * h0, b)
    goes_on = (valid & ~first)[:, None, None]
    h = _recur(torch.where(goes_on, a, 0.0), go, longest)
    y0 = (h * Cs).sum(-1) + s["D"] * x
    gate = z * _sigmoid(z)
    out = {"y": flip((y0 * gate).to(to))}
    begin, length = _spans(s)
    final = len(t) - 1 - begin if s["newest_first"] else begin + length - 1   # the row, in time order, that a sequence ends with
    out["state"] = torch.where((length > 0)[:, None, None], h[final.clamp(0, len(t) - 1)], s["state"])
    if not train:
        return out
    dy = rows("dy")
    sg = _sigmoid(z)
    gy = dy * gate
    ahead = torch.cat([torch.where(goes_on, a, 0.0)[1:], torch.zeros_like(a[:1])])
    lam = _recur(ahead.flip(0), (gy[:, :, None] * Cs).flip(0), longest).flip(0)
    before = torch.cat([h0[:1], h[:-1]])
    ah = a * torch.where(first[:, None, None], h0, before)
    s1, s2 = (lam * Bs).sum(-1), (s["A"] * lam * ah).sum(-1)
    ddelta = torch.where(on, x * s1 + s2, 0.0)
    draw_ = ddelta * _sigmoid(raw)
    per_group = lambda v: v.view(-1, grp, d // grp, n).sum(2).reshape(-1, grp * n)  # noqa: E731
    out.update(
        dx=flip((s["D"] * gy + delta * s1).to(to)), ddt=flip(draw_.to(to)), dz=flip((dy * y0 * sg * (1 + z * (1 - sg))).to(to)),
        dB=flip(per_group(torch.where(on[:, :, None], lam * (delta * x)[:, :, None], 0.0)).to(to)),
        dC=flip(per_group(gy[:, :, None] * h).to(to)),
        dA=torch.where(on[:, :, None], delta[:, :, None] * lam * ah, 0.0).sum(0, dtype=torch.float64).float(),
        dD=(gy * x).sum(0, dtype=torch.float64).float(), ddt_bias=draw_.sum(0, dtype=torch.float64).float())
    return out


def _plain_scan_step(s):
    to, grp = s["x"].dtype, s["groups"]
    d, n = s["A"].shape
    x, z, Bs, Cs = (s[k].float() for k in ("x", "z", "B", "C"))
    delta = _softplus(s["dt"].float() + s["dt_bias"])
    Bs, Cs = (v.view(-1, grp, 1, n).expand(-1, grp, d // grp, n).reshape(-1, d, n) for v in (Bs, Cs))
    h0 = s["state"] if s["idx"] is None else s["state"][s["idx"].long()]
    h = torch.exp(delta[:, :, None] * s["A"]) * h0 + (delta * x)[:, :, None] * Bs
    y = ((h * Cs).sum(-1) + s["D"] * x) * z * _sigmoid(z)
    if s["idx"] is None:
        s["state_out"].copy_(h)
    else:
        s["state_out"][s["idx"].long()] = h
    return {"y": y.to(to), "state": s["state_out"]}


def _plain_conv_step(s):
    to = s["x"].dtype
    h0 = s["state"] if s["idx"] is None else s["state"][s["idx"].long()]
    win = torch.cat([h0, s["x"][:, None]], 1)
    pre = (win.float() * s["weight"].t()).sum(1) + s["bias"]
    if s["idx"] is None:
        s["state_out"].copy_(win[:, 1:])
    else:
        s["state_out"][s["idx"].long()] = win[:, 1:]
    return {"y": (pre * _sigmoid(pre)).to(to), "state": s["state_out"]}


def _plain_conv(s):
    to, taps = s["x"].dtype, s["weight"].shape[1]
    seq, t, valid = _rows_of(s)
    flip = (lambda v: v.flip(0)) if s["newest_first"] else (lambda v: v)
    seq, t, valid = flip(seq), flip(t), flip(valid)
    n = t.numel()
    x, dy = (torch.where(valid[:, None], flip(s[k]).float(), 0.0) for k in ("x", "dy"))
    back = torch.arange(taps - 1, -1, -1, device="cuda")
    at, row = t[:, None] - back, (torch.arange(n, device="cuda")[:, None] - back).clamp(min=0)   # [n, taps]
    state = s["state"].float()
    win = torch.where((at >= 0)[:, :, None], x[row], state[seq[:, None], (at + taps - 1).clamp(0, max(0, taps - 2))])
    pre = (win * s["weight"].t()).sum(1) + s["bias"]
    sg = _sigmoid(pre)
    on = valid[:, None]
    g = torch.where(on, dy * sg * (1 + pre * (1 - sg)), 0.0)
    # the gradient of a row: from the rows that see it
    row = torch.arange(n, device="cuda")[:, None] + back
    inside = row < n
    row = row.clamp(max=n - 1)
    inside = inside & (seq[row] == seq[:, None]) & valid[row]
    dx = (torch.where(inside[:, :, None], g[row], 0.0) * s["weight"].t()).sum(1)
    dx = torch.where(on, dx, 0.0)
    # what the sequence ends with: its last taps - 1 rows, or what the state held before them
    begin, length = _spans(s)
    end_t = length[:, None] - (taps - 1) + torch.arange(taps - 1, device="cuda")
    off = length[:, None] - 1 - end_t if s["newest_first"] else end_t
    last = torch.where((end_t >= 0)[:, :, None], s["x"][(begin[:, None] + off).clamp(0, n - 1)],
                       s["state"][torch.arange(s["seqs"], device="cuda")[:, None], (end_t + taps - 1).clamp(0, max(0, taps - 2))])
    return {"y": flip(torch.where(on, pre * sg, 0.0).to(to)), "state": last, "dx": flip(dx.to(to)),
            "d_weight": (g[:, None] * win).sum(0, dtype=torch.float64).t().float().contiguous(),
            "d_bias": g.sum(0, dtype=torch.float64).float()}


def _plain_norm(s):
    to, x, dy = s["x"].dtype, s["x"].float(), s["dy"].float()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
    xh, g = (x - mean) * rstd, dy * s["weight"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return {"y": (xh * s["weight"] + s["bias"]).to(to), "dx": dx.to(to), "d_weight": (dy * xh).sum(0, dtype=torch.float64).float(),
            "d_bias": dy.sum(0, dtype=torch.float64).float()}


def _plain_clip(s):
    # over the flat buffers that hold the tensors: a squared sum and a scaled copy for each
    flat = [v.float() for v in s["flat"]]
    norm = sum(v.square().sum(dtype=torch.float64) for v in flat).sqrt()
    scale = (s["max_norm"] / norm).clamp(max=1.0).float()
    return {"norm": norm.float().view(1), "grads": [o.copy_(v * scale) for v, o in zip(flat, s["out_flat"])]}


# ---- one pass ----
def _own(s):
    from paper_2307_07649_amd import tgnn
    path = s["path"]
    if path == "clip":
        norm = tgnn.tgnn_clip_grads(s["grads"], s["max_norm"], out=s["out"])
        return {"norm": norm, "grads": s["out_flat"]}
    if path == "norm-train":
        y, mean, rstd = tgnn.tgnn_layer_norm_fwd(s["x"], s["weight"], s["bias"], EPS)
        dx, dw, db = tgnn.tgnn_layer_norm_bwd(s["dy"], s["x"], mean, rstd, s["weight"])
        return {"y": y, "dx": dx, "d_weight": dw, "d_bias": db}
    if not path.endswith("step"):
        seqs = tgnn.Seqs(s["x"].shape[0], s["seqs"], s["longest"], indptr=s["indptr"], cnt=s["cnt"], newest_first=s["newest_first"])
    if path == "conv-step":
        y = tgnn.tgnn_causal_conv_step(s["x"], s["weight"], s["bias"], silu=True, state_in=s["state"], state_out=s["state_out"],
                                       state_idx=s["idx"])
        return {"y": y, "state": s["state_out"]}
    if path == "conv-train":
        y = tgnn.tgnn_causal_conv_fwd(seqs, s["x"], s["weight"], s["bias"], silu=True, state_in=s["state"],
                                      state_out=s["state_out"])
        dx, dw, db = tgnn.tgnn_causal_conv_bwd(seqs, s["dy"], s["x"], s["weight"], s["bias"], silu=True, state_in=s["state"])
        return {"y": y, "state": s["state_out"], "dx": dx, "d_weight": dw, "d_bias": db}
    inputs = dict(D=s["D"], z=s["z"], dt_bias=s["dt_bias"], softplus=True, state_in=s["state"])
    if path == "scan-step":
        y = tgnn.tgnn_selective_scan_step(s["x"], s["dt"], s["A"], s["B"], s["C"], state_out=s["state_out"], state_idx=s["idx"],
                                          **inputs)
        return {"y": y, "state": s["state_out"]}
    if path == "scan":
        y = tgnn.tgnn_selective_scan_fwd(seqs, s["x"], s["dt"], s["A"], s["B"], s["C"], state_out=s["state_out"], **inputs)
        return {"y": y, "state": s["state_out"]}
    saved = tgnn.selective_scan_saved(seqs, s["A"])
    y = tgnn.tgnn_selective_scan_fwd(seqs, s["x"], s["dt"], s["A"], s["B"], s["C"], state_out=s["state_out"], saved=saved,
                                     **inputs)
    grads = tgnn.tgnn_selective_scan_bwd(seqs, s["dy"], s["x"], s["dt"], s["A"], s["B"], s["C"], saved=saved, **inputs)
    return {"y": y, "state": s["state_out"], **grads}


def run(s):
    if own:
        return _own(s)
    path = s["path"]
    if path.startswith("scan"):
        return _plain_scan_step(s) if path == "scan-step" else _plain_scan(s, path == "scan-train")
    return {"conv-step": _plain_conv_step, "conv-train": _plain_conv, "norm-train": _plain_norm, "clip": _plain_clip}[path](s)


def work(case):
    path = case["path"]
    if path == "clip":
        sizes = _tensor_sizes(case)
        size = sum(n * (2 if case["dtype"] == "mixed" and i % 3 == 1 else 4) for i, n in enumerate(sizes))
        return {"bytes": 2 * size, "flops": 3 * sum(sizes)}
    e, d = (4 if case["dtype"] == "f32" else 2), case["width"]
    if path == "norm-train":
        # forward: x in, y out; backward: dy and x in, dx out
        return {"bytes": 5 * case["rows"] * d * e + 4 * (4 * d + 4 * case["rows"]), "flops": 20 * case["rows"] * d}
    scan = path.startswith("scan")
    hidden = 4 * case["states"] if scan else (case["taps"] - 1) * e   # bytes of a column's state
    if path.endswith("step"):
        n = case["rows"]
        row = (4 * d + 2 * case["groups"] * case["states"]) * e if scan else 2 * d * e
        ops = 7 * case["states"] if scan else 2 * case["taps"]
        return {"bytes": n * (row + 2 * d * hidden), "flops": n * d * (ops + 8)}
    n = int(_lengths(case).sum())
    state = 2 * case["seqs"] * d * hidden
    if path == "conv-train":
        return {"bytes": max(1, 5 * n * d * e + state), "flops": max(1, n * d * (6 * case["taps"] + 12))}
    bc = 2 * case["groups"] * case["states"]
    if path == "scan":
        return {"bytes": n * (4 * d + bc) * e + state, "flops": n * d * (7 * case["states"] + 12)}
    # backward: x, dt, z, B, C and dy in, four gradient rows out; the states formed once more, then the way back
    return {"bytes": n * (11 * d + 3 * bc) * e + state, "flops": n * d * (26 * case["states"] + 40)}


# ---- the definitions in 64 bits, one event after the other ----
def _places(s):
    """Row of every (sequence, time), and whether there is one: [sequences, longest]."""
    if s["indptr"] is None:
        begin, length = np.arange(s["seqs"]) * s["longest"], s["cnt"].cpu().numpy().astype(np.int64)
    else:
        ends = s["indptr"].cpu().numpy()
        begin, length = ends[:-1], ends[1:] - ends[:-1]
    t = np.arange(s["longest"])[None]
    there = t < length[:, None]
    at = begin[:, None] + (length[:, None] - 1 - t if s["newest_first"] else t)
    return torch.from_numpy(np.where(there, at, 0)).cuda(), torch.from_numpy(there).cuda(), torch.from_numpy(length).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return {"scan": _exact_scan, "scan-train": _exact_scan, "scan-step": _exact_step, "conv-step": _exact_step,
                "conv-train": _exact_conv, "norm-train": _exact_norm, "clip": _exact_clip}[case["path"]](s)


def _exact_clip(s):
    total = sum(float((v.double() ** 2).sum()) for v in s["flat"])
    norm = math.sqrt(total)
    scale = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
    return {"norm": torch.tensor([norm], dtype=torch.float64), "grads": [v.double() * scale for v in s["flat"]]}


def _exact_norm(s):
    x, dy, w = s["x"].double(), s["dy"].double(), s["weight"].double()
    c = x.shape[1]
    mean = x.sum(1, keepdim=True) / c
    var = ((x - mean) ** 2).sum(1, keepdim=True) / c
    xh = (x - mean) / (var + EPS) ** 0.5
    # the Jacobian of the normalised row: (I - 1 1^T / c - xh xh^T / c) / sqrt(var + eps)
    g = w * dy
    dx = (g - g.sum(1, keepdim=True) / c - xh * (xh * g).sum(1, keepdim=True) / c) / (var + EPS) ** 0.5
    return {"y": w * xh + s["bias"].double(), "dx": dx, "d_weight": (xh * dy).sum(0), "d_bias": dy.sum(0)}


def _silu64(v):
    return v / (1 + (-v).exp())


def _silu_slope64(v):
    e = 1 / (1 + (-v).exp())
    return e + v * e * (1 - e)


def _exact_step(s):
    idx = torch.arange(s["x"].shape[0], device="cuda") if s["idx"] is None else s["idx"].long()
    out = torch.zeros_like(s["state"], dtype=torch.float64)
    x, h = s["x"].double(), s["state"][idx].double()
    if s["path"] == "conv-step":
        win = torch.cat([h, x[:, None]], 1)
        pre = torch.einsum("rtc,ct->rc", win, s["weight"].double()) + s["bias"].double()
        out[idx] = win[:, 1:]
        return {"y": _silu64(pre), "state": out}
    d = x.shape[1]
    group = torch.arange(d, device="cuda") // (d // s["groups"])
    B, C = (s[k].double().view(len(idx), s["groups"], -1)[:, group] for k in ("B", "C"))
    step = torch.logaddexp(s["dt"].double() + s["dt_bias"].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    h = (step[..., None] * s["A"].double()).exp() * h + (step * x)[..., None] * B
    out[idx] = h
    return {"y": ((h * C).sum(-1) + s["D"].double() * x) * _silu64(s["z"].double()), "state": out}


def _exact_conv(s):
    at, there, length = _places(s)
    n, taps = s["x"].shape[0], s["weight"].shape[1]
    w = s["weight"].double()
    x = torch.cat([s["state"].double(), s["x"][at].double() * there[:, :, None]], 1)       # [seqs, taps - 1 + longest, width]
    dy = s["dy"][at].double() * there[:, :, None]
    steps = s["longest"]
    pre = sum(x[:, j:j + steps] * w[:, j] for j in range(taps)) + s["bias"].double()
    g = dy * _silu_slope64(pre)
    dx = torch.zeros_like(x)
    for j in range(taps):
        dx[:, j:j + steps] += g * w[:, j]
    flat = lambda v: torch.zeros(n, v.shape[2], dtype=torch.float64, device="cuda").index_put_((at[there],), v[there])  # noqa: E731
    tail = length[:, None] + torch.arange(taps - 1, device="cuda")
    return {"y": flat(_silu64(pre)), "state": torch.gather(x, 1, tail[:, :, None].expand(-1, -1, x.shape[2])),
            "dx": flat(dx[:, taps - 1:]), "d_weight": torch.stack([(g * x[:, j:j + steps]).sum((0, 1)) for j in range(taps)], 1),
            "d_bias": g.sum((0, 1))}


def _exact_scan(s):
    at, there, length = _places(s)
    n, (d, states), train = s["x"].shape[0], s["A"].shape, s["path"] == "scan-train"
    if s["seqs"] * s["longest"] * d * (states if train else 12) > 4_000_000_000:
        return None
    group = torch.arange(d, device="cuda") // (d // s["groups"])
    A, D, bias = s["A"].double(), s["D"].double(), s["dt_bias"].double()
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    h = s["state"].double()
    names = ("y", "dx", "ddt", "dz") if train else ("y",)
    rows = {k: torch.zeros(n, d, dtype=torch.float64, device="cuda") for k in names}
    kept = []

    def inputs(t):
        who = at[:, t]
        B, C = (s[k][who].double().view(s["seqs"], s["groups"], states)[:, group] for k in ("B", "C"))
        raw = s["dt"][who].double() + bias
        return who, there[:, t], s["x"][who].double(), raw, torch.logaddexp(raw, zero), B, C

    for t in range(s["longest"]):
        who, on, x, raw, step, B, C = inputs(t)
        new = (step[..., None] * A).exp() * h + (step * x)[..., None] * B
        h = torch.where(on[:, None, None], new, h)
        if train:
            kept.append(h)
        y = (h * C).sum(-1) + D * x
        rows["y"].index_put_((who[on],), (y * _silu64(s["z"][who].double()))[on])
    out = {"y": rows["y"], "state": h}
    if not train:
        return out
    carry = torch.zeros_like(h)                       # d loss / d h[t] through the events after t
    dA, dD, dbias = torch.zeros_like(A), torch.zeros_like(D), torch.zeros_like(bias)
    dB = torch.zeros(n, s["groups"] * states, dtype=torch.float64, device="cuda")
    dC = torch.zeros_like(dB)
    by_group = lambda v: v.view(s["seqs"], s["groups"], d // s["groups"], states).sum(2).view(s["seqs"], -1)  # noqa: E731
    for t in range(s["longest"] - 1, -1, -1):
        who, on, x, raw, step, B, C = inputs(t)
        z, dy = s["z"][who].double(), s["dy"][who].double()
        before = kept[t - 1] if t else s["state"].double()
        y = (kept[t] * C).sum(-1) + D * x
        gy = dy * _silu64(z)
        lam = carry + gy[..., None] * C
        decay = (step[..., None] * A).exp()
        dstep = (lam * (A * decay * before + x[..., None] * B)).sum(-1)
        draw_ = dstep * (raw - torch.logaddexp(raw, zero)).exp()
        m = on[:, None].double()
        dA += (m[..., None] * step[..., None] * lam * decay * before).sum(0)
        dD += (m * gy * x).sum(0)
        dbias += (m * draw_).sum(0)
        rows["dx"].index_put_((who[on],), (D * gy + step * (lam * B).sum(-1))[on])
        rows["ddt"].index_put_((who[on],), draw_[on])
        rows["dz"].index_put_((who[on],), (dy * y * _silu_slope64(z))[on])
        dB.index_put_((who[on],), by_group(lam * (step * x)[..., None])[on])
        dC.index_put_((who[on],), by_group(gy[..., None] * kept[t])[on])
        carry = torch.where(on[:, None, None], lam * decay, carry)
    out.update(dx=rows["dx"], ddt=rows["ddt"], dz=rows["dz"], dB=dB, dC=dC, dA=dA, dD=dD, ddt_bias=dbias)
    return out
