"""Shared by the tests of the sequence-layer operators: types, roundings, comparison with a 64-bit reference."""
import numpy as np
import torch

U = 2.0 ** -24                                  # half a step of float32, relative: what one rounding to float may be off
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def dev(a, dtype=None):
    return torch.as_tensor(a).to("cuda", dtype=dtype)


def f64(t):
    return t.detach().cpu().double()


def within(got, ref, tol, label=""):
    """|got - ref| <= tol element by element, plus the rounding of the result to got's type (a float16 below its normal range is off by
    up to half of its smallest step, 2^-25)."""
    got_, ref = f64(got), torch.as_tensor(ref).double()
    assert got_.shape == ref.shape, (label, got_.shape, ref.shape)
    half = HALF[got.dtype]
    tol = torch.as_tensor(tol).double().expand_as(ref)
    # (the result is rounded from a float that may be off by tol itself)
    limit = tol + half * (ref.abs() + tol) + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    bad = ~((got_ - ref).abs() <= limit)
    assert not bad.any(), (label, int(bad.sum()), float((got_ - ref).abs()[bad].max()), float(limit[bad].min()), bad.nonzero()[:4].tolist())


def wide_rows(t, extra, shift=0, fill=float("nan")):
    """The same rows in a wider array: `extra` values of `fill` behind every row, the first row `shift` values behind the start."""
    n, c = t.shape
    buf = torch.full((shift + n * (c + extra),), fill, dtype=t.dtype, device=t.device)
    view = buf[shift:].view(n, c + extra)[:, :c]
    view.copy_(t)
    return view


def rng(seed):
    return np.random.default_rng(seed)
