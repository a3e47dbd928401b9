"""64-bit references of the scan and the convolution, one event after the other, that carry along how far float arithmetic
may be off: every value comes with a bound of its error, which each operation passes on and adds its own roundings to."""
import numpy as np
import torch

from ops_common import U, dev, f64, rng

D64 = torch.float64


class V:
    """A value and a bound of its error."""

    def __init__(self, v, e=None):
        self.v = torch.as_tensor(v, dtype=D64)
        self.e = torch.zeros_like(self.v) if e is None else e

    def __add__(self, o):
        v = self.v + o.v
        return V(v, self.e + o.e + U * v.abs())

    def __mul__(self, o):
        v = self.v * o.v
        return V(v, self.v.abs() * o.e + o.v.abs() * self.e + self.e * o.e + U * v.abs())

    def __getitem__(self, k):
        return V(self.v[k], self.e[k])

    def at_least(self, extra):
        return V(self.v, self.e + extra)

    def sum(self, dim, deep):
        """`deep`: additions that a value goes through at most."""
        return V(self.v.sum(dim), self.e.sum(dim) + deep * U * self.v.abs().sum(dim))


def exp_(a, slack=0.0):
    """The argument is scaled to base 2 (one rounding of it and one of the constant), the exponential itself is off by one step, 2 U."""
    v = torch.exp(a.v)
    e = a.e + (2 * U + slack * U) * a.v.abs()
    return V(v, v * torch.expm1(e) + 3 * U * v)


def sigmoid_(a):
    v = torch.sigmoid(a.v)
    return V(v, v * (1 - v) * torch.expm1(a.e + 2 * U * a.v.abs()) * 1.01 + 6 * U * v)


def softplus_(a):
    """Relative: max(v, 0) + log1p(e) by a series in s = e / (2 + e): a dozen roundings and an exponential of |v|."""
    v = torch.logaddexp(a.v, torch.zeros((), dtype=D64))
    s = torch.sigmoid(a.v)
    return V(v, s * a.e * 1.01 + (16 + 2 * a.v.abs()) * U * v)


def silu_(a):
    return a * sigmoid_(a)


def silu_slope_(a):
    s = sigmoid_(a)
    one = V(torch.ones_like(a.v))
    return s * (one + a * (one + V(-s.v, s.e)))


def places(n_rows, n_seqs, max_len, indptr=None, cnt=None, newest_first=False):
    """Rows of every sequence in time order, and its padding rows."""
    out = []
    for s in range(n_seqs):
        b, e = (s * max_len, (s + 1) * max_len) if indptr is None else (int(indptr[s]), int(indptr[s + 1]))
        if not (0 <= b <= e <= n_rows):
            b = e = 0
        n = e - b if cnt is None else int(cnt[s])
        if not 0 <= n <= e - b:
            n = 0
        rows = list(range(b, b + n))
        out.append((rows[::-1] if newest_first else rows, list(range(b + n, e))))
    return out


def scan_reference(seqs, p, dy=None, segment=64):
    """p: dict of cpu double tensors x, dt, A, B, C and optionally D, z, dt_bias, state; groups, softplus.  `segment`: events that a segment
    may have: its deltas are summed up in float.  -> dict of V (rows: zero where no sequence is), final states among them."""
    x, dt, A, B, C = (p[k] for k in ("x", "dt", "A", "B", "C"))
    rows, d = x.shape
    n = A.shape[1]
    G = p["groups"]
    group = torch.arange(d) // (d // G)
    zero = lambda *s: V(torch.zeros(*s, dtype=D64))  # noqa: E731
    out = {k: zero(rows, d) for k in ("y", "dx", "ddt", "dz")}
    out.update({k: zero(rows, G * n) for k in ("dB", "dC")})
    out.update(dA=zero(d, n), dD=zero(d), ddt_bias=zero(d), state=[])
    opt = lambda k: V(p[k]) if p.get(k) is not None else None  # noqa: E731
    D, bias, VA = opt("D"), opt("dt_bias"), V(A)

    def put(name, r, v):
        out[name].v[r], out[name].e[r] = v.v, v.e

    def acc(name, v):     # sums over events, in whatever order, are at most so deep
        out[name].v += v.v
        out[name].e += v.e + 80 * U * v.v.abs()

    def event(r):
        X, Bv, Cv = V(x[r]), V(B[r].view(G, n)[group]), V(C[r].view(G, n)[group])
        raw = V(dt[r]) + bias if bias is not None else V(dt[r])
        delta = softplus_(raw) if p.get("softplus", True) else raw
        a = exp_(delta[:, None] * VA, slack=segment)
        Z = V(p["z"][r]) if p.get("z") is not None else None
        return X, Bv, Cv, raw, delta, a, Z

    for s, (order, _) in enumerate(seqs):
        h0 = V(p["state"][s].clone()) if p.get("state") is not None else zero(d, n)
        h, hs = h0, []
        for r in order:
            X, Bv, Cv, raw, delta, a, Z = event(r)
            h = a * h + (delta * X)[:, None] * Bv
            hs.append(h)
            y0 = (h * Cv).sum(1, n + 2)
            if D is not None:
                y0 = y0 + D * X
            put("y", r, y0 * silu_(Z) if Z is not None else y0)
        out["state"].append(h)
        if dy is None:
            continue
        carry = zero(d, n)
        for i in range(len(order) - 1, -1, -1):
            r = order[i]
            X, Bv, Cv, raw, delta, a, Z = event(r)
            before = hs[i - 1] if i else h0
            dyv = V(dy[r])
            gy = dyv * silu_(Z) if Z is not None else dyv
            lam = Cv * gy[:, None] + carry
            ah = a * before
            s1 = (lam * Bv).sum(1, n + 2)
            s2 = (VA * (lam * ah)).sum(1, n + 2)
            dxv = delta * s1
            put("dx", r, D * gy + dxv if D is not None else dxv)
            dd = X * s1 + s2
            draw = dd * sigmoid_(raw) if p.get("softplus", True) else dd
            put("ddt", r, draw)
            if Z is not None:
                y0 = (hs[i] * Cv).sum(1, n + 2)
                if D is not None:
                    y0 = y0 + D * X
                put("dz", r, dyv * (y0 * silu_slope_(Z)))
            fold = lambda v: V(v.v.view(G, d // G, n).sum(1).reshape(-1),  # noqa: E731
                               (v.e + (24 + d / 64) * U * v.v.abs()).view(G, d // G, n).sum(1).reshape(-1))
            put("dB", r, fold(lam * (delta * X)[:, None]))
            put("dC", r, fold(gy[:, None] * hs[i]))
            acc("dA", delta[:, None] * (lam * ah))
            acc("dD", gy * X)
            acc("ddt_bias", draw)
            carry = a * lam
    return out


def conv_reference(seqs, p, dy=None):
    """p: x, weight, optionally bias, state [seqs, width - 1, d]; silu.  -> dict of V, state: the last width - 1 inputs of every sequence."""
    x, w = p["x"], p["weight"]
    rows, d = x.shape
    W = w.shape[1]
    zero = lambda *s: V(torch.zeros(*s, dtype=D64))  # noqa: E731
    out = dict(y=zero(rows, d), dx=zero(rows, d), d_weight=zero(d, W), d_bias=zero(d), state=[])
    for s, (order, _) in enumerate(seqs):
        head = p["state"][s] if p.get("state") is not None else torch.zeros(W - 1, d, dtype=D64)
        xs = torch.cat([head, x[order]])
        out["state"].append(xs[len(xs) - (W - 1):] if W > 1 else xs[:0])
        if not order:
            continue
        n = len(order)
        pre = V(torch.zeros(n, d, dtype=D64)) if p.get("bias") is None else V(p["bias"].expand(n, d))
        for j in range(W):
            pre = pre + V(xs[j:j + n]) * V(w[:, j])
        y = silu_(pre) if p.get("silu", True) else pre
        out["y"].v[order], out["y"].e[order] = y.v, y.e
        if dy is None:
            continue
        g = V(dy[order])
        if p.get("silu", True):
            g = g * silu_slope_(pre)
        for m in range(W):     # dx[u] += w[W - 1 - m] g[u + m]
            if m < n:
                t = g[m:] * V(w[:, W - 1 - m])
                at = order[:n - m]
                out["dx"].v[at] += t.v
                out["dx"].e[at] += t.e + (W + 1) * U * t.v.abs()
        for j in range(W):
            t = g * V(xs[j:j + n])
            out["d_weight"].v[:, j] += t.v.sum(0)
            out["d_weight"].e[:, j] += (t.e + (80 + n / 64) * U * t.v.abs()).sum(0)
        out["d_bias"].v += g.v.sum(0)
        out["d_bias"].e += (g.e + (80 + n / 64) * U * g.v.abs()).sum(0)
    return out


def packed(lens, behind=0):
    ip = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    return dict(n_rows=int(ip[-1]) + behind, n_seqs=len(lens), max_len=max(1, max(lens, default=1)), indptr=torch.from_numpy(ip))


def lists(counts, k, newest_first=True):
    return dict(n_rows=len(counts) * k, n_seqs=len(counts), max_len=k, cnt=torch.tensor(counts, dtype=torch.int32), newest_first=newest_first)


def on_gpu(tgnn, q, **over):
    q = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in {**q, **over}.items()}
    return tgnn.Seqs(**q)


def poison(t, q, value=float("nan")):
    """The rows that belong to no sequence hold `value`."""
    keep = torch.zeros(t.shape[0], dtype=torch.bool)
    for order, _ in places(**q):
        keep[order] = True
    t[~keep.to(t.device)] = value
    return t
