"""The state-space layer's operators in 64 bits, row after row: linear with epilogue, causal convolution, scan.

Each function also takes ``magnitude``: every term then enters by its absolute value (decays stay what they
are), which gives the size that the roundings of a 32-bit evaluation are relative to.
"""

import math

import numpy as np


def _erf(x):
    return np.vectorize(math.erf, otypes=[np.float64])(x)


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1 / (1 + e), e / (1 + e))


def act(name, p):
    """(act(p), act'(p))."""
    if name == "none":
        return p, np.ones_like(p)
    if name == "relu":
        return np.maximum(p, 0), (p > 0) * 1.0
    if name == "silu":
        s = sigmoid(p)
        return p * s, s * (1 + p * (1 - s))
    if name == "gelu":
        c = 0.5 * (1 + _erf(p / math.sqrt(2)))
        return p * c, c + p * np.exp(-p * p / 2) / math.sqrt(2 * math.pi)
    raise ValueError(name)


def linear(x, W, b, residual, name, dy=None):
    x, W = np.asarray(x, np.float64), np.asarray(W, np.float64)
    pre = x @ W.T + (0 if b is None else b)
    f, df = act(name, pre)
    out = dict(pre=pre, y=f if residual is None else f + residual)
    if dy is not None:
        g = np.asarray(dy, np.float64) * df
        out.update(g=g, dx=g @ W, dW=g.T @ x, db=g.sum(0))
    return out


def conv(lens, x, w, b, name, first=None, dy=None, magnitude=False):
    """first: [sequences, width - 1, d] or None.  Rows of all sequences one after the other."""
    k, d = w.shape
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    b = np.zeros(d) if b is None else np.asarray(b, np.float64)
    first = np.zeros((len(lens), k - 1, d)) if first is None else np.asarray(first, np.float64)
    a = np.abs if magnitude else (lambda v: v)
    pre, mag, last = np.zeros_like(x), np.zeros_like(x), first.copy()
    out = dict(dx=np.zeros_like(x), dw=np.zeros_like(w), db=np.zeros(d))
    r = 0
    for s, n in enumerate(lens):
        line = np.concatenate([first[s], x[r:r + n]])
        for t in range(n):
            pre[r + t] = b + (w * line[t:t + k]).sum(0)
            mag[r + t] = np.abs(b) + np.abs(w * line[t:t + k]).sum(0)
        if n:
            last[s] = line[n:n + k - 1]
        if dy is not None:
            slope = act(name, pre[r:r + n])[1]
            # a rounding of pre moves the slope by its second derivative, at most 1/2
            g = np.abs(dy[r:r + n]) * (1.2 + 0.5 * mag[r:r + n]) if magnitude else dy[r:r + n] * slope
            for t in range(n):
                out["dw"] += a(g[t] * line[t:t + k])
                out["db"] += a(g[t])
                for j in range(k):
                    if t + k - 1 - j < n:
                        out["dx"][r + t] += a(w[j] * g[t + k - 1 - j])
        r += n
    out.update(y=mag if magnitude else act(name, pre)[0], state=last)
    return out


def scan(lens, x, delta, A, B, C, D=None, z=None, bias=None, softplus=True, groups=1, first=None, dy=None,
         magnitude=False):
    """A, first rows [n, d]; B, C [rows, groups n]."""
    f64 = lambda v: None if v is None else np.asarray(v, np.float64)   # noqa: E731
    x, A, B, C, D, z, dy = f64(x), f64(A), f64(B), f64(C), f64(D), f64(z), f64(dy)
    n, d = A.shape
    u = f64(delta) + (0 if bias is None else f64(bias))
    dt = np.logaddexp(u, 0) if softplus else u
    wide = lambda m: np.repeat(m.reshape(-1, groups, n).transpose(0, 2, 1), d // groups, axis=2)   # noqa: E731
    narrow = lambda m: m.reshape(n, groups, d // groups).sum(2).T.reshape(-1)                      # noqa: E731
    B, C = wide(B), wide(C)
    decay = lambda t: np.exp(dt[t] * A)   # noqa: E731
    first = np.zeros((len(lens), n, d)) if first is None else f64(first)
    gate, dgate = (np.ones_like(x), np.zeros_like(x)) if z is None else act("silu", z)
    du_dt = sigmoid(u) if softplus else np.ones_like(u)
    Aval = A
    dtv = dt
    if magnitude:
        if z is not None:   # silu' = s + s z (1 - s): two terms that cancel near z = -1.28, each rounded at its own size
            dgate = sigmoid(z) * (1 + np.abs(z) * sigmoid(-z))
        x, B, C, first, gate, dgate, Aval, dtv = (np.abs(v) for v in (x, B, C, first, gate, dgate, A, dt))
        D = None if D is None else np.abs(D)
        dy = None if dy is None else np.abs(dy)
    raw, last = np.zeros_like(x), first.copy()
    out = {}
    if dy is not None:
        out = dict(dx=np.zeros_like(x), ddelta=np.zeros_like(x), dB=np.zeros((x.shape[0], groups * n)),
                   dC=np.zeros((x.shape[0], groups * n)), dA=np.zeros_like(A), dD=np.zeros(d))
    r = 0
    for s, m in enumerate(lens):
        h, before = first[s].copy(), []
        for t in range(r, r + m):
            before.append(h)
            h = decay(t) * h + dtv[t] * x[t] * B[t]
            raw[t] = (C[t] * h).sum(0) + (0 if D is None else D * x[t])
        if m:
            last[s] = h
        if dy is not None:
            flow = np.zeros((n, d))
            for t in range(r + m - 1, r - 1, -1):
                hp = before[t - r]
                e = dy[t] * gate[t]
                hn = decay(t) * hp + dtv[t] * x[t] * B[t]
                g = C[t] * e + flow
                out["dC"][t] = narrow(hn * e)
                out["dB"][t] = narrow(g * dtv[t] * x[t])
                inner = g * decay(t) * hp
                out["dA"] += inner * dtv[t]
                gb = (g * B[t]).sum(0)
                out["ddelta"][t] = ((inner * Aval).sum(0) + gb * x[t]) * du_dt[t]
                out["dx"][t] = gb * dtv[t] + (0 if D is None else D * e)
                out["dD"] += e * x[t]
                flow = decay(t) * g
        r += m
    out.update(y=raw * gate, state=last)
    if dy is not None:
        out.update(dz=dy * raw * dgate, ddelta_bias=out["ddelta"].sum(0))
    return out
