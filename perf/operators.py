"""The operators of a state-space layer over sequences of rows, as they are measured.

Three operators that a sequence memory is made of, next to the GRU and the recurrent cell: a linear
layer whose bias, activation and residual are part of its product, a short causal convolution per channel, and a
selective state space scan.  The last two take sequences of unequal lengths, laid one after the other
in the rows of a matrix, and start from and leave a carried state per sequence, found in a table by
slot (a node's, as the node memory's rows are).  Each has a form for whole sequences, one for training
(the forward call and the backward call), and, where there is a state, one for single rows.

Formulas, for row t of a sequence (t - 1 is the row before it or, at the first one, the carried state):

  linear   pre = W x + b,  y = act(pre) + residual
  conv     pre_t = b + sum_j w_j x_(t - width + 1 + j)  (per channel),  y = act(pre)
  scan     dt_t = softplus(delta_t + delta_bias)
           h_t[n, c] = exp(dt_t[c] A[n, c]) h_(t-1)[n, c] + dt_t[c] B_t[n] x_t[c]
           y_t[c] = (sum_n C_t[n] h_t[n, c] + D[c] x_t[c]) silu(z_t[c])

with act none, relu, silu or gelu, and B and C per group of channels.  Carried states are inputs of a
call, not differentiated.

``own`` chooses between the plain form (elementary torch operations in 32 bits) and this repository's
kernels; ``exact`` gives the values in 64 bits, row after row.
"""

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

ACTS = ("none", "relu", "silu", "gelu")


# --------------------------------------------------------------------------- cases

def _linear(name, kind, rows, d_in, d_out, act, dtype, bias=True, residual=False, pad=0):
    c = dict(kind=kind, rows=rows, d_in=d_in, d_out=d_out, act=act, dtype=dtype, bias=bias, residual=residual, pad=pad)
    return dict(c, name=name) if name else c


def _conv(name, kind, rows, d, width, act, dtype, seqs, skew=0.0, slots=0, bias=True, pad=0):
    c = dict(kind=kind, rows=rows, d=d, width=width, act=act, dtype=dtype, seqs=seqs, skew=skew, slots=slots, bias=bias,
             pad=pad)
    return dict(c, name=name) if name else c


def _scan(name, kind, rows, d, n, dtype, seqs, skew=0.0, slots=0, groups=1, gate=True, skip=True, pad=0):
    c = dict(kind=kind, rows=rows, d=d, n=n, dtype=dtype, seqs=seqs, skew=skew, slots=slots, groups=groups, gate=gate,
             skip=skip, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    """seqs: sequences in the rows; skew > 0: the rows' nodes follow a Zipf law of that exponent over `seqs`
    nodes (a batch's messages grouped by node: a few long sequences, many of one row), else lengths vary
    by a factor of about three; slots > 0: carried states in a table of so many slots; pad: rows behind the last."""
    return [
        # the input layer of a batch's messages (4,000 events, two messages each, the headline width)
        _linear("linear-events-f32", "linear_fwd", 8_000, 300, 200, "silu", "f32"),
        # the output layer over long sequences, with the residual stream
        _linear("linear-prompt-bf16", "linear_fwd", 16_384, 4_096, 2_048, "none", "bf16", residual=True),
        # a training step of a message layer with wide edge features: odd sizes, few rows
        _linear("linear-train-odd-f32", "linear_train", 2_399, 472, 100, "gelu", "f32", residual=True),
        # a training step of an inner layer over long sequences
        _linear("linear-train-bf16", "linear_train", 8_192, 1_024, 2_048, "silu", "bf16"),
        # a batch's messages by node, each sequence going on where its node stopped
        _conv("conv-events-f32", "conv_fwd", 8_000, 100, 4, "silu", "f32", 6_000, 1.2, 100_000, pad=100),
        # training over long sequences
        _conv("conv-train-bf16", "conv_train", 32_768, 2_048, 4, "silu", "bf16", 10),
        # serving: one row for each of many sequences
        _conv("conv-step-bf16", "conv_step", 4_000, 2_048, 4, "silu", "bf16", 4_000, 0.0, 6_000),
        # one row for each node of the smallest batch: latency
        _scan("scan-step-tiny-f32", "scan_step", 400, 32, 16, "f32", 400, 0.0, 1_000),
        # serving: one row for each of many sequences
        _scan("scan-step-bf16", "scan_step", 16_000, 256, 16, "bf16", 16_000, 0.0, 20_000),
        # a batch's messages by node, with the nodes' states
        _scan("scan-events-f32", "scan_fwd", 8_000, 100, 16, "f32", 6_000, 1.2, 100_000, pad=100),
        # long prompts
        _scan("scan-prompt-bf16", "scan_fwd", 32_768, 2_048, 16, "bf16", 5, slots=8),
        # training over sequences of mixed lengths
        _scan("scan-train-bf16", "scan_train", 16_384, 1_024, 16, "bf16", 24),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("linear_fwd", "linear_train", "conv_fwd", "conv_train", "conv_step", "scan_fwd", "scan_train",
                       "scan_step"))
    dtype = rng.choice(("f32", "bf16"))
    pad = rng.choice((0, 0, rng.randint(1, 200)))
    if kind.startswith("linear"):
        d_in, d_out = _log(rng, 16, 4_096), _log(rng, 16, 4_096)
        top = 16e9 if dtype == "f32" or kind == "linear_train" else 100e9
        rows = _log(rng, 1, max(2, min(60_000, top / (d_in * d_out))))
        return _linear(None, kind, rows, d_in, d_out, rng.choice(ACTS), dtype, rng.random() < 0.7, rng.random() < 0.5, pad)
    d = rng.choice((_log(rng, 8, 2_048), 32, 100, 128))
    step = kind.endswith("step")
    if kind.startswith("conv"):
        rows = _log(rng, 1, min(100_000, 60e6 / d))
    else:
        n = rng.choice((4, 8, 16, 16, 32, 64, rng.randint(1, 64)))
        rows = _log(rng, 1, min(60_000, 3e8 / (d * n)))
    seqs = rows if step else min(rows, _log(rng, 1, 20_000))
    skew = 0.0 if step else rng.choice((0.0, round(rng.uniform(0.6, 1.2), 2)))
    slots = seqs + rng.randint(0, 100) if step or rng.random() < 0.5 else 0
    if kind.startswith("conv"):
        return _conv(None, kind, rows, d, rng.randint(2, 4), rng.choice(("none", "silu")), dtype, seqs, skew, slots,
                     rng.random() < 0.7, pad)
    groups = rng.choice([g for g in (1, 1, 1, 2, 4) if d % g == 0])
    return _scan(None, kind, rows, d, n, dtype, seqs, skew, slots, groups, rng.random() < 0.7, rng.random() < 0.7, pad)


# --------------------------------------------------------------------------- inputs

def _dt(c):
    return torch.bfloat16 if c.dtype == "bf16" else torch.float32


def _lengths(c, seed):
    """Rows of each sequence (a few of them empty), adding up to c.rows."""
    rs = np.random.RandomState((int(seed) * 9176 + 11) % (1 << 31))
    if c.skew > 0:
        p = np.arange(1, c.seqs + 1, dtype=np.float64) ** -c.skew
        return rs.permutation(rs.multinomial(c.rows, p / p.sum()))
    w = rs.uniform(0.5, 1.5, c.seqs)
    n = np.floor(w / w.sum() * c.rows).astype(np.int64)
    for i in rs.randint(0, c.seqs, c.rows - int(n.sum())):
        n[i] += 1
    return n


def _inputs(case, seed):
    """What a program has in hand: the tensors of one call, made on the GPU from the seed."""
    c = SimpleNamespace(**case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 6007 + 29)
    dt, R = _dt(c), c.rows + c.pad
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")   # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=gen, device="cuda")     # noqa: E731
    v = SimpleNamespace(c=c, R=R, dt=dt)
    if c.kind.startswith("linear"):
        v.x = randn(R, c.d_in).to(dt)
        v.W = ((2 * rand(c.d_out, c.d_in) - 1) * math.sqrt(3.0 / c.d_in)).to(dt)
        v.b = (2 * rand(c.d_out) - 1) * 0.1 if c.bias else None
        v.res = randn(R, c.d_out).to(dt) if c.residual else None
        v.n_rows = torch.tensor([c.rows], dtype=torch.int32, device="cuda")
        if c.kind == "linear_train":
            v.dy = randn(R, c.d_out) * 0.01
        return v
    d = c.d
    S = c.seqs
    if c.kind.endswith("step"):
        v.off = None
        v.n_rows = torch.tensor([c.rows], dtype=torch.int32, device="cuda")
        S = R
    else:
        v.lens = _lengths(c, seed)
        v.off = torch.from_numpy(np.concatenate([[0], np.cumsum(v.lens)]).astype(np.int32)).cuda()
    v.S = S
    n_slots = max(c.slots, S) if c.slots else 0
    v.slot = torch.randperm(n_slots, generator=gen, device="cuda")[:S].int() if c.slots else None
    # the layer's inputs are column ranges of wider rows: x and the gate z of one projection's
    # output, B and C of another's
    wide = randn(R, 2 * d).to(dt)
    v.x, v.z = wide[:, :d], wide[:, d:]
    if c.kind.startswith("conv"):
        v.w = ((2 * rand(c.width, d) - 1) / math.sqrt(c.width)).to(dt)
        v.b = (2 * rand(d) - 1) * 0.1 if c.bias else None
        v.state = randn(n_slots, c.width - 1, d).to(dt) if c.slots else None
    else:
        if not c.gate:
            v.z = None
        v.delta = (0.5 * randn(R, d)).to(dt)
        step = torch.exp(rand(d) * math.log(100.0) + math.log(1e-3))   # steps from 1e-3 to 1e-1
        v.delta_bias = step + torch.log(-torch.expm1(-step))
        v.A = -torch.arange(1, c.n + 1, device="cuda", dtype=torch.float32)[:, None] * (0.5 + rand(c.n, d))
        gn = c.groups * c.n
        bc = randn(R, 2 * gn).to(dt)
        v.B, v.C = bc[:, :gn], bc[:, gn:]
        v.D = 0.5 + rand(d) if c.skip else None
        v.state = randn(n_slots, c.n, d) if c.slots else None
    if c.kind.endswith("train"):
        v.dy = randn(R, d) * 0.01
    return v


def prepare(case, seed):
    v = _inputs(case, seed)
    if own:
        _own_buffers(v)
    return v


def run(state):
    return (_OWN if own else _PLAIN)[state.c.kind](state)


# --------------------------------------------------------------------------- the plain forms, in 32 bits

def _f(t):
    return None if t is None else t.float()


def _act(name, p):
    if name == "relu":
        return torch.where(p > 0, p, torch.zeros_like(p))
    if name == "silu":
        return p / (1 + torch.exp(-p))
    if name == "gelu":
        return 0.5 * p * (1 + torch.erf(p * math.sqrt(0.5)))
    return p


def _dact(name, p):
    if name == "relu":
        return (p > 0).to(p.dtype)
    if name == "silu":
        s = 1 / (1 + torch.exp(-p))
        return s * (1 + p * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(p * math.sqrt(0.5))) + p * torch.exp(-0.5 * p * p) / math.sqrt(2 * math.pi)
    return torch.ones_like(p)


def _plain_linear_pre(v):
    n = v.c.rows
    p = _f(v.x[:n]) @ _f(v.W).t()
    return p if v.b is None else p + v.b


def _plain_linear(v):
    n = v.c.rows
    y = _act(v.c.act, _plain_linear_pre(v))
    if v.res is not None:
        y = y + _f(v.res[:n])
    y = y.to(v.dt)
    return y if n == v.R else torch.cat([y, torch.zeros(v.R - n, y.shape[1], dtype=y.dtype, device=y.device)])


def _plain_linear_train(v):
    n = v.c.rows
    p = _plain_linear_pre(v)
    y = _act(v.c.act, p)
    if v.res is not None:
        y = y + _f(v.res[:n])
    g = v.dy[:n] * _dact(v.c.act, p)
    y, dx = y.to(v.dt), g @ _f(v.W)
    if n != v.R:
        y = torch.cat([y, torch.zeros(v.R - n, y.shape[1], dtype=y.dtype, device=y.device)])
        dx = torch.cat([dx, torch.zeros(v.R - n, dx.shape[1], device=y.device)])
    out = dict(y=y, dx=dx, dW=g.t() @ _f(v.x[:n]))
    if v.b is not None:
        out["db"] = g.sum(0)
    return out


def _rows_of(v):
    """Of each row below c.rows: its sequence and its place in it."""
    lens = (v.off[1:] - v.off[:-1]).long()
    seq = torch.repeat_interleave(torch.arange(v.S, device="cuda"), lens, output_size=v.c.rows)
    pos = torch.arange(v.c.rows, device="cuda") - v.off[:-1].long()[seq]
    return seq, pos, lens


def _slots(v):
    return None if v.slot is None else v.slot.long()


def _conv_taps(v, x, seq, pos):
    """The inputs that meet w[j], for every j: x some rows back, or the carried state, or zero."""
    k, taps = v.c.width, []
    for j in range(k):
        back = k - 1 - j
        t = torch.zeros_like(x)
        if back == 0:
            t = x
        else:
            t[back:] = x[:-back] if back < x.shape[0] else 0
            miss = pos < back
            if v.state is None:
                t[miss] = 0
            else:
                t[miss] = v.state[_slots(v)[seq[miss]], pos[miss] + j].to(x.dtype)
        taps.append(t)
    return taps


def _plain_conv_state(v, x, lens):
    """Table of the carried states after the call (zeros in the slots that no sequence has)."""
    k = v.c.width
    new = torch.zeros_like(v.state)
    full = lens > 0
    sl, end = _slots(v)[full], v.off[1:][full].long()
    n = lens[full]
    for j in range(k - 1):
        back = k - 1 - j               # counted from the sequence's end
        inside = n >= back
        old = v.state[sl, (n + j).clamp_(max=k - 2)]
        new[sl, j] = torch.where(inside[:, None], x[(end - back).clamp_(min=0)].to(v.dt), old)
    return new


def _plain_conv(v):
    n = v.c.rows
    x = _f(v.x[:n])
    seq, pos, lens = _rows_of(v)
    w = _f(v.w)
    p = sum(w[j] * t for j, t in enumerate(_conv_taps(v, x, seq, pos)))
    if v.b is not None:
        p = p + v.b
    out = dict(y=_pad_rows(_act(v.c.act, p).to(v.dt), v))
    if v.state is not None:
        out["state"] = _plain_conv_state(v, x, lens)
    return out


def _pad_rows(t, v):
    n = t.shape[0]
    return t if n == v.R else torch.cat([t, torch.zeros(v.R - n, *t.shape[1:], dtype=t.dtype, device=t.device)])


def _plain_conv_train(v):
    n, k = v.c.rows, v.c.width
    x, w = _f(v.x[:n]), _f(v.w)
    seq, pos, lens = _rows_of(v)
    taps = _conv_taps(v, x, seq, pos)
    p = sum(w[j] * t for j, t in enumerate(taps))
    if v.b is not None:
        p = p + v.b
    g = v.dy[:n] * _dact(v.c.act, p)
    left = lens[seq] - 1 - pos         # rows of the sequence after this one
    dx = torch.zeros_like(x)
    for j in range(k):
        back = k - 1 - j
        t = g
        if back:
            t = torch.zeros_like(g)
            t[:-back] = g[back:] if back < n else 0
            t[left < back] = 0
        dx += w[j] * t
    out = dict(y=_pad_rows(_act(v.c.act, p).to(v.dt), v), dx=_pad_rows(dx, v),
               dw=torch.stack([(g * t).sum(0) for t in taps]))
    if v.b is not None:
        out["db"] = g.sum(0)
    if v.state is not None:
        out["state"] = _plain_conv_state(v, x, lens)
    return out


def _plain_conv_step(v):
    n, k = v.c.rows, v.c.width
    sl = _slots(v)[:n]
    past = torch.cat([v.state[sl], v.x[:n, None]], 1)
    p = (_f(past) * _f(v.w)).sum(1)
    if v.b is not None:
        p = p + v.b
    new = torch.zeros_like(v.state)
    new[sl] = past[:, 1:]
    return dict(y=_pad_rows(_act(v.c.act, p).to(v.dt), v), state=new)


def _softplus(u):
    return torch.clamp(u, min=0) + torch.log1p(torch.exp(-u.abs()))


def _channels(t, v):
    """[rows, groups * n] to [rows, n, d]: each channel its group's values."""
    c = v.c
    t = _f(t).reshape(t.shape[0], c.groups, c.n).transpose(1, 2)
    return t.repeat_interleave(c.d // c.groups, 2) if c.groups > 1 else t.expand(t.shape[0], c.n, c.d)


def _doubling(a, u, longest):
    """h_t = a_t h_(t-1) + u_t in place of u, over rows; a is zero at the rows that start a sequence."""
    s = 1
    while s < longest:
        u[s:] += a[s:] * u[:-s]
        a[s:] *= a[:-s].clone()
        s *= 2
    return u


def _plain_scan_parts(v):
    n = v.c.rows
    x, dt = _f(v.x[:n]), _softplus(_f(v.delta[:n]) + v.delta_bias)
    seq, pos, lens = _rows_of(v)
    first = torch.nonzero(pos == 0)[:, 0]
    a = torch.exp(dt[:, None] * v.A)
    u = (dt * x)[:, None] * _channels(v.B[:n], v)
    if v.state is not None:
        u[first] += a[first] * v.state[_slots(v)[seq[first]]]
    a[first] = 0
    h = _doubling(a, u, int(v.lens.max()))
    return x, dt, seq, pos, lens, first, h


def _plain_scan_out(v, x, h):
    n = v.c.rows
    y = (h * _channels(v.C[:n], v)).sum(1)
    return y if v.D is None else y + v.D * x


def _plain_scan_state(v, h, lens):
    new = torch.zeros_like(v.state)
    full = lens > 0
    new[_slots(v)[full]] = h[v.off[1:][full].long() - 1]
    return new


def _plain_scan(v):
    x, dt, seq, pos, lens, first, h = _plain_scan_parts(v)
    y = _plain_scan_out(v, x, h)
    if v.z is not None:
        y = y * _act("silu", _f(v.z[:v.c.rows]))
    out = dict(y=_pad_rows(y.to(v.dt), v))
    if v.state is not None:
        out["state"] = _plain_scan_state(v, h, lens)
    return out


def _by_group(t, v):
    """Sum over each group's channels: [rows, n, d] to [rows, groups * n]."""
    c = v.c
    return t.reshape(t.shape[0], c.n, c.groups, c.d // c.groups).sum(3).transpose(1, 2).reshape(t.shape[0], -1)


def _plain_scan_train(v):
    c, n = v.c, v.c.rows
    x, dt, seq, pos, lens, first, h = _plain_scan_parts(v)
    raw = _plain_scan_out(v, x, h)
    dy, out = v.dy[:n], {}
    y = raw
    if v.z is not None:
        z = _f(v.z[:n])
        y = raw * _act("silu", z)
        out["dz"] = _pad_rows(dy * raw * _dact("silu", z), v)
        dy = dy * _act("silu", z)
    out["y"] = _pad_rows(y.to(v.dt), v)
    if v.state is not None:
        out["state"] = _plain_scan_state(v, h, lens)
    # the state's gradient runs backwards over the rows: g_t = C_t dy_t + a_(t+1) g_(t+1)
    out["dC"] = _pad_rows(_by_group(h * dy[:, None], v), v)
    a = torch.exp(dt[:, None] * v.A)
    nxt = torch.zeros_like(a)
    nxt[:-1] = a[1:]
    nxt[lens[seq] - 1 == pos] = 0
    g = _doubling(nxt.flip(0), (_channels(v.C[:n], v) * dy[:, None]).flip(0), int(v.lens.max())).flip(0)
    del nxt
    out["dB"] = _pad_rows(_by_group(g * (dt * x)[:, None], v), v)
    prev = torch.zeros_like(h)
    prev[1:] = h[:-1]
    prev[first] = 0 if v.state is None else v.state[_slots(v)[seq[first]]]
    e = g * a * prev                    # the gradient of dt A
    gb = (g * _channels(v.B[:n], v)).sum(1)
    out["dA"] = (e * dt[:, None]).sum(0)
    du = ((e * v.A).sum(1) + gb * x) * (1 / (1 + torch.exp(-(_f(v.delta[:n]) + v.delta_bias))))
    out["ddelta"], out["ddelta_bias"] = _pad_rows(du, v), du.sum(0)
    dx = gb * dt
    if v.D is not None:
        dx = dx + v.D * dy
        out["dD"] = (dy * x).sum(0)
    out["dx"] = _pad_rows(dx, v)
    return out


def _plain_scan_step(v):
    n = v.c.rows
    x, dt = _f(v.x[:n]), _softplus(_f(v.delta[:n]) + v.delta_bias)
    sl = _slots(v)[:n]
    h = torch.exp(dt[:, None] * v.A) * v.state[sl] + (dt * x)[:, None] * _channels(v.B[:n], v)
    y = _plain_scan_out(v, x, h)
    if v.z is not None:
        y = y * _act("silu", _f(v.z[:n]))
    new = torch.zeros_like(v.state)
    new[sl] = h
    return dict(y=_pad_rows(y.to(v.dt), v), state=new)


_PLAIN = dict(linear_fwd=_plain_linear, linear_train=_plain_linear_train, conv_fwd=_plain_conv,
              conv_train=_plain_conv_train, conv_step=_plain_conv_step, scan_fwd=_plain_scan,
              scan_train=_plain_scan_train, scan_step=_plain_scan_step)


# --------------------------------------------------------------------------- this repository's kernels

def _own_buffers(v):
    """Outputs, saves and workspaces, as a program keeps them from call to call."""
    from paper_2608_16305_amd import mtgnn as M
    v.M, c, dt = M, v.c, v.dt
    code = M.BF16 if c.dtype == "bf16" else M.F32
    f32 = lambda *s: torch.zeros(*s, device="cuda")   # noqa: E731
    train = c.kind.endswith("train")
    v.save = v.ws = None
    if c.kind.startswith("linear"):
        v.d = M.linear_dims(c.d_in, c.d_out, code, ACTS.index(c.act))
        v.y = torch.zeros(v.R, c.d_out, dtype=dt, device="cuda")
        v.ws = M.alloc_bytes(M.linear_ws_bytes(v.d, v.R, train))
        v.pre = f32(v.R, c.d_out) if train else None
        if train:
            v.dx, v.dW, v.db = f32(v.R, c.d_in), f32(c.d_out, c.d_in), f32(c.d_out) if c.bias else None
        return
    v.y = torch.zeros(v.R, c.d, dtype=dt, device="cuda")
    v.state_out = torch.zeros_like(v.state) if v.state is not None else None
    if v.off is not None:
        v.q = M.seqs(v.off, v.R, slot=v.slot, n_slots=0 if v.state is None else v.state.shape[0])
    if train:
        v.dx = f32(v.R, c.d)
    if c.kind.startswith("conv"):
        v.d = M.conv_dims(c.d, c.width, code, ACTS.index(c.act))
        if train:
            v.dw, v.db = f32(c.width, c.d), f32(c.d) if c.bias else None
            v.ws = M.alloc_bytes(M.causal_conv_ws_bytes(v.d, v.R))
            v.save = M.alloc_bytes(M.causal_conv_save_bytes(v.d, v.S)) if v.state is not None else None
        return
    v.d = M.scan_dims(c.d, c.n, c.groups, code)
    v.inp = M.scan_inputs(v.d, v.x, v.delta, v.A, v.B, v.C, D=v.D, z=v.z, delta_bias=v.delta_bias)
    if c.kind == "scan_step":
        return
    v.ws = M.alloc_bytes(M.selective_scan_ws_bytes(v.d, v.R, v.S, train))
    if train:
        v.save = M.alloc_bytes(M.selective_scan_save_bytes(v.d, v.R, v.S, v.state is not None))
        v.g = dict(dx=v.dx, ddelta=f32(v.R, c.d), dA=f32(c.n, c.d), dB=f32(v.R, c.groups * c.n),
                   dC=f32(v.R, c.groups * c.n), dD=f32(c.d) if c.skip else None, dz=f32(v.R, c.d) if c.gate else None,
                   ddelta_bias=f32(c.d))
        v.grads = M.scan_grads(v.d, **v.g)


def _own_linear(v):
    v.M.mtgnn_linear(v.x, v.W, v.b, v.res, v.d, v.y, n_rows=v.n_rows, ws=v.ws)
    return v.y


def _own_linear_train(v):
    v.M.mtgnn_linear(v.x, v.W, v.b, v.res, v.d, v.y, pre=v.pre, n_rows=v.n_rows, ws=v.ws)
    v.M.mtgnn_linear_bwd(v.dy, v.pre, v.x, v.W, v.d, v.dx, v.dW, v.db, n_rows=v.n_rows, ws=v.ws)
    out = dict(y=v.y, dx=v.dx, dW=v.dW)
    if v.db is not None:
        out["db"] = v.db
    return out


def _with_state(v, out):
    if v.state is not None:
        out["state"] = v.state_out
    return out


def _own_conv(v):
    v.M.mtgnn_causal_conv(v.q, v.x, v.w, v.b, v.d, v.state, v.state_out, v.y)
    return _with_state(v, dict(y=v.y))


def _own_conv_train(v):
    v.M.mtgnn_causal_conv(v.q, v.x, v.w, v.b, v.d, v.state, v.state_out, v.y, save=v.save)
    v.M.mtgnn_causal_conv_bwd(v.q, v.dy, v.x, v.w, v.b, v.d, v.save, v.dx, v.dw, v.db, v.ws)
    out = dict(y=v.y, dx=v.dx, dw=v.dw)
    if v.db is not None:
        out["db"] = v.db
    return _with_state(v, out)


def _own_conv_step(v):
    v.M.mtgnn_causal_conv_step(v.slot, v.x, v.w, v.b, v.d, v.state, v.state_out, v.y, n_rows=v.n_rows)
    return dict(y=v.y, state=v.state_out)


def _own_scan(v):
    v.M.mtgnn_selective_scan(v.q, v.inp, v.d, v.state, v.state_out, v.y, ws=v.ws)
    return _with_state(v, dict(y=v.y))


def _own_scan_train(v):
    v.M.mtgnn_selective_scan(v.q, v.inp, v.d, v.state, v.state_out, v.y, save=v.save, ws=v.ws)
    v.M.mtgnn_selective_scan_bwd(v.q, v.dy, v.inp, v.d, v.save, v.grads, v.ws)
    return _with_state(v, dict(y=v.y, **{k: t for k, t in v.g.items() if t is not None}))


def _own_scan_step(v):
    v.M.mtgnn_selective_scan_step(v.slot, v.inp, v.d, v.state, v.state_out, v.y, n_rows=v.n_rows)
    return dict(y=v.y, state=v.state_out)


_OWN = dict(linear_fwd=_own_linear, linear_train=_own_linear_train, conv_fwd=_own_conv, conv_train=_own_conv_train,
            conv_step=_own_conv_step, scan_fwd=_own_scan, scan_train=_own_scan_train, scan_step=_own_scan_step)


# --------------------------------------------------------------------------- least work

def work(case):
    """Every input read once, every output written once; an exponential counts as one operation."""
    c = SimpleNamespace(**case)
    e, R = 2 if c.dtype == "bf16" else 4, c.rows
    train, step = c.kind.endswith("train"), c.kind.endswith("step")
    if c.kind.startswith("linear"):
        by = e * (R * c.d_in + c.d_out * c.d_in + (2 if c.residual else 1) * R * c.d_out) + 4 * c.d_out
        fl = 2 * R * c.d_in * c.d_out
        if train:
            by += 4 * (R * c.d_out + R * c.d_in + c.d_out * c.d_in)
            fl *= 3
        return dict(bytes=by, flops=fl)
    seqs = R if step else min(R, c.seqs)
    if c.kind.startswith("conv"):
        by = 2 * e * R * c.d + c.width * c.d * e + (2 * e * seqs * (c.width - 1) * c.d if c.slots else 0)
        fl = R * c.d * (2 * c.width + 6)
        if train:
            by += 8 * R * c.d + 4 * c.width * c.d
            fl += R * c.d * (4 * c.width + 8)
        return dict(bytes=by, flops=fl)
    gn = c.groups * c.n
    by = e * R * ((4 if c.gate else 3) * c.d + 2 * gn) + 4 * (c.n + 2) * c.d + (8 * seqs * c.n * c.d if c.slots else 0)
    fl = R * c.d * (7 * c.n + 12)
    if train:
        by += 4 * R * ((4 if c.gate else 3) * c.d + 2 * gn) + 4 * (c.n + 2) * c.d
        fl += R * c.d * (16 * c.n + 20)
    return dict(bytes=by, flops=fl)


# --------------------------------------------------------------------------- 64 bits, row after row

def exact(case, seed):
    v = _inputs(case, seed)
    return _EXACT[v.c.kind](v)


def _d(t):
    return None if t is None else t.double()


def _act64(name, p):
    """(act(p), its derivative)."""
    if name == "none":
        return p, torch.ones_like(p)
    if name == "relu":
        return p.clamp(min=0), torch.sign(p).clamp(min=0)
    if name == "silu":
        s = torch.sigmoid(p)
        return p * s, s + p * s * torch.sigmoid(-p)
    phi = 0.5 * torch.erfc(-p / math.sqrt(2.0))
    return p * phi, phi + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)


def _exact_linear(v):
    n, train = v.c.rows, v.c.kind == "linear_train"
    x, W = _d(v.x)[:n], _d(v.W)
    p = torch.mm(x, W.t().contiguous())
    if v.b is not None:
        p += _d(v.b)
    f, df = _act64(v.c.act, p)
    y = torch.zeros(v.R, v.c.d_out, dtype=torch.float64, device="cuda")
    y[:n] = f if v.res is None else f + _d(v.res)[:n]
    if not train:
        return y
    df *= _d(v.dy)[:n]
    dx = torch.zeros(v.R, v.c.d_in, dtype=torch.float64, device="cuda")
    dx[:n] = torch.mm(df, W)
    out = dict(y=y, dx=dx, dW=torch.mm(df.t().contiguous(), x))
    if v.b is not None:
        out["db"] = df.sum(0)
    return out


def _walk(v):
    """For each place in the sequences: (sequences that reach it, their rows there)."""
    if v.off is None:
        yield torch.arange(v.c.rows, device="cuda"), torch.arange(v.c.rows, device="cuda")
        return
    order = np.argsort(-v.lens, kind="stable")
    lens = v.lens[order]
    seq, start = torch.from_numpy(order).cuda(), v.off[:-1].long()
    for t in range(int(lens[0])):
        live = seq[:int(np.searchsorted(-lens, -t, side="left"))]
        yield live, start[live] + t


def _first64(v, shape):
    h = torch.zeros(v.S, *shape, dtype=torch.float64, device="cuda")
    if v.state is not None:
        h += v.state[v.slot.long()].double()
    return h


def _table64(v, h, moved):
    out = torch.zeros(v.state.shape, dtype=torch.float64, device="cuda")
    out[v.slot.long()[moved]] = h[moved]
    return out


def _moved(v):
    return torch.arange(v.c.rows, device="cuda") if v.off is None else torch.nonzero(v.off[1:] > v.off[:-1])[:, 0]


def _exact_conv(v):
    c, k = v.c, v.c.width
    x, w = _d(v.x), _d(v.w)
    b = 0.0 if v.b is None else _d(v.b)
    past = _first64(v, (k - 1, c.d))
    zeros = lambda: torch.zeros(v.R, c.d, dtype=torch.float64, device="cuda")   # noqa: E731
    y, slope, seen = zeros(), zeros(), []
    dw = torch.zeros(k, c.d, dtype=torch.float64, device="cuda")
    db = torch.zeros(c.d, dtype=torch.float64, device="cuda")
    train = c.kind == "conv_train"
    for live, row in _walk(v):
        win = torch.cat([past[live], x[row, None]], 1)
        y[row], s = _act64(c.act, (win * w).sum(1) + b)
        past[live] = win[:, 1:]
        if train:
            s = s * v.dy[row].double()
            slope[row] = s
            dw += (win * s[:, None]).sum(0)
            db += s.sum(0)
            seen.append((live, row))
    out = dict(y=y)
    if v.state is not None:
        out["state"] = _table64(v, past, _moved(v))
    if train:
        dx = zeros()
        ahead = torch.zeros(v.S, k, c.d, dtype=torch.float64, device="cuda")   # slopes of this row and the next ones
        for live, row in reversed(seen):
            win = torch.cat([slope[row, None], ahead[live, :-1]], 1)
            dx[row] = (win * w.flip(0)).sum(1)
            ahead[live] = win
        out.update(dx=dx, dw=dw)
        if v.b is not None:
            out["db"] = db
    return out


def _exact_scan(v):
    c = v.c
    train, per = c.kind == "scan_train", c.d // c.groups
    A, x = _d(v.A), _d(v.x)
    u = _d(v.delta) + _d(v.delta_bias)
    dt = torch.logaddexp(u, torch.zeros_like(u))
    wide = lambda t: t.reshape(-1, c.groups, c.n).transpose(1, 2).repeat_interleave(per, 2)   # noqa: E731
    h = _first64(v, (c.n, c.d))
    zeros = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")   # noqa: E731
    raw, seen = zeros(v.R, c.d), []
    before = zeros(c.rows, c.n, c.d) if train else None
    for live, row in _walk(v):
        if train:
            before[row] = h[live]
            seen.append((live, row))
        t = dt[row, None]
        new = torch.exp(t * A) * h[live] + t * x[row, None] * wide(v.B[row].double())
        h[live] = new
        raw[row] = (new * wide(v.C[row].double())).sum(1)
        if v.D is not None:
            raw[row] += v.D.double() * x[row]
    f, df = (1.0, None) if v.z is None else _act64("silu", _d(v.z))
    out = dict(y=raw * f)
    if v.state is not None:
        out["state"] = _table64(v, h, _moved(v))
    if not train:
        return out
    dy = _d(v.dy)
    dy[c.rows:] = 0
    if v.z is not None:
        out["dz"] = dy * raw * df
        dy = dy * f
    narrow = lambda t: t.reshape(-1, c.n, c.groups, per).sum(3).transpose(1, 2).reshape(t.shape[0], -1)   # noqa: E731
    gx, gu, dB, dC = zeros(v.R, c.d), zeros(v.R, c.d), zeros(v.R, c.groups * c.n), zeros(v.R, c.groups * c.n)
    dA, g = zeros(c.n, c.d), zeros(v.S, c.n, c.d)
    for live, row in reversed(seen):
        t, b = dt[row, None], wide(v.B[row].double())
        decay = torch.exp(t * A)
        g_row = g[live] + wide(v.C[row].double()) * dy[row, None]
        now = decay * before[row] + t * x[row, None] * b
        dC[row] = narrow(now * dy[row, None])
        dB[row] = narrow(g_row * t * x[row, None])
        gb = (g_row * b).sum(1)
        gx[row] = gb * dt[row]
        inner = g_row * decay * before[row]
        dA += (inner * t).sum(0)
        gu[row] = ((inner * A).sum(1) + gb * x[row]) * torch.sigmoid(u[row])
        g[live] = decay * g_row
    if v.D is not None:
        gx += dy * v.D.double()
        out["dD"] = (dy * x).sum(0)
    out.update(dx=gx, ddelta=gu, ddelta_bias=gu.sum(0), dA=dA, dB=dB, dC=dC)
    return out


_EXACT = dict(linear_fwd=_exact_linear, linear_train=_exact_linear, conv_fwd=_exact_conv, conv_train=_exact_conv,
              conv_step=_exact_conv, scan_fwd=_exact_scan, scan_train=_exact_scan, scan_step=_exact_scan)
