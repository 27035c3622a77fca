"""The operators of a model over all nodes in 64 bits: embedding, layer norm, softmax loss over all classes, AdamW with
states in 32 or 8 bits.  Written from the formulas, row by row where that is plainer."""

import math

import numpy as np


def embedding(ids, table, scale, dy=None):
    n, d = table.shape
    table = np.asarray(table, np.float64)
    y, dtable = np.zeros((len(ids), d)), np.zeros((n, d))
    for r, i in enumerate(ids):
        if 0 <= i < n:
            y[r] = scale * table[i]
            if dy is not None:
                dtable[i] += scale * np.asarray(dy[r], np.float64)
    return dict(y=y) if dy is None else dict(y=y, dtable=dtable)


def layer_norm(x, gamma, beta, eps, dy=None, past=None):
    x = np.asarray(x, np.float64)
    d = x.shape[1]
    gamma = np.ones(d) if gamma is None else np.asarray(gamma, np.float64)
    beta = np.zeros(d) if beta is None else np.asarray(beta, np.float64)
    m = x.mean(1, keepdims=True)
    q = 1 / np.sqrt(((x - m) ** 2).mean(1, keepdims=True) + eps)
    h = (x - m) * q
    out = dict(y=gamma * h + beta, mean=m[:, 0], q=q[:, 0], h=h)
    if dy is not None:
        dy = np.asarray(dy, np.float64)
        g = dy * gamma
        dx = q * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
        out.update(dx=dx if past is None else dx + past, dgamma=(dy * h).sum(0), dbeta=dy.sum(0))
    return out


def softmax_loss(x, W, b, label, dloss=None):
    """Loss, rows' losses, and (dloss given) dx, dW, db; P: of the rows with a label, before the scale."""
    x, W = np.asarray(x, np.float64), np.asarray(W, np.float64)
    n = W.shape[0]
    have = [r for r, c in enumerate(label) if 0 <= c < n]
    rows, dx, dW, db = np.zeros(len(label)), np.zeros(x.shape), np.zeros(W.shape), np.zeros(n)
    Ps = np.zeros((len(label), n))
    for r in have:
        logits = W @ x[r] + (0 if b is None else np.asarray(b, np.float64))
        top = logits.max()
        e = np.exp(logits - top)
        rows[r] = top + math.log(e.sum()) - logits[label[r]]
        P = e / e.sum()
        P[label[r]] -= 1
        Ps[r] = P
    out = dict(loss=rows[have].mean() if have else 0.0, rows=rows)
    if dloss is not None:
        s = dloss / len(have) if have else 0.0
        live = np.asarray(have, np.int64)
        dx[live] = Ps[live] @ W * s
        dW = Ps[live].T @ x[live] * s
        db = Ps[live].sum(0) * s
        out.update(dx=dx, dW=dW, db=db, P=Ps)
    return out


def e4m3(code):
    """The number of a code (sign, 4 bits of exponent with bias 7, 3 of mantissa; 0x7f and 0xff NaN)."""
    s, e, f = -1.0 if code & 0x80 else 1.0, code >> 3 & 15, code & 7
    if code & 0x7f == 0x7f:
        return math.nan
    return s * (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))


E4M3 = np.array([e4m3(c) for c in range(256)])


def nearest_code(a):
    """The code of the number nearest to a in [0, 448], of two equally near ones the even one."""
    best = min(range(127), key=lambda c: (abs(E4M3[c] - a), c & 1))
    return best


def to8(values, root=False):
    """(codes, biased exponents) of values, or of their roots, for blocks of 32."""
    v = np.asarray(values, np.float64).ravel()
    codes, exps = np.zeros(len(v), np.uint8), np.zeros(-(-len(v) // 32), np.uint8)
    for k in range(len(exps)):
        block = v[32 * k:32 * k + 32]
        block = np.sqrt(block) if root else block
        finite = np.abs(block[np.isfinite(block)])
        top = finite.max() if len(finite) else 0.0
        e = -127
        while e < 127 and top > 448 * 2.0 ** e:
            e += 1
        exps[k] = e + 127
        for j, x in enumerate(block):
            if not np.isfinite(x):
                codes[32 * k + j] = 0xff if x < 0 else 0x7f
                continue
            c = nearest_code(abs(x) * 2.0 ** -e)
            if root and x > 0 and c == 0:
                c = 1
            codes[32 * k + j] = c | (0x80 if x < 0 else 0)
    return codes, exps


def from8(codes, exps, root=False):
    v = E4M3[codes] * 2.0 ** (np.repeat(exps.astype(np.int64), 32)[:len(codes)] - 127)
    return v * v if root else v


def adamw(p, g, m, v, lr, beta1, beta2, eps, t, decay):
    """(p, m, v) after the step, all in 64 bits."""
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * (g * g)
    step = (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return p * (1 - lr * decay) - lr * step, m, v
