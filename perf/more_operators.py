"""The operators of a model that predicts among all nodes, as they are measured.

Four operators that such a model's training step chains, next to the memory update, the sequence operators and the link
loss with one negative an event: the rows of a table by id, a layer norm, the softmax cross entropy of each row's label
over all the nodes, and an AdamW step over all of the model's tensors.

Formulas:

  embed  y_r = scale table[id_r] (zeros where the id is no row);  dtable_i = scale sum of dy_r over the rows with id i
  norm   m = mean x_r, q = 1 / sqrt(mean (x_r - m)^2 + eps), h = (x_r - m) q,  y = gamma h + beta;
         with g = dy gamma:  dx = q (g - mean g - h mean(g h)) + past,  dgamma = sum dy h,  dbeta = sum dy
  loss   l = x W^T + b,  loss_r = log(sum_c exp l_rc) - l_r,label,  loss = their mean over the rows that have a label;
         P = (softmax(l) - [c is the label]) / rows with a label:  dx = P W,  dW = P^T x,  db = sum_r P
  adamw  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
         p = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)

with m and v held in float32, or in 8 bits: m and sqrt(v) as e4m3 numbers (to the nearest, ties to even, a sqrt(v) that is
not zero never to zero) times a power of two for each 32 elements, the least that keeps them within 448.

``own`` chooses between the plain form (elementary torch operations, in 32 bits, and in 64 what is then
rounded to 8) and this repository's kernels; ``exact`` gives the values in 64 bits.
"""

import math
import random
from types import SimpleNamespace

import torch

own = False

LR, BETA1, BETA2, EPS, STEP = 1e-3, 0.9, 0.999, 1e-8, 10


# --------------------------------------------------------------------------- cases

def _embed(name, kind, rows, n, d, dtype, scale=1.0, skew=1.0, missing=0.0, pad=0):
    c = dict(kind=kind, rows=rows, n=n, d=d, dtype=dtype, scale=scale, skew=skew, missing=missing, pad=pad)
    return dict(c, name=name) if name else c


def _norm(name, kind, rows, d, dtype, affine=True, past=False, pad=0, wide=0):
    c = dict(kind=kind, rows=rows, d=d, dtype=dtype, affine=affine, past=past, pad=pad, wide=wide)
    return dict(c, name=name) if name else c


def _loss(name, kind, rows, n, d, dtype, bias=True, ignored=0.0, pad=0):
    c = dict(kind=kind, rows=rows, n=n, d=d, dtype=dtype, bias=bias, ignored=ignored, pad=pad)
    return dict(c, name=name) if name else c


def _adamw(name, tensors, smallest, largest, mix, bits, shadow=False):
    c = dict(kind="adamw", tensors=tensors, smallest=smallest, largest=largest, mix=mix, bits=bits, shadow=shadow)
    return dict(c, name=name) if name else c


def listed():
    """missing: share of the ids that are no row (a node without a neighbour); ignored: share of the rows without a
    label; pad: rows behind the last; wide: columns beside x's in its matrix; mix: what the tensors' sizes are drawn by."""
    return [
        # serving: the rows of a few nodes, latency
        _embed("embed-step-tiny-f32", "embed_fwd", 16, 9_000, 100, "f32", pad=4),
        # training: both endpoints of a batch's events, a table of all nodes
        _embed("embed-train-events-f32", "embed_train", 8_000, 100_000, 100, "f32", 1.0, 1.2, 0.05, 100),
        # training over long sequences, a wide table, ids as skewed as the streams' nodes
        _embed("embed-train-bf16", "embed_train", 32_768, 50_000, 1_024, "bf16", 32.0, 1.0),
        # serving: one row for each of a few sequences
        _norm("norm-step-bf16", "norm_fwd", 24, 2_048, "bf16"),
        # training: a batch's rows of an odd width, x a column range of a wider matrix
        _norm("norm-train-odd-f32", "norm_train", 7_997, 445, "f32", pad=3, wide=100),
        # training over long sequences, with the residual stream's gradient
        _norm("norm-train-bf16", "norm_train", 16_384, 2_048, "bf16", past=True),
        # evaluation: one batch's events ranked among the smaller stream's nodes
        _loss("loss-eval-f32", "loss_fwd", 200, 9_000, 100, "f32", ignored=0.1),
        # training: the same with the events of a large batch, a few of them masked
        _loss("loss-train-events-f32", "loss_train", 4_000, 9_001, 100, "f32", ignored=0.15, pad=50),
        # serving: a few rows against a large table, for their likelihoods
        _loss("loss-eval-wide-bf16", "loss_fwd", 33, 100_003, 520, "bf16", bias=False),
        # training over long sequences, a few rows (those of a prompt) without a label
        _loss("loss-train-bf16", "loss_train", 8_192, 32_768, 1_024, "bf16", ignored=0.1),
        # the tensors of a small model, from biases to matrices
        _adamw("adamw-small-f32", 26, 1, 160_000, 1, 32, True),
        # the tensors of a large one, in 8 bits, with the copy that its products read
        _adamw("adamw-large-8bit", 150, 1_000, 8_000_000, 2, 8, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("embed_fwd", "embed_train", "norm_fwd", "norm_train", "loss_fwd", "loss_train", "adamw"))
    dtype = rng.choice(("f32", "bf16"))
    pad = rng.choice((0, 0, rng.randint(1, 200)))
    if kind == "adamw":
        bits, tensors = rng.choice((32, 8)), _log(rng, 1, 400)
        smallest = _log(rng, 1, 10_000)
        return _adamw(None, tensors, smallest, _log(rng, smallest, min(20e6, 4e8 / tensors)), rng.randint(3, 10 ** 6), bits,
                      rng.random() < 0.5)
    if kind.startswith("embed"):
        d = rng.choice((_log(rng, 1, 2_048), 32, 100, 128, 1_024))
        n = _log(rng, 2, min(1_000_000, 60e6 / d))
        return _embed(None, kind, _log(rng, 1, min(200_000, 40e6 / d)), n, d, dtype, rng.choice((1.0, 0.5, math.sqrt(d))),
                      round(rng.uniform(0.0, 1.3), 2), rng.choice((0.0, 0.05)), pad)
    if kind.startswith("norm"):
        d = rng.choice((_log(rng, 8, 16_384), 100, 1_024, 2_048, 4_096))
        return _norm(None, kind, _log(rng, 1, min(200_000, 33e6 / d)), d, dtype, rng.random() < 0.8, rng.random() < 0.5, pad,
                     rng.choice((0, 0, rng.randint(1, 200))))
    d = rng.choice((_log(rng, 8, 2_048), 32, 100, 128, 1_024))
    top = 2.2e11 if dtype == "bf16" else 4e10
    n = _log(rng, 2, min(200_000, top / d))
    return _loss(None, kind, _log(rng, 1, max(2, min(16_384, top / (n * d)))), n, d, dtype, rng.random() < 0.6,
                 rng.choice((0.0, 0.1, 0.5)), pad)


# --------------------------------------------------------------------------- inputs

def _dt(c):
    return torch.bfloat16 if c.dtype == "bf16" else torch.float32


def _sizes(c):
    rng = random.Random(c.mix)
    return [_log(rng, c.smallest, c.largest) for _ in range(c.tensors)]


def _zipf(gen, rows, n, skew):
    """Ids below n, the i-th most frequent one (i + 1)^-skew as often as the first, which id that is spread over the range."""
    p = torch.arange(1, n + 1, device="cuda", dtype=torch.float64) ** -skew
    p = torch.cumsum(p, 0)
    u = torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64) * p[-1]
    return torch.randperm(n, generator=gen, device="cuda")[torch.searchsorted(p, u).clamp_(max=n - 1)].int()


def _inputs(case, seed):
    """What a program has in hand: the tensors of one call, made on the GPU from the seed."""
    c = SimpleNamespace(**case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 6007 + 31)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")   # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=gen, device="cuda")     # noqa: E731
    v = SimpleNamespace(c=c)
    if c.kind == "adamw":
        # a tensor each in buffers for all of them, as a program keeps them that reduces or saves them together
        v.sizes = _sizes(c)
        v.room = [-(-n // 256) * 256 for n in v.sizes]
        total = sum(v.room)
        room = torch.tensor(v.room, device="cuda")
        behind = torch.arange(total, device="cuda")
        start = torch.cumsum(room, 0) - room
        behind -= torch.repeat_interleave(start, room, output_size=total)
        inside = behind < torch.repeat_interleave(torch.tensor(v.sizes, device="cuda"), room, output_size=total)
        del behind
        # gradients of unlike tensors are of unlike sizes
        size = 10 ** (torch.tensor([random.Random(c.mix + 1 + i).uniform(-5, -2) for i in range(c.tensors)], device="cuda"))
        each = torch.repeat_interleave(size, room, output_size=total) * inside
        v.p, v.g, v.m = randn(total) * 0.05 * inside, randn(total) * each, randn(total) * each * 0.3
        v.v = (each * (0.3 + rand(total))) ** 2
        del each, inside
        v.decay = [0.1 if n > 1_000 else 0.0 for n in v.sizes]   # none for biases and norms
        v.shadow = v.p.bfloat16() if c.shadow else None
        if c.bits == 8:
            (v.m, v.m_exp), (v.v, v.v_exp) = _to8(v.m.double(), False), _to8(v.v.double(), True)
        return v
    dt, R = _dt(c), c.rows + c.pad
    v.R, v.dt = R, dt
    v.n_rows = torch.tensor([c.rows], dtype=torch.int32, device="cuda")
    if c.kind.startswith("embed"):
        v.table = (randn(c.n, c.d) / math.sqrt(c.d)).to(dt)
        v.ids = _zipf(gen, R, c.n, c.skew)
        v.ids[rand(R) < c.missing] = -1
        if c.kind == "embed_train":
            v.dy = randn(R, c.d) * 0.01
    elif c.kind.startswith("norm"):
        # rows of unlike sizes, channels of unlike means, as a residual stream has them
        w = ((randn(R, c.d + c.wide) + 0.5 * randn(c.d + c.wide)) * torch.exp(0.5 * randn(R, 1))).to(dt)
        v.x = w[:, :c.d]
        v.gamma = 1 + 0.2 * randn(c.d) if c.affine else None
        v.beta = 0.1 * randn(c.d) if c.affine else None
        if c.kind == "norm_train":
            v.dy = randn(R, c.d) * 0.01
            v.past = randn(R, c.d) * 0.01 if c.past else None
    else:
        v.x = randn(R, c.d).to(dt)
        v.W = (randn(c.n, c.d) * (2 / math.sqrt(c.d))).to(dt)
        v.b = -torch.log(1 + c.n * rand(c.n)) if c.bias else None   # frequencies of a skewed stream
        v.label = _zipf(gen, R, c.n, 1.0)
        v.label[rand(R) < c.ignored] = -1
        v.label[0] = c.n - 1
    return v


def prepare(case, seed):
    v = _inputs(case, seed)
    if own:
        _own_buffers(v)
    return v


def run(state):
    return (_OWN if own else _PLAIN)[state.c.kind](state)


# --------------------------------------------------------------------------- numbers in 8 bits

def _blocks(t):
    """[blocks, 32], the last one filled with zeros."""
    n = t.numel()
    return torch.nn.functional.pad(t, (0, -n % 32)).view(-1, 32)


def _to8(t, square):
    """(e4m3 numbers, biased exponents) of t, or of its roots (square) in 64 bits: scale 2^(e - 127), the least that keeps a
    block within 448."""
    b = _blocks(t)
    b = torch.sqrt(b) if square else b
    top = b.abs().amax(1)
    f, e = torch.frexp(top)                              # top = f 2^e, f in [0.5, 1): 448 = 0.875 2^9
    e = torch.where(top > 0, e + (f > 0.875).int() - 9, torch.full_like(e, -127)).clamp(-127, 127)
    a = torch.ldexp(b, -e[:, None]).abs()
    step = torch.ldexp(torch.ones_like(a), torch.frexp(a)[1].clamp(min=-5) - 4)   # three bits behind the first; 2^-9 below 2^-6
    q = torch.round(a / step) * step
    if square:
        q = torch.where((a > 0) & (q == 0), torch.full_like(q, 2.0 ** -9), q)
    q = torch.copysign(q, b).view(-1)[:t.numel()]
    return q.float().to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _scale(e):
    """The block scales that exponents stand for."""
    return torch.exp2(e.float() - 127)


def _from8(q, e, square):
    v = torch.ldexp(_blocks(q.double()), e[:, None].int() - 127)
    v = v.view(-1)[:q.numel()]
    return v * v if square else v


# --------------------------------------------------------------------------- the plain forms, in 32 bits

def _pad_rows(t, v):
    n = t.shape[0]
    return t if n == v.R else torch.cat([t, torch.zeros(v.R - n, *t.shape[1:], dtype=t.dtype, device=t.device)])


def _plain_embed(v):
    c, ids = v.c, v.ids[:v.c.rows].long()
    known = (ids >= 0) & (ids < c.n)
    y = v.table[ids.clamp(0, c.n - 1)].float() * c.scale
    return _pad_rows(torch.where(known[:, None], y, torch.zeros_like(y)).to(v.dt), v)


def _plain_embed_train(v):
    c, ids = v.c, v.ids[:v.c.rows].long()
    dtable = torch.zeros(c.n + 1, c.d, device="cuda")   # the last row takes what has no id
    known = (ids >= 0) & (ids < c.n)
    dtable.index_add_(0, torch.where(known, ids, torch.full_like(ids, c.n)), v.dy[:c.rows])
    return dict(y=_plain_embed(v), dtable=dtable[:c.n] * c.scale)


def _plain_norm_parts(v):
    x = v.x[:v.c.rows].float()
    x = x - x.mean(1, keepdim=True)
    q = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5)
    h = x * q
    y = h if v.gamma is None else h * v.gamma + v.beta
    return h, q, _pad_rows(y.to(v.dt), v)


def _plain_norm(v):
    return _plain_norm_parts(v)[2]


def _plain_norm_train(v):
    h, q, y = _plain_norm_parts(v)
    dy = v.dy[:v.c.rows]
    g = dy if v.gamma is None else dy * v.gamma
    dx = q * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    if v.past is not None:
        dx = dx + v.past[:v.c.rows]
    out = dict(y=y, dx=_pad_rows(dx, v))
    if v.gamma is not None:
        out.update(dgamma=(dy * h).sum(0), dbeta=dy.sum(0))
    return out


def _plain_loss_parts(v):
    """(rows' losses, softmax, which rows have a label, labels)."""
    c = v.c
    label = v.label[:c.rows].long()
    has = (label >= 0) & (label < c.n)
    label = label.clamp(0, c.n - 1)
    logits = v.x[:c.rows].float() @ v.W.float().t()
    if v.b is not None:
        logits += v.b
    top = logits.max(1, keepdim=True).values
    at = (logits.gather(1, label[:, None]) - top)[:, 0]
    e = torch.exp(logits.sub_(top))
    s = e.sum(1, keepdim=True)
    rows = torch.where(has, torch.log(s[:, 0]) - at, torch.zeros_like(at))
    return rows, e.div_(s), has, label


def _plain_loss(v):
    rows, _, has, _ = _plain_loss_parts(v)
    return dict(loss=rows.sum() / has.sum(), rows=_pad_rows(rows, v))


def _plain_loss_train(v):
    rows, p, has, label = _plain_loss_parts(v)
    count = has.sum()
    p[torch.arange(v.c.rows, device="cuda"), label] -= 1
    p *= has[:, None] / count
    out = dict(loss=rows.sum() / count, rows=_pad_rows(rows, v), dx=_pad_rows(p @ v.W.float(), v),
               dW=p.t() @ v.x[:v.c.rows].float())
    if v.b is not None:
        out["db"] = p.sum(0)
    return out


def _plain_adamw(v):
    bc1, bc2 = 1 - BETA1 ** STEP, 1 - BETA2 ** STEP
    room = torch.tensor(v.room, device="cuda")
    decay = torch.repeat_interleave(torch.tensor(v.decay, device="cuda"), room, output_size=sum(v.room))
    if v.c.bits == 8:
        g = v.g.double()
        m = BETA1 * _from8(v.m, v.m_exp, False) + (1 - BETA1) * g
        s = BETA2 * _from8(v.v, v.v_exp, True) + (1 - BETA2) * g * g
        for store, exps, (q, e) in ((v.m, v.m_exp, _to8(m, False)), (v.v, v.v_exp, _to8(s, True))):
            store.copy_(q)
            exps.copy_(e)
        m, s = m.float(), s.float()
    else:
        m = v.m.mul_(BETA1).add_(v.g * (1 - BETA1))
        s = v.v.mul_(BETA2).add_(v.g * v.g * (1 - BETA2))
    v.p.mul_(1 - LR * decay).sub_(LR * (m / bc1) / (torch.sqrt(s / bc2) + EPS))
    if v.shadow is not None:
        v.shadow.copy_(v.p)
    return _adamw_out(v)


def _adamw_out(v):
    """What is held in 8 bits goes out as the numbers that it holds, and their blocks' scales."""
    out = dict(p=v.p, m=v.m, v=v.v)
    if v.c.bits == 8:
        out.update(m_scale=_scale(v.m_exp), v_scale=_scale(v.v_exp))
    if v.shadow is not None:
        out["shadow"] = v.shadow
    return out


_PLAIN = dict(embed_fwd=_plain_embed, embed_train=_plain_embed_train, norm_fwd=_plain_norm, norm_train=_plain_norm_train,
              loss_fwd=_plain_loss, loss_train=_plain_loss_train, adamw=_plain_adamw)


# --------------------------------------------------------------------------- this repository's kernels

def _own_buffers(v):
    """Outputs, saves and workspaces, as a program keeps them from call to call."""
    from paper_2608_16305_amd import mtgnn as M
    v.M, c = M, v.c
    f32 = lambda *s: torch.zeros(*s, device="cuda")   # noqa: E731
    if c.kind == "adamw":
        def each(t, per=1):
            return None if t is None else [x[:-(-n // per)] for x, n in zip(t.split([n // per for n in v.room]), v.sizes)]
        scales = dict(m_exp=each(v.m_exp, 32), v_exp=each(v.v_exp, 32)) if c.bits == 8 else {}
        v.tensors = M.adamw_tensors(each(v.p), each(v.g), each(v.m), each(v.v), shadow=each(v.shadow), decay=v.decay, **scales)
        return
    code, train = M.BF16 if c.dtype == "bf16" else M.F32, c.kind.endswith("train")
    rows = lambda *s: torch.zeros(v.R, *s, dtype=v.dt, device="cuda")   # noqa: E731
    if c.kind.startswith("embed"):
        v.d, v.y = M.embedding_dims(c.n, c.d, code, c.scale), rows(c.d)
        if train:
            v.dtable, v.ws = f32(c.n, c.d), M.alloc_bytes(M.embedding_ws_bytes(v.d, v.R))
    elif c.kind.startswith("norm"):
        v.d, v.y, v.stats = M.norm_dims(c.d, code, 1e-5), rows(c.d), f32(v.R, 2) if train else None
        if train:
            v.dx, v.ws = f32(v.R, c.d), M.alloc_bytes(M.layer_norm_ws_bytes(v.d, v.R))
            v.dgamma, v.dbeta = (f32(c.d), f32(c.d)) if c.affine else (None, None)
    else:
        v.d, v.loss, v.rows = M.loss_dims(c.n, c.d, code), f32(1), f32(v.R)
        v.ws = M.alloc_bytes(M.softmax_loss_ws_bytes(v.d, v.R, train))
        v.save = None
        if train:
            v.save = M.alloc_bytes(M.softmax_loss_save_bytes(v.d, v.R))
            v.dx, v.dW, v.db = f32(v.R, c.d), f32(c.n, c.d), f32(c.n) if c.bias else None


def _own_embed(v):
    v.M.mtgnn_embedding(v.ids, v.table, v.d, v.y, n_rows=v.n_rows)
    return v.y


def _own_embed_train(v):
    v.M.mtgnn_embedding(v.ids, v.table, v.d, v.y, n_rows=v.n_rows)
    v.M.mtgnn_embedding_bwd(v.ids, v.dy, v.d, v.dtable, v.ws, n_rows=v.n_rows)
    return dict(y=v.y, dtable=v.dtable)


def _own_norm(v):
    v.M.mtgnn_layer_norm(v.x, v.gamma, v.beta, v.d, v.y, n_rows=v.n_rows)
    return v.y


def _own_norm_train(v):
    v.M.mtgnn_layer_norm(v.x, v.gamma, v.beta, v.d, v.y, stats=v.stats, n_rows=v.n_rows)
    v.M.mtgnn_layer_norm_bwd(v.dy, v.x, v.gamma, v.stats, v.d, v.dx, v.dgamma, v.dbeta, past=v.past, n_rows=v.n_rows, ws=v.ws)
    out = dict(y=v.y, dx=v.dx)
    if v.gamma is not None:
        out.update(dgamma=v.dgamma, dbeta=v.dbeta)
    return out


def _own_loss(v):
    v.M.mtgnn_softmax_loss(v.x, v.W, v.b, v.label, v.d, v.loss, v.ws, row_loss=v.rows, n_rows=v.n_rows)
    return dict(loss=v.loss[0], rows=v.rows)


def _own_loss_train(v):
    v.M.mtgnn_softmax_loss(v.x, v.W, v.b, v.label, v.d, v.loss, v.ws, row_loss=v.rows, save=v.save, n_rows=v.n_rows)
    v.M.mtgnn_softmax_loss_bwd(v.x, v.W, v.b, v.label, v.d, v.save, v.dx, v.dW, v.db, v.ws, n_rows=v.n_rows)
    out = dict(loss=v.loss[0], rows=v.rows, dx=v.dx, dW=v.dW)
    if v.b is not None:
        out["db"] = v.db
    return out


def _own_adamw(v):
    v.M.mtgnn_adamw_step(v.tensors, LR, BETA1, BETA2, EPS, STEP)
    return _adamw_out(v)


_OWN = dict(embed_fwd=_own_embed, embed_train=_own_embed_train, norm_fwd=_own_norm, norm_train=_own_norm_train,
            loss_fwd=_own_loss, loss_train=_own_loss_train, adamw=_own_adamw)


# --------------------------------------------------------------------------- least work

def work(case):
    """Every input read once, every output written once; an exponential counts as one operation."""
    c = SimpleNamespace(**case)
    if c.kind == "adamw":
        n = sum(_sizes(c))
        return dict(bytes=n * ((28 if c.bits == 32 else 16.125) + (2 if c.shadow else 0)), flops=14 * n)
    e, R, train = 2 if c.dtype == "bf16" else 4, c.rows, c.kind.endswith("train")
    if c.kind.startswith("embed"):
        by, fl = R * (4 + 2 * e * c.d), R * c.d
        if train:
            by, fl = by + 4 * R * c.d + 4 * c.n * c.d, fl + R * c.d + c.n * c.d
    elif c.kind.startswith("norm"):
        by, fl = 2 * e * R * c.d + (8 * c.d if c.affine else 0), 8 * R * c.d
        if train:
            by, fl = by + (12 if c.past else 8) * R * c.d + (8 * c.d if c.affine else 0), fl + 14 * R * c.d
    else:
        live = R * (1 - c.ignored)
        by, fl = e * (live + c.n) * c.d + 8 * R + (4 * c.n if c.bias else 0), 2 * live * c.n * c.d + 3 * live * c.n
        if train:
            by, fl = by + 4 * (R + c.n) * c.d + (4 * c.n if c.bias else 0), fl + 4 * live * c.n * c.d + 3 * live * c.n
    return dict(bytes=by, flops=fl)


# --------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    v = _inputs(case, seed)
    return _EXACT[v.c.kind](v)


def _exact_embed(v):
    c = v.c
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")   # noqa: E731
    rows = torch.nonzero((v.ids[:c.rows] >= 0) & (v.ids[:c.rows] < c.n))[:, 0]
    at = v.ids[rows].long()
    y = z(v.R, c.d)
    y[rows] = c.scale * v.table.double()[at]
    if c.kind == "embed_fwd":
        return y
    # sums of runs of equal ids, as differences of the running sums: 64 bits hold them to 1e-12
    order = torch.argsort(at, stable=True)
    run = torch.cat([z(1, c.d), torch.cumsum(v.dy.double()[rows[order]], 0)])
    off = torch.searchsorted(at[order].contiguous(), torch.arange(c.n + 1, device="cuda"))
    return dict(y=y, dtable=c.scale * (run[off[1:]] - run[off[:-1]]))


def _exact_norm(v):
    n, x = v.c.rows, v.x[:v.c.rows].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    sd = torch.sqrt(var + 1e-5)
    gamma = torch.ones(v.c.d, dtype=torch.float64, device="cuda") if v.gamma is None else v.gamma.double()
    beta = 0.0 if v.beta is None else v.beta.double()
    zero = lambda: torch.zeros(v.R, v.c.d, dtype=torch.float64, device="cuda")   # noqa: E731
    y = zero()
    y[:n] = gamma * (x - mean) / sd + beta
    if v.c.kind == "norm_fwd":
        return y
    dy, h = v.dy[:n].double(), (x - mean) / sd
    # the slope without its parts along the ones and along h
    g, dx = dy * gamma, zero()
    g = g - g.sum(1, keepdim=True) / v.c.d
    dx[:n] = (g - h * ((g * h).sum(1, keepdim=True) / v.c.d)) / sd
    if v.past is not None:
        dx[:n] += v.past[:n].double()
    out = dict(y=y, dx=dx)
    if v.gamma is not None:
        out.update(dgamma=(h * dy).sum(0), dbeta=dy.sum(0))
    return out


def _exact_loss(v):
    c = v.c
    live = torch.nonzero((v.label[:c.rows] >= 0) & (v.label[:c.rows] < c.n))[:, 0]
    at, x, W = v.label[live].long(), v.x.double()[live], v.W.double()
    logits = torch.mm(x, W.t().contiguous())
    if v.b is not None:
        logits += v.b.double()
    total = torch.logsumexp(logits, 1)
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")   # noqa: E731
    rows = z(v.R)
    rows[live] = total - logits[torch.arange(live.numel(), device="cuda"), at]
    out = dict(loss=rows.sum() / live.numel(), rows=rows)
    if c.kind == "loss_fwd":
        return out
    p = torch.exp(logits - total[:, None]) / live.numel()
    dx, dW = z(v.R, c.d), torch.mm(p.t().contiguous(), x)
    dx[live] = torch.mm(p, W) - W[at] / live.numel()
    dW.index_put_((at,), -x / live.numel(), accumulate=True)
    out.update(dx=dx, dW=dW)
    if v.b is not None:
        out["db"] = p.sum(0) - torch.bincount(at, minlength=c.n) / live.numel()
    return out


def _code64(t, square):
    """_to8 by search among the 127 numbers that e4m3 has: (values in units of the block's scale, scales)."""
    codes = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    b = _blocks(t)
    top = b.abs().amax(1)
    limit = 448.0 ** 2 if square else 448.0
    grow = torch.arange(-127, 128, dtype=torch.float64, device="cuda")
    grow = torch.exp2(2 * grow if square else grow) * limit
    e = torch.searchsorted(grow, top).clamp(max=254)       # the first that is not below the largest
    unit = torch.exp2(e.double() - 127)
    a = (b / (unit * unit)[:, None]).clamp(min=0) if square else b.abs() / unit[:, None]
    mid = (codes[1:] + codes[:-1]) / 2
    mid = mid * mid if square else mid
    hi = torch.searchsorted(mid, a.contiguous())           # below a midpoint, or on it: the lower one ...
    tie = (hi < 126) & (a == mid[hi.clamp(max=125)]) & (hi % 2 == 1)
    hi = hi + tie.long()                                   # ... unless that one's code is odd
    if square:
        hi = torch.where((a > 0) & (hi == 0), torch.ones_like(hi), hi)
    q = torch.copysign(codes[hi], b).view(-1)[:t.numel()]
    return q, unit


def _exact_adamw(v):
    bc1, bc2 = 1 - BETA1 ** STEP, 1 - BETA2 ** STEP
    p, g, m, s = (t.double() for t in (v.p, v.g, v.m, v.v))
    if v.c.bits == 8:
        m = (m.view(-1, 32) * torch.exp2(v.m_exp.double() - 127)[:, None]).view(-1)
        s = (s.view(-1, 32) * torch.exp2(v.v_exp.double() - 127)[:, None]).view(-1) ** 2
    m = BETA1 * m + (1 - BETA1) * g
    s = BETA2 * s + (1 - BETA2) * g ** 2
    first = 0
    for n, decay in zip(v.room, v.decay):
        p[first:first + n] *= 1 - LR * decay
        first += n
    p -= LR * (m / bc1) / ((s / bc2) ** 0.5 + EPS)
    out = dict(p=p, m=m, v=s)
    if v.c.bits == 8:
        (out["m"], out["m_scale"]), (out["v"], out["v_scale"]) = _code64(m, False), _code64(s, True)
    if v.c.shadow:
        out["shadow"] = p
    return out


_EXACT = dict(embed_fwd=_exact_embed, embed_train=_exact_embed, norm_fwd=_exact_norm, norm_train=_exact_norm,
              loss_fwd=_exact_loss, loss_train=_exact_loss, adamw=_exact_adamw)
