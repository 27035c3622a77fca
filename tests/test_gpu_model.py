"""The operators of a model over all nodes on the GPU through the C ABI, against the 64-bit oracle.

Tolerances are those of a 32-bit evaluation, per element, from the magnitudes that its roundings are relative to
(u = 2^-24, half a step of float32):
  embedding  one product; the gradient n - 1 sums and a product for an id of n rows: (n + 1) u of the terms' magnitude;
  norm       a row's sums are chains of at most 64 + d / 256 additions: so many u of the mean magnitudes, which enter as the
             formulas say (a wrong mean moves every h by q of it), and a few u for each operation on an element;
  loss       a logit is a sum of d products, (d + 4) u of their magnitudes, and 8 u more where each float32 factor is two
             float16 parts (2 u each, and 4 u the product of the second parts); an exponential is off by that, its own two u
             and the difference's; a row's sum is a chain of at most 64 + n / 2,048; P is held to 2 u of itself or 2^-39;
             sums of K products add K u of their magnitudes; an element in float16 parts is held to 2^-39 of its
             matrix's largest where that is more;
  adamw      a few u of each term; in 8 bits the codes and exponents are the oracle's.
An output in bfloat16 is rounded once more, by 2^-8 of itself."""

import numpy as np
import pytest
import torch

from oracle import model
from oracle.bf16 import round_bf16
from paper_2608_16305_amd import mtgnn as M
from tests._gpu import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

U = 2.0 ** -24
MARK = 7.25                       # what untouched memory keeps
BOTH = pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])


def _vals(rs, bf16, *shape):
    v = rs.randn(*shape).astype(np.float32)
    return round_bf16(v) if bf16 else v


def _dev(v, bf16=False):
    return torch.from_numpy(np.ascontiguousarray(v, np.float32)).cuda().to(torch.bfloat16 if bf16 else torch.float32)


def _in_wide(v, bf16=False, left=3, right=2):
    """The matrix as a column range of a wider one (NaN around it)."""
    wide = torch.full((v.shape[0], left + v.shape[1] + right), float("nan"))
    wide[:, left:left + v.shape[1]] = torch.from_numpy(np.ascontiguousarray(v, np.float32))
    return wide.cuda().to(torch.bfloat16 if bf16 else torch.float32)[:, left:left + v.shape[1]]


def _marked(rows, cols, bf16=False, wide=False):
    t = torch.full((rows, cols + (5 if wide else 0)), MARK, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    return t[:, 2:2 + cols] if wide else t


def _behind(v, pad):
    return np.concatenate([v, np.full((pad,) + v.shape[1:], np.nan, np.float32)]) if pad else v


def _count(rows, pad):
    return torch.tensor([rows], dtype=torch.int32, device="cuda") if pad else None


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _close(name, got, want, tol, bf16=False):
    got = _np(got) if isinstance(got, torch.Tensor) else got
    tol = tol + (2.0 ** -8 if bf16 else U) * np.abs(want) + 1e-37
    assert np.isfinite(got).all(), name
    bad = np.abs(got - want) > tol
    assert not bad.any(), (name, np.argwhere(bad)[:4].tolist(), float((np.abs(got - want) / tol).max()))


def _kept(name, t, rows):
    assert (t[rows:].float() == MARK).all(), name


# --------------------------------------------------------------------------- embedding

EMBED = [  # rows, pad, n, d, scale, ids (how many different), share that is no row, wide
    (1, 0, 1, 1, 1.0, 1, 0.0, False),
    (1, 3, 5, 7, -2.5, 5, 0.0, True),
    (3, 0, 4, 4, 1.0, 4, 1.0, False),
    (64, 0, 100, 100, 0.5, 100, 0.1, False),
    (65, 7, 1000, 129, 1.0, 50, 0.3, True),
    (33, 0, 3, 8, 1.0, 1, 0.0, False),
    (32, 0, 3, 8, 3.0, 1, 0.0, True),
    (1000, 24, 7, 36, 1.0, 3, 0.2, False),
    (1025, 0, 2, 3, 1.0, 2, 0.0, False),
    (5000, 100, 300, 20, 0.125, 300, 0.05, True),
    (4099, 0, 70000, 12, 1.0, 70000, 0.0, False),
    (9000, 0, 1025, 260, 1.0, 5, 0.01, False),
    (20000, 0, 9001, 3, 1.0, 2, 0.0, False),
    (30000, 11, 8192, 9, 1.0, 1, 0.0, True),
    (17000, 3, 3000, 260, 0.5, 700, 0.01, True),
]


@BOTH
@pytest.mark.parametrize("case", EMBED, ids=str)
def test_embedding(case, bf16):
    rows, pad, n, d, scale, kinds, none, wide = case
    rs = np.random.RandomState(rows + n)
    table, dy = _vals(rs, bf16, n, d), _vals(rs, False, rows, d)
    ids = rs.permutation(n)[:kinds][rs.randint(0, kinds, rows)].astype(np.int32)
    ids[rs.rand(rows) < none] = rs.choice([-1, n, -2 ** 31, 2 ** 31 - 1])
    I = torch.from_numpy(np.concatenate([ids, np.zeros(pad, np.int32)])).cuda()
    e = M.embedding_dims(n, d, M.BF16 if bf16 else M.F32, scale)
    y, dtable = _marked(rows + pad, d, bf16, wide), _marked(n, d)
    G = (_in_wide if wide else _dev)(_behind(dy, pad))
    M.mtgnn_embedding(I, _dev(table, bf16), e, y, n_rows=_count(rows, pad))
    ws = M.alloc_bytes(M.embedding_ws_bytes(e, rows + pad)).fill_(255)
    M.mtgnn_embedding_bwd(I, G, e, dtable, ws, n_rows=_count(rows, pad))
    want, mag = model.embedding(ids, table, scale, dy), model.embedding(ids, table, abs(scale), np.abs(dy))
    _close("y", y[:rows], want["y"], 0, bf16)
    _kept("y", y, rows)
    count = np.bincount(ids[(ids >= 0) & (ids < n)], minlength=n)[:, None]
    _close("dtable", dtable, want["dtable"], (count + 1) * U * mag["dtable"])
    assert (_np(dtable)[count[:, 0] == 0] == 0).all()
    again = _marked(n, d)
    M.mtgnn_embedding_bwd(I, G, e, again, ws.fill_(1), n_rows=_count(rows, pad))
    assert torch.equal(again, dtable)


# --------------------------------------------------------------------------- layer norm

NORM = [  # rows, pad, d, affine, past, wide
    (1, 0, 1, True, False, False),
    (1, 0, 8, False, False, False),
    (2, 3, 7, True, True, True),
    (5, 0, 256, True, False, False),
    (65, 7, 100, True, True, False),
    (9, 0, 257, False, True, True),
    (7, 2, 445, True, False, True),
    (31, 0, 513, True, True, False),
    (6, 0, 1025, True, False, True),
    (2100, 20, 24, True, True, False),
    (1500, 0, 1032, True, False, False),
    (3, 1, 2049, False, True, False),
    (4, 0, 4097, True, True, True),
    (3, 0, 8193, True, False, True),
    (70, 2, 9000, True, True, False),
    (2, 0, 33000, True, True, True),
    (9000, 30, 21, True, True, True),
    (17001, 0, 8, True, False, False),
]


def _norm_tolerances(x, gamma, dy, past, want):
    d = x.shape[1]
    c = 64 + d / 256
    q, h = want["q"][:, None], want["h"]
    e_h = q * c * U * np.abs(x).mean(1, keepdims=True) + (c + 12) * U * np.abs(h) + q * 2 * U * np.abs(x)
    e_h = e_h + np.abs(h) * (q * c * U * np.abs(x).mean(1, keepdims=True)) ** 2
    ga = np.ones(d) if gamma is None else np.abs(gamma)
    out = dict(h=e_h, y=ga * e_h + 4 * U * (ga * np.abs(h)) + 2 * U * np.abs(want["y"]))
    if dy is not None:
        g = np.abs(dy) * ga
        mean = lambda v: v.mean(1, keepdims=True)   # noqa: E731
        e_b = (c + 4) * U * mean(g * np.abs(h)) + mean(g * e_h)
        b = np.abs(mean(dy * (1 if gamma is None else gamma) * h))
        size = g + mean(g) + np.abs(h) * b
        out["dx"] = q * (4 * U * g + (c + 4) * U * mean(g) + np.abs(h) * e_b + e_h * b + (c + 16) * U * size)
        if past is not None:
            out["dx"] = out["dx"] + 2 * U * np.abs(past)
        out["dgamma"] = ((len(x) + 4) * U * np.abs(dy) * np.abs(h) + np.abs(dy) * e_h).sum(0)
        out["dbeta"] = len(x) * U * np.abs(dy).sum(0)
    return out


@BOTH
@pytest.mark.parametrize("case", NORM, ids=str)
def test_layer_norm(case, bf16):
    rows, pad, d, affine, past, wide = case
    rs = np.random.RandomState(rows + d)
    x = _vals(rs, bf16, rows, d) * np.float32(2.0) ** rs.randint(-3, 4, (rows, 1)).astype(np.float32) + np.float32(2)
    x = round_bf16(x) if bf16 else x
    gamma, beta = (_vals(rs, False, d), _vals(rs, False, d)) if affine else (None, None)
    dy, extra = _vals(rs, False, rows, d), _vals(rs, False, rows, d) if past else None
    place = _in_wide if wide else _dev
    X, G = place(_behind(x, pad), bf16), place(_behind(dy, pad))
    E = place(_behind(extra, pad)) if past else None
    e = M.norm_dims(d, M.BF16 if bf16 else M.F32, 1e-5)
    dev = lambda v: None if v is None else _dev(v)   # noqa: E731
    y, stats, n = _marked(rows + pad, d, bf16, wide), _marked(rows + pad, 2), _count(rows, pad)
    M.mtgnn_layer_norm(X, dev(gamma), dev(beta), e, y, stats=stats, n_rows=n)
    y2 = _marked(rows + pad, d, bf16, wide)
    M.mtgnn_layer_norm(X, dev(gamma), dev(beta), e, y2, n_rows=n)
    want = model.layer_norm(x, gamma, beta, np.float32(1e-5), dy, extra)
    tol = _norm_tolerances(x, gamma, dy, extra, want)
    _close("y", y[:rows], want["y"], tol["y"], bf16)
    assert torch.equal(y2[:rows], y[:rows])
    _kept("y", y, rows)
    _kept("stats", stats, rows)
    ws = M.alloc_bytes(M.layer_norm_ws_bytes(e, rows + pad)).fill_(255)
    dx, dgamma, dbeta = _marked(rows + pad, d, wide=wide), _marked(1, d)[0], _marked(1, d)[0]
    M.mtgnn_layer_norm_bwd(G, X, dev(gamma), stats, e, dx, dgamma, dbeta, past=E, n_rows=n, ws=ws)
    _close("dx", dx[:rows], want["dx"], tol["dx"])
    _kept("dx", dx, rows)
    _close("dgamma", dgamma, want["dgamma"], tol["dgamma"])
    _close("dbeta", dbeta, want["dbeta"], tol["dbeta"])
    # without the sums over rows, dx in dy's place; then in past's
    own = G.clone(memory_format=torch.preserve_format) if not wide else G
    M.mtgnn_layer_norm_bwd(own, X, dev(gamma), stats, e, own, None, None, past=E, n_rows=n)
    assert torch.equal(own[:rows], dx[:rows])
    if past:
        G2 = place(_behind(dy, pad))
        M.mtgnn_layer_norm_bwd(G2, X, dev(gamma), stats, e, E, None, None, past=E, n_rows=n)
        assert torch.equal(E[:rows], dx[:rows])


def test_layer_norm_far_rows_and_constant_rows():
    """A row far from zero keeps its deviations; a constant row is beta; NaN and infinity stay in their row."""
    rs = np.random.RandomState(5)
    x = rs.randn(6, 96).astype(np.float32)
    x[1] += 4096.0
    x[2] = 0.1
    x[3, 5], x[4, 7] = np.nan, np.inf
    e, y = M.norm_dims(96, M.F32, 1e-5), _marked(6, 96)
    M.mtgnn_layer_norm(_dev(x), None, None, e, y)
    got = _np(y)
    want = model.layer_norm(x[[0, 1, 5]], None, None, np.float32(1e-5))
    _close("rows", got[[0, 1, 5]], want["y"], _norm_tolerances(x[[0, 1, 5]], None, None, None, want)["y"])
    assert np.abs(got[2]).max() <= 96 * U * 0.1 / np.sqrt(1e-5) + U   # what the mean's rounding leaves
    assert np.isnan(got[3]).all() and np.isnan(got[4]).all()


# --------------------------------------------------------------------------- softmax loss

LOSS = [  # rows, pad, n, d, bias, share without a label, wide, dloss
    (1, 0, 1, 1, True, 0.0, False, None),
    (1, 0, 2, 8, False, 0.0, False, None),
    (3, 2, 5, 7, True, 0.3, True, 0.5),
    (64, 0, 64, 64, False, 0.0, False, None),
    (65, 0, 65, 65, True, 0.0, False, None),
    (17, 15, 129, 100, True, 0.5, True, -3.0),
    (130, 0, 300, 72, True, 0.1, False, None),
    (200, 56, 127, 32, False, 0.9, False, 2.0),
    (129, 0, 1000, 130, True, 0.0, True, None),
    (300, 0, 257, 520, False, 0.2, False, None),
    (2100, 30, 40, 16, True, 0.1, False, None),
    (5, 0, 4000, 200, True, 0.0, False, None),
    (3, 2, 70000, 20, True, 0.0, True, None),
    (9000, 0, 5, 33, True, 0.1, True, 0.25),
    (5, 3, 9, 12, True, 1.0, False, None),
    (33, 5, 65, 130, True, 0.2, True, None),
    (100, 0, 70, 33, True, 1.0, False, None),
    (256, 0, 500, 129, True, 0.0, True, None),
    (250, 6, 33, 68, False, 0.6, False, -1.0),
    (64, 0, 33000, 100, True, 0.0, False, 2.0),
    (20, 0, 40000, 65, False, 0.1, True, None),
]
# enough tiles of 256 for the larger kernels, forward and backward; whole and ragged ones
LOSS_BIG = [(3333, 40, 3800, 72, True, 0.03, True, None), (3584, 0, 3584, 64, False, 0.0, False, 1.5)]


def _loss_case(case, bf16):
    rows, pad, n, d, bias, none, wide, dloss = case
    rs = np.random.RandomState(rows + n)
    x, W = _vals(rs, bf16, rows, d), _vals(rs, bf16, n, d) * np.float32(2.0 / 2 ** round(np.log2(d) / 2))
    b = _vals(rs, False, n) if bias else None
    label = rs.randint(0, n, rows).astype(np.int32)
    out = rs.rand(rows) < none
    label[out] = rs.choice([-1, n, -2 ** 31, 2 ** 31 - 1], out.sum())
    x[out] = np.nan               # what a row without a label holds does not count
    return x, W, b, label, 1.0 if dloss is None else dloss


def _loss_tolerances(x, W, b, label, want, dloss, bf16):
    n, d = W.shape
    live = np.nonzero((label >= 0) & (label < n))[0]
    s = abs(dloss) / max(1, len(live))
    ax, aW = np.abs(x[live]).astype(np.float64), np.abs(W).astype(np.float64)
    mag = ax @ aW.T + (0 if b is None else np.abs(b))
    FLOOR = 2.0 ** -39
    e_l = (d + 4) * U * mag
    if not bf16:
        e_l = e_l + 8 * U * mag + FLOOR * (ax.max(initial=0) * aW.sum(1) + aW.max() * ax.sum(1)[:, None])
    logits = x[live].astype(np.float64) @ W.astype(np.float64).T + (0 if b is None else b)
    gap = logits.max(1, keepdims=True) - logits
    worst = e_l.max(1, keepdims=True)
    chain = (64 + n / 2048) * U
    rows = np.zeros(len(label))
    rows[live] = 2 * worst[:, 0] + chain + 4 * U * (np.abs(logits).max(1) + 1)
    p = want["P"][live] + (np.arange(n) == label[live][:, None])
    e_p = p * (np.exp(2 * worst) * (2 * worst + chain + (8 + 4 * gap) * U)) + 2 * U * np.abs(want["P"][live])
    e_p = e_p + 2 * U * np.abs(want["P"][live]) + FLOOR
    aP, R = np.abs(want["P"][live]), len(live)
    dx = np.zeros(x.shape)
    dx[live] = s * (e_p @ aW + (n + 20) * U * (aP @ aW) + FLOOR * aW.max() * aP.sum(1)[:, None])
    dW = s * (e_p.T @ ax + (R + 20) * U * (aP.T @ ax) + FLOOR * ax.max(initial=0) * aP.sum(0)[:, None])
    return dict(rows=rows, loss=rows.sum() / max(1, R) + 2 * U * abs(want["loss"]), dx=dx, dW=dW, db=s * (e_p.sum(0) + (R + 12) * U * aP.sum(0)))


def _check_loss(case, bf16):
    rows, pad, n, d, bias, none, wide, dloss = case
    x, W, b, label, dl = _loss_case(case, bf16)
    X = (_in_wide if wide else _dev)(_behind(x, pad), bf16)
    Wd, bd = _dev(W, bf16), None if b is None else _dev(b)
    L = torch.from_numpy(np.concatenate([label, np.zeros(pad, np.int32)])).cuda()
    e, R, c = M.loss_dims(n, d, M.BF16 if bf16 else M.F32), rows + pad, _count(rows, pad)
    loss, per_row = _marked(1, 1)[0], _marked(R, 1)[:, 0]
    ws = M.alloc_bytes(M.softmax_loss_ws_bytes(e, R, True)).fill_(255)
    save = M.alloc_bytes(M.softmax_loss_save_bytes(e, R)).fill_(255)
    M.mtgnn_softmax_loss(X, Wd, bd, L, e, loss, ws, row_loss=per_row, save=save, n_rows=c)
    alone = _marked(1, 1)[0]
    M.mtgnn_softmax_loss(X, Wd, bd, L, e, alone, M.alloc_bytes(M.softmax_loss_ws_bytes(e, R)).fill_(255), n_rows=c)
    assert torch.equal(alone, loss)
    dx, dW, db = _marked(R, d, wide=wide), _marked(n, d), _marked(1, n)[0]
    up = None if dloss is None else _dev(np.array([dloss]))
    ws.fill_(255)
    M.mtgnn_softmax_loss_bwd(X, Wd, bd, L, e, save, dx, dW, db, ws, dloss=up, n_rows=c)
    want = model.softmax_loss(np.nan_to_num(x), W, b, label, dl)
    tol = _loss_tolerances(np.nan_to_num(x), W, b, label, want, dl, bf16)
    _close("loss", loss, np.array([want["loss"]]), tol["loss"])
    _close("rows", per_row[:rows], want["rows"], tol["rows"])
    _kept("rows", per_row, rows)
    _close("dx", dx[:rows], want["dx"], tol["dx"])
    _kept("dx", dx, rows)
    _close("dW", dW, want["dW"], tol["dW"])
    _close("db", db, want["db"], tol["db"])
    # each gradient alone is the same
    for k in range(3):
        part = [_marked(R, d), _marked(n, d), _marked(1, n)[0]]
        M.mtgnn_softmax_loss_bwd(X, Wd, bd, L, e, save, *[t if i == k else None for i, t in enumerate(part)], ws, dloss=up,
                                 n_rows=c)
        got, all_ = (part[k], (dx, dW, db)[k]) if k else (part[0][:rows], dx[:rows])
        assert torch.equal(got, all_)


@BOTH
@pytest.mark.parametrize("case", LOSS, ids=str)
def test_softmax_loss(case, bf16):
    _check_loss(case, bf16)


@BOTH
@pytest.mark.parametrize("case", LOSS_BIG, ids=str)
def test_softmax_loss_many_tiles(case, bf16):
    _check_loss(case, bf16)


@BOTH
def test_softmax_loss_without_labels(bf16):
    x, W = np.full((70, 24), np.nan, np.float32), np.ones((50, 24), np.float32)
    e, L = M.loss_dims(50, 24, M.BF16 if bf16 else M.F32), torch.full((70,), -1, dtype=torch.int32, device="cuda")
    X, Wd, loss, rows = _dev(x, bf16), _dev(W, bf16), _marked(1, 1)[0], _marked(70, 1)[:, 0]
    ws = M.alloc_bytes(M.softmax_loss_ws_bytes(e, 70, True)).fill_(255)
    save = M.alloc_bytes(M.softmax_loss_save_bytes(e, 70)).fill_(255)
    dx, dW, db = _marked(70, 24), _marked(50, 24), _marked(1, 50)[0]
    M.mtgnn_softmax_loss(X, Wd, None, L, e, loss, ws, row_loss=rows, save=save)
    M.mtgnn_softmax_loss_bwd(X, Wd, None, L, e, save, dx, dW, db, ws)
    for t in (loss, rows, dx, dW, db):
        assert (t == 0).all()


@BOTH
def test_softmax_loss_masked_classes(bf16):
    """Classes of bias -inf take no part; a label among them has the loss inf; a row of nothing but such is NaN; so is what a
    NaN of x reaches, and nothing else."""
    rs = np.random.RandomState(3)
    x, W = _vals(rs, bf16, 40, 64), _vals(rs, bf16, 300, 64) / np.float32(8)
    b = np.zeros(300, np.float32)
    b[::3] = -np.inf
    label = (3 * rs.randint(0, 100, 40) + 1).astype(np.int32)
    keep = np.arange(300) % 3 != 0
    want = model.softmax_loss(x, W[keep], None, np.array([2 * (c // 3) + c % 3 - 1 for c in label]), 1.0)
    e = M.loss_dims(300, 64, M.BF16 if bf16 else M.F32)
    ws, save = M.alloc_bytes(M.softmax_loss_ws_bytes(e, 40, True)), M.alloc_bytes(M.softmax_loss_save_bytes(e, 40))
    loss, rows, dx, dW, db = _marked(1, 1)[0], _marked(40, 1)[:, 0], _marked(40, 64), _marked(300, 64), _marked(1, 300)[0]

    def call(x, b, label):
        L = torch.from_numpy(label).cuda()
        M.mtgnn_softmax_loss(_dev(x, bf16), _dev(W, bf16), _dev(b), L, e, loss, ws, row_loss=rows, save=save)
        M.mtgnn_softmax_loss_bwd(_dev(x, bf16), _dev(W, bf16), _dev(b), L, e, save, dx, dW, db, ws)

    call(x, b, label)
    tol = _loss_tolerances(x, W[keep], None, np.array([2 * (c // 3) + c % 3 - 1 for c in label]), want, 1.0, bf16)
    _close("rows", rows, want["rows"], tol["rows"])
    _close("dx", dx, want["dx"], tol["dx"])
    _close("dW", dW[torch.from_numpy(keep).cuda()], want["dW"], tol["dW"])
    assert (dW[::3] == 0).all() and (db[::3] == 0).all()
    before = rows.clone()
    bad = label.copy()
    bad[7] = 0
    call(x, b, bad)
    assert torch.isinf(rows[7]) and rows[7] > 0 and torch.isinf(loss).all() and torch.isfinite(dx).all()
    assert torch.equal(torch.cat([rows[:7], rows[8:]]), torch.cat([before[:7], before[8:]]))
    worse = x.copy()
    worse[9, 3] = np.nan
    call(worse, b, label)
    assert torch.isnan(rows[9]) and torch.isnan(dx[9]).all() and torch.isnan(loss).all()
    assert torch.equal(torch.cat([rows[:9], rows[10:]]), torch.cat([before[:9], before[10:]]))
    assert torch.isfinite(torch.cat([dx[:9], dx[10:]])).all()
    call(x, np.full(300, -np.inf, np.float32), label)
    assert torch.isnan(rows).all()


def test_softmax_loss_far_logits():
    """Logits of hundreds: no overflow, and the label's exponential may vanish beside the others."""
    rs = np.random.RandomState(4)
    x, W = rs.randn(30, 40).astype(np.float32) * 20, rs.randn(200, 40).astype(np.float32) * 2
    label = rs.randint(0, 200, 30).astype(np.int32)
    e, L = M.loss_dims(200, 40), torch.from_numpy(label).cuda()
    loss, rows = _marked(1, 1)[0], _marked(30, 1)[:, 0]
    M.mtgnn_softmax_loss(_dev(x), _dev(W), None, L, e, loss, M.alloc_bytes(M.softmax_loss_ws_bytes(e, 30)), row_loss=rows)
    want = model.softmax_loss(x, W, None, label, 1.0)
    tol = _loss_tolerances(x, W, None, label, want, 1.0, False)
    assert want["rows"].max() > 300
    _close("rows", rows, want["rows"], tol["rows"])
    _close("loss", loss, np.array([want["loss"]]), tol["loss"])


# --------------------------------------------------------------------------- AdamW

SIZES = [(1,), (31,), (32,), (33,), (7, 9), (100, 41), (4096,), (4097,), (3, 5000), (70000,)]
CFG = dict(lr=3e-3, beta1=0.9, beta2=0.98, eps=1e-8, t=3)


def _adamw_tolerance(p, g, m, v, want, cfg, decay):
    lr, b1, b2, eps, t = (cfg[k] for k in ("lr", "beta1", "beta2", "eps", "t"))
    e_m = 4 * U * (np.abs(b1 * m) + np.abs((1 - b1) * g))
    e_v = 4 * U * want[2]
    den = np.sqrt(want[2] / (1 - b2 ** t)) + eps
    step = np.abs(want[1]) / (1 - b1 ** t) / den
    return dict(m=e_m, v=e_v, p=lr * (e_m / (1 - b1 ** t) / den + 16 * U * step) + 4 * U * np.abs(p) * (1 + lr * abs(decay)))


@pytest.mark.parametrize("many", [False, True], ids=["few", "many"])
def test_adamw(many):
    rs = np.random.RandomState(6)
    sizes = SIZES + [(int(k),) for k in rs.randint(0, 300, 90)] if many else SIZES
    made = [(rs.randn(*s).astype(np.float32), (rs.randn(*s) * 0.01).astype(np.float32), (rs.randn(*s) * 0.01).astype(np.float32),
             (rs.rand(*s) * 1e-4).astype(np.float32)) for s in sizes]
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    dev = [[torch.from_numpy(x).cuda() for x in col] for col in zip(*made)]
    shadow = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") if i % 2 else None for i, s in enumerate(sizes)]
    M.mtgnn_adamw_step(M.adamw_tensors(*dev, shadow=shadow, decay=decay), **CFG)
    for i, (p, g, m, v) in enumerate(made):
        want = model.adamw(p, g, m, v, decay=decay[i], **CFG)
        tol = _adamw_tolerance(p, g, m, v, want, CFG, decay[i])
        for k, name in enumerate("p m v".split()):
            _close((i, name), dev[(0, 2, 3)[k]][i], want[k], tol[name])
        assert torch.equal(dev[1][i], torch.from_numpy(g).cuda())
        if shadow[i] is not None:
            assert torch.equal(shadow[i], dev[0][i].bfloat16())


def _state8(rs, size, root):
    v = (rs.rand(size) if root else rs.randn(size)) * 10.0 ** rs.uniform(-6, 0, size)
    if size > 40:
        v[3:9] = 0
        v[32:min(size, 64)] = 0         # a whole block of zeros
    return model.to8(v * v if root else v, root)


def test_adamw_in_8_bits():
    rs = np.random.RandomState(8)
    sizes = [1, 31, 32, 33, 100, 4097, 9000]
    p = [rs.randn(n).astype(np.float32) for n in sizes]
    g = [(rs.randn(n) * 10.0 ** rs.uniform(-6, 0, n)).astype(np.float32) for n in sizes]
    for x in g:
        x[::7] = 0
    m8, v8 = [_state8(rs, n, False) for n in sizes], [_state8(rs, n, True) for n in sizes]
    # what is behind a tensor stays as it is
    place = lambda x: torch.from_numpy(np.concatenate([x, np.full(7, 77, x.dtype)])).cuda()   # noqa: E731
    dev = {k: [place(x) for x in xs] for k, xs in dict(p=p, g=g, m=[a for a, _ in m8], v=[a for a, _ in v8], me=[e for _, e in m8],
                                                       ve=[e for _, e in v8]).items()}
    cut = lambda k, per=1: [t[:-(-n // per)] for t, n in zip(dev[k], sizes)]   # noqa: E731
    shadow = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes]
    T = M.adamw_tensors(cut("p"), cut("g"), cut("m"), cut("v"), shadow=shadow, decay=[0.01] * len(sizes), m_exp=cut("me", 32),
                        v_exp=cut("ve", 32))
    M.mtgnn_adamw_step(T, **CFG)
    for i, n in enumerate(sizes):
        m, v = model.from8(*m8[i]), model.from8(*v8[i], root=True)
        want = model.adamw(p[i], g[i], m, v, decay=0.01, **CFG)
        _close((n, "p"), dev["p"][i][:n], want[0], _adamw_tolerance(p[i], g[i], m, v, want, CFG, 0.01)["p"])
        assert torch.equal(shadow[i], dev["p"][i][:n].bfloat16())
        for k, x, root in (("m", want[1], False), ("v", want[2], True)):
            codes, exps = model.to8(x, root)
            assert np.array_equal(dev[k][i][:n].cpu().numpy() & (0xff if k == "m" else 0x7f), codes), (n, k)
            assert np.array_equal(dev[k + "e"][i][:-(-n // 32)].cpu().numpy(), exps), (n, k)
        for k, t in dev.items():
            assert (t[i][-7:].float() == 77).all(), (n, k)


def test_adamw_8_bit_borders():
    """Ties go to the even code, a root never to zero, exponents to the least that holds the block; infinite and NaN gradients
    leave NaN codes in their own places."""
    n = 64
    cfg = dict(lr=0.0, beta1=0.5, beta2=0.0, eps=1e-8, t=1)
    # m = g / 2 here, v = g^2: sqrt(v) = |g|.  Midpoints of neighbouring codes in the first block, the range's ends in the second.
    g = np.zeros(n, np.float32)
    for i in range(28):
        g[i] = 2 * (model.E4M3[100 + i // 2] + model.E4M3[101 + i // 2]) / 2 * (-1 if i % 2 else 1) if i // 2 < 14 else 0
    g[30] = 2 * 448
    g[32], g[33], g[34], g[35], g[36] = 1.0, 2.0 ** -30, -2.0 ** -30, 0.875 * 2.0 ** 9, 3.0
    z = np.zeros(n, np.uint8)
    dev = lambda x: torch.from_numpy(x.copy()).cuda()   # noqa: E731
    p, m, v, me, ve = dev(np.ones(n, np.float32)), dev(z), dev(z), dev(z[:2]), dev(z[:2])
    M.mtgnn_adamw_step(M.adamw_tensors([p], [dev(g)], [m], [v], m_exp=[me], v_exp=[ve]), **cfg)
    _, wm, wv = model.adamw(np.ones(n), g, np.zeros(n), np.zeros(n), decay=0.0, **cfg)
    for got, exps, x, root in ((m, me, wm, False), (v, ve, wv, True)):
        codes, es = model.to8(x, root)
        assert np.array_equal(got.cpu().numpy(), codes) and np.array_equal(exps.cpu().numpy(), es)
    assert v[33] == 1 and m[33] == 0
    bad = g.copy()
    bad[2], bad[40] = np.nan, np.inf
    m2, v2, me2, ve2 = dev(z), dev(z), dev(z[:2]), dev(z[:2])
    M.mtgnn_adamw_step(M.adamw_tensors([p], [dev(bad)], [m2], [v2], m_exp=[me2], v_exp=[ve2]), **cfg)
    for a, b in ((m, m2), (v, v2)):
        assert (b[[2, 40]] & 0x7f == 0x7f).all()
        ok = [i for i in range(n) if i not in (2, 40)]
        assert torch.equal(a[ok], b[ok])


def test_adamw_8_bit_sums_on_borders():
    """beta1 = 0.9: old codes and gradients whose new m is a border of two codes in decimals.  Which side it falls on is decided by
    the roundings of the formula's operations in 64 bits, which the oracle's are."""
    c = np.asarray(model.E4M3[:127], np.float64)
    border = (c[:-1] + c[1:]) / 2
    old, to = (x.ravel() for x in np.meshgrid(c[1:], np.concatenate([border, -border])))
    g = (10 * to - 9 * old)              # (exact: a few bits each)
    assert np.array_equal(g, g.astype(np.float32))
    rows = np.stack([old, g], 1)[: len(old) // 31 * 31].reshape(-1, 31, 2)
    lead = np.full((len(rows), 1, 2), [448.0, 448.0])      # holds each block's exponent where it is
    rows = np.concatenate([lead, rows], 1).reshape(-1, 2) * 2.0 ** -20
    old, g = rows[:, 0], rows[:, 1].astype(np.float32)
    codes, exps = model.to8(old, False)
    assert np.array_equal(model.from8(codes, exps), old)
    dev = lambda x: torch.from_numpy(x.copy()).cuda()   # noqa: E731
    p, m, me = dev(np.zeros(len(g), np.float32)), dev(codes), dev(exps)
    v, ve = dev(np.zeros(len(g), np.uint8)), dev(np.zeros(len(exps), np.uint8))
    M.mtgnn_adamw_step(M.adamw_tensors([p], [dev(g)], [m], [v], m_exp=[me], v_exp=[ve]), 1e-3, 0.9, 0.999, 1e-8, 1)
    _, wm, wv = model.adamw(np.zeros(len(g)), g, old, np.zeros(len(g)), 1e-3, 0.9, 0.999, 1e-8, 1, 0.0)
    for got, e, x, root in ((m, me, wm, False), (v, ve, wv, True)):
        want, we = model.to8(x, root)
        assert np.array_equal(e.cpu().numpy(), we)
        assert np.array_equal(got.cpu().numpy(), want)


def test_adamw_refuses_a_tensor_listed_twice():
    x = [torch.ones(8, device="cuda") for _ in range(7)]
    M.adamw_tensors(x[:2], [x[6]] * 2, x[2:4], x[4:6])      # (a gradient is only read)
    with pytest.raises(M.MtgnnError, match="share memory"):
        M.adamw_tensors([x[0], x[0]], x[6:] * 2, x[2:4], x[4:6])
    with pytest.raises(M.MtgnnError, match="share memory"):
        M.adamw_tensors(x[:2], x[6:] * 2, x[2:4], [x[4], x[3]])
    wide = torch.ones(15, device="cuda")
    with pytest.raises(M.MtgnnError, match="share memory"):
        M.adamw_tensors([wide[:8], wide[7:]], x[6:] * 2, x[2:4], x[4:6])


def test_adamw_step_count_on_the_device():
    rs = np.random.RandomState(9)
    p, g = torch.from_numpy(rs.randn(1000).astype(np.float32)).cuda(), torch.from_numpy(rs.randn(1000).astype(np.float32)).cuda()
    made = [[p.clone()], [g], [torch.zeros_like(p)], [torch.zeros_like(p)]], [[p.clone()], [g], [torch.zeros_like(p)], [torch.zeros_like(p)]]
    step = torch.tensor([41], dtype=torch.int32, device="cuda")
    M.mtgnn_adamw_step(M.adamw_tensors(*made[0]), 1e-2, 0.9, 0.999, 1e-8, 0, step=step)
    M.mtgnn_adamw_step(M.adamw_tensors(*made[1]), 1e-2, 0.9, 0.999, 1e-8, 41)
    assert torch.allclose(made[0][0][0], made[1][0][0], rtol=4 * U, atol=1e-9)
    assert torch.equal(made[0][2][0], made[1][2][0])


# --------------------------------------------------------------------------- together

class Model:
    """ids -> embedding -> norm -> linear with silu and residual -> norm -> loss over all n, as a program keeps it."""

    def __init__(self, rows, n, d, seed=0):
        rs = np.random.RandomState(seed)
        self.rows, self.n, self.d = rows, n, d
        self.ids, self.label = rs.randint(0, n, rows).astype(np.int32), rs.randint(-1, n, rows).astype(np.int32)
        self.ids[3] = -1
        host = dict(table=rs.randn(n, d) * 0.3, g1=1 + 0.1 * rs.randn(d), b1=0.1 * rs.randn(d), W=rs.randn(d, d) / np.sqrt(d),
                    b=0.1 * rs.randn(d), g2=1 + 0.1 * rs.randn(d), b2=0.1 * rs.randn(d), out=rs.randn(n, d) / np.sqrt(d),
                    bias=0.1 * rs.randn(n))
        self.host = {k: v.astype(np.float32) for k, v in host.items()}
        self.p = {k: _dev(v) for k, v in self.host.items()}
        z = lambda *s: torch.zeros(*s, device="cuda")   # noqa: E731
        self.g = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.ids_d, self.label_d = torch.from_numpy(self.ids).cuda(), torch.from_numpy(self.label).cuda()
        self.e, self.nd, self.ld = M.embedding_dims(n, d, scale=2.0), M.norm_dims(d), M.linear_dims(d, d, act=M.ACT_SILU)
        self.od = M.loss_dims(n, d)
        r = rows
        self.x0, self.h1, self.x1, self.h2, self.pre = (z(r, d) for _ in range(5))
        self.s1, self.s2, self.loss, self.row_loss = z(r, 2), z(r, 2), z(1), z(r)
        self.da, self.db, self.dc = z(r, d), z(r, d), z(r, d)
        need = max(M.embedding_ws_bytes(self.e, r), M.layer_norm_ws_bytes(self.nd, r), M.linear_ws_bytes(self.ld, r, True),
                   M.softmax_loss_ws_bytes(self.od, r, True))
        self.ws, self.save = M.alloc_bytes(need), M.alloc_bytes(M.softmax_loss_save_bytes(self.od, r))
        names = list(self.p)
        self.m, self.v = ({k: torch.zeros_like(self.p[k]) for k in names} for _ in range(2))
        self.tensors = M.adamw_tensors(*([x[k] for k in names] for x in (self.p, self.g, self.m, self.v)),
                                       decay=[0.01 if self.p[k].dim() > 1 else 0.0 for k in names])
        self.step = torch.zeros(1, dtype=torch.int32, device="cuda")

    def gradients(self):
        p, g, ws = self.p, self.g, self.ws
        M.mtgnn_embedding(self.ids_d, p["table"], self.e, self.x0)
        M.mtgnn_layer_norm(self.x0, p["g1"], p["b1"], self.nd, self.h1, stats=self.s1)
        M.mtgnn_linear(self.h1, p["W"], p["b"], self.x0, self.ld, self.x1, pre=self.pre, ws=ws)
        M.mtgnn_layer_norm(self.x1, p["g2"], p["b2"], self.nd, self.h2, stats=self.s2)
        M.mtgnn_softmax_loss(self.h2, p["out"], p["bias"], self.label_d, self.od, self.loss, ws, row_loss=self.row_loss, save=self.save)
        M.mtgnn_softmax_loss_bwd(self.h2, p["out"], p["bias"], self.label_d, self.od, self.save, self.da, g["out"], g["bias"], ws)
        M.mtgnn_layer_norm_bwd(self.da, self.x1, p["g2"], self.s2, self.nd, self.db, g["g2"], g["b2"], ws=ws)
        M.mtgnn_linear_bwd(self.db, self.pre, self.h1, p["W"], self.ld, self.dc, g["W"], g["b"], ws=ws)
        # x0 reaches the loss through the norm and through the residual
        M.mtgnn_layer_norm_bwd(self.dc, self.x0, p["g1"], self.s1, self.nd, self.da, g["g1"], g["b1"], past=self.db, ws=ws)
        M.mtgnn_embedding_bwd(self.ids_d, self.da, self.e, g["table"], ws)

    def train(self):
        self.gradients()
        self.step.add_(1)
        M.mtgnn_adamw_step(self.tensors, 1e-2, 0.9, 0.99, 1e-8, 0, step=self.step)

    def reference(self):
        """Loss and gradients in 64 bits by torch's differentiation on the CPU."""
        p = {k: torch.from_numpy(v).double().requires_grad_() for k, v in self.host.items()}
        ids = torch.from_numpy(self.ids).long()
        x0 = 2.0 * p["table"][ids.clamp(min=0)] * (ids >= 0)[:, None]
        norm = lambda x, g, b: (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, correction=0, keepdim=True) + float(np.float32(1e-5))) * g + b   # noqa: E731
        x1 = torch.nn.functional.silu(norm(x0, p["g1"], p["b1"]) @ p["W"].T + p["b"]) + x0
        logits = norm(x1, p["g2"], p["b2"]) @ p["out"].T + p["bias"]
        loss = torch.nn.functional.cross_entropy(logits, torch.from_numpy(self.label).long(), ignore_index=-1)
        loss.backward()
        return loss.item(), {k: v.grad.numpy() for k, v in p.items()}


@pytest.mark.parametrize("rows,n,d", [(50, 70, 24), (300, 411, 64)])
def test_a_model_of_them(rows, n, d):
    """The gradients of the whole against 64 bits.  Each of seven stages adds a relative error of its sums, at most max(d, n, rows) u
    of terms that are up to about 8 times the sum in norm (they cancel like random ones): 56 max(d, n, rows) u of the norm."""
    m = Model(rows, n, d)
    m.gradients()
    loss, want = m.reference()
    rel = 56 * max(rows, n, d) * U
    assert abs(float(m.loss) - loss) <= rel * loss
    for k, g in want.items():
        off = np.linalg.norm(_np(m.g[k]) - g) / np.linalg.norm(g)
        assert off <= rel, (k, off, rel)
    assert (m.g["table"][[i for i in range(n) if i not in m.ids]] == 0).all()


def test_training_steps_in_a_graph():
    """A captured step, replayed between eager work and synchronizations, is the eager step bit for bit, its step count too."""
    a, b = Model(200, 300, 40), Model(200, 300, 40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.gradients()             # (warms up; changes no parameter)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.train()
    losses = []
    for k in range(4):
        a.train()
        graph.replay()
        torch.cuda.synchronize()
        torch.randn(1000, device="cuda").sum()
        assert torch.equal(a.loss, b.loss), k
        for name in a.p:
            assert torch.equal(a.g[name], b.g[name]) and torch.equal(a.p[name], b.p[name]), (k, name)
        losses.append(float(a.loss))
    assert int(a.step) == int(b.step) == 4 and len(set(losses)) == 4


@BOTH
@pytest.mark.parametrize("rows,n,d", [(60, 700, 36), (200, 90, 130), (300, 40, 65)])
def test_captured_losses_follow_the_count(rows, n, d, bf16):
    """One capture of the loss and its gradients, replayed for other counts of rows (none, too), is the eager call's bits each time."""
    rs = np.random.RandomState(rows)
    x, W, b = _dev(_vals(rs, bf16, rows, d), bf16), _dev(_vals(rs, bf16, n, d), bf16), _dev(_vals(rs, False, n))
    L = torch.from_numpy(rs.randint(-1, n, rows).astype(np.int32)).cuda()
    e, c = M.loss_dims(n, d, M.BF16 if bf16 else M.F32), torch.tensor([rows], dtype=torch.int32, device="cuda")
    ws, save = M.alloc_bytes(M.softmax_loss_ws_bytes(e, rows, True)), M.alloc_bytes(M.softmax_loss_save_bytes(e, rows))
    out = [_marked(1, 1)[0], _marked(1, rows)[0], _marked(rows, d), _marked(n, d), _marked(1, n)[0]]
    marked = [t.clone() for t in out]

    def both():
        M.mtgnn_softmax_loss(x, W, b, L, e, out[0], ws, row_loss=out[1], save=save, n_rows=c)
        M.mtgnn_softmax_loss_bwd(x, W, b, L, e, save, out[2], out[3], out[4], ws, n_rows=c)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for count in (rows, 1, 0, 33, rows - 1, 0, rows):
        got = []
        for run in (graph.replay, both):
            c.fill_(count)
            for t, m in zip(out, marked):
                t.copy_(m)
            ws.fill_(255)
            save.fill_(255)
            run()
            torch.cuda.synchronize()
            got.append([t.clone() for t in out])
        for k, (a, w) in enumerate(zip(*got)):
            assert torch.equal(a.view(torch.int32), w.view(torch.int32)), (count, k)
        assert torch.equal(got[0][1][count:], marked[1][count:]) and torch.equal(got[0][2][count:], marked[2][count:])
        if count == 0:
            assert float(got[0][0]) == 0 and not got[0][3].any() and not got[0][4].any()


def test_two_streams_at_once():
    """Two models on two streams, each with a workspace of its own, give what one after the other gives."""
    want, got = [Model(257, 500, 33, s) for s in (1, 2)], [Model(257, 500, 33, s) for s in (1, 2)]
    for m in want:
        m.gradients()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in got]
    for _ in range(3):
        for m, s in zip(got, streams):
            with torch.cuda.stream(s):
                m.gradients()
    torch.cuda.synchronize()
    for x, y in zip(want, got):
        assert torch.equal(x.loss, y.loss)
        for k in x.g:
            assert torch.equal(x.g[k], y.g[k]), k


# --------------------------------------------------------------------------- far offsets and limits

def test_rows_past_32_bits():
    """Elements behind the 2^31st of a table, a gradient, a norm's rows and an optimizer's tensor."""
    n, d = 2_200_000, 1024
    table = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    table[-1], table[0] = 3.0, 1.0
    ids = torch.tensor([n - 1, 0, n - 1], dtype=torch.int32, device="cuda")
    e, y = M.embedding_dims(n, d, M.BF16), torch.empty(3, d, dtype=torch.bfloat16, device="cuda")
    M.mtgnn_embedding(ids, table, e, y)
    assert (y[0] == 3).all() and (y[1] == 1).all()
    del table
    dtable = torch.full((n, d), MARK, device="cuda")
    dy = torch.ones(3, d, device="cuda")
    M.mtgnn_embedding_bwd(ids, dy, e, dtable, M.alloc_bytes(M.embedding_ws_bytes(e, 3)))
    assert (dtable[-1] == 2).all() and (dtable[0] == 1).all() and (dtable[1:-1] == 0).all()
    m, v = torch.zeros_like(dtable), torch.zeros_like(dtable)
    p = torch.ones_like(dtable)
    M.mtgnn_adamw_step(M.adamw_tensors([p], [dtable], [m], [v]), 0.5, 0.5, 0.5, 0.0, 1)
    assert (m[-1] == 1).all() and (v[-1] == 2).all() and (p[-1] == 0.5).all() and torch.isnan(p[-2]).all()   # (0 / 0: eps is 0)
    del dtable, m, v, p
    wide = torch.zeros(2100, 1 << 20, device="cuda")   # rows 2^20 elements apart
    x, y = wide[:, :64], wide[:, 64:128]
    x.copy_(torch.arange(64, device="cuda"))
    M.mtgnn_layer_norm(x, None, None, M.norm_dims(64), y)
    assert torch.equal(y[0], y[-1]) and y[-1].std() > 0.9


def test_embedding_of_the_most_ids():
    n = 1 << 26
    ids = torch.tensor([n - 1, 5, n - 1, n, 8192], dtype=torch.int32, device="cuda")
    e, dtable = M.embedding_dims(n, 1, scale=2.0), torch.full((n, 1), MARK, device="cuda")
    M.mtgnn_embedding_bwd(ids, torch.ones(5, 1, device="cuda"), e, dtable, M.alloc_bytes(M.embedding_ws_bytes(e, 5)))
    assert dtable[n - 1] == 4 and dtable[5] == 2 and dtable[8192] == 2 and int((dtable != 0).sum()) == 3


def _check_loss_large(rows, n, d, bf16, scale):
    """Against torch's float64 products on the GPU, with the tolerances of _loss_tolerances."""
    rs = np.random.RandomState(rows + n)
    x, W, b = _vals(rs, bf16, rows, d), _vals(rs, bf16, n, d) * np.float32(scale), _vals(rs, False, n)
    label = rs.randint(0, n, rows).astype(np.int32)
    label[rs.rand(rows) < 0.02] = -1
    e, L = M.loss_dims(n, d, M.BF16 if bf16 else M.F32), torch.from_numpy(label).cuda()
    X, Wd, bd = _dev(x, bf16), _dev(W, bf16), _dev(b)
    ws, save = M.alloc_bytes(M.softmax_loss_ws_bytes(e, rows, True)).fill_(255), M.alloc_bytes(M.softmax_loss_save_bytes(e, rows)).fill_(255)
    loss, per_row, dx, dW, db = _marked(1, 1)[0], _marked(rows, 1)[:, 0], _marked(rows, d), _marked(n, d), _marked(1, n)[0]
    M.mtgnn_softmax_loss(X, Wd, bd, L, e, loss, ws, row_loss=per_row, save=save)
    M.mtgnn_softmax_loss_bwd(X, Wd, bd, L, e, save, dx, dW, db, ws)
    live = torch.nonzero(L >= 0)[:, 0]
    at, R = L[live].long(), int(live.numel())
    xd, Wq = X.double()[live], Wd.double()
    ax, aW = xd.abs(), Wq.abs()
    floor = 2.0 ** -39
    logits = xd @ Wq.t().contiguous() + bd.double()
    e_l = (d + (4 if bf16 else 12)) * U * (ax @ aW.t().contiguous() + bd.double().abs())
    if not bf16:
        e_l += floor * (ax.max() * aW.sum(1) + aW.max() * ax.sum(1)[:, None])
    lse = torch.logsumexp(logits, 1)
    rows_want = lse - logits[torch.arange(R, device="cuda"), at]
    worst, chain = e_l.max(1).values, (64 + n / 2048) * U
    tol = 2 * worst + chain + 4 * U * (logits.abs().max(1).values + 1)
    assert bool(((per_row[live].double() - rows_want).abs() <= tol + U * rows_want).all())
    assert abs(float(loss) - float(rows_want.mean())) <= float(tol.mean()) + 4 * U * float(rows_want.mean())
    P = torch.exp(logits - lse[:, None])
    e_p = P * (torch.exp(2 * worst)[:, None] * (2 * worst[:, None] + chain + (8 + 4 * (logits.max(1, keepdim=True).values - logits)) * U))
    del logits, e_l
    P[torch.arange(R, device="cuda"), at] -= 1
    aP = P.abs()
    e_p += 4 * U * aP + floor
    t = lambda m: m.t().contiguous()   # noqa: E731
    full = torch.zeros(rows, d, dtype=torch.float64, device="cuda")
    full[live] = P @ Wq
    room = torch.zeros_like(full)
    room[live] = e_p @ aW + (n + 20) * U * (aP @ aW) + floor * aW.max() * aP.sum(1)[:, None]
    for name, got, want, tol in (("dx", dx, full, room),
                                 ("dW", dW, t(P) @ xd, t(e_p) @ ax + (R + 20) * U * (t(aP) @ ax) + floor * ax.max() * aP.sum(0)[:, None]),
                                 ("db", db, P.sum(0), e_p.sum(0) + (R + 12) * U * aP.sum(0))):
        off = (got.double() - want / R).abs()
        assert bool((off <= tol / R + 4 * U * want.abs() / R).all()), (name, float((off / tol * R).max()))


@BOTH
def test_softmax_loss_in_pieces(bf16):
    """More rows and classes than one piece of P holds: 66,000 rows of 3,840 classes at a time, the last piece not a whole one."""
    e = M.loss_dims(4_500, 8, M.BF16 if bf16 else M.F32)
    assert M.softmax_loss_ws_bytes(e, 66_000, True) < 4 * 66_000 * 4_600   # (P of all classes would take more)
    _check_loss_large(66_000, 4_500, 8, bf16, 0.5)


@BOTH
@pytest.mark.parametrize("rows,n,d", [(2100, 16500, 1000), (2304, 16384, 1024)])
def test_softmax_loss_large_tiles(rows, n, d, bf16):
    """The gradients' products in tiles of 256, their sums shared by blocks; ragged and whole."""
    _check_loss_large(rows, n, d, bf16, 2 / np.sqrt(d))
