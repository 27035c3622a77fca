"""The softmax loss over numbers of unlike sizes, on the GPU through the C ABI, against the 64-bit oracle: one far element of W or x,
classes whose probability is far below the others'.  What a float32 evaluation holds, the kernels hold: every tolerance is
relative to the terms that enter an element, none to a matrix's largest.

With u = 2^-24, half a step of float32:
  logits     a sum of d products, (d + 4) u of their magnitudes; a float32 factor in three bfloat16 parts is held to u, and the
             products of parts that are left out, second by third and third by third, are below 2^-8 2^-16 2 = 2 u: 8 u more;
  P          of the exponentials' share p: its own logit's error and the row's sum's (the logits' errors in the mean that p is the
             weight of), a chain of at most 64 + n / 2,048 sums, 8 u for the operations and 4 u of the logit's distance from
             the largest; of P = p - [label] the subtraction's and the parts' 2 u;
  gradients  sums of n (dx) or of rows (dW) products, so many u of their magnitudes and 20 for the parts, shares and scale."""

import numpy as np
import pytest
import torch

from oracle import model
from paper_2608_16305_amd import mtgnn as M
from tests._gpu import needs_gpu
from tests.test_gpu_model import BOTH, U, _close, _dev, _marked, _vals

pytestmark = [pytest.mark.gpu, needs_gpu]

FAR = np.float32(2.0 ** 30)
SIZES = pytest.mark.parametrize("rows,n,d", [(300, 200, 72), (300, 130, 65), (100, 257, 64), (40, 500, 129)])


def _tolerances(x, W, b, label, want, bf16):
    n, d = W.shape
    ax, aW, at = np.abs(x).astype(np.float64), np.abs(W).astype(np.float64), np.arange(len(x))
    logits = x.astype(np.float64) @ W.astype(np.float64).T + b
    e_l = (d + (4 if bf16 else 12)) * U * (ax @ aW.T + np.abs(b))
    p = want["P"] + (np.arange(n) == label[:, None])
    mean, chain = (p * e_l).sum(1, keepdims=True), (64 + n / 2048) * U
    gap = logits.max(1, keepdims=True) - logits
    aP, R = np.abs(want["P"]), len(x)
    e_p = p * np.expm1(np.minimum(e_l + mean + chain + (8 + 4 * gap) * U, 50)) + 4 * U * aP
    return dict(rows=mean[:, 0] + e_l[at, label] + chain + 4 * U * (np.abs(logits).max(1) + 1),
                dx=(e_p @ aW + (n + 20) * U * (aP @ aW)) / R, dW=(e_p.T @ ax + (R + 20) * U * (aP.T @ ax)) / R,
                db=(e_p.sum(0) + (R + 12) * U * aP.sum(0)) / R)


def _check(x, W, b, label, bf16):
    (rows, d), n = x.shape, len(W)
    e, L = M.loss_dims(n, d, M.BF16 if bf16 else M.F32), torch.from_numpy(label).cuda()
    X, Wd, bd = _dev(x, bf16), _dev(W, bf16), _dev(b)
    ws, save = M.alloc_bytes(M.softmax_loss_ws_bytes(e, rows, True)).fill_(255), M.alloc_bytes(M.softmax_loss_save_bytes(e, rows)).fill_(255)
    loss, per_row, dx, dW, db = _marked(1, 1)[0], _marked(rows, 1)[:, 0], _marked(rows, d), _marked(n, d), _marked(1, n)[0]
    M.mtgnn_softmax_loss(X, Wd, bd, L, e, loss, ws, row_loss=per_row, save=save)
    M.mtgnn_softmax_loss_bwd(X, Wd, bd, L, e, save, dx, dW, db, ws)
    want = model.softmax_loss(x, W, b, label, 1.0)
    tol = _tolerances(x, W, b, label, want, bf16)
    for name, got in (("rows", per_row), ("dx", dx), ("dW", dW), ("db", db)):
        _close(name, got, want[name], tol[name])
    return want


def _inputs(rows, n, d, bf16):
    rs = np.random.RandomState(rows + n + d)
    x, W = _vals(rs, bf16, rows, d), _vals(rs, bf16, n, d) / np.float32(8)
    return x, W, _vals(rs, False, n), rs.randint(0, n, rows).astype(np.int32)


@BOTH
@SIZES
def test_a_far_element_of_w_leaves_the_others_as_they_are(rows, n, d, bf16):
    """x is zero where it would meet that element: no logit has it, and of dx the one column."""
    x, W, b, label = _inputs(rows, n, d, bf16)
    x[:, 2], W[3, 2] = 0, FAR
    _check(x, W, b, label, bf16)


@BOTH
@SIZES
def test_a_far_row_of_x_leaves_the_others_as_they_are(rows, n, d, bf16):
    """That row's label is certain: P is zero in it, and no gradient of a class has it."""
    x, W, b, label = _inputs(rows, n, d, bf16)
    W[:, 2] = 0
    x[5], x[5, 2], W[label[5], 2] = 0, FAR, 1
    want = _check(x, W, b, label, bf16)
    assert (want["P"][5] == 0).all()


@BOTH
@SIZES
def test_rare_classes_have_their_gradient(rows, n, d, bf16):
    """Classes some e^-60 times as likely as the others: their rows of dW are held as well as the others'."""
    x, W, b, label = _inputs(rows, n, d, bf16)
    b[::3] -= 60
    label = label % (n // 3) * 3 + 1 + label % 2
    want = _check(x, W, b, label.astype(np.int32), bf16)
    assert 0 < np.abs(want["dW"][::3]).max() < 1e-20


@BOTH
@SIZES
@pytest.mark.parametrize("power", [-80, 60])
def test_operands_of_unlike_sizes(rows, n, d, power, bf16):
    """Rows of x larger or smaller by a power of two than W's are smaller or larger: the logits are ordinary ones."""
    x, W, b, label = _inputs(rows, n, d, bf16)
    _check(np.ldexp(x, power), np.ldexp(W, -power), b, label, bf16)


@BOTH
@pytest.mark.parametrize("rows", [10, 70, 200, 1100])
@pytest.mark.parametrize("at", [5, 500])
def test_a_nan_beside_an_infinite_logit_is_nan(rows, at, bf16):
    """log sum exp of an infinite logit is infinite, of one and a NaN, in the same tile or in another, NaN; a row without a label is 0."""
    rs = np.random.RandomState(rows)
    n, d = 600, 24
    x, W, b = _vals(rs, bf16, rows, d), _vals(rs, bf16, n, d), _vals(rs, False, n)
    label = rs.randint(4, n, rows).astype(np.int32)
    label[0], label[1] = -1, 3
    e, L = M.loss_dims(n, d, M.BF16 if bf16 else M.F32), torch.from_numpy(label).cuda()
    loss, per_row, dx = _marked(1, 1)[0], _marked(rows, 1)[:, 0], _marked(rows, d)
    ws, save = M.alloc_bytes(M.softmax_loss_ws_bytes(e, rows, True)), M.alloc_bytes(M.softmax_loss_save_bytes(e, rows))
    for nan in (False, True):
        b[3] = np.inf
        b[at] = np.nan if nan else 0.5
        X, Wd, bd = _dev(x, bf16), _dev(W, bf16), _dev(b)
        M.mtgnn_softmax_loss(X, Wd, bd, L, e, loss, ws, row_loss=per_row, save=save)
        M.mtgnn_softmax_loss_bwd(X, Wd, bd, L, e, save, dx, None, None, ws)
        assert per_row[0] == 0 and torch.isnan(per_row[1]) and torch.isnan(loss).all()
        assert torch.isnan(per_row[2:]).all() if nan else (per_row[2:] == np.inf).all()
        assert torch.isnan(dx[1:]).all() and not dx[0].any()
