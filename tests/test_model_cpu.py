"""The operators of a model over all nodes without a GPU: the 64-bit oracle's gradients against differences, its 8-bit numbers
against their definition, and the C entry points' refusals (none of these calls reaches a launch)."""

import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

from oracle import model
from paper_2608_16305_amd import mtgnn as M

built = pytest.mark.skipif(not os.path.exists(M.LIB_PATH), reason="libmtgnn.so not built")

P = C.c_void_p(256)
BIG = 1 << 40


def _slope(f, v, direction, h=1e-6):
    return (f(v + h * direction) - f(v - h * direction)) / (2 * h)


def _check(f, v, grad, seed=0):
    """grad in a random direction against the difference of f: h^2 times the third derivative, and the sums' rounding over 2h."""
    d = np.random.RandomState(seed).randn(*v.shape)
    num, ana = _slope(f, v, d), (grad * d).sum()
    assert abs(num - ana) <= 1e-6 * (1 + abs(ana)), (num, ana)


def test_embedding_gradient():
    rs = np.random.RandomState(1)
    table, dy = rs.randn(6, 3), rs.randn(9, 3)
    ids = [0, 5, -1, 0, 2, 6, 0, 2, 1]
    got = model.embedding(ids, table, 0.7, dy)
    _check(lambda t: (model.embedding(ids, t, 0.7)["y"] * dy).sum(), table, got["dtable"])
    assert (got["dtable"][[3, 4]] == 0).all() and (got["y"][[2, 5]] == 0).all()


@pytest.mark.parametrize("past", [False, True])
def test_layer_norm_gradients(past):
    rs = np.random.RandomState(2)
    x, gamma, beta, dy = rs.randn(5, 7) + 1, rs.randn(7), rs.randn(7), rs.randn(5, 7)
    extra = rs.randn(5, 7) if past else None
    got = model.layer_norm(x, gamma, beta, 1e-3, dy, extra)
    call = lambda x, g, b: (model.layer_norm(x, g, b, 1e-3)["y"] * dy).sum() + (0 if extra is None else (x * extra).sum())   # noqa: E731
    _check(lambda v: call(v, gamma, beta), x, got["dx"])
    _check(lambda v: call(x, v, beta), gamma, got["dgamma"])
    _check(lambda v: call(x, gamma, v), beta, got["dbeta"])


def test_softmax_loss_gradients():
    rs = np.random.RandomState(3)
    x, W, b = rs.randn(6, 4), rs.randn(9, 4), rs.randn(9)
    label = np.array([0, 8, -1, 3, 9, 3])
    got = model.softmax_loss(x, W, b, label, 1.0)
    _check(lambda v: model.softmax_loss(v, W, b, label)["loss"], x, got["dx"])
    _check(lambda v: model.softmax_loss(x, v, b, label)["loss"], W, got["dW"])
    _check(lambda v: model.softmax_loss(x, W, v, label)["loss"], b, got["db"])
    half = model.softmax_loss(x, W, b, label, 0.5)
    assert np.allclose(half["dW"], got["dW"] / 2, rtol=1e-14) and (got["dx"][[2, 4]] == 0).all()
    assert model.softmax_loss(x, W, b, np.full(6, -1), 1.0)["loss"] == 0


def test_e4m3_numbers():
    assert model.E4M3[0x7e] == 448 and model.E4M3[1] == 2.0 ** -9 and model.E4M3[0x38] == 1 and math.isnan(model.E4M3[0x7f])
    torch_says = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(torch_says, nan=7e7), np.nan_to_num(model.E4M3, nan=7e7))
    rs = np.random.RandomState(4)
    v = np.concatenate([rs.rand(200) * 448, 10.0 ** rs.uniform(-4, 2, 200), model.E4M3[:127], (model.E4M3[:126] + model.E4M3[1:127]) / 2])
    want = torch.from_numpy(v).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()   # (all of them float32 but the first)
    got = np.array([model.nearest_code(float(np.float32(x))) for x in v])
    assert np.array_equal(got, want)


def test_states_in_8_bits_round_trip():
    rs = np.random.RandomState(5)
    m = rs.randn(100) * 10.0 ** rs.uniform(-8, 3, 100)
    codes, exps = model.to8(m)
    back = model.from8(codes, exps)
    unit = 2.0 ** (np.repeat(exps.astype(int), 32)[:100] - 127)
    assert (np.abs(back - m) <= np.maximum(np.abs(m) / 16, unit * 2.0 ** -10) * (1 + 1e-12)).all()
    again = model.to8(back)
    assert np.array_equal(again[0] & 0x7f, codes & 0x7f) and np.array_equal(again[1], exps)
    v = m * m
    codes, exps = model.to8(v, root=True)
    assert ((codes == 0) == (v == 0)).all()
    top = np.array([np.sqrt(v[32 * k:32 * k + 32]).max() for k in range(4)])
    assert (top <= 448 * 2.0 ** (exps.astype(int) - 127)).all() and (top > 224 * 2.0 ** (exps.astype(int) - 127)).all()


def test_adamw_step_by_hand():
    p, m, v = model.adamw([2.0], [0.5], [0.1], [0.04], 0.1, 0.9, 0.99, 0.0, 2, 0.01)
    assert abs(m[0] - 0.14) < 1e-15 and abs(v[0] - 0.0421) < 1e-15
    assert abs(p[0] - (2 * 0.999 - 0.1 * (0.14 / 0.19) / math.sqrt(0.0421 / 0.0199))) < 1e-14


# --------------------------------------------------------------------------- refusals

@built
def test_embedding_refusals():
    L = M.lib()
    good = dict(n=100, d=8, dtype=M.F32, scale=1.0)
    dims = lambda **k: C.byref(M.embedding_dims(*dict(good, **k).values()))   # noqa: E731

    def fwd(ids=P, rows=10, table=C.c_void_p(1 << 30), d=None, y=P, ldy=8, **k):
        return L.mtgnn_embedding(ids, None, rows, table, d or dims(**k), y, ldy, None)

    def bwd(ids=P, rows=10, dy=P, lddy=8, d=None, to=C.c_void_p(1 << 30), ws=P, room=BIG, **k):
        return L.mtgnn_embedding_bwd(ids, None, rows, dy, lddy, d or dims(**k), to, ws, room, None)

    for f in (fwd, bwd):
        assert f(dtype=3) == -2
        for k in (dict(n=0), dict(n=-1), dict(scale=math.inf), dict(scale=math.nan)):
            assert f(**k) in (-1, -2), k
        assert f(ids=None) == -1 and f(rows=-1) == -1 and f(rows=1 << 31) == -1
    assert fwd(rows=0) == 0 and bwd(rows=0) == -1
    assert fwd(table=None) == -1 and fwd(y=None) == -1 and fwd(ldy=7) == -1 and fwd(table=P) == -1
    assert fwd(rows=(1 << 31) - 65, ldy=64, d=C.byref(M.embedding_dims(100, 64, M.F32))) == -2
    assert bwd(dy=None) == -1 and bwd(to=None) == -1 and bwd(lddy=7) == -1 and bwd(to=P) == -1
    assert bwd(room=M.embedding_ws_bytes(M.embedding_dims(100, 8), 10) - 1) == -3
    assert bwd(ws=None) == -1 and bwd(ws=C.c_void_p(264)) == -1
    assert bwd(d=C.byref(M.embedding_dims((1 << 26) + 1, 1))) == -2
    assert M.embedding_ws_bytes(M.embedding_dims(0, 8), 10) == 0 and M.embedding_ws_bytes(M.embedding_dims(5, 8), -1) == 0


@built
def test_layer_norm_refusals():
    L = M.lib()
    d8 = M.norm_dims(8)
    far = C.c_void_p(1 << 30)

    def fwd(x=P, ldx=8, rows=10, d=C.byref(d8), y=far, ldy=8, stats=None):
        return L.mtgnn_layer_norm(x, ldx, None, rows, None, None, d, y, ldy, stats, None)

    def bwd(dy=P, lddy=8, x=far, ldx=8, stats=C.c_void_p(1 << 32), rows=10, past=None, ldp=8, d=C.byref(d8), dx=C.c_void_p(1 << 34), lddx=8,
            dgamma=P, ws=P, n=BIG):
        return L.mtgnn_layer_norm_bwd(dy, lddy, x, ldx, stats, None, rows, None, past, ldp, d, dx, lddx, dgamma, None, ws, n, None)

    for f in (fwd, bwd):
        assert f(d=None) == -1
        for e in (-1e-5, math.nan, math.inf):
            assert f(d=C.byref(M.norm_dims(8, M.F32, e))) == -1
        assert f(d=C.byref(M.norm_dims(0))) == -1 and f(d=C.byref(M.norm_dims(8, 5))) == -2
        assert f(d=C.byref(M.norm_dims((1 << 20) + 1))) == -2
        assert f(rows=-1) == -1 and f(x=None) == -1 and f(ldx=7) == -1
        assert f(rows=1 << 27) == -2          # 64 threads a row
    assert fwd(rows=0) == 0 and bwd(rows=0) == -1
    assert fwd(y=None) == -1 and fwd(ldy=7) == -1
    assert fwd(y=C.c_void_p(256 + 4)) == -1 and fwd(y=P, ldy=9) == -1 and fwd(y=P, stats=far) == -1
    assert bwd(dy=None) == -1 and bwd(stats=None) == -1 and bwd(dx=None) == -1 and bwd(lddx=7) == -1 and bwd(lddy=7) == -1
    assert bwd(past=P, ldp=7) == -1 and bwd(dx=far) == -1 and bwd(dx=P, lddx=9) == -1 and bwd(dx=C.c_void_p(260)) == -1
    assert bwd(past=C.c_void_p(1 << 36), dx=C.c_void_p((1 << 36) + 4)) == -1 and bwd(stats=C.c_void_p((1 << 32) + 4)) == -1
    assert bwd(n=M.layer_norm_ws_bytes(d8, 10) - 1) == -3 and bwd(ws=None) == -1 and bwd(ws=C.c_void_p(264)) == -1
    assert M.layer_norm_ws_bytes(M.norm_dims(0), 10) == 0


@built
def test_layer_norm_stats_are_aligned_in_both_directions():
    """What the backward would refuse, the forward does too."""
    L, d = M.lib(), M.norm_dims(8)
    for at, want in ((4, -1), (12, -1), (1, -1)):
        stats, far = C.c_void_p((1 << 32) + at), C.c_void_p(1 << 30)
        assert L.mtgnn_layer_norm(P, 8, None, 10, None, None, C.byref(d), far, 8, stats, None) == want
        assert L.mtgnn_layer_norm_bwd(P, 8, far, 8, stats, None, 10, None, None, 8, C.byref(d), C.c_void_p(1 << 34), 8, None, None, None, 0,
                                      None) == want


@built
def test_softmax_loss_refusals():
    L = M.lib()
    good = M.loss_dims(100, 8)
    far, farther = C.c_void_p(1 << 30), C.c_void_p(1 << 32)

    def fwd(x=P, ldx=8, rows=10, W=P, label=P, d=C.byref(good), loss=P, save=None, ws=P, n=BIG):
        return L.mtgnn_softmax_loss(x, ldx, None, rows, W, None, label, d, loss, None, save, ws, n, None)

    def bwd(rows=10, W=P, label=P, d=C.byref(good), save=P, dx=far, lddx=8, dW=farther, ws=P, n=BIG):
        return L.mtgnn_softmax_loss_bwd(None, rows, W, None, label, d, save, None, dx, lddx, dW, None, ws, n, None)

    for f in (fwd, bwd):
        assert f(d=None) == -1 and f(d=C.byref(M.loss_dims(0, 8))) == -1 and f(d=C.byref(M.loss_dims(5, 0))) == -1
        assert f(d=C.byref(M.loss_dims(5, 8, 9))) == -2 and f(d=C.byref(M.loss_dims(5, (1 << 20) + 1))) == -2
        assert f(d=C.byref(M.loss_dims((1 << 31) - 64, 8))) == -2
        assert f(rows=0) == -1 and f(rows=-1) == -1 and f(W=None) == -1 and f(label=None) == -1 and f(ws=None) == -1
        assert f(ws=C.c_void_p(264)) == -1 and f(save=C.c_void_p(264)) == -1
        assert f(rows=1 << 30, d=C.byref(M.loss_dims(1 << 30, 8))) == -2
    assert fwd(x=None) == -1 and fwd(loss=None) == -1 and fwd(ldx=7) == -1
    assert fwd(n=M.softmax_loss_ws_bytes(good, 10) - 1) == -3
    assert bwd(save=None) == -1 and bwd(lddx=7) == -1 and bwd(dx=P) == -1 and bwd(dx=farther) == -1 and bwd(dW=P) == -1
    assert bwd(dx=None, dW=None) == 0
    assert M.softmax_loss_ws_bytes(good, 10, True) > 0 and M.softmax_loss_save_bytes(good, 10) > 0
    assert M.softmax_loss_ws_bytes(M.loss_dims(0, 8), 10) == 0 and M.softmax_loss_save_bytes(good, -1) == 0


def test_softmax_loss_memory():
    """Not the logits: a gigabyte of P at most, beside the copies of x and W."""
    if not os.path.exists(M.LIB_PATH):
        pytest.skip("libmtgnn.so not built")
    rows, n, d = 16384, 200_000, 1024
    e = M.loss_dims(n, d, M.BF16)
    copies = 2 * 1.1 * (rows + n) * d
    assert M.softmax_loss_ws_bytes(e, rows, True) < copies + 1.1 * 2 ** 30 + rows * n // 16
    assert M.softmax_loss_ws_bytes(e, rows, True) < rows * n


@built
def test_softmax_loss_has_room_for_a_copy_of_w():
    """Of a bfloat16 W at any address, which the workspace's size does not know, in the forward and the backward."""
    for n, d, rows in ((100_000, 64, 5), (3000, 520, 200), (70, 8, 1)):
        for back in (False, True):
            assert M.softmax_loss_ws_bytes(M.loss_dims(n, d, M.BF16), rows, back) >= 2 * n * d


@built
@pytest.mark.parametrize("rows", [8_000, 16_384, 100_000, 262_144, 349_500])
def test_softmax_loss_takes_a_gigabyte_for_p(rows):
    """The padding of P's rows counts too.  A twentieth more for what else is there: copies of 8 columns, tiles' and columns' sums."""
    for n in (2000, 30_000):
        assert M.softmax_loss_ws_bytes(M.loss_dims(n, 8, M.BF16), rows, True) < 1.05 * 2 ** 30 + rows * n // 16


@built
def test_adamw_refusals():
    L = M.lib()
    t = (M.AdamwTensor * 2)()
    cfg = lambda **k: C.byref(M.AdamConfig(*dict(dict(lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, t=1), **k).values()))   # noqa: E731
    call = lambda n=2, c=None, step=None, tensors=t: L.mtgnn_adamw_step(tensors, n, c or cfg(), step, None)   # noqa: E731
    assert call() == 0 and call(n=0, tensors=None) == 0        # tensors without elements: nothing to do
    assert call(n=-1) == -1 and call(tensors=None) == -1 and L.mtgnn_adamw_step(t, 2, None, None, None) == -1
    for bad in (dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=math.nan), dict(eps=-1.0), dict(eps=math.nan), dict(lr=math.inf),
                dict(t=0)):
        assert call(c=cfg(**bad)) == -1, bad
    assert call(c=cfg(t=0), step=P) == 0
    names = ("param", "grad", "m", "v")
    for missing in names:
        for k in names:
            setattr(t[1], k, None if k == missing else P)
        t[1].n = 4
        assert call() == -1, missing
    for k in names:
        setattr(t[1], k, P)
    t[1].m_exp = P
    assert call() == -1
    t[1].m_exp, t[1].n = None, -1
    assert call() == -1
    t[1].n = (1 << 33) + 1
    assert call() == -2
    t[1].n, t[1].decay = 4, math.nan
    assert call() == -1


@built
def test_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros(4, 8)
    with pytest.raises(M.MtgnnError, match="GPU tensor"):
        M.mtgnn_layer_norm(x, None, None, M.norm_dims(8), x)
    with pytest.raises(M.MtgnnError, match="GPU tensor"):
        M.mtgnn_softmax_loss(x, x, None, torch.zeros(4, dtype=torch.int32), M.loss_dims(4, 8), x[0, :1], None)
    with pytest.raises(M.MtgnnError, match="vector of int32"):
        M.mtgnn_embedding(torch.zeros(2, 2, dtype=torch.int32), x, M.embedding_dims(4, 8), x)
    with pytest.raises(M.MtgnnError, match="2 tensors for 1"):
        M.adamw_tensors([x], [x, x], [x], [x])
    with pytest.raises(M.MtgnnError, match="GPU tensor"):
        M.adamw_tensors([x], [x], [x], [x])
