"""The operators of a model over all nodes at addresses and sizes between the ordinary ones, against the 64-bit oracle, with the
tolerances of tests/test_gpu_model.py: tensors that start at any element of a packed buffer, many wide rows of the layer
norm, tiles of the embedding's ordering with several rounds."""

import numpy as np
import pytest
import torch

from oracle import model
from paper_2608_16305_amd import mtgnn as M
from tests._gpu import needs_gpu
from tests.test_gpu_model import (BOTH, CFG, U, _adamw_tolerance, _check_loss, _close, _dev, _loss_tolerances, _marked, _norm_tolerances,
                                  _vals)
from tests.test_gpu_model import test_embedding as _embedding_case
from tests.test_gpu_model import test_layer_norm as _norm_case

pytestmark = [pytest.mark.gpu, needs_gpu]


def _packed(v, bf16=False, at=1):
    """The tensor from element `at` of a buffer on (NaN around it)."""
    flat = torch.full((at + v.size + 5,), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    flat[at:at + v.size] = _dev(v, bf16).view(-1)
    out = flat[at:at + v.size].view(v.shape)
    assert out.data_ptr() % 16 == at * (2 if bf16 else 4) % 16
    return out


@BOTH
@pytest.mark.parametrize("at", [1, 2, 3, 6])
@pytest.mark.parametrize("rows,n,d", [(70, 300, 64), (33, 1000, 72), (300, 260, 65), (1030, 129, 8), (5, 70, 520)])
def test_softmax_loss_of_a_packed_w(rows, n, d, at, bf16):
    rs = np.random.RandomState(rows + n)
    x, W, b = _vals(rs, bf16, rows, d), _vals(rs, bf16, n, d) / np.float32(4), _vals(rs, False, n)
    label = rs.randint(0, n, rows).astype(np.int32)
    label[::7] = -1
    e, L = M.loss_dims(n, d, M.BF16 if bf16 else M.F32), torch.from_numpy(label).cuda()
    X, Wd, bd = _packed(x, bf16, at), _packed(W, bf16, at), _packed(b, at=at)
    loss, per_row, dx = _marked(1, 1)[0], _marked(rows, 1)[:, 0], _marked(rows, d)
    dW, db = _packed(np.zeros((n, d), np.float32), at=at), _packed(np.zeros(n, np.float32), at=at)
    save = M.alloc_bytes(M.softmax_loss_save_bytes(e, rows)).fill_(255)
    M.mtgnn_softmax_loss(X, Wd, bd, L, e, loss, M.alloc_bytes(M.softmax_loss_ws_bytes(e, rows)).fill_(255), row_loss=per_row, save=save)
    M.mtgnn_softmax_loss_bwd(X, Wd, bd, L, e, save, dx, dW, db, M.alloc_bytes(M.softmax_loss_ws_bytes(e, rows, True)).fill_(255))
    want = model.softmax_loss(x, W, b, label, 1.0)
    tol = _loss_tolerances(x, W, b, label, want, 1.0, bf16)
    _close("loss", loss, np.array([want["loss"]]), tol["loss"])
    for name, got in (("rows", per_row), ("dx", dx), ("dW", dW), ("db", db)):
        _close(name, got, want[name], tol[name])
    for t in (dW, db):      # what lies around a result stays
        around = torch.as_strided(t, (at + t.numel() + 5,), (1,), t.storage_offset() - at)
        assert torch.isnan(around[:at]).all() and torch.isnan(around[-5:]).all()


def test_adamw_refuses_a_gradient_in_what_is_written():
    p, g, m, v, sh = (torch.ones(24, device="cuda") for _ in range(5))
    sh = sh.bfloat16()
    lists = lambda g, **k: M.adamw_tensors([p[:8], p[8:16]], g, [m[:8], m[8:16]], [v[:8], v[8:16]], **k)   # noqa: E731
    lists([g[:8], g[4:12]])                              # gradients are only read
    lists([p[16:], v[16:]])                              # beside a parameter, not in it
    lists([g[:8], m[16:]], shadow=[sh[:8], None])
    for bad in (p[:8], p[15:23], p[8:16], m[7:15], v[:8], v[15:23]):
        with pytest.raises(M.MtgnnError, match="gradient shares memory"):
            lists([g[:8], bad])
        with pytest.raises(M.MtgnnError, match="gradient shares memory"):
            lists([bad, g[:8]])
    in_shadow = sh.view(torch.float32)[:8]
    with pytest.raises(M.MtgnnError, match="gradient shares memory"):
        lists([g[:8], in_shadow], shadow=[None, sh[8:16]])
    empty = torch.empty(0, device="cuda")
    M.adamw_tensors([empty, p[:8]], [empty, g[:8]], [empty, m[:8]], [empty, v[:8]])


# float32: three groups of 64 rows that share W, more blocks than the card has at once; and one row more, by parts
@BOTH
@pytest.mark.parametrize("case", [(150, 42, 17_003, 40, True, 0.1, True, None), (192, 0, 20_000, 33, False, 0.0, False, 2.0),
                                  (193, 0, 20_000, 33, True, 0.0, False, None), (3, 189, 17_000, 64, True, 0.0, False, None)], ids=str)
def test_softmax_loss_of_three_groups_of_rows(case, bf16):
    _check_loss(case, bf16)


# 2,048 rows and more of these widths have a wave each forward, of 16 or 32 elements a lane
@BOTH
@pytest.mark.parametrize("case", [(2100, 20, 777, True, True, True), (2050, 0, 1500, True, False, False), (2048, 0, 2048, True, True, False),
                                  (2049, 3, 513, False, True, False), (2048, 0, 1025, True, True, True)], ids=str)
def test_layer_norm_of_many_wide_rows(case, bf16):
    _norm_case(case, bf16)


# 65,537 rows and more: a tile of the ordering has two rounds of 1,024; n <= 8,192: one pass, else two
@BOTH
@pytest.mark.parametrize("case", [(65_537, 0, 9, 2, 1.0, 9, 0.1, False), (70_001, 30, 8192, 3, 0.5, 8000, 0.0, True),
                                  (140_000, 7, 8193, 1, 1.0, 3, 0.05, False), (131_073, 0, 70_000, 5, -1.0, 70_000, 0.01, False)], ids=str)
def test_embedding_of_many_rows(case, bf16):
    _embedding_case(case, bf16)


@BOTH
@pytest.mark.parametrize("at", [1, 3])
def test_packed_embedding(at, bf16):
    rows, n, d = 700, 300, 37
    rs = np.random.RandomState(1)
    table, dy, ids = _vals(rs, bf16, n, d), _vals(rs, False, rows, d), rs.randint(-1, n, rows).astype(np.int32)
    e, I = M.embedding_dims(n, d, M.BF16 if bf16 else M.F32, 0.5), torch.from_numpy(ids).cuda()
    y, dtable = _packed(np.zeros((rows, d)), bf16, at), _packed(np.zeros((n, d)), at=at)
    M.mtgnn_embedding(I, _packed(table, bf16, at), e, y)
    M.mtgnn_embedding_bwd(I, _packed(dy, at=at), e, dtable, M.alloc_bytes(M.embedding_ws_bytes(e, rows)).fill_(255))
    want, mag = model.embedding(ids, table, 0.5, dy), model.embedding(ids, table, 0.5, np.abs(dy))
    _close("y", y, want["y"], 0, bf16)
    count = np.bincount(ids[ids >= 0], minlength=n)[:, None]
    _close("dtable", dtable, want["dtable"], (count + 1) * U * mag["dtable"])


@BOTH
@pytest.mark.parametrize("at", [1, 3])
@pytest.mark.parametrize("rows,d", [(9, 256), (33, 445), (5, 2050), (3, 9001), (2, 33001)])
def test_packed_layer_norm(rows, d, at, bf16):
    rs = np.random.RandomState(d)
    x, gamma, beta, dy, past = _vals(rs, bf16, rows, d), *(_vals(rs, False, *s) for s in ((d,), (d,), (rows, d), (rows, d)))
    e, X, G = M.norm_dims(d, M.BF16 if bf16 else M.F32, 1e-5), _packed(x, bf16, at), _packed(gamma, at=at)
    y, stats, dx = _packed(np.zeros((rows, d)), bf16, at), _marked(rows, 2), _packed(np.zeros((rows, d)), at=at)
    dgamma, dbeta = _packed(np.zeros(d), at=at), _packed(np.zeros(d), at=at)
    M.mtgnn_layer_norm(X, G, _packed(beta, at=at), e, y, stats=stats)
    M.mtgnn_layer_norm_bwd(_packed(dy, at=at), X, G, stats, e, dx, dgamma, dbeta, past=_packed(past, at=at),
                           ws=M.alloc_bytes(M.layer_norm_ws_bytes(e, rows)).fill_(255))
    want = model.layer_norm(x, gamma, beta, np.float32(1e-5), dy, past)
    tol = _norm_tolerances(x, gamma, dy, past, want)
    _close("y", y, want["y"], tol["y"], bf16)
    for name, got in (("dx", dx), ("dgamma", dgamma), ("dbeta", dbeta)):
        _close(name, got, want[name], tol[name])


@pytest.mark.parametrize("at", [1, 2, 3])
def test_packed_adamw(at):
    rs = np.random.RandomState(at)
    sizes = [1, 5, 127, 2048, 4099]
    made = [(rs.randn(n).astype(np.float32), (rs.randn(n) * 0.01).astype(np.float32), (rs.randn(n) * 0.01).astype(np.float32),
             (rs.rand(n) * 1e-4).astype(np.float32)) for n in sizes]
    dev = [[_packed(v, at=at) for v in col] for col in zip(*made)]
    shadow = [_packed(np.zeros(n), True, at) for n in sizes]
    M.mtgnn_adamw_step(M.adamw_tensors(*dev, shadow=shadow, decay=[0.1] * len(sizes)), **CFG)
    for i, (p, g, m, v) in enumerate(made):
        want = model.adamw(p, g, m, v, decay=0.1, **CFG)
        tol = _adamw_tolerance(p, g, m, v, want, CFG, 0.1)
        for k, name in enumerate("p m v".split()):
            _close((i, name), dev[(0, 2, 3)[k]][i], want[k], tol[name])
        assert torch.equal(shadow[i], dev[0][i].bfloat16())
