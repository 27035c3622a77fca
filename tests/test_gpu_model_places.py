"""The operators of a model over all nodes at addresses and sizes between the ordinary ones, against the 64-bit oracle, with the
tolerances of tests/test_gpu_model.py: tensors that start at any element of a packed buffer."""

import numpy as np
import pytest
import torch

from oracle import model
from paper_2608_16305_amd import mtgnn as M
from tests._gpu import needs_gpu
from tests.test_gpu_model import BOTH, _close, _dev, _loss_tolerances, _marked, _vals

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
