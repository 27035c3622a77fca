"""The state-space layer's operators without a GPU: the 64-bit oracle's gradients against differences, and the
C entry points' refusals (none of these calls reaches a launch)."""

import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import layer
from paper_2608_16305_amd import mtgnn as M

built = pytest.mark.skipif(not os.path.exists(M.LIB_PATH), reason="libmtgnn.so not built")


def _slope(f, v, direction, h=1e-6):
    return (f(v + h * direction) - f(v - h * direction)) / (2 * h)


def _check_gradients(call, inputs, names, seed=0):
    """Each gradient in a random direction against the difference of sum(dy y)."""
    rs = np.random.RandomState(seed)
    y0 = call(**inputs)["y"]
    dy = rs.randn(*y0.shape)
    grads = call(dy=dy, **inputs)
    for name, grad in names.items():
        v = np.asarray(inputs[name], np.float64)
        dirn = rs.randn(*v.shape)
        num = _slope(lambda a, name=name: (call(**dict(inputs, **{name: a}))["y"] * dy).sum(), v, dirn)
        ana = (grads[grad] * dirn).sum()
        # central differences: h^2 times the third derivative, and rounding of the sums over 2h
        assert abs(num - ana) <= 1e-6 * (1 + abs(ana)), (name, num, ana)


@pytest.mark.parametrize("name", ["none", "silu", "gelu"])
def test_linear_gradients(name):
    rs = np.random.RandomState(1)
    i = dict(x=rs.randn(7, 5), W=rs.randn(4, 5), b=rs.randn(4), residual=rs.randn(7, 4))
    _check_gradients(lambda dy=None, **k: layer.linear(name=name, dy=dy, **k), i, dict(x="dx", W="dW", b="db"))


@pytest.mark.parametrize("name,width", [("none", 2), ("silu", 3), ("silu", 4)])
def test_conv_gradients(name, width):
    rs = np.random.RandomState(2)
    lens = [3, 0, 1, 6, 2]
    i = dict(x=rs.randn(12, 3), w=rs.randn(width, 3), b=rs.randn(3), first=rs.randn(5, width - 1, 3))
    _check_gradients(lambda dy=None, **k: layer.conv(lens, name=name, dy=dy, **k), i, dict(x="dx", w="dw", b="db"))


@pytest.mark.parametrize("softplus,groups", [(True, 1), (False, 2)])
def test_scan_gradients(softplus, groups):
    rs = np.random.RandomState(3)
    lens = [4, 1, 0, 5]
    i = dict(x=rs.randn(10, 4), delta=rs.rand(10, 4), A=-rs.rand(3, 4) * 2, B=rs.randn(10, 3 * groups),
             C=rs.randn(10, 3 * groups), D=rs.randn(4), z=rs.randn(10, 4), bias=0.1 * rs.rand(4))
    first = rs.randn(4, 3, 4)
    _check_gradients(lambda dy=None, **k: layer.scan(lens, softplus=softplus, groups=groups, first=first, dy=dy, **k), i,
                     dict(x="dx", delta="ddelta", A="dA", B="dB", C="dC", D="dD", z="dz", bias="ddelta_bias"))


def test_a_sequence_is_its_pieces():
    """A sequence cut in two, the second piece from the first one's state, gives the whole one's rows."""
    rs = np.random.RandomState(4)
    x, delta, A, B, C_ = rs.randn(9, 2), rs.randn(9, 2), -rs.rand(3, 2), rs.randn(9, 3), rs.randn(9, 3)
    whole = layer.scan([9], x, delta, A, B, C_)
    one = layer.scan([4], x[:4], delta[:4], A, B[:4], C_[:4])
    two = layer.scan([5], x[4:], delta[4:], A, B[4:], C_[4:], first=one["state"])
    assert np.allclose(np.concatenate([one["y"], two["y"]]), whole["y"], rtol=1e-13, atol=1e-13)
    w = rs.randn(4, 2)
    whole = layer.conv([9], x, w, None, "silu")
    one = layer.conv([2], x[:2], w, None, "silu")
    two = layer.conv([7], x[2:], w, None, "silu", first=one["state"])
    assert np.allclose(np.concatenate([one["y"], two["y"]]), whole["y"], rtol=1e-13, atol=1e-13)


P = C.c_void_p(256)
BIG = 1 << 40


def _q(max_rows=10, max_seq=3, n_slots=4, off=P):
    return C.byref(M.Seqs(max_rows, max_seq, n_slots, off, None, None))


@built
def test_linear_refusals():
    L = M.lib()

    def fwd(d=(8, 4, 0, 2), rows=10, x=P, ldx=8, W=P, res=None, ldr=0, y=P, ldy=4, ws=P, wb=BIG):
        dims = C.byref(M.LinearDims(*d)) if d else None
        return L.mtgnn_linear(x, ldx, None, rows, W, None, res, ldr, dims, y, ldy, None, ws, wb, None)

    assert fwd(d=None) == -1 and fwd(d=(0, 4, 0, 2)) == -1 and fwd(d=(8, -1, 0, 2)) == -1
    assert fwd(d=(8, 4, 5, 2)) == -2 and fwd(d=(8, 4, 0, 4)) == -2 and fwd(d=(8, 4, 0, -1)) == -2
    assert fwd(rows=-1) == -1 and fwd(rows=(1 << 31) - 1) == -1
    assert fwd(x=None) == -1 and fwd(W=None) == -1 and fwd(y=None) == -1
    assert fwd(ldx=7) == -1 and fwd(ldy=3) == -1 and fwd(res=P, ldr=3) == -1
    assert fwd(rows=0) == 0
    need = L.mtgnn_linear_ws_bytes(C.byref(M.LinearDims(8, 4, 0, 2)), 10, 0)
    assert need == 0 or fwd(wb=need - 1) == -3
    assert L.mtgnn_linear_ws_bytes(C.byref(M.LinearDims(8, 4, 0, 9)), 10, 0) == 0

    def bwd(d=(8, 4, 0, 2), rows=10, dy=P, lddy=4, pre=P, x=P, ldx=8, W=P, dx=P, lddx=8, dW=P, ws=P, wb=BIG):
        return L.mtgnn_linear_bwd(dy, lddy, pre, x, ldx, None, rows, W, C.byref(M.LinearDims(*d)), dx, lddx, dW, None,
                                  ws, wb, None)

    assert bwd(rows=0) == -1 and bwd(dy=None) == -1 and bwd(pre=None) == -1 and bwd(dW=None) == -1
    assert bwd(lddy=3) == -1 and bwd(ldx=2) == -1 and bwd(lddx=7) == -1 and bwd(x=None) == -1 and bwd(W=None) == -1
    need = L.mtgnn_linear_ws_bytes(C.byref(M.LinearDims(8, 4, 0, 2)), 10, 1)
    assert need > 0 and bwd(wb=need - 1) == -3 and bwd(ws=None) == -1


@built
def test_conv_refusals():
    L = M.lib()

    def fwd(d=(8, 4, 0, 2), q=None, x=P, ldx=8, w=P, y=P, ldy=8):
        return L.mtgnn_causal_conv(q or _q(), x, ldx, w, None, C.byref(M.ConvDims(*d)), None, None, y, ldy, None, None)

    assert fwd(d=(0, 4, 0, 2)) == -1 and fwd(d=(8, 1, 0, 2)) == -2 and fwd(d=(8, 5, 0, 2)) == -2
    assert fwd(d=(8, 4, 2, 2)) == -2 and fwd(d=(8, 4, 0, 1)) == -2
    assert fwd(q=_q(off=None)) == -1 and fwd(q=_q(max_rows=-1)) == -1 and fwd(q=_q(max_seq=-1)) == -1
    assert fwd(q=_q(n_slots=-1)) == -1
    assert fwd(x=None) == -1 and fwd(w=None) == -1 and fwd(y=None) == -1 and fwd(ldx=7) == -1 and fwd(ldy=7) == -1
    assert fwd(q=_q(max_rows=0)) == 0 and fwd(q=_q(max_seq=0, off=None)) == 0
    assert L.mtgnn_causal_conv(None, P, 8, P, None, C.byref(M.ConvDims(8, 4, 0, 2)), None, None, P, 8, None, None) == -1

    def bwd(q=None, dy=P, lddy=8, x=P, ldx=8, w=P, dx=P, lddx=8, dw=P, ws=P, wb=BIG):
        return L.mtgnn_causal_conv_bwd(q or _q(), dy, lddy, x, ldx, w, None, C.byref(M.ConvDims(8, 4, 0, 2)), None, dx,
                                       lddx, dw, None, ws, wb, None)

    assert bwd(q=_q(max_rows=0)) == -1 and bwd(dy=None) == -1 and bwd(dx=None) == -1 and bwd(dw=None) == -1
    assert bwd(lddy=7) == -1 and bwd(lddx=7) == -1 and bwd(ws=None) == -1 and bwd(wb=16) == -3

    def step(rows=10, n_slots=4, x=P, y=P, ldx=8):
        return L.mtgnn_causal_conv_step(None, None, rows, n_slots, x, ldx, P, None, C.byref(M.ConvDims(8, 4, 0, 2)),
                                        None, None, y, 8, None)

    assert step(rows=-1) == -1 and step(n_slots=-1) == -1 and step(x=None) == -1 and step(y=None) == -1
    assert step(ldx=7) == -1 and step(rows=0) == 0


def _inp(**kw):
    v = dict(x=P, delta=P, B=P, C=P, z=None, ldx=8, lddelta=8, ldB=4, ldC=4, ldz=0, A=P, D=None, delta_bias=None)
    v.update(kw)
    return C.byref(M.ScanInputs(*[v[f] for f, _ in M.ScanInputs._fields_]))


@built
def test_scan_refusals():
    L = M.lib()

    def fwd(d=(8, 4, 1, 0, 1), q=None, inp=None, y=P, ldy=8, ws=P, wb=BIG):
        return L.mtgnn_selective_scan(q or _q(), inp or _inp(), C.byref(M.ScanDims(*d)), None, None, y, ldy, None, ws,
                                      wb, None)

    assert fwd(d=(0, 4, 1, 0, 1)) == -1 and fwd(d=(8, 0, 1, 0, 1)) == -1 and fwd(d=(8, 4, 3, 0, 1)) == -1
    assert fwd(d=(8, 65, 1, 0, 1)) == -2 and fwd(d=(8, 4, 1, 3, 1)) == -2
    for name in ("x", "delta", "B", "C", "A"):
        assert fwd(inp=_inp(**{name: None})) == -1
    for name in ("ldx", "lddelta"):
        assert fwd(inp=_inp(**{name: 7})) == -1
    for name in ("ldB", "ldC"):
        assert fwd(inp=_inp(**{name: 3})) == -1
    assert fwd(inp=_inp(z=P, ldz=7)) == -1 and fwd(y=None) == -1 and fwd(ldy=7) == -1
    assert fwd(ws=None) == -1 and fwd(wb=16) == -3 and fwd(q=_q(off=None)) == -1
    assert fwd(q=_q(max_rows=0)) == 0 and fwd(q=_q(max_seq=0, off=None)) == 0

    def bwd(d=(8, 4, 1, 0, 1), q=None, inp=None, dy=P, lddy=8, save=P, ws=P, wb=BIG, **kw):
        v = dict(dx=P, ddelta=P, dB=P, dC=P, dz=None, lddx=8, ldddelta=8, lddB=4, lddC=4, lddz=8, dA=P, dD=None,
                 ddelta_bias=None)
        v.update(kw)
        g = M.ScanGrads(*[v[f] for f, _ in M.ScanGrads._fields_])
        return L.mtgnn_selective_scan_bwd(q or _q(), dy, lddy, inp or _inp(), C.byref(M.ScanDims(*d)), save, C.byref(g),
                                          ws, wb, None)

    for name in ("dx", "ddelta", "dB", "dC", "dA"):
        assert bwd(**{name: None}) == -1
    for name in ("lddx", "ldddelta"):
        assert bwd(**{name: 7}) == -1
    for name in ("lddB", "lddC"):
        assert bwd(**{name: 3}) == -1
    assert bwd(dz=P) == -1 and bwd(dD=P) == -1 and bwd(ddelta_bias=P) == -1
    assert bwd(inp=_inp(z=P, ldz=8)) == -1 and bwd(inp=_inp(z=P, ldz=8), dz=P, lddz=7) == -1
    assert bwd(dy=None) == -1 and bwd(save=None) == -1 and bwd(lddy=7) == -1
    assert bwd(ws=None) == -1 and bwd(wb=16) == -3 and bwd(q=_q(max_rows=0)) == -1

    def step(rows=10, n_slots=4, inp=None, y=P):
        return L.mtgnn_selective_scan_step(None, None, rows, n_slots, inp or _inp(), C.byref(M.ScanDims(8, 4, 1, 0, 1)),
                                           None, None, y, 8, None)

    assert step(rows=-1) == -1 and step(n_slots=-1) == -1 and step(y=None) == -1 and step(inp=_inp(A=None)) == -1
    assert step(rows=0) == 0


@built
def test_sizes():
    d = M.scan_dims(100, 16)
    assert 0 < M.selective_scan_ws_bytes(d, 100, 5) <= M.selective_scan_ws_bytes(d, 100, 5, True)
    a, b = M.selective_scan_save_bytes(d, 100, 5, False), M.selective_scan_save_bytes(d, 100, 5, True)
    assert a >= 100 // 8 * 16 * 100 * 4 and b - a >= 5 * 16 * 100 * 4
    assert M.selective_scan_ws_bytes(M.scan_dims(100, 16, 3), 100, 5) == 0
    c = M.conv_dims(100, 4, M.BF16)
    assert M.causal_conv_save_bytes(c, 7) == 7 * 3 * 100 * 2 and M.causal_conv_ws_bytes(c, 100) > 0


@built
def test_binding_refuses_host_tensors():
    with pytest.raises(M.MtgnnError):
        M.mtgnn_linear(torch.zeros(3, 4), torch.zeros(5, 4), None, None, M.linear_dims(4, 5), torch.zeros(3, 5))
    with pytest.raises(M.MtgnnError):
        M.seqs(torch.zeros(3, dtype=torch.int32), 4)


@built
def test_sizes_without_rows():
    for act in (M.ACT_NONE, M.ACT_SILU):
        d = M.linear_dims(64, 64, act=act)
        assert M.linear_ws_bytes(d, 0) == 0 and M.linear_ws_bytes(d, 0, True) >= 0
    assert M.causal_conv_ws_bytes(M.conv_dims(8, 4), 0) >= 0 and M.causal_conv_save_bytes(M.conv_dims(8, 4), 0) == 0
    s = M.scan_dims(8, 4)
    assert M.selective_scan_ws_bytes(s, 0, 0, True) >= 0 and M.selective_scan_save_bytes(s, 0, 0, True) >= 0


@built
def test_launches_of_too_many_threads_are_refused():
    """Refused with EUNSUPPORTED before anything is launched; the sizes just below are not tried."""
    L = M.lib()
    many = 1 << 29   # rows of eight channels
    conv, scan, lin = C.byref(M.ConvDims(8, 4, 0, 2)), C.byref(M.ScanDims(8, 4, 1, 0, 1)), C.byref(M.LinearDims(8, 1, 0, 0))
    assert L.mtgnn_causal_conv_step(None, None, many, 4, P, 8, P, None, conv, P, P, P, 8, None) == -2
    assert L.mtgnn_causal_conv(_q(max_seq=many), P, 8, P, None, conv, P, P, P, 8, None, None) == -2
    assert L.mtgnn_causal_conv(_q(max_seq=many), P, 8, P, None, conv, P, None, P, 8, P, None) == -2
    assert L.mtgnn_selective_scan_step(None, None, many, 4, _inp(), scan, P, P, P, 8, None) == -2
    g = M.ScanGrads(P, P, P, P, None, 8, 8, 4, 4, 0, P, None, None)
    assert L.mtgnn_selective_scan_bwd(_q(max_rows=many), P, 8, _inp(), scan, P, C.byref(g), P, 1 << 62, None) == -2
    assert L.mtgnn_linear_bwd(P, 1, None, P, 8, None, many, P, lin, P, 8, P, P, P, 1 << 62, None) == -2


@built
def test_workspaces_that_are_not_aligned_are_refused():
    L, off = M.lib(), C.c_void_p(260)
    lin, conv, scan = M.LinearDims(8, 4, 0, 2), M.ConvDims(8, 4, 0, 2), M.ScanDims(8, 4, 1, 0, 1)
    few = M.LinearDims(1024, 4, 0, 2)   # a sum in shares: the forward has a workspace
    assert L.mtgnn_linear_ws_bytes(C.byref(few), 10, 0) > 0
    assert L.mtgnn_linear(P, 1024, None, 10, P, None, None, 0, C.byref(few), P, 4, None, off, BIG, None) == -1
    assert L.mtgnn_linear_bwd(P, 4, P, P, 8, None, 10, P, C.byref(lin), P, 8, P, None, off, BIG, None) == -1
    assert L.mtgnn_causal_conv_bwd(_q(), P, 8, P, 8, P, None, C.byref(conv), None, P, 8, P, None, off, BIG, None) == -1
    g = M.ScanGrads(P, P, P, P, None, 8, 8, 4, 4, 0, P, None, None)
    for ws, save in ((off, P), (P, off)):
        assert L.mtgnn_selective_scan(_q(), _inp(), C.byref(scan), None, None, P, 8, save, ws, BIG, None) == -1
        assert L.mtgnn_selective_scan_bwd(_q(), P, 8, _inp(), C.byref(scan), save, C.byref(g), ws, BIG, None) == -1


@built
def test_inputs_of_other_dims_are_refused():
    d, q = M.scan_dims(8, 4), M.Seqs(10, 3, 4, P, None, None)
    inp, g = M.ScanInputs(), M.ScanGrads()
    for other in ((16, 4, 1, M.F32), (8, 5, 1, M.F32), (8, 4, 2, M.F32), (8, 4, 1, M.BF16)):
        inp.rows, inp.dims = 10, other
        g.rows, g.dims = 10, other
        for call in (lambda: M.mtgnn_selective_scan(q, inp, d, None, None, None),
                     lambda: M.mtgnn_selective_scan_step(None, inp, d, None, None, None),
                     lambda: M.mtgnn_selective_scan_bwd(q, None, inp, d, None, g, None)):
            with pytest.raises(M.MtgnnError, match="made for"):
                call()
        inp.dims = (8, 4, 1, M.F32)
        with pytest.raises(M.MtgnnError, match="gradients were made for"):
            M.mtgnn_selective_scan_bwd(q, None, inp, d, None, g, None)


@built
def test_gradients_over_what_is_still_read_are_refused():
    """dx over operands that other blocks, or the product after it, read: refused, by the bytes that rows share."""
    L = M.lib()
    at = lambda b: C.c_void_p(1 << 20 | b)   # noqa: E731
    far = C.c_void_p(1 << 30)

    def conv(dy, x, dx, ld=8, dtype=M.F32, ws=far):
        d = M.ConvDims(8, 4, dtype, 2)
        return L.mtgnn_causal_conv_bwd(_q(), dy, ld, x, ld, P, None, C.byref(d), None, dx, ld, P, None, ws,
                                       BIG, None)

    for dx in (0, 4, 32, 9 * 32 + 28, -28):            # the same rows, shifted by an element, by a row, the last and first element
        assert conv(at(4096), far, at(4096 + dx)) == -1 and b"overlaps dy" in L.mtgnn_last_error()
        assert conv(far, at(4096), at(4096 + dx)) == -1 and b"overlaps x" in L.mtgnn_last_error()
    assert conv(far, at(4096), at(4096 + 9 * 16 + 12), dtype=M.BF16) == -1    # the strides differ: the last row's second half
    assert conv(at(4096), far, at(4096 + 28), ld=16) == -1 and conv(at(4096), far, at(4096 + 36), ld=16) == -1

    def lin(dy, x, dx, act=0, d_in=8, d_out=8, ldd=8, ldx=8):
        d = M.LinearDims(d_in, d_out, M.F32, act)
        return L.mtgnn_linear_bwd(dy, ldd, far, x, ldx, None, 10, P, C.byref(d), dx, ldx, P, None, far, BIG, None)

    assert lin(at(4096), far, at(4096)) == -1 and b"overlaps dy" in L.mtgnn_last_error()
    assert lin(far, at(4096), at(4096)) == -1 and b"overlaps x" in L.mtgnn_last_error()
    assert lin(at(4096), at(4096), at(4096), act=2) == -1 and b"overlaps x" in L.mtgnn_last_error()
    assert lin(at(4096), far, at(4096 + 300), d_out=9, ldd=9) == -1


def test_descriptors_keep_their_tensors(monkeypatch):
    """seqs, scan_inputs and scan_grads hold addresses: the tensors live as long as they do."""
    import gc
    import weakref
    monkeypatch.setattr(M, "_ptr", lambda t, *a, **k: None if t is None else C.c_void_p(t.data_ptr()))
    monkeypatch.setattr(M, "_rows", lambda t, *a, **k: (None, 8) if t is None else (C.c_void_p(t.data_ptr()), 8))
    alive = []

    def new(*shape, dtype=torch.float32):
        t = torch.zeros(*shape, dtype=dtype)
        alive.append(weakref.ref(t))
        return t

    i32 = torch.int32
    q = M.seqs(new(4, dtype=i32), 10, n_seq=new(1, dtype=i32), slot=new(3, dtype=i32), n_slots=2)
    d = M.scan_dims(8, 4)
    inp = M.scan_inputs(d, new(10, 8), new(10, 8), new(4, 8), new(10, 4), new(10, 4), D=new(8), z=new(10, 8),
                        delta_bias=new(8))
    g = M.scan_grads(d, new(10, 8), new(10, 8), new(4, 8), new(10, 4), new(10, 4), dD=new(8), dz=new(10, 8),
                     ddelta_bias=new(8))
    gc.collect()
    assert len(alive) == 19 and all(r() is not None for r in alive)
    del q, inp, g
    gc.collect()
    assert all(r() is None for r in alive)


def test_tensors_of_another_device_are_refused(monkeypatch):
    """Every kind of operand, as if the current device were another one."""
    class Elsewhere:
        is_cuda, device, shape, dtype = True, torch.device("cuda", 1), (4, 8), torch.float32
        numel, dim, get_device, stride = (lambda s: 32), (lambda s: 2), (lambda s: 1), (lambda s, i: (8, 1)[i])

    monkeypatch.setattr(M, "_ptr", lambda t, *a, **k: C.c_void_p(256))
    monkeypatch.setattr(torch, "Tensor", Elsewhere)
    monkeypatch.setattr(M, "_device", lambda: 0)
    t = Elsewhere()
    for call in (lambda: M._rows(t, torch.float32, "m", 4, 8, dev=0), lambda: M._work(t, 0), lambda: M.seqs(t, 4),
                 lambda: M._table(t, torch.float32, "m", (4, 8), dev=0), lambda: M._count(t, 3, "m", dev=0),
                 lambda: M._bytes(t, 16, "m", dev=0)):
        with pytest.raises(M.MtgnnError, match="current device is 0"):
            call()
    # what holds addresses was made there, and is used here
    monkeypatch.setattr(M, "_device", lambda: 1)
    q, d, c = M.seqs(t, 4), M.scan_dims(8, 4), M.conv_dims(8, 4)
    inp, g = M.ScanInputs(), M.ScanGrads()
    inp.rows = g.rows = 4
    inp.dims = g.dims = (8, 4, 1, M.F32)
    inp.device = g.device = 1
    monkeypatch.setattr(M, "_device", lambda: 0)
    for call in (lambda: M.mtgnn_causal_conv(q, None, None, None, c, None, None, None),
                 lambda: M.mtgnn_causal_conv_bwd(q, None, None, None, None, c, None, None, None, None, None),
                 lambda: M.mtgnn_selective_scan(q, inp, d, None, None, None),
                 lambda: M.mtgnn_selective_scan_step(None, inp, d, None, None, None),
                 lambda: M.mtgnn_selective_scan_bwd(q, None, inp, d, None, g, None)):
        with pytest.raises(M.MtgnnError, match="current device is 0"):
            call()


def test_a_lost_part_shows_in_a_single_product():
    """What the GPU tests hold single products to (3 u): six products of bfloat16 parts keep to it, three where one operand
    is bfloat16 itself, and none of those can be left out."""
    from itertools import product

    from oracle.bf16 import round_bf16
    rs = np.random.RandomState(5)
    a, b = (((1 + rs.rand(20000)) * rs.choice([-1, 1], 20000)).astype(np.float32) for _ in range(2))

    def parts(v):
        out, left = [], v.astype(np.float32)
        for _ in range(3):
            out.append(round_bf16(left))
            left = (left - out[-1]).astype(np.float32)
        return out

    def off(terms, w):
        s = np.zeros_like(a)
        for i, j in sorted(terms, key=lambda t: -sum(t)):   # the smallest first, each sum rounded to float32
            s = (s + parts(a)[i].astype(np.float64) * parts(w)[j].astype(np.float64)).astype(np.float32)
        exact = a.astype(np.float64) * w.astype(np.float64)
        return float((np.abs(s - exact) / np.abs(exact)).max()) * 2.0 ** 24

    six = [(i, j) for i, j in product(range(3), range(3)) if i + j < 3]
    assert off(six, b) < 3
    for t in six:
        assert off([s for s in six if s != t], b) > 30, t
    three = [(0, 0), (1, 0), (2, 0)]
    assert off(three, round_bf16(b)) < 3
    for t in three:
        assert off([s for s in three if s != t], round_bf16(b)) > 30, t
