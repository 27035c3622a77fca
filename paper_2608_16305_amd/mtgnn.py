"""ctypes binding of libmtgnn.so.

Argument marshalling only: every function checks that its tensors live on the
GPU with the expected dtype and layout, passes their device pointers and the
current HIP stream to the C entry point of the same name, and raises
``MtgnnError`` on a non-zero status.  No computation happens here, and there
is no fallback: if the library is missing, the first call raises.
"""

import bisect
import ctypes as C
import os

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmtgnn.so")

F32, BF16 = 0, 1
OP_BUILD_QUERIES, OP_AGGREGATE_LAST, OP_BUILD_MESSAGES, OP_GRU_UPDATE, OP_SAMPLE_RECENT = 0, 1, 2, 3, 4
OP_TEMPORAL_ATTN, OP_TEMPORAL_ATTN_BWD, OP_GRU_UPDATE_BWD, OP_BUILD_MESSAGES_BWD, OP_BUILD_CSR = 5, 6, 7, 8, 9
OP_LINK_LOSS, OP_MIXED_BATCHES, OP_RNN_UPDATE, OP_RNN_UPDATE_BWD, OP_TIME_PROJECTION_BWD = 10, 11, 12, 13, 14

ENTRY_POINTS = (
    "mtgnn_build_queries", "mtgnn_aggregate_last", "mtgnn_build_messages", "mtgnn_gru_update",
    "mtgnn_sample_recent", "mtgnn_temporal_attn", "mtgnn_temporal_attn_prepare", "mtgnn_temporal_attn_prepare_weights",
    "mtgnn_temporal_attn_prepare_weights_link",
    "mtgnn_temporal_attn_prepare_slots", "mtgnn_temporal_attn_prepared",
    "mtgnn_temporal_attn_bwd", "mtgnn_temporal_attn_bwd_overlap", "mtgnn_temporal_attn_bwd_group",
    "mtgnn_temporal_attn_bwd_grouped",
    "mtgnn_gru_update_bwd", "mtgnn_link_loss", "mtgnn_link_loss_overlap", "mtgnn_link_prepare_weights",
    "mtgnn_link_loss_prepared",
    "mtgnn_build_messages_bwd", "mtgnn_build_messages_bwd_noalloc", "mtgnn_build_temporal_csr",
    "mtgnn_dependency_scan", "mtgnn_mixed_batches", "mtgnn_rnn_update", "mtgnn_rnn_update_bwd",
    "mtgnn_time_projection", "mtgnn_time_projection_bwd", "mtgnn_controller_create", "mtgnn_controller_destroy",
    "mtgnn_controller_decide", "mtgnn_controller_observe", "mtgnn_controller_state", "mtgnn_grad_norm_ws_bytes",
    "mtgnn_grad_norm", "mtgnn_prune_aux", "mtgnn_cache_refresh", "mtgnn_adam_step", "mtgnn_workspace_bytes", "mtgnn_save_bytes",
    "mtgnn_linear_ws_bytes", "mtgnn_linear", "mtgnn_linear_bwd", "mtgnn_causal_conv_save_bytes",
    "mtgnn_causal_conv_ws_bytes", "mtgnn_causal_conv", "mtgnn_causal_conv_bwd", "mtgnn_causal_conv_step",
    "mtgnn_selective_scan_ws_bytes", "mtgnn_selective_scan_save_bytes", "mtgnn_selective_scan",
    "mtgnn_selective_scan_bwd", "mtgnn_selective_scan_step",
    "mtgnn_embedding", "mtgnn_embedding_ws_bytes", "mtgnn_embedding_bwd", "mtgnn_layer_norm", "mtgnn_layer_norm_ws_bytes",
    "mtgnn_layer_norm_bwd", "mtgnn_softmax_loss_save_bytes", "mtgnn_softmax_loss_ws_bytes", "mtgnn_softmax_loss",
    "mtgnn_softmax_loss_bwd", "mtgnn_adamw_step",
    "mtgnn_status_string", "mtgnn_last_error", "mtgnn_version", "mtgnn_timer_start", "mtgnn_timer_stop",
)


class MtgnnError(RuntimeError):
    pass


class Dims(C.Structure):
    _fields_ = [("n_nodes", C.c_int64), ("d_mem", C.c_int32), ("d_time", C.c_int32), ("d_edge", C.c_int32),
                ("d_attn", C.c_int32), ("n_heads", C.c_int32), ("k", C.c_int32), ("dtype", C.c_int32)]


class Batch(C.Structure):
    _fields_ = [("n", C.c_int64), ("src", C.c_void_p), ("dst", C.c_void_p), ("eid", C.c_void_p),
                ("t", C.c_void_p), ("flags", C.c_void_p)]


_ATTN = ("W_q", "W_k", "W_v", "W_o", "W_1", "W_2", "b_q", "b_k", "b_v", "b_o", "b_1", "b_2")


class AttnParams(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _ATTN]


class AttnGrads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _ATTN]


_LINK = ("W_d1", "b_d1", "W_d2", "b_d2")


class ControllerConfig(C.Structure):
    _fields_ = [("alpha", C.c_double), ("beta", C.c_double), ("tau_g", C.c_double), ("tau_c", C.c_double),
                ("interval", C.c_int32)]


class AdamConfig(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("t", C.c_int32)]


class LinkParams(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _LINK]


class LinkGrads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _LINK]


ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = 0, 1, 2, 3


class Seqs(C.Structure):
    _fields_ = [("max_rows", C.c_int64), ("max_seq", C.c_int64), ("n_slots", C.c_int64), ("off", C.c_void_p),
                ("n_seq", C.c_void_p), ("slot", C.c_void_p)]


class LinearDims(C.Structure):
    _fields_ = [("d_in", C.c_int32), ("d_out", C.c_int32), ("dtype", C.c_int32), ("act", C.c_int32)]


class ConvDims(C.Structure):
    _fields_ = [("d", C.c_int32), ("width", C.c_int32), ("dtype", C.c_int32), ("act", C.c_int32)]


class ScanDims(C.Structure):
    _fields_ = [("d", C.c_int32), ("n", C.c_int32), ("groups", C.c_int32), ("dtype", C.c_int32),
                ("softplus", C.c_int32)]


class ScanInputs(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("x", "delta", "B", "C", "z")]
                + [(n, C.c_int64) for n in ("ldx", "lddelta", "ldB", "ldC", "ldz")]
                + [(n, C.c_void_p) for n in ("A", "D", "delta_bias")])


class ScanGrads(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("dx", "ddelta", "dB", "dC", "dz")]
                + [(n, C.c_int64) for n in ("lddx", "ldddelta", "lddB", "lddC", "lddz")]
                + [(n, C.c_void_p) for n in ("dA", "dD", "ddelta_bias")])


class EmbeddingDims(C.Structure):
    _fields_ = [("n", C.c_int64), ("d", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float)]


class NormDims(C.Structure):
    _fields_ = [("d", C.c_int32), ("dtype", C.c_int32), ("eps", C.c_float)]


class LossDims(C.Structure):
    _fields_ = [("n", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32)]


class AdamwTensor(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("param", "grad", "m", "v", "m_exp", "v_exp", "shadow")]
                + [("n", C.c_int64), ("decay", C.c_float)])


_P = C.c_void_p
_I64 = C.c_int64
_I32 = C.c_int32
_SZ = C.c_size_t
_SIGS = {
    "mtgnn_build_queries": [C.POINTER(Batch), _P, _P, _P, _P, _P, _SZ, _P],
    "mtgnn_aggregate_last": [C.POINTER(Batch), _I64, _P, _P, _P, _P, _SZ, _P],
    "mtgnn_build_messages": [C.POINTER(Batch), _P, _P, _P, _I64, _P, _P, _P, _P, _P, C.POINTER(Dims), _P, _P, _P],
    "mtgnn_gru_update": [C.POINTER(Batch), _P, _P, _P, _I64, _P, _P, _P, _P, _P, C.POINTER(Dims), _P, _P, _P, _P, _SZ,
                         _P],
    "mtgnn_sample_recent": [_P, _P, _P, _P, _I64, _P, _P, _P, _I64, _I32, _P, _P, _P, _P],
    "mtgnn_temporal_attn": [_P, _P, _P, _I64, _P, _P, _P, _P, _P, _P, _P, C.POINTER(AttnParams), C.POINTER(Dims), _P,
                            _P, _P, _SZ, _P],
    "mtgnn_temporal_attn_prepare": [_P, _P, _I64, C.POINTER(AttnParams), _P, _P, C.POINTER(Dims), _P, _P, _SZ, _P],
    "mtgnn_temporal_attn_prepare_weights": [C.POINTER(AttnParams), _P, _P, C.POINTER(Dims), _P, _P],
    "mtgnn_temporal_attn_prepare_weights_link": [C.POINTER(AttnParams), _P, _P, C.POINTER(Dims), _P,
                                                 C.POINTER(LinkParams), _I64, _P, _SZ, _P],
    "mtgnn_temporal_attn_prepare_slots": [_P, _P, _I64, C.POINTER(Dims), _P, _P, _SZ, _P],
    "mtgnn_temporal_attn_prepared": [_P, _P, _P, _I64, _P, _P, _P, _P, _P, _P, _P, C.POINTER(AttnParams),
                                     C.POINTER(Dims), _P, _P, _P],
    "mtgnn_temporal_attn_bwd": [_P, _P, _P, _I64, _P, _P, _P, _P, _P, _P, _I64, _P, _P, C.POINTER(AttnParams),
                                C.POINTER(Dims), C.POINTER(AttnGrads), _P, _P, _P, _P, _SZ, _P],
    "mtgnn_temporal_attn_bwd_overlap": [_P, _P, _P, _I64, _P, _P, _P, _P, _P, _P, _I64, _P, _P,
                                        C.POINTER(AttnParams), C.POINTER(Dims), C.POINTER(AttnGrads), _P, _P, _P, _P,
                                        _SZ, _P, _P, _P, _P],
    "mtgnn_temporal_attn_bwd_group": [_P, _P, _I64, _P, _P, _P, _P, _I64, C.POINTER(Dims), _P, _SZ, _P],
    "mtgnn_temporal_attn_bwd_grouped": [_P, _P, _P, _I64, _P, _P, _P, _P, _P, _P, _I64, _P, _P,
                                        C.POINTER(AttnParams), C.POINTER(Dims), C.POINTER(AttnGrads), _P, _P, _P, _P,
                                        _SZ, _P, _P, _P, _P],
    "mtgnn_gru_update_bwd": [_P, _P, _P, _P, _I64, _P, _P, C.POINTER(Dims), _P, _P, _P, _P, _P, _P, _SZ, _P],
    "mtgnn_link_loss": [_P, _P, _I64, C.POINTER(LinkParams), C.POINTER(Dims), _P, _P, _P, C.POINTER(LinkGrads), _P,
                        _SZ, _P],
    "mtgnn_link_loss_overlap": [_P, _P, _I64, C.POINTER(LinkParams), C.POINTER(Dims), _P, _P, _P,
                                C.POINTER(LinkGrads), _P, _SZ, _P, _P, _P],
    "mtgnn_link_prepare_weights": [C.POINTER(LinkParams), C.POINTER(Dims), _I64, _P, _SZ, _P],
    "mtgnn_link_loss_prepared": [_P, _P, _I64, C.POINTER(LinkParams), C.POINTER(Dims), _P, _P, _P,
                                 C.POINTER(LinkGrads), _P, _SZ, _P, _P, _P],
    "mtgnn_build_messages_bwd": [_P, _P, _P, _I64, _P, _P, C.POINTER(Dims), _P, _P, _P, _SZ, _P],
    "mtgnn_build_messages_bwd_noalloc": [_P, _P, _P, _I64, _P, _P, C.POINTER(Dims), _P, _P, _P],
    "mtgnn_build_temporal_csr": [_P, _P, _P, _I64, _I64, _P, _P, _P, _P, _P, _SZ, _P],
    "mtgnn_dependency_scan": [_P, _P, _I64, _P, _I64, _I32, _I64, _I32, _P, _P, _P],
    "mtgnn_rnn_update": [C.POINTER(Batch), _P, _P, _P, _I64, _P, _P, _P, _P, _P, C.POINTER(Dims), _P, _P, _P, _P, _SZ,
                         _P],
    "mtgnn_rnn_update_bwd": [_P, _P, _P, _P, _I64, _P, _P, C.POINTER(Dims), _P, _P, _P, _P, _P, _P, _SZ, _P],
    "mtgnn_time_projection": [_P, _P, _P, _I64, _P, _P, _P, _P, C.c_float, C.POINTER(Dims), _P, _P],
    "mtgnn_time_projection_bwd": [_P, _P, _P, _I64, _P, _P, _P, _P, C.c_float, _P, _P, _P, _I64, C.POINTER(Dims),
                                  _P, _P, _P, _P, _SZ, _P],
    "mtgnn_controller_create": [C.POINTER(ControllerConfig), C.POINTER(C.c_void_p)],
    "mtgnn_controller_destroy": [_P],
    "mtgnn_controller_decide": [_P, _I64, C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_int32)],
    "mtgnn_controller_observe": [_P, C.c_double, C.c_double],
    "mtgnn_controller_state": [_P] + [C.POINTER(C.c_double)] * 4,
    "mtgnn_grad_norm_ws_bytes": [C.POINTER(C.c_int64), _I32],
    "mtgnn_grad_norm": [C.POINTER(C.c_void_p), C.POINTER(C.c_int64), _I32, _P, _P, _SZ, _P],
    "mtgnn_prune_aux": [_P, _I64, _I32, _P],
    "mtgnn_cache_refresh": [_P, _I64, _P, _P, C.POINTER(Dims), _P, _P, _P],
    "mtgnn_adam_step": [C.POINTER(C.c_void_p)] * 5 + [C.POINTER(C.c_int64), _I32, C.POINTER(AdamConfig), _P],
    "mtgnn_mixed_batches": [_P, _I64, _I64, _P, _P, _P, _P, _SZ, _P],
    "mtgnn_embedding": [_P, _P, _I64, _P, C.POINTER(EmbeddingDims), _P, _I64, _P],
    "mtgnn_embedding_ws_bytes": [C.POINTER(EmbeddingDims), _I64],
    "mtgnn_embedding_bwd": [_P, _P, _I64, _P, _I64, C.POINTER(EmbeddingDims), _P, _P, _SZ, _P],
    "mtgnn_layer_norm": [_P, _I64, _P, _I64, _P, _P, C.POINTER(NormDims), _P, _I64, _P, _P],
    "mtgnn_layer_norm_ws_bytes": [C.POINTER(NormDims), _I64],
    "mtgnn_layer_norm_bwd": [_P, _I64, _P, _I64, _P, _P, _I64, _P, _P, _I64, C.POINTER(NormDims), _P, _I64, _P, _P, _P, _SZ, _P],
    "mtgnn_softmax_loss_save_bytes": [C.POINTER(LossDims), _I64],
    "mtgnn_softmax_loss_ws_bytes": [C.POINTER(LossDims), _I64, _I32],
    "mtgnn_softmax_loss": [_P, _I64, _P, _I64, _P, _P, _P, C.POINTER(LossDims), _P, _P, _P, _P, _SZ, _P],
    "mtgnn_softmax_loss_bwd": [_P, _I64, _P, _P, _P, C.POINTER(LossDims), _P, _P, _P, _I64, _P, _P, _P, _SZ, _P],
    "mtgnn_adamw_step": [C.POINTER(AdamwTensor), _I64, C.POINTER(AdamConfig), _P, _P],
    "mtgnn_linear_ws_bytes": [C.POINTER(LinearDims), _I64, _I32],
    "mtgnn_linear": [_P, _I64, _P, _I64, _P, _P, _P, _I64, C.POINTER(LinearDims), _P, _I64, _P, _P, _SZ, _P],
    "mtgnn_linear_bwd": [_P, _I64, _P, _P, _I64, _P, _I64, _P, C.POINTER(LinearDims), _P, _I64, _P, _P, _P, _SZ, _P],
    "mtgnn_causal_conv_save_bytes": [C.POINTER(ConvDims), _I64],
    "mtgnn_causal_conv_ws_bytes": [C.POINTER(ConvDims), _I64],
    "mtgnn_causal_conv": [C.POINTER(Seqs), _P, _I64, _P, _P, C.POINTER(ConvDims), _P, _P, _P, _I64, _P, _P],
    "mtgnn_causal_conv_bwd": [C.POINTER(Seqs), _P, _I64, _P, _I64, _P, _P, C.POINTER(ConvDims), _P, _P, _I64, _P, _P,
                              _P, _SZ, _P],
    "mtgnn_causal_conv_step": [_P, _P, _I64, _I64, _P, _I64, _P, _P, C.POINTER(ConvDims), _P, _P, _P, _I64, _P],
    "mtgnn_selective_scan_ws_bytes": [C.POINTER(ScanDims), _I64, _I64, _I32],
    "mtgnn_selective_scan_save_bytes": [C.POINTER(ScanDims), _I64, _I64, _I32],
    "mtgnn_selective_scan": [C.POINTER(Seqs), C.POINTER(ScanInputs), C.POINTER(ScanDims), _P, _P, _P, _I64, _P, _P,
                             _SZ, _P],
    "mtgnn_selective_scan_bwd": [C.POINTER(Seqs), _P, _I64, C.POINTER(ScanInputs), C.POINTER(ScanDims), _P,
                                 C.POINTER(ScanGrads), _P, _SZ, _P],
    "mtgnn_selective_scan_step": [_P, _P, _I64, _I64, C.POINTER(ScanInputs), C.POINTER(ScanDims), _P, _P, _P, _I64,
                                  _P],
    "mtgnn_workspace_bytes": [C.c_int, C.POINTER(Dims), _I64, _I64],
    "mtgnn_save_bytes": [C.c_int, C.POINTER(Dims), _I64, _I64],
    "mtgnn_status_string": [C.c_int],
    "mtgnn_last_error": [],
    "mtgnn_version": [],
    "mtgnn_timer_start": [C.c_char_p, C.c_int],
    "mtgnn_timer_stop": [C.POINTER(C.c_double), C.POINTER(C.c_int)],
}
_RES = {"mtgnn_workspace_bytes": _SZ, "mtgnn_save_bytes": _SZ, "mtgnn_grad_norm_ws_bytes": _SZ,
        "mtgnn_linear_ws_bytes": _SZ, "mtgnn_causal_conv_save_bytes": _SZ, "mtgnn_causal_conv_ws_bytes": _SZ,
        "mtgnn_selective_scan_ws_bytes": _SZ, "mtgnn_selective_scan_save_bytes": _SZ,
        "mtgnn_embedding_ws_bytes": _SZ, "mtgnn_layer_norm_ws_bytes": _SZ, "mtgnn_softmax_loss_save_bytes": _SZ,
        "mtgnn_softmax_loss_ws_bytes": _SZ,
        "mtgnn_controller_destroy": None, "mtgnn_status_string": C.c_char_p,
        "mtgnn_last_error": C.c_char_p, "mtgnn_version": C.c_int}

_lib = None


def lib() -> C.CDLL:
    """Load the in-tree libmtgnn.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MtgnnError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = C.CDLL(LIB_PATH)
        for name, args in _SIGS.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = _RES.get(name, C.c_int)
        _lib = L
    return _lib


def _check(status: int, name: str):
    if status != 0:
        L = lib()
        raise MtgnnError(f"{name}: {L.mtgnn_status_string(status).decode()} "
                         f"({L.mtgnn_last_error().decode()})")


# The current stream's handle without a Stream object around it (2.5 us less a call), where torch offers it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None and _raw_stream is not None:
        return C.c_void_p(_raw_stream(torch.cuda.current_device()))
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


_DT = {F32: torch.float32, BF16: torch.bfloat16}


def _ptr(t, dtype=None, name="tensor", optional=False):
    if t is None:
        if optional:
            return None
        raise MtgnnError(f"{name} is required")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise MtgnnError(f"{name} must be a GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise MtgnnError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise MtgnnError(f"{name} must be contiguous")
    return C.c_void_p(t.data_ptr())


def _ws(ws):
    if ws is None:
        return None, 0
    return _ptr(ws, torch.uint8, "ws"), ws.numel()


def dims(n_nodes, d_mem, d_time, d_edge, d_attn, n_heads, k, dtype=F32) -> Dims:
    return Dims(int(n_nodes), int(d_mem), int(d_time), int(d_edge), int(d_attn), int(n_heads), int(k), int(dtype))


def batch(src, dst, t, eid=None, flags=None) -> Batch:
    n = int(src.numel())
    return Batch(n, _ptr(src, torch.int32, "src"), _ptr(dst, torch.int32, "dst"),
                 _ptr(eid, torch.int32, "eid", optional=True), _ptr(t, torch.float32, "t"),
                 _ptr(flags, torch.uint8, "flags", optional=True))


def workspace_bytes(op, d: Dims = None, max_rows=0, max_q=0) -> int:
    return int(lib().mtgnn_workspace_bytes(op, C.byref(d) if d is not None else None, int(max_rows), int(max_q)))


def save_bytes(op, d: Dims, max_rows=0, max_q=0) -> int:
    return int(lib().mtgnn_save_bytes(op, C.byref(d), int(max_rows), int(max_q)))


def alloc_bytes(n, device="cuda"):
    return torch.empty(max(int(n), 1), dtype=torch.uint8, device=device)


# ----------------------------------------------------------------------------- entry points

def mtgnn_build_queries(b: Batch, neg, q_node, q_t, n_q, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_build_queries(C.byref(b), _ptr(neg, torch.int32, "neg"), _ptr(q_node, torch.int32, "q_node"),
                                     _ptr(q_t, torch.float32, "q_t"), _ptr(n_q, torch.int32, "n_q"), wp, wb,
                                     _stream(stream)), "mtgnn_build_queries")


def mtgnn_aggregate_last(b: Batch, n_nodes, uniq, winner, n_uniq, ws, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_aggregate_last(C.byref(b), int(n_nodes), _ptr(uniq, torch.int32, "uniq"),
                                      _ptr(winner, torch.int32, "winner"), _ptr(n_uniq, torch.int32, "n_uniq"), wp, wb,
                                      _stream(stream)), "mtgnn_aggregate_last")


def mtgnn_build_messages(b: Batch, uniq, winner, n_rows, max_rows, memory, last_update, edge_feat, time_w, time_b,
                         d: Dims, msg, dt, stream=None):
    md = _DT[d.dtype]
    _check(lib().mtgnn_build_messages(C.byref(b), _ptr(uniq, torch.int32, "uniq"), _ptr(winner, torch.int32, "winner"),
                                      _ptr(n_rows, torch.int32, "n_rows", True), int(max_rows),
                                      _ptr(memory, md, "memory"), _ptr(last_update, torch.float32, "last_update"),
                                      _ptr(edge_feat, torch.float32, "edge_feat", True),
                                      _ptr(time_w, torch.float32, "time_w"), _ptr(time_b, torch.float32, "time_b"),
                                      C.byref(d), _ptr(msg, md, "msg"), _ptr(dt, torch.float32, "dt"),
                                      _stream(stream)), "mtgnn_build_messages")


def mtgnn_gru_update(b: Batch, uniq, winner, n_rows, max_rows, msg, W_ih, W_hh, b_ih, b_hh, d: Dims, memory,
                     last_update, save, ws, stream=None):
    md = _DT[d.dtype]
    wp, wb = _ws(ws)
    _check(lib().mtgnn_gru_update(C.byref(b), _ptr(uniq, torch.int32, "uniq"), _ptr(winner, torch.int32, "winner"),
                                  _ptr(n_rows, torch.int32, "n_rows", True), int(max_rows), _ptr(msg, md, "msg"),
                                  _ptr(W_ih, md, "W_ih"), _ptr(W_hh, md, "W_hh"), _ptr(b_ih, torch.float32, "b_ih"),
                                  _ptr(b_hh, torch.float32, "b_hh"), C.byref(d), _ptr(memory, md, "memory"),
                                  _ptr(last_update, torch.float32, "last_update"),
                                  _ptr(save, torch.uint8, "save", True), wp, wb, _stream(stream)), "mtgnn_gru_update")


def mtgnn_sample_recent(csr_off, csr_nbr, csr_t, csr_eid, n_nodes, q_node, q_t, n_q, max_q, k, out_nbr, out_t,
                        out_eid, stream=None):
    _check(lib().mtgnn_sample_recent(_ptr(csr_off, torch.int64, "csr_off"), _ptr(csr_nbr, torch.int32, "csr_nbr"),
                                     _ptr(csr_t, torch.float32, "csr_t"), _ptr(csr_eid, torch.int32, "csr_eid"),
                                     int(n_nodes), _ptr(q_node, torch.int32, "q_node"), _ptr(q_t, torch.float32, "q_t"),
                                     _ptr(n_q, torch.int32, "n_q", True), int(max_q), int(k),
                                     _ptr(out_nbr, torch.int32, "out_nbr"), _ptr(out_t, torch.float32, "out_t"),
                                     _ptr(out_eid, torch.int32, "out_eid"), _stream(stream)), "mtgnn_sample_recent")


def attn_params(p: dict, d: Dims) -> AttnParams:
    md = _DT[d.dtype]
    return AttnParams(*[_ptr(p[n], md if n.startswith("W") else torch.float32, n) for n in _ATTN])


def attn_grads(g: dict) -> AttnGrads:
    return AttnGrads(*[_ptr(g[n], torch.float32, "d" + n) for n in _ATTN])


def mtgnn_temporal_attn(q_node, q_t, n_q, max_q, nbr, nt, neid, memory, edge_feat, time_w, time_b,
                        params: AttnParams, d: Dims, z, save, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_temporal_attn(_ptr(q_node, torch.int32, "q_node"), _ptr(q_t, torch.float32, "q_t"),
                                     _ptr(n_q, torch.int32, "n_q", True), int(max_q), _ptr(nbr, torch.int32, "nbr"),
                                     _ptr(nt, torch.float32, "nt"), _ptr(neid, torch.int32, "neid"),
                                     _ptr(memory, _DT[d.dtype], "memory"),
                                     _ptr(edge_feat, torch.float32, "edge_feat", True),
                                     _ptr(time_w, torch.float32, "time_w"), _ptr(time_b, torch.float32, "time_b"),
                                     C.byref(params), C.byref(d), _ptr(z, torch.float32, "z"),
                                     _ptr(save, torch.uint8, "save"), wp, wb, _stream(stream)), "mtgnn_temporal_attn")


def mtgnn_temporal_attn_prepare(nbr, n_q, max_q, params: AttnParams, time_w, time_b, d: Dims, save, ws=None,
                                stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_temporal_attn_prepare(_ptr(nbr, torch.int32, "nbr"), _ptr(n_q, torch.int32, "n_q", True),
                                             int(max_q), C.byref(params), _ptr(time_w, torch.float32, "time_w"),
                                             _ptr(time_b, torch.float32, "time_b"), C.byref(d),
                                             _ptr(save, torch.uint8, "save"), wp, wb, _stream(stream)),
           "mtgnn_temporal_attn_prepare")


def mtgnn_temporal_attn_prepare_weights(params: AttnParams, time_w, time_b, d: Dims, save, stream=None):
    _check(lib().mtgnn_temporal_attn_prepare_weights(C.byref(params), _ptr(time_w, torch.float32, "time_w"),
                                                     _ptr(time_b, torch.float32, "time_b"), C.byref(d),
                                                     _ptr(save, torch.uint8, "save"), _stream(stream)),
           "mtgnn_temporal_attn_prepare_weights")


def mtgnn_temporal_attn_prepare_weights_link(params: AttnParams, time_w, time_b, d: Dims, save, link: LinkParams,
                                             max_q, link_ws, stream=None):
    wp, wb = _ws(link_ws)
    _check(lib().mtgnn_temporal_attn_prepare_weights_link(C.byref(params), _ptr(time_w, torch.float32, "time_w"),
                                                          _ptr(time_b, torch.float32, "time_b"), C.byref(d),
                                                          _ptr(save, torch.uint8, "save"), C.byref(link), int(max_q),
                                                          wp, wb, _stream(stream)),
           "mtgnn_temporal_attn_prepare_weights_link")


def mtgnn_temporal_attn_prepare_slots(nbr, n_q, max_q, d: Dims, save, ws=None, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_temporal_attn_prepare_slots(_ptr(nbr, torch.int32, "nbr"), _ptr(n_q, torch.int32, "n_q", True),
                                                   int(max_q), C.byref(d), _ptr(save, torch.uint8, "save"), wp, wb,
                                                   _stream(stream)), "mtgnn_temporal_attn_prepare_slots")


def mtgnn_temporal_attn_prepared(q_node, q_t, n_q, max_q, nbr, nt, neid, memory, edge_feat, time_w, time_b,
                                 params: AttnParams, d: Dims, z, save, stream=None):
    _check(lib().mtgnn_temporal_attn_prepared(_ptr(q_node, torch.int32, "q_node"), _ptr(q_t, torch.float32, "q_t"),
                                              _ptr(n_q, torch.int32, "n_q", True), int(max_q),
                                              _ptr(nbr, torch.int32, "nbr"), _ptr(nt, torch.float32, "nt"),
                                              _ptr(neid, torch.int32, "neid"), _ptr(memory, _DT[d.dtype], "memory"),
                                              _ptr(edge_feat, torch.float32, "edge_feat", True),
                                              _ptr(time_w, torch.float32, "time_w"),
                                              _ptr(time_b, torch.float32, "time_b"), C.byref(params), C.byref(d),
                                              _ptr(z, torch.float32, "z"), _ptr(save, torch.uint8, "save"),
                                              _stream(stream)), "mtgnn_temporal_attn_prepared")


def mtgnn_temporal_attn_bwd(q_node, q_t, n_q, max_q, nbr, nt, dz, save, uniq, n_rows, max_rows, time_w, time_b,
                            params: AttnParams, d: Dims, grads: AttnGrads, d_mem, d_time_w, d_time_b, ws,
                            stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_temporal_attn_bwd(_ptr(q_node, torch.int32, "q_node"), _ptr(q_t, torch.float32, "q_t"),
                                         _ptr(n_q, torch.int32, "n_q", True), int(max_q),
                                         _ptr(nbr, torch.int32, "nbr"), _ptr(nt, torch.float32, "nt"),
                                         _ptr(dz, torch.float32, "dz"), _ptr(save, torch.uint8, "save"),
                                         _ptr(uniq, torch.int32, "uniq", True), _ptr(n_rows, torch.int32, "n_rows", True),
                                         int(max_rows), _ptr(time_w, torch.float32, "time_w"),
                                         _ptr(time_b, torch.float32, "time_b"), C.byref(params), C.byref(d),
                                         C.byref(grads), _ptr(d_mem, torch.float32, "d_mem", True),
                                         _ptr(d_time_w, torch.float32, "d_time_w"),
                                         _ptr(d_time_b, torch.float32, "d_time_b"), wp, wb, _stream(stream)),
           "mtgnn_temporal_attn_bwd")


_hip = None


def _hip_rt():
    # the HIP runtime already loaded in this process (torch's, which the library resolves to as well)
    global _hip
    if _hip is None:
        _hip = C.CDLL("libamdhip64.so.7", mode=C.RTLD_GLOBAL)
        for f in ("hipEventCreateWithFlags", "hipEventRecord", "hipStreamWaitEvent", "hipEventDestroy"):
            getattr(_hip, f).restype = C.c_int
    return _hip


def _hip_check(rc, what):
    if rc != 0:
        raise MtgnnError(f"{what} failed with HIP error {rc}")


class DeviceEvent:
    """An event that orders work between two streams of the current device.

    No timing, and a device-scope release when it is recorded (hipEventDisableSystemFence): both streams
    run on one GPU, so the system-scope fence of a default event, a cache write-back and invalidate that
    costs several microseconds per record, is not needed.  Methods follow torch.cuda.Event's:
    record(stream) and wait(stream) (the stream waits for the event)."""

    _FLAGS = 0x2 | 0x20000000   # hipEventDisableTiming | hipEventDisableSystemFence

    def __init__(self):
        self._rt = _hip_rt()
        h = C.c_void_p()
        _hip_check(self._rt.hipEventCreateWithFlags(C.byref(h), C.c_uint(self._FLAGS)), "hipEventCreateWithFlags")
        self.handle = h

    def record(self, stream=None):
        _hip_check(self._rt.hipEventRecord(self.handle, _stream(stream)), "hipEventRecord")

    def wait(self, stream=None):
        _hip_check(self._rt.hipStreamWaitEvent(_stream(stream), self.handle, C.c_uint(0)), "hipStreamWaitEvent")

    def __del__(self):
        try:   # may run at interpreter exit, after the runtime (or this module's globals) are gone
            if getattr(self, "handle", None) and self.handle.value:
                self._rt.hipEventDestroy(self.handle)
                self.handle = None
        except Exception:
            pass


def _event(e, name):
    if isinstance(e, DeviceEvent):
        return e.handle
    h = e.cuda_event if isinstance(e, torch.cuda.Event) else 0
    if not h:
        raise MtgnnError(f"{name}: a torch.cuda.Event that has been recorded once (so that it exists) is required")
    return C.c_void_p(h)


def mtgnn_temporal_attn_bwd_group(q_node, n_q, max_q, nbr, save, uniq, n_rows, max_rows, d: Dims, ws, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_temporal_attn_bwd_group(
        _ptr(q_node, torch.int32, "q_node"), _ptr(n_q, torch.int32, "n_q", True), int(max_q),
        _ptr(nbr, torch.int32, "nbr"), _ptr(save, torch.uint8, "save"), _ptr(uniq, torch.int32, "uniq", True),
        _ptr(n_rows, torch.int32, "n_rows", True), int(max_rows), C.byref(d), wp, wb, _stream(stream)),
        "mtgnn_temporal_attn_bwd_group")


def mtgnn_temporal_attn_bwd_overlap(q_node, q_t, n_q, max_q, nbr, nt, dz, save, uniq, n_rows, max_rows, time_w,
                                    time_b, params: AttnParams, d: Dims, grads: AttnGrads, d_mem, d_time_w, d_time_b,
                                    ws, dmem_stream, fork, join, stream=None, grouped=False):
    """grouped=True calls mtgnn_temporal_attn_bwd_grouped (the grouping left in ws by
    mtgnn_temporal_attn_bwd_group on dmem_stream); there join may be None (the caller joins)."""
    wp, wb = _ws(ws)
    name = "mtgnn_temporal_attn_bwd_grouped" if grouped else "mtgnn_temporal_attn_bwd_overlap"
    _check(getattr(lib(), name)(
        _ptr(q_node, torch.int32, "q_node"), _ptr(q_t, torch.float32, "q_t"), _ptr(n_q, torch.int32, "n_q", True),
        int(max_q), _ptr(nbr, torch.int32, "nbr"), _ptr(nt, torch.float32, "nt"), _ptr(dz, torch.float32, "dz"),
        _ptr(save, torch.uint8, "save"), _ptr(uniq, torch.int32, "uniq", True),
        _ptr(n_rows, torch.int32, "n_rows", True), int(max_rows), _ptr(time_w, torch.float32, "time_w"),
        _ptr(time_b, torch.float32, "time_b"), C.byref(params), C.byref(d), C.byref(grads),
        _ptr(d_mem, torch.float32, "d_mem", True), _ptr(d_time_w, torch.float32, "d_time_w"),
        _ptr(d_time_b, torch.float32, "d_time_b"), wp, wb, _stream(stream), _stream(dmem_stream),
        _event(fork, "fork"), None if (grouped and join is None) else _event(join, "join")), name)


def mtgnn_gru_update_bwd(d_mem, save, msg, n_rows, max_rows, W_ih, W_hh, d: Dims, dW_ih, dW_hh, db_ih, db_hh,
                         dmsg_time, ws, stream=None):
    md = _DT[d.dtype]
    wp, wb = _ws(ws)
    _check(lib().mtgnn_gru_update_bwd(_ptr(d_mem, torch.float32, "d_mem"), _ptr(save, torch.uint8, "save"),
                                      _ptr(msg, md, "msg"), _ptr(n_rows, torch.int32, "n_rows", True), int(max_rows),
                                      _ptr(W_ih, md, "W_ih"), _ptr(W_hh, md, "W_hh"), C.byref(d),
                                      _ptr(dW_ih, torch.float32, "dW_ih"), _ptr(dW_hh, torch.float32, "dW_hh"),
                                      _ptr(db_ih, torch.float32, "db_ih"), _ptr(db_hh, torch.float32, "db_hh"),
                                      _ptr(dmsg_time, torch.float32, "dmsg_time", True), wp, wb, _stream(stream)),
           "mtgnn_gru_update_bwd")


def link_params(p: dict) -> LinkParams:
    return LinkParams(*[_ptr(p[n], torch.float32, n) for n in _LINK])


def link_grads(g: dict) -> LinkGrads:
    return LinkGrads(*[_ptr(g[n], torch.float32, "d" + n) for n in _LINK])


def mtgnn_link_prepare_weights(params: LinkParams, d: Dims, max_q, ws, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_link_prepare_weights(C.byref(params), C.byref(d), int(max_q), wp, wb, _stream(stream)),
           "mtgnn_link_prepare_weights")


def mtgnn_link_loss(z, n_q, max_q, params: LinkParams, d: Dims, loss, scores, dz, grads: LinkGrads, ws, stream=None,
                    dw_stream=None, fork=None, prepared=False):
    """dw_stream and fork given: mtgnn_link_loss_overlap (W_d1's gradient on dw_stream after fork).
    prepared: mtgnn_link_loss_prepared (ws holds mtgnn_link_prepare_weights' copies of params' W_d1)."""
    wp, wb = _ws(ws)
    args = (_ptr(z, torch.float32, "z"), _ptr(n_q, torch.int32, "n_q", True), int(max_q), C.byref(params), C.byref(d),
            _ptr(loss, torch.float32, "loss"), _ptr(scores, torch.float32, "scores", True), _ptr(dz, torch.float32, "dz"),
            C.byref(grads), wp, wb, _stream(stream))
    if prepared:
        ov = dw_stream is not None
        _check(lib().mtgnn_link_loss_prepared(*args, _stream(dw_stream) if ov else None,
                                              _event(fork, "fork") if ov else None), "mtgnn_link_loss_prepared")
    elif dw_stream is None:
        _check(lib().mtgnn_link_loss(*args), "mtgnn_link_loss")
    else:
        _check(lib().mtgnn_link_loss_overlap(*args, _stream(dw_stream), _event(fork, "fork")),
               "mtgnn_link_loss_overlap")


def mtgnn_build_messages_bwd(dmsg_time, dt, n_rows, max_rows, time_w, time_b, d: Dims, d_time_w, d_time_b, ws,
                             stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_build_messages_bwd(_ptr(dmsg_time, torch.float32, "dmsg_time"), _ptr(dt, torch.float32, "dt"),
                                          _ptr(n_rows, torch.int32, "n_rows", True), int(max_rows),
                                          _ptr(time_w, torch.float32, "time_w"), _ptr(time_b, torch.float32, "time_b"),
                                          C.byref(d), _ptr(d_time_w, torch.float32, "d_time_w"),
                                          _ptr(d_time_b, torch.float32, "d_time_b"), wp, wb, _stream(stream)),
           "mtgnn_build_messages_bwd")


def mtgnn_build_messages_bwd_noalloc(dmsg_time, dt, n_rows, max_rows, time_w, time_b, d: Dims, d_time_w, d_time_b,
                                     stream=None):
    _check(lib().mtgnn_build_messages_bwd_noalloc(
        _ptr(dmsg_time, torch.float32, "dmsg_time"), _ptr(dt, torch.float32, "dt"),
        _ptr(n_rows, torch.int32, "n_rows", True), int(max_rows), _ptr(time_w, torch.float32, "time_w"),
        _ptr(time_b, torch.float32, "time_b"), C.byref(d), _ptr(d_time_w, torch.float32, "d_time_w"),
        _ptr(d_time_b, torch.float32, "d_time_b"), _stream(stream)), "mtgnn_build_messages_bwd_noalloc")


def mtgnn_build_temporal_csr(src, dst, t, n_nodes, csr_off, csr_nbr, csr_t, csr_eid, ws, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_build_temporal_csr(_ptr(src, torch.int32, "src"), _ptr(dst, torch.int32, "dst"),
                                          _ptr(t, torch.float32, "t"), int(src.numel()), int(n_nodes),
                                          _ptr(csr_off, torch.int64, "csr_off"), _ptr(csr_nbr, torch.int32, "csr_nbr"),
                                          _ptr(csr_t, torch.float32, "csr_t"), _ptr(csr_eid, torch.int32, "csr_eid"),
                                          wp, wb, _stream(stream)), "mtgnn_build_temporal_csr")


def mtgnn_dependency_scan(src, dst, owner, n_workers, batch, window, role, sync_bits, stream=None):
    _check(lib().mtgnn_dependency_scan(_ptr(src, torch.int32, "src"), _ptr(dst, torch.int32, "dst"), int(src.numel()),
                                       _ptr(owner, torch.int32, "owner"), int(owner.numel()), int(n_workers),
                                       int(batch), int(window), _ptr(role, torch.uint8, "role"),
                                       _ptr(sync_bits, torch.int32, "sync_bits"), _stream(stream)),
           "mtgnn_dependency_scan")


def mtgnn_mixed_batches(role, batch, eid_out, flags_out, batch_off, ws, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_mixed_batches(_ptr(role, torch.uint8, "role"), int(role.numel()), int(batch),
                                     _ptr(eid_out, torch.int32, "eid_out"), _ptr(flags_out, torch.uint8, "flags_out"),
                                     _ptr(batch_off, torch.int32, "batch_off"), wp, wb, _stream(stream)),
           "mtgnn_mixed_batches")


def mtgnn_rnn_update(b: Batch, uniq, winner, n_rows, max_rows, msg, W_ih, W_hh, b_ih, b_hh, d: Dims, memory,
                     last_update, save, ws, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_rnn_update(C.byref(b), _ptr(uniq, torch.int32, "uniq"), _ptr(winner, torch.int32, "winner"),
                                  _ptr(n_rows, torch.int32, "n_rows", True), int(max_rows), _ptr(msg, _DT[d.dtype], "msg"),
                                  _ptr(W_ih, _DT[d.dtype], "W_ih"), _ptr(W_hh, _DT[d.dtype], "W_hh"),
                                  _ptr(b_ih, torch.float32, "b_ih"), _ptr(b_hh, torch.float32, "b_hh"), C.byref(d),
                                  _ptr(memory, _DT[d.dtype], "memory"), _ptr(last_update, torch.float32, "last_update"),
                                  _ptr(save, torch.uint8, "save", True), wp, wb, _stream(stream)), "mtgnn_rnn_update")


def mtgnn_rnn_update_bwd(d_mem, save, msg, n_rows, max_rows, W_ih, W_hh, d: Dims, dW_ih, dW_hh, db_ih, db_hh,
                         dmsg_time, ws, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_rnn_update_bwd(_ptr(d_mem, torch.float32, "d_mem"), _ptr(save, torch.uint8, "save"),
                                      _ptr(msg, _DT[d.dtype], "msg"), _ptr(n_rows, torch.int32, "n_rows", True),
                                      int(max_rows), _ptr(W_ih, _DT[d.dtype], "W_ih"), _ptr(W_hh, _DT[d.dtype], "W_hh"),
                                      C.byref(d), _ptr(dW_ih, torch.float32, "dW_ih"),
                                      _ptr(dW_hh, torch.float32, "dW_hh"), _ptr(db_ih, torch.float32, "db_ih"),
                                      _ptr(db_hh, torch.float32, "db_hh"),
                                      _ptr(dmsg_time, torch.float32, "dmsg_time", True), wp, wb, _stream(stream)),
           "mtgnn_rnn_update_bwd")


def mtgnn_time_projection(q_node, q_t, n_q, max_q, memory, last_update, W_p, b_p, time_scale, d: Dims, z,
                          stream=None):
    _check(lib().mtgnn_time_projection(_ptr(q_node, torch.int32, "q_node"), _ptr(q_t, torch.float32, "q_t"),
                                       _ptr(n_q, torch.int32, "n_q", True), int(max_q),
                                       _ptr(memory, _DT[d.dtype], "memory"),
                                       _ptr(last_update, torch.float32, "last_update"), _ptr(W_p, torch.float32, "W_p"),
                                       _ptr(b_p, torch.float32, "b_p"), float(time_scale), C.byref(d),
                                       _ptr(z, torch.float32, "z"), _stream(stream)), "mtgnn_time_projection")


def mtgnn_time_projection_bwd(q_node, q_t, n_q, max_q, memory, last_update, W_p, b_p, time_scale, dz, uniq, n_rows,
                              max_rows, d: Dims, dW_p, db_p, d_mem, ws, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_time_projection_bwd(
        _ptr(q_node, torch.int32, "q_node"), _ptr(q_t, torch.float32, "q_t"), _ptr(n_q, torch.int32, "n_q", True),
        int(max_q), _ptr(memory, _DT[d.dtype], "memory"), _ptr(last_update, torch.float32, "last_update"),
        _ptr(W_p, torch.float32, "W_p"), _ptr(b_p, torch.float32, "b_p"), float(time_scale),
        _ptr(dz, torch.float32, "dz"), _ptr(uniq, torch.int32, "uniq"), _ptr(n_rows, torch.int32, "n_rows", True),
        int(max_rows), C.byref(d), _ptr(dW_p, torch.float32, "dW_p"), _ptr(db_p, torch.float32, "db_p"),
        _ptr(d_mem, torch.float32, "d_mem"), wp, wb, _stream(stream)), "mtgnn_time_projection_bwd")


class Controller:
    """The library's host-side runtime controller (Eq. 6-9): decisions before a batch, observations after."""

    def __init__(self, alpha, beta, tau_g, tau_c, interval):
        h = C.c_void_p()
        _check(lib().mtgnn_controller_create(C.byref(ControllerConfig(alpha, beta, tau_g, tau_c, int(interval))),
                                             C.byref(h)), "mtgnn_controller_create")
        self._h = h

    def decide(self, r):
        """(boundary, S_r, H_r) before batch r."""
        b, sy, hv = C.c_int32(), C.c_int32(), C.c_int32()
        _check(lib().mtgnn_controller_decide(self._h, int(r), C.byref(b), C.byref(sy), C.byref(hv)),
               "mtgnn_controller_decide")
        return b.value, sy.value, hv.value

    def observe(self, grad_norm, batch_time):
        _check(lib().mtgnn_controller_observe(self._h, float(grad_norm), float(batch_time)),
               "mtgnn_controller_observe")

    def state(self):
        v = [C.c_double() for _ in range(4)]
        _check(lib().mtgnn_controller_state(self._h, *[C.byref(x) for x in v]), "mtgnn_controller_state")
        return tuple(x.value for x in v)

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _lib is not None:
            _lib.mtgnn_controller_destroy(h)
            self._h = None


def _ptr_array(ts, dtype, name):
    arr = (C.c_void_p * len(ts))()
    for i, t in enumerate(ts):
        arr[i] = _ptr(t, dtype, name).value
    return arr


def _sizes(ts):
    return (C.c_int64 * len(ts))(*[int(t.numel()) for t in ts])


def grad_norm_ws_bytes(tensors) -> int:
    return int(lib().mtgnn_grad_norm_ws_bytes(_sizes(tensors), len(tensors)))


def mtgnn_grad_norm(grads, norm, ws, stream=None):
    wp, wb = _ws(ws)
    _check(lib().mtgnn_grad_norm(_ptr_array(grads, torch.float32, "grad"), _sizes(grads), len(grads),
                                 _ptr(norm, torch.float64, "norm"), wp, wb, _stream(stream)), "mtgnn_grad_norm")


def mtgnn_prune_aux(flags, heavy, stream=None):
    _check(lib().mtgnn_prune_aux(_ptr(flags, torch.uint8, "flags"), int(flags.numel()), int(heavy), _stream(stream)),
           "mtgnn_prune_aux")


def mtgnn_cache_refresh(sync_bits, n_nodes, auth_memory, auth_lu, d: Dims, memory, last_update, stream=None):
    _check(lib().mtgnn_cache_refresh(_ptr(sync_bits, torch.int32, "sync_bits"), int(n_nodes),
                                     _ptr(auth_memory, None, "auth_memory"), _ptr(auth_lu, torch.float32, "auth_lu"),
                                     C.byref(d), _ptr(memory, None, "memory"),
                                     _ptr(last_update, torch.float32, "last_update"), _stream(stream)),
           "mtgnn_cache_refresh")


def mtgnn_adam_step(params, grads, m, v, shadow, lr, beta1, beta2, eps, t, stream=None):
    """params, grads, m, v: lists of float32 tensors; shadow: None or a list of (None | bf16 tensor)."""
    sh = None
    if shadow is not None:
        sh = (C.c_void_p * len(shadow))()
        for i, x in enumerate(shadow):
            sh[i] = None if x is None else _ptr(x, torch.bfloat16, "shadow").value
    _check(lib().mtgnn_adam_step(_ptr_array(params, torch.float32, "param"), _ptr_array(grads, torch.float32, "grad"),
                                 _ptr_array(m, torch.float32, "m"), _ptr_array(v, torch.float32, "v"), sh,
                                 _sizes(params), len(params), C.byref(AdamConfig(lr, beta1, beta2, eps, int(t))),
                                 _stream(stream)), "mtgnn_adam_step")


# ----------------------------------------------------------------------------- state-space layer

def _device() -> int:
    """The current device, on which all tensors of a call have to be (-1: no GPU tensor can exist yet)."""
    return torch.cuda.current_device() if torch.cuda.is_initialized() else -1


def _elsewhere(t, name, dev):
    if t.is_cuda:
        raise MtgnnError(f"{name} is on {t.device}, the current device is {dev}")


def _made_here(what, name, dev):
    """Refuses what holds the addresses of another device's tensors (a bare structure has its own)."""
    if getattr(what, "device", dev) != dev:
        raise MtgnnError(f"{name} are on device {what.device}, the current device is {dev}")


def _rows(t, dtype, name, rows, cols, optional=False, dev=-1):
    """(pointer, row stride) of a [rows or more, cols] matrix whose rows are dense."""
    if t is None:
        if optional:
            return None, cols
        raise MtgnnError(f"{name} is required")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise MtgnnError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise MtgnnError(f"{name} must be {dtype}, got {t.dtype}")
    shape, ld = t.shape, t.stride(0) if t.dim() == 2 else 0
    if len(shape) != 2 or shape[0] < rows or shape[1] != cols:
        raise MtgnnError(f"{name} must be [{rows}, {cols}], got {tuple(shape)}")
    if (cols > 1 and t.stride(1) != 1) or (shape[0] > 1 and ld < cols):
        raise MtgnnError(f"{name} must have dense rows, got strides {t.stride()}")
    if t.get_device() != dev:
        _elsewhere(t, name, dev)
    return C.c_void_p(t.data_ptr()), max(ld, cols)


def _table(t, dtype, name, shape, optional=False, dev=-1):
    """Pointer of a dense tensor of the given shape."""
    if t is None:
        return _ptr(t, dtype, name, optional)
    if t.shape != shape:
        raise MtgnnError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    p = _ptr(t, dtype, name)
    if t.get_device() != dev:
        _elsewhere(t, name, dev)
    return p


def _count(t, n, name, dev=-1):
    """Pointer of an int32 tensor of n entries or more, or NULL."""
    if t is None:
        return None
    if t.numel() < n:
        raise MtgnnError(f"{name} must have {n} entries, got {t.numel()}")
    p = _ptr(t, torch.int32, name)
    if t.get_device() != dev:
        _elsewhere(t, name, dev)
    return p


def _bytes(t, need, name, optional=False, dev=-1):
    if t is not None and t.numel() < need:
        raise MtgnnError(f"{name} must have {need} bytes, got {t.numel()}")
    p = _ptr(t, torch.uint8, name, optional)
    if t is not None and t.get_device() != dev:
        _elsewhere(t, name, dev)
    return p


def _work(ws, dev):
    """(pointer, bytes) of a workspace, or (None, 0)."""
    return (None, 0) if ws is None else (_bytes(ws, 0, "ws", dev=dev), ws.numel())


def seqs(off, max_rows, n_seq=None, slot=None, n_slots=0) -> Seqs:
    """Sequences in the rows of a matrix: sequence s has rows off[s] .. off[s + 1] - 1 (off int32, one entry more
    than there are sequences at most).  It keeps its tensors."""
    dev = _device()
    max_seq = int(off.numel()) - 1
    if max_seq < 0:
        raise MtgnnError("off must have one entry more than there are sequences")
    s = Seqs(int(max_rows), max_seq, int(n_slots), _count(off, 1, "off", dev=dev), _count(n_seq, 1, "n_seq", dev=dev),
             _count(slot, max_seq, "slot", dev=dev))
    s.tensors, s.device = (off, n_seq, slot), dev
    return s


def linear_dims(d_in, d_out, dtype=F32, act=ACT_NONE) -> LinearDims:
    return LinearDims(int(d_in), int(d_out), int(dtype), int(act))


def conv_dims(d, width, dtype=F32, act=ACT_SILU) -> ConvDims:
    return ConvDims(int(d), int(width), int(dtype), int(act))


def scan_dims(d, n, groups=1, dtype=F32, softplus=True) -> ScanDims:
    return ScanDims(int(d), int(n), int(groups), int(dtype), int(softplus))


def linear_ws_bytes(d: LinearDims, max_rows, backward=False) -> int:
    return int(lib().mtgnn_linear_ws_bytes(C.byref(d), int(max_rows), int(backward)))


def causal_conv_ws_bytes(d: ConvDims, max_rows) -> int:
    return int(lib().mtgnn_causal_conv_ws_bytes(C.byref(d), int(max_rows)))


def causal_conv_save_bytes(d: ConvDims, max_seq) -> int:
    return int(lib().mtgnn_causal_conv_save_bytes(C.byref(d), int(max_seq)))


def selective_scan_ws_bytes(d: ScanDims, max_rows, max_seq, backward=False) -> int:
    return int(lib().mtgnn_selective_scan_ws_bytes(C.byref(d), int(max_rows), int(max_seq), int(backward)))


def selective_scan_save_bytes(d: ScanDims, max_rows, max_seq, carried) -> int:
    return int(lib().mtgnn_selective_scan_save_bytes(C.byref(d), int(max_rows), int(max_seq), int(carried)))


def mtgnn_linear(x, W, b, residual, d: LinearDims, y, pre=None, n_rows=None, ws=None, stream=None):
    """y = act(x W^T + b) + residual; pre: where the backward will find x W^T + b."""
    dev = _device()
    md, R = _DT[d.dtype], int(x.shape[0])
    xp, ldx = _rows(x, md, "x", R, d.d_in, dev=dev)
    rp, ldr = _rows(residual, md, "residual", R, d.d_out, optional=True, dev=dev)
    yp, ldy = _rows(y, md, "y", R, d.d_out, dev=dev)
    wp, wb = _work(ws, dev)
    _check(lib().mtgnn_linear(xp, ldx, _count(n_rows, 1, "n_rows", dev=dev), R,
                              _table(W, md, "W", (d.d_out, d.d_in), dev=dev),
                              _table(b, torch.float32, "b", (d.d_out,), True, dev=dev), rp, ldr, C.byref(d), yp, ldy,
                              _table(pre, torch.float32, "pre", (R, d.d_out), True, dev=dev), wp, wb, _stream(stream)),
           "mtgnn_linear")


def mtgnn_linear_bwd(dy, pre, x, W, d: LinearDims, dx, dW, db, n_rows=None, ws=None, stream=None):
    dev = _device()
    md, R, f32 = _DT[d.dtype], int(x.shape[0]), torch.float32
    gp, lddy = _rows(dy, f32, "dy", R, d.d_out, dev=dev)
    xp, ldx = _rows(x, md, "x", R, d.d_in, dev=dev)
    dp, lddx = _rows(dx, f32, "dx", R, d.d_in, optional=True, dev=dev)
    wp, wb = _work(ws, dev)
    _check(lib().mtgnn_linear_bwd(gp, lddy, _table(pre, f32, "pre", (R, d.d_out), d.act == ACT_NONE, dev=dev), xp, ldx,
                                  _count(n_rows, 1, "n_rows", dev=dev), R,
                                  _table(W, md, "W", (d.d_out, d.d_in), dev=dev), C.byref(d), dp, lddx,
                                  _table(dW, f32, "dW", (d.d_out, d.d_in), dev=dev),
                                  _table(db, f32, "db", (d.d_out,), True, dev=dev), wp, wb, _stream(stream)),
           "mtgnn_linear_bwd")


def mtgnn_causal_conv(q: Seqs, x, w, b, d: ConvDims, state_in, state_out, y, save=None, stream=None):
    dev = _device()
    md = _DT[d.dtype]
    _made_here(q, "seqs", dev)
    xp, ldx = _rows(x, md, "x", q.max_rows, d.d, dev=dev)
    yp, ldy = _rows(y, md, "y", q.max_rows, d.d, dev=dev)
    st = (q.n_slots, d.width - 1, d.d)
    _check(lib().mtgnn_causal_conv(C.byref(q), xp, ldx, _table(w, md, "w", (d.width, d.d), dev=dev),
                                   _table(b, torch.float32, "b", (d.d,), True, dev=dev), C.byref(d),
                                   _table(state_in, md, "state_in", st, True, dev=dev),
                                   _table(state_out, md, "state_out", st, True, dev=dev), yp, ldy,
                                   _bytes(save, causal_conv_save_bytes(d, q.max_seq), "save", True, dev=dev),
                                   _stream(stream)), "mtgnn_causal_conv")


def mtgnn_causal_conv_bwd(q: Seqs, dy, x, w, b, d: ConvDims, save, dx, dw, db, ws, stream=None):
    dev = _device()
    md, f32 = _DT[d.dtype], torch.float32
    _made_here(q, "seqs", dev)
    gp, lddy = _rows(dy, f32, "dy", q.max_rows, d.d, dev=dev)
    xp, ldx = _rows(x, md, "x", q.max_rows, d.d, dev=dev)
    dp, lddx = _rows(dx, f32, "dx", q.max_rows, d.d, dev=dev)
    wp, wb = _work(ws, dev)
    _check(lib().mtgnn_causal_conv_bwd(C.byref(q), gp, lddy, xp, ldx, _table(w, md, "w", (d.width, d.d), dev=dev),
                                       _table(b, f32, "b", (d.d,), True, dev=dev), C.byref(d),
                                       _bytes(save, causal_conv_save_bytes(d, q.max_seq), "save", True, dev=dev), dp, lddx,
                                       _table(dw, f32, "dw", (d.width, d.d), dev=dev),
                                       _table(db, f32, "db", (d.d,), True, dev=dev), wp, wb, _stream(stream)),
           "mtgnn_causal_conv_bwd")


def mtgnn_causal_conv_step(slot, x, w, b, d: ConvDims, state_in, state_out, y, n_rows=None, stream=None):
    """One row each: x[r] is the next row of slot[r] (None: slot r)."""
    dev = _device()
    md, R = _DT[d.dtype], int(x.shape[0])
    xp, ldx = _rows(x, md, "x", R, d.d, dev=dev)
    yp, ldy = _rows(y, md, "y", R, d.d, dev=dev)
    n = _n_slots(state_in, state_out)
    st = (n, d.width - 1, d.d)
    _check(lib().mtgnn_causal_conv_step(_count(slot, R, "slot", dev=dev), _count(n_rows, 1, "n_rows", dev=dev), R, n,
                                        xp, ldx,
                                        _table(w, md, "w", (d.width, d.d), dev=dev),
                                        _table(b, torch.float32, "b", (d.d,), True, dev=dev), C.byref(d),
                                        _table(state_in, md, "state_in", st, True, dev=dev),
                                        _table(state_out, md, "state_out", st, True, dev=dev), yp, ldy, _stream(stream)),
           "mtgnn_causal_conv_step")


def _n_slots(state_in, state_out):
    t = state_in if state_in is not None else state_out
    return 0 if t is None else int(t.shape[0])


def scan_inputs(d: ScanDims, x, delta, A, B, C_, D=None, z=None, delta_bias=None) -> ScanInputs:
    """The scan's inputs; it keeps its tensors."""
    dev = _device()
    md, f32, R, gn = _DT[d.dtype], torch.float32, int(x.shape[0]), d.groups * d.n
    r = [_rows(x, md, "x", R, d.d, dev=dev), _rows(delta, md, "delta", R, d.d, dev=dev),
         _rows(B, md, "B", R, gn, dev=dev), _rows(C_, md, "C", R, gn, dev=dev),
         _rows(z, md, "z", R, d.d, optional=True, dev=dev)]
    s = ScanInputs(*[p for p, _ in r], *[ld for _, ld in r], _table(A, f32, "A", (d.n, d.d), dev=dev),
                   _table(D, f32, "D", (d.d,), True, dev=dev),
                   _table(delta_bias, f32, "delta_bias", (d.d,), True, dev=dev))
    s.rows, s.dims = R, (d.d, d.n, d.groups, d.dtype)
    s.tensors, s.device = (x, delta, A, B, C_, D, z, delta_bias), dev
    return s


def scan_grads(d: ScanDims, dx, ddelta, dA, dB, dC, dD=None, dz=None, ddelta_bias=None) -> ScanGrads:
    dev = _device()
    f32, R, gn = torch.float32, int(dx.shape[0]), d.groups * d.n
    r = [_rows(dx, f32, "dx", R, d.d, dev=dev), _rows(ddelta, f32, "ddelta", R, d.d, dev=dev),
         _rows(dB, f32, "dB", R, gn, dev=dev), _rows(dC, f32, "dC", R, gn, dev=dev),
         _rows(dz, f32, "dz", R, d.d, optional=True, dev=dev)]
    s = ScanGrads(*[p for p, _ in r], *[ld for _, ld in r], _table(dA, f32, "dA", (d.n, d.d), dev=dev),
                  _table(dD, f32, "dD", (d.d,), True, dev=dev),
                  _table(ddelta_bias, f32, "ddelta_bias", (d.d,), True, dev=dev))
    s.rows, s.dims = R, (d.d, d.n, d.groups, d.dtype)
    s.tensors, s.device = (dx, ddelta, dA, dB, dC, dD, dz, ddelta_bias), dev
    return s


def _fit(what, d, rows, name, dev):
    """The tensors were checked against the dims of this call, and have its rows."""
    if what.dims != (d.d, d.n, d.groups, d.dtype):
        raise MtgnnError(f"{name} were made for (d, n, groups, dtype) = {what.dims}")
    if what.rows < rows:
        raise MtgnnError(f"{name} have {what.rows} rows, the sequences {rows}")
    _made_here(what, name, dev)


def mtgnn_selective_scan(q: Seqs, inp: ScanInputs, d: ScanDims, state_in, state_out, y, save=None, ws=None,
                         stream=None):
    dev = _device()
    _fit(inp, d, q.max_rows, "the scan's inputs", dev)
    _made_here(q, "seqs", dev)
    yp, ldy = _rows(y, _DT[d.dtype], "y", q.max_rows, d.d, dev=dev)
    st, f32 = (q.n_slots, d.n, d.d), torch.float32
    need = selective_scan_save_bytes(d, q.max_rows, q.max_seq, state_in is not None)
    wp, wb = _work(ws, dev)
    _check(lib().mtgnn_selective_scan(C.byref(q), C.byref(inp), C.byref(d),
                                      _table(state_in, f32, "state_in", st, True, dev=dev),
                                      _table(state_out, f32, "state_out", st, True, dev=dev), yp, ldy,
                                      _bytes(save, need, "save", True, dev=dev), wp, wb, _stream(stream)),
           "mtgnn_selective_scan")


def mtgnn_selective_scan_bwd(q: Seqs, dy, inp: ScanInputs, d: ScanDims, save, grads: ScanGrads, ws, stream=None):
    dev = _device()
    _fit(inp, d, q.max_rows, "the scan's inputs", dev)
    _fit(grads, d, q.max_rows, "the scan's gradients", dev)
    _made_here(q, "seqs", dev)
    gp, lddy = _rows(dy, torch.float32, "dy", q.max_rows, d.d, dev=dev)
    need = selective_scan_save_bytes(d, q.max_rows, q.max_seq, False)
    wp, wb = _work(ws, dev)
    _check(lib().mtgnn_selective_scan_bwd(C.byref(q), gp, lddy, C.byref(inp), C.byref(d),
                                          _bytes(save, need, "save", dev=dev), C.byref(grads), wp, wb,
                                          _stream(stream)), "mtgnn_selective_scan_bwd")


def mtgnn_selective_scan_step(slot, inp: ScanInputs, d: ScanDims, state_in, state_out, y, n_rows=None, stream=None):
    """One row each: row r of the inputs is the next row of slot[r] (None: slot r)."""
    dev = _device()
    R, f32 = inp.rows, torch.float32
    _fit(inp, d, R, "the scan's inputs", dev)
    yp, ldy = _rows(y, _DT[d.dtype], "y", R, d.d, dev=dev)
    n = _n_slots(state_in, state_out)
    st = (n, d.n, d.d)
    _check(lib().mtgnn_selective_scan_step(_count(slot, R, "slot", dev=dev), _count(n_rows, 1, "n_rows", dev=dev), R, n,
                                           C.byref(inp), C.byref(d), _table(state_in, f32, "state_in", st, True, dev=dev),
                                           _table(state_out, f32, "state_out", st, True, dev=dev), yp, ldy, _stream(stream)),
           "mtgnn_selective_scan_step")


# ----------------------------------------------------------------------------- a model over all nodes

def embedding_dims(n, d, dtype=F32, scale=1.0) -> EmbeddingDims:
    return EmbeddingDims(int(n), int(d), int(dtype), float(scale))


def norm_dims(d, dtype=F32, eps=1e-5) -> NormDims:
    return NormDims(int(d), int(dtype), float(eps))


def loss_dims(n, d, dtype=F32) -> LossDims:
    """n classes, rows of width d."""
    return LossDims(int(n), int(d), int(dtype))


def embedding_ws_bytes(d: EmbeddingDims, max_rows) -> int:
    return int(lib().mtgnn_embedding_ws_bytes(C.byref(d), int(max_rows)))


def layer_norm_ws_bytes(d: NormDims, max_rows) -> int:
    return int(lib().mtgnn_layer_norm_ws_bytes(C.byref(d), int(max_rows)))


def softmax_loss_save_bytes(d: LossDims, max_rows) -> int:
    return int(lib().mtgnn_softmax_loss_save_bytes(C.byref(d), int(max_rows)))


def softmax_loss_ws_bytes(d: LossDims, max_rows, backward=False) -> int:
    return int(lib().mtgnn_softmax_loss_ws_bytes(C.byref(d), int(max_rows), int(backward)))


def _ids(t, name, dev):
    if t is None or t.dim() != 1:
        raise MtgnnError(f"{name} must be a vector of int32")
    return _count(t, 0, name, dev=dev), int(t.shape[0])


def mtgnn_embedding(ids, table, d: EmbeddingDims, y, n_rows=None, stream=None):
    """y[r] = scale table[ids[r]], zeros for an id outside the table."""
    dev = _device()
    md = _DT[d.dtype]
    ip, R = _ids(ids, "ids", dev)
    yp, ldy = _rows(y, md, "y", R, d.d, dev=dev)
    _check(lib().mtgnn_embedding(ip, _count(n_rows, 1, "n_rows", dev=dev), R, _table(table, md, "table", (d.n, d.d), dev=dev),
                                 C.byref(d), yp, ldy, _stream(stream)), "mtgnn_embedding")


def mtgnn_embedding_bwd(ids, dy, d: EmbeddingDims, dtable, ws, n_rows=None, stream=None):
    dev = _device()
    f32 = torch.float32
    ip, R = _ids(ids, "ids", dev)
    gp, lddy = _rows(dy, f32, "dy", R, d.d, dev=dev)
    wp, wb = _work(ws, dev)
    _check(lib().mtgnn_embedding_bwd(ip, _count(n_rows, 1, "n_rows", dev=dev), R, gp, lddy, C.byref(d),
                                     _table(dtable, f32, "dtable", (d.n, d.d), dev=dev), wp, wb, _stream(stream)),
           "mtgnn_embedding_bwd")


def mtgnn_layer_norm(x, gamma, beta, d: NormDims, y, stats=None, n_rows=None, stream=None):
    """Each row normed; stats [rows, 2]: where the backward will find the rows' means and scales."""
    dev = _device()
    md, R, f32 = _DT[d.dtype], int(x.shape[0]), torch.float32
    xp, ldx = _rows(x, md, "x", R, d.d, dev=dev)
    yp, ldy = _rows(y, md, "y", R, d.d, dev=dev)
    _check(lib().mtgnn_layer_norm(xp, ldx, _count(n_rows, 1, "n_rows", dev=dev), R,
                                  _table(gamma, f32, "gamma", (d.d,), True, dev=dev),
                                  _table(beta, f32, "beta", (d.d,), True, dev=dev), C.byref(d), yp, ldy,
                                  _table(stats, f32, "stats", (R, 2), True, dev=dev), _stream(stream)), "mtgnn_layer_norm")


def mtgnn_layer_norm_bwd(dy, x, gamma, stats, d: NormDims, dx, dgamma, dbeta, past=None, n_rows=None, ws=None, stream=None):
    """past: a gradient that reaches x beside the norm, added to dx."""
    dev = _device()
    md, R, f32 = _DT[d.dtype], int(x.shape[0]), torch.float32
    gp, lddy = _rows(dy, f32, "dy", R, d.d, dev=dev)
    xp, ldx = _rows(x, md, "x", R, d.d, dev=dev)
    pp, ldp = _rows(past, f32, "past", R, d.d, optional=True, dev=dev)
    dp, lddx = _rows(dx, f32, "dx", R, d.d, dev=dev)
    wp, wb = _work(ws, dev)
    _check(lib().mtgnn_layer_norm_bwd(gp, lddy, xp, ldx, _table(stats, f32, "stats", (R, 2), dev=dev),
                                      _count(n_rows, 1, "n_rows", dev=dev), R,
                                      _table(gamma, f32, "gamma", (d.d,), True, dev=dev), pp, ldp, C.byref(d), dp, lddx,
                                      _table(dgamma, f32, "dgamma", (d.d,), True, dev=dev),
                                      _table(dbeta, f32, "dbeta", (d.d,), True, dev=dev), wp, wb, _stream(stream)),
           "mtgnn_layer_norm_bwd")


def mtgnn_softmax_loss(x, W, b, label, d: LossDims, loss, ws, row_loss=None, save=None, n_rows=None, stream=None):
    """loss[0] = mean over the rows with a label of log sum exp(x W^T + b) - the label's."""
    dev = _device()
    md, R, f32 = _DT[d.dtype], int(x.shape[0]), torch.float32
    xp, ldx = _rows(x, md, "x", R, d.d, dev=dev)
    wp, wb = _work(ws, dev)
    _check(lib().mtgnn_softmax_loss(xp, ldx, _count(n_rows, 1, "n_rows", dev=dev), R, _table(W, md, "W", (d.n, d.d), dev=dev),
                                    _table(b, f32, "b", (d.n,), True, dev=dev),
                                    _table(label, torch.int32, "label", (R,), dev=dev), C.byref(d),
                                    _table(loss, f32, "loss", (1,), dev=dev),
                                    _table(row_loss, f32, "row_loss", (R,), True, dev=dev),
                                    _bytes(save, softmax_loss_save_bytes(d, R), "save", True, dev=dev), wp, wb,
                                    _stream(stream)), "mtgnn_softmax_loss")


def mtgnn_softmax_loss_bwd(x, W, b, label, d: LossDims, save, dx, dW, db, ws, dloss=None, n_rows=None, stream=None):
    """dx, dW, db (each or None) of the loss times dloss ([1] or None: 1).  Of x only the rows count: their values are in save."""
    dev = _device()
    md, R, f32 = _DT[d.dtype], int(x.shape[0]), torch.float32
    _rows(x, md, "x", R, d.d, dev=dev)
    dp, lddx = _rows(dx, f32, "dx", R, d.d, optional=True, dev=dev)
    wp, wb = _work(ws, dev)
    _check(lib().mtgnn_softmax_loss_bwd(_count(n_rows, 1, "n_rows", dev=dev), R, _table(W, md, "W", (d.n, d.d), dev=dev),
                                        _table(b, f32, "b", (d.n,), True, dev=dev),
                                        _table(label, torch.int32, "label", (R,), dev=dev), C.byref(d),
                                        _bytes(save, softmax_loss_save_bytes(d, R), "save", dev=dev),
                                        _table(dloss, f32, "dloss", (1,), True, dev=dev), dp, lddx,
                                        _table(dW, f32, "dW", (d.n, d.d), True, dev=dev),
                                        _table(db, f32, "db", (d.n,), True, dev=dev), wp, wb, _stream(stream)),
           "mtgnn_softmax_loss_bwd")


class AdamwTensors:
    """The tensors of mtgnn_adamw_step, described once: lists of as many dense tensors each.  shadow: None or a list of (None |
    bf16 tensor); decay: None or a list of numbers; m_exp, v_exp: None, or lists of (None | uint8 tensor of ceil(n / 32)),
    where given m and v hold 8-bit codes (uint8 or float8_e4m3fn).  It keeps its tensors."""

    def __init__(self, params, grads, m, v, shadow=None, decay=None, m_exp=None, v_exp=None):
        f32, n, dev = torch.float32, len(params), _device()
        none = [None] * n
        lists = dict(grads=grads, m=m, v=v, shadow=shadow or none, decay=decay or [0.0] * n, m_exp=m_exp or none,
                     v_exp=v_exp or none)
        for name, x in lists.items():
            if len(x) != n:
                raise MtgnnError(f"{name}: {len(x)} tensors for {n} parameters")
        self.array = (AdamwTensor * n)()
        for t, p, g, a, b, sh, de, ea, eb in zip(self.array, params, *lists.values()):
            shape, size, blocks = tuple(p.shape), int(p.numel()), -(-int(p.numel()) // 32)
            state = f32 if ea is None else a.dtype
            if ea is not None and (a.dtype not in (torch.uint8, torch.float8_e4m3fn) or b.dtype != a.dtype):
                raise MtgnnError(f"m and v must be uint8 or float8_e4m3fn beside exponents, got {a.dtype} and {b.dtype}")
            t.param, t.grad = (_table(x, f32, k, shape, dev=dev) for x, k in ((p, "param"), (g, "grad")))
            t.m, t.v = (_table(x, state, k, shape, dev=dev) for x, k in ((a, "m"), (b, "v")))
            t.m_exp, t.v_exp = (_table(x, torch.uint8, k, (blocks,), True, dev=dev) for x, k in ((ea, "m_exp"), (eb, "v_exp")))
            t.shadow = _table(sh, torch.bfloat16, "shadow", shape, True, dev=dev)
            t.n, t.decay = size, float(de)
        written = sorted((x.data_ptr(), x.numel() * x.element_size())
                         for x in (*params, *m, *v, *lists["shadow"], *lists["m_exp"], *lists["v_exp"]) if x is not None and x.numel())
        if any(a + size > b for (a, size), (b, _) in zip(written, written[1:])):
            raise MtgnnError("two of the tensors share memory (a parameter may be listed once)")
        for g in grads:   # (only read: two may be one)
            k = bisect.bisect_left(written, (g.data_ptr() + g.numel() * 4,)) - 1   # the last that starts before its end
            if g.numel() and k >= 0 and sum(written[k]) > g.data_ptr():
                raise MtgnnError("a gradient shares memory with a parameter or a state")
        self.tensors, self.device = (list(params), *(list(x) for x in lists.values())), dev


def adamw_tensors(params, grads, m, v, shadow=None, decay=None, m_exp=None, v_exp=None) -> AdamwTensors:
    return AdamwTensors(params, grads, m, v, shadow, decay, m_exp, v_exp)


def mtgnn_adamw_step(tensors: AdamwTensors, lr, beta1, beta2, eps, t, step=None, stream=None):
    """t: the step's number, or step: an int32 tensor on the device that holds it."""
    dev = _device()
    _made_here(tensors, "the tensors", dev)
    _check(lib().mtgnn_adamw_step(tensors.array, len(tensors.array), C.byref(AdamConfig(lr, beta1, beta2, eps, int(t))),
                                  _count(step, 1, "step", dev=dev), _stream(stream)), "mtgnn_adamw_step")


def timer_start(kernel: str, max_launches: int):
    """Arm the library's launch timer for `kernel` (instrumentation)."""
    _check(lib().mtgnn_timer_start(kernel.encode(), int(max_launches)), "mtgnn_timer_start")


def timer_stop():
    """Disarm the timer; returns (summed milliseconds, number of timed launches)."""
    ms, n = C.c_double(0.0), C.c_int(0)
    _check(lib().mtgnn_timer_stop(C.byref(ms), C.byref(n)), "mtgnn_timer_stop")
    return ms.value, n.value
