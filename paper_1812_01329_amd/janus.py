"""ctypes binding of libjanus.so (declared in include/janus.h).

Argument marshalling only: every function passes device pointers taken from
torch tensors (``tensor.data_ptr()``), host int32 arrays and the current HIP
stream to the C entry point of the same name, and raises ``JanusError`` on a
non-OK status.  Nothing here computes any part of the training step.

The shared library is loaded from the package directory; if it is missing
or fails to load, every call raises immediately (there is no fallback).
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libjanus.so")

OK, ERR_INVALID_ARG, ERR_LENGTH, ERR_TREE, ERR_TOKEN, ERR_WORKSPACE, ERR_UNSUPPORTED, ERR_DEVICE = range(8)
F32, BF16 = 0, 1
EMBED_FWD, XENT_FWD_BWD, EMBED_BWD = 0, 1, 2
LOSS_SUMSQ, LOSS_MEAN = 0, 1
CONV_LINEAR, CONV_SILU = 0, 1
SCAN_SOFTPLUS, SCAN_KEEP = 1, 2
ADAMW_F32, ADAMW_8BIT = 0, 1

EXPORTS = [
    "janus_lstm_workspace_bytes", "janus_lstm_seq_fwd", "janus_lstm_seq_bwd", "janus_lstm_device_report",
    "janus_lstm_fault_flag", "janus_lstm_schedule",
    "janus_treelstm_workspace_bytes", "janus_tree_schedule_build", "janus_treelstm_fwd",
    "janus_treelstm_bwd", "janus_treelstm_device_report", "janus_xent_workspace_bytes", "janus_embed_softmax_xent",
    "janus_mse_workspace_bytes", "janus_linear_mse", "janus_loss_reduce", "janus_trace_begin",
    "janus_trace_end", "janus_status_string", "janus_version", "janus_last_error",
    "janus_sgd_workspace_bytes", "janus_sgd_clip_update", "janus_sgd_clip_update_noalloc",
    "janus_lstm_state_carry",
    "janus_treernn_workspace_bytes", "janus_treernn_fwd", "janus_treernn_bwd", "janus_treernn_device_report",
    "janus_childsum_workspace_bytes", "janus_childsum_fwd", "janus_childsum_bwd", "janus_childsum_device_report",
    "janus_causal_conv_workspace_bytes", "janus_causal_conv_fwd", "janus_causal_conv_bwd", "janus_causal_conv_step",
    "janus_selective_scan_workspace_bytes", "janus_selective_scan_fwd", "janus_selective_scan_bwd",
    "janus_selective_scan_step", "janus_policy_workspace_bytes", "janus_policy_loss",
    "janus_layer_norm_workspace_bytes", "janus_layer_norm_fwd", "janus_layer_norm_bwd",
    "janus_sample_workspace_bytes", "janus_sample", "janus_adamw_workspace_bytes", "janus_adamw_update",
]


class JanusError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        self.detail = detail
        super().__init__(f"{where}: {status_string(status)} (status {status})" + (f": {detail}" if detail else ""))


class LstmDesc(C.Structure):
    _fields_ = [("L", C.c_int32), ("I", C.c_int32), ("H", C.c_int32), ("B", C.c_int32),
                ("T", C.c_int32), ("dtype", C.c_int)]


class TreeDesc(C.Structure):
    _fields_ = [("E", C.c_int32), ("H", C.c_int32), ("V", C.c_int32), ("dtype", C.c_int)]


class TreeBatchC(C.Structure):
    _fields_ = [("num_trees", C.c_int32), ("num_nodes", C.c_int32),
                ("left", C.POINTER(C.c_int32)), ("right", C.POINTER(C.c_int32)),
                ("word", C.POINTER(C.c_int32)), ("root", C.POINTER(C.c_int32))]


class NaryBatchC(C.Structure):
    _fields_ = [("num_trees", C.c_int32), ("num_nodes", C.c_int32),
                ("child_offsets", C.POINTER(C.c_int32)), ("children", C.POINTER(C.c_int32)),
                ("word", C.POINTER(C.c_int32)), ("root", C.POINTER(C.c_int32))]


class XentDesc(C.Structure):
    _fields_ = [("V", C.c_int32), ("H", C.c_int32), ("rows", C.c_int32), ("dtype", C.c_int)]


class TraceStat(C.Structure):
    _fields_ = [("label", C.c_char * 48), ("launches", C.c_int64), ("total_ms", C.c_double),
                ("flops", C.c_double), ("bytes", C.c_double)]


class LstmReport(C.Structure):
    _fields_ = [("timed_out", C.c_int32), ("bwd_groups", C.c_int32), ("bwd_local_groups", C.c_int32),
                ("fwd_groups", C.c_int32), ("fwd_local_groups", C.c_int32)]


class MseDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("H", C.c_int32), ("P", C.c_int32), ("dtype", C.c_int)]


class SgdDesc(C.Structure):
    _fields_ = [("n", C.c_int32), ("dtype", C.c_int), ("lr", C.c_float), ("max_norm", C.c_float)]


class ConvDesc(C.Structure):
    _fields_ = [("D", C.c_int32), ("K", C.c_int32), ("B", C.c_int32), ("T", C.c_int32), ("dtype", C.c_int),
                ("act", C.c_int), ("ldx", C.c_int64), ("ldy", C.c_int64)]


class ScanDesc(C.Structure):
    _fields_ = [("D", C.c_int32), ("N", C.c_int32), ("G", C.c_int32), ("B", C.c_int32), ("T", C.c_int32),
                ("dtype", C.c_int), ("flags", C.c_int32), ("ldx", C.c_int64), ("ldt", C.c_int64),
                ("ldb", C.c_int64), ("ldc", C.c_int64), ("ldz", C.c_int64), ("ldy", C.c_int64)]


class PolicyDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("V", C.c_int32), ("dtype", C.c_int), ("ld", C.c_int64),
                ("clip_low", C.c_float), ("clip_high", C.c_float), ("kl_coef", C.c_float), ("ent_coef", C.c_float)]


class NormDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int), ("eps", C.c_float), ("ldx", C.c_int64),
                ("ldh", C.c_int64), ("ldy", C.c_int64)]


class SampleDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("V", C.c_int32), ("dtype", C.c_int), ("ld", C.c_int64),
                ("temperature", C.c_float), ("top_k", C.c_int32), ("top_p", C.c_float), ("min_p", C.c_float)]


class AdamWDesc(C.Structure):
    _fields_ = [("n", C.c_int32), ("states", C.c_int), ("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float),
                ("eps", C.c_float), ("max_norm", C.c_float), ("seed", C.c_uint32)]


class AdamWTensor(C.Structure):
    _fields_ = [("p", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("scale", C.c_void_p),
                ("master", C.c_void_p), ("size", C.c_int64), ("decay", C.c_float), ("dtype", C.c_int)]


_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_1812_01329_amd.build`")
        # torch brings its own HIP runtime.  Loaded first, it is the one the
        # library binds to; loaded after the library, a second runtime would
        # come up beside the system one, and the library's launches would fail
        # (hipErrorNoDevice) on buffers torch allocated.
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        pi32 = C.POINTER(C.c_int32)
        L.janus_status_string.restype = C.c_char_p
        L.janus_status_string.argtypes = [C.c_int]
        L.janus_version.restype = C.c_char_p
        L.janus_last_error.restype = C.c_char_p
        L.janus_lstm_workspace_bytes.restype = sz
        L.janus_lstm_workspace_bytes.argtypes = [C.POINTER(LstmDesc)]
        L.janus_lstm_seq_fwd.argtypes = [C.POINTER(LstmDesc), vp, pi32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.janus_lstm_seq_bwd.argtypes = [C.POINTER(LstmDesc), vp, pi32, vp, vp, vp, sz, vp, vp, vp, vp, vp, vp,
                                         vp, vp, vp, vp]
        L.janus_lstm_schedule.argtypes = [i32, i32, pi32, pi32, pi32, pi32, pi32]
        L.janus_lstm_device_report.argtypes = [C.POINTER(LstmDesc), vp, sz, C.POINTER(LstmReport), vp]
        L.janus_lstm_fault_flag.argtypes = [C.POINTER(LstmDesc), vp, sz, C.POINTER(vp)]
        L.janus_treelstm_workspace_bytes.restype = sz
        L.janus_treelstm_workspace_bytes.argtypes = [C.POINTER(TreeDesc), i32, i32]
        L.janus_tree_schedule_build.argtypes = [C.POINTER(TreeBatchC), i32, pi32, pi32, pi32, pi32]
        L.janus_treelstm_fwd.argtypes = [C.POINTER(TreeDesc), C.POINTER(TreeBatchC), vp, vp, vp, vp, vp, vp, sz, vp]
        L.janus_treelstm_bwd.argtypes = [C.POINTER(TreeDesc), C.POINTER(TreeBatchC), vp, vp, vp, vp, sz, vp, vp, vp,
                                         vp, vp, vp]
        L.janus_treelstm_device_report.argtypes = [C.POINTER(TreeDesc), C.POINTER(TreeBatchC), vp, sz,
                                                   C.POINTER(i32), vp]
        L.janus_treernn_workspace_bytes.restype = sz
        L.janus_treernn_workspace_bytes.argtypes = [C.POINTER(TreeDesc), i32, i32]
        L.janus_treernn_fwd.argtypes = [C.POINTER(TreeDesc), C.POINTER(TreeBatchC), vp, vp, vp, vp, vp, sz, vp]
        L.janus_treernn_bwd.argtypes = [C.POINTER(TreeDesc), C.POINTER(TreeBatchC), vp, vp, sz, vp, vp, vp, vp, vp]
        L.janus_treernn_device_report.argtypes = [C.POINTER(TreeDesc), C.POINTER(TreeBatchC), vp, sz,
                                                  C.POINTER(i32), vp]
        L.janus_childsum_workspace_bytes.restype = sz
        L.janus_childsum_workspace_bytes.argtypes = [C.POINTER(TreeDesc), i32]
        L.janus_childsum_fwd.argtypes = [C.POINTER(TreeDesc), C.POINTER(NaryBatchC), vp, vp, vp, vp, vp, vp, sz, vp]
        L.janus_childsum_bwd.argtypes = [C.POINTER(TreeDesc), C.POINTER(NaryBatchC), vp, vp, vp, vp, sz, vp, vp, vp,
                                         vp, vp, vp]
        L.janus_childsum_device_report.argtypes = [C.POINTER(TreeDesc), C.POINTER(NaryBatchC), vp, sz,
                                                   C.POINTER(i32), vp]
        L.janus_xent_workspace_bytes.restype = sz
        L.janus_xent_workspace_bytes.argtypes = [C.POINTER(XentDesc), C.c_int]
        L.janus_embed_softmax_xent.argtypes = [C.POINTER(XentDesc), C.c_int, pi32, vp, vp, vp, vp, vp, vp, vp, vp,
                                               vp, sz, vp]
        L.janus_lstm_state_carry.argtypes = [C.POINTER(LstmDesc), i32, vp, vp, vp, vp, vp]
        L.janus_sgd_workspace_bytes.restype = sz
        L.janus_sgd_workspace_bytes.argtypes = [C.POINTER(SgdDesc)]
        L.janus_sgd_clip_update.argtypes = [C.POINTER(SgdDesc), C.POINTER(vp), C.POINTER(vp),
                                            C.POINTER(C.c_int64), vp, vp, vp, sz, vp]
        L.janus_sgd_clip_update_noalloc.argtypes = [C.POINTER(SgdDesc), C.POINTER(vp), C.POINTER(vp),
                                                    C.POINTER(C.c_int64), vp, vp, vp]
        L.janus_mse_workspace_bytes.restype = sz
        L.janus_mse_workspace_bytes.argtypes = [C.POINTER(MseDesc)]
        L.janus_linear_mse.argtypes = [C.POINTER(MseDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.janus_loss_reduce.argtypes = [C.c_int, vp, i64, vp, vp, vp]
        L.janus_causal_conv_workspace_bytes.restype = sz
        L.janus_causal_conv_workspace_bytes.argtypes = [C.POINTER(ConvDesc)]
        L.janus_causal_conv_fwd.argtypes = [C.POINTER(ConvDesc), vp, pi32, vp, vp, vp, vp, vp, vp]
        L.janus_causal_conv_bwd.argtypes = [C.POINTER(ConvDesc), vp, pi32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz,
                                            vp]
        L.janus_causal_conv_step.argtypes = [C.POINTER(ConvDesc), vp, vp, vp, vp, i32, vp, vp, vp]
        L.janus_selective_scan_workspace_bytes.restype = sz
        L.janus_selective_scan_workspace_bytes.argtypes = [C.POINTER(ScanDesc)]
        L.janus_selective_scan_fwd.argtypes = [C.POINTER(ScanDesc)] + [vp] * 8 + [pi32] + [vp] * 4 + [sz, vp]
        L.janus_selective_scan_bwd.argtypes = [C.POINTER(ScanDesc)] + [vp] * 8 + [pi32] + [vp] * 13 + [sz, vp]
        L.janus_selective_scan_step.argtypes = [C.POINTER(ScanDesc)] + [vp] * 9 + [i32, vp, vp, vp]
        L.janus_policy_workspace_bytes.restype = sz
        L.janus_policy_workspace_bytes.argtypes = [C.POINTER(PolicyDesc)]
        L.janus_policy_loss.argtypes = [C.POINTER(PolicyDesc)] + [vp] * 11 + [sz, vp]
        L.janus_layer_norm_workspace_bytes.restype = sz
        L.janus_layer_norm_workspace_bytes.argtypes = [C.POINTER(NormDesc)]
        L.janus_layer_norm_fwd.argtypes = [C.POINTER(NormDesc)] + [vp] * 9
        L.janus_layer_norm_bwd.argtypes = [C.POINTER(NormDesc)] + [vp] * 10 + [sz, vp]
        L.janus_sample_workspace_bytes.restype = sz
        L.janus_sample_workspace_bytes.argtypes = [C.POINTER(SampleDesc)]
        L.janus_sample.argtypes = [C.POINTER(SampleDesc)] + [vp] * 11 + [sz, vp]
        L.janus_adamw_workspace_bytes.restype = sz
        L.janus_adamw_workspace_bytes.argtypes = [C.POINTER(AdamWDesc)]
        L.janus_adamw_update.argtypes = [C.POINTER(AdamWDesc), C.POINTER(AdamWTensor)] + [vp] * 5 + [sz, vp]
        L.janus_trace_begin.argtypes = []
        L.janus_trace_end.argtypes = [C.POINTER(TraceStat), i32, C.POINTER(C.c_int32)]
        for name in EXPORTS:
            if name not in ("janus_status_string", "janus_version", "janus_last_error") and "workspace_bytes" not in name:
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().janus_status_string(status).decode()


def version() -> str:
    return lib().janus_version().decode()


# ---------------------------------------------------------------- helpers
def _p(t) -> Optional[int]:
    """Device pointer of a tensor (or None)."""
    return None if t is None else t.data_ptr()


def _stream(stream=None) -> Optional[int]:
    if stream is not None:
        return stream
    import torch
    # (the handle alone: a torch.cuda.Stream object costs more than the rest of a small call)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _stream_of(where: str, stream, *tensors) -> Optional[int]:
    """The given stream, or the current one, which the tensors (None aside) have
    to be on the device of: a kernel that got a host tensor's address would fault."""
    if stream is not None:
        return stream
    devices = {t.get_device() for t in tensors if t is not None}
    if -1 in devices:
        raise ValueError(f"{where}: a tensor is not on the GPU")
    import torch
    now = torch.cuda.current_device()
    if devices - {now}:
        raise ValueError(f"{where}: tensors on the devices {sorted(devices)}, the current device is {now}")
    return torch._C._cuda_getCurrentRawStream(now)


def _ptr_array(tensors: Sequence) -> C.Array:
    arr = (C.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = _p(t)
    return arr


def _i32(a) -> Optional[np.ndarray]:
    return None if a is None else np.ascontiguousarray(a, dtype=np.int32)


def _i32p(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.POINTER(C.c_int32))


def last_error() -> str:
    """Which HIP call failed behind the last DEVICE status on this thread."""
    return lib().janus_last_error().decode()


def _check(st: int, where: str):
    if st != OK:
        raise JanusError(st, where, last_error() if st == ERR_DEVICE else "")


def _tree_c(left, right, word, root):
    arrs = [_i32(a) for a in (left, right, word, root)]
    tb = TreeBatchC(len(arrs[3]), len(arrs[0]), *[_i32p(a) for a in arrs])
    return tb, arrs   # keep the arrays alive with the struct


# ---------------------------------------------------------------- LSTM
def janus_lstm_workspace_bytes(L, I, H, B, T, dtype) -> int:
    return int(lib().janus_lstm_workspace_bytes(C.byref(LstmDesc(L, I, H, B, T, dtype))))


def janus_lstm_seq_fwd(desc: LstmDesc, x, lengths, Wx, Wh, b, h0, c0, y, hT, cT, ws, stream=None):
    lens = _i32(lengths)
    st = lib().janus_lstm_seq_fwd(C.byref(desc), _p(x), _i32p(lens), _ptr_array(Wx), _ptr_array(Wh),
                                  _ptr_array(b), _p(h0), _p(c0), _p(y), _p(hT), _p(cT), _p(ws),
                                  ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "janus_lstm_seq_fwd")


def janus_lstm_seq_bwd(desc: LstmDesc, x, lengths, Wx, Wh, ws, dy, dhT, dcT, dx, dh0, dc0, dWx, dWh, db,
                       stream=None):
    lens = _i32(lengths)
    st = lib().janus_lstm_seq_bwd(C.byref(desc), _p(x), _i32p(lens), _ptr_array(Wx), _ptr_array(Wh), _p(ws),
                                  ws.numel() * ws.element_size(), _p(dy), _p(dhT), _p(dcT), _p(dx), _p(dh0),
                                  _p(dc0), _ptr_array(dWx), _ptr_array(dWh), _ptr_array(db), _stream(stream))
    _check(st, "janus_lstm_seq_bwd")


def janus_lstm_device_report(desc: LstmDesc, ws, stream=None) -> dict:
    """Synchronises the stream and returns the report of the current step on
    this workspace (the last forward and the backward after it); raises
    JanusError(DEVICE) if a barrier wait ran out."""
    rep = LstmReport()
    st = lib().janus_lstm_device_report(C.byref(desc), _p(ws), ws.numel() * ws.element_size(), C.byref(rep),
                                        _stream(stream))
    _check(st, "janus_lstm_device_report")
    return dict(timed_out=int(rep.timed_out), bwd_groups=int(rep.bwd_groups),
                bwd_local_groups=int(rep.bwd_local_groups), fwd_groups=int(rep.fwd_groups),
                fwd_local_groups=int(rep.fwd_local_groups))


def janus_lstm_fault_flag(desc: LstmDesc, ws) -> int:
    """Device address of the workspace's timeout word (see janus.h)."""
    out = C.c_void_p(0)
    st = lib().janus_lstm_fault_flag(C.byref(desc), _p(ws), ws.numel() * ws.element_size(), C.byref(out))
    _check(st, "janus_lstm_fault_flag")
    return int(out.value)


def janus_lstm_schedule(B: int, T: int, lengths):
    """Host-only schedule: returns (perm, active[T], offsets[T+1], t_eff)."""
    lens = _i32(lengths)
    perm = np.zeros(B, np.int32)
    active = np.zeros(max(T, 1), np.int32)
    offsets = np.zeros(T + 1, np.int32)
    t_eff = C.c_int32(0)
    st = lib().janus_lstm_schedule(B, T, _i32p(lens), _i32p(perm), _i32p(active), _i32p(offsets), C.byref(t_eff))
    _check(st, "janus_lstm_schedule")
    return perm, active[:T], offsets, int(t_eff.value)


# ---------------------------------------------------------------- TreeLSTM
def janus_treelstm_workspace_bytes(E, H, V, dtype, max_nodes, max_trees) -> int:
    return int(lib().janus_treelstm_workspace_bytes(C.byref(TreeDesc(E, H, V, dtype)), max_nodes, max_trees))


def janus_tree_schedule_build(left, right, word, root, V):
    """Host-only frontier schedule: returns (node_level, level_offsets, level_nodes, num_levels)."""
    tb, keep = _tree_c(left, right, word, root)
    N = tb.num_nodes
    level = np.zeros(max(N, 1), np.int32)
    offsets = np.zeros(N + 1, np.int32)
    nodes = np.zeros(max(N, 1), np.int32)
    L = C.c_int32(0)
    st = lib().janus_tree_schedule_build(C.byref(tb), V, _i32p(level), _i32p(offsets), _i32p(nodes), C.byref(L))
    _check(st, "janus_tree_schedule_build")
    L = int(L.value)
    return level[:N], offsets[:L + 1], nodes[:N], L


def janus_treelstm_fwd(desc: TreeDesc, trees, emb, W, U, b, h_root, ws, stream=None):
    tb, keep = _tree_c(trees.left, trees.right, trees.word, trees.root)
    st = lib().janus_treelstm_fwd(C.byref(desc), C.byref(tb), _p(emb), _p(W), _p(U), _p(b), _p(h_root), _p(ws),
                                  ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "janus_treelstm_fwd")


def janus_treelstm_bwd(desc: TreeDesc, trees, emb, W, U, ws, dh_root, demb, dW, dU, db, stream=None):
    tb, keep = _tree_c(trees.left, trees.right, trees.word, trees.root)
    st = lib().janus_treelstm_bwd(C.byref(desc), C.byref(tb), _p(emb), _p(W), _p(U), _p(ws),
                                  ws.numel() * ws.element_size(), _p(dh_root), _p(demb), _p(dW), _p(dU), _p(db),
                                  _stream(stream))
    _check(st, "janus_treelstm_bwd")


def janus_treelstm_device_report(desc: TreeDesc, trees, ws, stream=None) -> int:
    """Synchronises the stream and returns 1 if a level barrier of the last
    TreeLSTM forward or backward on this workspace ran out of its wait (the
    call then raises JanusError(DEVICE)), else 0."""
    tb, keep = _tree_c(trees.left, trees.right, trees.word, trees.root)
    out = C.c_int32(0)
    st = lib().janus_treelstm_device_report(C.byref(desc), C.byref(tb), _p(ws), ws.numel() * ws.element_size(),
                                            C.byref(out), _stream(stream))
    _check(st, "janus_treelstm_device_report")
    return int(out.value)


def janus_treernn_device_report(desc: TreeDesc, trees, ws, stream=None) -> int:
    """Synchronises the stream and returns 1 if a level barrier of the last
    TreeRNN forward or backward on this workspace ran out of its wait (the
    call then raises JanusError(DEVICE)), else 0."""
    tb, keep = _tree_c(trees.left, trees.right, trees.word, trees.root)
    out = C.c_int32(0)
    st = lib().janus_treernn_device_report(C.byref(desc), C.byref(tb), _p(ws), ws.numel() * ws.element_size(),
                                           C.byref(out), _stream(stream))
    _check(st, "janus_treernn_device_report")
    return int(out.value)


def janus_treernn_workspace_bytes(H, V, max_nodes, max_trees) -> int:
    return int(lib().janus_treernn_workspace_bytes(C.byref(TreeDesc(H, H, V, F32)), max_nodes, max_trees))


def janus_treernn_fwd(desc: TreeDesc, trees, emb, W, b, h_root, ws, stream=None):
    tb, keep = _tree_c(trees.left, trees.right, trees.word, trees.root)
    st = lib().janus_treernn_fwd(C.byref(desc), C.byref(tb), _p(emb), _p(W), _p(b), _p(h_root), _p(ws),
                                 ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "janus_treernn_fwd")


def janus_treernn_bwd(desc: TreeDesc, trees, W, ws, dh_root, demb, dW, db, stream=None):
    tb, keep = _tree_c(trees.left, trees.right, trees.word, trees.root)
    st = lib().janus_treernn_bwd(C.byref(desc), C.byref(tb), _p(W), _p(ws), ws.numel() * ws.element_size(),
                                 _p(dh_root), _p(demb), _p(dW), _p(db), _stream(stream))
    _check(st, "janus_treernn_bwd")


def _nary_c(trees):
    arrs = [np.ascontiguousarray(a, dtype=np.int32) for a in
            (trees.child_offsets, trees.children, trees.word, trees.root)]
    tb = NaryBatchC(len(arrs[3]), len(arrs[2]), *[_i32p(a) for a in arrs])
    return tb, arrs   # keep the arrays alive with the struct


def janus_childsum_workspace_bytes(E, H, V, max_nodes) -> int:
    return int(lib().janus_childsum_workspace_bytes(C.byref(TreeDesc(E, H, V, F32)), max_nodes))


def janus_childsum_fwd(desc: TreeDesc, trees, emb, W, U, b, h_root, ws, stream=None):
    tb, keep = _nary_c(trees)
    st = lib().janus_childsum_fwd(C.byref(desc), C.byref(tb), _p(emb), _p(W), _p(U), _p(b), _p(h_root), _p(ws),
                                  ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "janus_childsum_fwd")


def janus_childsum_bwd(desc: TreeDesc, trees, emb, W, U, ws, dh_root, demb, dW, dU, db, stream=None):
    tb, keep = _nary_c(trees)
    st = lib().janus_childsum_bwd(C.byref(desc), C.byref(tb), _p(emb), _p(W), _p(U), _p(ws),
                                  ws.numel() * ws.element_size(), _p(dh_root), _p(demb), _p(dW), _p(dU), _p(db),
                                  _stream(stream))
    _check(st, "janus_childsum_bwd")


def janus_childsum_device_report(desc: TreeDesc, trees, ws, stream=None) -> int:
    """Synchronises the stream and returns 1 if a level barrier of the last
    Child-Sum forward or backward on this workspace ran out of its wait (the
    call then raises JanusError(DEVICE)), else 0."""
    tb, keep = _nary_c(trees)
    out = C.c_int32(0)
    st = lib().janus_childsum_device_report(C.byref(desc), C.byref(tb), _p(ws), ws.numel() * ws.element_size(),
                                            C.byref(out), _stream(stream))
    _check(st, "janus_childsum_device_report")
    return int(out.value)


# ---------------------------------------------------------------- heads
def janus_xent_workspace_bytes(V, H, rows, dtype, op) -> int:
    return int(lib().janus_xent_workspace_bytes(C.byref(XentDesc(V, H, rows, dtype)), op))


def janus_embed_softmax_xent(desc: XentDesc, op, ids_host, ids_dev, table=None, bias=None, inp=None, out=None,
                             dtable=None, dbias=None, loss=None, ws=None, stream=None):
    ids = _i32(ids_host)
    st = lib().janus_embed_softmax_xent(C.byref(desc), op, _i32p(ids), _p(ids_dev), _p(table), _p(bias), _p(inp),
                                        _p(out), _p(dtable), _p(dbias), _p(loss), _p(ws),
                                        0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "janus_embed_softmax_xent")


def janus_mse_workspace_bytes(rows, H, P, dtype) -> int:
    return int(lib().janus_mse_workspace_bytes(C.byref(MseDesc(rows, H, P, dtype))))


def janus_linear_mse(desc: MseDesc, h, W, b, target, dh, dW, db, loss, ws, stream=None):
    st = lib().janus_linear_mse(C.byref(desc), _p(h), _p(W), _p(b), _p(target), _p(dh), _p(dW), _p(db), _p(loss),
                                _p(ws), ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "janus_linear_mse")


def janus_loss_reduce(kind, h, n, loss, dh, stream=None):
    st = lib().janus_loss_reduce(kind, _p(h), n, _p(loss), _p(dh), _stream(stream))
    _check(st, "janus_loss_reduce")


def janus_lstm_state_carry(desc: LstmDesc, B_prev: int, hT, cT, h0, c0, stream=None):
    """Initial state of the next batch (desc.B rows) from the final state of
    the previous one (B_prev rows)."""
    st = lib().janus_lstm_state_carry(C.byref(desc), int(B_prev), _p(hT), _p(cT), _p(h0), _p(c0), _stream(stream))
    _check(st, "janus_lstm_state_carry")


# ---------------------------------------------------------------- convolution and scan
def janus_causal_conv_workspace_bytes(desc: ConvDesc) -> int:
    return int(lib().janus_causal_conv_workspace_bytes(C.byref(desc)))


def janus_causal_conv_fwd(desc: ConvDesc, x, lengths, w, bias, s0, y, sT=None, stream=None):
    lens = _i32(lengths)
    st = lib().janus_causal_conv_fwd(C.byref(desc), _p(x), _i32p(lens), _p(w), _p(bias), _p(s0), _p(y), _p(sT),
                                     _stream(stream))
    _check(st, "janus_causal_conv_fwd")


def janus_causal_conv_bwd(desc: ConvDesc, x, lengths, w, bias, s0, dy, dsT, dx, dw, dbias, ds0, ws, stream=None):
    lens = _i32(lengths)
    st = lib().janus_causal_conv_bwd(C.byref(desc), _p(x), _i32p(lens), _p(w), _p(bias), _p(s0), _p(dy), _p(dsT),
                                     _p(dx), _p(dw), _p(dbias), _p(ds0), _p(ws), ws.numel() * ws.element_size(),
                                     _stream(stream))
    _check(st, "janus_causal_conv_bwd")


def janus_causal_conv_step(desc: ConvDesc, x, w, bias, state, y, slots=None, stream=None):
    """One token of desc.B sequences; ``state`` [n_slots, K-1, D] is updated
    in place, ``slots`` a device int32 tensor (None: row b has slot b)."""
    n_slots = desc.B if state is None else state.shape[0]
    st = lib().janus_causal_conv_step(C.byref(desc), _p(x), _p(w), _p(bias), _p(slots), n_slots, _p(state), _p(y),
                                      _stream(stream))
    _check(st, "janus_causal_conv_step")


def janus_selective_scan_workspace_bytes(desc: ScanDesc) -> int:
    return int(lib().janus_selective_scan_workspace_bytes(C.byref(desc)))


def janus_selective_scan_fwd(desc: ScanDesc, x, dt, A, Bm, Cm, lengths, y, ws=None, Dskip=None, z=None, dt_bias=None,
                             h0=None, hT=None, stream=None):
    lens = _i32(lengths)
    st = lib().janus_selective_scan_fwd(C.byref(desc), _p(x), _p(dt), _p(A), _p(Bm), _p(Cm), _p(Dskip), _p(z),
                                        _p(dt_bias), _i32p(lens), _p(h0), _p(y), _p(hT), _p(ws),
                                        0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "janus_selective_scan_fwd")


def janus_selective_scan_bwd(desc: ScanDesc, x, dt, A, Bm, Cm, lengths, dy, ws, dx, ddt, dA, dBm, dCm, Dskip=None,
                             z=None, dt_bias=None, h0=None, dhT=None, dDskip=None, dz=None, ddt_bias=None, dh0=None,
                             stream=None):
    lens = _i32(lengths)
    st = lib().janus_selective_scan_bwd(C.byref(desc), _p(x), _p(dt), _p(A), _p(Bm), _p(Cm), _p(Dskip), _p(z),
                                        _p(dt_bias), _i32p(lens), _p(h0), _p(dy), _p(dhT), _p(dx), _p(ddt), _p(dA),
                                        _p(dBm), _p(dCm), _p(dDskip), _p(dz), _p(ddt_bias), _p(dh0), _p(ws),
                                        ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "janus_selective_scan_bwd")


def janus_selective_scan_step(desc: ScanDesc, x, dt, A, Bm, Cm, state, y, Dskip=None, z=None, dt_bias=None,
                              slots=None, stream=None):
    """One token of desc.B sequences; ``state`` [n_slots, D, N] float32 is
    updated in place, ``slots`` as in janus_causal_conv_step."""
    st = lib().janus_selective_scan_step(C.byref(desc), _p(x), _p(dt), _p(A), _p(Bm), _p(Cm), _p(Dskip), _p(z),
                                         _p(dt_bias), _p(slots), state.shape[0], _p(state), _p(y), _stream(stream))
    _check(st, "janus_selective_scan_step")


# ---------------------------------------------------------------- policy loss
def janus_policy_workspace_bytes(desc: PolicyDesc) -> int:
    return int(lib().janus_policy_workspace_bytes(C.byref(desc)))


def janus_policy_loss(desc: PolicyDesc, logits, actions, old_logp=None, adv=None, ref_logp=None, weights=None,
                      dlogits=None, logp=None, entropy=None, stats=None, ws=None, stream=None):
    """Loss statistics and logits' gradient, or (without old_logp, adv and
    dlogits) only the rows' log-probabilities and entropies."""
    st = lib().janus_policy_loss(C.byref(desc), _p(logits), _p(actions), _p(old_logp), _p(adv), _p(ref_logp),
                                 _p(weights), _p(dlogits), _p(logp), _p(entropy), _p(stats), _p(ws),
                                 0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    _check(st, "janus_policy_loss")


# ---------------------------------------------------------------- layer norm
def janus_layer_norm_workspace_bytes(desc: NormDesc) -> int:
    return int(lib().janus_layer_norm_workspace_bytes(C.byref(desc)))


def janus_layer_norm_fwd(desc: NormDesc, x, gamma, beta, y, r=None, h=None, mean=None, rstd=None, stream=None):
    """y of the rows x, or of h = x + r with a residual ``r``; ``mean`` and
    ``rstd`` (and ``h``) are what the backward reads."""
    st = lib().janus_layer_norm_fwd(C.byref(desc), _p(x), _p(r), _p(gamma), _p(beta), _p(h), _p(y), _p(mean), _p(rstd),
                                    _stream_of("janus_layer_norm_fwd", stream, x, r, gamma, beta, h, y, mean, rstd))
    _check(st, "janus_layer_norm_fwd")


def janus_layer_norm_bwd(desc: NormDesc, h, gamma, mean, rstd, dy, dx, ws=None, dgamma=None, dbeta=None, dh=None,
                         stream=None):
    """``h``: the rows that were normalised (the forward's h, or its x without
    a residual); ``dh``: the gradient they have from elsewhere."""
    st = lib().janus_layer_norm_bwd(C.byref(desc), _p(h), _p(gamma), _p(mean), _p(rstd), _p(dy), _p(dh), _p(dx),
                                    _p(dgamma), _p(dbeta), _p(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                    _stream_of("janus_layer_norm_bwd", stream, h, gamma, mean, rstd, dy, dh, dx, dgamma, dbeta,
                                               ws))
    _check(st, "janus_layer_norm_bwd")


# ---------------------------------------------------------------- drawing tokens
def janus_sample_workspace_bytes(desc: SampleDesc) -> int:
    return int(lib().janus_sample_workspace_bytes(C.byref(desc)))


def janus_sample(desc: SampleDesc, logits, u, tokens, temperature=None, top_k=None, top_p=None, min_p=None, logp=None,
                 draw_logp=None, kept=None, ws=None, stream=None):
    """A token of each row by the uniform numbers ``u``; ``temperature``,
    ``top_k``, ``top_p`` and ``min_p``: device tensors with a setting a row, or
    None for the descriptor's."""
    st = lib().janus_sample(C.byref(desc), _p(logits), _p(u), _p(temperature), _p(top_k), _p(top_p), _p(min_p),
                            _p(tokens), _p(logp), _p(draw_logp), _p(kept), _p(ws),
                            0 if ws is None else ws.numel() * ws.element_size(),
                            _stream_of("janus_sample", stream, logits, u, temperature, top_k, top_p, min_p, tokens, logp,
                                       draw_logp, kept, ws))
    _check(st, "janus_sample")


# ---------------------------------------------------------------- update
def sgd_workspace_bytes(desc: SgdDesc) -> int:
    return int(lib().janus_sgd_workspace_bytes(C.byref(desc)))


def janus_sgd_clip_update(desc: SgdDesc, params, grads, stats=None, ws=None, stream=None, hold=None):
    """SGD step with global-norm clipping on lists of flat device tensors
    (parameters updated in place; float32 gradients).  ``hold``: a device
    address (int) of a uint32 that, when non-zero, keeps the update from
    writing anything (janus_lstm_fault_flag's word)."""
    n = len(params)
    S = (C.c_int64 * n)(*[int(t.numel()) for t in params])
    wsb = 0 if ws is None else ws.numel() * ws.element_size()
    st = lib().janus_sgd_clip_update(C.byref(desc), _ptr_array(params), _ptr_array(grads), S, _p(stats),
                                     None if hold is None else C.c_void_p(int(hold)), _p(ws), wsb, _stream(stream))
    _check(st, "janus_sgd_clip_update")


SGD_NOALLOC_MAX_TENSORS = 256   # JANUS_SGD_NOALLOC_MAX_TENSORS


def janus_sgd_clip_update_noalloc(desc: SgdDesc, params, grads, stats=None, stream=None, hold=None):
    """janus_sgd_clip_update without a workspace (the library's fixed
    per-device array; at most SGD_NOALLOC_MAX_TENSORS tensors)."""
    n = len(params)
    S = (C.c_int64 * n)(*[int(t.numel()) for t in params])
    st = lib().janus_sgd_clip_update_noalloc(C.byref(desc), _ptr_array(params), _ptr_array(grads), S, _p(stats),
                                             None if hold is None else C.c_void_p(int(hold)), _stream(stream))
    _check(st, "janus_sgd_clip_update_noalloc")


def adamw_tensors(params, grads, m, v, scale=None, master=None, decay=0.0) -> C.Array:
    """The tensors of janus_adamw_update, as it takes them: lists of device
    tensors (``scale`` of 8-bit states; ``master`` with None where a parameter has
    none), ``decay`` one number or one for each.  Made once for an update's every step.
    Raises ValueError where sizes or types do not go together."""
    import torch
    n = len(params)
    out = (AdamWTensor * n)()
    state = torch.float32 if scale is None else (torch.uint8, torch.float8_e4m3fn)
    for i in range(n):
        w = None if master is None else master[i]
        size, f32 = params[i].numel(), torch.float32
        for name, t, dts, least in (("p", params[i], (f32, torch.bfloat16), size), ("g", grads[i], f32, size), ("m", m[i], state, size),
                                    ("v", v[i], state, size), ("master", w, f32, size),
                                    ("scale", None if scale is None else scale[i], f32, -(-size // 256) * 2)):
            if t is not None and (t.numel() != least or not t.is_contiguous() or
                                  t.dtype not in (dts if isinstance(dts, tuple) else (dts,))):
                raise ValueError(f"adamw_tensors: {name} of tensor {i}: {t.dtype} {tuple(t.shape)} for {size} parameters")
        out[i] = AdamWTensor(_p(params[i]), _p(grads[i]), _p(m[i]), _p(v[i]), None if scale is None else _p(scale[i]), _p(w),
                             size, float(decay if np.isscalar(decay) else decay[i]),
                             BF16 if params[i].dtype == torch.bfloat16 else F32)
    out.tensors = [t for ts in (params, grads, m, v, scale or [], master or []) for t in ts if t is not None]   # (kept alive)
    devices = {t.get_device() for t in out.tensors}
    if len(devices) > 1:
        raise ValueError(f"adamw_tensors: tensors on the devices {sorted(devices)}")
    return out


def janus_adamw_workspace_bytes(desc: AdamWDesc) -> int:
    return int(lib().janus_adamw_workspace_bytes(C.byref(desc)))


def janus_adamw_update(desc: AdamWDesc, tensors: C.Array, step, lr=None, stats=None, ws=None, stream=None, hold=None):
    """One AdamW step on ``tensors`` (adamw_tensors); ``step`` an int64 device
    tensor that counts the steps taken, ``lr`` a float32 device tensor or None
    for the descriptor's, ``hold`` as in janus_sgd_clip_update."""
    st = lib().janus_adamw_update(C.byref(desc), tensors, _p(step), _p(lr), _p(stats),
                                  None if hold is None else C.c_void_p(int(hold)), _p(ws),
                                  0 if ws is None else ws.numel() * ws.element_size(),
                                  _stream_of("janus_adamw_update", stream, step, lr, stats, ws, *getattr(tensors, "tensors", ())[:1]))
    _check(st, "janus_adamw_update")


# ---------------------------------------------------------------- tracing
def janus_trace_begin():
    _check(lib().janus_trace_begin(), "janus_trace_begin")


def janus_trace_end(max_out: int = 128):
    """Per-label kernel statistics of the launches since janus_trace_begin."""
    out = (TraceStat * max_out)()
    n = C.c_int32(0)
    _check(lib().janus_trace_end(out, max_out, C.byref(n)), "janus_trace_end")
    return [dict(label=out[i].label.decode(), launches=int(out[i].launches), total_ms=float(out[i].total_ms),
                 flops=float(out[i].flops), bytes=float(out[i].bytes)) for i in range(min(n.value, max_out))]
