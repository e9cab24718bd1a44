"""ctypes binding of libtgm (include/tgm.h), function for function.

Argument marshalling only: device arrays are torch tensors on the GPU (passed
by data pointer), streams are torch streams.  Every computation happens in
the library's HIP kernels.  A missing library is an error, never a fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtgm.so")

TGM_OK, TGM_EINVAL, TGM_ERANGE, TGM_EORDER, TGM_ESIZE, TGM_EDEVICE, TGM_ENOMEM = \
    0, -1, -2, -3, -4, -5, -6
MAX_SAMPLE_SETS = 16                     # TGM_MAX_SAMPLE_SETS
MITIGATE_NOALLOC_MAX_NODES = 32768       # TGM_MITIGATE_NOALLOC_MAX_NODES

# Every exported symbol of include/tgm.h
SYMBOLS = ["tgm_status_str", "tgm_last_device_error", "tgm_version", "tgm_alloc_count",
           "tgm_graph_create",
           "tgm_graph_destroy", "tgm_graph_info", "tgm_batch_roots", "tgm_sample", "tgm_sample_batch",
           "tgm_node_set", "tgm_sample_nodes", "tgm_state_create", "tgm_state_destroy", "tgm_state_reset",
           "tgm_state_flush", "tgm_state_read", "tgm_state_load", "tgm_state_checkpoint_bytes",
           "tgm_state_save", "tgm_state_restore", "tgm_fetch_memory",
           "tgm_model_create", "tgm_model_destroy", "tgm_update_memory", "tgm_embed",
           "tgm_stage_run", "tgm_mitigator_create", "tgm_mitigator_destroy", "tgm_mitigate",
           "tgm_mitigator_read", "tgm_state_set_mitigation", "tgm_min_staleness",
           "tgm_mitigate_noalloc", "tgm_trainer_create", "tgm_trainer_destroy",
           "tgm_trainer_info", "tgm_trainer_read", "tgm_train_step", "tgm_state_set_training",
           "tgm_apan_create", "tgm_apan_destroy", "tgm_apan_step", "tgm_apan_flush",
           "tgm_apan_reset", "tgm_apan_load",
           "tgm_apan_read", "tgm_apan_fetched",
           "tgm_embed_projection",
           "tgm_norm", "tgm_norm_work_bytes", "tgm_norm_backward",
           "tgm_linear", "tgm_linear_work_bytes", "tgm_linear_backward",
           "tgm_scan", "tgm_scan_carry_rows", "tgm_scan_work_bytes", "tgm_scan_backward",
           "tgm_scan_step", "tgm_rotary", "tgm_rotary_frequencies",
           "tgm_decay_attn", "tgm_decay_attn_work_bytes", "tgm_decay_attn_backward",
           "tgm_decay_attn_step", "tgm_xent",
           "tgm_xent_work_bytes", "tgm_xent_backward",
           "tgm_profile_enable", "tgm_profile_reset", "tgm_profile_count", "tgm_profile_get"]


class TgmError(RuntimeError):
    def __init__(self, fn, code):
        self.code = code
        super().__init__(f"{fn}: {status_str(code)} ({code})")


class SampleBuffers(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in (
        "root", "root_ts", "nbr", "eid", "nts", "cnt", "nodes", "n_nodes", "root_pos", "nbr_pos")]


class FetchBuffers(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in ("mem", "mem_ts", "mail", "mail_ts", "ver")]


class ModelDesc(C.Structure):
    _fields_ = [("M", C.c_int32), ("D_e", C.c_int32), ("D_t", C.c_int32), ("H", C.c_int32),
                ("nb", C.c_int32), ("max_nodes", C.c_int32), ("max_roots", C.c_int32),
                ("kind", C.c_int32)]


TGM_MODEL_TGN, TGM_MODEL_JODIE = 0, 1
MODEL_KINDS = {"tgn": TGM_MODEL_TGN, "jodie": TGM_MODEL_JODIE}


_fp = C.POINTER(C.c_float)
_dp = C.POINTER(C.c_double)


class Weights(C.Structure):
    _fields_ = [("W_ih", _fp), ("W_hh", _fp), ("b_ih", _fp), ("b_hh", _fp),
                ("omega", _dp), ("beta", _dp),
                ("W_q", _fp), ("b_q", _fp), ("W_k", _fp), ("b_k", _fp), ("W_v", _fp),
                ("b_v", _fp), ("W_o", _fp), ("b_o", _fp), ("w_t", _fp)]


class ApanDesc(C.Structure):
    _fields_ = [("N", C.c_int32), ("M", C.c_int32), ("D_e", C.c_int32), ("D_t", C.c_int32),
                ("nb", C.c_int32), ("K_mb", C.c_int32), ("propagate", C.c_int32),
                ("s", C.c_int32), ("max_batch", C.c_int32), ("max_nodes", C.c_int32)]


class Predictor(C.Structure):
    _fields_ = [("W_src", _fp), ("W_dst", _fp), ("b_p", _fp), ("w_out", _fp),
                ("b_out", C.c_float)]


class Optimizer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("lr", C.c_float), ("beta1", C.c_float),
                ("beta2", C.c_float), ("eps", C.c_float)]


TGM_OPT_SGD, TGM_OPT_ADAM = 0, 1
OPTIMIZERS = {"sgd": TGM_OPT_SGD, "adam": TGM_OPT_ADAM}
N_PARAM_TENSORS = 17   # TGM_N_PARAM_TENSORS

class NormDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32),
                ("out_dtype", C.c_int32), ("eps", C.c_float), ("ld_x", C.c_int64),
                ("ld_res", C.c_int64), ("ld_total", C.c_int64), ("ld_y", C.c_int64)]


class LinearDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("N", C.c_int32), ("K", C.c_int32), ("dtype", C.c_int32),
                ("out_dtype", C.c_int32), ("act", C.c_int32), ("ld_x", C.c_int64),
                ("ld_w", C.c_int64), ("ld_res", C.c_int64), ("ld_z", C.c_int64),
                ("ld_y", C.c_int64), ("ld_dx", C.c_int64), ("ld_dw", C.c_int64)]


class ScanDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("S", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32),
                ("reverse", C.c_int32), ("ld_g", C.c_int64), ("ld_x", C.c_int64),
                ("ld_y", C.c_int64), ("ld_dg", C.c_int64), ("ld_dx", C.c_int64)]


class RotaryDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("H", C.c_int32), ("d", C.c_int32), ("rot", C.c_int32),
                ("dtype", C.c_int32), ("pos_type", C.c_int32), ("layout", C.c_int32),
                ("inverse", C.c_int32), ("amplitude", C.c_float), ("ld_x", C.c_int64),
                ("ld_y", C.c_int64)]


class DecayAttnDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("S", C.c_int32), ("H", C.c_int32), ("H_kv", C.c_int32),
                ("d_k", C.c_int32), ("d_v", C.c_int32), ("dtype", C.c_int32),
                ("reverse", C.c_int32), ("scale", C.c_float), ("ld_q", C.c_int64),
                ("ld_k", C.c_int64), ("ld_v", C.c_int64), ("ld_o", C.c_int64),
                ("ld_dq", C.c_int64), ("ld_dk", C.c_int64), ("ld_dv", C.c_int64)]


class XentDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("N", C.c_int32), ("K", C.c_int32), ("dtype", C.c_int32),
                ("ld_x", C.c_int64), ("ld_w", C.c_int64), ("ld_dx", C.c_int64),
                ("ld_dw", C.c_int64)]


TGM_F32, TGM_BF16, TGM_F16, TGM_E4M3 = 0, 1, 2, 3
TGM_ACT_NONE, TGM_ACT_RELU, TGM_ACT_SILU, TGM_ACT_GELU = 0, 1, 2, 3
ACTS = {"none": TGM_ACT_NONE, "relu": TGM_ACT_RELU, "silu": TGM_ACT_SILU, "gelu": TGM_ACT_GELU}
TGM_ROTARY_HALF, TGM_ROTARY_INTERLEAVED = 0, 1
ROTARY_LAYOUTS = {"half": TGM_ROTARY_HALF, "interleaved": TGM_ROTARY_INTERLEAVED}
TGM_POS_I32, TGM_POS_I64, TGM_POS_F64 = 0, 1, 2
TGM_ROTARY_PLAIN, TGM_ROTARY_LINEAR, TGM_ROTARY_BASE, TGM_ROTARY_PARTS = 0, 1, 2, 3
ROTARY_SCALINGS = {"none": TGM_ROTARY_PLAIN, "linear": TGM_ROTARY_LINEAR,
                   "base": TGM_ROTARY_BASE, "parts": TGM_ROTARY_PARTS}

_lib = None
V, I32, I64, P = C.c_void_p, C.c_int32, C.c_int64, C.c_void_p


def lib():
    """Load libtgm.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -c 'import __graft_entry__ as g; g.build()'`")
        L = C.CDLL(LIB_PATH)
        L.tgm_status_str.argtypes = [I32]
        L.tgm_status_str.restype = C.c_char_p
        L.tgm_last_device_error.restype = I32
        L.tgm_version.restype = I32
        sig = {
            "tgm_graph_create": [I32, I64, P, P, P, P, P, I32, V, C.POINTER(V)],
            "tgm_graph_destroy": [V],
            "tgm_graph_info": [V, P, P, P, P],
            "tgm_batch_roots": [V, I64, I32, P, P, V],
            "tgm_sample": [V, P, P, I32, I32, P, P, P, P, V],
            "tgm_sample_batch": [V, I64, I32, I32, P, P, P, P, P, P, V],
            "tgm_node_set": [V, P, I32, P, I32, P, P, I32, P, P, V],
            "tgm_sample_nodes": [V, I64, I32, I32, P, P, P, P, P, P, P, P, I32, P, P, V],
            "tgm_state_create": [I32, I32, I32, I32, I32, V, C.POINTER(V)],
            "tgm_state_destroy": [V],
            "tgm_state_reset": [V, V],
            "tgm_state_flush": [V, V],
            "tgm_state_read": [V, P, P, P, P, P, V],
            "tgm_state_load": [V, I64, P, P, P, P, P, V],
            "tgm_state_checkpoint_bytes": [V, C.POINTER(C.c_size_t)],
            "tgm_state_save": [V, P, C.c_size_t, V],
            "tgm_state_restore": [V, P, C.c_size_t, V],
            "tgm_fetch_memory": [V, I64, P, P, I32, P, P, P, P, P, V],
            "tgm_model_create": [C.POINTER(ModelDesc), C.POINTER(Weights), V, C.POINTER(V)],
            "tgm_model_destroy": [V],
            "tgm_update_memory": [V, V, V, I64, P, P, I32, P, P, P, P, P, I64, I32, P, P, P, P, P,
                                  V],
            "tgm_embed": [V, V, I32, I32, P, P, P, P, P, P, P, P, I32, P, V],
            "tgm_stage_run": [V, V, V, I64, I64, I32, I32, I32, C.POINTER(SampleBuffers), I32,
                              C.POINTER(FetchBuffers), P, P, P, P, P, P, V, V],
            "tgm_alloc_count": [C.POINTER(I64)],
            "tgm_trainer_create": [V, C.POINTER(Weights), C.POINTER(Predictor),
                                   C.POINTER(Optimizer), V, C.POINTER(V)],
            "tgm_trainer_destroy": [V],
            "tgm_trainer_info": [V, C.POINTER(I64), C.POINTER(I64), C.POINTER(I64)],
            "tgm_trainer_read": [V, P, P, P, V],
            "tgm_train_step": [V, V, V, I32, C.POINTER(SampleBuffers), C.POINTER(FetchBuffers),
                               P, P, I32, P, V],
            "tgm_state_set_training": [V, V, P, I64],
            "tgm_apan_create": [C.POINTER(ApanDesc), C.POINTER(Weights), V, C.POINTER(V)],
            "tgm_apan_destroy": [V],
            "tgm_apan_step": [V, V, I64, C.POINTER(SampleBuffers), I32, P, P, P, V],
            "tgm_apan_flush": [V, V],
            "tgm_apan_reset": [V, V],
            "tgm_apan_load": [V, I64, P, P, P, P, P, P, V],
            "tgm_apan_read": [V, P, P, P, P, P, P, V],
            "tgm_apan_fetched": [V, P, P, P, P, P, P, V],
            "tgm_mitigator_create": [I32, I32, I32, C.POINTER(V)],
            "tgm_mitigator_destroy": [V],
            "tgm_mitigate": [V, V, I64, P, P, I32, P, P, I32, C.c_double, C.c_float, V],
            "tgm_mitigate_noalloc": [V, I64, P, P, I32, P, P, I32, I32, I32, C.c_double,
                                     C.c_float, V],
            "tgm_mitigator_read": [V, P, P, P, P, V],
            "tgm_state_set_mitigation": [V, V, C.c_double, C.c_float],
            "tgm_min_staleness": [P, I64, I32, P, P, P, P, P],
            "tgm_embed_projection": [V, I32, P, P, P, P, P, I32, P, V],
            "tgm_linear_work_bytes": [I32, I32, I32, I32, I32, I32, C.POINTER(C.c_size_t)],
            "tgm_linear": [C.POINTER(LinearDesc), P, P, P, P, P, P, P, P, P, P, C.c_size_t, V],
            "tgm_linear_backward": [C.POINTER(LinearDesc), P, P, P, P, P, P, P, P, P,
                                    C.c_size_t, V],
            "tgm_scan": [C.POINTER(ScanDesc), P, P, P, P, P, P, P, P, P, C.c_size_t, V],
            "tgm_scan_carry_rows": [I64, I32, I32, C.POINTER(I64)],
            "tgm_scan_work_bytes": [I64, I32, I32, C.POINTER(C.c_size_t)],
            "tgm_scan_backward": [C.POINTER(ScanDesc), P, P, P, P, P, P, P, P, P, P, P, P,
                                  C.c_size_t, V],
            "tgm_scan_step": [C.POINTER(ScanDesc), P, P, P, P, P, P, V],
            "tgm_norm": [C.POINTER(NormDesc), P, P, P, P, P, P, P, V],
            "tgm_norm_work_bytes": [I32, I32, C.POINTER(C.c_size_t)],
            "tgm_norm_backward": [C.POINTER(NormDesc), P, P, P, P, P, P, P, P, C.c_size_t, V],
            "tgm_rotary": [C.POINTER(RotaryDesc), P, P, P, P, P, V],
            "tgm_rotary_frequencies": [I32, I32, C.c_double, C.c_double, C.c_double, C.c_double,
                                       C.c_double, P, C.POINTER(C.c_float)],
            "tgm_decay_attn_work_bytes": [I64, I32, I32, I32, I32, I32, I32, I32,
                                          C.POINTER(C.c_size_t)],
            "tgm_decay_attn": [C.POINTER(DecayAttnDesc), P, P, P, P, P, P, P, P, P, P, C.c_size_t,
                               V],
            "tgm_decay_attn_backward": [C.POINTER(DecayAttnDesc), P, P, P, P, P, P, P, P, P, P, P,
                                        P, P, P, C.c_size_t, V],
            "tgm_decay_attn_step": [C.POINTER(DecayAttnDesc), P, P, P, P, P, P, P, P, V],
            "tgm_xent_work_bytes": [I32, I32, I32, I32, I32, C.POINTER(C.c_size_t)],
            "tgm_xent": [C.POINTER(XentDesc), P, P, P, P, P, P, P, P, C.c_size_t, V],
            "tgm_xent_backward": [C.POINTER(XentDesc), P, P, P, P, P, P, P, P, P, P, P,
                                  C.c_size_t, V],
        }
        sig["tgm_profile_enable"] = [I32]
        sig["tgm_profile_reset"] = []
        sig["tgm_profile_count"] = []
        sig["tgm_profile_get"] = [I32, C.POINTER(C.c_char_p), C.POINTER(I64),
                                  C.POINTER(C.c_double)]
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = I32
        _lib = L
    return _lib


def status_str(code: int) -> str:
    return lib().tgm_status_str(int(code)).decode()


def _check(fn, rc):
    if rc != TGM_OK:
        raise TgmError(fn, rc)


def _p(t):
    """Device pointer of a tensor (None -> NULL)."""
    if t is None:
        return None
    return C.c_void_p(t.data_ptr())


def _s(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def last_device_error() -> int:
    return lib().tgm_last_device_error()


def version() -> int:
    return lib().tgm_version()


def tgm_profile_enable(on: bool):
    _check("tgm_profile_enable", lib().tgm_profile_enable(1 if on else 0))


def tgm_profile_reset():
    _check("tgm_profile_reset", lib().tgm_profile_reset())


def tgm_profile_read() -> dict:
    """{kernel name: (launches, total ms)}; synchronises the recorded events."""
    L = lib()
    out = {}
    for k in range(L.tgm_profile_count()):
        name, n, ms = C.c_char_p(), C.c_int64(), C.c_double()
        _check("tgm_profile_get", L.tgm_profile_get(k, C.byref(name), C.byref(n), C.byref(ms)))
        out[name.value.decode()] = (n.value, ms.value)
    return out


# ------------------------------------------------------------------ graph
def tgm_graph_create(N, src, dst, t, neg, efeat, stream=None):
    E = int(src.numel())
    D_e = 0 if efeat is None else int(efeat.shape[1])
    h = V()
    _check("tgm_graph_create", lib().tgm_graph_create(N, E, _p(src), _p(dst), _p(t), _p(neg),
                                                      _p(efeat), D_e, _s(stream), C.byref(h)))
    return h


def tgm_graph_destroy(g):
    _check("tgm_graph_destroy", lib().tgm_graph_destroy(g))


def tgm_graph_info(g):
    N, E, D_e, n_adj = C.c_int32(), C.c_int64(), C.c_int32(), C.c_int64()
    _check("tgm_graph_info", lib().tgm_graph_info(g, C.byref(N), C.byref(E), C.byref(D_e),
                                                  C.byref(n_adj)))
    return N.value, E.value, D_e.value, n_adj.value


def tgm_batch_roots(g, first_event, b, root, root_ts, stream=None):
    _check("tgm_batch_roots", lib().tgm_batch_roots(g, first_event, b, _p(root), _p(root_ts),
                                                    _s(stream)))


def tgm_sample(g, root, root_ts, R, nb, nbr, eid, nts, cnt, stream=None):
    _check("tgm_sample", lib().tgm_sample(g, _p(root), _p(root_ts), R, nb, _p(nbr), _p(eid),
                                          _p(nts), _p(cnt), _s(stream)))


def tgm_sample_batch(g, first_event, b, nb, root, root_ts, nbr, eid, nts, cnt, stream=None):
    _check("tgm_sample_batch", lib().tgm_sample_batch(g, first_event, b, nb, _p(root),
                                                      _p(root_ts), _p(nbr), _p(eid), _p(nts),
                                                      _p(cnt), _s(stream)))


def tgm_node_set(g, root, R, nbr, nb, nodes, n_nodes, cap, root_pos, nbr_pos, stream=None):
    _check("tgm_node_set", lib().tgm_node_set(g, _p(root), R, _p(nbr), nb, _p(nodes),
                                              _p(n_nodes), cap, _p(root_pos), _p(nbr_pos),
                                              _s(stream)))


def tgm_sample_nodes(g, first_event, b, nb, root, root_ts, nbr, eid, nts, cnt, nodes, n_nodes, cap,
                     root_pos, nbr_pos, stream=None):
    _check("tgm_sample_nodes", lib().tgm_sample_nodes(
        g, first_event, b, nb, _p(root), _p(root_ts), _p(nbr), _p(eid), _p(nts), _p(cnt),
        _p(nodes), _p(n_nodes), cap, _p(root_pos), _p(nbr_pos), _s(stream)))


# ------------------------------------------------------------------ state
def tgm_state_create(N, M, D_m, s, max_batch, stream=None):
    h = V()
    _check("tgm_state_create", lib().tgm_state_create(N, M, D_m, s, max_batch, _s(stream),
                                                      C.byref(h)))
    return h


def tgm_state_destroy(st):
    _check("tgm_state_destroy", lib().tgm_state_destroy(st))


def tgm_state_reset(st, stream=None):
    _check("tgm_state_reset", lib().tgm_state_reset(st, _s(stream)))


def tgm_state_flush(st, stream=None):
    _check("tgm_state_flush", lib().tgm_state_flush(st, _s(stream)))


def tgm_state_read(st, mem, mem_ts, mail, mail_ts, ver, stream=None):
    _check("tgm_state_read", lib().tgm_state_read(st, _p(mem), _p(mem_ts), _p(mail),
                                                  _p(mail_ts), _p(ver), _s(stream)))


def tgm_state_load(st, it, mem, mem_ts, mail, mail_ts, ver, stream=None):
    _check("tgm_state_load", lib().tgm_state_load(st, it, _p(mem), _p(mem_ts), _p(mail),
                                                  _p(mail_ts), _p(ver), _s(stream)))


def tgm_state_checkpoint_bytes(st) -> int:
    n = C.c_size_t(0)
    _check("tgm_state_checkpoint_bytes", lib().tgm_state_checkpoint_bytes(st, C.byref(n)))
    return n.value


def tgm_state_save(st, stream=None, nbytes=None):
    """The state's checkpoint as a host uint8 array (after the work already on
    `stream`; returns once it is copied)."""
    import numpy as np
    n = tgm_state_checkpoint_bytes(st) if nbytes is None else nbytes
    buf = np.zeros(n, dtype=np.uint8)
    _check("tgm_state_save", lib().tgm_state_save(st, buf.ctypes.data, n, _s(stream)))
    return buf


def tgm_state_restore(st, buf, stream=None):
    """Load a checkpoint (a contiguous host uint8 array) into st."""
    import numpy as np
    buf = np.ascontiguousarray(buf, dtype=np.uint8)
    _check("tgm_state_restore", lib().tgm_state_restore(st, buf.ctypes.data, buf.nbytes,
                                                        _s(stream)))


def tgm_fetch_memory(st, it, nodes, n_nodes, cap, mem, mem_ts, mail, mail_ts, ver, stream=None):
    _check("tgm_fetch_memory", lib().tgm_fetch_memory(st, it, _p(nodes), _p(n_nodes), cap,
                                                      _p(mem), _p(mem_ts), _p(mail), _p(mail_ts),
                                                      _p(ver), _s(stream)))


def buffers(struct, **tensors):
    """A SampleBuffers / FetchBuffers holding the device pointers of the named tensors."""
    return struct(*[tensors[f].data_ptr() for f, _ in struct._fields_])


def tgm_stage_run(g, st, m, i0, n, B, nb, cap, sample_bufs, fetch_bufs, mem_new, new_mem_ts,
                  winner, h, stream, prefetch_stream, h_trace=None, s_trace=None):
    """sample_bufs: a (SampleBuffers * nsb) array; fetch_bufs: a FetchBuffers;
    h_trace [n x 3B x M] and s_trace [n x cap x M] optional per-iteration
    copies of h and mem_new."""
    _check("tgm_stage_run", lib().tgm_stage_run(
        g, st, m, i0, n, B, nb, cap, sample_bufs, len(sample_bufs), C.byref(fetch_bufs),
        _p(mem_new), _p(new_mem_ts), _p(winner), _p(h), _p(h_trace), _p(s_trace), _s(stream),
        _s(prefetch_stream)))


def alloc_count() -> int:
    """Device allocations the library has made in this process so far."""
    c = I64()
    _check("tgm_alloc_count", lib().tgm_alloc_count(C.byref(c)))
    return int(c.value)


# ------------------------------------------------------------- mitigation
def tgm_mitigator_create(max_nodes, nb, K):
    h = V()
    _check("tgm_mitigator_create", lib().tgm_mitigator_create(max_nodes, nb, K, C.byref(h)))
    return h


def tgm_mitigator_destroy(mt):
    _check("tgm_mitigator_destroy", lib().tgm_mitigator_destroy(mt))


def tgm_mitigate(mt, g, first_event, nodes, n_nodes, cap, mem, mem_ts, M, p, lam, stream=None):
    _check("tgm_mitigate", lib().tgm_mitigate(mt, g, first_event, _p(nodes), _p(n_nodes), cap,
                                              _p(mem), _p(mem_ts), M, float(p), float(lam),
                                              _s(stream)))


def tgm_mitigate_noalloc(g, first_event, nodes, n_nodes, cap, mem, mem_ts, M, nb, K, p, lam,
                         stream=None):
    _check("tgm_mitigate_noalloc", lib().tgm_mitigate_noalloc(
        g, first_event, _p(nodes), _p(n_nodes), cap, _p(mem), _p(mem_ts), M, nb, K, float(p),
        float(lam), _s(stream)))


def tgm_mitigator_read(mt, gamma, n_stale, stale, omega, stream=None):
    _check("tgm_mitigator_read", lib().tgm_mitigator_read(mt, _p(gamma), _p(n_stale), _p(stale),
                                                          _p(omega), _s(stream)))


def tgm_state_set_mitigation(st, mt, p=1.0, lam=1.0):
    _check("tgm_state_set_mitigation", lib().tgm_state_set_mitigation(st, mt, float(p),
                                                                      float(lam)))


# ------------------------------------------------------------- staleness bound
def tgm_min_staleness(tau, n, k_max):
    """Host solver of the minimal-staleness bound: returns (k, fetch_start,
    stall, b, e) for iterations 1..n as numpy arrays (b, e: [n x 5])."""
    import numpy as np
    t = np.ascontiguousarray(tau, dtype=np.float64)
    if t.shape != (5,):
        raise ValueError("tau holds the five stage durations")
    n = int(n)
    k = np.zeros(max(n, 1), np.int32)
    fs, st = np.zeros(max(n, 1)), np.zeros(max(n, 1))
    b, e = np.zeros((max(n, 1), 5)), np.zeros((max(n, 1), 5))
    _check("tgm_min_staleness", lib().tgm_min_staleness(
        t.ctypes.data, n, int(k_max), k.ctypes.data, fs.ctypes.data, st.ctypes.data,
        b.ctypes.data, e.ctypes.data))
    return k[:n], fs[:n], st[:n], b[:n], e[:n]


# ------------------------------------------------------------------ model
def _weights_struct(w, keep):
    def arr(name, dt):
        v = getattr(w, name, None)
        if v is None:
            return None
        a = np.ascontiguousarray(v, dtype=dt)
        keep[name] = a
        return a.ctypes.data_as(_fp if dt == np.float32 else _dp)

    ws = Weights()
    for name in ("W_ih", "W_hh", "b_ih", "b_hh", "W_q", "b_q", "W_k", "b_k", "W_v", "b_v",
                 "W_o", "b_o", "w_t"):
        setattr(ws, name, arr(name, np.float32))
    ws.omega = arr("omega", np.float64)
    ws.beta = arr("beta", np.float64)
    return ws


def tgm_trainer_create(m, w, pred, opt="adam", lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8,
                       stream=None):
    """``w`` the model's numpy weights (workloads.Weights), ``pred`` a
    workloads.Predictor."""
    keep = {}
    ws = _weights_struct(w, keep)
    pa = {k: np.ascontiguousarray(getattr(pred, k), dtype=np.float32)
          for k in ("W_src", "W_dst", "b_p", "w_out")}
    ps = Predictor(*[pa[k].ctypes.data_as(_fp) for k in ("W_src", "W_dst", "b_p", "w_out")],
                   float(pred.b_out))
    os_ = Optimizer(OPTIMIZERS[opt], float(lr), float(beta1), float(beta2), float(eps))
    h = V()
    _check("tgm_trainer_create", lib().tgm_trainer_create(m, C.byref(ws), C.byref(ps),
                                                          C.byref(os_), _s(stream), C.byref(h)))
    return h


def tgm_apan_create(N, M, D_e, D_t, nb, K_mb, propagate, s, max_batch, max_nodes, w,
                    stream=None):
    """``w`` the APAN weights (workloads.make_weights(model='apan'))."""
    keep = {}
    ws = _weights_struct(w, keep)
    d = ApanDesc(N, M, D_e, D_t, nb, K_mb, 1 if propagate else 0, s, max_batch, max_nodes)
    h = V()
    _check("tgm_apan_create", lib().tgm_apan_create(C.byref(d), C.byref(ws), _s(stream),
                                                    C.byref(h)))
    return h


def tgm_apan_destroy(a):
    _check("tgm_apan_destroy", lib().tgm_apan_destroy(a))


def tgm_apan_step(a, g, it, sample_bufs, cap, mem_new, new_mem_ts, h, stream=None):
    _check("tgm_apan_step", lib().tgm_apan_step(a, g, it, C.byref(sample_bufs), cap,
                                                _p(mem_new), _p(new_mem_ts), _p(h),
                                                _s(stream)))


def tgm_apan_flush(a, stream=None):
    _check("tgm_apan_flush", lib().tgm_apan_flush(a, _s(stream)))


def tgm_apan_reset(a, stream=None):
    _check("tgm_apan_reset", lib().tgm_apan_reset(a, _s(stream)))


def tgm_apan_load(a, it, mem, mem_ts, ver, mb, mb_ts, mb_cnt, stream=None):
    _check("tgm_apan_load", lib().tgm_apan_load(a, it, _p(mem), _p(mem_ts), _p(ver), _p(mb),
                                                _p(mb_ts), _p(mb_cnt), _s(stream)))


def tgm_apan_read(a, mem=None, mem_ts=None, ver=None, mb=None, mb_ts=None, mb_cnt=None,
                  stream=None):
    _check("tgm_apan_read", lib().tgm_apan_read(a, _p(mem), _p(mem_ts), _p(ver), _p(mb),
                                                _p(mb_ts), _p(mb_cnt), _s(stream)))


def tgm_apan_fetched(a, mem=None, mem_ts=None, ver=None, mb=None, mb_ts=None, mb_cnt=None,
                     stream=None):
    _check("tgm_apan_fetched", lib().tgm_apan_fetched(a, _p(mem), _p(mem_ts), _p(ver), _p(mb),
                                                      _p(mb_ts), _p(mb_cnt), _s(stream)))


def tgm_trainer_destroy(tr):
    _check("tgm_trainer_destroy", lib().tgm_trainer_destroy(tr))


def tgm_trainer_info(tr):
    """(n_params, [sizes of the 17 tensors], optimizer steps taken)."""
    n, st = I64(), I64()
    sz = (I64 * N_PARAM_TENSORS)()
    _check("tgm_trainer_info", lib().tgm_trainer_info(tr, C.byref(n), sz, C.byref(st)))
    return int(n.value), [int(x) for x in sz], int(st.value)


def tgm_trainer_read(tr, params=None, grad=None, loss=None, stream=None):
    _check("tgm_trainer_read", lib().tgm_trainer_read(tr, _p(params), _p(grad), _p(loss),
                                                      _s(stream)))


def tgm_train_step(tr, m, g, b, sample_bufs, fetch_bufs, mem_new, h, cap, loss=None,
                   stream=None):
    _check("tgm_train_step", lib().tgm_train_step(tr, m, g, b, C.byref(sample_bufs),
                                                  C.byref(fetch_bufs), _p(mem_new), _p(h), cap,
                                                  _p(loss), _s(stream)))


def tgm_state_set_training(st, tr, loss_log=None):
    n = 0 if loss_log is None else int(loss_log.numel())
    _check("tgm_state_set_training", lib().tgm_state_set_training(st, tr, _p(loss_log), n))


def tgm_model_create(M, D_e, D_t, H, nb, max_nodes, max_roots, w, stream=None):
    """``w`` holds numpy weights (fp32; omega and beta fp64), see workloads.Weights."""
    kind = MODEL_KINDS[getattr(w, "kind", "tgn")]
    d = ModelDesc(M, D_e, D_t, H, nb, max_nodes, max_roots, kind)
    keep = {}

    def arr(name, dt):
        v = getattr(w, name, None)
        if v is None:
            return None
        a = np.ascontiguousarray(v, dtype=dt)
        keep[name] = a
        return a.ctypes.data_as(_fp if dt == np.float32 else _dp)

    ws = Weights()
    for name in ("W_ih", "W_hh", "b_ih", "b_hh", "W_q", "b_q", "W_k", "b_k", "W_v", "b_v",
                 "W_o", "b_o", "w_t"):
        setattr(ws, name, arr(name, np.float32))
    ws.omega = arr("omega", np.float64)
    ws.beta = arr("beta", np.float64)
    h = V()
    _check("tgm_model_create", lib().tgm_model_create(C.byref(d), C.byref(ws), _s(stream),
                                                      C.byref(h)))
    return h


def tgm_model_destroy(m):
    _check("tgm_model_destroy", lib().tgm_model_destroy(m))


def tgm_update_memory(st, m, g, it, nodes, n_nodes, cap, mem, mem_ts, mail, mail_ts, ver,
                      first_event, b, src_pos, dst_pos, mem_new, new_mem_ts=None, winner=None,
                      stream=None):
    _check("tgm_update_memory", lib().tgm_update_memory(
        st, m, g, it, _p(nodes), _p(n_nodes), cap, _p(mem), _p(mem_ts), _p(mail), _p(mail_ts),
        _p(ver), first_event, b, _p(src_pos), _p(dst_pos), _p(mem_new), _p(new_mem_ts),
        _p(winner), _s(stream)))


def tgm_embed_projection(m, R, root_pos, root_ts, mem_new, new_mem_ts, n_nodes, cap, h,
                         stream=None):
    _check("tgm_embed_projection", lib().tgm_embed_projection(
        m, R, _p(root_pos), _p(root_ts), _p(mem_new), _p(new_mem_ts), _p(n_nodes), cap, _p(h),
        _s(stream)))


def tgm_embed(m, g, R, nb, root_pos, root_ts, nbr_pos, eid, nts, cnt, mem_new, n_nodes, cap, h,
              stream=None):
    _check("tgm_embed", lib().tgm_embed(m, g, R, nb, _p(root_pos), _p(root_ts), _p(nbr_pos),
                                        _p(eid), _p(nts), _p(cnt), _p(mem_new), _p(n_nodes), cap,
                                        _p(h), _s(stream)))


# ------------------------------------------------------------------ sequence operators
_codes = {}   # torch types to TGM_F32, ...


def dtype_code(dtype) -> int:
    """TGM_F32, ... of a torch type."""
    if not _codes:
        import torch
        _codes.update({torch.float32: TGM_F32, torch.bfloat16: TGM_BF16, torch.float16: TGM_F16,
                       torch.float8_e4m3fn: TGM_E4M3})
    code = _codes.get(dtype)
    if code is None:
        raise ValueError(f"no operator takes {dtype}")
    return code


def _arg(name, t, dtype, shape, gpu):
    """Check a tensor argument and return (address, row stride).  ``gpu`` is the
    index of the device of the call's tensors.  The stride is 0 where there is no
    second row for it to lead to."""
    # a call costs a few us in all: the usual argument by one test
    if t is not None and t.dtype is dtype and t.shape == shape and t.get_device() == gpu >= 0 \
            and t.is_contiguous():
        return t.data_ptr(), shape[1] if len(shape) == 2 and shape[0] > 1 else 0
    if t is None:
        raise ValueError(f"{name} is missing")
    if t.dtype is not dtype:
        raise ValueError(f"{name} has type {t.dtype}, not {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    ld = 0
    if len(shape) == 2:
        ld, step = t.stride()
        if t.numel():
            if step != 1 and shape[1] > 1:
                raise ValueError(f"{name}'s columns are not contiguous")
            if shape[0] > 1 and ld < shape[1]:
                raise ValueError(f"{name}'s rows overlap (stride {ld}, width {shape[1]})")
        if shape[0] <= 1:
            ld = 0
    elif not t.is_contiguous():
        raise ValueError(f"{name} is not contiguous")
    if gpu < 0 or t.get_device() != gpu:
        raise ValueError(f"{name} is on {t.device}: every tensor of a call is on one GPU")
    return t.data_ptr(), ld


def _opt(name, t, dtype, shape, gpu):
    return (None, 0) if t is None else _arg(name, t, dtype, shape, gpu)


def _dense(name, t, dtype, shape, gpu):
    """Address of an optional tensor without gaps between its rows."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError(f"{name} is not contiguous")
    return _arg(name, t, dtype, shape, gpu)[0]


def _work_arg(work, gpu):
    import torch
    if work is None:
        return None, 0
    if work.get_device() != gpu or work.dtype is not torch.uint8 or not work.is_contiguous():
        raise ValueError("work is a contiguous uint8 tensor on the call's GPU")
    return work.data_ptr(), work.numel()


def _call(fn, gpu, stream, *args):
    """fn(*args, stream) with the tensors' device current."""
    import torch
    if gpu < 0:
        raise ValueError(f"{fn}: the operators run on a GPU")
    if stream is None:
        # the address alone: a Stream object takes ten times as long to make
        s = torch._C._cuda_getCurrentRawStream(gpu)
    elif stream.device_index != gpu:
        raise ValueError(f"{fn}: a stream of {stream.device} for tensors on cuda:{gpu}")
    else:
        s = stream.cuda_stream
    f = getattr(lib(), fn)
    if torch.cuda.current_device() == gpu:
        rc = f(*args, s)
    else:
        with torch.cuda.device(gpu):
            rc = f(*args, s)
    if rc:
        _check(fn, rc)


def _sizes(fn, args, types):
    """Refuse whole numbers that the C types would cut short."""
    for v, t in zip(args, types):
        if t(v).value != v:
            raise ValueError(f"{fn}: {v} is out of range")


def _bytes(fn, *args) -> int:
    _sizes(fn, args, getattr(lib(), fn).argtypes)
    n = C.c_size_t(0)
    _check(fn, getattr(lib(), fn)(*args, C.byref(n)))
    return int(n.value)


def _shape2(name, t):
    if t is None or t.dim() != 2:
        raise ValueError(f"{name} is a matrix")
    shape = rows, columns = tuple(t.shape)
    if rows >= 1 << 31 or columns >= 1 << 31:
        raise ValueError(f"{name} has too many rows or columns: {shape}")
    return shape


def tgm_norm(x, w, y, eps, res=None, total=None, scale=None, n_rows=None, stream=None):
    """y = t / rms(t) * w with t = x + res; ``y`` of x's type, or float8_e4m3fn
    with ``scale`` [rows] fp32; ``total`` receives t."""
    import torch
    rows, D = _shape2("x", x)
    gpu, dt = x.get_device(), x.dtype
    out = y.dtype if y is not None and y.dtype == torch.float8_e4m3fn else dt
    px, lx = _arg("x", x, dt, (rows, D), gpu)
    pr, lr = _opt("res", res, dt, (rows, D), gpu)
    pw, _ = _arg("w", w, dt, (D,), gpu)
    pt, lt = _opt("total", total, dt, (rows, D), gpu)
    py, ly = _arg("y", y, out, (rows, D), gpu)
    ps, _ = _opt("scale", scale, torch.float32, (rows,), gpu)
    pn, _ = _opt("n_rows", n_rows, torch.int32, (1,), gpu)
    d = NormDesc(rows, D, dtype_code(dt), dtype_code(out), eps, lx, lr, lt, ly)
    _call("tgm_norm", gpu, stream, C.byref(d), px, pr, pw, pn, pt, py, ps)


def tgm_norm_work_bytes(rows, D) -> int:
    return _bytes("tgm_norm_work_bytes", rows, D)


def tgm_norm_backward(t, w, dy, eps, dx, dw, work, dtotal=None, n_rows=None, stream=None):
    import torch
    rows, D = _shape2("t", t)
    gpu, dt = t.get_device(), t.dtype
    px, lx = _arg("t", t, dt, (rows, D), gpu)
    pw, _ = _arg("w", w, dt, (D,), gpu)
    py, ly = _arg("dy", dy, dt, (rows, D), gpu)
    pd, ld = _opt("dtotal", dtotal, dt, (rows, D), gpu)
    po, lo = _arg("dx", dx, dt, (rows, D), gpu)
    pg, _ = _opt("dw", dw, dt, (D,), gpu)
    pn, _ = _opt("n_rows", n_rows, torch.int32, (1,), gpu)
    pk, nk = _work_arg(work, gpu)
    d = NormDesc(rows, D, dtype_code(dt), dtype_code(dt), eps, lx, ld, lo, ly)
    _call("tgm_norm_backward", gpu, stream, C.byref(d), px, pw, py, pd, pn, po, pg, pk, nk)


def _act(name) -> int:
    if name not in ACTS:
        raise ValueError(f"act is one of {sorted(ACTS)}, not {name!r}")
    return ACTS[name]


def tgm_linear_work_bytes(rows, N, K, dtype, act="none", backward=False) -> int:
    return _bytes("tgm_linear_work_bytes", rows, N, K, dtype_code(dtype), _act(act),
                  1 if backward else 0)


def tgm_linear(x, w, y, work, act="none", bias=None, residual=None, z=None, scale_x=None,
               scale_w=None, n_rows=None, stream=None):
    """y = act(x w^T + bias) + residual; float8_e4m3fn x and w with ``scale_x``
    [rows] and ``scale_w`` [N]; ``z`` receives the pre-activation."""
    import torch
    (rows, K), (N, _), out = _shape2("x", x), _shape2("w", w), None if y is None else y.dtype
    gpu, dt = x.get_device(), x.dtype
    px, lx = _arg("x", x, dt, (rows, K), gpu)
    pw, lw = _arg("w", w, dt, (N, K), gpu)
    psx, _ = _opt("scale_x", scale_x, torch.float32, (rows,), gpu)
    psw, _ = _opt("scale_w", scale_w, torch.float32, (N,), gpu)
    pb, _ = _opt("bias", bias, out, (N,), gpu)
    pr, lr = _opt("residual", residual, out, (rows, N), gpu)
    pz, lz = _opt("z", z, out, (rows, N), gpu)
    py, ly = _arg("y", y, out, (rows, N), gpu)
    pn, _ = _opt("n_rows", n_rows, torch.int32, (1,), gpu)
    pk, nk = _work_arg(work, gpu)
    d = LinearDesc(rows, N, K, dtype_code(dt), dtype_code(out), _act(act), lx, lw, lr, lz, ly, 0,
                   0)
    _call("tgm_linear", gpu, stream, C.byref(d), px, psx, pw, psw, pb, pr, pn, pz, py, pk, nk)


def tgm_linear_backward(x, w, dy, work, act="none", z=None, dx=None, dw=None, db=None,
                        n_rows=None, stream=None):
    """dx, dw and db (each optional) from dy and, unless act is none, the ``z``
    that tgm_linear wrote."""
    import torch
    (rows, K), (N, _) = _shape2("x", x), _shape2("w", w)
    gpu, dt = x.get_device(), x.dtype
    px, lx = _arg("x", x, dt, (rows, K), gpu)
    pw, lw = _arg("w", w, dt, (N, K), gpu)
    pz, lz = _opt("z", z, dt, (rows, N), gpu)
    py, ly = _arg("dy", dy, dt, (rows, N), gpu)
    pdx, ldx = _opt("dx", dx, dt, (rows, K), gpu)
    pdw, ldw = _opt("dw", dw, dt, (N, K), gpu)
    pdb, _ = _opt("db", db, dt, (N,), gpu)
    pn, _ = _opt("n_rows", n_rows, torch.int32, (1,), gpu)
    pk, nk = _work_arg(work, gpu)
    d = LinearDesc(rows, N, K, dtype_code(dt), dtype_code(dt), _act(act), lx, lw, 0, lz, ly, ldx,
                   ldw)
    _call("tgm_linear_backward", gpu, stream, C.byref(d), px, pw, pz, py, pn, pdx, pdw, pdb, pk,
          nk)


def tgm_scan_carry_rows(rows, S, packed) -> int:
    _sizes("tgm_scan_carry_rows", (rows, S), (I64, I32))
    n = I64()
    _check("tgm_scan_carry_rows", lib().tgm_scan_carry_rows(rows, S, 1 if packed else 0,
                                                            C.byref(n)))
    return int(n.value)


def tgm_scan_work_bytes(rows, D, S) -> int:
    return _bytes("tgm_scan_work_bytes", rows, D, S)


def _scan_args(g, x, S, offsets, length, h0):
    import torch
    rows, D = _shape2("g", g)
    if not 0 <= S < 1 << 31:
        raise ValueError(f"S is {S}")
    gpu, dt = g.get_device(), g.dtype
    pg, lg = _arg("g", g, dt, (rows, D), gpu)
    px, lx = _arg("x", x, dt, (rows, D), gpu)
    po, _ = _opt("offsets", offsets, torch.int64, (S + 1,), gpu)
    pl, _ = _opt("length", length, torch.int32, (S,), gpu)
    ph = _dense("h0", h0, torch.float32, (S, D), gpu)
    return rows, D, gpu, dt, pg, lg, px, lx, po, pl, ph


def tgm_scan(g, x, y, S, work, offsets=None, length=None, h0=None, h_last=None, carry=None,
             reverse=False, stream=None):
    """h_t = a_t h_(t-1) + (1 - a_t) x_t, a = sigmoid(g), along S sequences:
    packed by ``offsets`` [S + 1], or padded (rows / S rows each)."""
    import torch
    rows, D, gpu, dt, pg, lg, px, lx, po, pl, ph = _scan_args(g, x, S, offsets, length, h0)
    py, ly = _arg("y", y, dt, (rows, D), gpu)
    pe = _dense("h_last", h_last, torch.float32, (S, D), gpu)
    pc = None
    if carry is not None:
        n = tgm_scan_carry_rows(rows, S, offsets is not None)
        pc = _dense("carry", carry, torch.float32, (n, D), gpu)
    pk, nk = _work_arg(work, gpu)
    d = ScanDesc(rows, S, D, dtype_code(dt), 1 if reverse else 0, lg, lx, ly, 0, 0)
    _call("tgm_scan", gpu, stream, C.byref(d), pg, px, po, pl, ph, py, pe, pc, pk, nk)


def tgm_scan_backward(g, x, dy, carry, dg, dx, S, work, offsets=None, length=None, h0=None,
                      dh_last=None, dh0=None, reverse=False, stream=None):
    """Gradients of tgm_scan with the same inputs, sequences and the ``carry``
    that it left."""
    import torch
    rows, D, gpu, dt, pg, lg, px, lx, po, pl, ph = _scan_args(g, x, S, offsets, length, h0)
    n = tgm_scan_carry_rows(rows, S, offsets is not None)
    pc = _dense("carry", carry, torch.float32, (n, D), gpu)
    py, ly = _arg("dy", dy, dt, (rows, D), gpu)
    pe = _dense("dh_last", dh_last, torch.float32, (S, D), gpu)
    pdg, ldg = _arg("dg", dg, dt, (rows, D), gpu)
    pdx, ldx = _arg("dx", dx, dt, (rows, D), gpu)
    p0 = _dense("dh0", dh0, torch.float32, (S, D), gpu)
    pk, nk = _work_arg(work, gpu)
    d = ScanDesc(rows, S, D, dtype_code(dt), 1 if reverse else 0, lg, lx, ly, ldg, ldx)
    _call("tgm_scan_backward", gpu, stream, C.byref(d), pg, px, po, pl, ph, pc, py, pe, pdg, pdx,
          p0, pk, nk)


def tgm_scan_step(g, x, state, y, slots=None, n_rows=None, stream=None):
    """One row of the scan for each row of g and x, into ``state`` [slots x D]
    in place."""
    import torch
    rows, D = _shape2("g", g)
    gpu, dt = g.get_device(), g.dtype
    S, _ = _shape2("state", state)
    pg, lg = _arg("g", g, dt, (rows, D), gpu)
    px, lx = _arg("x", x, dt, (rows, D), gpu)
    ps = _dense("state", state, torch.float32, (S, D), gpu)
    py, ly = _opt("y", y, dt, (rows, D), gpu)
    pt, _ = _opt("slots", slots, torch.int32, (rows,), gpu)
    pn, _ = _opt("n_rows", n_rows, torch.int32, (1,), gpu)
    d = ScanDesc(rows, S, D, dtype_code(dt), 0, lg, lx, ly, 0, 0)
    _call("tgm_scan_step", gpu, stream, C.byref(d), pg, px, pt, pn, ps, py)


def _choice(what, name, choices) -> int:
    if name not in choices:
        raise ValueError(f"{what} is one of {sorted(choices)}, not {name!r}")
    return choices[name]


_pos_codes = {}   # torch types to TGM_POS_I32, ...


def tgm_rotary(x, y, heads, omega, pos=None, layout="half", amplitude=1.0, inverse=False,
               n_rows=None, stream=None):
    """y = x [rows x heads d] with the first 2 len(omega) columns of each head turned by
    ``pos`` (int32, int64 or float64; the row's number without) times ``omega`` (float64, on
    the GPU); ``inverse`` turns back, which is the gradient."""
    import torch
    if not _pos_codes:
        _pos_codes.update({torch.int32: TGM_POS_I32, torch.int64: TGM_POS_I64,
                           torch.float64: TGM_POS_F64})
    rows, W = _shape2("x", x)
    gpu, dt = x.get_device(), x.dtype
    if not 0 < heads <= W or W % heads:
        raise ValueError(f"x's {W} columns are no {heads} heads")
    if omega is None or omega.dim() != 1:
        raise ValueError("omega is a vector")
    pairs = omega.shape[0]
    if 2 * pairs > W // heads:
        raise ValueError(f"{pairs} pairs in heads of {W // heads} columns")
    kind = TGM_POS_I32
    if pos is not None:
        kind = _pos_codes.get(pos.dtype)
        if kind is None:
            raise ValueError(f"pos has type {pos.dtype}")
    px, lx = _arg("x", x, dt, (rows, W), gpu)
    py, ly = _arg("y", y, dt, (rows, W), gpu)
    pw, _ = _arg("omega", omega, torch.float64, (pairs,), gpu)
    pp, _ = _opt("pos", pos, pos.dtype if pos is not None else None, (rows,), gpu)
    pn, _ = _opt("n_rows", n_rows, torch.int32, (1,), gpu)
    d = RotaryDesc(rows, heads, W // heads, 2 * pairs, dtype_code(dt), kind,
                   _choice("layout", layout, ROTARY_LAYOUTS), 1 if inverse else 0, amplitude, lx,
                   ly)
    _call("tgm_rotary", gpu, stream, C.byref(d), px, pw, pp, pn, py)


def tgm_rotary_frequencies(rot, scaling="none", base=10000.0, factor=1.0, original=0.0,
                           often=32.0, seldom=1.0):
    """(omega, amplitude): a float64 numpy array of rot / 2 frequencies, for histories
    ``factor`` times as long as the ``original`` positions, and the factor of cos and sin."""
    code = _choice("scaling", scaling, ROTARY_SCALINGS)
    _sizes("tgm_rotary_frequencies", (rot,), (I32,))
    omega, a = np.zeros(max(1, rot // 2)), C.c_float(0)
    _check("tgm_rotary_frequencies", lib().tgm_rotary_frequencies(
        rot, code, base, factor, original, often, seldom, omega.ctypes.data, C.byref(a)))
    return omega, float(a.value)


def tgm_xent_work_bytes(rows, N, K, dtype, backward=False) -> int:
    return _bytes("tgm_xent_work_bytes", rows, N, K, dtype_code(dtype), 1 if backward else 0)


def _xent_args(x, w, target, bias, n_rows):
    import torch
    (rows, K), (N, _) = _shape2("x", x), _shape2("w", w)
    gpu, dt = x.get_device(), x.dtype
    px, lx = _arg("x", x, dt, (rows, K), gpu)
    pw, lw = _arg("w", w, dt, (N, K), gpu)
    pb, _ = _opt("bias", bias, dt, (N,), gpu)
    pt, _ = _arg("target", target, torch.int32, (rows,), gpu)
    pn, _ = _opt("n_rows", n_rows, torch.int32, (1,), gpu)
    return rows, N, K, gpu, dt, px, lx, pw, lw, pb, pt, pn


def tgm_xent(x, w, target, loss, work, lse=None, bias=None, n_rows=None, stream=None):
    """loss = log sum exp(x w^T + bias) - (x w^T + bias)[target] a row, and ``lse``, the
    first term (each optional, fp32); rows whose target is outside the classes lose 0."""
    import torch
    rows, N, K, gpu, dt, px, lx, pw, lw, pb, pt, pn = _xent_args(x, w, target, bias, n_rows)
    pl, _ = _opt("loss", loss, torch.float32, (rows,), gpu)
    pe, _ = _opt("lse", lse, torch.float32, (rows,), gpu)
    pk, nk = _work_arg(work, gpu)
    d = XentDesc(rows, N, K, dtype_code(dt), lx, lw, 0, 0)
    _call("tgm_xent", gpu, stream, C.byref(d), px, pw, pb, pt, pn, pl, pe, pk, nk)


def tgm_xent_backward(x, w, target, lse, dloss, work, bias=None, dx=None, dw=None, db=None,
                      n_rows=None, stream=None):
    """dx, dw and db (each optional) of sum(dloss * loss), with the ``lse`` that tgm_xent
    wrote."""
    import torch
    rows, N, K, gpu, dt, px, lx, pw, lw, pb, pt, pn = _xent_args(x, w, target, bias, n_rows)
    pe, _ = _arg("lse", lse, torch.float32, (rows,), gpu)
    pd, _ = _arg("dloss", dloss, torch.float32, (rows,), gpu)
    pdx, ldx = _opt("dx", dx, dt, (rows, K), gpu)
    pdw, ldw = _opt("dw", dw, dt, (N, K), gpu)
    pdb, _ = _opt("db", db, dt, (N,), gpu)
    pk, nk = _work_arg(work, gpu)
    d = XentDesc(rows, N, K, dtype_code(dt), lx, lw, ldx, ldw)
    _call("tgm_xent_backward", gpu, stream, C.byref(d), px, pw, pb, pt, pe, pd, pn, pdx, pdw, pdb,
          pk, nk)


def tgm_decay_attn_work_bytes(rows, S, heads, d_k, d_v, dtype, kv_heads=None,
                              backward=False) -> int:
    return _bytes("tgm_decay_attn_work_bytes", rows, S, heads, kv_heads or heads, d_k, d_v,
                  dtype_code(dtype), 1 if backward else 0)


def _state(name, t, shape, gpu):
    """Address of an optional dense fp32 table of states."""
    import torch
    if t is None:
        return None
    if t.dtype is not torch.float32 or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name} is a contiguous float32 tensor of {shape}")
    if gpu < 0 or t.get_device() != gpu:
        raise ValueError(f"{name} is on {t.device}: every tensor of a call is on one GPU")
    return t.data_ptr()


def _decay_args(q, k, v, decay, kv_heads):
    """What the calls share: sizes, device, addresses and strides."""
    import torch
    (rows, wq), (_, wk), (_, wv) = _shape2("q", q), _shape2("k", k), _shape2("v", v)
    if decay is None or decay.dim() != 1:
        raise ValueError("decay is a vector, a number for each head")
    H = decay.shape[0]
    G = H if kv_heads is None else kv_heads
    if H < 1 or G < 1 or H % G:
        raise ValueError(f"{H} heads share {G} heads of k and v")
    if wq % H or wk % G or wv % G or wq // H != wk // G:
        raise ValueError(f"q, k and v of {wq}, {wk} and {wv} columns are no {H} and {G} heads")
    gpu, dt = q.get_device(), q.dtype
    pq, lq = _arg("q", q, dt, (rows, wq), gpu)
    pk, lk = _arg("k", k, dt, (rows, wk), gpu)
    pv, lv = _arg("v", v, dt, (rows, wv), gpu)
    pd, _ = _arg("decay", decay, torch.float32, (H,), gpu)
    return rows, H, G, wq // H, wv // G, gpu, dt, pq, lq, pk, lk, pv, lv, pd


def _sequences(S, offsets, length, gpu):
    import torch
    if not 0 <= S < 1 << 31:
        raise ValueError(f"S is {S}")
    return (_opt("offsets", offsets, torch.int64, (S + 1,), gpu)[0],
            _opt("length", length, torch.int32, (S,), gpu)[0])


def tgm_decay_attn(q, k, v, decay, o, S, work, scale=1.0, kv_heads=None, offsets=None, length=None,
                   state=None, state_last=None, reverse=False, stream=None):
    """S_t = exp(decay) S_(t-1) + k_t v_t^T, o_t = scale q_t S_t for each head, along S
    sequences: packed by ``offsets`` [S + 1], or padded (rows / S rows each).  q [rows x H
    d_k], k [rows x kv_heads d_k], v [rows x kv_heads d_v], decay [H] (log a), o [rows x H
    d_v], states [S, H, d_k, d_v] fp32."""
    rows, H, G, dk, dv, gpu, dt, pq, lq, pk, lk, pv, lv, pd = _decay_args(q, k, v, decay, kv_heads)
    pf, pl = _sequences(S, offsets, length, gpu)
    po, lo = _arg("o", o, dt, (rows, H * dv), gpu)
    ps = _state("state", state, (S, H, dk, dv), gpu)
    pe = _state("state_last", state_last, (S, H, dk, dv), gpu)
    pw, nw = _work_arg(work, gpu)
    d = DecayAttnDesc(rows, S, H, G, dk, dv, dtype_code(dt), 1 if reverse else 0, scale, lq, lk, lv,
                      lo, 0, 0, 0)
    _call("tgm_decay_attn", gpu, stream, C.byref(d), pq, pk, pv, pd, pf, pl, ps, po, pe, pw, nw)


def tgm_decay_attn_backward(q, k, v, decay, do, dq, dk, dv, S, work, scale=1.0, kv_heads=None,
                            offsets=None, length=None, state=None, dstate_last=None, dstate=None,
                            reverse=False, stream=None):
    """Gradients of tgm_decay_attn with the same inputs and sequences; dq, dk, dv and dstate
    are optional."""
    rows, H, G, nk, nv, gpu, dt, pq, lq, pk, lk, pv, lv, pd = _decay_args(q, k, v, decay, kv_heads)
    pf, pl = _sequences(S, offsets, length, gpu)
    po, lo = _arg("do", do, dt, (rows, H * nv), gpu)
    ps = _state("state", state, (S, H, nk, nv), gpu)
    pe = _state("dstate_last", dstate_last, (S, H, nk, nv), gpu)
    pb = _state("dstate", dstate, (S, H, nk, nv), gpu)
    pdq, ldq = _opt("dq", dq, dt, (rows, H * nk), gpu)
    pdk, ldk = _opt("dk", dk, dt, (rows, G * nk), gpu)
    pdv, ldv = _opt("dv", dv, dt, (rows, G * nv), gpu)
    pw, nw = _work_arg(work, gpu)
    d = DecayAttnDesc(rows, S, H, G, nk, nv, dtype_code(dt), 1 if reverse else 0, scale, lq, lk, lv,
                      lo, ldq, ldk, ldv)
    _call("tgm_decay_attn_backward", gpu, stream, C.byref(d), pq, pk, pv, pd, pf, pl, ps, po, pe,
          pdq, pdk, pdv, pb, pw, nw)


def tgm_decay_attn_step(q, k, v, decay, state, o, scale=1.0, kv_heads=None, slots=None,
                        n_rows=None, stream=None):
    """One row of tgm_decay_attn for each row of q, k and v, into ``state``
    [slots, H, d_k, d_v] in place."""
    import torch
    rows, H, G, dk, dv, gpu, dt, pq, lq, pk, lk, pv, lv, pd = _decay_args(q, k, v, decay, kv_heads)
    if state is None or state.dim() != 4:
        raise ValueError("state is a table of states [slots, H, d_k, d_v]")
    S = state.shape[0]
    ps = _state("state", state, (S, H, dk, dv), gpu)
    po, lo = _opt("o", o, dt, (rows, H * dv), gpu)
    pt, _ = _opt("slots", slots, torch.int32, (rows,), gpu)
    pn, _ = _opt("n_rows", n_rows, torch.int32, (1,), gpu)
    d = DecayAttnDesc(rows, S, H, G, dk, dv, dtype_code(dt), 0, scale, lq, lk, lv, lo, 0, 0, 0)
    _call("tgm_decay_attn_step", gpu, stream, C.byref(d), pq, pk, pv, pd, pt, pn, ps, po)
