"""ctypes binding of libcortex.so (the C ABI in include/cortex.h).

The functions below carry the C names and only marshal arguments: every step
of linearization and of the forward pass runs in the library's HIP kernels.
PyTorch serves as the allocator of device memory and the source of streams.
Loading fails loudly when the library has not been built; there is no
fallback path.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcortex.so")

CORTEX_OK = 0
CORTEX_E_INVAL = -1
CORTEX_E_HIP = -2
CORTEX_E_TOO_LARGE = -3
CORTEX_E_WORKSPACE = -4

CORTEX_ST_OK = 0
CORTEX_ST_CHILD_RANGE = 1
CORTEX_ST_CYCLE = 2
CORTEX_ST_BARRIER_TIMEOUT = 3
CORTEX_ST_BAD_LINEARIZATION = 4
CORTEX_ST_INPUT_RANGE = 5
CORTEX_ST_EPOCH_WRAP = 6
CORTEX_ST_SEQ_OFFSETS = 7

CORTEX_F32 = 0
CORTEX_BF16 = 1

CORTEX_NORM_NONE = 0
CORTEX_NORM_RMS = 1
CORTEX_NORM_L2 = 2

CORTEX_TREE_RNN = 0
CORTEX_NARY_TREELSTM = 1
CORTEX_CHILDSUM_TREELSTM = 2
CORTEX_MVRNN = 3
CORTEX_CHILDSUM_TREEGRU = 4
CORTEX_SIMPLE_TREEGRU = 5

CORTEX_KNOB_LIN_BLOCKS = 0
CORTEX_KNOB_FWD_NODE_GROUPS = 1
CORTEX_KNOB_BARRIER_TIMEOUT_US = 2
CORTEX_KNOB_COOPERATIVE = 3
CORTEX_KNOB_FWD_SLICE_UNITS = 4
CORTEX_KNOB_LEVEL_SYNC = 5
CORTEX_KNOB_TREE_UNROLL = 6
CORTEX_KNOB_ABLATE = 7

CELL_IDS = {"tree_rnn": CORTEX_TREE_RNN, "nary_treelstm": CORTEX_NARY_TREELSTM,
            "childsum_treelstm": CORTEX_CHILDSUM_TREELSTM, "mvrnn": CORTEX_MVRNN,
            "childsum_treegru": CORTEX_CHILDSUM_TREEGRU, "simple_treegru": CORTEX_SIMPLE_TREEGRU}

EXPORTED = [
    "cortex_linearize_workspace_bytes", "cortex_linearize", "cortex_forward_workspace_bytes",
    "cortex_tree_forward", "cortex_dag_forward", "cortex_tree_infer_workspace_bytes", "cortex_tree_infer",
    "cortex_tree_infer_noalloc",
    "cortex_dag_infer_workspace_bytes", "cortex_dag_infer",
    "cortex_set_knob", "cortex_get_knob",
    "cortex_last_grid", "cortex_version",
    "cortex_probe_mfma_sink_floats", "cortex_probe_mfma_flops", "cortex_probe_mfma",
    "cortex_probe_levels_workspace_bytes", "cortex_probe_levels",
    "cortex_conv_forward", "cortex_conv_step", "cortex_scan_workspace_bytes", "cortex_scan_forward",
    "cortex_scan_step", "cortex_logits_workspace_bytes", "cortex_logits_process",
    "cortex_delta_workspace_bytes", "cortex_delta_forward", "cortex_delta_step", "cortex_qk_norm",
    "cortex_delta_segment_tokens",
    "cortex_quant_i8", "cortex_linear_i8_workspace_bytes", "cortex_linear_i8",
]


class cortex_lin_t(ctypes.Structure):
    _fields_ = [("num_nodes", ctypes.c_int32), ("max_arity", ctypes.c_int32),
                ("num_levels", ctypes.c_void_p), ("height", ctypes.c_void_p),
                ("level_offsets", ctypes.c_void_p), ("level_nodes", ctypes.c_void_p),
                ("node_row", ctypes.c_void_p), ("child_rows", ctypes.c_void_p)]


class cortex_weights_t(ctypes.Structure):
    _fields_ = [("W", ctypes.c_void_p), ("U", ctypes.c_void_p), ("b", ctypes.c_void_p),
                ("W_M", ctypes.c_void_p)]


def _fields(text: str):
    """(name, ctype) pairs from "i name ..." groups: i int32, f float, l int64, p pointer."""
    kinds = {"i": ctypes.c_int32, "f": ctypes.c_float, "l": ctypes.c_int64, "p": ctypes.c_void_p}
    return [(n, kinds[group.split()[0]]) for group in text.split(";") for n in group.split()[1:]]


def _packer(text: str, cls):
    """The structure's bytes from its members' values in order; a call then costs
    the host a third of what filling a ctypes structure does."""
    kinds = {"i": "i", "f": "f", "l": "q", "p": "P"}
    s = struct.Struct("@" + "".join(kinds[group.split()[0]] * len(group.split()[1:]) for group in text.split(";")))
    assert s.size == ctypes.sizeof(cls)
    return s.pack


_CONV = ("i dtype num_seqs num_tokens channels width silu state_rows; p seq_offsets state_index x; l x_ld;"
         "p weight bias state_in state_out y; l y_ld")
_SCAN = ("i dtype num_seqs num_tokens channels head_dim groups state_size softplus state_rows;"
         "p seq_offsets state_index x z dt B C; l x_ld z_ld dt_ld B_ld C_ld;"
         "p A skip dt_bias state_in state_out y; l y_ld")
_LOGITS = ("i dtype rows vocab history_cap num_biases mask_rows; p logits; l logits_ld; p history; l history_ld;"
           "p history_len prompt_len repetition frequency presence bias_offsets bias_tokens bias_values mask;"
           "l mask_ld; p mask_index out; l out_ld; p token lse")
_DELTA = ("i dtype num_seqs num_tokens heads key_heads key_dim value_dim softplus sigmoid state_rows; f scale;"
          "p seq_offsets state_index q k v b dt; l q_ld k_ld v_ld b_ld dt_ld;"
          "p A dt_bias state_in state_out y; l y_ld")
_QK_NORM = ("i dtype num_tokens heads key_heads head_dim rotary_dim interleaved norm; f eps; p q k; l q_ld k_ld;"
            "p q_weight k_weight positions freqs q_out k_out; l q_out_ld k_out_ld")
_QUANT = "i dtype rows columns; p x; l x_ld; p q; l q_ld; p scale"
_LINEAR = "i dtype tokens inputs outputs; p x; l x_ld; p x_scale w; l w_ld; p w_scale bias y; l y_ld"


class cortex_conv_t(ctypes.Structure):
    _fields_ = _fields(_CONV)


class cortex_scan_t(ctypes.Structure):
    _fields_ = _fields(_SCAN)


class cortex_logits_t(ctypes.Structure):
    _fields_ = _fields(_LOGITS)


class cortex_delta_t(ctypes.Structure):
    _fields_ = _fields(_DELTA)


class cortex_qk_norm_t(ctypes.Structure):
    _fields_ = _fields(_QK_NORM)


class cortex_quant_i8_t(ctypes.Structure):
    _fields_ = _fields(_QUANT)


class cortex_linear_i8_t(ctypes.Structure):
    _fields_ = _fields(_LINEAR)


_pack_conv = _packer(_CONV, cortex_conv_t)
_pack_scan = _packer(_SCAN, cortex_scan_t)
_pack_logits = _packer(_LOGITS, cortex_logits_t)
_pack_delta = _packer(_DELTA, cortex_delta_t)
_pack_qk_norm = _packer(_QK_NORM, cortex_qk_norm_t)
_pack_quant = _packer(_QUANT, cortex_quant_i8_t)
_pack_linear = _packer(_LINEAR, cortex_linear_i8_t)


_lib: Optional[ctypes.CDLL] = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libcortex.so and declare the signatures (raises if it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError("libcortex.so is not built (%s); run paper_2011_01383_amd.build" % path)
    lib = ctypes.CDLL(path)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.cortex_linearize_workspace_bytes.argtypes = [I32, I32]
    lib.cortex_linearize_workspace_bytes.restype = SZ
    lib.cortex_linearize.argtypes = [P, I32, I32, ctypes.POINTER(cortex_lin_t), P, P, SZ, P]
    lib.cortex_linearize.restype = ctypes.c_int
    lib.cortex_forward_workspace_bytes.argtypes = [I32, I32, I32]
    lib.cortex_forward_workspace_bytes.restype = SZ
    lib.cortex_tree_forward.argtypes = [I32, I32, ctypes.POINTER(cortex_lin_t), P, I32, P, P,
                                        ctypes.POINTER(cortex_weights_t), P, P, P, P, SZ, P]
    lib.cortex_tree_forward.restype = ctypes.c_int
    lib.cortex_dag_forward.argtypes = [I32, ctypes.POINTER(cortex_lin_t), P, P, P, P, P, P, P, SZ, P]
    lib.cortex_dag_forward.restype = ctypes.c_int
    lib.cortex_tree_infer_workspace_bytes.argtypes = [I32, I32, I32, I32]
    lib.cortex_tree_infer_workspace_bytes.restype = SZ
    lib.cortex_tree_infer.argtypes = [I32, I32, P, ctypes.POINTER(cortex_lin_t), P, I32, P, P,
                                      ctypes.POINTER(cortex_weights_t), P, P, P, P, SZ, P]
    lib.cortex_tree_infer.restype = ctypes.c_int
    lib.cortex_tree_infer_noalloc.argtypes = [I32, I32, P, ctypes.POINTER(cortex_lin_t), P, I32, P, P,
                                              ctypes.POINTER(cortex_weights_t), P, P, P, P]
    lib.cortex_tree_infer_noalloc.restype = ctypes.c_int
    lib.cortex_dag_infer_workspace_bytes.argtypes = [I32, I32, I32]
    lib.cortex_dag_infer_workspace_bytes.restype = SZ
    lib.cortex_dag_infer.argtypes = [I32, P, ctypes.POINTER(cortex_lin_t), P, P, P, P, P, P, P, SZ, P]
    lib.cortex_dag_infer.restype = ctypes.c_int
    lib.cortex_set_knob.argtypes = [I32, I64]
    lib.cortex_set_knob.restype = ctypes.c_int
    lib.cortex_get_knob.argtypes = [I32]
    lib.cortex_get_knob.restype = I64
    lib.cortex_last_grid.argtypes = [I32]
    lib.cortex_last_grid.restype = I32
    lib.cortex_probe_mfma_sink_floats.argtypes = []
    lib.cortex_probe_mfma_sink_floats.restype = SZ
    lib.cortex_probe_mfma_flops.argtypes = [I32]
    lib.cortex_probe_mfma_flops.restype = ctypes.c_double
    lib.cortex_probe_mfma.argtypes = [P, I32, P]
    lib.cortex_probe_mfma.restype = ctypes.c_int
    lib.cortex_probe_levels_workspace_bytes.argtypes = []
    lib.cortex_probe_levels_workspace_bytes.restype = SZ
    lib.cortex_probe_levels.argtypes = [I32, I32, I32, P, P, SZ, P]
    lib.cortex_probe_levels.restype = ctypes.c_int
    lib.cortex_conv_forward.argtypes = [P, P, P]
    lib.cortex_conv_forward.restype = ctypes.c_int
    lib.cortex_conv_step.argtypes = [P, P, P]
    lib.cortex_conv_step.restype = ctypes.c_int
    lib.cortex_scan_workspace_bytes.argtypes = [I32, I32, I32, I32, I32]
    lib.cortex_scan_workspace_bytes.restype = SZ
    lib.cortex_scan_forward.argtypes = [P, P, P, SZ, P]
    lib.cortex_scan_forward.restype = ctypes.c_int
    lib.cortex_scan_step.argtypes = [P, P, P]
    lib.cortex_scan_step.restype = ctypes.c_int
    lib.cortex_logits_workspace_bytes.argtypes = [I32, I32]
    lib.cortex_logits_workspace_bytes.restype = SZ
    lib.cortex_logits_process.argtypes = [P, P, P, SZ, P]
    lib.cortex_logits_process.restype = ctypes.c_int
    lib.cortex_delta_workspace_bytes.argtypes = [I32, I32, I32, I32, I32]
    lib.cortex_delta_workspace_bytes.restype = SZ
    lib.cortex_delta_segment_tokens.argtypes = [I32, I32, I32, I32, I32]
    lib.cortex_delta_segment_tokens.restype = I32
    lib.cortex_delta_forward.argtypes = [P, P, P, SZ, P]
    lib.cortex_delta_forward.restype = ctypes.c_int
    lib.cortex_delta_step.argtypes = [P, P, P]
    lib.cortex_delta_step.restype = ctypes.c_int
    lib.cortex_qk_norm.argtypes = [P, P, P]
    lib.cortex_qk_norm.restype = ctypes.c_int
    lib.cortex_quant_i8.argtypes = [P, P, P]
    lib.cortex_quant_i8.restype = ctypes.c_int
    lib.cortex_linear_i8_workspace_bytes.argtypes = [I32, I32, I32]
    lib.cortex_linear_i8_workspace_bytes.restype = SZ
    lib.cortex_linear_i8.argtypes = [P, P, P, SZ, P]
    lib.cortex_linear_i8.restype = ctypes.c_int
    lib.cortex_version.argtypes = []
    lib.cortex_version.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _need(t, name: str, dtype: torch.dtype, min_numel: int, optional: bool = False) -> None:
    """Reject a tensor the library would misread: the library takes raw
    pointers, so a wrong dtype, a strided view, too few elements or host
    memory would be read as something else (or past the allocation)."""
    _need_all([(t, name, dtype, min_numel, optional)])


def _need_all(specs) -> None:
    """_need over several tensors: every dtype, layout and size first, then
    that each tensor is in device memory."""
    for t, _, dtype, min_numel, optional in specs:
        if t is None:
            if not optional:
                break
        elif not (type(t) is torch.Tensor and (dtype is None or t.dtype is dtype) and t.is_contiguous()
                  and t.numel() >= min_numel and t.is_cuda):
            break
    else:
        return                          # nothing to refuse: the usual call
    for t, name, dtype, min_numel, optional in specs:
        if t is None:
            if optional:
                continue
            raise ValueError("%s is required" % name)
        if not isinstance(t, torch.Tensor):
            raise ValueError("%s must be a torch.Tensor, got %s" % (name, type(t).__name__))
        if dtype is not None and t.dtype != dtype:
            raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
        if t.numel() < min_numel:
            raise ValueError("%s holds %d elements, needs at least %d" % (name, t.numel(), min_numel))
    for t, name, _, _, _ in specs:
        if t is not None and not t.is_cuda:
            raise ValueError("%s must be in device memory" % name)


def _need_count(v: int, name: str) -> None:
    if int(v) < 0:
        raise ValueError("%s must be non-negative, got %d" % (name, int(v)))


# Elements of each weight tensor per cell, as functions of H (layouts of the
# header: row-major [out, in] float32).
_WEIGHT_ELEMS = {
    CORTEX_TREE_RNN: {"W": lambda H: 2 * H * H, "b": lambda H: H},
    CORTEX_NARY_TREELSTM: {"U": lambda H: 10 * H * H, "b": lambda H: 5 * H},
    CORTEX_CHILDSUM_TREELSTM: {"W": lambda H: 4 * H * H, "U": lambda H: 4 * H * H, "b": lambda H: 4 * H},
    CORTEX_MVRNN: {"W": lambda H: 2 * H * H, "W_M": lambda H: 2 * H * H},
    CORTEX_CHILDSUM_TREEGRU: {"W": lambda H: 3 * H * H, "U": lambda H: 3 * H * H, "b": lambda H: 3 * H},
    CORTEX_SIMPLE_TREEGRU: {"W": lambda H: 3 * H * H, "U": lambda H: 3 * H * H, "b": lambda H: 3 * H},
}


_NO_WS = object()        # the entry point takes no workspace


def _check_tree_args(cell: int, H: int, N: int, x_table, x_rows: int, x_index, leaf_mat, weights: dict, h,
                     c_or_P, status, ws) -> None:
    if cell not in _WEIGHT_ELEMS:
        return                      # the library rejects the cell id itself
    _need_count(H, "H")
    _need_count(x_rows, "x_rows")
    f32, i32 = torch.float32, torch.int32
    specs = [(x_table, "x_table", f32, x_rows * H, x_rows == 0), (x_index, "x_index", i32, N, False)]
    if cell == CORTEX_MVRNN:
        specs.append((leaf_mat, "leaf_mat", f32, x_rows * H * H, x_rows == 0))
    for name, elems in _WEIGHT_ELEMS[cell].items():
        specs.append((weights.get(name), name, f32, elems(H), False))
    specs.append((h, "h", f32, N * H, False))
    if cell in (CORTEX_NARY_TREELSTM, CORTEX_CHILDSUM_TREELSTM):
        specs.append((c_or_P, "c", f32, N * H, False))
    elif cell == CORTEX_MVRNN:
        specs.append((c_or_P, "P", f32, N * H * H, False))
    specs.append((status, "status", i32, 1, False))
    if ws is not _NO_WS:
        specs.append((ws, "ws", None, 1, False))
    _need_all(specs)


def _check_dag_args(H: int, N: int, x, W, U, b, h, status, ws) -> None:
    _need_count(H, "H")
    f32 = torch.float32
    _need_all([(x, "x", f32, N * H, False), (W, "W", f32, H * H, False), (U, "U", f32, 2 * H * H, False),
               (b, "b", f32, H, False), (h, "h", f32, N * H, False), (status, "status", torch.int32, 1, False),
               (ws, "ws", None, 1, False)])


def _check_lin(lin: "Linearization", N: int, K: int) -> None:
    if not isinstance(lin, Linearization):
        raise ValueError("lin must be a Linearization")
    if lin.N != N or lin.K != K:
        raise ValueError("lin was allocated for N=%d K=%d, the call has N=%d K=%d" % (lin.N, lin.K, N, K))


def _stream(stream) -> Optional[int]:
    if stream is None:
        # the handle that torch.cuda.current_stream() wraps in an object (2.7 us of host time a call)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch._C._cuda_getDevice())
    return getattr(stream, "cuda_stream", stream)


# ---- the C entry points, same names -------------------------------------------

def cortex_linearize_workspace_bytes(N: int, K: int) -> int:
    return load().cortex_linearize_workspace_bytes(N, K)


def cortex_forward_workspace_bytes(cell: int, N: int, H: int) -> int:
    return load().cortex_forward_workspace_bytes(cell, N, H)


def cortex_linearize(children: torch.Tensor, N: int, K: int, lin: "Linearization",
                     status: torch.Tensor, ws: torch.Tensor, stream=None) -> int:
    _need_count(N, "N")
    _need_count(K, "K")
    _need(children, "children", torch.int32, N * K)
    _check_lin(lin, N, K)
    _need(status, "status", torch.int32, 1)
    _need(ws, "ws", None, 1)
    return load().cortex_linearize(_ptr(children), N, K, ctypes.byref(lin.struct), _ptr(status),
                                   _ptr(ws), ws.numel() * ws.element_size(), _stream(stream))


def cortex_tree_forward(cell: int, H: int, lin: "Linearization", x_table: Optional[torch.Tensor],
                        x_rows: int, x_index: torch.Tensor, leaf_mat: Optional[torch.Tensor],
                        W=None, U=None, b=None, W_M=None, h: torch.Tensor = None,
                        c_or_P: Optional[torch.Tensor] = None, status: torch.Tensor = None,
                        ws: torch.Tensor = None, stream=None) -> int:
    _check_lin(lin, lin.N, lin.K)
    _check_tree_args(cell, H, lin.N, x_table, x_rows, x_index, leaf_mat, {"W": W, "U": U, "b": b, "W_M": W_M},
                     h, c_or_P, status, ws)
    w = cortex_weights_t(_ptr(W), _ptr(U), _ptr(b), _ptr(W_M))
    return load().cortex_tree_forward(cell, H, ctypes.byref(lin.struct), _ptr(x_table), x_rows,
                                      _ptr(x_index), _ptr(leaf_mat), ctypes.byref(w), _ptr(h),
                                      _ptr(c_or_P), _ptr(status), _ptr(ws),
                                      ws.numel() * ws.element_size(), _stream(stream))


def cortex_dag_forward(H: int, lin: "Linearization", x: torch.Tensor, W: torch.Tensor,
                       U: torch.Tensor, b: torch.Tensor, h: torch.Tensor, status: torch.Tensor,
                       ws: torch.Tensor, stream=None) -> int:
    _check_lin(lin, lin.N, lin.K)
    _check_dag_args(H, lin.N, x, W, U, b, h, status, ws)
    return load().cortex_dag_forward(H, ctypes.byref(lin.struct), _ptr(x), _ptr(W), _ptr(U), _ptr(b),
                                     _ptr(h), _ptr(status), _ptr(ws), ws.numel() * ws.element_size(),
                                     _stream(stream))


def cortex_tree_infer_workspace_bytes(cell: int, N: int, K: int, H: int) -> int:
    return load().cortex_tree_infer_workspace_bytes(cell, N, K, H)


def cortex_tree_infer(cell: int, H: int, children: torch.Tensor, lin: "Linearization",
                      x_table: Optional[torch.Tensor], x_rows: int, x_index: torch.Tensor,
                      leaf_mat: Optional[torch.Tensor], W=None, U=None, b=None, W_M=None,
                      h: torch.Tensor = None, c_or_P: Optional[torch.Tensor] = None,
                      status: torch.Tensor = None, ws: torch.Tensor = None, stream=None) -> int:
    _check_lin(lin, lin.N, lin.K)
    _need(children, "children", torch.int32, lin.N * lin.K)
    _check_tree_args(cell, H, lin.N, x_table, x_rows, x_index, leaf_mat, {"W": W, "U": U, "b": b, "W_M": W_M},
                     h, c_or_P, status, ws)
    w = cortex_weights_t(_ptr(W), _ptr(U), _ptr(b), _ptr(W_M))
    return load().cortex_tree_infer(cell, H, _ptr(children), ctypes.byref(lin.struct), _ptr(x_table), x_rows,
                                    _ptr(x_index), _ptr(leaf_mat), ctypes.byref(w), _ptr(h), _ptr(c_or_P),
                                    _ptr(status), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream))


def cortex_tree_infer_noalloc(cell: int, H: int, children: torch.Tensor, lin: "Linearization",
                              x_table: Optional[torch.Tensor], x_rows: int, x_index: torch.Tensor,
                              leaf_mat: Optional[torch.Tensor], W=None, U=None, b=None, W_M=None,
                              h: torch.Tensor = None, c_or_P: Optional[torch.Tensor] = None,
                              status: torch.Tensor = None, stream=None) -> int:
    _check_lin(lin, lin.N, lin.K)
    _need(children, "children", torch.int32, lin.N * lin.K)
    _check_tree_args(cell, H, lin.N, x_table, x_rows, x_index, leaf_mat, {"W": W, "U": U, "b": b, "W_M": W_M},
                     h, c_or_P, status, _NO_WS)
    w = cortex_weights_t(_ptr(W), _ptr(U), _ptr(b), _ptr(W_M))
    return load().cortex_tree_infer_noalloc(cell, H, _ptr(children), ctypes.byref(lin.struct), _ptr(x_table), x_rows,
                                            _ptr(x_index), _ptr(leaf_mat), ctypes.byref(w), _ptr(h), _ptr(c_or_P),
                                            _ptr(status), _stream(stream))


def cortex_dag_infer_workspace_bytes(N: int, K: int, H: int) -> int:
    return load().cortex_dag_infer_workspace_bytes(N, K, H)


def cortex_dag_infer(H: int, children: torch.Tensor, lin: "Linearization", x: torch.Tensor, W: torch.Tensor,
                     U: torch.Tensor, b: torch.Tensor, h: torch.Tensor, status: torch.Tensor, ws: torch.Tensor,
                     stream=None) -> int:
    _check_lin(lin, lin.N, lin.K)
    _need(children, "children", torch.int32, lin.N * lin.K)
    _check_dag_args(H, lin.N, x, W, U, b, h, status, ws)
    return load().cortex_dag_infer(H, _ptr(children), ctypes.byref(lin.struct), _ptr(x), _ptr(W), _ptr(U),
                                   _ptr(b), _ptr(h), _ptr(status), _ptr(ws), ws.numel() * ws.element_size(),
                                   _stream(stream))


def cortex_set_knob(knob: int, value: int) -> int:
    return load().cortex_set_knob(knob, value)


def cortex_get_knob(knob: int) -> int:
    return load().cortex_get_knob(knob)


def cortex_last_grid(which: int) -> int:
    return load().cortex_last_grid(which)


def cortex_probe_mfma_sink_floats() -> int:
    return load().cortex_probe_mfma_sink_floats()


def cortex_probe_mfma_flops(iters: int) -> float:
    return load().cortex_probe_mfma_flops(iters)


def cortex_probe_mfma(sink: torch.Tensor, iters: int, stream=None) -> int:
    _need(sink, "sink", torch.float32, cortex_probe_mfma_sink_floats())
    return load().cortex_probe_mfma(_ptr(sink), iters, _stream(stream))


def cortex_probe_levels_workspace_bytes() -> int:
    return load().cortex_probe_levels_workspace_bytes()


def cortex_probe_levels(mode: int, grid: int, levels: int, status: torch.Tensor, ws: torch.Tensor,
                        stream=None) -> int:
    _need(status, "status", torch.int32, 1)
    _need(ws, "ws", None, 1)
    return load().cortex_probe_levels(mode, grid, levels, _ptr(status), _ptr(ws), ws.numel() * ws.element_size(),
                                      _stream(stream))


# ---- sequences ------------------------------------------------------------------

_DTYPES = {torch.float32: CORTEX_F32, torch.bfloat16: CORTEX_BF16}


def _at(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _rows(t, name: str, dtype, rows: int, cols: int) -> int:
    """A [rows, cols] tensor whose rows are whole and may be apart (the columns
    of a wider array): its row stride."""
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s is required" % name if t is None else
                         "%s must be a torch.Tensor, got %s" % (name, type(t).__name__))
    if t.dtype is not dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    shape = t.shape
    if len(shape) != 2 or shape[0] != rows or shape[1] != cols:
        raise ValueError("%s must be [%d, %d], got %s" % (name, rows, cols, list(shape)))
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        raise ValueError("%s must have contiguous rows" % name)
    if ld < cols:
        if rows > 1:
            raise ValueError("%s must have rows that do not overlap" % name)
        return cols                    # one row: its stride is never used
    return ld


def _on_device(names: str, *tensors) -> None:
    for i, t in enumerate(tensors):
        if t is not None and not t.is_cuda:
            raise ValueError("%s must be in device memory" % names.split()[i])


def _shape2(t, name: str):
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError("%s must be a 2-dimensional torch.Tensor" % name)
    if t.dtype not in _DTYPES:
        raise ValueError("%s must be torch.float32 or torch.bfloat16, got %s" % (name, t.dtype))
    return t.shape


def _state_specs(state_in, state_out, state_index, S: int, dtype, tail: tuple):
    """Rows of the state pools and what they have to hold."""
    rows = -1
    for t in (state_in,) if state_out is state_in else (state_in, state_out):
        if t is None:
            continue
        shape = t.shape if isinstance(t, torch.Tensor) else ()
        if len(shape) != 3 or shape[1:] != tail or (rows >= 0 and shape[0] != rows):
            raise ValueError("state_in and state_out must be [rows, %d, %d], with the same rows" % tail)
        rows = shape[0]
    if rows < 0:
        rows = 0
    elif state_index is None and rows < S:
        raise ValueError("the states have %d rows, %d sequences need as many" % (rows, S))
    n = rows * tail[0] * tail[1]
    return rows, [(state_in, "state_in", dtype, n, True), (state_out, "state_out", dtype, n, True),
                  (state_index, "state_index", torch.int32, S, True)]


def _conv(step: bool, x, weight, offsets, y, bias, silu, state_in, state_out, state_index, status, stream) -> int:
    T, C = _shape2(x, "x")
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2 or weight.shape[0] != C:
        raise ValueError("weight must be [%d, W]" % C)
    W, f32, i32 = weight.shape[1], torch.float32, torch.int32
    if step:
        S = T
        specs = []
    else:
        if not isinstance(offsets, torch.Tensor) or offsets.numel() < 1:
            raise ValueError("offsets must be a torch.Tensor of S + 1 elements")
        S = offsets.numel() - 1
        specs = [(offsets, "offsets", i32, S + 1, False)]
    rows, state = _state_specs(state_in, state_out, state_index, S, x.dtype, (W - 1, C))
    x_ld, y_ld = _rows(x, "x", x.dtype, T, C), _rows(y, "y", x.dtype, T, C)
    _need_all(specs + state + [(weight, "weight", f32, C * W, False), (bias, "bias", f32, C, True),
                               (status, "status", i32, 1, False)])
    _on_device("x y", x, y)
    args = _pack_conv(_DTYPES[x.dtype], S, T, C, W, 1 if silu else 0, rows, _at(offsets), _at(state_index), x.data_ptr(),
                      x_ld, weight.data_ptr(), _at(bias), _at(state_in), _at(state_out), y.data_ptr(), y_ld)
    lib = load()
    call = lib.cortex_conv_step if step else lib.cortex_conv_forward
    return call(args, status.data_ptr(), _stream(stream))


def cortex_conv_forward(x: torch.Tensor, weight: torch.Tensor, offsets: torch.Tensor, y: torch.Tensor, *, bias=None,
                        silu: bool = True, state_in=None, state_out=None, state_index=None,
                        status: torch.Tensor = None, stream=None) -> int:
    """x, y [T, C]; weight [C, W]; offsets [S + 1]; states [rows, W - 1, C]."""
    return _conv(False, x, weight, offsets, y, bias, silu, state_in, state_out, state_index, status, stream)


def cortex_conv_step(x: torch.Tensor, weight: torch.Tensor, y: torch.Tensor, *, bias=None, silu: bool = True,
                     state_in=None, state_out=None, state_index=None, status: torch.Tensor = None, stream=None) -> int:
    """One token of each of S sequences: x, y [S, C]."""
    return _conv(True, x, weight, None, y, bias, silu, state_in, state_out, state_index, status, stream)


def _group_rows(t, name: str, dtype, T: int):
    """A [T, G, N] tensor with the groups of a row side by side: G, N and its row stride."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError("%s must be a [T, G, N] torch.Tensor" % name)
    if t.dtype is not dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    rows, G, N = t.shape
    if rows != T:
        raise ValueError("%s must have %d rows, got %d" % (name, T, rows))
    ld, between, inner = t.stride()
    if (inner != 1 and N > 1) or (between != N and G > 1):
        raise ValueError("%s must have contiguous rows" % name)
    if ld < G * N:
        if rows > 1:
            raise ValueError("%s must have rows that do not overlap" % name)
        ld = G * N
    return G, N, ld


def _scan(step: bool, x, dt, A, B, C, offsets, y, skip, z, dt_bias, softplus, state_in, state_out, state_index, status,
          ws, stream) -> int:
    T, D = _shape2(x, "x")
    typ, f32, i32 = x.dtype, torch.float32, torch.int32
    if not isinstance(A, torch.Tensor) or A.dim() not in (1, 2):
        raise ValueError("A must be [D, N] (decays per channel) or [heads] (decays per head)")
    G, N, B_ld = _group_rows(B, "B", typ, T)
    G2, N2, C_ld = _group_rows(C, "C", typ, T)
    if (G, N) != (G2, N2):
        raise ValueError("B and C must have the same groups and state size")
    H = A.shape[0]
    if A.dim() == 2:
        if H != D or A.shape[1] != N:
            raise ValueError("A must be [%d, %d], got %s" % (D, N, list(A.shape)))
        P = 0
    else:
        if H < 1 or D % H:
            raise ValueError("A must hold a divisor of %d heads, got %d" % (D, H))
        P = D // H
    if step:
        S = T
        specs = []
    else:
        if not isinstance(offsets, torch.Tensor) or offsets.numel() < 1:
            raise ValueError("offsets must be a torch.Tensor of S + 1 elements")
        S = offsets.numel() - 1
        specs = [(offsets, "offsets", i32, S + 1, False), (ws, "ws", None, 1, False)]
    rows, state = _state_specs(state_in, state_out, state_index, S, f32, (D, N))
    x_ld, y_ld, dt_ld = _rows(x, "x", typ, T, D), _rows(y, "y", typ, T, D), _rows(dt, "dt", typ, T, H)
    z_ld = 0 if z is None else _rows(z, "z", typ, T, D)
    _need_all(specs + state + [(A, "A", f32, A.numel(), False), (skip, "D", f32, H, True),
                               (dt_bias, "dt_bias", f32, H, True), (status, "status", i32, 1, False)])
    _on_device("x dt B C z y", x, dt, B, C, z, y)
    args = _pack_scan(_DTYPES[typ], S, T, D, P, G, N, 1 if softplus else 0, rows, _at(offsets), _at(state_index),
                      x.data_ptr(), _at(z), dt.data_ptr(), B.data_ptr(), C.data_ptr(), x_ld, z_ld, dt_ld, B_ld, C_ld,
                      A.data_ptr(), _at(skip), _at(dt_bias), _at(state_in), _at(state_out), y.data_ptr(), y_ld)
    lib = load()
    if step:
        return lib.cortex_scan_step(args, status.data_ptr(), _stream(stream))
    return lib.cortex_scan_forward(args, status.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(),
                                   _stream(stream))


def cortex_scan_workspace_bytes(T: int, S: int, D: int, N: int, head_dim: int = 0) -> int:
    return load().cortex_scan_workspace_bytes(T, S, D, N, head_dim)


def cortex_scan_forward(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor,
                        offsets: torch.Tensor, y: torch.Tensor, *, D=None, z=None, dt_bias=None, softplus: bool = True,
                        state_in=None, state_out=None, state_index=None, status: torch.Tensor = None,
                        ws: torch.Tensor = None, stream=None) -> int:
    """x, y, z [T, D]; B, C [T, G, N]; A [D, N] with dt [T, D], or A [heads] with
    dt [T, heads]; the skip D and dt_bias like dt's rows; states [rows, D, N]."""
    return _scan(False, x, dt, A, B, C, offsets, y, D, z, dt_bias, softplus, state_in, state_out, state_index, status, ws,
                 stream)


def cortex_scan_step(x: torch.Tensor, dt: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor,
                     y: torch.Tensor, *, D=None, z=None, dt_bias=None, softplus: bool = True, state_in=None,
                     state_out=None, state_index=None, status: torch.Tensor = None, stream=None) -> int:
    """One token of each of S sequences: x, y, z [S, D], dt and B, C likewise."""
    return _scan(True, x, dt, A, B, C, None, y, D, z, dt_bias, softplus, state_in, state_out, state_index, status, None,
                 stream)


def cortex_logits_workspace_bytes(rows: int, vocab: int) -> int:
    return load().cortex_logits_workspace_bytes(rows, vocab)


def cortex_logits_process(logits: torch.Tensor, *, out=None, token=None, lse=None, history=None, history_len=None,
                          prompt_len=None, repetition=None, frequency=None, presence=None, bias_offsets=None,
                          bias_tokens=None, bias_values=None, mask=None, mask_index=None, status: torch.Tensor = None,
                          ws: torch.Tensor = None, stream=None) -> int:
    """logits, out [R, V]; history [R, columns]; mask [states, ceil(V / 32)] of int32 words."""
    R, V = _shape2(logits, "logits")
    f32, i32 = torch.float32, torch.int32
    if out is None and token is None and lse is None:
        raise ValueError("out, token or lse is required")
    specs = [(token, "token", i32, R, True), (lse, "lse", f32, R, True), (status, "status", i32, 1, False),
             (ws, "ws", None, 1, False)]
    cap = history_ld = biases = states = mask_ld = 0
    if history is not None:
        if not isinstance(history, torch.Tensor) or history.dim() != 2:
            raise ValueError("history must be a 2-dimensional torch.Tensor")
        cap = history.shape[1]
        history_ld = _rows(history, "history", i32, R, cap)
        specs += [(history_len, "history_len", i32, R, False), (prompt_len, "prompt_len", i32, R, True),
                  (repetition, "repetition", f32, R, True), (frequency, "frequency", f32, R, True),
                  (presence, "presence", f32, R, True)]
    elif any(t is not None for t in (history_len, prompt_len, repetition, frequency, presence)):
        raise ValueError("history is required with its lengths and penalties")
    if bias_offsets is not None:
        if bias_tokens is not None and not isinstance(bias_tokens, torch.Tensor):
            raise ValueError("bias_tokens must be a torch.Tensor, got %s" % type(bias_tokens).__name__)
        biases = 0 if bias_tokens is None else bias_tokens.numel()
        specs += [(bias_offsets, "bias_offsets", i32, R + 1, False), (bias_tokens, "bias_tokens", i32, 0, False),
                  (bias_values, "bias_values", f32, biases, False)]
    elif bias_tokens is not None or bias_values is not None:
        raise ValueError("bias_offsets is required with the biases")
    if mask is not None:
        if not isinstance(mask, torch.Tensor) or mask.dim() != 2:
            raise ValueError("mask must be a 2-dimensional torch.Tensor")
        states = mask.shape[0]
        mask_ld = _rows(mask, "mask", i32, states, (V + 31) // 32)
        specs.append((mask_index, "mask_index", i32, R, True))
        if mask_index is None and states < R:
            raise ValueError("mask has %d rows, %d rows of logits need as many" % (states, R))
    elif mask_index is not None:
        raise ValueError("mask is required with mask_index")
    logits_ld = _rows(logits, "logits", logits.dtype, R, V)
    out_ld = 0 if out is None else _rows(out, "out", logits.dtype, R, V)
    _need_all(specs)
    _on_device("logits out history mask", logits, out, history, mask)
    args = _pack_logits(_DTYPES[logits.dtype], R, V, cap, biases, states, logits.data_ptr(), logits_ld, _at(history),
                        history_ld, _at(history_len), _at(prompt_len), _at(repetition), _at(frequency), _at(presence),
                        _at(bias_offsets), _at(bias_tokens), _at(bias_values), _at(mask), mask_ld, _at(mask_index),
                        _at(out), out_ld, _at(token), _at(lse))
    return load().cortex_logits_process(args, status.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(),
                                        _stream(stream))


def _all_here(specs, names: str, *tensors) -> None:
    """_need_all over `specs`, and that these and `tensors` (views, named in `names`) are in the
    memory of the current device, to which the launch goes."""
    device = tensors[0].get_device()
    if device >= 0:
        for t in tensors:
            if t is not None and t.get_device() != device:
                break
        else:
            for t, _, dtype, min_numel, optional in specs:
                if t is None:
                    if not optional:
                        break
                elif not (type(t) is torch.Tensor and (dtype is None or t.dtype is dtype) and t.is_contiguous()
                          and t.numel() >= min_numel and t.get_device() == device):
                    break
            else:
                if device == torch._C._cuda_getDevice():
                    return              # nothing to refuse: the usual call
    _need_all(specs)
    _on_device(names, *tensors)
    current = torch.cuda.current_device()
    for name, t in [*zip(names.split(), tensors), *((s[1], s[0]) for s in specs)]:
        if t is not None and t.get_device() != current:
            raise ValueError("%s must be on the current device (%d), got %d" % (name, current, t.get_device()))


def _head_rows(t, name: str, dtype, T: int, like=None):
    """A [T, heads, elements] tensor: heads, elements and its row stride."""
    if type(t) is torch.Tensor and t.dtype is dtype:
        shape = t.shape
        if len(shape) == 3:
            rows, H, P = shape
            ld, between, inner = t.stride()
            if rows == T and inner == 1 and between == P and ld >= H * P and (like is None or like == (H, P)):
                return H, P, ld         # the usual rows
    H, P, ld = _group_rows(t, name, dtype, T)
    if like is not None and (H, P) != like:
        raise ValueError("%s must be [%d, %d, %d], got %s" % (name, T, like[0], like[1], list(t.shape)))
    return H, P, ld


def _number(v, name: str) -> float:
    if type(v) is float:
        return v
    if isinstance(v, torch.Tensor) or isinstance(v, str):
        raise ValueError("%s must be a number, got %s" % (name, type(v).__name__))
    return float(v)


def _delta(step: bool, q, k, v, b, offsets, y, dt, A, dt_bias, softplus, sigmoid, scale, state_in, state_out, state_index,
           status, ws, stream) -> int:
    if not isinstance(v, torch.Tensor) or v.dim() != 3 or v.dtype not in _DTYPES:
        raise ValueError("v must be a [T, H, V] torch.Tensor of torch.float32 or torch.bfloat16")
    scale = _number(scale, "scale")
    T, typ, f32, i32 = v.shape[0], v.dtype, torch.float32, torch.int32
    H, V, v_ld = _head_rows(v, "v", typ, T)
    G, K, q_ld = _head_rows(q, "q", typ, T)
    _, _, k_ld = _head_rows(k, "k", typ, T, (G, K))
    _, _, y_ld = _head_rows(y, "y", typ, T, (H, V))
    b_ld = _rows(b, "b", typ, T, H)
    if A is None:
        if dt is not None or dt_bias is not None:
            raise ValueError("A is required with dt and dt_bias")
        dt_ld = 0
    else:
        dt_ld = _rows(dt, "dt", typ, T, H)
    if step:
        S = T
        specs = []
    else:
        if not isinstance(offsets, torch.Tensor) or offsets.numel() < 1:
            raise ValueError("offsets must be a torch.Tensor of S + 1 elements")
        S = offsets.numel() - 1
        specs = [(offsets, "offsets", i32, S + 1, False), (ws, "ws", None, 1, False)]
    rows, state = _state_specs(state_in, state_out, state_index, S, f32, (H * V, K))
    _all_here(specs + state + [(A, "A", f32, H, True), (dt_bias, "dt_bias", f32, H, True), (status, "status", i32, 1, False)],
              "q k v b dt y", q, k, v, b, dt, y)
    args = _pack_delta(_DTYPES[typ], S, T, H, G, K, V, 1 if softplus else 0, 1 if sigmoid else 0, rows,
                       scale, _at(offsets), _at(state_index), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                       b.data_ptr(), _at(dt), q_ld, k_ld, v_ld, b_ld, dt_ld, _at(A), _at(dt_bias), _at(state_in),
                       _at(state_out), y.data_ptr(), y_ld)
    lib = load()
    if step:
        return lib.cortex_delta_step(args, status.data_ptr(), _stream(stream))
    return lib.cortex_delta_forward(args, status.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream))


def cortex_delta_workspace_bytes(T: int, S: int, H: int, K: int, V: int) -> int:
    return load().cortex_delta_workspace_bytes(T, S, H, K, V)


def cortex_delta_segment_tokens(T: int, S: int, H: int, K: int, V: int) -> int:
    return load().cortex_delta_segment_tokens(T, S, H, K, V)


def cortex_delta_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, b: torch.Tensor, offsets: torch.Tensor,
                         y: torch.Tensor, *, dt=None, A=None, dt_bias=None, softplus: bool = True, sigmoid: bool = True,
                         scale: float = 1.0, state_in=None, state_out=None, state_index=None,
                         status: torch.Tensor = None, ws: torch.Tensor = None, stream=None) -> int:
    """q, k [T, key heads, K]; v, y [T, H, V]; b, dt [T, H]; A, dt_bias [H]; states [rows, H V, K]."""
    return _delta(False, q, k, v, b, offsets, y, dt, A, dt_bias, softplus, sigmoid, scale, state_in, state_out, state_index,
                  status, ws, stream)


def cortex_delta_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, b: torch.Tensor, y: torch.Tensor, *, dt=None,
                      A=None, dt_bias=None, softplus: bool = True, sigmoid: bool = True, scale: float = 1.0, state_in=None,
                      state_out=None, state_index=None, status: torch.Tensor = None, stream=None) -> int:
    """One token of each of S sequences: q, k [S, key heads, K] and the others likewise."""
    return _delta(True, q, k, v, b, None, y, dt, A, dt_bias, softplus, sigmoid, scale, state_in, state_out, state_index,
                  status, None, stream)


def cortex_qk_norm(q: torch.Tensor, q_out: torch.Tensor, *, k=None, k_out=None, norm: int = CORTEX_NORM_RMS,
                   eps: float = 1e-6, q_weight=None, k_weight=None, positions=None, freqs=None, interleaved: bool = False,
                   status: torch.Tensor = None, stream=None) -> int:
    """q, q_out [T, H, P]; k, k_out [T, key heads, P]; weights [P]; positions [T]; freqs [R / 2]."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.dtype not in _DTYPES:
        raise ValueError("q must be a [T, H, P] torch.Tensor of torch.float32 or torch.bfloat16")
    if not isinstance(norm, int):
        raise ValueError("norm must be one of CORTEX_NORM_*, got %r" % (norm,))
    eps = _number(eps, "eps")
    T, typ, f32 = q.shape[0], q.dtype, torch.float32
    H, P, q_ld = _head_rows(q, "q", typ, T)
    _, _, qo_ld = _head_rows(q_out, "q_out", typ, T, (H, P))
    G = k_ld = ko_ld = R = 0
    if k is not None:
        G, K, k_ld = _head_rows(k, "k", typ, T)
        if K != P:
            raise ValueError("k must be [%d, heads, %d], got %s" % (T, P, list(k.shape)))
        _, _, ko_ld = _head_rows(k_out, "k_out", typ, T, (G, P))
    elif k_out is not None or k_weight is not None:
        raise ValueError("k is required with k_out and k_weight")
    if freqs is not None:
        if not isinstance(freqs, torch.Tensor):
            raise ValueError("freqs must be a torch.Tensor, got %s" % type(freqs).__name__)
        R = 2 * freqs.numel()
    elif positions is not None:
        raise ValueError("freqs is required with positions")
    _all_here([(q_weight, "q_weight", f32, P, True), (k_weight, "k_weight", f32, P, True),
               (positions, "positions", torch.int32, T, freqs is None), (freqs, "freqs", f32, 0, True),
               (status, "status", torch.int32, 1, False)], "q q_out k k_out", q, q_out, k, k_out)
    args = _pack_qk_norm(_DTYPES[typ], T, H, G, P, R, 1 if interleaved else 0, norm, eps, q.data_ptr(), _at(k),
                         q_ld, k_ld, _at(q_weight), _at(k_weight), _at(positions), _at(freqs), q_out.data_ptr(), _at(k_out),
                         qo_ld, ko_ld)
    return load().cortex_qk_norm(args, status.data_ptr(), _stream(stream))


def cortex_quant_i8(x: torch.Tensor, q: torch.Tensor, scale: torch.Tensor, *, status: torch.Tensor = None,
                    stream=None) -> int:
    """x [rows, columns] to q (int8) of the same shape and scale [rows]."""
    rows, cols = _shape2(x, "x")
    x_ld, q_ld = _rows(x, "x", x.dtype, rows, cols), _rows(q, "q", torch.int8, rows, cols)
    _all_here([(scale, "scale", torch.float32, rows, False), (status, "status", torch.int32, 1, False)], "x q", x, q)
    args = _pack_quant(_DTYPES[x.dtype], rows, cols, x.data_ptr(), x_ld, q.data_ptr(), q_ld, scale.data_ptr())
    return load().cortex_quant_i8(args, status.data_ptr(), _stream(stream))


def cortex_linear_i8_workspace_bytes(T: int, N: int, K: int) -> int:
    return load().cortex_linear_i8_workspace_bytes(T, N, K)


def cortex_linear_i8(x: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, y: torch.Tensor, *, x_scale=None, bias=None,
                     status: torch.Tensor = None, ws: torch.Tensor = None, stream=None) -> int:
    """x [T, K] of y's type, or int8 with x_scale [T]; w [N, K] int8 in rows that start at
    16-byte boundaries; w_scale, bias [N]; y [T, N]."""
    T, N = _shape2(y, "y")
    f32, i8 = torch.float32, torch.int8
    if not isinstance(w, torch.Tensor) or w.dim() != 2:
        raise ValueError("w must be a 2-dimensional torch.Tensor")
    K = w.shape[1]
    w_ld = _rows(w, "w", i8, N, K)
    if N == 1:                         # its stride is never used
        w_ld = (K + 15) // 16 * 16
    x_ld, y_ld = _rows(x, "x", y.dtype if x_scale is None else i8, T, K), _rows(y, "y", y.dtype, T, N)
    if w_ld % 16 or w.data_ptr() % 16:
        raise ValueError("w must have rows that start at 16-byte boundaries")
    if K % 16 and N > 0 and w.storage_offset() + (N - 1) * w_ld + (K + 15) // 16 * 16 > w.untyped_storage().nbytes():
        raise ValueError("w must hold whole pieces of 16 bytes, its last row too")
    _all_here([(w_scale, "w_scale", f32, N, False), (x_scale, "x_scale", f32, T, True), (bias, "bias", f32, N, True),
               (status, "status", torch.int32, 1, False), (ws, "ws", None, 1, False)], "x w y", x, w, y)
    args = _pack_linear(_DTYPES[y.dtype], T, K, N, x.data_ptr(), x_ld, _at(x_scale), w.data_ptr(), w_ld, w_scale.data_ptr(),
                        _at(bias), y.data_ptr(), y_ld)
    return load().cortex_linear_i8(args, status.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream))


def cortex_version() -> str:
    return load().cortex_version().decode()


# ---- device-memory plumbing ---------------------------------------------------

@dataclass
class Linearization:
    """Caller-owned device arrays of a linearization (cortex_lin_t)."""
    N: int
    K: int
    num_levels: torch.Tensor
    height: torch.Tensor
    level_offsets: torch.Tensor
    level_nodes: torch.Tensor
    node_row: torch.Tensor
    child_rows: torch.Tensor

    def __post_init__(self):
        sizes = {"num_levels": 1, "height": self.N, "level_offsets": self.N + 1, "level_nodes": self.N,
                 "node_row": self.N, "child_rows": self.N * self.K}
        for name, n in sizes.items():
            _need(getattr(self, name), name, torch.int32, n)
        self.struct = cortex_lin_t(self.N, self.K, _ptr(self.num_levels), _ptr(self.height),
                                   _ptr(self.level_offsets), _ptr(self.level_nodes),
                                   _ptr(self.node_row), _ptr(self.child_rows))

    @staticmethod
    def alloc(N: int, K: int, device="cuda") -> "Linearization":
        e = lambda n: torch.empty(max(n, 1), dtype=torch.int32, device=device)
        return Linearization(N, K, e(1), e(N), e(N + 1), e(N), e(N), e(N * K))


def workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """Zero-filled workspace (the library requires zeros before first use)."""
    return torch.zeros(max(1, (nbytes + 255) // 256 * 256), dtype=torch.uint8, device=device)


def check(rc: int, what: str = "cortex call") -> None:
    if rc != CORTEX_OK:
        raise RuntimeError("%s failed with host code %d" % (what, rc))
