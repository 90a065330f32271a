"""Thin Python binding of the C ABI in ``include/fold.h`` (ctypes).

Argument marshalling only: every step of the hot path runs in the HIP library.
PyTorch provides device memory (``tensor.data_ptr()``) and streams
(``torch.cuda.current_stream().cuda_stream``).  If ``libfold.so`` is missing the
binding raises -- there is no fallback.

The functions keep the ABI's names:
    fold_schedule, fold_sched_get_info, fold_sched_free, fold_trim,
    fold_pack_params, fold_packed_free, fold_workspace_size,
    fold_forward, fold_backward, fold_row_ld, fold_last_error,
    fold_graph_create, fold_graph_launch, fold_graph_num_nodes, fold_graph_free,
    fold_vocab_logits, fold_vocab_backward, fold_loss_distill, fold_token_logprobs,
    fold_layer_norm, fold_layer_norm_backward, fold_linear, fold_linear_backward,
    fold_cross_create, fold_cross_free, fold_cross_workspace_size, fold_cross_attend, fold_cross_backward
``Schedule`` / ``Packed`` / ``StepGraph`` / ``VocabHead`` / ``Linear`` / ``CrossAttention``, ``distill_loss``,
``token_logprobs``, ``layer_norm`` and ``layer_norm_backward`` wrap them for tensors.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
from ctypes import POINTER, byref, c_int32, c_int64, c_size_t, c_void_p
from typing import NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfold.so")

FOLD_OK = 0
ERRORS = {-1: "FOLD_E_INVALID", -2: "FOLD_E_OP", -3: "FOLD_E_ARITY", -4: "FOLD_E_CHILD",
          -5: "FOLD_E_INPUT", -6: "FOLD_E_CYCLE", -7: "FOLD_E_NOMEM", -8: "FOLD_E_DEVICE",
          -9: "FOLD_E_MISMATCH"}
FOLD_E_INVALID, FOLD_E_OP, FOLD_E_ARITY, FOLD_E_CHILD, FOLD_E_INPUT, FOLD_E_CYCLE = -1, -2, -3, -4, -5, -6
FOLD_E_NOMEM, FOLD_E_DEVICE, FOLD_E_MISMATCH = -7, -8, -9
FOLD_EMBED, FOLD_TREERNN, FOLD_TREELSTM, FOLD_LSTM, FOLD_PROJ = 0, 1, 2, 3, 4
FOLD_ATTN_SCORE, FOLD_ATTN_SUM, FOLD_ATTN_OUT = 5, 6, 7
FOLD_F32, FOLD_BF16 = 0, 1
GATES = {FOLD_EMBED: 0, FOLD_TREERNN: 1, FOLD_TREELSTM: 5, FOLD_LSTM: 4, FOLD_PROJ: 1,
         FOLD_ATTN_SCORE: 0, FOLD_ATTN_SUM: 0, FOLD_ATTN_OUT: 0}


class fold_op(ctypes.Structure):
    _fields_ = [("kind", c_int32), ("arity", c_int32), ("has_input", c_int32), ("param_set", c_int32)]


class fold_batch(ctypes.Structure):
    _fields_ = [("num_graphs", c_int32), ("num_nodes", c_int32), ("num_edges", c_int32),
                ("num_ops", c_int32), ("num_inputs", c_int32),
                ("graph_ptr", c_void_p), ("node_op", c_void_p), ("child_ptr", c_void_p),
                ("child_idx", c_void_p), ("node_input", c_void_p), ("ops", POINTER(fold_op))]


_I32P = c_void_p


class fold_sched_info(ctypes.Structure):
    _fields_ = [("num_nodes", c_int32), ("num_edges", c_int32), ("num_graphs", c_int32),
                ("num_ops", c_int32), ("num_levels", c_int32), ("num_groups", c_int32),
                ("num_roots", c_int32), ("max_parents", c_int32),
                ("depth", _I32P), ("node_pos", _I32P), ("pos_node", _I32P), ("level_ptr", _I32P),
                ("group_level", _I32P), ("group_op", _I32P), ("group_row_begin", _I32P),
                ("group_rows", _I32P), ("group_idx_off", _I32P), ("child_pos", _I32P),
                ("input_idx", _I32P), ("root_pos", _I32P),
                ("h_level_ptr", POINTER(c_int32)), ("h_group_level", POINTER(c_int32)),
                ("h_group_op", POINTER(c_int32)), ("h_group_row_begin", POINTER(c_int32)),
                ("h_group_rows", POINTER(c_int32)), ("h_group_idx_off", POINTER(c_int32)),
                ("group_child_base0", _I32P), ("group_child_base1", _I32P),
                ("h_group_child_base0", POINTER(c_int32)), ("h_group_child_base1", POINTER(c_int32))]


class fold_typed_op(ctypes.Structure):
    _fields_ = [("num_inputs", c_int32), ("num_outputs", c_int32), ("in_type", POINTER(c_int32)),
                ("out_type", POINTER(c_int32))]


class fold_typed_batch(ctypes.Structure):
    _fields_ = [("num_graphs", c_int32), ("num_nodes", c_int32), ("num_edges", c_int32), ("num_ops", c_int32),
                ("num_types", c_int32), ("graph_ptr", c_void_p), ("node_op", c_void_p), ("in_ptr", c_void_p),
                ("in_node", c_void_p), ("in_slot", c_void_p), ("ops", POINTER(fold_typed_op))]


class fold_typed_sched_info(ctypes.Structure):
    _fields_ = [("num_levels", c_int32), ("num_batches", c_int32), ("num_passes", c_int32),
                ("num_items", c_int32), ("num_gather", c_int32), ("num_ops", c_int32), ("num_types", c_int32),
                ("depth", _I32P), ("batch_depth", _I32P), ("batch_op", _I32P), ("batch_rows", _I32P),
                ("batch_gather_off", _I32P), ("batch_item_begin", _I32P), ("item_node", _I32P),
                ("gather", _I32P), ("pass_node", _I32P), ("pass_slot", _I32P), ("pass_depth", _I32P),
                ("state_size", _I32P), ("edge_index", _I32P),
                ("h_batch_depth", POINTER(c_int32)), ("h_batch_op", POINTER(c_int32)),
                ("h_batch_rows", POINTER(c_int32)), ("h_batch_gather_off", POINTER(c_int32)),
                ("h_state_size", POINTER(c_int32))]


class fold_param_set(ctypes.Structure):
    _fields_ = [("kind", c_int32), ("in_dim", c_int32), ("arity", c_int32),
                ("W_in", c_void_p), ("W_rec", c_void_p), ("bias", c_void_p)]


class fold_params(ctypes.Structure):
    _fields_ = [("dtype", c_int32), ("hidden", c_int32), ("num_sets", c_int32),
                ("sets", POINTER(fold_param_set))]


class fold_param_grads(ctypes.Structure):
    _fields_ = [("dW_in", c_void_p), ("dW_rec", c_void_p), ("dbias", c_void_p)]


class fold_grads(ctypes.Structure):
    _fields_ = [("num_sets", c_int32), ("sets", POINTER(fold_param_grads)), ("d_leaf_table", c_void_p)]


class fold_step_buffers(ctypes.Structure):
    _fields_ = [("leaf_table", c_void_p), ("leaf_rows", c_int64), ("h_pool", c_void_p), ("c_pool", c_void_p),
                ("roots_out", c_void_p), ("dh_roots", c_void_p), ("dh_nodes", c_void_p),
                ("grads", POINTER(fold_grads)), ("dh_out", c_void_p), ("dc_out", c_void_p),
                ("ws", c_void_p), ("ws_bytes", c_size_t)]


FOLD_STEP_BACKWARD, FOLD_STEP_ZERO_GRADS = 1, 2
FOLD_VOCAB_ACCUMULATE = 1
FOLD_ACT_NONE, FOLD_ACT_RELU, FOLD_ACT_TANH, FOLD_ACT_GELU = 0, 1, 2, 3
FOLD_BLOCK_ACCUMULATE = 1
ACTIVATIONS = {"none": FOLD_ACT_NONE, "relu": FOLD_ACT_RELU, "tanh": FOLD_ACT_TANH, "gelu": FOLD_ACT_GELU}


class fold_cross_batch(ctypes.Structure):
    _fields_ = [("dtype", c_int32), ("heads", c_int32), ("kv_heads", c_int32), ("head_dim", c_int32),
                ("num_seqs", c_int32), ("num_sources", c_int32), ("num_queries", c_int32), ("num_keys", c_int32),
                ("num_query_rows", c_int32), ("num_key_rows", c_int32), ("query_ptr", c_void_p), ("query_row", c_void_p),
                ("key_ptr", c_void_p), ("key_row", c_void_p), ("source", c_void_p)]


class fold_kernel_stat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("launches", c_int64), ("total_ms", ctypes.c_double),
                ("max_ms", ctypes.c_double)]


class fold_launch_time(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("group", c_int32), ("op", c_int32), ("ms", ctypes.c_double)]


class FoldError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


EXPORTS = ["fold_schedule", "fold_sched_get_info", "fold_sched_free", "fold_pack_params",
           "fold_packed_free", "fold_row_ld", "fold_workspace_size", "fold_forward",
           "fold_backward", "fold_last_error", "fold_profile_enable", "fold_profile_read",
           "fold_profile_read_launches",
           "fold_probe_mfma", "fold_probe_mfma_random", "fold_probe_copy", "fold_graph_create", "fold_graph_launch",
           "fold_graph_num_nodes", "fold_graph_free", "fold_pack_update", "fold_loss_softmax_ce",
           "fold_loss_workspace_size", "fold_adam_step", "fold_forward_dropout", "fold_backward_dropout",
           "fold_dropout_mask", "fold_forward_noalloc", "fold_schedule_typed", "fold_typed_sched_get_info",
           "fold_typed_sched_free", "fold_level_launches", "fold_trim", "fold_vocab_logits", "fold_vocab_backward",
           "fold_vocab_workspace_size", "fold_loss_distill", "fold_distill_workspace_size", "fold_token_logprobs",
           "fold_token_workspace_size", "fold_layer_norm", "fold_layer_norm_workspace_size", "fold_layer_norm_backward",
           "fold_linear", "fold_linear_workspace_size", "fold_linear_backward", "fold_cross_create",
           "fold_cross_free", "fold_cross_workspace_size", "fold_cross_attend", "fold_cross_backward"]

_lib = None


def lib():
    """Load libfold.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_1702_02181_amd.build_lib.build()")
    # torch first: its HIP runtime (same soname) is then the one the library's calls reach.  Loaded the other
    # way round, the process would map two HIP runtimes and the library's would see no device.
    import torch  # noqa: F401
    L = ctypes.CDLL(LIB_PATH)
    L.fold_last_error.restype = ctypes.c_char_p
    L.fold_last_error.argtypes = []
    L.fold_row_ld.restype = c_int32
    L.fold_row_ld.argtypes = [c_int32]
    L.fold_schedule.restype = c_int32
    L.fold_schedule.argtypes = [POINTER(fold_batch), c_void_p, POINTER(c_void_p)]
    L.fold_sched_get_info.restype = c_int32
    L.fold_sched_get_info.argtypes = [c_void_p, POINTER(fold_sched_info)]
    L.fold_sched_free.restype = c_int32
    L.fold_sched_free.argtypes = [c_void_p]
    L.fold_trim.restype = c_int32
    L.fold_trim.argtypes = [POINTER(c_size_t)]
    L.fold_pack_params.restype = c_int32
    L.fold_pack_params.argtypes = [POINTER(fold_params), c_void_p, POINTER(c_void_p)]
    L.fold_packed_free.restype = c_int32
    L.fold_packed_free.argtypes = [c_void_p]
    L.fold_workspace_size.restype = c_int32
    L.fold_workspace_size.argtypes = [c_void_p, c_void_p, POINTER(c_size_t), POINTER(c_size_t)]
    L.fold_forward.restype = c_int32
    L.fold_forward.argtypes = [c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p,
                               c_void_p, c_size_t, c_void_p]
    L.fold_backward.restype = c_int32
    L.fold_backward.argtypes = [c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p,
                                c_void_p, POINTER(fold_grads), c_void_p, c_void_p, c_void_p, c_size_t,
                                c_void_p]
    L.fold_forward_dropout.restype = c_int32
    L.fold_forward_dropout.argtypes = [c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p,
                                       c_void_p, c_void_p, c_size_t, c_void_p]
    L.fold_backward_dropout.restype = c_int32
    L.fold_backward_dropout.argtypes = [c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p,
                                        c_void_p, c_void_p, POINTER(fold_grads), c_void_p, c_void_p, c_void_p,
                                        c_size_t, c_void_p]
    L.fold_level_launches.restype = c_int32
    L.fold_level_launches.argtypes = [c_int32]
    L.fold_schedule_typed.restype = c_int32
    L.fold_schedule_typed.argtypes = [POINTER(fold_typed_batch), c_void_p, POINTER(c_void_p)]
    L.fold_typed_sched_get_info.restype = c_int32
    L.fold_typed_sched_get_info.argtypes = [c_void_p, POINTER(fold_typed_sched_info)]
    L.fold_typed_sched_free.restype = c_int32
    L.fold_typed_sched_free.argtypes = [c_void_p]
    L.fold_forward_noalloc.restype = c_int32
    L.fold_forward_noalloc.argtypes = [c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p]
    L.fold_dropout_mask.restype = c_int32
    L.fold_dropout_mask.argtypes = [c_void_p, c_int32, ctypes.c_double, ctypes.c_uint64, ctypes.c_uint64, c_void_p,
                                    c_void_p]
    L.fold_graph_create.restype = c_int32
    L.fold_graph_create.argtypes = [c_void_p, c_void_p, POINTER(fold_step_buffers), c_int32, POINTER(c_void_p)]
    L.fold_graph_launch.restype = c_int32
    L.fold_graph_launch.argtypes = [c_void_p, c_void_p]
    L.fold_graph_num_nodes.restype = c_int32
    L.fold_graph_num_nodes.argtypes = [c_void_p, POINTER(c_int32)]
    L.fold_graph_free.restype = c_int32
    L.fold_graph_free.argtypes = [c_void_p]
    L.fold_profile_enable.restype = c_int32
    L.fold_profile_enable.argtypes = [c_int32]
    L.fold_profile_read.restype = c_int32
    L.fold_profile_read.argtypes = [POINTER(fold_kernel_stat), c_int32, POINTER(c_int32)]
    L.fold_profile_read_launches.restype = c_int32
    L.fold_profile_read_launches.argtypes = [POINTER(fold_launch_time), c_int32, POINTER(c_int32)]
    L.fold_probe_mfma.restype = c_int32
    L.fold_probe_mfma.argtypes = [c_int32, c_void_p, POINTER(ctypes.c_double)]
    L.fold_probe_mfma_random.restype = c_int32
    L.fold_probe_mfma_random.argtypes = [c_int32, c_void_p, POINTER(ctypes.c_double)]
    L.fold_probe_copy.restype = c_int32
    L.fold_probe_copy.argtypes = [c_void_p, c_void_p, c_size_t, c_void_p, POINTER(ctypes.c_double)]
    L.fold_pack_update.restype = c_int32
    L.fold_pack_update.argtypes = [c_void_p, POINTER(fold_params), c_void_p]
    L.fold_loss_softmax_ce.restype = c_int32
    L.fold_loss_softmax_ce.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                       ctypes.c_float, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                       c_void_p]
    L.fold_loss_workspace_size.restype = c_int32
    L.fold_loss_workspace_size.argtypes = [c_void_p, c_int32, POINTER(c_size_t)]
    L.fold_adam_step.restype = c_int32
    L.fold_adam_step.argtypes = [c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, ctypes.c_double,
                                 ctypes.c_double, ctypes.c_double, ctypes.c_double, c_int32, c_void_p]
    L.fold_vocab_logits.restype = c_int32
    L.fold_vocab_logits.argtypes = [c_int32, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_void_p,
                                    c_void_p]
    L.fold_vocab_workspace_size.restype = c_int32
    L.fold_vocab_workspace_size.argtypes = [c_int32, c_int64, c_int32, c_int32, POINTER(c_size_t)]
    L.fold_vocab_backward.restype = c_int32
    L.fold_vocab_backward.argtypes = [c_int32, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                      c_void_p, c_void_p, c_int32, c_void_p, c_size_t, c_void_p]
    L.fold_distill_workspace_size.restype = c_int32
    L.fold_distill_workspace_size.argtypes = [c_int32, c_int64, c_int32, c_int32, POINTER(c_size_t)]
    L.fold_loss_distill.restype = c_int32
    L.fold_loss_distill.argtypes = [c_void_p, c_int32, c_int64, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_void_p,
                                    ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float, c_void_p, c_int32,
                                    c_void_p, c_void_p, c_size_t, c_void_p]
    L.fold_token_workspace_size.restype = c_int32
    L.fold_token_workspace_size.argtypes = [c_int32, c_int64, c_int32, c_int32, POINTER(c_size_t)]
    L.fold_token_logprobs.restype = c_int32
    L.fold_token_logprobs.argtypes = [c_void_p, c_int32, c_int64, c_int32, c_void_p, c_int32, c_void_p, c_void_p,
                                      c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    L.fold_layer_norm.restype = c_int32
    L.fold_layer_norm.argtypes = [c_int32, c_int64, c_int32, c_void_p, c_void_p, c_void_p, ctypes.c_float, c_void_p,
                                  c_void_p, c_void_p, c_void_p]
    L.fold_layer_norm_workspace_size.restype = c_int32
    L.fold_layer_norm_workspace_size.argtypes = [c_int32, c_int64, c_int32, POINTER(c_size_t)]
    L.fold_layer_norm_backward.restype = c_int32
    L.fold_layer_norm_backward.argtypes = [c_int32, c_int64, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_int32,
                                           c_void_p, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_void_p,
                                           c_size_t, c_void_p]
    L.fold_linear.restype = c_int32
    L.fold_linear.argtypes = [c_int32, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_void_p,
                              c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    L.fold_linear_workspace_size.restype = c_int32
    L.fold_linear_workspace_size.argtypes = [c_int32, c_int64, c_int32, c_int32, POINTER(c_size_t), POINTER(c_size_t)]
    L.fold_linear_backward.restype = c_int32
    L.fold_linear_backward.argtypes = [c_int32, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                       c_void_p, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_int32, c_void_p,
                                       c_size_t, c_void_p]
    L.fold_cross_create.restype = c_int32
    L.fold_cross_create.argtypes = [POINTER(fold_cross_batch), c_void_p, POINTER(c_void_p)]
    L.fold_cross_free.restype = c_int32
    L.fold_cross_free.argtypes = [c_void_p]
    L.fold_cross_workspace_size.restype = c_int32
    L.fold_cross_workspace_size.argtypes = [c_void_p, POINTER(c_size_t), POINTER(c_size_t)]
    L.fold_cross_attend.restype = c_int32
    L.fold_cross_attend.argtypes = [c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                                    ctypes.c_float, c_void_p, c_int64, c_void_p, c_void_p, c_size_t, c_void_p]
    L.fold_cross_backward.restype = c_int32
    L.fold_cross_backward.argtypes = [c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                                      ctypes.c_float, c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_void_p, c_int64,
                                      c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_size_t, c_void_p]
    _lib = L
    return L


def _check(rc: int):
    if rc != FOLD_OK:
        raise FoldError(rc, lib().fold_last_error().decode())


def fold_last_error() -> str:
    return lib().fold_last_error().decode()


def fold_profile_enable(on: bool):
    _check(lib().fold_profile_enable(1 if on else 0))


def fold_profile_read() -> dict:
    """{kernel class: (launches, total_ms, max_ms)}; waits for the recorded events and clears them."""
    cap = 128
    arr = (fold_kernel_stat * cap)()
    n = c_int32()
    _check(lib().fold_profile_read(arr, cap, byref(n)))
    return {arr[i].name.decode(): (int(arr[i].launches), float(arr[i].total_ms), float(arr[i].max_ms))
            for i in range(min(n.value, cap))}


def fold_profile_read_launches() -> list:
    """[(kernel class, group, op, ms)] in launch order; waits for the recorded events and clears them."""
    n = c_int32()
    _check(lib().fold_profile_read_launches(None, 0, byref(n)))  # count only
    cap = n.value
    arr = (fold_launch_time * max(cap, 1))()
    _check(lib().fold_profile_read_launches(arr, cap, byref(n)) if cap else 0)
    return [(arr[i].name.decode(), int(arr[i].group), int(arr[i].op), float(arr[i].ms))
            for i in range(min(n.value, cap))]


def fold_probe_mfma(dtype: int, stream=None) -> float:
    t = ctypes.c_double()
    _check(lib().fold_probe_mfma(int(dtype), _stream(stream), byref(t)))
    return float(t.value)


def fold_probe_mfma_random(dtype: int, stream=None) -> float:
    t = ctypes.c_double()
    _check(lib().fold_probe_mfma_random(int(dtype), _stream(stream), byref(t)))
    return float(t.value)


def fold_probe_copy(dst, src, nbytes: int, stream=None) -> float:
    g = ctypes.c_double()
    _check(lib().fold_probe_copy(_ptr(dst), _ptr(src), int(nbytes), _stream(stream), byref(g)))
    return float(g.value)


def fold_row_ld(width: int) -> int:
    return int(lib().fold_row_ld(int(width)))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


# ----------------------------------------------------------------------------- raw calls

def fold_schedule(batch: fold_batch, stream=None) -> c_void_p:
    h = c_void_p()
    _check(lib().fold_schedule(byref(batch), _stream(stream), byref(h)))
    return h


def fold_sched_get_info(handle) -> fold_sched_info:
    info = fold_sched_info()
    _check(lib().fold_sched_get_info(handle, byref(info)))
    return info


def fold_sched_free(handle):
    _check(lib().fold_sched_free(handle))


def fold_trim() -> int:
    """Give back the device memory that the library keeps between schedules; the bytes given back.  (PyTorch's allocator
    cannot reclaim it by itself.)"""
    n = c_size_t()
    _check(lib().fold_trim(byref(n)))
    return int(n.value)


def fold_pack_params(params: fold_params, stream=None) -> c_void_p:
    h = c_void_p()
    _check(lib().fold_pack_params(byref(params), _stream(stream), byref(h)))
    return h


def fold_pack_update(handle, params: fold_params, stream=None):
    _check(lib().fold_pack_update(handle, byref(params), _stream(stream)))


def fold_loss_workspace_size(packed, num_classes) -> int:
    n = c_size_t()
    _check(lib().fold_loss_workspace_size(packed, int(num_classes), byref(n)))
    return int(n.value)


def fold_loss_softmax_ce(sched, packed, h_pool, labels, num_classes, W_cls, b_cls, scale, node_loss, dh_nodes,
                         dW_cls, db_cls, ws, ws_bytes, stream=None):
    _check(lib().fold_loss_softmax_ce(sched, packed, _ptr(h_pool), _ptr(labels), int(num_classes), _ptr(W_cls),
                                      _ptr(b_cls), float(scale), _ptr(node_loss), _ptr(dh_nodes), _ptr(dW_cls),
                                      _ptr(db_cls), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_adam_step(n, param, param_bf16, grad, m, v, lr, beta1, beta2, eps, step, stream=None):
    _check(lib().fold_adam_step(int(n), _ptr(param), _ptr(param_bf16), _ptr(grad), _ptr(m), _ptr(v), float(lr),
                                float(beta1), float(beta2), float(eps), int(step), _stream(stream)))


def fold_level_launches(on) -> bool:
    """Turn level launches on or off for later calls; returns the previous setting."""
    return bool(lib().fold_level_launches(1 if on else 0))


def fold_forward_noalloc(sched, packed, table, table_rows, h_pool, c_pool, roots, stream=None):
    _check(lib().fold_forward_noalloc(sched, packed, _ptr(table), int(table_rows), _ptr(h_pool), _ptr(c_pool),
                                      _ptr(roots), _stream(stream)))


def fold_dropout_mask(sched, hidden, p, seed, step, mask, stream=None):
    _check(lib().fold_dropout_mask(sched, int(hidden), float(p), int(seed) & (2 ** 64 - 1), int(step) & (2 ** 64 - 1),
                                   _ptr(mask), _stream(stream)))


def fold_vocab_logits(dtype, rows, hidden, vocab, states, W, bias, logits_dtype, logits, stream=None):
    _check(lib().fold_vocab_logits(int(dtype), int(rows), int(hidden), int(vocab), _ptr(states), _ptr(W), _ptr(bias),
                                   int(logits_dtype), _ptr(logits), _stream(stream)))


def fold_vocab_workspace_size(dtype, rows, hidden, vocab) -> int:
    n = c_size_t()
    _check(lib().fold_vocab_workspace_size(int(dtype), int(rows), int(hidden), int(vocab), byref(n)))
    return int(n.value)


def fold_vocab_backward(dtype, rows, hidden, vocab, states, W, dlogits, d_states, dW, dbias, flags, ws, ws_bytes,
                        stream=None):
    _check(lib().fold_vocab_backward(int(dtype), int(rows), int(hidden), int(vocab), _ptr(states), _ptr(W),
                                     _ptr(dlogits), _ptr(d_states), _ptr(dW), _ptr(dbias), int(flags), _ptr(ws),
                                     int(ws_bytes), _stream(stream)))


def fold_distill_workspace_size(dtype, rows, vocab, num_teacher) -> int:
    n = c_size_t()
    _check(lib().fold_distill_workspace_size(int(dtype), int(rows), int(vocab), int(num_teacher), byref(n)))
    return int(n.value)


def fold_loss_distill(sched, dtype, rows, vocab, logits, num_teacher, teacher_token, teacher_logit, labels, temperature,
                      soft_weight, hard_weight, scale, row_loss, grad_dtype, dlogits, ws, ws_bytes, stream=None):
    _check(lib().fold_loss_distill(sched, int(dtype), int(rows), int(vocab), _ptr(logits), int(num_teacher),
                                   _ptr(teacher_token), _ptr(teacher_logit), _ptr(labels), float(temperature),
                                   float(soft_weight), float(hard_weight), float(scale), _ptr(row_loss),
                                   int(grad_dtype), _ptr(dlogits), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_token_workspace_size(dtype, rows, vocab, top_k) -> int:
    n = c_size_t()
    _check(lib().fold_token_workspace_size(int(dtype), int(rows), int(vocab), int(top_k), byref(n)))
    return int(n.value)


def fold_token_logprobs(sched, dtype, rows, vocab, logits, num_tokens, tokens, logp, entropy, top_k, top_token,
                        top_logp, ws, ws_bytes, stream=None):
    _check(lib().fold_token_logprobs(sched, int(dtype), int(rows), int(vocab), _ptr(logits), int(num_tokens),
                                     _ptr(tokens), _ptr(logp), _ptr(entropy), int(top_k), _ptr(top_token),
                                     _ptr(top_logp), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_layer_norm(dtype, rows, width, x, gamma, beta, eps, y, mean, rstd, stream=None):
    _check(lib().fold_layer_norm(int(dtype), int(rows), int(width), _ptr(x), _ptr(gamma), _ptr(beta), float(eps), _ptr(y),
                                 _ptr(mean), _ptr(rstd), _stream(stream)))


def fold_layer_norm_workspace_size(dtype, rows, width) -> int:
    n = c_size_t()
    _check(lib().fold_layer_norm_workspace_size(int(dtype), int(rows), int(width), byref(n)))
    return int(n.value)


def fold_layer_norm_backward(dtype, rows, width, x, gamma, mean, rstd, dy_dtype, dy, residual_dtype, residual, dx_dtype, dx,
                             dgamma, dbeta, flags, ws, ws_bytes, stream=None):
    _check(lib().fold_layer_norm_backward(int(dtype), int(rows), int(width), _ptr(x), _ptr(gamma), _ptr(mean), _ptr(rstd),
                                          int(dy_dtype), _ptr(dy), int(residual_dtype), _ptr(residual), int(dx_dtype),
                                          _ptr(dx), _ptr(dgamma), _ptr(dbeta), int(flags), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_linear(dtype, rows, in_dim, out_dim, x, W, bias, act, residual, out, pre, ws, ws_bytes, stream=None):
    _check(lib().fold_linear(int(dtype), int(rows), int(in_dim), int(out_dim), _ptr(x), _ptr(W), _ptr(bias), int(act),
                             _ptr(residual), _ptr(out), _ptr(pre), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_linear_workspace_size(dtype, rows, in_dim, out_dim):
    f, b = c_size_t(), c_size_t()
    _check(lib().fold_linear_workspace_size(int(dtype), int(rows), int(in_dim), int(out_dim), byref(f), byref(b)))
    return int(f.value), int(b.value)


def fold_linear_backward(dtype, rows, in_dim, out_dim, x, W, act, pre, dout, dpre, dx_dtype, dx, dw_dtype, dW, dbias, flags,
                         ws, ws_bytes, stream=None):
    _check(lib().fold_linear_backward(int(dtype), int(rows), int(in_dim), int(out_dim), _ptr(x), _ptr(W), int(act),
                                      _ptr(pre), _ptr(dout), _ptr(dpre), int(dx_dtype), _ptr(dx), int(dw_dtype), _ptr(dW),
                                      _ptr(dbias), int(flags), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_cross_create(batch: fold_cross_batch, stream=None) -> c_void_p:
    h = c_void_p()
    _check(lib().fold_cross_create(byref(batch), _stream(stream), byref(h)))
    return h


def fold_cross_free(handle):
    _check(lib().fold_cross_free(handle))


def fold_cross_workspace_size(cross):
    f, b = c_size_t(), c_size_t()
    _check(lib().fold_cross_workspace_size(cross, byref(f), byref(b)))
    return int(f.value), int(b.value)


def fold_cross_attend(cross, q, ldq, k, ldk, v, ldv, key_mask, scale, out, ldo, lse, ws, ws_bytes, stream=None):
    _check(lib().fold_cross_attend(cross, _ptr(q), int(ldq), _ptr(k), int(ldk), _ptr(v), int(ldv), _ptr(key_mask),
                                   float(scale), _ptr(out), int(ldo), _ptr(lse), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_cross_backward(cross, q, ldq, k, ldk, v, ldv, key_mask, scale, out, ldo, lse, dout, lddo, dq, lddq, dk, lddk, dv,
                        lddv, ws, ws_bytes, stream=None):
    _check(lib().fold_cross_backward(cross, _ptr(q), int(ldq), _ptr(k), int(ldk), _ptr(v), int(ldv), _ptr(key_mask),
                                     float(scale), _ptr(out), int(ldo), _ptr(lse), _ptr(dout), int(lddo), _ptr(dq), int(lddq),
                                     _ptr(dk), int(lddk), _ptr(dv), int(lddv), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_packed_free(handle):
    _check(lib().fold_packed_free(handle))


def fold_workspace_size(sched, packed):
    f, b = c_size_t(), c_size_t()
    _check(lib().fold_workspace_size(sched, packed, byref(f), byref(b)))
    return int(f.value), int(b.value)


def fold_forward(sched, packed, leaf_table, leaf_rows, h_pool, c_pool, roots_out, ws, ws_bytes, stream=None):
    _check(lib().fold_forward(sched, packed, _ptr(leaf_table), int(leaf_rows), _ptr(h_pool), _ptr(c_pool),
                              _ptr(roots_out), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_backward(sched, packed, leaf_table, leaf_rows, h_pool, c_pool, dh_roots, dh_nodes, grads,
                  dh_out, dc_out, ws, ws_bytes, stream=None):
    _check(lib().fold_backward(sched, packed, _ptr(leaf_table), int(leaf_rows), _ptr(h_pool), _ptr(c_pool),
                               _ptr(dh_roots), _ptr(dh_nodes), None if grads is None else byref(grads),
                               _ptr(dh_out), _ptr(dc_out), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_forward_dropout(sched, packed, leaf_table, leaf_rows, h_pool, c_pool, roots_out, u_mask, ws, ws_bytes,
                         stream=None):
    _check(lib().fold_forward_dropout(sched, packed, _ptr(leaf_table), int(leaf_rows), _ptr(h_pool), _ptr(c_pool),
                                      _ptr(roots_out), _ptr(u_mask), _ptr(ws), int(ws_bytes), _stream(stream)))


def fold_backward_dropout(sched, packed, leaf_table, leaf_rows, h_pool, c_pool, u_mask, dh_roots, dh_nodes, grads,
                          dh_out, dc_out, ws, ws_bytes, stream=None):
    _check(lib().fold_backward_dropout(sched, packed, _ptr(leaf_table), int(leaf_rows), _ptr(h_pool), _ptr(c_pool),
                                       _ptr(u_mask), _ptr(dh_roots), _ptr(dh_nodes),
                                       None if grads is None else byref(grads), _ptr(dh_out), _ptr(dc_out), _ptr(ws),
                                       int(ws_bytes), _stream(stream)))


def fold_graph_create(sched, packed, buffers: fold_step_buffers, flags: int) -> c_void_p:
    h = c_void_p()
    _check(lib().fold_graph_create(sched, packed, byref(buffers), int(flags), byref(h)))
    return h


def fold_graph_launch(graph, stream=None):
    _check(lib().fold_graph_launch(graph, _stream(stream)))


def fold_graph_num_nodes(graph) -> int:
    n = c_int32()
    _check(lib().fold_graph_num_nodes(graph, byref(n)))
    return int(n.value)


def fold_graph_free(graph):
    _check(lib().fold_graph_free(graph))


# ----------------------------------------------------------------------------- tensor wrappers

def _dev_copy_to_host(ptr: int, count: int) -> np.ndarray:
    """Copy `count` int32 from a library-owned device array to host (the schedule call has synchronised)."""
    out = np.empty(count, dtype=np.int32)
    if count:
        rc = _hip().hipMemcpy(c_void_p(out.ctypes.data), c_void_p(ptr), c_size_t(4 * count), 2)
        if rc != 0:
            raise RuntimeError(f"hipMemcpy failed ({rc})")
    return out


_hiplib = None


def _hip():
    global _hiplib
    if _hiplib is None:
        _hiplib = ctypes.CDLL("libamdhip64.so")
        _hiplib.hipMemcpy.restype = ctypes.c_int
        _hiplib.hipMemcpy.argtypes = [c_void_p, c_void_p, c_size_t, ctypes.c_int]
        _hiplib.hipMemcpyAsync.restype = ctypes.c_int
        _hiplib.hipMemcpyAsync.argtypes = [c_void_p, c_void_p, c_size_t, ctypes.c_int, c_void_p]
    return _hiplib


class Schedule:
    """fold_schedule over int32 CUDA tensors; frees the handle when collected."""

    def __init__(self, graph_ptr, node_op, child_ptr, child_idx, node_input, ops, num_inputs, stream=None):
        self._keep = (graph_ptr, node_op, child_ptr, child_idx, node_input)
        self._ops = (fold_op * len(ops))(*[fold_op(*o) for o in ops])
        b = fold_batch()
        b.num_graphs = graph_ptr.numel() - 1
        b.num_nodes = node_op.numel()
        b.num_edges = child_idx.numel()
        b.num_ops = len(ops)
        b.num_inputs = int(num_inputs)
        b.graph_ptr, b.node_op, b.child_ptr = _ptr(graph_ptr), _ptr(node_op), _ptr(child_ptr)
        b.child_idx = _ptr(child_idx) if child_idx.numel() else c_void_p(graph_ptr.data_ptr())
        b.node_input = _ptr(node_input)
        b.ops = self._ops
        self.batch = b
        self.handle = fold_schedule(b, stream)
        self.info = fold_sched_get_info(self.handle)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            try:
                fold_sched_free(h)
            except Exception:
                pass
            self.handle = None

    @property
    def num_levels(self):
        return self.info.num_levels

    def host_groups(self) -> dict:
        i = self.info
        ng = i.num_groups

        def arr(p, n):
            return np.ctypeslib.as_array(p, shape=(n,)).copy() if n else np.zeros(0, np.int32)
        return dict(level_ptr=arr(i.h_level_ptr, i.num_levels + 1), group_level=arr(i.h_group_level, ng),
                    group_op=arr(i.h_group_op, ng), group_row_begin=arr(i.h_group_row_begin, ng),
                    group_rows=arr(i.h_group_rows, ng), group_idx_off=arr(i.h_group_idx_off, ng),
                    group_child_base0=arr(i.h_group_child_base0, ng),
                    group_child_base1=arr(i.h_group_child_base1, ng))

    def arrays(self) -> dict:
        """Every schedule array, copied to host numpy (device arrays and the host group table)."""
        i = self.info
        n, e, ng, D, R = i.num_nodes, i.num_edges, i.num_groups, i.num_levels, i.num_roots
        out = dict(num_levels=D, num_groups=ng, num_roots=R, max_parents=i.max_parents)
        for name, cnt in (("depth", n), ("node_pos", n), ("pos_node", n), ("level_ptr", D + 1),
                          ("group_level", ng), ("group_op", ng), ("group_row_begin", ng), ("group_rows", ng),
                          ("group_idx_off", ng), ("child_pos", e), ("input_idx", n), ("root_pos", R),
                          ("group_child_base0", ng), ("group_child_base1", ng)):
            p = getattr(i, name)
            out[name] = _dev_copy_to_host(p, cnt) if p else np.zeros(0, np.int32)
        out["host"] = self.host_groups()
        return out


class TypedSchedule:
    """fold_schedule_typed over CUDA int32 tensors (the paper's form: typed per-depth states, pass-throughs).
    ops: list of (in_types, out_types)."""

    def __init__(self, graph_ptr, node_op, in_ptr, in_node, in_slot, ops, num_types, stream=None):
        self._keep = [graph_ptr, node_op, in_ptr, in_node, in_slot]
        self._types = []
        arr = (fold_typed_op * len(ops))()
        for k, (ins, outs) in enumerate(ops):
            a = (c_int32 * max(1, len(ins)))(*ins)
            b = (c_int32 * max(1, len(outs)))(*outs)
            self._types += [a, b]
            arr[k] = fold_typed_op(len(ins), len(outs), a, b)
        self._ops = arr
        bt = fold_typed_batch(int(graph_ptr.numel()) - 1, int(node_op.numel()), int(in_node.numel()), len(ops),
                              int(num_types), _ptr(graph_ptr), _ptr(node_op), _ptr(in_ptr), _ptr(in_node),
                              _ptr(in_slot), arr)
        h = c_void_p()
        _check(lib().fold_schedule_typed(ctypes.byref(bt), _stream(stream), ctypes.byref(h)))
        self.handle = h
        self.info = fold_typed_sched_info()
        _check(lib().fold_typed_sched_get_info(h, ctypes.byref(self.info)))
        self.num_nodes, self.num_edges = int(node_op.numel()), int(in_node.numel())

    def __del__(self):
        if getattr(self, "handle", None) is not None and _lib is not None:
            _lib.fold_typed_sched_free(self.handle)
            self.handle = None

    def arrays(self) -> dict:
        i = self.info
        D, T, nb, P, M, G = i.num_levels, i.num_types, i.num_batches, i.num_passes, i.num_items, i.num_gather

        def dev(name, n):
            p = getattr(i, name)
            return _dev_copy_to_host(p, n) if (p and n) else np.zeros(0, np.int32)

        def host(p, n):
            return np.ctypeslib.as_array(p, shape=(n,)).copy() if n else np.zeros(0, np.int32)
        out = dict(num_levels=D, num_batches=nb, num_passes=P, num_items=M, num_gather=G)
        for name, n in (("depth", self.num_nodes), ("batch_depth", nb), ("batch_op", nb), ("batch_rows", nb),
                        ("batch_gather_off", nb), ("batch_item_begin", nb), ("item_node", M), ("gather", G),
                        ("pass_node", P), ("pass_slot", P), ("pass_depth", P), ("state_size", (D + 1) * T),
                        ("edge_index", self.num_edges)):
            out[name] = dev(name, n)
        out["host"] = dict(batch_depth=host(i.h_batch_depth, nb), batch_op=host(i.h_batch_op, nb),
                           batch_rows=host(i.h_batch_rows, nb), batch_gather_off=host(i.h_batch_gather_off, nb),
                           state_size=host(i.h_state_size, (D + 1) * T))
        return out


class Packed:
    """fold_pack_params over CUDA tensors (weights of the params' dtype, fp32 biases)."""

    def __init__(self, dtype: int, hidden: int, sets, stream=None):
        # sets: list of dict(kind, in_dim, arity, W_in, W_rec, bias) with tensors or None
        self._keep = sets
        arr = (fold_param_set * len(sets))()
        for k, s in enumerate(sets):
            arr[k] = fold_param_set(s["kind"], s["in_dim"], s["arity"], _ptr(s.get("W_in")),
                                    _ptr(s.get("W_rec")), _ptr(s.get("bias")))
        self._sets = arr
        p = fold_params(dtype, hidden, len(sets), arr)
        self.handle = fold_pack_params(p, stream)
        self.dtype, self.hidden, self.num_sets = dtype, hidden, len(sets)

    def update(self, sets, stream=None):
        """fold_pack_update: re-pack new values of the same parameters (same shapes) in place."""
        arr = (fold_param_set * len(sets))()
        for k, s in enumerate(sets):
            arr[k] = fold_param_set(s["kind"], s["in_dim"], s["arity"], _ptr(s.get("W_in")),
                                    _ptr(s.get("W_rec")), _ptr(s.get("bias")))
        fold_pack_update(self.handle, fold_params(self.dtype, self.hidden, len(sets), arr), stream)
        self._keep, self._sets = sets, arr

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            try:
                fold_packed_free(h)
            except Exception:
                pass
            self.handle = None


def make_grads(sets_tensors, d_leaf_table=None) -> fold_grads:
    """sets_tensors: list of (dW_in, dW_rec, dbias) fp32 CUDA tensors or None."""
    arr = (fold_param_grads * len(sets_tensors))()
    for k, (a, b, c) in enumerate(sets_tensors):
        arr[k] = fold_param_grads(_ptr(a), _ptr(b), _ptr(c))
    g = fold_grads(len(sets_tensors), arr, _ptr(d_leaf_table))
    g._keep = (arr, sets_tensors, d_leaf_table)
    return g


class StepGraph:
    """fold_graph_create over CUDA tensors: one recorded forward (+ backward) step.  Keeps every
    tensor it was built on alive; frees the graph when collected."""

    def __init__(self, sched, packed, leaf_table, leaf_rows, h_pool, c_pool, roots_out, ws, ws_bytes,
                 backward=False, dh_roots=None, dh_nodes=None, grads=None, dh_out=None, dc_out=None,
                 zero_grads=False):
        self._keep = (sched, packed, leaf_table, h_pool, c_pool, roots_out, ws, dh_roots, dh_nodes, grads,
                      dh_out, dc_out)
        b = fold_step_buffers()
        b.leaf_table, b.leaf_rows = _ptr(leaf_table), int(leaf_rows)
        b.h_pool, b.c_pool, b.roots_out = _ptr(h_pool), _ptr(c_pool), _ptr(roots_out)
        b.dh_roots, b.dh_nodes = _ptr(dh_roots), _ptr(dh_nodes)
        b.grads = None if grads is None else ctypes.pointer(grads)
        b.dh_out, b.dc_out = _ptr(dh_out), _ptr(dc_out)
        b.ws, b.ws_bytes = _ptr(ws), int(ws_bytes)
        flags = (FOLD_STEP_BACKWARD if backward else 0) | (FOLD_STEP_ZERO_GRADS if zero_grads else 0)
        self.handle = fold_graph_create(sched.handle, packed.handle, b, flags)
        self.num_nodes = fold_graph_num_nodes(self.handle)

    def launch(self, stream=None):
        fold_graph_launch(self.handle, stream)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            try:
                fold_graph_free(h)
            except Exception:
                pass
            self.handle = None


# ----------------------------------------------------------------------------- the vocabulary head

def _row_ld(width: int) -> int:
    return (width + 63) // 64 * 64


def _code(dtype) -> int:
    import torch
    if dtype == torch.float32:
        return FOLD_F32
    if dtype == torch.bfloat16:
        return FOLD_BF16
    raise ValueError(f"expected float32 or bfloat16, got {dtype}")


def _matrix(name, t, width, dtype=None, rows=None):
    """A dense matrix [rows, fold_row_ld(width)] on the current device, as the library reads it."""
    import torch
    if not (t.is_cuda and t.dim() == 2 and t.is_contiguous()):
        raise ValueError(f"{name}: a contiguous 2-D CUDA tensor is needed")
    if t.shape[1] != _row_ld(width):
        raise ValueError(f"{name}: rows of {_row_ld(width)} elements are needed (width {width}), got {t.shape[1]}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if rows is not None and t.shape[0] != rows:
        raise ValueError(f"{name}: expected {rows} rows, got {t.shape[0]}")
    _here(name, t)
    return t


def _vector(name, t, dtype, *shape):
    if not (t.is_cuda and t.is_contiguous()) or t.dtype != dtype or tuple(t.shape) != shape:
        raise ValueError(f"{name}: a contiguous CUDA tensor {list(shape)} of {dtype} is needed, got "
                         f"{list(t.shape)} of {t.dtype}")
    _here(name, t)
    return t


def _here(name, t):
    import torch
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{torch.cuda.current_device()}")


_HERE_STREAM = contextlib.nullcontext()


def _on(stream):
    """New tensors belong to the stream that the call runs on."""
    import torch
    if stream is None:
        return _HERE_STREAM
    _here("stream", stream)
    return torch.cuda.stream(stream)


class _Raw:
    """The current stream as the calls take it, without the object that torch.cuda.current_stream() makes (3 us, where a
    whole call on one row takes 15)."""

    @property
    def cuda_stream(self):
        import torch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


_CURRENT = _Raw()


# sizes by sizes: pure functions of their arguments
_vocab_ws = functools.lru_cache(256)(fold_vocab_workspace_size)
_distill_ws = functools.lru_cache(256)(fold_distill_workspace_size)
_token_ws = functools.lru_cache(256)(fold_token_workspace_size)


class VocabHead:
    """The head z = s W^T + bias of a vocabulary (fold_vocab_logits, fold_vocab_backward).

    weight: [vocab, fold_row_ld(hidden)], float32 or bfloat16, laid out as a leaf table (which may be it: tied
    weights); bias: [vocab] float32 or None.  Results and workspaces are new tensors of the calls' stream."""

    def __init__(self, weight, bias=None, hidden=None):
        import torch
        self.hidden = int(weight.shape[1] if hidden is None else hidden)
        self.weight = _matrix("weight", weight, self.hidden)
        self.vocab, self.dtype = int(weight.shape[0]), weight.dtype
        self.code = _code(weight.dtype)
        self.bias = None if bias is None else _vector("bias", bias, torch.float32, self.vocab)

    def logits(self, states, dtype=None, out=None, stream=None):
        """[rows, fold_row_ld(vocab)] logits of `states` [rows, fold_row_ld(hidden)], of dtype (the head's)."""
        import torch
        _matrix("states", states, self.hidden, self.dtype)
        _here("weight", self.weight)
        rows = states.shape[0]
        with _on(stream):
            if out is None:
                out = torch.empty((rows, _row_ld(self.vocab)), dtype=dtype or self.dtype, device=states.device)
            else:
                _matrix("out", out, self.vocab, dtype, rows)
            fold_vocab_logits(self.code, rows, self.hidden, self.vocab, states, self.weight, self.bias,
                              _code(out.dtype), out, stream or _CURRENT)
        return out

    def backward(self, states, dlogits, d_states=True, dW=True, dbias=True, accumulate=False, stream=None):
        """(d_states, dW, dbias) of `dlogits` [rows, fold_row_ld(vocab)].  Each of the three: True for a new tensor, a
        tensor to write, or None to leave it out.  accumulate: dW and dbias are added to the tensors given."""
        import torch
        _matrix("states", states, self.hidden, self.dtype)
        _here("weight", self.weight)
        rows = states.shape[0]
        _matrix("dlogits", dlogits, self.vocab, self.dtype, rows)
        if accumulate and (dW is True or dbias is True):
            raise ValueError("accumulate needs the dW and dbias to add to (or None)")
        f32 = dict(dtype=torch.float32, device=states.device)
        with _on(stream):
            if d_states is True:
                d_states = torch.empty((rows, _row_ld(self.hidden)), **f32)
            elif d_states is not None:
                _matrix("d_states", d_states, self.hidden, torch.float32, rows)
            if dW is True:
                dW = torch.empty((self.vocab, _row_ld(self.hidden)), **f32)
            elif dW is not None:
                _matrix("dW", dW, self.hidden, torch.float32, self.vocab)
            if dbias is True:
                dbias = torch.empty(self.vocab, **f32)
            elif dbias is not None:
                _vector("dbias", dbias, torch.float32, self.vocab)
            n = _vocab_ws(self.code, rows, self.hidden, self.vocab)
            ws = torch.empty(n, dtype=torch.uint8, device=states.device) if n else None
            fold_vocab_backward(self.code, rows, self.hidden, self.vocab, states, self.weight, dlogits, d_states, dW,
                                dbias, FOLD_VOCAB_ACCUMULATE if accumulate else 0, ws, n, stream or _CURRENT)
        return d_states, dW, dbias


def distill_loss(logits, vocab, teacher_token=None, teacher_logit=None, labels=None, temperature=1.0, soft_weight=1.0,
                 hard_weight=0.0, scale=1.0, dlogits=True, grad_dtype=None, sched=None, stream=None):
    """(losses [rows], gradient [rows, fold_row_ld(vocab)]) of fold_loss_distill.

    teacher_token, teacher_logit: [rows, num_teacher] int32, float32; labels: [rows] int32.  sched: a Schedule whose
    pool rows the logits are; targets and losses are then in node order.  dlogits: True for a new tensor (of grad_dtype,
    the logits' type by default), a tensor to write (the logits themselves, for one), or None for the losses alone."""
    import torch
    _matrix("logits", logits, vocab)
    code, rows, k = _code(logits.dtype), logits.shape[0], 0
    if (teacher_token is None) != (teacher_logit is None):
        raise ValueError("teacher_token and teacher_logit come together")
    if teacher_token is not None:
        k = int(teacher_token.shape[-1])
        _vector("teacher_token", teacher_token, torch.int32, rows, k)
        _vector("teacher_logit", teacher_logit, torch.float32, rows, k)
    if labels is not None:
        _vector("labels", labels, torch.int32, rows)
    with _on(stream):
        if dlogits is True:
            dlogits = torch.empty(logits.shape, dtype=grad_dtype or logits.dtype, device=logits.device)
        elif dlogits is not None:
            _matrix("dlogits", dlogits, vocab, grad_dtype, rows)
        loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
        n = _distill_ws(code, rows, vocab, k)
        ws = torch.empty(n, dtype=torch.uint8, device=logits.device) if n else None
        fold_loss_distill(None if sched is None else sched.handle, code, rows, vocab, logits, k, teacher_token,
                          teacher_logit, labels, temperature, soft_weight, hard_weight, scale, loss,
                          code if dlogits is None else _code(dlogits.dtype), dlogits, ws, n, stream or _CURRENT)
    return loss, dlogits


class TokenLogprobs(NamedTuple):
    """logp [rows, num_tokens], entropy [rows], top_token and top_logp [rows, top_k]; None for what was not asked for."""
    logp: object
    entropy: object
    top_token: object
    top_logp: object


def token_logprobs(logits, vocab, tokens=None, top_k=0, entropy=True, sched=None, stream=None) -> TokenLogprobs:
    """Log probabilities of `tokens` [rows, num_tokens] int32, the rows' entropy and their top_k alternatives
    (fold_token_logprobs).  sched: as in distill_loss."""
    import torch
    _matrix("logits", logits, vocab)
    code, rows, J, top_k = _code(logits.dtype), logits.shape[0], 0, int(top_k)
    if tokens is not None:
        J = int(tokens.shape[-1])
        _vector("tokens", tokens, torch.int32, rows, J)
    n = _token_ws(code, rows, vocab, top_k)
    with _on(stream):
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=logits.device)  # noqa: E731
        out = TokenLogprobs(new(rows, J) if J else None, new(rows) if entropy else None,
                            new(rows, top_k, dtype=torch.int32) if top_k else None, new(rows, top_k) if top_k else None)
        ws = new(n, dtype=torch.uint8) if n else None
        fold_token_logprobs(None if sched is None else sched.handle, code, rows, vocab, logits, J, tokens, out.logp,
                            out.entropy, top_k, out.top_token, out.top_logp, ws, n, stream or _CURRENT)
    return out


# ----------------------------------------------------------------------------- the attention block

_norm_ws = functools.lru_cache(256)(fold_layer_norm_workspace_size)
_linear_ws = functools.lru_cache(256)(fold_linear_workspace_size)


def _bytes(n, device):
    import torch
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def layer_norm(x, width, gamma=None, beta=None, eps=1e-5, stats=True, out=None, stream=None):
    """(y, mean [rows], rstd [rows]) of fold_layer_norm for x [rows, fold_row_ld(width)]; without stats the last two are
    None.  gamma, beta: [width] float32 or None.  out: a tensor to write, x itself for one."""
    import torch
    _matrix("x", x, width)
    code, rows = _code(x.dtype), x.shape[0]
    for name, t in (("gamma", gamma), ("beta", beta)):
        if t is not None:
            _vector(name, t, torch.float32, width)
    with _on(stream):
        out = torch.empty_like(x) if out is None else _matrix("out", out, width, x.dtype, rows)
        mean = torch.empty(rows, dtype=torch.float32, device=x.device) if stats else None
        rstd = torch.empty_like(mean) if stats else None
        fold_layer_norm(code, rows, width, x, gamma, beta, eps, out, mean, rstd, stream or _CURRENT)
    return out, mean, rstd


def layer_norm_backward(x, width, dy, mean, rstd, gamma=None, residual=None, dx=True, dgamma=True, dbeta=True, dtype=None,
                        accumulate=False, stream=None):
    """(dx, dgamma, dbeta) of fold_layer_norm_backward.  dy: of x's type or float32; residual: a gradient that goes by the
    norm, added to dx, of either type.  Each of the three: True for a new tensor (dx of `dtype`, the residual's or x's type by
    default), a tensor to write, or None to leave it out.  accumulate: dgamma and dbeta are added to the tensors given."""
    import torch
    _matrix("x", x, width)
    rows = x.shape[0]
    _matrix("dy", dy, width, None, rows)
    _vector("mean", mean, torch.float32, rows)
    _vector("rstd", rstd, torch.float32, rows)
    if gamma is not None:
        _vector("gamma", gamma, torch.float32, width)
    if accumulate and (dgamma is True or dbeta is True):
        raise ValueError("accumulate needs the dgamma and dbeta to add to (or None)")
    f32 = dict(dtype=torch.float32, device=x.device)
    with _on(stream):
        if dx is True:
            dx = torch.empty_like(x, dtype=dtype or (x.dtype if residual is None else residual.dtype))
        elif dx is not None:
            _matrix("dx", dx, width, dtype, rows)
        if residual is not None:
            _matrix("residual", residual, width, None, rows)
        dgamma = torch.empty(width, **f32) if dgamma is True else dgamma
        dbeta = torch.empty(width, **f32) if dbeta is True else dbeta
        for name, t in (("dgamma", dgamma), ("dbeta", dbeta)):
            if t is not None:
                _vector(name, t, torch.float32, width)
        code = _code(x.dtype)
        n = _norm_ws(code, rows, width) if dgamma is not None or dbeta is not None else 0
        ws = _bytes(n, x.device)
        fold_layer_norm_backward(code, rows, width, x, gamma, mean, rstd, _code(dy.dtype), dy,
                                 code if residual is None else _code(residual.dtype), residual,
                                 code if dx is None else _code(dx.dtype), dx, dgamma, dbeta,
                                 FOLD_BLOCK_ACCUMULATE if accumulate else 0, ws, n, stream or _CURRENT)
    return dx, dgamma, dbeta


class Linear:
    """The layer out = act(x W^T + bias) + residual (fold_linear, fold_linear_backward).

    weight: [out_dim, fold_row_ld(in_dim)], float32 or bfloat16; bias: [out_dim] float32 or None; activation: "none", "relu",
    "tanh" or "gelu".  Results and workspaces are new tensors of the calls' stream."""

    def __init__(self, weight, bias=None, in_dim=None, activation="none"):
        import torch
        self.in_dim = int(weight.shape[1] if in_dim is None else in_dim)
        self.weight = _matrix("weight", weight, self.in_dim)
        self.out_dim, self.dtype = int(weight.shape[0]), weight.dtype
        self.code = _code(weight.dtype)
        self.bias = None if bias is None else _vector("bias", bias, torch.float32, self.out_dim)
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation: one of {sorted(ACTIVATIONS)}, got {activation!r}")
        self.act = ACTIVATIONS[activation]

    def forward(self, x, residual=None, pre=None, out=None, stream=None):
        """out [rows, fold_row_ld(out_dim)] for x [rows, fold_row_ld(in_dim)]; with pre (True, or a tensor to write) a pair
        of it and the values before the activation, which backward() needs of a layer that has one."""
        import torch
        _matrix("x", x, self.in_dim, self.dtype)
        _here("weight", self.weight)
        rows = x.shape[0]
        if residual is not None:
            _matrix("residual", residual, self.out_dim, self.dtype, rows)
        shape, ret = (rows, _row_ld(self.out_dim)), pre is not None and pre is not False
        with _on(stream):
            new = lambda: torch.empty(shape, dtype=self.dtype, device=x.device)  # noqa: E731
            out = new() if out is None else _matrix("out", out, self.out_dim, self.dtype, rows)
            pre = None if not ret else new() if pre is True else _matrix("pre", pre, self.out_dim, self.dtype, rows)
            n = _linear_ws(self.code, rows, self.in_dim, self.out_dim)[0]
            ws = _bytes(n, x.device)
            fold_linear(self.code, rows, self.in_dim, self.out_dim, x, self.weight, self.bias, self.act, residual, out, pre,
                        ws, n, stream or _CURRENT)
        return (out, pre) if ret else out

    def backward(self, x, dout, pre=None, dx=True, dW=True, dbias=True, dpre=None, dx_dtype=None, dw_dtype=None,
                 accumulate=False, stream=None):
        """(dx, dW, dbias) of `dout` [rows, fold_row_ld(out_dim)].  Each of the three: True for a new tensor (dx of dx_dtype,
        dW of dw_dtype; float32 by default), a tensor to write, or None to leave it out.  pre: what forward() gave (a layer
        with an activation); dpre: a tensor for the gradient there (pre or dout itself, for one).  accumulate: dW and dbias
        are added to the tensors given."""
        import torch
        _matrix("x", x, self.in_dim, self.dtype)
        _here("weight", self.weight)
        rows = x.shape[0]
        _matrix("dout", dout, self.out_dim, self.dtype, rows)
        if accumulate and (dW is True or dbias is True):
            raise ValueError("accumulate needs the dW and dbias to add to (or None)")
        if (self.act != FOLD_ACT_NONE) != (pre is not None):
            raise ValueError("pre: what forward() gave, for a layer with an activation")
        with _on(stream):
            if dx is True:
                dx = torch.empty(x.shape, dtype=dx_dtype or torch.float32, device=x.device)
            elif dx is not None:
                _matrix("dx", dx, self.in_dim, dx_dtype, rows)
            if dW is True:
                dW = torch.empty(self.weight.shape, dtype=dw_dtype or torch.float32, device=x.device)
            elif dW is not None:
                _matrix("dW", dW, self.in_dim, dw_dtype, self.out_dim)
            if dbias is True:
                dbias = torch.empty(self.out_dim, dtype=torch.float32, device=x.device)
            elif dbias is not None:
                _vector("dbias", dbias, torch.float32, self.out_dim)
            if pre is not None:
                _matrix("pre", pre, self.out_dim, self.dtype, rows)
                if dpre is not None:
                    _matrix("dpre", dpre, self.out_dim, self.dtype, rows)
                elif any(t is not None for t in (dx, dW, dbias)):
                    dpre = torch.empty_like(pre)
            elif dpre is not None:
                raise ValueError("dpre belongs to a layer with an activation")
            n = _linear_ws(self.code, rows, self.in_dim, self.out_dim)[1]
            ws = _bytes(n, x.device)
            fold_linear_backward(self.code, rows, self.in_dim, self.out_dim, x, self.weight, self.act, pre, dout, dpre,
                                 FOLD_F32 if dx is None else _code(dx.dtype), dx,
                                 FOLD_F32 if dW is None else _code(dW.dtype), dW, dbias,
                                 FOLD_BLOCK_ACCUMULATE if accumulate else 0, ws, n, stream or _CURRENT)
        return dx, dW, dbias


def _columns(name, t, width, dtype, rows):
    """A matrix [rows, width or more] whose rows may lie apart (columns of a wider matrix)."""
    if not (t.is_cuda and t.dim() == 2 and t.shape[1] >= width and (t.stride(1) == 1 or t.shape[1] <= 1)):
        raise ValueError(f"{name}: a 2-D CUDA tensor with rows of at least {width} neighbouring elements is needed")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape[0] != rows:
        raise ValueError(f"{name}: expected {rows} rows, got {t.shape[0]}")
    _here(name, t)
    return t


def _stride(t):
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


class CrossAttention:
    """Cross attention of query sequences to key sequences (fold_cross_create; forward: fold_cross_attend, backward:
    fold_cross_backward).

    query_ptr [sequences + 1], key_ptr [sources + 1], query_rows [list entries], key_rows, source [sequences]: int32 CUDA
    tensors; rows None: row i is list entry i.  With schedules: graph_ptr and the schedule's node_pos (`schedule_rows`).
    num_query_rows, num_key_rows: rows of the matrices (the list entries by default).  The object is made once for a batch
    (it synchronises); its calls may be captured.  Results and workspaces are new tensors of the calls' stream."""

    def __init__(self, heads, head_dim, query_ptr, key_ptr, query_rows=None, key_rows=None, num_query_rows=None,
                 num_key_rows=None, source=None, kv_heads=None, dtype=None, num_queries=None, num_keys=None, stream=None):
        import torch
        self.heads, self.head_dim = int(heads), int(head_dim)
        self.kv_heads = self.heads if kv_heads is None else int(kv_heads)
        self.dtype = torch.bfloat16 if dtype is None else dtype
        for name, t in (("query_ptr", query_ptr), ("key_ptr", key_ptr), ("query_rows", query_rows), ("key_rows", key_rows),
                        ("source", source)):
            if t is not None:
                _vector(name, t, torch.int32, t.numel())
        if query_ptr.numel() < 1 or key_ptr.numel() < 1:
            raise ValueError("query_ptr and key_ptr have an entry more than there are sequences")
        # (without a list and a count the end of ptr is read, which waits for the GPU, as making the plan does)
        count = lambda rows, n, ptr: int(rows.numel()) if rows is not None else int(ptr[-1]) if n is None else int(n)  # noqa: E731
        with _on(stream):
            self.num_queries = count(query_rows, num_queries, query_ptr)
            self.num_keys = count(key_rows, num_keys, key_ptr)
        self.query_rows = self.num_queries if num_query_rows is None else int(num_query_rows)
        self.key_rows = self.num_keys if num_key_rows is None else int(num_key_rows)
        if source is not None and source.numel() != query_ptr.numel() - 1:
            raise ValueError("source has an entry for each query sequence")
        b = fold_cross_batch(_code(self.dtype), self.heads, self.kv_heads, self.head_dim, query_ptr.numel() - 1,
                             key_ptr.numel() - 1, self.num_queries, self.num_keys, self.query_rows, self.key_rows,
                             _ptr(query_ptr), _ptr(query_rows), _ptr(key_ptr), _ptr(key_rows), _ptr(source))
        self.handle = None
        with _on(stream):
            self.handle = fold_cross_create(b, stream)
        self.ws_bytes = fold_cross_workspace_size(self.handle)
        self.whole = self.num_queries == self.query_rows, self.num_keys == self.key_rows  # every row is listed

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            try:
                fold_cross_free(h)
            except Exception:
                pass
            self.handle = None

    def _new(self, rows, width, whole, like):
        """Zeros where the call leaves something alone: rows that are not listed, pad columns."""
        import torch
        make = torch.empty if whole and width % 64 == 0 else torch.zeros
        return make((rows, _row_ld(width)), dtype=self.dtype, device=like.device)

    def _inputs(self, q, k, v, key_mask, scale):
        import torch
        wq, wk = self.heads * self.head_dim, self.kv_heads * self.head_dim
        _columns("q", q, wq, self.dtype, self.query_rows)
        _columns("k", k, wk, self.dtype, self.key_rows)
        _columns("v", v, wk, self.dtype, self.key_rows)
        if key_mask is not None:
            if key_mask.dtype == torch.bool:
                key_mask = key_mask.view(torch.uint8)
            _vector("key_mask", key_mask, torch.uint8, self.num_keys)
        return wq, wk, key_mask, self.head_dim ** -0.5 if scale is None else float(scale)

    def forward(self, q, k, v, key_mask=None, scale=None, out=None, lse=True, stream=None):
        """(out [query rows, fold_row_ld(heads * head_dim)], lse [query rows, heads]) of q [query rows, ...] and k, v [key
        rows, ...] (columns of wider matrices, for one).  key_mask: uint8 or bool [num_keys] in list order; scale:
        head_dim^-1/2 by default; out: a tensor to write; lse: a tensor to write, or None to leave it out."""
        import torch
        wq, _, key_mask, scale = self._inputs(q, k, v, key_mask, scale)
        with _on(stream):
            out = self._new(self.query_rows, wq, self.whole[0], q) if out is None else _columns(
                "out", out, wq, self.dtype, self.query_rows)
            if lse is True:
                lse = (torch.empty if self.whole[0] else torch.zeros)((self.query_rows, self.heads), dtype=torch.float32,
                                                                      device=q.device)
            elif lse is not None:
                _vector("lse", lse, torch.float32, self.query_rows, self.heads)
            n = self.ws_bytes[0]
            ws = _bytes(n, q.device)
            fold_cross_attend(self.handle, q, _stride(q), k, _stride(k), v, _stride(v), key_mask, scale, out, _stride(out),
                              lse, ws, n, stream or _CURRENT)
        return out, lse

    def backward(self, q, k, v, out, lse, dout, key_mask=None, scale=None, dq=True, dk=True, dv=True, stream=None):
        """(dq, dk, dv) of `dout`, shaped as q, k and v are made by forward()'s rules; out and lse as it gave them.  Each of
        the three: True for a new tensor, a tensor to write (columns of a wider one, for instance), or None."""
        import torch
        wq, wk, key_mask, scale = self._inputs(q, k, v, key_mask, scale)
        _columns("out", out, wq, self.dtype, self.query_rows)
        _columns("dout", dout, wq, self.dtype, self.query_rows)
        _vector("lse", lse, torch.float32, self.query_rows, self.heads)
        with _on(stream):
            made = []
            for name, t, rows, w, whole in (("dq", dq, self.query_rows, wq, self.whole[0]),
                                            ("dk", dk, self.key_rows, wk, self.whole[1]),
                                            ("dv", dv, self.key_rows, wk, self.whole[1])):
                made.append(self._new(rows, w, whole, q) if t is True else None if t is None
                            else _columns(name, t, w, self.dtype, rows))
            dq, dk, dv = made
            ld = lambda t: 0 if t is None else _stride(t)  # noqa: E731
            n = self.ws_bytes[1]
            ws = _bytes(n, q.device)
            fold_cross_backward(self.handle, q, _stride(q), k, _stride(k), v, _stride(v), key_mask, scale, out, _stride(out),
                                lse, dout, _stride(dout), dq, ld(dq), dk, ld(dk), dv, ld(dv), ws, n, stream or _CURRENT)
        return dq, dk, dv


def schedule_rows(sched, stream=None) -> "torch.Tensor":  # noqa: F821
    """The schedule's node_pos as a new int32 tensor of `stream` (the current one by default): the pool row of every node, which
    with graph_ptr lists a batch's graphs for CrossAttention.  Waits for the copy, so that any stream may read it."""
    import torch
    n = sched.info.num_nodes
    with _on(stream):
        out = torch.empty(n, dtype=torch.int32, device="cuda")
        if n:  # (a plain hipMemcpy on the device goes through the null stream, which torch's streams do not wait for)
            st = torch.cuda.current_stream()
            rc = _hip().hipMemcpyAsync(out.data_ptr(), sched.info.node_pos, 4 * n, 3, st.cuda_stream)
            if rc != 0:
                raise RuntimeError(f"hipMemcpyAsync failed ({rc})")
            st.synchronize()
    return out
