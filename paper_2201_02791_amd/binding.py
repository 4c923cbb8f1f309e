"""Thin ctypes binding of ``libkge_mi355.so``: argument marshalling only.

Function names mirror the C ABI (``include/kge_mi355.h``) without the ``kge_`` prefix.
PyTorch is used for device memory and streams; every step of the training path runs in
the library's HIP kernels.  There is no CPU fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes as C
import os
import sys
from typing import List, Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libkge_mi355.so")
_lib = None

EXPORTED = ["kge_build_partition", "kge_partition_info", "kge_partition_export",
            "kge_partition_destroy", "kge_workspace_bytes", "kge_workspace_slice", "kge_rgcn_forward",
            "kge_rgcn_backward", "kge_sample_negatives", "kge_distmult_score_loss",
            "kge_profile_enable", "kge_profile_collect", "kge_last_error", "kge_cgraph_create",
            "kge_cgraph_destroy", "kge_compute_graph", "kge_cgraph_export", "kge_optimizer_step",
            "kge_optimizer_step_rows", "kge_eval_filter_create", "kge_eval_filter_destroy",
            "kge_eval_workspace_bytes", "kge_eval_rank_all", "kge_eval_rank_candidates", "kge_eval_metrics",
            "kge_eval_debug_scores", "kge_eval_rank_all_static", "kge_cgraph_input_rows", "kge_score_index_create", "kge_score_index_destroy",
            "kge_partition_bad_ids", "kge_test_set_rel_slab", "kge_test_pair_query", "kge_dense_forward",
            "kge_dense_workspace_bytes", "kge_dense_backward", "kge_layer_norm_forward", "kge_layer_norm_workspace_bytes",
            "kge_layer_norm_backward", "kge_adamw_step"]

ACT_IDENTITY, ACT_RELU, ACT_SILU = 0, 1, 2       # ACT_SILU: dense layers only
ORDER_PROJECT_FIRST, ORDER_RELATION_WEIGHTS = 0, 2
OPT_SGD, OPT_ADAM = 0, 1
OPT_ADAMW = 2                     # TrainStep: adamw_step over all parameters (not a kind of optimizer_step)
MSG_F32, MSG_BF16 = 0, 1
DT_F32, DT_BF16 = 0, 1
ROWS_ALL, ROWS_MASK, ROWS_NONZERO = 0, 1, 2
ADAMW_BLOCK = 256                 # KGE_ADAMW_BLOCK
NEG_TAIL, NEG_HEAD_OR_TAIL = 0, 1
DOMAIN_CORE, DOMAIN_ALL = 0, 1
EVAL_STATIC_BYTES = 32 << 20      # KGE_EVAL_STATIC_BYTES

ARRAYS = {"vert_gid": (0, np.int32), "core_eid": (1, np.int32), "core_h": (2, np.int32),
          "core_r": (3, np.int32), "core_t": (4, np.int32), "seg_ptr": (5, np.int32),
          "seg_rel": (6, np.int32), "seg_dst": (7, np.int32), "inv_c": (8, np.float32),
          "col_src": (9, np.int32), "edge_id": (10, np.int32), "cand": (11, np.int32),
          "dm_ptr": (12, np.int32), "dm_src": (13, np.int32), "dm_rel": (14, np.int32),
          "dm_invc": (15, np.float32), "sm_ptr": (16, np.int32), "sm_dst": (17, np.int32),
          "sm_rel": (18, np.int32), "sm_invc": (19, np.float32), "rel_ptr": (20, np.int32),
          "dr_ptr": (21, np.int32), "dr_seg": (22, np.int32), "dr_rel": (23, np.int32),
          "sm_seg": (24, np.int32)}


class KgeError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("kge status %d: %s" % (status, msg))
        self.status = status


class _PartInfo(C.Structure):
    _fields_ = [("n_vert", C.c_int64), ("n_edge", C.c_int64), ("n_seg", C.c_int64),
                ("n_core", C.c_int64), ("n_cand", C.c_int64), ("n_triples", C.c_int64),
                ("n_entities", C.c_int32), ("n_relations", C.c_int32), ("n_parts", C.c_int32),
                ("part_id", C.c_int32), ("n_hops", C.c_int32), ("neg_domain", C.c_int32),
                ("max_in_degree", C.c_int32), ("max_out_degree", C.c_int32)]


class _Layer(C.Structure):
    _fields_ = [("d_in", C.c_int32), ("d_out", C.c_int32), ("n_bases", C.c_int32), ("act", C.c_int32),
                ("order", C.c_int32), ("V", C.c_void_p), ("a", C.c_void_p), ("W0", C.c_void_p),
                ("dropout", C.c_float), ("drop_seed", C.c_uint64), ("drop_step", C.c_uint64)]


class _LayerGrad(C.Structure):
    _fields_ = [("dV", C.c_void_p), ("da", C.c_void_p), ("dW0", C.c_void_p)]


class _Opt(C.Structure):
    _fields_ = [("kind", C.c_int32), ("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float),
                ("eps", C.c_float), ("t", C.c_int64)]


class _Dense(C.Structure):
    _fields_ = [("d_in", C.c_int32), ("d_out", C.c_int32), ("act", C.c_int32), ("dtype", C.c_int32),
                ("W", C.c_void_p), ("b", C.c_void_p)]


class _Norm(C.Structure):
    _fields_ = [("d", C.c_int32), ("x_dtype", C.c_int32), ("y_dtype", C.c_int32), ("eps", C.c_float),
                ("gamma", C.c_void_p), ("beta", C.c_void_p)]


class _AdamWTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("copy", C.c_void_p), ("row_mask", C.c_void_p),
                ("n_rows", C.c_int64), ("d", C.c_int64), ("state_bits", C.c_int32), ("rows", C.c_int32),
                ("weight_decay", C.c_float)]


class _AdamW(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("t", C.c_int64), ("t_dev", C.c_void_p)]


class _ProfEntry(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("total_ms", C.c_double), ("calls", C.c_int64)]


def load():
    """Load the shared library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("%s is missing: run `python -m paper_2201_02791_amd.build` "
                              "(there is no CPU fallback)" % LIB_PATH)
        # torch first: its bundled HIP runtime must be the one this process initialises; loading
        # the library before it brings in a second runtime that then finds no device
        import torch  # noqa: F401
        lib = C.CDLL(LIB_PATH)
        lib.kge_last_error.restype = C.c_char_p
        lib.kge_workspace_bytes.restype = C.c_size_t
        lib.kge_partition_destroy.restype = None
        lib.kge_cgraph_destroy.restype = None
        lib.kge_score_index_destroy.restype = None
        lib.kge_eval_filter_destroy.restype = None
        lib.kge_eval_workspace_bytes.restype = C.c_size_t
        lib.kge_dense_workspace_bytes.restype = C.c_size_t
        lib.kge_layer_norm_workspace_bytes.restype = C.c_size_t
        # with argument types ctypes takes plain integers: a call of the block costs half the time on the host
        p, i64, size = C.c_void_p, C.c_int64, C.c_size_t
        lib.kge_dense_forward.argtypes = [p, i64] + [p, i64] * 4 + [p]
        lib.kge_dense_workspace_bytes.argtypes = [p, i64]
        lib.kge_dense_backward.argtypes = [p, i64] + [p, i64] * 5 + [p, p, p, size, p]
        lib.kge_layer_norm_forward.argtypes = [p, i64] + [p, i64] * 2 + [p, p, p]
        lib.kge_layer_norm_workspace_bytes.argtypes = [p, i64]
        lib.kge_layer_norm_backward.argtypes = [p, i64, p, i64, p, p, p, i64, p, i64, p, p, p, size, p]
        lib.kge_adamw_step.argtypes = [p, p, C.c_int32, p]
        _lib = lib
    return _lib


def _check(rc: int):
    if rc != 0:
        raise KgeError(rc, load().kge_last_error().decode())


def _ptr(t) -> C.c_void_p:
    return C.c_void_p(0 if t is None else t.data_ptr())


def _stream(stream) -> C.c_void_p:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return C.c_void_p(getattr(stream, "cuda_stream", stream))


class Partition:
    """Owner of a ``kge_partition*``."""

    def __init__(self, handle):
        self._h = C.c_void_p(handle)
        info = _PartInfo()
        _check(load().kge_partition_info(self._h, C.byref(info)))
        for name, _ in _PartInfo._fields_:
            setattr(self, name, int(getattr(info, name)))

    @property
    def handle(self):
        return self._h

    def export(self, name: str) -> np.ndarray:
        return partition_export(self, name)

    def bad_ids(self) -> int:
        """Ids outside the partition that the per-step kernels have met (and not used) so far; synchronises."""
        n = C.c_int64()
        _check(load().kge_partition_bad_ids(self._h, C.byref(n)))
        return int(n.value)

    def destroy(self):
        if self._h is not None and self._h.value:
            load().kge_partition_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def set_rel_slab_for_tests(vertices: int, min_runs: int = 0):
    """Test hook: slab size (destinations) and cutting threshold (runs) of the range order that partitions built
    afterwards give the transposed per-run products; (0, 0) restores the library's values."""
    load().kge_test_set_rel_slab(C.c_int32(vertices), C.c_int32(min_runs))


def pair_query_for_tests(n_known, at: int):
    """Test hook: (query whose row the evaluation's per-query kernel reads for place `at` of a block whose queries have
    n_known known answers each, number of places)."""
    known = np.ascontiguousarray(n_known, np.int64)
    n_pairs = C.c_int64()
    i = load().kge_test_pair_query(known.ctypes.data_as(C.c_void_p), C.c_int32(len(known)), C.c_int64(at), C.byref(n_pairs))
    return i, n_pairs.value


def build_partition(head, rel, tail, n_entities: int, n_relations: int, n_parts: int = 1,
                    part_id: int = 0, n_hops: int = 2, neg_domain: int = DOMAIN_CORE) -> Partition:
    head = np.ascontiguousarray(head, np.int32)
    rel = np.ascontiguousarray(rel, np.int32)
    tail = np.ascontiguousarray(tail, np.int32)
    assert len(head) == len(rel) == len(tail)
    out = C.c_void_p()
    _check(load().kge_build_partition(head.ctypes.data_as(C.c_void_p), rel.ctypes.data_as(C.c_void_p),
                                      tail.ctypes.data_as(C.c_void_p), C.c_int64(len(head)),
                                      C.c_int32(n_entities), C.c_int32(n_relations), C.c_int32(n_parts),
                                      C.c_int32(part_id), C.c_int32(n_hops), C.c_int32(neg_domain),
                                      C.byref(out)))
    return Partition(out.value)


def partition_info(part: Partition) -> dict:
    return {name: getattr(part, name) for name, _ in _PartInfo._fields_}


def partition_export(part: Partition, name: str) -> np.ndarray:
    which, dt = ARRAYS[name]
    n = {"vert_gid": part.n_vert, "core_eid": part.n_core, "core_h": part.n_core, "core_r": part.n_core,
         "core_t": part.n_core, "seg_ptr": part.n_seg + 1, "seg_rel": part.n_seg, "seg_dst": part.n_seg,
         "inv_c": part.n_seg, "col_src": part.n_edge, "edge_id": part.n_edge, "cand": part.n_cand,
         "dm_ptr": part.n_vert + 1, "dm_src": part.n_edge, "dm_rel": part.n_edge, "dm_invc": part.n_edge,
         "sm_ptr": part.n_vert + 1, "sm_dst": part.n_edge, "sm_rel": part.n_edge, "sm_invc": part.n_edge,
         "rel_ptr": 2 * part.n_relations + 1, "dr_ptr": part.n_vert + 1, "dr_seg": part.n_seg,
         "dr_rel": part.n_seg, "sm_seg": part.n_edge}[name]
    arr = np.empty(n, dt)
    _check(load().kge_partition_export(part.handle, C.c_int32(which), arr.ctypes.data_as(C.c_void_p),
                                       C.c_int64(arr.nbytes)))
    return arr


def partition_destroy(part: Partition):
    part.destroy()


def _layers(layers: Sequence[dict]):
    arr = (_Layer * len(layers))()
    for i, l in enumerate(layers):
        V, a, W0 = l["V"], l["a"], l["W0"]
        arr[i].n_bases, arr[i].d_in, arr[i].d_out = V.shape
        arr[i].act = int(l["act"])
        arr[i].order = int(l.get("order", ORDER_PROJECT_FIRST))
        arr[i].V, arr[i].a, arr[i].W0 = V.data_ptr(), a.data_ptr(), W0.data_ptr()
        arr[i].dropout = float(l.get("dropout", 0.0))
        arr[i].drop_seed, arr[i].drop_step = int(l.get("drop_seed", 0)), int(l.get("drop_step", 0))
    return arr


def workspace_bytes(part: Partition, layers: Sequence[dict], msg_dtype: int = MSG_F32) -> int:
    n = load().kge_workspace_bytes(part.handle, _layers(layers), C.c_int32(len(layers)), C.c_int32(msg_dtype))
    if n == 0:
        raise KgeError(-1, load().kge_last_error().decode())
    return int(n)


class ComputeGraph:
    """Owner of a ``kge_cgraph*``: the flags of one batch's computational sub-graph."""

    def __init__(self, part: Partition, n_layers: int):
        out = C.c_void_p()
        _check(load().kge_cgraph_create(part.handle, C.c_int32(n_layers), C.byref(out)))
        self._h = C.c_void_p(out.value)
        self.n_layers, self.n_vert = n_layers, part.n_vert

    @property
    def handle(self):
        return self._h

    def export(self):
        """(active uint8 [n_layers][N], counts int64 [n_layers][4] = vertices, edges in, runs, edges out)."""
        active = np.zeros((self.n_layers, self.n_vert), np.uint8)
        stats = np.zeros((self.n_layers, 4), np.int64)
        _check(load().kge_cgraph_export(self._h, active.ctypes.data_as(C.c_void_p),
                                        stats.ctypes.data_as(C.c_void_p)))
        return active, stats

    def input_rows_ptr(self) -> int:
        """Device address of the flags (uint8 [N]) of the first layer's input rows the batch reads."""
        ptr = C.c_void_p()
        _check(load().kge_cgraph_input_rows(self._h, C.byref(ptr), None, None))
        return ptr.value

    def input_rows(self):
        """(flags uint8 [N] on the host, their count): the first layer's input rows the batch reads."""
        flags = np.zeros(self.n_vert, np.uint8)
        count = C.c_int64()
        _check(load().kge_cgraph_input_rows(self._h, None, flags.ctypes.data_as(C.c_void_p), C.byref(count)))
        return flags, int(count.value)

    def destroy(self):
        if self._h is not None and self._h.value:
            load().kge_cgraph_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def _cg(cg) -> C.c_void_p:
    return C.c_void_p(0) if cg is None else cg.handle


def compute_graph(part: Partition, cg: ComputeGraph, pos_core_idx, neg_ent=None, stream=None):
    n_neg_entries = 0 if neg_ent is None else neg_ent.numel()
    _check(load().kge_compute_graph(part.handle, cg.handle, _ptr(pos_core_idx), C.c_int64(pos_core_idx.numel()),
                                    _ptr(neg_ent if n_neg_entries else None), C.c_int64(n_neg_entries),
                                    _stream(stream)))


def rgcn_forward(part: Partition, layers: Sequence[dict], H0, workspace, H_out,
                 msg_dtype: int = MSG_F32, stream=None, cg: ComputeGraph = None):
    _check(load().kge_rgcn_forward(part.handle, _cg(cg), _layers(layers), C.c_int32(len(layers)), C.c_int32(msg_dtype),
                                   _ptr(H0), _ptr(workspace), C.c_size_t(workspace.numel() * workspace.element_size()),
                                   _ptr(H_out), _stream(stream)))


def rgcn_backward(part: Partition, layers: Sequence[dict], H0, workspace, dH_out, grads: Sequence[dict],
                  dH0=None, msg_dtype: int = MSG_F32, stream=None, cg: ComputeGraph = None):
    g = (_LayerGrad * len(layers))()
    for i, gr in enumerate(grads):
        g[i].dV, g[i].da, g[i].dW0 = gr["dV"].data_ptr(), gr["da"].data_ptr(), gr["dW0"].data_ptr()
    _check(load().kge_rgcn_backward(part.handle, _cg(cg), _layers(layers), C.c_int32(len(layers)), C.c_int32(msg_dtype),
                                    _ptr(H0), _ptr(workspace), C.c_size_t(workspace.numel() * workspace.element_size()),
                                    _ptr(dH_out), g, _ptr(dH0), _stream(stream)))


def sample_negatives(part: Partition, pos_core_idx, n_neg: int, mode: int, seed: int, step: int,
                     neg_ent, neg_side, stream=None):
    _check(load().kge_sample_negatives(part.handle, _ptr(pos_core_idx), C.c_int64(pos_core_idx.numel()),
                                       C.c_int32(n_neg), C.c_int32(mode), C.c_uint64(seed), C.c_uint64(step),
                                       _ptr(neg_ent), _ptr(neg_side), _stream(stream)))


class ScoreIndex:
    """Owner of a ``kge_score_index*``: scratch of the atomic-free scoring call for batches up to a given size."""

    def __init__(self, part: Partition, max_pos: int, max_neg: int, d: int):
        out = C.c_void_p()
        _check(load().kge_score_index_create(part.handle, C.c_int64(max_pos), C.c_int32(max_neg), C.c_int32(d),
                                             C.byref(out)))
        self._h = C.c_void_p(out.value)

    @property
    def handle(self):
        return self._h

    def destroy(self):
        if self._h is not None and self._h.value:
            load().kge_score_index_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def distmult_score_loss(part: Partition, H, M, pos_core_idx, neg_ent, neg_side, n_neg: int, scores, loss,
                        dH, dM, stream=None, index: "ScoreIndex" = None):
    _check(load().kge_distmult_score_loss(part.handle, index.handle if index is not None else C.c_void_p(0),
                                          _ptr(H), _ptr(M), C.c_int32(H.shape[1]),
                                          _ptr(pos_core_idx), C.c_int64(pos_core_idx.numel()),
                                          _ptr(neg_ent), _ptr(neg_side), C.c_int32(n_neg), _ptr(scores),
                                          _ptr(loss), _ptr(dH), _ptr(dM), _stream(stream)))


def profile_enable(on: bool):
    _check(load().kge_profile_enable(C.c_int32(1 if on else 0)))


def profile_collect() -> dict:
    """{kernel name: (total milliseconds, launches)} since profiling was enabled / last collected."""
    arr = (_ProfEntry * 64)()
    n = C.c_int32(0)
    _check(load().kge_profile_collect(arr, C.c_int32(64), C.byref(n)))
    return {arr[i].name.decode(): (float(arr[i].total_ms), int(arr[i].calls)) for i in range(n.value)}


WS_P, WS_H, WS_G, WS_DP, WS_DH, WS_Z, WS_U, WS_HD = 0, 1, 2, 3, 4, 5, 7, 8


def workspace_slice(part: Partition, layers: Sequence[dict], which: int, layer: int,
                    msg_dtype: int = MSG_F32):
    """(byte offset, byte size) of one intermediate inside the workspace."""
    off, nbytes = C.c_size_t(0), C.c_size_t(0)
    _check(load().kge_workspace_slice(part.handle, _layers(layers), C.c_int32(len(layers)), C.c_int32(msg_dtype),
                                      C.c_int32(which), C.c_int32(layer), C.byref(off), C.byref(nbytes)))
    return int(off.value), int(nbytes.value)


def optimizer_step(kind: int, param, grad, m=None, v=None, lr=0.01, beta1=0.9, beta2=0.999, eps=1e-8, t=1,
                   rows: bool = False, row_mask=None, stream=None):
    """One optimizer step in place on device tensors.  rows=True: the row form on a 2-D tensor."""
    o = _Opt(kind, lr, beta1, beta2, eps, t)
    if rows:
        mask = C.c_void_p(row_mask) if isinstance(row_mask, int) else _ptr(row_mask)     # raw device address or tensor
        _check(load().kge_optimizer_step_rows(C.byref(o), _ptr(param), _ptr(grad), _ptr(m), _ptr(v),
                                              C.c_int64(param.shape[0]), C.c_int32(param.shape[1]),
                                              mask, _stream(stream)))
    else:
        _check(load().kge_optimizer_step(C.byref(o), _ptr(param), _ptr(grad), _ptr(m), _ptr(v),
                                         C.c_int64(param.numel()), _stream(stream)))


# ---- vertex-feature block (dense layer, layer norm) and AdamW over a list of tensors ------------

# These calls are short enough for the host's time to count: a caller's tensors mean that torch is loaded, and looking it up is
# cheaper than importing it again.

def _need(ok, msg: str):
    """An argument check of this layer: the library's own status for it (KGE_EINVAL)."""
    if not ok:
        raise KgeError(-1, msg)


def _rows(t, name: str, width=None, n=None, dtype=None):
    """(address, row stride) of a 2-D device tensor whose rows are dense; None is no tensor."""
    if t is None:
        return 0, 0
    if t.dim() != 2:
        raise KgeError(-1, "%s: a matrix of rows is wanted, not %d dimensions" % (name, t.dim()))
    rows, cols = t.shape
    if (width is not None and cols != width) or (n is not None and rows != n):
        raise KgeError(-1, "%s: %s x %s is wanted, not %d x %d" % (name, "any" if n is None else n, "any" if width is None else width, rows, cols))
    if dtype is not None and t.dtype != dtype:
        raise KgeError(-1, "%s: %s is wanted, not %s" % (name, dtype, t.dtype))
    ld, one = t.stride()
    if (cols > 1 and one != 1) or (rows > 1 and ld < cols):
        raise KgeError(-1, "%s: a row's elements must lie side by side, and rows apart" % name)
    return t.data_ptr(), ld if rows > 1 else cols


def _vector(t, name: str, width: int, need=False):
    """Address of `width` contiguous floats; None is no tensor unless it is needed."""
    torch = sys.modules["torch"]
    if t is None:
        _need(not need, "%s is missing" % name)
        return 0
    if t.dtype != torch.float32 or t.numel() != width or not t.is_contiguous():
        raise KgeError(-1, "%s: %d contiguous floats are wanted" % (name, width))
    return t.data_ptr()


def _new(X, shape, dtype, stream):
    """What a call makes by itself is memory of the stream that it runs on: the current one's may still be in use there, and would
    be given away again in the current one's order."""
    if stream is None or not X.is_cuda:
        return X.new_empty(shape, dtype=dtype)
    torch = sys.modules["torch"]
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(stream, X.device) if stream else torch.cuda.default_stream(X.device)
    with torch.cuda.stream(stream):
        return X.new_empty(shape, dtype=dtype)


def _workspace(t, need: int, X, stream):
    """The caller's workspace, or one from torch's allocator."""
    if t is None:
        return _new(X, max(need, 1), sys.modules["torch"].uint8, stream)
    _need(t.is_contiguous(), "workspace: contiguous memory is wanted")
    return t


def _call(function, stream, first, others, *args):
    """One library call on the device that all of its tensors are on, on `stream` or that device's current one.  Asked of torch by
    number and without its wrappers, device and stream cost a tenth of what they do otherwise."""
    torch = sys.modules["torch"]
    if not first.is_cuda:
        raise KgeError(-1, "device tensors are wanted (there is no CPU fallback)")
    at = first.get_device()
    for t in others:
        if t is not None and t.get_device() != at:
            raise KgeError(-1, "all tensors of a call must be on one device")
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(at)
    else:
        stream = getattr(stream, "cuda_stream", stream)
    if torch._C._cuda_getDevice() == at:
        rc = function(*args, stream)
    else:
        with torch.cuda.device(at):
            rc = function(*args, stream)
    if rc != 0:
        _check(rc)


def _type_of(dtype, name: str) -> int:
    torch = sys.modules["torch"]
    _need(dtype in (torch.float32, torch.bfloat16), "%s: float32 or bfloat16 is wanted, not %s" % (name, dtype))
    return DT_F32 if dtype == torch.float32 else DT_BF16


def _dense(layer: dict, X):
    W = layer["W"]
    if W.dim() != 2 or not W.is_contiguous():
        raise KgeError(-1, "W: a contiguous matrix is wanted")
    dt = _type_of(X.dtype, "X")
    _need(W.dtype == X.dtype, "W and X must be of one type")
    return _Dense(W.shape[0], W.shape[1], int(layer["act"]), dt, W.data_ptr(), _vector(layer.get("b"), "b", W.shape[1]))


def dense_workspace_bytes(layer: dict, n_rows: int) -> int:
    W = layer["W"]
    d = _Dense(W.shape[0], W.shape[1], int(layer["act"]), _type_of(W.dtype, "W"), None, None)
    n = load().kge_dense_workspace_bytes(C.byref(d), n_rows)
    if n == 0:
        raise KgeError(-1, load().kge_last_error().decode())
    return int(n)


def dense_forward(layer: dict, X, R=None, keep_pre: bool = False, Y=None, pre=None, stream=None):
    """(Y, pre): Y = act(X W + b) + R on the rows of X; layer = dict(W=, b= or None, act=).  pre (keep_pre, or a tensor to
    write it to): act's argument, which dense_backward takes; otherwise None."""
    d, dtype = _dense(layer, X), X.dtype
    x, ldx = _rows(X, "X", d.d_in)
    n, wide = X.shape[0], d.d_out
    r, ldr = _rows(R, "R", wide, n, dtype)
    if Y is None:
        Y = _new(X, (n, wide), dtype, stream)
    if pre is None and keep_pre:
        pre = _new(X, (n, wide), dtype, stream)
    y, ldy = _rows(Y, "Y", wide, n, dtype)
    z, ldz = _rows(pre, "pre", wide, n, dtype)
    _call(load().kge_dense_forward, stream, X, (layer["W"], layer.get("b"), R, Y, pre), C.byref(d), n, x, ldx, r, ldr, y, ldy, z, ldz)
    return Y, pre


def dense_backward(layer: dict, X, pre, dY, add=None, need_dX: bool = True, need_dW: bool = True, dX=None, dW=None, db=None,
                   workspace=None, stream=None) -> dict:
    """dict(dX=, dW=, db=) of dense_forward (dX: need_dX; dW, db: need_dW); add: a gradient that reaches X past the layer."""
    torch = sys.modules["torch"]
    d, dtype = _dense(layer, X), X.dtype
    x, ldx = _rows(X, "X", d.d_in)
    n = X.shape[0]
    z, ldz = _rows(pre, "pre", d.d_out, n, dtype)
    g, ldg = _rows(dY, "dY", d.d_out, n, dtype)
    if not need_dX:
        dX = None
    elif dX is None:
        dX = _new(X, (n, d.d_in), dtype, stream)
    ws_bytes = 0
    if need_dW:
        dW = _new(X, (d.d_in, d.d_out), torch.float32, stream) if dW is None else dW
        db = _new(X, d.d_out, torch.float32, stream) if db is None else db
        _need(dW.dim() == 2 and dW.shape[0] == d.d_in, "dW: %d x %d is wanted" % (d.d_in, d.d_out))
        workspace = _workspace(workspace, dense_workspace_bytes(layer, n), X, stream)
        ws_bytes = workspace.numel() * workspace.element_size()
    else:
        dW = db = workspace = None
    o, ldo = _rows(dX, "dX", d.d_in, n, dtype)
    a, lda = _rows(add, "add", d.d_in, n, dtype)
    pw, pb = _vector(dW, "dW", d.d_in * d.d_out), _vector(db, "db", d.d_out)
    _call(load().kge_dense_backward, stream, X, (layer["W"], pre, dY, add, dX, dW, db, workspace), C.byref(d), n, x, ldx, z, ldz, g, ldg,
          a, lda, o, ldo, pw, pb, 0 if workspace is None else workspace.data_ptr(), ws_bytes)
    return dict(dX=dX, dW=dW, db=db)


def _norm(norm: dict, d: int, x_dtype, y_dtype):
    return _Norm(d, _type_of(x_dtype, "X"), _type_of(y_dtype, "Y"), float(norm.get("eps", 1e-5)),
                 _vector(norm.get("gamma"), "gamma", d), _vector(norm.get("beta"), "beta", d))


def layer_norm_workspace_bytes(d: int, n_rows: int) -> int:
    p = _Norm(d, DT_F32, DT_F32, 0.0, None, None)
    n = load().kge_layer_norm_workspace_bytes(C.byref(p), n_rows)
    if n == 0:
        raise KgeError(-1, load().kge_last_error().decode())
    return int(n)


def layer_norm_forward(norm: dict, X, out_dtype=None, Y=None, mean=None, rstd=None, stream=None):
    """(Y, mean, rstd) of X's rows; norm = dict(gamma= or None, beta= or None, eps=); Y in out_dtype (X's by default)."""
    torch = sys.modules["torch"]
    x, ldx = _rows(X, "X")
    n, d = X.shape
    Y = _new(X, (n, d), out_dtype or X.dtype, stream) if Y is None else Y
    mean = _new(X, n, torch.float32, stream) if mean is None else mean
    rstd = _new(X, n, torch.float32, stream) if rstd is None else rstd
    p = _norm(norm, d, X.dtype, Y.dtype)
    y, ldy = _rows(Y, "Y", d, n)
    pm, pr = _vector(mean, "mean", n), _vector(rstd, "rstd", n)
    _call(load().kge_layer_norm_forward, stream, X, (norm.get("gamma"), norm.get("beta"), Y, mean, rstd), C.byref(p), n, x, ldx, y, ldy,
          pm, pr)
    return Y, mean, rstd


def layer_norm_backward(norm: dict, X, mean, rstd, dY, need_dX: bool = True, dX=None, dgamma=None, dbeta=None, workspace=None,
                        stream=None) -> dict:
    """dict(dX=, dgamma=, dbeta=) of layer_norm_forward (dX: need_dX)."""
    torch = sys.modules["torch"]
    x, ldx = _rows(X, "X")
    n, d = X.shape
    p = _norm(norm, d, X.dtype, dY.dtype)
    g, ldg = _rows(dY, "dY", d, n)
    if not need_dX:
        dX = None
    elif dX is None:
        dX = _new(X, (n, d), X.dtype, stream)
    o, ldo = _rows(dX, "dX", d, n, X.dtype)
    dgamma = _new(X, d, torch.float32, stream) if dgamma is None else dgamma
    dbeta = _new(X, d, torch.float32, stream) if dbeta is None else dbeta
    pm, pr = _vector(mean, "mean", n, True), _vector(rstd, "rstd", n, True)
    pg, pb = _vector(dgamma, "dgamma", d), _vector(dbeta, "dbeta", d)
    workspace = _workspace(workspace, layer_norm_workspace_bytes(d, n), X, stream)
    _call(load().kge_layer_norm_backward, stream, X, (norm.get("gamma"), norm.get("beta"), mean, rstd, dY, dX, dgamma, dbeta, workspace),
          C.byref(p), n, x, ldx, pm, pr, g, ldg, o, ldo, pg, pb, workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return dict(dX=dX, dgamma=dgamma, dbeta=dbeta)


class AdamWTensors:
    """The descriptions of the tensors that adamw_step updates, laid out once (the tensors are kept alive).  Each is a dict:
    param, grad; m, v and, for moments of 8 bits, m_scale, v_scale (adamw_state makes them); and, as wanted, weight_decay (0),
    rows ("all", "mask", "nonzero"), row_mask (a tensor or a device address), copy (bf16).  A parameter of two dimensions is held
    by rows, any other as one row.  What a step writes may overlap nothing else in the list: a parameter in it twice is refused."""

    def __init__(self, tensors: Sequence[dict]):
        torch = sys.modules["torch"]
        self.tensors = [dict(t) for t in tensors]
        self.array = (_AdamWTensor * max(len(self.tensors), 1))()
        places = []                        # (first byte, end, whether a step writes it, tensor, name)
        for i, t in enumerate(self.tensors):
            a, p = self.array[i], t["param"]
            name = "tensor %d: " % i
            rows, d = _row_shape(p)
            _need(p.dtype == torch.float32 and p.is_contiguous(), name + "param: contiguous floats are wanted")
            _need(t["grad"].dtype == torch.float32 and t["grad"].is_contiguous() and t["grad"].numel() == p.numel(),
                  name + "grad: contiguous floats are wanted, as many as param's")
            eight = t.get("m_scale") is not None
            for k, dt in (("m", torch.float8_e4m3fn if eight else torch.float32), ("v", torch.float8_e5m2 if eight else torch.float32)):
                _need(t[k].dtype == dt and t[k].is_contiguous() and t[k].numel() == p.numel(),
                      name + "%s: contiguous %s is wanted, as many as param's" % (k, dt))
            if eight:
                for k in ("m_scale", "v_scale"):
                    _need(t.get(k) is not None and t[k].dtype == torch.float32 and t[k].is_contiguous() and
                          t[k].numel() == rows * -(-d // ADAMW_BLOCK), name + "%s: a float for each block of %d is wanted" % (k, ADAMW_BLOCK))
            else:
                _need(t.get("v_scale") is None, name + "v_scale without m_scale")
            copy, mask, how = t.get("copy"), t.get("row_mask"), t.get("rows", "all")
            _need(copy is None or (copy.dtype == torch.bfloat16 and copy.is_contiguous() and copy.numel() == p.numel()),
                  name + "copy: contiguous bfloat16 is wanted, as many as param's")
            _need(how in ("all", "mask", "nonzero"), name + "rows: all, mask or nonzero is wanted")
            if mask is not None and not isinstance(mask, int):
                _need(mask.dtype in (torch.uint8, torch.bool) and mask.is_contiguous() and mask.numel() == rows,
                      name + "row_mask: a byte for each row is wanted")
            on = [x for x in (t["grad"], t["m"], t["v"], t.get("m_scale"), t.get("v_scale"), copy, mask) if hasattr(x, "device")]
            _need(all(x.device == self.tensors[0]["param"].device for x in on + [p]), "all tensors of a call must be on one device")
            a.param, a.grad, a.m, a.v = (t[k].data_ptr() for k in ("param", "grad", "m", "v"))
            a.m_scale, a.v_scale, a.copy = (_ptr(t.get(k)).value for k in ("m_scale", "v_scale", "copy"))
            a.row_mask = mask if isinstance(mask, int) else _ptr(mask).value
            a.n_rows, a.d, a.state_bits = rows, d, 8 if eight else 32
            a.rows, a.weight_decay = dict(all=ROWS_ALL, mask=ROWS_MASK, nonzero=ROWS_NONZERO)[how], float(t.get("weight_decay", 0.0))
            for k in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy"):
                if t.get(k) is not None:
                    places.append((t[k].data_ptr(), t[k].data_ptr() + t[k].numel() * t[k].element_size(), k != "grad", i, k))
            if a.row_mask:
                places.append((a.row_mask, a.row_mask + rows, False, i, "row_mask"))
        last = written = (0, 0, False, 0, "")        # of the places before: the one that ends last, and of those that are written
        for at in sorted(p for p in places if p[1] > p[0]):
            over = last if at[2] else written
            _need(at[0] >= over[1], "tensor %d: its %s overlaps %s of tensor %d" % (at[3], at[4], over[4], over[3]))
            last = max(last, at, key=lambda p: p[1])
            if at[2]:
                written = max(written, at, key=lambda p: p[1])


def _row_shape(p):
    return (p.shape[0], p.shape[1]) if p.dim() == 2 else (1, p.numel())


def adamw_state(param, bits: int = 32) -> dict:
    """Zeroed moments of a parameter: dict(m=, v=, m_scale=, v_scale=), the scales None with 32 bits."""
    torch = sys.modules["torch"]
    _need(bits in (8, 32), "moments have 32 or 8 bits")
    if bits == 32:
        return dict(m=torch.zeros_like(param), v=torch.zeros_like(param), m_scale=None, v_scale=None)
    rows, d = _row_shape(param)
    scales = lambda: torch.zeros((rows, -(-d // ADAMW_BLOCK)), dtype=torch.float32, device=param.device)
    codes = lambda dt: torch.zeros(param.shape, dtype=torch.uint8, device=param.device).view(dt)
    return dict(m=codes(torch.float8_e4m3fn), v=codes(torch.float8_e5m2), m_scale=scales(), v_scale=scales())


def adamw_step(tensors, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, t=1, t_dev=None, stream=None):
    """One AdamW step in place on all tensors: an AdamWTensors or a list of its dicts.  t_dev: the step number as a device
    int64 tensor of one element, in place of t."""
    torch = sys.modules["torch"]
    plan = tensors if isinstance(tensors, AdamWTensors) else AdamWTensors(tensors)
    _need(t_dev is None or (t_dev.dtype == torch.int64 and t_dev.numel() == 1), "t_dev: one int64 is wanted")
    o = _AdamW(lr, beta1, beta2, eps, int(t), _ptr(t_dev).value)
    if not plan.tensors:
        return
    _call(load().kge_adamw_step, stream, plan.tensors[0]["param"], (t_dev,), C.byref(o), plan.array, len(plan.tensors))


# ---- link-prediction evaluation (filtered ranks, MRR, Hits@k) ----------------------------------

class EvalFilter:
    """Owner of a ``kge_eval_filter*``: the known triples whose corruptions the filtered setting drops."""

    def __init__(self, head, rel, tail, n_entities: int, n_relations: int):
        head = np.ascontiguousarray(head, np.int32)
        rel = np.ascontiguousarray(rel, np.int32)
        tail = np.ascontiguousarray(tail, np.int32)
        assert len(head) == len(rel) == len(tail)
        out = C.c_void_p()
        _check(load().kge_eval_filter_create(head.ctypes.data_as(C.c_void_p), rel.ctypes.data_as(C.c_void_p),
                                             tail.ctypes.data_as(C.c_void_p), C.c_int64(len(head)),
                                             C.c_int32(n_entities), C.c_int32(n_relations), C.byref(out)))
        self._h = C.c_void_p(out.value)

    @property
    def handle(self):
        return self._h

    def destroy(self):
        if self._h is not None and self._h.value:
            load().kge_eval_filter_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def eval_workspace_bytes(n_queries: int, d: int) -> int:
    n = load().kge_eval_workspace_bytes(C.c_int64(n_queries), C.c_int32(d))
    if n == 0:
        raise KgeError(-1, load().kge_last_error().decode())
    return int(n)


def _eval_ws(n_queries, d, device, workspace):
    import torch
    need = eval_workspace_bytes(n_queries, d)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace


def eval_rank_all(H, M, test_h, test_r, test_t, filt: EvalFilter = None, workspace=None, stream=None):
    """(higher, equal) int32 [2 n_test] on the device: tail queries of all test triples, then head queries."""
    import torch
    n_test = test_h.numel()
    ws = _eval_ws(2 * n_test, H.shape[1], H.device, workspace)
    higher = torch.empty(2 * n_test, dtype=torch.int32, device=H.device)
    equal = torch.empty_like(higher)
    _check(load().kge_eval_rank_all(filt.handle if filt is not None else C.c_void_p(0), _ptr(H), C.c_int64(H.shape[0]),
                                    C.c_int32(H.shape[1]), _ptr(M), C.c_int32(M.shape[0]), _ptr(test_h), _ptr(test_r),
                                    _ptr(test_t), C.c_int64(n_test), _ptr(ws), C.c_size_t(ws.numel()), _ptr(higher),
                                    _ptr(equal), _stream(stream)))
    return higher, equal


def eval_rank_all_static(H, M, test_h, test_r, test_t, higher, equal, filt: EvalFilter = None, stream=None):
    """kge_eval_rank_all_static: the caller brings the outputs (int32 [2 n_test] each); nothing is allocated."""
    _check(load().kge_eval_rank_all_static(filt.handle if filt is not None else C.c_void_p(0), _ptr(H),
                                           C.c_int64(H.shape[0]), C.c_int32(H.shape[1]), _ptr(M), C.c_int32(M.shape[0]),
                                           _ptr(test_h), _ptr(test_r), _ptr(test_t), C.c_int64(test_h.numel()),
                                           _ptr(higher), _ptr(equal), _stream(stream)))


def eval_rank_candidates(H, M, fixed, rel, answer, cand, workspace=None, stream=None):
    """(higher, equal) int32 [n_queries] against each query's own candidate list cand [n_queries, n_cand]."""
    import torch
    nq = fixed.numel()
    ws = _eval_ws(nq, H.shape[1], H.device, workspace)
    higher = torch.empty(nq, dtype=torch.int32, device=H.device)
    equal = torch.empty_like(higher)
    _check(load().kge_eval_rank_candidates(_ptr(H), C.c_int64(H.shape[0]), C.c_int32(H.shape[1]), _ptr(M),
                                           C.c_int32(M.shape[0]), _ptr(fixed), _ptr(rel), _ptr(answer), C.c_int64(nq),
                                           _ptr(cand), C.c_int32(cand.shape[1] if cand.dim() == 2 else 0), _ptr(ws),
                                           C.c_size_t(ws.numel()), _ptr(higher), _ptr(equal), _stream(stream)))
    return higher, equal


def eval_metrics(higher, equal, ks=(1, 3, 10), stream=None):
    """Device tensor of doubles: MRR, then Hits@k for each k."""
    import torch
    out = torch.empty(1 + len(ks), dtype=torch.float64, device=higher.device)
    karr = (C.c_int32 * max(len(ks), 1))(*ks)
    _check(load().kge_eval_metrics(_ptr(higher), _ptr(equal), C.c_int64(higher.numel()), karr, C.c_int32(len(ks)),
                                   _ptr(out), _stream(stream)))
    return out


def eval_debug_scores(H, M, test_h, test_r, test_t, stream=None):
    """Test hook: (scores [2 n_test, n_entities] from the tile kernel, answer scores [2 n_test] from the
    per-query kernel)."""
    import torch
    n_test = test_h.numel()
    ws = _eval_ws(2 * n_test, H.shape[1], H.device, None)
    scores = torch.empty((2 * n_test, H.shape[0]), dtype=torch.float32, device=H.device)
    ans = torch.empty(2 * n_test, dtype=torch.float32, device=H.device)
    _check(load().kge_eval_debug_scores(_ptr(H), C.c_int64(H.shape[0]), C.c_int32(H.shape[1]), _ptr(M),
                                        C.c_int32(M.shape[0]), _ptr(test_h), _ptr(test_r), _ptr(test_t),
                                        C.c_int64(n_test), _ptr(ws), C.c_size_t(ws.numel()), _ptr(scores), _ptr(ans),
                                        _stream(stream)))
    return scores, ans
