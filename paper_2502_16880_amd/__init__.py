"""Thin Python binding of libcoral_lmhead.so (argument marshalling only).

Every step of the grouped / dense LM head (paper section 3.3 and the appendix on
the LM head router) runs in the HIP kernels behind the C ABI declared in
include/coral_lmhead.h.  PyTorch is used for device memory and the current
stream, nothing else.  There is no CPU fallback: if the built library is missing
the import of this package fails.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import NamedTuple, Optional, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcoral_lmhead.so")

CORAL_OK = 0
CORAL_F32 = 0
CORAL_BF16 = 1
CORAL_F16 = 2


class CoralError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"coral_lmhead status {status}: {message}")
        self.status = status


class _GroupIndexStruct(ctypes.Structure):
    _fields_ = [("G", ctypes.c_int32),
                ("group_offsets_host", ctypes.c_void_p),
                ("group_offsets", ctypes.c_void_p),
                ("group_rows", ctypes.c_void_p)]


class _RopeStruct(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("inv_freq", ctypes.c_void_p), ("eps", ctypes.c_float), ("rot_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32)]


class _Kv4CacheStruct(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class _LogitRulesStruct(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("history_ranges", ctypes.c_void_p),
                ("penalties", ctypes.c_void_p), ("bias_ids", ctypes.c_void_p),
                ("bias_values", ctypes.c_void_p), ("bias_ranges", ctypes.c_void_p),
                ("mask", ctypes.c_void_p), ("n_history", ctypes.c_int32), ("n_biases", ctypes.c_int32)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'` "
            "(there is no fallback path)")
    L = ctypes.CDLL(LIB_PATH)
    c = ctypes
    L.coral_status_string.restype = c.c_char_p
    L.coral_status_string.argtypes = [c.c_int]
    L.coral_group_index_validate.restype = c.c_int
    L.coral_group_index_validate.argtypes = [c.c_void_p, c.c_void_p, c.c_int, c.c_int]
    L.coral_lmhead_workspace_bytes.restype = c.c_size_t
    L.coral_lmhead_workspace_bytes.argtypes = [c.c_int] * 7
    L.coral_lmhead_path.restype = c.c_int
    L.coral_lmhead_path.argtypes = [c.c_int] * 8
    L.coral_lmhead_logprob_path.restype = c.c_int
    L.coral_lmhead_logprob_path.argtypes = [c.c_int] * 7
    L.coral_lmhead_workspace_init.restype = c.c_int
    L.coral_lmhead_workspace_init.argtypes = [c.c_void_p, c.c_size_t, c.c_void_p]
    L.coral_lmhead_grouped.restype = c.c_int
    L.coral_lmhead_grouped.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
                                       c.POINTER(_GroupIndexStruct)] + [c.c_int] * 6 + \
                                      [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_size_t,
                                       c.c_void_p]
    L.coral_lmhead_grouped_noalloc.restype = c.c_int
    L.coral_lmhead_grouped_noalloc.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
                                               c.POINTER(_GroupIndexStruct)] + [c.c_int] * 6 + \
                                              [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p]
    L.coral_lmhead_dense.restype = c.c_int
    L.coral_lmhead_dense.argtypes = [c.c_void_p, c.c_void_p] + [c.c_int] * 5 + \
                                    [c.c_void_p, c.c_void_p, c.c_void_p, c.c_size_t, c.c_void_p]
    L.coral_lmhead_grouped_profiled.restype = c.c_int
    L.coral_lmhead_grouped_profiled.argtypes = L.coral_lmhead_grouped.argtypes + [c.c_void_p] * 2
    L.coral_lmhead_grouped_logprob.restype = c.c_int
    L.coral_lmhead_grouped_logprob.argtypes = L.coral_lmhead_grouped.argtypes
    L.coral_lmhead_grouped_logprob_profiled.restype = c.c_int
    L.coral_lmhead_grouped_logprob_profiled.argtypes = L.coral_lmhead_grouped_profiled.argtypes
    L.coral_lmhead_dense_profiled.restype = c.c_int
    L.coral_lmhead_dense_profiled.argtypes = L.coral_lmhead_dense.argtypes + [c.c_void_p] * 2
    L.coral_probe_read.restype = c.c_int
    L.coral_probe_read.argtypes = [c.c_void_p, c.c_size_t, c.c_int, c.c_void_p, c.c_void_p, c.c_void_p]
    L.coral_router_premix.restype = c.c_int
    L.coral_router_premix.argtypes = [c.c_void_p, c.c_void_p, c.c_int, c.c_int, c.c_int, c.c_int,
                                      c.c_void_p, c.c_void_p]
    L.coral_tree_expand.restype = c.c_int
    L.coral_tree_expand.argtypes = [c.c_void_p] * 3 + [c.c_int] * 3 + [c.c_void_p] * 4
    L.coral_lmhead_draft_level.restype = c.c_int
    L.coral_lmhead_draft_level.argtypes = [c.c_void_p] * 5 + [c.POINTER(_GroupIndexStruct)] + \
                                          [c.c_int] * 6 + [c.c_void_p, c.c_int] + [c.c_void_p] * 7 + \
                                          [c.c_size_t, c.c_void_p]
    L.coral_lmhead_grouped_routed.restype = c.c_int
    L.coral_lmhead_grouped_routed.argtypes = [c.c_void_p] * 5 + [c.POINTER(_GroupIndexStruct)] + \
                                             [c.c_int] * 7 + [c.c_void_p] * 4 + \
                                             [c.c_size_t, c.c_void_p]
    L.coral_matvec_w4.restype = c.c_int
    L.coral_matvec_w4.argtypes = [c.c_void_p] * 6 + [c.c_int] * 8 + [c.c_void_p] * 2
    L.coral_logits_adjust.restype = c.c_int
    L.coral_logits_adjust.argtypes = [c.c_void_p, c.POINTER(_LogitRulesStruct)] + [c.c_int] * 3 + [c.c_void_p] * 2
    L.coral_logits_topk_workspace_bytes.restype = c.c_size_t
    L.coral_logits_topk_workspace_bytes.argtypes = [c.c_int] * 3
    L.coral_logits_topk.restype = c.c_int
    L.coral_logits_topk.argtypes = [c.c_void_p, c.POINTER(_LogitRulesStruct)] + [c.c_int] * 4 + \
                                   [c.c_void_p] * 3 + [c.c_size_t, c.c_void_p]
    p, i, i64 = c.c_void_p, c.c_int, c.c_int64
    L.coral_qk_norm_rope.restype = c.c_int
    L.coral_qk_norm_rope.argtypes = [p, i64, p, i64, c.POINTER(_RopeStruct), i, i, i, i, i, p, i64, p, i64,
                                     c.POINTER(_Kv4CacheStruct), p, i64, p, p]
    L.coral_kv4_append.restype = c.c_int
    L.coral_kv4_append.argtypes = [c.POINTER(_Kv4CacheStruct), p, i64, p, i64, p, i, i, p]
    L.coral_kv4_read.restype = c.c_int
    L.coral_kv4_read.argtypes = [c.POINTER(_Kv4CacheStruct), p, i, i, p, p, p]
    L.coral_attention_kv4_workspace_bytes.restype = c.c_size_t
    L.coral_attention_kv4_workspace_bytes.argtypes = [i] * 7
    L.coral_attention_kv4.restype = c.c_int
    L.coral_attention_kv4.argtypes = [p, i64, c.POINTER(_Kv4CacheStruct), p, i, p, p, p, p, i, i, i, i, i, c.c_float, i, p, p,
                                      c.c_size_t, p]
    L.coral_attention_prompt.restype = c.c_int
    L.coral_attention_prompt.argtypes = [p, i64, p, i64, p, i64, p, p, i, i, i, i, i, i, c.c_float, i, p, p]
    return L


_L = _load()


def coral_status_string(status: int) -> str:
    return _L.coral_status_string(int(status)).decode()


def _raise(status: int):
    if status != CORAL_OK:
        raise CoralError(status, coral_status_string(status))


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return CORAL_BF16
    if t.dtype == torch.float16:
        return CORAL_F16
    if t.dtype == torch.float32:
        return CORAL_F32
    raise TypeError(f"hidden/gate_W/lm_W must be bfloat16, float16 or float32, got {t.dtype}")


def _dev_ptr(t: Optional[torch.Tensor], name: str, dtype=None) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous (row-major, no padding)")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def device_tensor(a: np.ndarray, storage: str, device="cuda") -> torch.Tensor:
    """Upload a host array; storage 'bf16' and 'f16' take uint16 bit patterns, 'f32' float32."""
    if storage in ("bf16", "f16"):
        if a.dtype != np.uint16:
            raise TypeError(f"{storage} storage expects uint16 bit patterns")
        return torch.from_numpy(a.view(np.int16)).to(device).view(
            torch.bfloat16 if storage == "bf16" else torch.float16)
    if storage == "f32":
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device)
    raise ValueError(f"unknown storage {storage!r}")


class GroupIndex:
    """CSR partition of the vocabulary into groups: host offsets + device copies."""

    def __init__(self, group_offsets: np.ndarray, group_rows, device="cuda", validate=True):
        self.offsets_host = np.ascontiguousarray(group_offsets, dtype=np.int32)
        self.G = int(self.offsets_host.size - 1)
        if isinstance(group_rows, torch.Tensor):
            if validate:
                raise ValueError("validation needs the rows on the host; pass a numpy array")
            self.rows = group_rows
        else:
            rows_host = np.ascontiguousarray(group_rows, dtype=np.int32)
            if validate:
                group_index_validate(self.offsets_host, rows_host)
            self.rows = torch.from_numpy(rows_host).to(device)
        self.V = int(self.rows.numel())
        self.offsets = torch.from_numpy(self.offsets_host).to(device)
        self._struct = _GroupIndexStruct(self.G, self.offsets_host.ctypes.data,
                                         _dev_ptr(self.offsets, "group_offsets", torch.int32),
                                         _dev_ptr(self.rows, "group_rows", torch.int32))

    def struct(self):
        return ctypes.byref(self._struct)


def group_index_validate(group_offsets: np.ndarray, group_rows: np.ndarray) -> None:
    off = np.ascontiguousarray(group_offsets, dtype=np.int32)
    rows = np.ascontiguousarray(group_rows, dtype=np.int32)
    _raise(_L.coral_group_index_validate(off.ctypes.data, rows.ctypes.data, off.size - 1, rows.size))


def coral_lmhead_workspace_bytes(M: int, H: int, V: int, G: int, g: int, k: int, dt: int) -> int:
    return int(_L.coral_lmhead_workspace_bytes(M, H, V, G, g, k, dt))


PATH_NAMES = {0: "general", 1: "single-launch", 2: "tiles", -1: "unsupported"}


def coral_lmhead_path(dense: bool, M: int, H: int, V: int, G: int, g: int, k: int, dt: int) -> int:
    return int(_L.coral_lmhead_path(1 if dense else 0, M, H, V, G, g, k, dt))


def coral_lmhead_logprob_path(M: int, H: int, V: int, G: int, g: int, k: int, dt: int) -> int:
    return int(_L.coral_lmhead_logprob_path(M, H, V, G, g, k, dt))


def coral_lmhead_workspace_init(workspace: torch.Tensor, stream=None) -> None:
    _raise(_L.coral_lmhead_workspace_init(_dev_ptr(workspace, "workspace"),
                                          workspace.numel() * workspace.element_size(),
                                          _stream_ptr(stream)))


def alloc_workspace(M, H, V, G, g, k, dt, device="cuda", stream=None) -> torch.Tensor:
    """A prepared workspace (allocated through PyTorch, control words zeroed on `stream`, the
    stream the head will be enqueued on; None = the current stream)."""
    n = coral_lmhead_workspace_bytes(M, H, V, G, g, k, dt)
    if n == 0:
        raise ValueError("invalid sizes for the workspace")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    coral_lmhead_workspace_init(ws, stream)
    if stream is not None:
        ws.record_stream(stream)       # the caching allocator must not reuse it under that stream
    return ws


def _marshal_grouped(hidden, gate_W, gate_bias, lm_W, gi, g, k, topk_ids, topk_logits, sel_groups,
                     workspace, stream, events, logprob, gate_hidden, level):
    """Checks and marshals the arguments of the grouped entry points once: returns the entry
    point, its arguments up to (not including) the stream, those behind the stream, and the
    output tensors."""
    dt = _dtype_code(hidden)
    if gate_W.dtype != hidden.dtype or lm_W.dtype != hidden.dtype:
        raise TypeError("hidden, gate_W and lm_W must share one dtype")
    if hidden.dim() != 2 or gate_W.dim() != 2 or lm_W.dim() != 2:
        raise ValueError("hidden, gate_W and lm_W must be 2-D")
    M, H = hidden.shape
    V = lm_W.shape[0]
    if lm_W.shape[1] != H or gate_W.shape != (gi.G, H) or gi.V != V:
        raise ValueError("inconsistent shapes")
    if gate_bias is not None and gate_bias.shape != (gi.G,):
        raise ValueError("gate_bias must be [G]")
    dev = hidden.device
    if topk_ids is None:
        topk_ids = torch.empty((M, k), dtype=torch.int32, device=dev)
    if topk_logits is None:
        topk_logits = torch.empty((M, k), dtype=torch.float32, device=dev)
    if sel_groups is None:
        sel_groups = torch.empty((M, g), dtype=torch.int32, device=dev)
    if topk_ids.shape != (M, k) or topk_logits.shape != (M, k) or sel_groups.shape != (M, g):
        raise ValueError("output shapes must be [M,k], [M,k], [M,g]")
    if workspace is None:
        workspace = alloc_workspace(M, H, V, gi.G, g, k, dt, dev, stream)
    args = (_dev_ptr(hidden, "hidden"), _dev_ptr(gate_W, "gate_W"),
            _dev_ptr(gate_bias, "gate_bias", torch.float32), _dev_ptr(lm_W, "lm_W"), gi.struct(),
            M, H, V, g, k, dt, _dev_ptr(topk_ids, "topk_ids", torch.int32),
            _dev_ptr(topk_logits, "topk_logits", torch.float32),
            _dev_ptr(sel_groups, "sel_groups", torch.int32), _dev_ptr(workspace, "workspace"),
            workspace.numel() * workspace.element_size())
    if gate_hidden is not None and (gate_hidden.dtype != hidden.dtype or gate_hidden.shape != hidden.shape):
        raise ValueError("gate_hidden must match hidden in dtype and shape")
    behind = ()
    if level is not None:
        if events is not None:
            raise ValueError("the draft-level entry point has no measurement variant")
        parent_score, n_next, next_parent, next_token, next_score = level
        fn = _L.coral_lmhead_draft_level
        args = (args[0], _dev_ptr(gate_hidden, "gate_hidden"), *args[1:11],
                _dev_ptr(parent_score, "parent_score", torch.float32), int(n_next), *args[11:14],
                _dev_ptr(next_parent, "next_parent", torch.int32),
                _dev_ptr(next_token, "next_token", torch.int32),
                _dev_ptr(next_score, "next_score", torch.float32), *args[14:])
    elif gate_hidden is not None:
        if events is not None:
            raise ValueError("the routed entry point has no measurement variant")
        fn = _L.coral_lmhead_grouped_routed
        args = (args[0], _dev_ptr(gate_hidden, "gate_hidden"), *args[1:11], 1 if logprob else 0, *args[11:])
    elif events is None:
        fn = _L.coral_lmhead_grouped_logprob if logprob else _L.coral_lmhead_grouped
    else:
        fn = _L.coral_lmhead_grouped_logprob_profiled if logprob else _L.coral_lmhead_grouped_profiled
        behind = (events[0], events[1])
    keep = (hidden, gate_W, gate_bias, lm_W, gi, workspace, gate_hidden, level)
    return fn, args, behind, (topk_ids, topk_logits, sel_groups), keep


def coral_lmhead_grouped(hidden: torch.Tensor, gate_W: torch.Tensor,
                         gate_bias: Optional[torch.Tensor], lm_W: torch.Tensor, gi: GroupIndex,
                         g: int, k: int, topk_ids: Optional[torch.Tensor] = None,
                         topk_logits: Optional[torch.Tensor] = None,
                         sel_groups: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, stream=None, events=None,
                         logprob: bool = False, gate_hidden: Optional[torch.Tensor] = None,
                         level=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """events: optional (hipEvent_t, hipEvent_t) raw handles; selects the _profiled entry.
    logprob: call coral_lmhead_grouped_logprob (the second result then holds log p(x)).
    gate_hidden: call coral_lmhead_grouped_routed (the router sees this [M,H] tensor).
    level: (parent_score or None, n_next, next_parent, next_token, next_score): call
    coral_lmhead_draft_level (see coral_lmhead_draft_level below)."""
    fn, args, behind, out, _ = _marshal_grouped(hidden, gate_W, gate_bias, lm_W, gi, g, k, topk_ids,
                                                topk_logits, sel_groups, workspace, stream, events,
                                                logprob, gate_hidden, level)
    _raise(fn(*args, _stream_ptr(stream), *behind))
    return out


class PreparedGrouped:
    """A grouped-head call whose arguments are checked and marshalled once, for loops that
    issue the same call many times (a draft loop, a benchmark): calling the object only looks
    the stream up and enters the library.  Takes coral_lmhead_grouped's arguments (a workspace
    is required: the call must not allocate); .out holds the output tensors.  The tensors are
    kept alive by the object and must not be resized or freed while it is in use."""

    def __init__(self, hidden, gate_W, gate_bias, lm_W, gi, g, k, workspace, topk_ids=None,
                 topk_logits=None, sel_groups=None, logprob=False, gate_hidden=None, level=None):
        if workspace is None:
            raise ValueError("a prepared call needs its workspace")
        self._fn, self._args, _, self.out, self._keep = _marshal_grouped(
            hidden, gate_W, gate_bias, lm_W, gi, g, k, topk_ids, topk_logits, sel_groups, workspace,
            None, None, logprob, gate_hidden, level)

    def __call__(self, stream=None):
        st = self._fn(*self._args, _stream_ptr(stream))
        if st:
            _raise(st)
        return self.out


NOALLOC_SCRATCH_BYTES = 8 << 20      # CORAL_NOALLOC_SCRATCH_BYTES of the header


def coral_lmhead_grouped_noalloc(hidden: torch.Tensor, gate_W: torch.Tensor,
                                 gate_bias: Optional[torch.Tensor], lm_W: torch.Tensor, gi: GroupIndex,
                                 g: int, k: int, topk_ids: torch.Tensor, topk_logits: torch.Tensor,
                                 sel_groups: Optional[torch.Tensor] = None, stream=None) -> None:
    """coral_lmhead_grouped_noalloc of the C ABI: the grouped head on the library's static
    scratch.  Nothing is allocated here either: the caller passes every output tensor."""
    dt = _dtype_code(hidden)
    if gate_W.dtype != hidden.dtype or lm_W.dtype != hidden.dtype:
        raise TypeError("hidden, gate_W and lm_W must share one dtype")
    if hidden.dim() != 2 or gate_W.dim() != 2 or lm_W.dim() != 2:
        raise ValueError("hidden, gate_W and lm_W must be 2-D")
    M, H = hidden.shape
    V = lm_W.shape[0]
    if lm_W.shape[1] != H or gate_W.shape != (gi.G, H) or gi.V != V:
        raise ValueError("inconsistent shapes")
    if gate_bias is not None and gate_bias.shape != (gi.G,):
        raise ValueError("gate_bias must be [G]")
    if topk_ids.shape != (M, k) or topk_logits.shape != (M, k) or \
            (sel_groups is not None and sel_groups.shape != (M, g)):
        raise ValueError("output shapes must be [M,k], [M,k], [M,g]")
    _raise(_L.coral_lmhead_grouped_noalloc(
        _dev_ptr(hidden, "hidden"), _dev_ptr(gate_W, "gate_W"),
        _dev_ptr(gate_bias, "gate_bias", torch.float32), _dev_ptr(lm_W, "lm_W"), gi.struct(),
        M, H, V, g, k, dt, _dev_ptr(topk_ids, "topk_ids", torch.int32),
        _dev_ptr(topk_logits, "topk_logits", torch.float32),
        _dev_ptr(sel_groups, "sel_groups", torch.int32), _stream_ptr(stream)))


def coral_probe_read(src: torch.Tensor, nbytes: int, waves: int, events, stream=None) -> None:
    """coral_probe_read of the C ABI: a kernel that only reads the first nbytes of src."""
    if not src.is_cuda or not src.is_contiguous() or src.numel() * src.element_size() < nbytes:
        raise ValueError("src must be a contiguous device tensor of at least nbytes bytes")
    _raise(_L.coral_probe_read(src.data_ptr(), int(nbytes), int(waves), _stream_ptr(stream),
                               events[0], events[1]))


ACTIVATIONS = {"silu": 0, "relu": 1, "identity": 2}


def coral_router_premix(hidden: torch.Tensor, W1: torch.Tensor, act: str = "silu",
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """coral_router_premix of the C ABI: u = act(W1 hidden) + hidden, [M,H] in hidden's dtype."""
    dt = _dtype_code(hidden)
    if W1.dtype != hidden.dtype:
        raise TypeError("hidden and W1 must share one dtype")
    if hidden.dim() != 2 or W1.shape != (hidden.shape[1], hidden.shape[1]):
        raise ValueError("W1 must be [H,H]")
    if act not in ACTIVATIONS:
        raise ValueError(f"unknown activation {act!r}")
    M, H = hidden.shape
    if out is None:
        out = torch.empty_like(hidden)
    if out.shape != hidden.shape or out.dtype != hidden.dtype:
        raise ValueError("out must match hidden")
    _raise(_L.coral_router_premix(_dev_ptr(hidden, "hidden"), _dev_ptr(W1, "W1"), M, H, dt,
                                  ACTIVATIONS[act], _dev_ptr(out, "out"), _stream_ptr(stream)))
    return out


def coral_tree_expand(parent_score: Optional[torch.Tensor], cand_ids: torch.Tensor,
                      cand_logp: torch.Tensor, n_next: int, stream=None
                      ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """coral_tree_expand of the C ABI: (parent index, token id, cumulative score), each [n_next]."""
    if cand_ids.dim() != 2 or cand_logp.shape != cand_ids.shape:
        raise ValueError("cand_ids and cand_logp must both be [M,k]")
    M, k = cand_ids.shape
    if parent_score is not None and parent_score.shape != (M,):
        raise ValueError("parent_score must be [M]")
    dev = cand_ids.device
    parent = torch.empty(n_next, dtype=torch.int32, device=dev)
    token = torch.empty(n_next, dtype=torch.int32, device=dev)
    score = torch.empty(n_next, dtype=torch.float32, device=dev)
    _raise(_L.coral_tree_expand(_dev_ptr(parent_score, "parent_score", torch.float32),
                                _dev_ptr(cand_ids, "cand_ids", torch.int32),
                                _dev_ptr(cand_logp, "cand_logp", torch.float32), M, k, int(n_next),
                                _dev_ptr(parent, "next_parent"), _dev_ptr(token, "next_token"),
                                _dev_ptr(score, "next_score"), _stream_ptr(stream)))
    return parent, token, score


def coral_lmhead_draft_level(hidden, gate_W, gate_bias, lm_W, gi, g, k, n_next: int,
                             parent_score: Optional[torch.Tensor] = None,
                             next_parent: Optional[torch.Tensor] = None,
                             next_token: Optional[torch.Tensor] = None,
                             next_score: Optional[torch.Tensor] = None, **kw):
    """coral_lmhead_draft_level of the C ABI: the log-probability head for the M nodes of a tree
    level and the level's expansion.  Returns (ids, log-probabilities, selected groups,
    parent index, token id, cumulative score), the last three [n_next]."""
    M = hidden.shape[0]
    dev = hidden.device
    if parent_score is not None and parent_score.shape != (M,):
        raise ValueError("parent_score must be [M]")
    if next_parent is None:
        next_parent = torch.empty(n_next, dtype=torch.int32, device=dev)
    if next_token is None:
        next_token = torch.empty(n_next, dtype=torch.int32, device=dev)
    if next_score is None:
        next_score = torch.empty(n_next, dtype=torch.float32, device=dev)
    if next_parent.shape != (n_next,) or next_token.shape != (n_next,) or next_score.shape != (n_next,):
        raise ValueError("next_parent, next_token and next_score must be [n_next]")
    ids, logp, sel = coral_lmhead_grouped(hidden, gate_W, gate_bias, lm_W, gi, g, k, logprob=True,
                                          level=(parent_score, n_next, next_parent, next_token, next_score),
                                          **kw)
    return ids, logp, sel, next_parent, next_token, next_score


def coral_lmhead_grouped_logprob(hidden, gate_W, gate_bias, lm_W, gi, g, k, **kw):
    """coral_lmhead_grouped_logprob of the C ABI: (ids, log-probabilities, selected groups)."""
    return coral_lmhead_grouped(hidden, gate_W, gate_bias, lm_W, gi, g, k, logprob=True, **kw)


def coral_lmhead_dense(hidden: torch.Tensor, lm_W: torch.Tensor, k: int,
                       topk_ids: Optional[torch.Tensor] = None,
                       topk_logits: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None, events=None
                       ) -> Tuple[torch.Tensor, torch.Tensor]:
    dt = _dtype_code(hidden)
    if lm_W.dtype != hidden.dtype:
        raise TypeError("hidden and lm_W must share one dtype")
    if hidden.dim() != 2 or lm_W.dim() != 2 or lm_W.shape[1] != hidden.shape[1]:
        raise ValueError("inconsistent shapes")
    M, H = hidden.shape
    V = lm_W.shape[0]
    dev = hidden.device
    if topk_ids is None:
        topk_ids = torch.empty((M, k), dtype=torch.int32, device=dev)
    if topk_logits is None:
        topk_logits = torch.empty((M, k), dtype=torch.float32, device=dev)
    if topk_ids.shape != (M, k) or topk_logits.shape != (M, k):
        raise ValueError("output shapes must be [M,k]")
    if workspace is None:
        workspace = alloc_workspace(M, H, V, 0, 0, k, dt, dev, stream)
    args = (_dev_ptr(hidden, "hidden"), _dev_ptr(lm_W, "lm_W"), M, H, V, k, dt,
            _dev_ptr(topk_ids, "topk_ids", torch.int32),
            _dev_ptr(topk_logits, "topk_logits", torch.float32), _dev_ptr(workspace, "workspace"),
            workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if events is None:
        st = _L.coral_lmhead_dense(*args)
    else:
        st = _L.coral_lmhead_dense_profiled(*args, events[0], events[1])
    _raise(st)
    return topk_ids, topk_logits


# ---------------------------------------------------------------- 4-bit products, rules on logits
def _same_device_ptr(t: Optional[torch.Tensor], name: str, device, dtype, shape) -> Optional[int]:
    """Pointer of a contiguous tensor of this type, device and shape (None: any 1-D one); None stays None."""
    if t is None:
        return None
    if t.dtype == dtype and t.device == device and (t.shape == shape if shape is not None else t.dim() == 1) \
            and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must live on {device}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous (row-major, no padding)")
    raise ValueError(f"{name} must be {'1-D' if shape is None else list(shape)}, got {list(t.shape)}")


# The device's current stream as a raw handle: without the object that torch.cuda.current_stream makes
# (1.8 of the 11 us that a call cost the host) where this PyTorch has that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _enqueue(fn, device, stream, *args) -> None:
    """Calls the library on the tensors' device and the given stream (None: the device's current one)."""
    if stream is None:
        handle = _raw_stream(device.index)
    elif stream.device != device:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors to {device}")
    else:
        handle = stream.cuda_stream
    if device.index == _current_device():
        st = fn(*args, handle)
    else:
        with torch.cuda.device(device):
            st = fn(*args, handle)
    if st:
        _raise(st)


def _new(shape, dtype, device, stream) -> torch.Tensor:
    """An output tensor whose memory the caching allocator holds for the stream that writes it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


_INT_MAX = 2 ** 31 - 1              # of the library's arguments: ctypes passes the lower half of what is larger


W4_CODES = {"int": 0, "e2m1": 1}
W4_MAX_K = 1 << 20                   # CORAL_W4_MAX_K of the header


def coral_matvec_w4(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, zeros: Optional[torch.Tensor] = None,
                    group: int = 128, code_type: str = "int", bias: Optional[torch.Tensor] = None,
                    residual: Optional[torch.Tensor] = None, act: str = "identity",
                    out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """coral_matvec_w4 of the C ABI: act(x W^T + bias) + residual with W [N,K] in 4 bits.

    codes [N,K/2] uint8, column 2j in the low half of byte j; scales [N,ceil(K/group)] in x's dtype;
    zeros the same shape in uint8 (None: 8; none for code_type "e2m1").  out_dtype: float32 (the
    default) or x's dtype."""
    dt = _dtype_code(x)
    if not x.is_cuda:
        raise ValueError("x must live in device memory")
    if x.dim() != 2 or codes.dim() != 2:
        raise ValueError("x and codes must be 2-D")
    if code_type not in W4_CODES:
        raise ValueError(f"unknown code type {code_type!r}")
    if act not in ACTIVATIONS:
        raise ValueError(f"unknown activation {act!r}")
    group = int(group)
    if group < 1:
        raise ValueError("group must be positive")
    M, K = x.shape
    N = codes.shape[0]
    if M > _INT_MAX or N > _INT_MAX or K > _INT_MAX or group > _INT_MAX:
        raise ValueError("sizes and group must fit 32 bits")
    n_groups = -(-K // group)
    if out is not None:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out must be {out_dtype}, got {out.dtype}")
        out_dtype = out.dtype
    elif out_dtype is None:
        out_dtype = torch.float32
    if out_dtype != torch.float32 and out_dtype != x.dtype:
        raise TypeError(f"the output must be float32 or {x.dtype}, got {out_dtype}")
    dev = x.device
    args = (_same_device_ptr(x, "x", dev, x.dtype, (M, K)),
            _same_device_ptr(codes, "codes", dev, torch.uint8, (N, K // 2)),
            _same_device_ptr(scales, "scales", dev, x.dtype, (N, n_groups)),
            _same_device_ptr(zeros, "zeros", dev, torch.uint8, (N, n_groups)),
            _same_device_ptr(bias, "bias", dev, torch.float32, (N,)),
            _same_device_ptr(residual, "residual", dev, x.dtype, (M, N)),
            M, N, K, group, W4_CODES[code_type], dt, ACTIVATIONS[act],
            CORAL_F32 if out_dtype == torch.float32 else dt)
    if out is None:
        out = _new((M, N), out_dtype, dev, stream)
    _enqueue(_L.coral_matvec_w4, dev, stream, *args, _same_device_ptr(out, "out", dev, out_dtype, (M, N)))
    return out


def _logit_rules(logits, history, ranges, penalties, bias_ids, bias_values, bias_ranges, mask):
    """The checked arguments of the calls on logits: (pointer, rules or None, M, V, storage type)."""
    dt = _dtype_code(logits)
    if not logits.is_cuda:
        raise ValueError("logits must live in device memory")
    if logits.dim() != 2:
        raise ValueError("logits must be [M,V]")
    if (history is None) != (ranges is None) or (history is None) != (penalties is None):
        raise ValueError("history, ranges and penalties go together")
    if (bias_ids is None) != (bias_values is None) or (bias_ids is None) != (bias_ranges is None):
        raise ValueError("bias_ids, bias_values and bias_ranges go together")
    M, V = logits.shape
    if M > _INT_MAX or V > _INT_MAX:
        raise ValueError("sizes must fit 32 bits")
    dev = logits.device
    rules = None
    if history is not None or bias_ids is not None or mask is not None:
        i32, f32 = torch.int32, torch.float32
        n_history = 0 if history is None else history.numel()
        n_biases = 0 if bias_ids is None else bias_ids.numel()
        if max(n_history, n_biases) > 1 << 29:
            raise ValueError("at most 2^29 tokens of history, and biases")
        rules = ctypes.byref(_LogitRulesStruct(
            _same_device_ptr(history, "history", dev, i32, None),
            _same_device_ptr(ranges, "ranges", dev, i32, (M, 4)),
            _same_device_ptr(penalties, "penalties", dev, f32, (M, 3)),
            _same_device_ptr(bias_ids, "bias_ids", dev, i32, None),
            _same_device_ptr(bias_values, "bias_values", dev, f32, (n_biases,)),
            _same_device_ptr(bias_ranges, "bias_ranges", dev, i32, (M, 2)),
            _same_device_ptr(mask, "mask", dev, i32, (M, -(-V // 32))), n_history, n_biases))
    return _same_device_ptr(logits, "logits", dev, logits.dtype, (M, V)), rules, M, V, dt


def coral_logits_adjust(logits: torch.Tensor, history: Optional[torch.Tensor] = None,
                        ranges: Optional[torch.Tensor] = None, penalties: Optional[torch.Tensor] = None,
                        bias_ids: Optional[torch.Tensor] = None, bias_values: Optional[torch.Tensor] = None,
                        bias_ranges: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """coral_logits_adjust of the C ABI: logits [M,V] under their rules, in their dtype.

    history [T] int32 token ids with ranges [M,4] int32 (prompt begin and end, output begin and end)
    and penalties [M,3] float32 (repetition, frequency, presence); bias_ids [B] int32 and bias_values
    [B] float32 with bias_ranges [M,2] int32; mask [M,ceil(V/32)] int32, bit v % 32 of word v // 32.
    out may be logits itself."""
    ptr, rules, M, V, dt = _logit_rules(logits, history, ranges, penalties, bias_ids, bias_values, bias_ranges, mask)
    if out is None:
        out = _new((M, V), logits.dtype, logits.device, stream)
    _enqueue(_L.coral_logits_adjust, logits.device, stream, ptr, rules, M, V, dt,
             _same_device_ptr(out, "out", logits.device, logits.dtype, (M, V)))
    return out


def coral_logits_topk_workspace_bytes(M: int, V: int, k: int) -> int:
    if not 0 < min(M, V, k) <= max(M, V, k) <= _INT_MAX:
        return 0
    return int(_L.coral_logits_topk_workspace_bytes(M, V, k))


def coral_logits_topk(logits: torch.Tensor, k: int, history: Optional[torch.Tensor] = None,
                      ranges: Optional[torch.Tensor] = None, penalties: Optional[torch.Tensor] = None,
                      bias_ids: Optional[torch.Tensor] = None, bias_values: Optional[torch.Tensor] = None,
                      bias_ranges: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                      topk_ids: Optional[torch.Tensor] = None, topk_logprob: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """coral_logits_topk of the C ABI: (ids, log-probabilities), each [M,k], of the k best tokens per
    row under the rules (arguments as for coral_logits_adjust); (-1, -inf) behind a row's last
    candidate.  workspace: prepared by coral_lmhead_workspace_init or zeros, and not shared by calls
    that may overlap; None allocates one."""
    ptr, rules, M, V, dt = _logit_rules(logits, history, ranges, penalties, bias_ids, bias_values, bias_ranges, mask)
    k = int(k)
    if abs(k) > _INT_MAX:
        raise ValueError("k must fit 32 bits")
    dev = logits.device
    if topk_ids is None:
        topk_ids = _new((M, max(k, 0)), torch.int32, dev, stream)
    if topk_logprob is None:
        topk_logprob = _new((M, max(k, 0)), torch.float32, dev, stream)
    if workspace is None:
        workspace = _new((max(coral_logits_topk_workspace_bytes(M, V, k), 1 << 15),), torch.uint8, dev, stream)
        _enqueue(_L.coral_lmhead_workspace_init, dev, stream, workspace.data_ptr(), workspace.numel())
    ws = _same_device_ptr(workspace, "workspace", dev, torch.uint8, None)
    _enqueue(_L.coral_logits_topk, dev, stream, ptr, rules, M, V, k, dt,
             _same_device_ptr(topk_ids, "topk_ids", dev, torch.int32, (M, k)),
             _same_device_ptr(topk_logprob, "topk_logprob", dev, torch.float32, (M, k)), ws, workspace.numel())
    return topk_ids, topk_logprob


# ---------------------------------------------------------------- a drafter's attention
class KV4Cache(NamedTuple):
    """Keys and values held in 4 bits (coral_kv4_cache of the C ABI), all uint8 and contiguous: codes
    [pages, kv_heads, page_size, head_dim/2], scales [pages, kv_heads, page_size, head_dim/32].  The
    calls take any tuple of these four."""
    k_codes: torch.Tensor
    k_scales: torch.Tensor
    v_codes: torch.Tensor
    v_scales: torch.Tensor


def alloc_kv4_cache(pages: int, page_size: int, kv_heads: int, head_dim: int, device="cuda") -> KV4Cache:
    """A cache of zeros."""
    return KV4Cache(*(torch.zeros((pages, kv_heads, page_size, n), dtype=torch.uint8, device=device)
                      for n in (head_dim // 2, head_dim // 32) * 2))


def _kv4_cache(cache, device):
    """(struct, page_size, kv_heads, head_dim) of four checked tensors."""
    k_codes, k_scales, v_codes, v_scales = cache
    codes = k_codes.shape
    if len(codes) != 4:
        raise ValueError("the cache's codes must be [pages, kv_heads, page_size, head_dim/2]")
    pages, kv_heads, page_size, half = codes
    if max(codes) > _INT_MAX // 2:
        raise ValueError("sizes must fit 32 bits")
    u8, scales = torch.uint8, (pages, kv_heads, page_size, half // 16)
    # what _same_device_ptr checks of each, in one expression (1 us less a call); it names what is wrong
    if not (k_codes.dtype is u8 and v_codes.dtype is u8 and k_scales.dtype is u8 and v_scales.dtype is u8
            and k_codes.device == device and v_codes.device == device and k_scales.device == device and v_scales.device == device
            and v_codes.shape == codes and k_scales.shape == scales and v_scales.shape == scales
            and k_codes.is_contiguous() and v_codes.is_contiguous() and k_scales.is_contiguous() and v_scales.is_contiguous()):
        for t, name in zip(cache, KV4Cache._fields):
            _same_device_ptr(t, name, device, u8, codes if name.endswith("codes") else scales)
    struct = _Kv4CacheStruct(k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr(), pages, page_size, kv_heads, half * 2)
    return ctypes.byref(struct), page_size, kv_heads, half * 2


def _like(t: torch.Tensor) -> torch.Tensor:
    """A dense tensor of this shape, type and device (1.3 us; torch.empty with the three of them 2.2)."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _heads_ptr(t: torch.Tensor, name: str, device, dtype) -> Tuple[int, int]:
    """(pointer, elements from token to token) of [T, heads, head_dim] with dense heads."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must live on {device}, got {t.device}")
    shape = t.shape
    if len(shape) != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim], got {list(shape)}")
    T, heads, D = shape
    if T > _INT_MAX or heads > _INT_MAX or D > _INT_MAX:
        raise ValueError("sizes must fit 32 bits")
    row, head, one = t.stride()
    if (one != 1 or head != D) and ((D > 1 and one != 1) or (heads > 1 and head != D)) and T and heads and D:
        raise ValueError(f"{name} must have its heads one behind the other (only the tokens may be further apart)")
    return t.data_ptr(), row if T > 1 and heads and D else heads * D


def _heads_out(out, like, name, device, stream) -> Tuple[torch.Tensor, int, int]:
    """(tensor, pointer, elements from token to token) of an output like `like`: the one given, or a new dense one."""
    if out is None:
        shape = like.shape
        out = _like(like) if stream is None else _new(shape, like.dtype, device, stream)
        return out, out.data_ptr(), shape[1] * shape[2]
    if out.shape != like.shape:
        raise ValueError(f"{name} must be {list(like.shape)}, got {list(out.shape)}")
    return (out, *_heads_ptr(out, name, device, like.dtype))


def _on_device(t: torch.Tensor, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    return t.device


def coral_qk_norm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: Optional[torch.Tensor] = None,
                       inv_freq: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                       k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                       q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, cache=None,
                       v: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None, stream=None
                       ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """coral_qk_norm_rope of the C ABI: (q, k) with each head's norm (weights [head_dim]; None: no norm) and
    rotated by positions [T] int32 times inv_freq [rot_dim/2] float32 (both None: no rotation).

    q [T,q_heads,head_dim] and k [T,kv_heads,head_dim] may be columns of a wider matrix, and one of them
    None; q_out and k_out may be q and k themselves.  With cache (see KV4Cache), v [T,kv_heads,head_dim]
    and slots [T] int32 the keys and values are appended to it too; k_out=False then leaves out the keys'
    own output (None comes back)."""
    first = q if q is not None else k
    if first is None:
        raise ValueError("q or k is needed")
    dt, dev, dtype = _dtype_code(first), _on_device(first, "q" if q is not None else "k"), first.dtype
    q_ptr = k_ptr = v_ptr = qo_ptr = ko_ptr = struct = slot_ptr = None
    q_row = k_row = v_row = qo_row = ko_row = q_heads = kv_heads = 0
    if q is not None:
        q_ptr, q_row = _heads_ptr(q, "q", dev, dtype)
        T, q_heads, D = q.shape
    if k is not None:
        k_ptr, k_row = _heads_ptr(k, "k", dev, dtype)
        k_tokens, kv_heads, k_dim = k.shape
        if q is None:
            T, D = k_tokens, k_dim
        elif k_tokens != T or k_dim != D:
            raise ValueError("q and k must have the same tokens and head_dim")
    if (positions is None) != (inv_freq is None):
        raise ValueError("positions and inv_freq go together")
    rope = _RopeStruct(_same_device_ptr(q_weight, "q_weight", dev, dtype, (D,)),
                       _same_device_ptr(k_weight, "k_weight", dev, dtype, (D,)),
                       _same_device_ptr(positions, "positions", dev, torch.int32, (T,)),
                       _same_device_ptr(inv_freq, "inv_freq", dev, torch.float32, None), float(eps),
                       0 if inv_freq is None else min(2 * inv_freq.numel(), _INT_MAX - 1), 1 if interleaved else 0)
    if cache is not None:
        if k is None or v is None or slots is None:
            raise ValueError("a cache goes with k, v and slots")
        struct = _kv4_cache(cache, dev)[0]
        v_ptr, v_row = _heads_ptr(v, "v", dev, dtype)
        if v.shape != k.shape:
            raise ValueError("v must have the shape of k")
        slot_ptr = _same_device_ptr(slots, "slots", dev, torch.int32, (T,))
    elif v is not None or slots is not None or k_out is False:
        raise ValueError("v, slots and k_out=False go with a cache")
    if q is None:
        q_out = None
    else:
        q_out, qo_ptr, qo_row = _heads_out(q_out, q, "q_out", dev, stream)
    if k is None or k_out is False:
        k_out = None
    else:
        k_out, ko_ptr, ko_row = _heads_out(k_out, k, "k_out", dev, stream)
    _enqueue(_L.coral_qk_norm_rope, dev, stream, q_ptr, q_row, k_ptr, k_row, ctypes.byref(rope), T, q_heads, kv_heads, D, dt,
             qo_ptr, qo_row, ko_ptr, ko_row, struct, v_ptr, v_row, slot_ptr)
    return q_out, k_out


def coral_kv4_append(cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, stream=None) -> None:
    """coral_kv4_append of the C ABI: tokens' keys and values [T,kv_heads,head_dim] into the places slots [T]
    int32 of the cache (page * page_size + place in the page; outside the cache: passed over)."""
    dt, dev = _dtype_code(k), _on_device(k, "k")
    struct, _, kv_heads, D = _kv4_cache(cache, dev)
    k_ptr, k_row = _heads_ptr(k, "k", dev, k.dtype)
    v_ptr, v_row = _heads_ptr(v, "v", dev, k.dtype)
    T, k_heads, k_dim = k.shape
    if k_heads != kv_heads or k_dim != D or v.shape != k.shape:
        raise ValueError(f"k and v must be [T, {kv_heads}, {D}] as the cache is")
    _enqueue(_L.coral_kv4_append, dev, stream, struct, k_ptr, k_row, v_ptr, v_row,
             _same_device_ptr(slots, "slots", dev, torch.int32, (T,)), T, dt)


def coral_kv4_read(cache, slots: torch.Tensor, dtype: torch.dtype, k_out: Optional[torch.Tensor] = None,
                   v_out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """coral_kv4_read of the C ABI: (k, v), each [T,kv_heads,head_dim] of dtype, as the cache holds them in the
    places slots [T] int32.  Rows of slots outside the cache are left as k_out and v_out were."""
    dev = _on_device(slots, "slots")
    struct, _, kv_heads, D = _kv4_cache(cache, dev)
    slot_ptr = _same_device_ptr(slots, "slots", dev, torch.int32, None)
    T = slots.numel()
    if T > _INT_MAX:
        raise ValueError("sizes must fit 32 bits")
    shape = (T, kv_heads, D)
    if k_out is None:
        k_out = _new(shape, dtype, dev, stream)
        k_ptr = k_out.data_ptr()
    else:
        k_ptr = _same_device_ptr(k_out, "k_out", dev, dtype, shape)
    if v_out is None:
        v_out = _like(k_out) if stream is None else _new(shape, dtype, dev, stream)
        v_ptr = v_out.data_ptr()
    else:
        v_ptr = _same_device_ptr(v_out, "v_out", dev, dtype, shape)
    _enqueue(_L.coral_kv4_read, dev, stream, struct, slot_ptr, T, _dtype_code(k_out), k_ptr, v_ptr)
    return k_out, v_out


KV4_MAX_ROWS = 64                    # rows of a sequence in one call of attention over the cache


def coral_attention_kv4_workspace_bytes(S: int, max_rows: int, max_length: int, q_heads: int, kv_heads: int, head_dim: int,
                                        dt: int) -> int:
    if not 0 <= min(S, max_rows, max_length, q_heads, kv_heads, head_dim) <= max(S, max_rows, max_length, q_heads, kv_heads, head_dim) <= _INT_MAX:
        return 0
    return int(_L.coral_attention_kv4_workspace_bytes(S, max_rows, max_length, q_heads, kv_heads, head_dim, dt))


def _scale_of(scale: Optional[float], head_dim: int) -> float:
    return 1.0 / math.sqrt(head_dim) if scale is None else float(scale)


def coral_attention_kv4(q: torch.Tensor, cache, page_table: torch.Tensor, lengths: torch.Tensor, q_offsets: torch.Tensor,
                        max_rows: int, max_length: Optional[int] = None, history: Optional[torch.Tensor] = None,
                        tree: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                        out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """coral_attention_kv4 of the C ABI: attention of q [T,q_heads,head_dim] over the 4-bit cache, [T,q_heads,head_dim].

    Sequence s has rows q_offsets[s] .. q_offsets[s+1] (int32 [S+1]; at most max_rows, 64), lengths[s] cached tokens
    (int32 [S], the rows' own among them) in pages page_table[s] (int32 [S,max_pages]).  Without tree a row sees itself
    and all older tokens; with history (int32 [S]) and tree (int64 [T]) the tokens before history[s], and of the 64 from
    there on those whose bit is set.  max_length: what the lengths may come to (None: what the page table holds).
    scale: None for 1/sqrt(head_dim).  workspace: coral_attention_kv4_workspace_bytes, prepared by
    coral_lmhead_workspace_init or zeros, and not shared by calls that may overlap; None allocates and fills one for
    this call (about 5 us)."""
    dt, dev, dtype = _dtype_code(q), _on_device(q, "q"), q.dtype
    struct, page_size, kv_heads, D = _kv4_cache(cache, dev)
    q_ptr, q_row = _heads_ptr(q, "q", dev, dtype)
    T, q_heads, q_dim = q.shape
    if q_dim != D:
        raise ValueError(f"q must be [T, q_heads, {D}] as the cache is")
    if page_table.dim() != 2:
        raise ValueError("page_table must be [S, max_pages]")
    S, max_pages = page_table.shape
    i32, max_rows = torch.int32, int(max_rows)
    max_length = min(max_pages * page_size, _INT_MAX) if max_length is None else int(max_length)
    if S > _INT_MAX or max_pages > _INT_MAX or abs(max_rows) > _INT_MAX or abs(max_length) > _INT_MAX:
        raise ValueError("sizes must fit 32 bits")
    args = (_same_device_ptr(page_table, "page_table", dev, i32, (S, max_pages)), max_pages,
            _same_device_ptr(lengths, "lengths", dev, i32, (S,)), _same_device_ptr(q_offsets, "q_offsets", dev, i32, (S + 1,)),
            _same_device_ptr(history, "history", dev, i32, (S,)), _same_device_ptr(tree, "tree", dev, torch.int64, (T,)))
    if out is None:
        out = _like(q) if stream is None else _new((T, q_heads, D), dtype, dev, stream)
        out_ptr = out.data_ptr()
    else:
        out_ptr = _same_device_ptr(out, "out", dev, dtype, (T, q_heads, D))
    if workspace is None:
        n = coral_attention_kv4_workspace_bytes(S, max_rows, max_length, q_heads, kv_heads, D, dt)
        workspace = _new((max(n, 512),), torch.uint8, dev, stream)
        _enqueue(_L.coral_lmhead_workspace_init, dev, stream, workspace.data_ptr(), workspace.numel())
    _enqueue(_L.coral_attention_kv4, dev, stream, q_ptr, q_row, struct, *args, T, S, max_rows, max_length, q_heads,
             _scale_of(scale, D), dt, out_ptr, _same_device_ptr(workspace, "workspace", dev, torch.uint8, None), workspace.numel())
    return out


def coral_attention_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor,
                           k_offsets: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                           out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """coral_attention_prompt of the C ABI: causal attention over packed sequences, [T,q_heads,head_dim].

    q [T,q_heads,head_dim]; k and v [keys,kv_heads,head_dim]; sequence s has rows q_offsets[s] .. q_offsets[s+1] (int32
    [S+1]) and keys k_offsets[s] .. k_offsets[s+1] (None: the same), its last row sees its last key.  scale: None for
    1/sqrt(head_dim)."""
    dt, dev, dtype = _dtype_code(q), _on_device(q, "q"), q.dtype
    q_ptr, q_row = _heads_ptr(q, "q", dev, dtype)
    k_ptr, k_row = _heads_ptr(k, "k", dev, dtype)
    v_ptr, v_row = _heads_ptr(v, "v", dev, dtype)
    T, q_heads, D = q.shape
    keys, kv_heads, k_dim = k.shape
    if k_dim != D or v.shape != k.shape:
        raise ValueError("k and v must have one shape, and q's head_dim")
    S = q_offsets.numel() - 1
    if S > _INT_MAX:
        raise ValueError("sizes must fit 32 bits")
    offsets_ptr = _same_device_ptr(q_offsets, "q_offsets", dev, torch.int32, (S + 1,))
    k_offsets_ptr = _same_device_ptr(k_offsets, "k_offsets", dev, torch.int32, (S + 1,))
    if out is None:
        out = _like(q) if stream is None else _new((T, q_heads, D), dtype, dev, stream)
        out_ptr = out.data_ptr()
    else:
        out_ptr = _same_device_ptr(out, "out", dev, dtype, (T, q_heads, D))
    _enqueue(_L.coral_attention_prompt, dev, stream, q_ptr, q_row, k_ptr, k_row, v_ptr, v_row, offsets_ptr, k_offsets_ptr, T, keys,
             S, q_heads, kv_heads, D, _scale_of(scale, D), dt, out_ptr)
    return out
