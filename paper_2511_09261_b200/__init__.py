"""Python binding of libgnnco (argument marshalling only).

Every step of the path runs inside the CUDA library; this module turns torch tensors
into raw pointers and calls the C ABI declared in ``include/gnnco.h`` with the same
names.  PyTorch is used for device memory and streams, nothing else.  There is no CPU
fallback: if the shared library is missing or cannot be loaded, importing the binding's
entry points raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

from . import _build

MAX_LAYERS = 8
OK = 0
INVALID_ARGUMENT, OUT_OF_RANGE, NOT_SIMPLE_GRAPH, UNSUPPORTED, WORKSPACE_TOO_SMALL, CUDA_ERROR, INTERNAL = (
    -1, -2, -3, -4, -5, -6, -7)
F32, BF16 = 0, 1
WANT_DX, FORWARD_ONLY, AX_STORE, AX_REUSE, WEIGHTS_UNTOUCHED, ACTIVE_ONLY, ONE_KERNEL_LAYERS = 1, 2, 4, 8, 16, 32, 64

EXPORTS = [
    "gnnco_status_string", "gnnco_partition_workspace_bytes", "gnnco_partition_load", "gnnco_graph_info",
    "gnnco_gather_rows", "gnnco_train_workspace_bytes", "gnnco_train_step", "gnnco_train_host_workspace_bytes",
    "gnnco_train_step_host", "gnnco_decode_boundary", "gnnco_async_status", "gnnco_launch_count", "gnnco_destroy",
    "gnnco_profile_begin", "gnnco_profile_end", "gnnco_objective_static", "gnnco_conflict_workspace_bytes",
    "gnnco_conflict_actions", "gnnco_apply_actions", "gnnco_gumbel_softmax", "gnnco_embedding_update",
    "gnnco_repair_boundary", "gnnco_partition_quality", "gnnco_active_plan_bytes", "gnnco_active_plan",
    "gnnco_louvain_workspace_bytes", "gnnco_louvain", "gnnco_embedding_lookup", "gnnco_embedding_plan_bytes",
    "gnnco_embedding_plan", "gnnco_embedding_grad", "gnnco_block_norm", "gnnco_block_norm_workspace_bytes",
    "gnnco_block_norm_backward", "gnnco_muon_workspace_bytes", "gnnco_muon_update", "gnnco_orthogonalise",
    "gnnco_dropout", "gnnco_gated_ff_workspace_bytes", "gnnco_gated_ff", "gnnco_gated_ff_backward",
]

_vp, _i32, _i64, _u32, _f32, _sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_float,
                                    ctypes.c_size_t)


class GraphDesc(ctypes.Structure):
    _fields_ = [("n", _i64), ("E", _i64), ("S", _i32), ("edge_u", _vp), ("edge_v", _vp), ("part", _vp)]


class GraphView(ctypes.Structure):
    _fields_ = [("n", _i64), ("S", _i32), ("E_in", _i64), ("E_b", _i64), ("max_row", _i32), ("perm", _vp),
                ("inv_perm", _vp), ("part_ptr", _vp), ("node_part", _vp), ("rowptr", _vp), ("colidx", _vp),
                ("bnd_u", _vp), ("bnd_v", _vp), ("inv_deg", _vp), ("is_boundary", _vp)]


class ModelDesc(ctypes.Structure):
    _fields_ = [("L", _i32), ("dims", _i32 * (MAX_LAYERS + 1)), ("feat_dtype", _i32), ("weight_sets", _i32),
                ("W", _vp * MAX_LAYERS)]


class Objective(ctypes.Structure):
    _fields_ = [("alpha", _f32), ("beta", _f32), ("lam", _f32), ("pen", _vp)]


class AdamState(ctypes.Structure):
    _fields_ = [("lr", _f32), ("beta1", _f32), ("beta2", _f32), ("eps", _f32), ("step", _i64),
                ("m", _vp * MAX_LAYERS), ("v", _vp * MAX_LAYERS), ("active", _vp), ("step_dev", _vp)]


class TrainOut(ctypes.Structure):
    _fields_ = [("loss", _vp), ("p", _vp), ("z", _vp), ("dW", _vp * MAX_LAYERS), ("dX", _vp), ("ax_cache", _vp)]


class ProfileEntry(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("calls", _i64), ("total_ms", ctypes.c_double)]


class BlockNormDesc(ctypes.Structure):
    _fields_ = [("rows", _i64), ("F", _i32), ("feat_dtype", _i32), ("eps", _f32), ("scale", _f32), ("x", _vp),
                ("x_ld", _i64), ("y", _vp), ("y_ld", _i64), ("gate", _vp), ("gate_ld", _i64), ("w_pre", _vp),
                ("w_post", _vp)]


class BlockNormGrads(ctypes.Structure):
    _fields_ = [("dx_out", _vp), ("dx_out_ld", _i64), ("dh", _vp), ("dh_ld", _i64), ("dx", _vp), ("dx_ld", _i64),
                ("dy", _vp), ("dy_ld", _i64), ("dgate", _vp), ("dgate_ld", _i64), ("dw_pre", _vp), ("dw_post", _vp)]


class MuonParams(ctypes.Structure):
    _fields_ = [("lr", _f32), ("momentum", _f32), ("weight_decay", _f32), ("nesterov", _i32), ("steps", _i32),
                ("a", _f32), ("b", _f32), ("c", _f32), ("eps", _f32), ("active", _vp)]


class DropoutParams(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("layer", _u32), ("step", _u32), ("step_dev", _vp)]


class GatedFfDesc(ctypes.Structure):
    _fields_ = [("rows", _i64), ("F", _i32), ("H", _i32), ("F_out", _i32), ("feat_dtype", _i32), ("w_dtype", _i32),
                ("sets", _i32), ("act", _i32), ("x", _vp), ("x_ld", _i64), ("w_gate", _vp), ("w_up", _vp),
                ("w_down", _vp), ("drop", ctypes.POINTER(DropoutParams))]


class GatedFfGrads(ctypes.Structure):
    _fields_ = [("dx", _vp), ("dx_ld", _i64), ("dw_gate", _vp), ("dw_up", _vp), ("dw_down", _vp), ("dw_dtype", _i32)]


class GnncoError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__("%s: %s (status %d)" % (what, status_string(status), status))
        self.status = status


_lib = None


def lib_path() -> str:
    return _build.LIB_PATH


def load_library(build_if_missing: bool = True):
    """Load libgnnco.so (building it in-tree first if it is absent or stale and nvcc is
    available).  Raises if the library cannot be produced or loaded."""
    global _lib
    if _lib is not None:
        return _lib
    if build_if_missing and _build.needs_build():
        _build.build()
    if not os.path.exists(_build.LIB_PATH):
        raise RuntimeError("libgnnco.so is missing: build it with paper_2511_09261_b200._build.build()")
    lib = ctypes.CDLL(_build.LIB_PATH)
    lib.gnnco_status_string.argtypes = [_i32]
    lib.gnnco_status_string.restype = ctypes.c_char_p
    lib.gnnco_partition_workspace_bytes.argtypes = [_i64, _i64, _i32, ctypes.POINTER(_sz), ctypes.POINTER(_sz)]
    lib.gnnco_partition_load.argtypes = [ctypes.POINTER(GraphDesc), _vp, _sz, _vp, _sz, _vp, ctypes.POINTER(_vp)]
    lib.gnnco_graph_info.argtypes = [_vp, ctypes.POINTER(GraphView)]
    lib.gnnco_gather_rows.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp]
    lib.gnnco_train_workspace_bytes.argtypes = [_vp, ctypes.POINTER(ModelDesc), _u32, ctypes.POINTER(_sz)]
    lib.gnnco_train_host_workspace_bytes.argtypes = [_vp, ctypes.POINTER(ModelDesc), _u32, ctypes.POINTER(_sz)]
    lib.gnnco_train_step.argtypes = [_vp, ctypes.POINTER(ModelDesc), _vp, ctypes.POINTER(Objective),
                                     ctypes.POINTER(AdamState), ctypes.POINTER(TrainOut), _u32, _vp, _sz, _vp]
    lib.gnnco_train_step_host.argtypes = [_vp, ctypes.POINTER(ModelDesc), _vp, _f32, _f32, _f32, _vp,
                                          ctypes.POINTER(AdamState), _vp, _vp, _u32, _vp, _sz, _vp]
    lib.gnnco_decode_boundary.argtypes = [_vp, _vp, _f32, _vp, _vp, _vp, _vp, _vp]
    lib.gnnco_async_status.argtypes = [_vp, _vp, ctypes.POINTER(_i32)]
    lib.gnnco_launch_count.argtypes = [_vp]
    lib.gnnco_launch_count.restype = _i64
    lib.gnnco_destroy.argtypes = [_vp]
    lib.gnnco_objective_static.argtypes = [_vp, _vp, ctypes.POINTER(Objective), _vp, _vp]
    lib.gnnco_profile_begin.argtypes = [_vp]
    lib.gnnco_profile_end.argtypes = [_vp, _vp, ctypes.POINTER(ProfileEntry), _i32, ctypes.POINTER(_i32)]
    lib.gnnco_conflict_workspace_bytes.argtypes = [_vp, ctypes.POINTER(_sz)]
    lib.gnnco_conflict_actions.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
    lib.gnnco_apply_actions.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.gnnco_partition_quality.argtypes = [_vp, _vp, _vp, _vp, _vp]
    lib.gnnco_repair_boundary.argtypes = [_vp, _vp, _vp, _vp, _vp]
    lib.gnnco_louvain_workspace_bytes.argtypes = [_i64, _i64, ctypes.POINTER(_sz)]
    lib.gnnco_louvain.argtypes = [_i64, _i64, _vp, _vp, _i32, _i32, _vp, ctypes.POINTER(_i32), ctypes.POINTER(_i64),
                                  ctypes.POINTER(_i64), ctypes.POINTER(_i32), ctypes.POINTER(_i32), _vp, _sz, _vp]
    lib.gnnco_active_plan_bytes.argtypes = [_vp, ctypes.POINTER(_sz)]
    lib.gnnco_active_plan.argtypes = [_vp, _vp, _vp, _sz, _vp, ctypes.POINTER(_i32)]
    lib.gnnco_gumbel_softmax.argtypes = [_vp, _i32, _i32, _vp, _vp, _f32, _vp, _vp]
    lib.gnnco_embedding_update.argtypes = [_vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _f32, _f32, _f32, _f32, _i64, _vp]
    lib.gnnco_embedding_lookup.argtypes = [_vp, _i32, _i32, _i64, _i32, _i32, _vp, _vp, _i64, _f32, _vp, _i64, _vp]
    lib.gnnco_embedding_plan_bytes.argtypes = [_i64, _i32, _i32, ctypes.POINTER(_sz)]
    lib.gnnco_embedding_plan.argtypes = [_vp, _vp, _i64, _i32, _i32, _vp, _sz, _vp]
    lib.gnnco_embedding_grad.argtypes = [_vp, _i32, _i32, _i64, _i32, _i32, _vp, _i64, _f32, _vp, _sz, _vp, _i64, _vp]
    lib.gnnco_block_norm.argtypes = [_vp, ctypes.POINTER(BlockNormDesc), _vp, _i64, _vp, _i64, _vp]
    lib.gnnco_block_norm_workspace_bytes.argtypes = [_vp, _i32, ctypes.POINTER(_sz)]
    lib.gnnco_block_norm_backward.argtypes = [_vp, ctypes.POINTER(BlockNormDesc), ctypes.POINTER(BlockNormGrads), _vp,
                                              _sz, _vp]
    lib.gnnco_muon_workspace_bytes.argtypes = [_vp, _i64, _i32, _i32, ctypes.POINTER(_sz)]
    lib.gnnco_muon_update.argtypes = [_vp, _i64, _i32, _i32, _vp, _vp, _vp, ctypes.POINTER(MuonParams), _vp, _sz, _vp]
    lib.gnnco_orthogonalise.argtypes = [_vp, _i32, _i32, _i64, _i32, _i32, _vp, _vp, ctypes.POINTER(MuonParams), _vp, _sz,
                                        _vp]
    lib.gnnco_dropout.argtypes = [_vp, _i32, _i64, _i32, _vp, _i64, ctypes.POINTER(DropoutParams), _vp, _i64, _vp]
    lib.gnnco_gated_ff_workspace_bytes.argtypes = [_vp, ctypes.POINTER(GatedFfDesc), _i32, ctypes.POINTER(_sz)]
    lib.gnnco_gated_ff.argtypes = [_vp, ctypes.POINTER(GatedFfDesc), _vp, _i64, _vp, _sz, _vp]
    lib.gnnco_gated_ff_backward.argtypes = [_vp, ctypes.POINTER(GatedFfDesc), _vp, _i64, ctypes.POINTER(GatedFfGrads),
                                            _vp, _sz, _vp]
    for name in EXPORTS:
        if name not in ("gnnco_status_string", "gnnco_launch_count"):
            getattr(lib, name).restype = _i32
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().gnnco_status_string(int(status)).decode()


def _check(status: int, what: str) -> None:
    if status != OK:
        raise GnncoError(status, what)


_current_raw_stream = None


def _stream_ptr(stream=None) -> int:
    """The given stream or the current one, as the pointer the C ABI takes.  (Asking torch for the pointer without
    building a Stream object takes 0.1 of the 3 microseconds: calls on small graphs are as long as that.)"""
    global _current_raw_stream
    if stream is not None:
        return int(stream.cuda_stream)
    if _current_raw_stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is None:
            _current_raw_stream = lambda: int(torch.cuda.current_stream().cuda_stream)  # noqa: E731
        else:
            torch.cuda.init()
            device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
            _current_raw_stream = lambda: raw(device())  # noqa: E731
    return _current_raw_stream()


def _dptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _require(t, dtype, what: str, device_type: str = "cuda"):
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_contiguous() or t.device.type != device_type:
        raise TypeError("%s must be a contiguous %s tensor of dtype %s" % (what, device_type, dtype))
    return t


def _int32(*sizes) -> None:
    """Refuses what the C ABI's 32-bit arguments would cut off (ctypes does not)."""
    for n in sizes:
        if not -0x80000000 <= n <= 0x7fffffff:
            raise ValueError("%d does not fit in 32 bits" % n)


_feat_codes = {}


def _feat_code(t, what: str) -> int:
    if not _feat_codes:
        import torch
        _feat_codes.update({torch.float32: F32, torch.bfloat16: BF16})
    code = _feat_codes.get(getattr(t, "dtype", None))
    if code is None:
        raise TypeError("%s must be a float32 or bfloat16 tensor" % what)
    return code


def _empty(shape, dtype, like, stream):
    """A tensor on ``like``'s device for a call on ``stream``: its memory comes from that stream's pool, so that work
    still queued on the current stream cannot own it."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    import torch
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _empty_as(like, shape, dtype, stream):
    """``_empty``, a little sooner where ``like`` has this very shape and type (small blocks take as long as their call)."""
    if stream is None and like.shape == shape and like.dtype == dtype and like.is_contiguous():
        import torch
        return torch.empty_like(like)
    return _empty(tuple(shape), dtype, like, stream)


ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}
MUON_COEFS = (3.4445, -4.7750, 2.0315)


class Model:
    """Shape and weights of the GCN (``gnnco_model_desc``).  ``W[l]`` is a float32 CUDA
    tensor [weight_sets, dims[l], dims[l+1]]."""

    def __init__(self, dims: Sequence[int], W: Sequence, feat_dtype: int = F32):
        import torch
        self.dims = [int(d) for d in dims]
        self.L = len(self.dims) - 1
        if self.L < 1 or self.L > MAX_LAYERS or len(W) != self.L:
            raise ValueError("need 1..%d layers and one weight tensor per layer" % MAX_LAYERS)
        self.W = [_require(w, torch.float32, "W[%d]" % l) for l, w in enumerate(W)]
        self.weight_sets = int(self.W[0].shape[0])
        for l, w in enumerate(self.W):
            if tuple(w.shape) != (self.weight_sets, self.dims[l], self.dims[l + 1]):
                raise ValueError("W[%d] has shape %s" % (l, tuple(w.shape)))
        self.feat_dtype = int(feat_dtype)

    def desc(self) -> ModelDesc:
        d = ModelDesc()
        d.L = self.L
        for k, v in enumerate(self.dims):
            d.dims[k] = v
        d.feat_dtype = self.feat_dtype
        d.weight_sets = self.weight_sets
        for l, w in enumerate(self.W):
            d.W[l] = w.data_ptr()
        return d

    @property
    def torch_feat_dtype(self):
        import torch
        return torch.bfloat16 if self.feat_dtype == BF16 else torch.float32


class Adam:
    """Adam moments and hyper-parameters (``gnnco_adam_state``); ``step`` is advanced by
    ``PartitionedGraph.train_step`` after each update."""

    def __init__(self, model: Model, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                 device_step: bool = False):
        import torch
        self.lr, self.beta1, self.beta2, self.eps = lr, beta1, beta2, eps
        self.step = 1
        self.active = None          # uint8 [S] device tensor: subgraphs being fine-tuned (None = all)
        # ``gnnco_adam_state.step_dev``: number of updates done so far, kept on the device (steps that use it can be
        # recorded in a CUDA graph and replayed)
        self.step_dev = torch.zeros(1, dtype=torch.int32, device=model.W[0].device) if device_step else None
        self.m = [torch.zeros_like(w) for w in model.W]
        self.v = [torch.zeros_like(w) for w in model.W]

    def desc(self) -> AdamState:
        a = AdamState()
        a.lr, a.beta1, a.beta2, a.eps, a.step = self.lr, self.beta1, self.beta2, self.eps, self.step
        for l in range(len(self.m)):
            a.m[l] = self.m[l].data_ptr()
            a.v[l] = self.v[l].data_ptr()
        a.active = _dptr(self.active)
        a.step_dev = _dptr(self.step_dev)
        return a


class Muon:
    """Momentum and hyper-parameters of orthogonalised updates (``gnnco_muon_params``) for every weight of a model;
    ``PartitionedGraph.muon_step`` applies one.  (A layer of width 1 gets its normalised gradient: the one singular
    vector there is.)"""

    def __init__(self, model: Model, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True,
                 weight_decay: float = 0.0, steps: int = 5, coefs: Sequence[float] = MUON_COEFS, eps: float = 1e-7):
        import torch
        self.lr, self.momentum, self.nesterov, self.weight_decay = lr, momentum, nesterov, weight_decay
        self.steps, self.coefs, self.eps = steps, tuple(coefs), eps
        self.active = None          # uint8 [weight_sets] device tensor: sets that are updated (None = all)
        self.m = [torch.zeros_like(w) for w in model.W]


class EmbeddingPlan:
    """Rows ordered by token (``gnnco_embedding_plan``); serves every gradient with the same tokens and width <= F."""

    def __init__(self, rows: int, V: int, F: int, ws, made_on: int):
        self.rows, self.V, self.F, self.ws = rows, V, F, ws
        self.made_on = made_on      # the stream that ws belongs to


class Dropout:
    """Which elements are dropped (``gnnco_dropout_params``): each with probability ``p``, decided by ``seed`` (64 bits),
    ``layer`` and ``step``.  ``step`` is advanced by the caller, after the backward pass; ``step_dev`` (int32 device tensor
    of one element, added to ``step``) is its form for recorded graphs."""

    def __init__(self, p: float, seed: int, layer: int = 0, step: int = 0, step_dev=None):
        self.p, self.seed, self.layer, self.step, self.step_dev = float(p), int(seed), int(layer), int(step), step_dev

    def params(self, device) -> DropoutParams:
        import torch
        if not 0.0 <= self.p <= 1.0:
            raise ValueError("p must be in [0, 1]")
        if self.seed >> 64 or self.layer >> 32 or self.step >> 32:
            raise ValueError("seed must fit in 64 bits, layer and step in 32, none below zero")
        if self.step_dev is not None:
            _require(self.step_dev, torch.int32, "step_dev")
            if self.step_dev.numel() != 1 or self.step_dev.device != device:
                raise ValueError("step_dev must be one int32 on %s" % device)
        return DropoutParams(self.p, self.seed, self.layer, self.step, _dptr(self.step_dev))


class PartitionedGraph:
    """Handle returned by ``gnnco_partition_load`` plus the torch buffers it lives in."""

    def __init__(self, edge_u, edge_v, part, S: int, stream=None):
        import torch
        lib = load_library()
        self._lib = lib
        self._handle = None
        n, E = int(part.numel()), int(edge_u.numel())
        _require(part, torch.int32, "part")
        _require(edge_u, torch.int32, "edge_u")
        _require(edge_v, torch.int32, "edge_v")
        if int(edge_v.numel()) != E:
            raise ValueError("edge_u and edge_v differ in length")
        self.device = part.device
        pb, sb = _sz(0), _sz(0)
        _check(lib.gnnco_partition_workspace_bytes(n, E, S, ctypes.byref(pb), ctypes.byref(sb)),
               "gnnco_partition_workspace_bytes")
        self._persistent = torch.empty(pb.value, dtype=torch.uint8, device=self.device)
        scratch = torch.empty(sb.value, dtype=torch.uint8, device=self.device)
        g = GraphDesc(n, E, S, _dptr(edge_u) if E else None, _dptr(edge_v) if E else None, _dptr(part))
        hp = _vp(0)
        st = lib.gnnco_partition_load(ctypes.byref(g), self._persistent.data_ptr(), pb.value, scratch.data_ptr(),
                                      sb.value, _stream_ptr(stream), ctypes.byref(hp))
        _check(st, "gnnco_partition_load")
        self._handle = hp
        del scratch
        v = GraphView()
        _check(lib.gnnco_graph_info(self._handle, ctypes.byref(v)), "gnnco_graph_info")
        self.n, self.S, self.E_in, self.E_b, self.max_row = int(v.n), int(v.S), int(v.E_in), int(v.E_b), int(v.max_row)
        self._view = v
        self._ws = None
        self._ws_key = None
        self._plan_ws = None
        self._plan_active = None
        self._plan_sizes = {}
        self._norm_sizes = {}

    # ---- views of the persistent area as torch tensors (no copies)
    def _view_tensor(self, ptr: int, count: int, dtype):
        import torch
        esz = torch.empty(0, dtype=dtype).element_size()
        off = ptr - self._persistent.data_ptr()
        return self._persistent[off: off + count * esz].view(dtype)

    def arrays(self) -> dict:
        import torch
        v = self._view
        return dict(
            perm=self._view_tensor(v.perm, self.n, torch.int32),
            inv_perm=self._view_tensor(v.inv_perm, self.n, torch.int32),
            part_ptr=self._view_tensor(v.part_ptr, self.S + 1, torch.int32),
            node_part=self._view_tensor(v.node_part, self.n, torch.int32),
            rowptr=self._view_tensor(v.rowptr, self.n + 1, torch.int32),
            colidx=self._view_tensor(v.colidx, 2 * self.E_in, torch.int32),
            bnd_u=self._view_tensor(v.bnd_u, self.E_b, torch.int32),
            bnd_v=self._view_tensor(v.bnd_v, self.E_b, torch.int32),
            inv_deg=self._view_tensor(v.inv_deg, self.n, torch.float32),
            is_boundary=self._view_tensor(v.is_boundary, self.n, torch.uint8),
        )

    def gather_rows(self, src, index, out=None, stream=None):
        """out[i] = src[index[i]] (``gnnco_gather_rows``)."""
        import torch
        rows = int(index.numel())
        row_bytes = src[0].numel() * src.element_size() if src.dim() > 1 else src.element_size()
        if out is None:
            out = torch.empty((rows,) + tuple(src.shape[1:]), dtype=src.dtype, device=src.device)
        _check(self._lib.gnnco_gather_rows(self._handle, src.data_ptr(), out.data_ptr(), index.data_ptr(), rows,
                                           row_bytes, _stream_ptr(stream)), "gnnco_gather_rows")
        return out

    def _workspace(self, model: Model, flags: int, host: bool):
        import torch
        key = (tuple(model.dims), model.feat_dtype, model.weight_sets, flags & FORWARD_ONLY, host)
        if self._ws_key != key:
            b = _sz(0)
            md = model.desc()
            fn = self._lib.gnnco_train_host_workspace_bytes if host else self._lib.gnnco_train_workspace_bytes
            _check(fn(self._handle, ctypes.byref(md), flags, ctypes.byref(b)), "gnnco_train_workspace_bytes")
            self._ws = None
            self._ws = torch.empty(max(256, b.value), dtype=torch.uint8, device=self.device)
            self._ws_key = key
        return self._ws

    def train_step(self, model: Model, X, alpha: float, beta: float, lam: float = 0.0, pen=None,
                   opt: Optional[Adam] = None, loss=None, p=None, z=None, dW: Optional[List] = None, dX=None,
                   flags: int = 0, stream=None, ax_cache=None):
        """One ``gnnco_train_step``.  Returns (loss, p).  Optional outputs are written
        into the tensors passed as ``z``, ``dW`` (list, entries may be None) and ``dX``;
        ``ax_cache`` ([n, dims[0]], the features' type) goes with AX_STORE / AX_REUSE."""
        import torch
        _require(X, model.torch_feat_dtype, "X")
        if tuple(X.shape) != (self.n, model.dims[0]):
            raise ValueError("X must be [n, dims[0]]")
        if loss is None:
            loss = torch.empty(self.S, dtype=torch.float32, device=self.device)
        if p is None:
            p = torch.empty(self.n, dtype=torch.float32, device=self.device)
        ws = self._workspace(model, flags, host=False)
        md = model.desc()
        obj = Objective(alpha, beta, lam, _dptr(pen))
        out = TrainOut()
        out.loss, out.p, out.z, out.dX = _dptr(loss), _dptr(p), _dptr(z), _dptr(dX)
        if ax_cache is not None:
            _require(ax_cache, model.torch_feat_dtype, "ax_cache")
            if tuple(ax_cache.shape) != (self.n, model.dims[0]):
                raise ValueError("ax_cache must be [n, dims[0]]")
            out.ax_cache = ax_cache.data_ptr()
        if dW is not None:
            for l, t in enumerate(dW):
                out.dW[l] = _dptr(t)
        ad = opt.desc() if opt is not None else None
        st = self._lib.gnnco_train_step(self._handle, ctypes.byref(md), X.data_ptr(), ctypes.byref(obj),
                                        ctypes.byref(ad) if ad is not None else None, ctypes.byref(out), flags,
                                        ws.data_ptr(), ws.numel(), _stream_ptr(stream))
        _check(st, "gnnco_train_step")
        if opt is not None and not (flags & FORWARD_ONLY):
            opt.step += 1
        return loss, p

    def train_step_host(self, model: Model, X_host, alpha: float, beta: float, lam: float = 0.0, pen_host=None,
                        opt: Optional[Adam] = None, loss_host=None, p_host=None, flags: int = 0, stream=None):
        """``gnnco_train_step_host``: per-step inputs and outputs are HOST tensors (pinned
        recommended); returns (loss_host, p_host) after the stream has been synchronised."""
        import torch
        _require(X_host, model.torch_feat_dtype, "X_host", "cpu")
        if loss_host is None:
            loss_host = torch.empty(self.S, dtype=torch.float32).pin_memory()
        if p_host is None:
            p_host = torch.empty(self.n, dtype=torch.float32).pin_memory()
        ws = self._workspace(model, flags, host=True)
        md = model.desc()
        ad = opt.desc() if opt is not None else None
        st = self._lib.gnnco_train_step_host(self._handle, ctypes.byref(md), X_host.data_ptr(), alpha, beta, lam,
                                             _dptr(pen_host), ctypes.byref(ad) if ad is not None else None,
                                             loss_host.data_ptr(), p_host.data_ptr(), flags, ws.data_ptr(),
                                             ws.numel(), _stream_ptr(stream))
        _check(st, "gnnco_train_step_host")
        if opt is not None and not (flags & FORWARD_ONLY):
            opt.step += 1
        return loss_host, p_host

    def decode_boundary(self, p, threshold: float = 0.5, x=None, viol=None, per_part=None, counts=None,
                        want_viol: bool = True, want_per_part: bool = True, stream=None):
        """``gnnco_decode_boundary``.  Returns dict(x, viol, per_part, counts) of device
        tensors; counts = int64[3] (set size, intra violations, boundary violations)."""
        import torch
        _require(p, torch.float32, "p")
        if x is None:
            x = torch.empty(self.n, dtype=torch.uint8, device=self.device)
        if viol is None and want_viol:
            viol = torch.empty(self.E_b, dtype=torch.uint8, device=self.device)
        if per_part is None and want_per_part:
            per_part = torch.empty(self.S, dtype=torch.int32, device=self.device)
        if counts is None:
            counts = torch.empty(3, dtype=torch.int64, device=self.device)
        st = self._lib.gnnco_decode_boundary(self._handle, p.data_ptr(), threshold, x.data_ptr(), _dptr(viol),
                                             _dptr(per_part), counts.data_ptr(), _stream_ptr(stream))
        _check(st, "gnnco_decode_boundary")
        return dict(x=x, viol=viol, per_part=per_part, counts=counts)

    def active_plan(self, active, stream=None) -> int:
        """``gnnco_active_plan``: work lists of the subgraphs with ``active[s] != 0`` (uint8 [S] device tensor,
        kept alive by the caller while the plan is in use) for steps with ACTIVE_ONLY.  Synchronises the
        stream; returns the number of active subgraphs."""
        import torch
        _require(active, torch.uint8, "active")
        if tuple(active.shape) != (self.S,):
            raise ValueError("active must be [S]")
        need = _sz(0)
        _check(self._lib.gnnco_active_plan_bytes(self._handle, ctypes.byref(need)), "gnnco_active_plan_bytes")
        if self._plan_ws is None or self._plan_ws.numel() < need.value:
            self._plan_ws = torch.empty(max(256, need.value), dtype=torch.uint8, device=self.device)
        count = _i32(0)
        _check(self._lib.gnnco_active_plan(self._handle, active.data_ptr(), self._plan_ws.data_ptr(),
                                           self._plan_ws.numel(), _stream_ptr(stream), ctypes.byref(count)),
               "gnnco_active_plan")
        self._plan_active = active
        return int(count.value)

    def conflict_actions(self, viol, p=None, want_action: bool = True, stream=None):
        """``gnnco_conflict_actions``.  Returns dict(conflict_idx, action, count): int32 [E_b]
        and uint8 [E_b] buffers of which the first ``count`` entries are valid, and the device
        int32 count itself (no host synchronisation)."""
        import torch
        _require(viol, torch.uint8, "viol")
        if want_action:
            _require(p, torch.float32, "p")
        need = _sz(0)
        _check(self._lib.gnnco_conflict_workspace_bytes(self._handle, ctypes.byref(need)),
               "gnnco_conflict_workspace_bytes")
        ws = torch.empty(need.value, dtype=torch.uint8, device=self.device)
        idx = torch.empty(self.E_b, dtype=torch.int32, device=self.device)
        action = torch.empty(self.E_b, dtype=torch.uint8, device=self.device) if want_action else None
        count = torch.empty(1, dtype=torch.int32, device=self.device)
        _check(self._lib.gnnco_conflict_actions(self._handle, viol.data_ptr(), _dptr(p) if want_action else None,
                                                idx.data_ptr(), _dptr(action), count.data_ptr(), ws.data_ptr(),
                                                need.value, _stream_ptr(stream)), "gnnco_conflict_actions")
        return dict(conflict_idx=idx, action=action, count=count)

    def apply_actions(self, conflict_idx, action, count, pen=None, active=None, stream=None):
        """``gnnco_apply_actions``.  Returns dict(pen, active, chosen): float32 [n], uint8 [S]
        and a device int32 with the number of distinct chosen nodes."""
        import torch
        _require(conflict_idx, torch.int32, "conflict_idx")
        _require(action, torch.uint8, "action")
        _require(count, torch.int32, "count")
        if pen is None:
            pen = torch.empty(self.n, dtype=torch.float32, device=self.device)
        if active is None:
            active = torch.empty(self.S, dtype=torch.uint8, device=self.device)
        chosen = torch.empty(1, dtype=torch.int32, device=self.device)
        _check(self._lib.gnnco_apply_actions(self._handle, conflict_idx.data_ptr(), action.data_ptr(),
                                             count.data_ptr(), pen.data_ptr(), active.data_ptr(), chosen.data_ptr(),
                                             _stream_ptr(stream)), "gnnco_apply_actions")
        return dict(pen=pen, active=active, chosen=chosen)

    def partition_quality(self, stream=None):
        """``gnnco_partition_quality``: dict(in_edges int64 [S], tot int64 [S], Q float64 [1]) on the device."""
        import torch
        in_edges = torch.empty(self.S, dtype=torch.int64, device=self.device)
        tot = torch.empty(self.S, dtype=torch.int64, device=self.device)
        Q = torch.empty(1, dtype=torch.float64, device=self.device)
        _check(self._lib.gnnco_partition_quality(self._handle, in_edges.data_ptr(), tot.data_ptr(), Q.data_ptr(),
                                                 _stream_ptr(stream)), "gnnco_partition_quality")
        return dict(in_edges=in_edges, tot=tot, Q=Q)

    def repair_boundary(self, pen, x, stream=None):
        """``gnnco_repair_boundary``: clears, in place, every chosen node (``pen`` != 0) from the
        mask ``x``; returns a device int32 with the number of selected nodes removed."""
        import torch
        _require(pen, torch.float32, "pen")
        _require(x, torch.uint8, "x")
        removed = torch.empty(1, dtype=torch.int32, device=self.device)
        _check(self._lib.gnnco_repair_boundary(self._handle, pen.data_ptr(), x.data_ptr(), removed.data_ptr(),
                                               _stream_ptr(stream)), "gnnco_repair_boundary")
        return removed

    def gumbel_softmax(self, E, U=None, tau: float = 1.0, out=None, stream=None):
        """``gnnco_gumbel_softmax``: rows of ``E`` ([n, F], float32 or bfloat16) through the
        Gumbel-softmax with uniforms ``U`` ([n, F] float32 in (0, 1), or None for no noise)."""
        import torch
        if E.dtype not in (torch.float32, torch.bfloat16) or E.dim() != 2 or E.shape[0] != self.n:
            raise ValueError("E must be [n, F] float32 or bfloat16")
        _require(E, E.dtype, "E")
        if U is not None:
            _require(U, torch.float32, "U")
            if tuple(U.shape) != tuple(E.shape):
                raise ValueError("U must have the shape of E")
        if out is None:
            out = torch.empty_like(E)
        _require(out, E.dtype, "out")
        dt = BF16 if E.dtype == torch.bfloat16 else F32
        _check(self._lib.gnnco_gumbel_softmax(self._handle, dt, int(E.shape[1]), E.data_ptr(), _dptr(U), float(tau),
                                              out.data_ptr(), _stream_ptr(stream)), "gnnco_gumbel_softmax")
        return out

    def embedding_update(self, dX, X_master, m, v, X, lr: float, step: int, beta1: float = 0.9,
                         beta2: float = 0.999, eps: float = 1e-8, stream=None):
        """``gnnco_embedding_update``: one Adam step on the float32 master embeddings with the
        gradient ``dX`` of a WANT_DX training step; ``X`` receives them in the features' type."""
        import torch
        for t, what in ((X_master, "X_master"), (m, "m"), (v, "v")):
            _require(t, torch.float32, what)
        _require(dX, X.dtype, "dX")
        _require(X, X.dtype, "X")
        if X.dtype not in (torch.float32, torch.bfloat16) or X.dim() != 2 or X.shape[0] != self.n:
            raise ValueError("X must be [n, F] float32 or bfloat16")
        for t in (dX, X_master, m, v):
            if tuple(t.shape) != tuple(X.shape):
                raise ValueError("dX, X_master, m, v and X must have the same shape")
        dt = BF16 if X.dtype == torch.bfloat16 else F32
        _check(self._lib.gnnco_embedding_update(self._handle, dt, int(X.shape[1]), dX.data_ptr(), X_master.data_ptr(),
                                                m.data_ptr(), v.data_ptr(), X.data_ptr(), float(lr), float(beta1),
                                                float(beta2), float(eps), int(step), _stream_ptr(stream)),
               "gnnco_embedding_update")
        return X

    # ---- shared input embeddings, norms around a block, orthogonalised updates

    def _rows(self, t, dtype, rows: int, F: int, what: str) -> int:
        """Checks a [rows, F] tensor whose rows are consecutive elements; returns the distance between rows."""
        if getattr(t, "dtype", None) != dtype or t.device != self.device or t.dim() != 2:
            raise TypeError("%s must be a 2-D %s tensor on %s" % (what, dtype, self.device))
        r, f = t.shape
        if r != rows or f != F:
            raise ValueError("%s must be [%d, %d]" % (what, rows, F))
        ld, step = t.stride()
        if r and f > 1 and step != 1 or r > 1 and ld < f:       # (without rows the strides mean nothing)
            raise ValueError("%s must have rows of consecutive elements that do not overlap" % what)
        return ld if r > 1 else max(f, 1)

    def _tokens(self, tokens) -> int:
        import torch
        _require(tokens, torch.int32, "tokens")
        if tokens.dim() != 1 or tokens.device != self.device:
            raise ValueError("tokens must be one-dimensional and on %s" % self.device)
        return tokens.shape[0]

    def embedding_lookup(self, table, tokens, scale: float = 1.0, out=None, out_dtype=None, stream=None):
        """``gnnco_embedding_lookup``: scale * table[tokens] for ``tokens`` int32 [rows]; a negative token gives zeros.
        ``table`` [V, F] and ``out`` [rows, F] are float32 or bfloat16 (``out_dtype`` defaults to the table's) and
        may be columns of wider tensors."""
        td = _feat_code(table, "table")
        rows = self._tokens(tokens)
        if table.dim() != 2 or 0 in table.shape:
            raise ValueError("table must be [V, F]")
        V, F = table.shape
        if (V | F) >> 31:
            _int32(V, F)
        table_ld = self._rows(table, table.dtype, V, F, "table")
        if out is None:
            if out_dtype is not None and out_dtype not in _feat_codes:
                raise TypeError("out_dtype must be float32 or bfloat16")
            out = _empty((rows, F), out_dtype or table.dtype, table, stream)
            od, out_ld = _feat_codes[out.dtype], F
        else:
            od = _feat_code(out, "out")
            out_ld = self._rows(out, out.dtype, rows, F, "out")
        _check(self._lib.gnnco_embedding_lookup(self._handle, td, od, rows, V, F, tokens.data_ptr(), table.data_ptr(),
                                                table_ld, scale, out.data_ptr(), out_ld, _stream_ptr(stream)),
               "gnnco_embedding_lookup")
        return out

    def embedding_plan(self, tokens, V: int, F: int, stream=None) -> EmbeddingPlan:
        """``gnnco_embedding_plan``: order of ``tokens`` (int32 [rows]) for gradients of tables [V, <= F].  No host
        synchronisation."""
        import torch
        rows = self._tokens(tokens)
        if (V | F) >> 31:
            _int32(V, F)
        need = self._plan_sizes.get((rows, V, F))
        if need is None:
            b = _sz(0)
            _check(self._lib.gnnco_embedding_plan_bytes(rows, V, F, ctypes.byref(b)), "gnnco_embedding_plan_bytes")
            need = self._plan_sizes[(rows, V, F)] = b.value
        ws = _empty((need,), torch.uint8, tokens, stream)
        on = _stream_ptr(stream)
        _check(self._lib.gnnco_embedding_plan(self._handle, tokens.data_ptr(), rows, V, F, ws.data_ptr(), need, on),
               "gnnco_embedding_plan")
        return EmbeddingPlan(rows, V, F, ws, on)

    def embedding_grad(self, plan: EmbeddingPlan, dout, scale: float = 1.0, out=None, out_dtype=None, stream=None):
        """``gnnco_embedding_grad``: gradient [V, F] of the table of ``embedding_lookup`` for the plan's tokens, from
        ``dout`` [rows, F] (float32 or bfloat16); float32 unless ``out`` or ``out_dtype`` says bfloat16."""
        import torch
        gd = _feat_code(dout, "dout")
        if dout.dim() != 2 or not 1 <= dout.shape[1] <= plan.F:
            raise ValueError("dout must be [rows, F] with F up to the plan's")
        F, V, ws = dout.shape[1], plan.V, plan.ws
        if ws.device != self.device:
            raise ValueError("plan must be one of %s" % self.device)
        dout_ld = self._rows(dout, dout.dtype, plan.rows, F, "dout")
        if out is None:
            if out_dtype is not None and out_dtype not in _feat_codes:
                raise TypeError("out_dtype must be float32 or bfloat16")
            out = _empty((V, F), out_dtype or torch.float32, dout, stream)
            od, out_ld = _feat_codes[out.dtype], F
        else:
            od = _feat_code(out, "out")
            out_ld = self._rows(out, out.dtype, V, F, "out")
        on = _stream_ptr(stream)
        _check(self._lib.gnnco_embedding_grad(self._handle, gd, od, plan.rows, V, F, dout.data_ptr(), dout_ld, scale,
                                              ws.data_ptr(), ws.shape[0], out.data_ptr(), out_ld, on),
               "gnnco_embedding_grad")
        if on != plan.made_on:      # the area must outlive this use, wherever the plan is dropped
            ws.record_stream(torch.cuda.current_stream() if stream is None else stream)
        return out

    def _weight(self, w, F, what: str):
        import torch
        if w is None:
            return None
        _require(w, torch.float32, what)
        if w.dim() != 1 or w.shape[0] != F or w.device != self.device:
            raise ValueError("%s must be [F] on %s" % (what, self.device))
        return w.data_ptr()

    def _block_desc(self, x, w_pre, y, w_post, gate, scale, eps):
        dt = _feat_code(x, "x")
        if x.dim() != 2 or x.shape[1] < 1:
            raise ValueError("x must be [rows, F]")
        if y is None and (gate is not None or w_post is not None):
            raise ValueError("gate and w_post belong to a block output y")
        rows, F = x.shape
        if F >> 31:
            _int32(F)
        d = BlockNormDesc(rows, F, dt, eps, scale, x.data_ptr(), self._rows(x, x.dtype, rows, F, "x"))
        if y is not None:
            d.y, d.y_ld = y.data_ptr(), self._rows(y, x.dtype, rows, F, "y")
        if gate is not None:
            if gate.dim() == 1:
                d.gate = self._weight(gate, F, "gate")
            else:
                d.gate, d.gate_ld = gate.data_ptr(), self._rows(gate, x.dtype, rows, F, "gate")
        d.w_pre, d.w_post = self._weight(w_pre, F, "w_pre"), self._weight(w_post, F, "w_post")
        return d

    def block_norm(self, x, w_pre=None, y=None, w_post=None, gate=None, scale: float = 1.0, eps: float = 1e-6, x_out=None,
                   h_out=None, want_h: bool = True, stream=None):
        """``gnnco_block_norm``: (x_out, h) with x_out = x + scale * gate * norm(y) * w_post and h = norm(x_out) * w_pre.
        Without ``y`` x_out is x; with want_h=False h is None.  ``gate``: None, float32 [F] or [rows, F] like x."""
        d = self._block_desc(x, w_pre, y, w_post, gate, scale, eps)
        rows, F, dtype = d.rows, d.F, x.dtype
        x_ld = h_ld = F
        if y is None:
            if x_out is not None:
                raise ValueError("x_out belongs to a block output y")
        elif x_out is None:
            x_out = _empty((rows, F), dtype, x, stream)
        else:
            x_ld = self._rows(x_out, dtype, rows, F, "x_out")
        if h_out is not None:
            h_ld = self._rows(h_out, dtype, rows, F, "h_out")
        elif want_h:
            h_out = _empty((rows, F), dtype, x, stream)
        _check(self._lib.gnnco_block_norm(self._handle, ctypes.byref(d), _dptr(x_out), x_ld, _dptr(h_out), h_ld,
                                          _stream_ptr(stream)), "gnnco_block_norm")
        return (x if y is None else x_out), h_out

    def block_norm_backward(self, x, dh=None, w_pre=None, dx_out=None, y=None, w_post=None, gate=None, scale: float = 1.0,
                            eps: float = 1e-6, dx=None, dy=None, dgate=None, stream=None):
        """``gnnco_block_norm_backward``: ``x`` is the stream after the block (the forward call's x_out).  Returns
        dict(dx, dy, dgate, dw_pre, dw_post); entries whose input was not given are None."""
        import torch
        d = self._block_desc(x, w_pre, y, w_post, gate, scale, eps)
        if y is None and dy is not None or gate is None and dgate is not None:
            raise ValueError("dy belongs to a block output y, dgate to a gate")
        rows, F, dtype = d.rows, d.F, x.dtype
        shape = (rows, F)
        g = BlockNormGrads()
        if dh is not None:
            g.dh, g.dh_ld = dh.data_ptr(), self._rows(dh, dtype, rows, F, "dh")
        if dx_out is not None:
            g.dx_out, g.dx_out_ld = dx_out.data_ptr(), self._rows(dx_out, dtype, rows, F, "dx_out")
        if dx is None:
            dx = _empty(shape, dtype, x, stream)
        g.dx, g.dx_ld = dx.data_ptr(), self._rows(dx, dtype, rows, F, "dx")
        if y is not None:
            if dy is None:
                dy = _empty(shape, dtype, x, stream)
            g.dy, g.dy_ld = dy.data_ptr(), self._rows(dy, dtype, rows, F, "dy")
        # the sums over rows share one allocation
        summed = (w_pre is not None) + (w_post is not None) + (gate is not None and gate.dim() == 1 and dgate is None)
        vectors = iter(_empty((summed, F), torch.float32, x, stream).unbind(0) if summed else ())
        if gate is not None:
            if gate.dim() == 1:
                if dgate is None:
                    dgate = next(vectors)
                g.dgate = self._weight(dgate, F, "dgate")
            else:
                if dgate is None:
                    dgate = _empty(shape, dtype, x, stream)
                g.dgate, g.dgate_ld = dgate.data_ptr(), self._rows(dgate, dtype, rows, F, "dgate")
        dw_pre = dw_post = None
        if w_pre is not None:
            dw_pre = next(vectors)
            g.dw_pre = dw_pre.data_ptr()
        if w_post is not None:
            dw_post = next(vectors)
            g.dw_post = dw_post.data_ptr()
        # a work area of its own for every call: callers on other threads and recorded graphs must not share one
        need = self._norm_sizes.get(F)
        if need is None:
            b = _sz(0)
            _check(self._lib.gnnco_block_norm_workspace_bytes(self._handle, F, ctypes.byref(b)),
                   "gnnco_block_norm_workspace_bytes")
            need = self._norm_sizes[F] = b.value
        ws = _empty((need,), torch.uint8, x, stream)
        _check(self._lib.gnnco_block_norm_backward(self._handle, ctypes.byref(d), ctypes.byref(g), ws.data_ptr(), need,
                                                   _stream_ptr(stream)), "gnnco_block_norm_backward")
        return dict(dx=dx, dy=dy, dgate=dgate, dw_pre=dw_pre, dw_post=dw_post)

    def dropout(self, x, drop: Dropout, out=None, stream=None):
        """``gnnco_dropout``: ``x`` [rows, F] with the elements that ``drop`` names set to 0 and the others scaled by
        1 / (1 - p).  Its gradient is the same call on the gradient."""
        dt = _feat_code(x, "x")
        if x.dim() != 2 or x.shape[1] < 1:
            raise ValueError("x must be [rows, F]")
        rows, F = x.shape
        if F >> 31:
            _int32(F)
        d = drop.params(self.device)
        x_ld = self._rows(x, x.dtype, rows, F, "x")
        out_ld = F
        if out is None:
            out = _empty_as(x, (rows, F), x.dtype, stream)
        else:
            out_ld = self._rows(out, x.dtype, rows, F, "out")
        _check(self._lib.gnnco_dropout(self._handle, dt, rows, F, x.data_ptr(), x_ld, ctypes.byref(d), out.data_ptr(), out_ld,
                                       _stream_ptr(stream)), "gnnco_dropout")
        return out

    def _gated_ff_desc(self, x, w_gate, w_up, w_down, act, drop):
        xd, wd = _feat_code(x, "x"), _feat_code(w_gate, "w_gate")
        if x.dim() != 2 or w_gate.dim() != 3:
            raise ValueError("x must be [rows, F], w_gate [sets, F, H]")
        rows, F = x.shape
        sets, _, H = w_gate.shape
        dtype, device = w_gate.dtype, self.device
        for w, what in ((w_gate, "w_gate"), (w_up, "w_up"), (w_down, "w_down")):
            if getattr(w, "dtype", None) != dtype or not w.is_contiguous() or w.device != device:
                raise TypeError("%s must be a contiguous %s tensor on %s" % (what, dtype, device))
        F_out = w_down.shape[-1]
        if (w_gate.shape != (sets, F, H) or w_up.shape != (sets, F, H) or w_down.shape != (sets, H, F_out)
                or not (sets and F and H and F_out)):
            raise ValueError("x [rows, F] takes w_gate and w_up [sets, F, H] and w_down [sets, H, F_out]")
        if sets != 1 and (sets != self.S or rows != self.n):
            raise ValueError("weights of %d sets need the %d rows of %d subgraphs" % (sets, self.n, self.S))
        code = ACTIVATIONS.get(act)
        if code is None:
            raise ValueError("act must be one of %s" % ", ".join(ACTIVATIONS))
        if (F | H | F_out) >> 31:
            _int32(F, H, F_out)
        d = GatedFfDesc(rows, F, H, F_out, xd, wd, sets, code, x.data_ptr(), self._rows(x, x.dtype, rows, F, "x"),
                        w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr())
        if drop is not None:
            d.drop = ctypes.pointer(drop.params(device))
        return d

    def _gated_ff_area(self, d, backward, like, ws, stream):
        import torch
        need = _sz(0)
        _check(self._lib.gnnco_gated_ff_workspace_bytes(self._handle, ctypes.byref(d), backward, ctypes.byref(need)),
               "gnnco_gated_ff_workspace_bytes")
        if ws is None:
            return _empty((need.value,), torch.uint8, like, stream)
        _require(ws, torch.uint8, "ws")
        if ws.device != self.device:
            raise ValueError("ws must be on %s" % self.device)
        return ws

    def gated_ff(self, x, w_gate, w_up, w_down, act: str = "silu", drop: Optional[Dropout] = None, out=None, ws=None,
                 stream=None):
        """``gnnco_gated_ff``: drop((act(x Wg) * (x Wu)) Wd) for ``x`` [rows, F], ``w_gate`` and ``w_up`` [sets, F, H] and
        ``w_down`` [sets, H, F_out], one set for all rows or one per subgraph.  The weights have x's type or are float32.
        ``ws`` may be a uint8 tensor kept between calls that follow each other on one stream."""
        d = self._gated_ff_desc(x, w_gate, w_up, w_down, act, drop)
        y_ld = d.F_out
        if out is None:
            out = _empty_as(x, (d.rows, y_ld), x.dtype, stream)
        else:
            y_ld = self._rows(out, x.dtype, d.rows, y_ld, "out")
        ws = self._gated_ff_area(d, 0, x, ws, stream)
        _check(self._lib.gnnco_gated_ff(self._handle, ctypes.byref(d), out.data_ptr(), y_ld, ws.data_ptr(), ws.numel(),
                                        _stream_ptr(stream)), "gnnco_gated_ff")
        return out

    def gated_ff_backward(self, x, dy, w_gate, w_up, w_down, act: str = "silu", drop: Optional[Dropout] = None,
                          want_dx: bool = True, want_dw: bool = True, dw_dtype=None, dx=None, ws=None, stream=None):
        """``gnnco_gated_ff_backward``: gradients of ``gated_ff`` for the gradient ``dy`` [rows, F_out] of its result, from the
        same ``x`` (nothing else is kept from the forward call), as dict(dx, dw_gate, dw_up, dw_down); None for what is not
        wanted.  The weights' gradients have the weights' type unless ``dw_dtype`` says otherwise."""
        d = self._gated_ff_desc(x, w_gate, w_up, w_down, act, drop)
        dy_ld = self._rows(dy, x.dtype, d.rows, d.F_out, "dy")
        if not (want_dx or want_dw) or dx is not None and not want_dx:
            raise ValueError("nothing is wanted, or dx is given and not wanted")
        g = GatedFfGrads()
        if want_dx:
            g.dx_ld = d.F
            if dx is None:
                dx = _empty_as(x, (d.rows, d.F), x.dtype, stream)
            else:
                g.dx_ld = self._rows(dx, x.dtype, d.rows, d.F, "dx")
            g.dx = dx.data_ptr()
        dws = [None, None, None]
        if want_dw:
            dw_dtype = dw_dtype or w_gate.dtype
            if dw_dtype not in _feat_codes:
                raise TypeError("dw_dtype must be float32 or bfloat16")
            dws = [_empty_as(w, w.shape, dw_dtype, stream) for w in (w_gate, w_up, w_down)]
            g.dw_gate, g.dw_up, g.dw_down = (t.data_ptr() for t in dws)
            g.dw_dtype = _feat_codes[dw_dtype]
        ws = self._gated_ff_area(d, 1, x, ws, stream)
        _check(self._lib.gnnco_gated_ff_backward(self._handle, ctypes.byref(d), dy.data_ptr(), dy_ld, ctypes.byref(g),
                                                 ws.data_ptr(), ws.numel(), _stream_ptr(stream)),
               "gnnco_gated_ff_backward")
        return dict(dx=dx, dw_gate=dws[0], dw_up=dws[1], dw_down=dws[2])

    def _muon_call(self, like, steps, active, stream, ws):
        import torch
        sets, r, c = like.shape
        if (r | c | steps) >> 31:
            _int32(r, c, steps)
        if active is not None:
            _require(active, torch.uint8, "active")
            if tuple(active.shape) != (sets,) or active.device != self.device:
                raise ValueError("active must be [sets]")
        need = _sz(0)
        _check(self._lib.gnnco_muon_workspace_bytes(self._handle, sets, r, c, ctypes.byref(need)),
               "gnnco_muon_workspace_bytes")
        if ws is None:
            ws = _empty((max(256, need.value),), torch.uint8, like, stream)
        else:
            _require(ws, torch.uint8, "ws")
            if ws.device != self.device:
                raise ValueError("ws must be on %s" % self.device)
        return sets, r, c, ws

    def muon_update(self, W, m, dW, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True,
                    weight_decay: float = 0.0, steps: int = 5, coefs: Sequence[float] = MUON_COEFS, eps: float = 1e-7,
                    active=None, ws=None, stream=None):
        """``gnnco_muon_update``: one orthogonalised update of ``W`` [sets, d_in, d_out] (float32, in place) with the
        gradient ``dW`` and the momentum ``m`` (in place); ``active`` uint8 [sets] restricts it.  ``ws`` may be a
        uint8 tensor kept between calls."""
        import torch
        for t, what in ((W, "W"), (m, "m"), (dW, "dW")):
            _require(t, torch.float32, what)
            if t.dim() != 3 or t.shape != W.shape or t.device != self.device:
                raise ValueError("W, m and dW must be [sets, d_in, d_out] on %s" % self.device)
        sets, r, c, ws = self._muon_call(W, steps, active, stream, ws)
        p = MuonParams(lr, momentum, weight_decay, int(nesterov), steps, coefs[0], coefs[1], coefs[2], eps, _dptr(active))
        _check(self._lib.gnnco_muon_update(self._handle, sets, r, c, W.data_ptr(), m.data_ptr(), dW.data_ptr(),
                                           ctypes.byref(p), ws.data_ptr(), ws.numel(), _stream_ptr(stream)),
               "gnnco_muon_update")
        return W

    def muon_step(self, model: Model, opt: Muon, dW: Sequence, stream=None) -> None:
        """One ``muon_update`` of every layer of ``model`` with the gradients ``dW`` of a training step."""
        if not len(model.W) == len(opt.m) == len(dW):
            raise ValueError("%d layers, %d momenta, %d gradients" % (len(model.W), len(opt.m), len(dW)))
        for W, m, g in zip(model.W, opt.m, dW):
            self.muon_update(W, m, g, opt.lr, opt.momentum, opt.nesterov, opt.weight_decay, opt.steps, opt.coefs, opt.eps,
                             opt.active, stream=stream)

    def orthogonalise(self, G, out=None, out_dtype=None, steps: int = 5, coefs: Sequence[float] = MUON_COEFS,
                      eps: float = 1e-7, active=None, ws=None, stream=None):
        """``gnnco_orthogonalise``: the Newton-Schulz iterate of every matrix of ``G`` [sets, rows, cols] (float32 or
        bfloat16)."""
        gd = _feat_code(G, "G")
        _require(G, G.dtype, "G")
        if G.dim() != 3 or 0 in G.shape or G.device != self.device:
            raise ValueError("G must be [sets, rows, cols] on %s" % self.device)
        if out is None:
            out = _empty(tuple(G.shape), out_dtype or G.dtype, G, stream)
        od = _feat_code(out, "out")
        _require(out, out.dtype, "out")
        if out.shape != G.shape or out.device != self.device:
            raise ValueError("out must have the shape of G")
        sets, r, c, ws = self._muon_call(G, steps, active, stream, ws)
        p = MuonParams(0.0, 0.0, 0.0, 0, steps, coefs[0], coefs[1], coefs[2], eps, _dptr(active))
        _check(self._lib.gnnco_orthogonalise(self._handle, gd, od, sets, r, c, G.data_ptr(), out.data_ptr(),
                                             ctypes.byref(p), ws.data_ptr(), ws.numel(), _stream_ptr(stream)),
               "gnnco_orthogonalise")
        return out

    def objective_static(self, p, alpha: float, beta: float, lam: float = 0.0, pen=None, loss=None, stream=None):
        """``gnnco_objective_static``: per-subgraph objective of given probabilities, with no
        work area and no allocation inside the library (``loss`` must be passed by callers
        that cannot allocate; it is created here only as a convenience)."""
        import torch
        _require(p, torch.float32, "p")
        if loss is None:
            loss = torch.empty(self.S, dtype=torch.float32, device=self.device)
        obj = Objective(alpha, beta, lam, _dptr(pen))
        _check(self._lib.gnnco_objective_static(self._handle, p.data_ptr(), ctypes.byref(obj), loss.data_ptr(),
                                                _stream_ptr(stream)), "gnnco_objective_static")
        return loss

    def async_status(self, stream=None) -> int:
        s = _i32(0)
        _check(self._lib.gnnco_async_status(self._handle, _stream_ptr(stream), ctypes.byref(s)), "gnnco_async_status")
        return int(s.value)

    def profile_begin(self) -> None:
        _check(self._lib.gnnco_profile_begin(self._handle), "gnnco_profile_begin")

    def profile_end(self, stream=None) -> dict:
        """``gnnco_profile_end``: {kernel family: (calls, total_ms)} since profile_begin."""
        entries = (ProfileEntry * 32)()
        count = _i32(0)
        _check(self._lib.gnnco_profile_end(self._handle, _stream_ptr(stream), entries, 32, ctypes.byref(count)),
               "gnnco_profile_end")
        return {entries[k].name.decode(): (int(entries[k].calls), float(entries[k].total_ms))
                for k in range(count.value)}

    def launch_count(self) -> int:
        return int(self._lib.gnnco_launch_count(self._handle))

    def close(self) -> None:
        if self._handle is not None:
            self._lib.gnnco_destroy(self._handle)
            self._handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def gnnco_partition_load(edge_u, edge_v, part, S: int, stream=None) -> PartitionedGraph:
    return PartitionedGraph(edge_u, edge_v, part, S, stream)


def gnnco_train_step(graph: PartitionedGraph, *args, **kwargs):
    return graph.train_step(*args, **kwargs)


def gnnco_decode_boundary(graph: PartitionedGraph, *args, **kwargs):
    return graph.decode_boundary(*args, **kwargs)


def gnnco_louvain(edge_u, edge_v, n: int, max_levels: int = 32, max_sweeps: int = 64, stream=None):
    """``gnnco_louvain``: deterministic Louvain partition of the graph (int32 device tensors ``edge_u``,
    ``edge_v``).  Returns dict(part [n] int32 device tensor, S, qnum, two_m, Q, levels, sweeps)."""
    import torch
    lib = load_library()
    _require(edge_u, torch.int32, "edge_u")
    _require(edge_v, torch.int32, "edge_v")
    E = int(edge_u.numel())
    need = _sz(0)
    _check(lib.gnnco_louvain_workspace_bytes(n, E, ctypes.byref(need)), "gnnco_louvain_workspace_bytes")
    ws = torch.empty(max(256, need.value), dtype=torch.uint8, device=edge_u.device)
    part = torch.empty(n, dtype=torch.int32, device=edge_u.device)
    S, levels, sweeps = _i32(0), _i32(0), _i32(0)
    qnum, two_m = _i64(0), _i64(0)
    _check(lib.gnnco_louvain(n, E, edge_u.data_ptr() if E else None, edge_v.data_ptr() if E else None, max_levels,
                             max_sweeps, part.data_ptr(), ctypes.byref(S), ctypes.byref(qnum), ctypes.byref(two_m),
                             ctypes.byref(levels), ctypes.byref(sweeps), ws.data_ptr(), ws.numel(), _stream_ptr(stream)),
           "gnnco_louvain")
    q = qnum.value / float(two_m.value) ** 2 if two_m.value else 0.0
    return dict(part=part, S=int(S.value), qnum=int(qnum.value), two_m=int(two_m.value), Q=q, levels=int(levels.value),
                sweeps=int(sweeps.value))
