"""Thin ctypes binding of libjanus (argument marshalling only).

Every computation runs in the HIP library; PyTorch is used here only to
allocate device memory and to pick the stream.  Importing this module loads
the in-tree ``_lib/libjanus.so`` and raises if it has not been built: there
is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import NamedTuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libjanus.so")

JANUS_OK, JANUS_EINVAL, JANUS_ECAPACITY, JANUS_ENOMEM, JANUS_EHIP, JANUS_EUNSUPPORTED = 0, -1, -2, -3, -4, -5


class JanusError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {_lib().janus_strerror(code).decode()} (code {code})")


class Config(C.Structure):
    _fields_ = [
        ("n_species", C.c_int32), ("d", C.c_int32), ("n_rbf", C.c_int32), ("n_blocks", C.c_int32),
        ("n_experts", C.c_int32), ("top_k", C.c_int32), ("d_hidden", C.c_int32), ("env_p", C.c_int32),
        ("r_cut", C.c_float), ("three_body", C.c_int32), ("r_cut3", C.c_float), ("n_experts3", C.c_int32),
        ("top_k3", C.c_int32), ("d_hidden3", C.c_int32), ("n_legendre", C.c_int32), ("w_E", C.c_float),
        ("w_F", C.c_float), ("atom_moe", C.c_int32), ("n_experts_f", C.c_int32), ("top_k_f", C.c_int32),
        ("d_hidden_f", C.c_int32), ("w_S", C.c_float), ("n_heads", C.c_int32), ("n_tasks", C.c_int32),
        ("n_charges", C.c_int32), ("n_spins", C.c_int32), ("robust", C.c_int32), ("huber_delta", C.c_float),
        ("robust_tau", C.c_float), ("route_feat", C.c_int32),
    ]


class TensorDesc(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("offset", C.c_int64), ("ndim", C.c_int32), ("shape", C.c_int64 * 3)]


class Edges(C.Structure):
    _fields_ = [("n_edges", C.c_int64), ("ei", C.c_void_p), ("ej", C.c_void_p), ("shift", C.c_void_p),
                ("rowptr", C.c_void_p), ("rev", C.c_void_p)]


class Labels(C.Structure):
    _fields_ = [("task", C.c_void_p), ("charge", C.c_void_p), ("spin", C.c_void_p)]


class Norm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("d", C.c_int32), ("type", C.c_int32), ("eps", C.c_float), ("n_seq", C.c_int32),
                ("w_post", C.c_void_p), ("scale", C.c_void_p), ("w_pre", C.c_void_p), ("gate", C.c_void_p),
                ("ldg", C.c_int64), ("gate_off", C.c_void_p)]


class Experts(C.Structure):
    _fields_ = [("d", C.c_int32), ("d_hidden", C.c_int32), ("n_experts", C.c_int32), ("top_k", C.c_int32),
                ("type", C.c_int32), ("normalize", C.c_int32), ("router", C.c_void_p), ("beta", C.c_void_p),
                ("w_up", C.c_void_p), ("w_down", C.c_void_p)]


class ProfileEntry(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("launches", C.c_int64), ("ms", C.c_double), ("flops", C.c_double),
                ("bytes", C.c_double)]


class Debug(C.Structure):
    _fields_ = [("eid", C.c_void_p), ("gate", C.c_void_p), ("counts", C.c_void_p), ("pos", C.c_void_p),
                ("basis", C.c_void_p), ("tri_e", C.c_void_p), ("tri_e2", C.c_void_p), ("eid3", C.c_void_p),
                ("gate3", C.c_void_p), ("eidf", C.c_void_p), ("gatef", C.c_void_p), ("gap", C.c_void_p)]

    KEYS = ("eid", "gate", "counts", "pos", "basis", "tri_e", "tri_e2", "eid3", "gate3", "eidf", "gatef", "gap")


_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"libjanus is not built ({LIB_PATH}); run paper_2604_15821_amd.build")
        # PyTorch's HIP runtime must be in the process before the library is: loaded
        # first, the library would bring in a second runtime (its link-time one), and
        # device memory of one runtime is not valid in the other
        import torch  # noqa: F401
        lib = C.CDLL(LIB_PATH)
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        lib.janus_strerror.restype = C.c_char_p
        lib.janus_strerror.argtypes = [C.c_int]
        lib.janus_create.argtypes = [C.POINTER(Config), C.POINTER(vp)]
        lib.janus_destroy.argtypes = [vp]
        lib.janus_destroy.restype = None
        lib.janus_weight_layout.argtypes = [C.POINTER(Config), C.POINTER(TensorDesc), C.POINTER(i32), C.POINTER(i64)]
        lib.janus_build_edges.argtypes = [vp, vp, vp, vp, i32, i32, i64, vp, vp, vp, vp, vp, C.POINTER(i64), vp]
        lib.janus_step.argtypes = [vp, vp, vp, vp, vp, i32, i32, C.POINTER(Edges), vp, vp, vp, vp, vp, vp, vp,
                                   C.POINTER(Debug), vp]
        lib.janus_step_stress.argtypes = [vp, vp, vp, vp, vp, i32, i32, C.POINTER(Edges), vp, vp, vp, vp, vp, vp,
                                          vp, vp, vp, C.POINTER(Debug), vp]
        lib.janus_step_ex.argtypes = [vp, vp, vp, vp, vp, i32, i32, C.POINTER(Edges), vp, vp, vp, vp,
                                      C.POINTER(Labels), vp, vp, vp, vp, vp, C.POINTER(Debug), vp]
        lib.janus_step_pos.argtypes = [vp, vp, vp, vp, vp, i32, i32, C.POINTER(Edges), vp, vp, vp, vp,
                                       C.POINTER(Labels), vp, vp, vp, vp, vp, vp, C.POINTER(Debug), vp]
        lib.janus_grouped_gemm.argtypes = [vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, vp]
        lib.janus_grouped_wgrad.argtypes = [vp, vp, vp, vp, vp, i32, i64, i32, i32, vp]
        lib.janus_grouped_gemm_noalloc.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, vp]
        lib.janus_wgrad_chunk_rows.argtypes = [i64, i32, i32]
        lib.janus_wgrad_chunk_rows.restype = i32
        lib.janus_residual_norm.argtypes = [C.POINTER(Norm), vp, i64, vp, i64, vp, i64, vp, i64, vp]
        lib.janus_residual_norm_grad_workspace.argtypes = [C.POINTER(Norm)]
        lib.janus_residual_norm_grad_workspace.restype = i64
        lib.janus_residual_norm_grad.argtypes = [C.POINTER(Norm), vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64,
                                                 vp, vp, vp, vp, i64, vp, i64, vp]
        lib.janus_expert_layer_workspace.argtypes = [C.POINTER(Experts), i32]
        lib.janus_expert_layer_workspace.restype = i64
        lib.janus_expert_layer.argtypes = [C.POINTER(Experts), vp, i64, i32, vp, i64, vp, vp, vp, i64, vp]
        lib.janus_pack_rows.argtypes = [vp, i64, i32, i64, i32, vp, i64, vp, i64, vp]
        lib.janus_unpack_rows.argtypes = [vp, i64, vp, i64, i64, i32, i32, i32, vp, i64, vp, i64, vp, i64, vp]
        lib.janus_packed_wgrad_workspace.argtypes = [i64, i32, i32, i32, i32]
        lib.janus_packed_wgrad_workspace.restype = i64
        lib.janus_packed_wgrad.argtypes = [vp, i64, vp, i64, vp, i64, i32, vp, vp, i32, i64, i32, i32, vp, i64, vp]
        lib.janus_set_workspace_limit.argtypes = [vp, i64]
        lib.janus_set_concurrency.argtypes = [vp, C.c_int]
        lib.janus_set_edge_builder.argtypes = [vp, C.c_int32]
        lib.janus_last_chunks.argtypes = [vp]
        lib.janus_last_triplets.argtypes = [vp]
        lib.janus_last_triplets.restype = i64
        lib.janus_profile_enable.argtypes = [vp, C.c_int]
        lib.janus_profile_read.argtypes = [vp, C.POINTER(ProfileEntry), i32]
        _LIB = lib
    return _LIB


def exported_symbols():
    """Names the library exports (checked against include/janus.h by the CPU tests)."""
    lib = _lib()
    names = ["janus_create", "janus_destroy", "janus_weight_layout", "janus_build_edges", "janus_step",
             "janus_step_stress", "janus_step_ex", "janus_step_pos",
             "janus_grouped_gemm", "janus_grouped_gemm_noalloc", "janus_grouped_wgrad", "janus_wgrad_chunk_rows",
             "janus_residual_norm", "janus_residual_norm_grad", "janus_residual_norm_grad_workspace",
             "janus_expert_layer", "janus_expert_layer_workspace", "janus_pack_rows", "janus_unpack_rows",
             "janus_packed_wgrad", "janus_packed_wgrad_workspace",
             "janus_profile_enable",
             "janus_profile_read",
             "janus_set_workspace_limit", "janus_set_concurrency", "janus_set_edge_builder", "janus_last_chunks",
             "janus_last_triplets", "janus_strerror"]
    return [n for n in names if hasattr(lib, n)]


def wgrad_chunk_rows(M: int, P: int, Q: int) -> int:
    """Row-chunk length of the weight-gradient contraction over M rows into P x Q blocks."""
    r = int(_lib().janus_wgrad_chunk_rows(int(M), int(P), int(Q)))
    if r < 0:
        raise JanusError(r, "janus_wgrad_chunk_rows")
    return r


def make_config(model) -> Config:
    """Config from a ModelConfig-like object (attribute names as in the C struct)."""
    c = Config()
    for name, _ in Config._fields_:
        v = getattr(model, name)
        setattr(c, name, int(v) if not isinstance(v, float) else v)
    return c


def weight_layout(model):
    """[(name, offset, shape)] and the blob size, from the library."""
    lib = _lib()
    cfg = make_config(model)
    n = C.c_int32(0)
    tot = C.c_int64(0)
    rc = lib.janus_weight_layout(C.byref(cfg), None, C.byref(n), C.byref(tot))
    if rc:
        raise JanusError(rc, "janus_weight_layout")
    descs = (TensorDesc * n.value)()
    rc = lib.janus_weight_layout(C.byref(cfg), descs, C.byref(n), C.byref(tot))
    if rc:
        raise JanusError(rc, "janus_weight_layout")
    out = [(d.name.decode(), int(d.offset), tuple(int(d.shape[k]) for k in range(d.ndim))) for d in descs]
    return out, int(tot.value)


def pack_weights(weights: dict, model) -> np.ndarray:
    layout, total = weight_layout(model)
    blob = np.zeros(total, np.float32)
    for name, off, shape in layout:
        w = np.asarray(weights[name], np.float32)
        if w.shape != shape:
            raise ValueError(f"{name}: shape {w.shape} != {shape}")
        blob[off:off + w.size] = w.reshape(-1)
    return blob


def unpack(blob: np.ndarray, model) -> dict:
    layout, _ = weight_layout(model)
    return {name: blob[off:off + int(np.prod(shape))].reshape(shape) for name, off, shape in layout}


def _ptr(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


_DTYPES = {"f32": "float32", "i32": "int32", "i8": "int8"}


def _arg(t, name, kind, shape=None, device=None, optional=False):
    """Check one tensor argument before its address goes to the library: the
    library reads raw memory, so a wrong dtype, a strided view, a host tensor or
    a wrong size would be misread rather than rejected.  `shape` may use None
    for a free dimension; returns the tensor."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name}: required")
    import torch
    want = getattr(torch, _DTYPES[kind])
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.dtype != want:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {want}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a device tensor (got {t.device})")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")
    if shape is not None:
        if t.dim() != len(shape) or any(w is not None and int(n) != int(w) for n, w in zip(t.shape, shape)):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


@dataclass
class NeighborList:
    n_edges: int
    ei: object
    ej: object
    shift: object
    rowptr: object
    rev: object

    def as_struct(self) -> Edges:
        return Edges(self.n_edges, _ptr(self.ei).value, _ptr(self.ej).value, _ptr(self.shift).value,
                     _ptr(self.rowptr).value, _ptr(self.rev).value)


class Context:
    """A libjanus context on the current device."""

    def __init__(self, model):
        import torch
        # PyTorch carries its own HIP runtime next to the library's; when the library's
        # initialises first, PyTorch's then finds no device, so PyTorch goes first
        if torch.cuda.is_available():
            torch.cuda.current_device()
        self.model = model
        self.cfg = make_config(model)
        h = C.c_void_p()
        rc = _lib().janus_create(C.byref(self.cfg), C.byref(h))
        if rc:
            raise JanusError(rc, "janus_create")
        self.h = h
        self.n_weights = weight_layout(model)[1]
        self.capacity = 0
        self._nl_bufs = None

    def close(self):
        if self.h:
            import torch
            torch.cuda.synchronize()
            _lib().janus_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---------------------------------------------------------------- edges
    def build_edges(self, pos, cell, offsets, capacity=None) -> NeighborList:
        """Neighbour list of device tensors pos [N,3] f32, cell [S,3,3] f32, offsets [S+1] i32."""
        import torch
        dev = pos.device
        N = pos.shape[0]
        S = cell.shape[0]
        self._check_geometry(pos, cell, offsets)
        rowptr = torch.empty(N + 1, dtype=torch.int32, device=dev)
        ne = C.c_int64(0)
        cap = int(capacity if capacity is not None else max(self.capacity, 1))
        for _ in range(2):
            ei = torch.empty(cap, dtype=torch.int32, device=dev)
            ej = torch.empty(cap, dtype=torch.int32, device=dev)
            rev = torch.empty(cap, dtype=torch.int32, device=dev)
            sh = torch.empty(cap * 3, dtype=torch.int8, device=dev)
            rc = _lib().janus_build_edges(self.h, _ptr(pos), _ptr(cell), _ptr(offsets), N, S, cap, _ptr(ei), _ptr(ej),
                                          _ptr(sh), _ptr(rowptr), _ptr(rev), C.byref(ne), _stream())
            if rc == JANUS_ECAPACITY and capacity is None:
                cap = int(ne.value)
                self.capacity = cap
                continue
            if rc:
                raise JanusError(rc, "janus_build_edges")
            n = int(ne.value)
            return NeighborList(n, ei[:n], ej[:n], sh[:3 * n].view(n, 3) if n else sh[:0].view(0, 3), rowptr,
                                rev[:n])
        raise RuntimeError("edge capacity did not converge")

    def build_edges_into(self, pos, cell, offsets, nl: NeighborList):
        """Rebuild into existing buffers (capacity = their size); returns the edge count."""
        ne = C.c_int64(0)
        cap = int(nl.ei.shape[0])
        self._check_geometry(pos, cell, offsets)
        self._check_edges(nl, pos.shape[0], pos.device, room=True)
        rc = _lib().janus_build_edges(self.h, _ptr(pos), _ptr(cell), _ptr(offsets), pos.shape[0], cell.shape[0],
                                      cap, _ptr(nl.ei), _ptr(nl.ej), _ptr(nl.shift), _ptr(nl.rowptr), _ptr(nl.rev),
                                      C.byref(ne), _stream())
        if rc:
            raise JanusError(rc, "janus_build_edges")
        return int(ne.value)

    # ------------------------------------------------------- argument checks
    @staticmethod
    def _check_geometry(pos, cell, offsets):
        dev = pos.device
        _arg(pos, "pos", "f32", (None, 3))
        _arg(cell, "cell", "f32", (None, 3, 3), dev)
        _arg(offsets, "offsets", "i32", (cell.shape[0] + 1,), dev)

    @staticmethod
    def _check_edges(nl, N, dev, room=False):
        """Edge arrays of a neighbour list: [Ne] each ([capacity] with room=True: the
        buffers a rebuild writes into), shift [Ne, 3], rowptr [N+1]."""
        n = int(nl.ei.shape[0]) if room else nl.n_edges
        _arg(nl.rowptr, "nl.rowptr", "i32", (N + 1,), dev)
        for name, t in (("nl.ei", nl.ei), ("nl.ej", nl.ej), ("nl.rev", nl.rev)):
            _arg(t, name, "i32", (n,), dev)
        sh = nl.shift.reshape(-1) if nl.shift is not None and nl.shift.is_contiguous() else nl.shift
        _arg(sh, "nl.shift", "i8", (3 * n,), dev)

    def _check_step(self, pos, cell, species, offsets, nl, W, E_ref, F_ref, out, S_ref, stress, labels):
        m = self.model
        dev = pos.device
        self._check_geometry(pos, cell, offsets)
        N, S = pos.shape[0], cell.shape[0]
        _arg(species, "species", "i32", (N,), dev)
        self._check_edges(nl, N, dev)
        total = self.n_weights
        _arg(W, "W", "f32", (total,), dev)
        _arg(E_ref, "E_ref", "f32", (S,), dev)
        _arg(F_ref, "F_ref", "f32", (N, 3), dev)
        # a missing S_ref (with w_S > 0) or missing labels (with n_tasks > 0) is the library's
        # JANUS_EINVAL; only the layout of what is passed is checked here
        _arg(S_ref, "S_ref", "f32", (S, 3, 3), dev, optional=True)
        _arg(stress, "stress", "f32", (S, 3, 3), dev, optional=True)
        if out is not None:
            loss, E, F, dW = out
            _arg(loss, "loss", "f32", (1,), dev)
            _arg(E, "E", "f32", (S,), dev)
            _arg(F, "F", "f32", (N, 3), dev)
            _arg(dW, "dLdW", "f32", (total,), dev)
        if labels is not None:
            for name, t in zip(("task", "charge", "spin"), labels):
                _arg(t, f"labels.{name}", "i32", (S,), dev)

    # ----------------------------------------------------------------- step
    def step(self, pos, cell, species, offsets, nl: NeighborList, W, E_ref, F_ref, out=None, debug=None,
             S_ref=None, stress=None, labels=None, dLdR=None):
        """One training step; returns (loss [1], E [S], F [N,3], dLdW [like W]) device tensors.

        With S_ref [S,3,3] (needed when the model's w_S > 0) or a stress output
        tensor [S,3,3], writes the stress into `stress`; labels = (task, charge,
        spin) int32 device tensors [S] (needed when the model has n_tasks > 0);
        with a dLdR tensor [N,3], also writes the loss gradient in the positions."""
        import torch
        dev = pos.device
        N = pos.shape[0]
        S = cell.shape[0]
        self._check_step(pos, cell, species, offsets, nl, W, E_ref, F_ref, out, S_ref, stress, labels)
        if out is None:
            out = (torch.empty(1, dtype=torch.float32, device=dev), torch.empty(S, dtype=torch.float32, device=dev),
                   torch.empty(N, 3, dtype=torch.float32, device=dev), torch.empty_like(W))
        loss, E, F, dW = out
        edges = nl.as_struct()
        dbg = None
        if debug is not None:
            dbg = Debug(*[_ptr(debug.get(k)).value for k in Debug.KEYS])
        dbgp = C.byref(dbg) if dbg is not None else None
        _arg(dLdR, "dLdR", "f32", (N, 3), dev, optional=True)
        if dLdR is not None:
            lab = Labels(*[_ptr(x).value for x in labels]) if labels is not None else None
            rc = _lib().janus_step_pos(self.h, _ptr(pos), _ptr(cell), _ptr(species), _ptr(offsets), N, S,
                                       C.byref(edges), _ptr(W), _ptr(E_ref), _ptr(F_ref), _ptr(S_ref),
                                       C.byref(lab) if lab is not None else None, _ptr(loss), _ptr(E), _ptr(F),
                                       _ptr(stress), _ptr(dW), _ptr(dLdR), dbgp, _stream())
        elif S_ref is None and stress is None and labels is None:
            rc = _lib().janus_step(self.h, _ptr(pos), _ptr(cell), _ptr(species), _ptr(offsets), N, S, C.byref(edges),
                                   _ptr(W), _ptr(E_ref), _ptr(F_ref), _ptr(loss), _ptr(E), _ptr(F), _ptr(dW), dbgp,
                                   _stream())
        elif labels is None:
            rc = _lib().janus_step_stress(self.h, _ptr(pos), _ptr(cell), _ptr(species), _ptr(offsets), N, S,
                                          C.byref(edges), _ptr(W), _ptr(E_ref), _ptr(F_ref), _ptr(S_ref), _ptr(loss),
                                          _ptr(E), _ptr(F), _ptr(stress), _ptr(dW), dbgp, _stream())
        else:
            lab = Labels(*[_ptr(x).value for x in labels])
            rc = _lib().janus_step_ex(self.h, _ptr(pos), _ptr(cell), _ptr(species), _ptr(offsets), N, S,
                                      C.byref(edges), _ptr(W), _ptr(E_ref), _ptr(F_ref), _ptr(S_ref), C.byref(lab),
                                      _ptr(loss), _ptr(E), _ptr(F), _ptr(stress), _ptr(dW), dbgp, _stream())
        if rc:
            raise JanusError(rc, "janus_step")
        return loss, E, F, dW

    # ------------------------------------------------------------ workspace
    def set_workspace_limit(self, nbytes: int):
        rc = _lib().janus_set_workspace_limit(self.h, int(nbytes))
        if rc:
            raise JanusError(rc, "janus_set_workspace_limit")

    def set_concurrency(self, on: bool):
        """Expert weight gradients on the context's second stream (True) or on the caller's (False, the default)."""
        rc = _lib().janus_set_concurrency(self.h, int(bool(on)))
        if rc:
            raise JanusError(rc, "janus_set_concurrency")

    def set_edge_builder(self, mode: int):
        """Candidate search of build_edges: 0 automatic, 1 cell list everywhere, 2 all pairs everywhere."""
        rc = _lib().janus_set_edge_builder(self.h, int(mode))
        if rc:
            raise JanusError(rc, "janus_set_edge_builder")

    def last_chunks(self) -> int:
        return int(_lib().janus_last_chunks(self.h))

    def last_triplets(self) -> int:
        return int(_lib().janus_last_triplets(self.h))

    # ------------------------------------------------------------- profiler
    PROFILE_FAMILIES = ["expert_gemm", "expert_wgrad", "dense_gemm", "edge", "atom", "route", "graph", "other",
                        "attention"]

    def profile(self, on: bool, families=None):
        """Start (on) or stop the event profiler; `families` restricts it to some kernel families."""
        mask = 0
        if on:
            mask = -1 if families is None else sum(1 << self.PROFILE_FAMILIES.index(f) for f in families)
        rc = _lib().janus_profile_enable(self.h, mask)
        if rc:
            raise JanusError(rc, "janus_profile_enable")

    def profile_read(self) -> dict:
        """{family: {launches, ms, flops, bytes}} since profile(True) or the last read."""
        buf = (ProfileEntry * 16)()
        n = _lib().janus_profile_read(self.h, buf, 16)
        if n < 0:
            raise JanusError(n, "janus_profile_read")
        return {buf[q].name.decode(): {"launches": int(buf[q].launches), "ms": float(buf[q].ms),
                                        "flops": float(buf[q].flops), "bytes": float(buf[q].bytes)}
                for q in range(n)}

    # ---------------------------------------------------------------- GEMMs
    def grouped_gemm(self, A, B, row_off, K, N, trans_b, out=None):
        import torch
        M = A.shape[0]
        dev = A.device
        G = row_off.shape[0] - 1
        _arg(A, "A", "f32", (M, K))
        _arg(B, "B", "f32", (G, N, K) if trans_b else (G, K, N), dev)
        _arg(row_off, "row_off", "i32", (G + 1,), dev)
        if out is None:
            out = torch.empty(M, N, dtype=torch.float32, device=A.device)
        _arg(out, "out", "f32", (M, N), dev)
        rc = _lib().janus_grouped_gemm(self.h, _ptr(A), _ptr(B), _ptr(out), _ptr(row_off), row_off.shape[0] - 1, M,
                                       K, N, int(trans_b), _stream())
        if rc:
            raise JanusError(rc, "janus_grouped_gemm")
        return out

    def grouped_wgrad(self, A, B, row_off, out=None):
        import torch
        M, P = A.shape
        Q = B.shape[1]
        G = row_off.shape[0] - 1
        dev = A.device
        _arg(A, "A", "f32", (M, P))
        _arg(B, "B", "f32", (M, Q), dev)
        _arg(row_off, "row_off", "i32", (G + 1,), dev)
        if out is None:
            out = torch.empty(G, P, Q, dtype=torch.float32, device=A.device)
        _arg(out, "out", "f32", (G, P, Q), dev)
        rc = _lib().janus_grouped_wgrad(self.h, _ptr(A), _ptr(B), _ptr(out), _ptr(row_off), G, M, P, Q, _stream())
        if rc:
            raise JanusError(rc, "janus_grouped_wgrad")
        return out


def grouped_gemm_noalloc(A, B, row_off, K, N, trans_b, out):
    """janus_grouped_gemm_noalloc on the current device: C = A x B_g per row group into
    the caller's `out`, with the tile table in the library's fixed scratch (no allocation)."""
    M = A.shape[0]
    dev = A.device
    G = row_off.shape[0] - 1
    _arg(A, "A", "f32", (M, K))
    _arg(B, "B", "f32", (G, N, K) if trans_b else (G, K, N), dev)
    _arg(row_off, "row_off", "i32", (G + 1,), dev)
    _arg(out, "out", "f32", (M, N), dev)
    rc = _lib().janus_grouped_gemm_noalloc(_ptr(A), _ptr(B), _ptr(out), _ptr(row_off), G, M, K, N, int(trans_b),
                                           _stream())
    if rc:
        raise JanusError(rc, "janus_grouped_gemm_noalloc")
    return out


# ------------------------------------------------------- operators around an expert block
#
# Calls on tensors' data, like the rest of this module: outputs carry no autograd history, gradients have calls of their own.

ACT = {"none": 0, "silu": 1}


_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

_MOST = 2 ** 31 - 1   # of what the library counts in 32 bits: ctypes would cut off more without a word


def _type_of(t, name):
    """janus_type of a tensor or of a torch dtype."""
    dt = t.dtype if isinstance(t, torch.Tensor) else t
    code = _TYPES.get(dt)
    if code is None:
        raise TypeError(f"{name}: {dt}, expected float32, bfloat16 or float16")
    return code


def _rows(t, name, dtype, shape, device):
    """Check a [rows, width] tensor whose rows may lie apart; returns (address, row distance)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if device.index is None or t.get_device() != device.index:
        raise ValueError(f"{name}: on {t.device}, expected a device tensor on {device}")
    n, w = shape
    if n == 0 or w == 0:
        return 0, w
    ld, step = t.stride()
    if step != 1 and w > 1:
        raise ValueError(f"{name}: the values of a row must lie next to each other")
    if n == 1:
        ld = w
    if ld < w:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr(), ld


def _param(t, name, d, device):
    """Address of an optional fp32 parameter vector of d values (None: NULL)."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.dtype == torch.float32 and t.shape == (d,) and t.stride() == (1,) and \
            t.get_device() == device.index:
        return t.data_ptr()
    return _arg(t, name, "f32", (d,), device).data_ptr()   # says what is wrong, or takes a vector of one value


def _matrix(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.dim() != 2:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected two dimensions")
    if t.shape[1] > _MOST:
        raise ValueError(f"{name}: {t.shape[1]} columns, at most {_MOST}")
    return t.shape[0], t.shape[1], t.device


def _offsets(t, name, device):
    """Check the offsets of groups or sequences; returns how many of these there are."""
    if isinstance(t, torch.Tensor) and t.numel() > _MOST:
        raise ValueError(f"{name}: {t.numel()} offsets, at most {_MOST}")
    return _arg(t, name, "i32", (None,), device).shape[0] - 1


def _call(rc, where):
    if rc < 0:
        raise JanusError(rc, where)
    return rc


def _launch(device, where, call, *args):
    """The library call on the current stream of the tensors' device, which is made the current one where it is not."""
    # the stream's handle itself: current_stream() builds an object around it, 3 us of a call of 12
    stream = torch._C._cuda_getCurrentRawStream(device.index)
    if torch.cuda.current_device() == device.index:
        rc = call(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = call(*args, stream)
    if rc < 0:
        raise JanusError(rc, where)


def _norm(rows, d, like, device, w_post, gate, gate_off, scale, w_pre, eps):
    p = Norm(rows, d, _type_of(like, "b"), float(eps), 0, _param(w_post, "w_post", d, device),
             _param(scale, "scale", d, device), _param(w_pre, "w_pre", d, device), None, d, None)
    if gate_off is not None:
        if gate is None:
            raise ValueError("gate_off: without a gate")
        p.n_seq = _offsets(gate_off, "gate_off", device)
        if p.n_seq < 0:
            raise ValueError("gate_off: needs at least one offset")
        p.gate_off = gate_off.data_ptr()
    if gate is not None:
        p.gate, p.ldg = _rows(gate, "gate", like.dtype, (rows if gate_off is None else p.n_seq, d), device)
        # a gate without rows has no address and is never read, but has to be told from none
        p.gate = p.gate or (gate_off if gate_off is not None else w_post if w_post is not None else like).data_ptr() or 16
    return p


def residual_norm(x, b, w_post=None, gate=None, gate_off=None, scale=None, w_pre=None, eps=1e-6, out=None):
    """The norms after and before a block, with its gate and residual scale:

        u = w_post * b / rms(b),   r = x + scale * gate * u,   n = w_pre * r / rms(r)

    x, b [rows, d] float32, bfloat16 or float16 device tensors (rows may lie apart); w_post, scale
    and w_pre [d] float32 or None; gate None, [rows, d], or one row per sequence [n_seq, d] with gate_off
    [n_seq + 1] int32 (rows behind the last sequence are left alone: zero in new outputs, as they
    were in `out`).  Returns (r, n), n None without w_pre; out = (r, n) to write into, where r may be x and
    n may be b."""
    rows, d, dev = _matrix(b, "b")
    pb, ldb = _rows(b, "b", b.dtype, (rows, d), dev)
    px, ldx = _rows(x, "x", b.dtype, (rows, d), dev)
    p = _norm(rows, d, b, dev, w_post, gate, gate_off, scale, w_pre, eps)
    if out is None:
        new = torch.empty if gate_off is None else torch.zeros
        r = new(rows, d, dtype=b.dtype, device=dev)
        n = None if w_pre is None else new(rows, d, dtype=b.dtype, device=dev)
    else:
        r, n = out
        if (n is None) != (w_pre is None):
            raise ValueError("out: n is given exactly where w_pre is")
    pr, ldr = _rows(r, "r", b.dtype, (rows, d), dev)
    pn, ldn = (None, 0) if n is None else _rows(n, "n", b.dtype, (rows, d), dev)
    _launch(dev, "janus_residual_norm", _lib().janus_residual_norm, C.byref(p), px, ldx, pb, ldb, pr, ldr, pn, ldn)
    return r, n


class NormGrads(NamedTuple):
    """Gradients of residual_norm; None where the forward pass had no such input."""
    dx: object
    db: object
    dw_post: object
    dgate: object
    dscale: object
    dw_pre: object


def residual_norm_grad(dr, dn, r, b, w_post=None, gate=None, gate_off=None, scale=None, w_pre=None, eps=1e-6, out=None):
    """Gradients of residual_norm in all its inputs, at the stored r and b, from the gradients dr and
    dn of its outputs (dr None: zero; dn and r None without w_pre).  out = (dx, db) to write into, where
    dx may be dr and db may be dn.  Rows behind the last sequence add to no gradient."""
    rows, d, dev = _matrix(b, "b")
    dt = b.dtype
    like = lambda t, name: (None, 0) if t is None else _rows(t, name, dt, (rows, d), dev)  # noqa: E731
    pb, ldb = _rows(b, "b", dt, (rows, d), dev)
    p = _norm(rows, d, b, dev, w_post, gate, gate_off, scale, w_pre, eps)
    if w_pre is not None and (dn is None or r is None):
        raise ValueError("dn, r: required with w_pre")
    if w_pre is None and dn is not None:
        raise ValueError("dn: without w_pre")
    pdr, lddr = like(dr, "dr")
    pdn, lddn = like(dn, "dn")
    pr, ldr = like(r, "r")
    if out is None:
        new = torch.empty if gate_off is None else torch.zeros
        dx, db = new(rows, d, dtype=dt, device=dev), new(rows, d, dtype=dt, device=dev)
    else:
        dx, db = out
    pdx, lddx = _rows(dx, "dx", dt, (rows, d), dev)
    pdb, lddb = _rows(db, "db", dt, (rows, d), dev)
    dw = iter(torch.empty(3, d, dtype=torch.float32, device=dev))
    dw_post, dscale, dw_pre = (None if w is None else next(dw) for w in (w_post, scale, w_pre))
    dgate = None if gate is None else torch.empty(gate.shape, dtype=dt, device=dev)
    adr = lambda t: None if t is None or t.numel() == 0 else t.data_ptr()  # noqa: E731
    lib = _lib()
    size = _call(lib.janus_residual_norm_grad_workspace(C.byref(p)), "janus_residual_norm_grad_workspace")
    work = torch.empty(size, dtype=torch.uint8, device=dev)
    _launch(dev, "janus_residual_norm_grad", lib.janus_residual_norm_grad, C.byref(p), pdr, lddr, pdn, lddn, pr, ldr, pb,
            ldb, pdx, lddx, pdb, lddb, adr(dw_post), adr(dscale), adr(dw_pre), adr(dgate), d, work.data_ptr(), size)
    return NormGrads(dx, db, dw_post, dgate, dscale, dw_pre)


def _weights(t, name, dtype, shape, device):
    """Address of a contiguous weight tensor."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    if device.index is None or t.get_device() != device.index or not t.is_contiguous():
        raise ValueError(f"{name}: must be a contiguous tensor on {device}")
    return t.data_ptr()


def expert_layer(x, router, w_up, w_down, top_k, beta=None, normalize=False, out=None):
    """A whole expert layer for up to 64 tokens x [tokens, d]: logits x router + beta, the top_k largest,
    gates their softmax probabilities (normalize: divided by their sum), and
    y = sum_c gate_c SiLU(x w_up[e_c]) w_down[e_c].

    router [d, n] float32, beta [n] float32 or None, w_up [n, d, h] and w_down [n, h, d] of x's type; d and h
    multiples of 16.  Returns (y [tokens, d], expert ids [tokens, top_k] int32, gates float32)."""
    tokens, d, dev = _matrix(x, "x")
    if not isinstance(w_up, torch.Tensor) or w_up.dim() != 3:
        raise ValueError("w_up: expected a tensor [experts, d, hidden]")
    n, _, h = w_up.shape
    if n > _MOST or h > _MOST:
        raise ValueError(f"w_up: {n} experts of {h} hidden values, at most {_MOST} of both")
    top_k = int(top_k)
    if not -_MOST <= top_k <= _MOST:
        raise ValueError(f"top_k: {top_k}, at most {_MOST}")
    code = _type_of(x, "x")
    px, ldx = _rows(x, "x", x.dtype, (tokens, d), dev)
    pr = _weights(router, "router", torch.float32, (d, n), dev)
    pu = _weights(w_up, "w_up", x.dtype, (n, d, h), dev)
    pw = _weights(w_down, "w_down", x.dtype, (n, h, d), dev)
    p = Experts(d, h, n, top_k, code, int(bool(normalize)), pr, _param(beta, "beta", n, dev), pu, pw)
    lib = _lib()
    size = _call(lib.janus_expert_layer_workspace(C.byref(p), tokens), "janus_expert_layer_workspace")
    y = torch.empty(tokens, d, dtype=x.dtype, device=dev) if out is None else out
    py, ldy = _rows(y, "out", x.dtype, (tokens, d), dev)
    eid = torch.empty(tokens, p.top_k, dtype=torch.int32, device=dev)
    gate = torch.empty(tokens, p.top_k, dtype=torch.float32, device=dev)
    work = torch.empty(size, dtype=torch.uint8, device=dev)
    _launch(dev, "janus_expert_layer", lib.janus_expert_layer, C.byref(p), px, ldx, tokens, py, ldy, eid.data_ptr(),
            gate.data_ptr(), work.data_ptr(), size)
    return y, eid, gate


class PackedRows(NamedTuple):
    """Activations in 8 bits: values q [rows, d] int8 and one code per 32 columns, code
    [rows, ceil(d / 32)] uint8; a value stands for q 2^(code - 127), code 255 for NaN."""
    q: object
    code: object


def _packed(p, device=None):
    rows, d, dev = _matrix(p.q, "q")
    if device is not None and dev != device:
        raise ValueError(f"q: on {dev}, expected {device}")
    pq, ldq = _rows(p.q, "q", torch.int8, (rows, d), dev)
    pc, ldc = _rows(p.code, "code", torch.uint8, (rows, (d + 31) // 32), dev)
    return rows, d, dev, (pq, ldq, pc, ldc)


def pack_rows(x, out=None) -> PackedRows:
    """x [rows, d] (float32, bfloat16 or float16) in 8 bits.  The values' rows start on multiples of 16 bytes;
    out = PackedRows to write into."""
    rows, d, dev = _matrix(x, "x")
    code = _type_of(x, "x")
    px, ldx = _rows(x, "x", x.dtype, (rows, d), dev)
    if out is None:
        wide = (d + 15) // 16 * 16
        q = torch.empty(rows, wide, dtype=torch.int8, device=dev)
        out = PackedRows(q if wide == d else q[:, :d], torch.empty(rows, (d + 31) // 32, dtype=torch.uint8, device=dev))
        at = (q.data_ptr(), wide, out.code.data_ptr(), (d + 31) // 32)
    else:
        n, w, _, at = _packed(out, dev)
        if (n, w) != (rows, d):
            raise ValueError(f"out: {n} x {w}, expected {rows} x {d}")
    _launch(dev, "janus_pack_rows", _lib().janus_pack_rows, px, ldx, code, rows, d, *at)
    return out


def unpack_rows(packed, dtype, act="none", grad=None, value=None, out=None):
    """What packed rows stand for, as `dtype`.

    act "none": returns X.  act "silu": returns SiLU(X), or with grad [rows, d] the gradient
    grad * SiLU'(X), or with grad and value=True both as (gradient, SiLU(X)).  `out`: tensor for the
    first result (it may be grad)."""
    rows, d, dev, at = _packed(packed)
    code = _type_of(dtype, "dtype")
    if act not in ACT:
        raise ValueError(f"act: {act!r}, expected one of {sorted(ACT)}")
    if grad is not None and act == "none":
        raise ValueError("grad: without an activation")
    pg, ldg = (None, 0) if grad is None else _rows(grad, "grad", dtype, (rows, d), dev)
    first = torch.empty(rows, d, dtype=dtype, device=dev) if out is None else out
    pf, ldf = _rows(first, "out", dtype, (rows, d), dev)
    second = torch.empty(rows, d, dtype=dtype, device=dev) if grad is not None and value else None
    ps, lds = (None, 0) if second is None else _rows(second, "value", dtype, (rows, d), dev)
    if grad is None:
        ps, lds, pf, ldf = pf, ldf, None, 0
    _launch(dev, "janus_unpack_rows", _lib().janus_unpack_rows, *at, rows, d, code, ACT[act], pg, ldg, pf, ldf, ps, lds)
    return first if second is None else (first, second)


def packed_wgrad(packed, B, row_off, out=None):
    """Grouped weight gradient from activations in 8 bits: G_g = X_g^T B_g over the rows
    row_off[g] .. row_off[g + 1] - 1 of X (packed [rows, P]) and B [rows, Q] (float32, bfloat16 or
    float16); returns G [groups, P, Q] float32.  row_off [groups + 1] int32 on the device."""
    rows, P, dev, at = _packed(packed)
    n, Q, _ = _matrix(B, "B")
    code = _type_of(B, "B")
    pb, ldb = _rows(B, "B", B.dtype, (rows, Q), dev)
    G = _offsets(row_off, "row_off", dev)
    if out is None:
        out = torch.empty(max(G, 0), P, Q, dtype=torch.float32, device=dev)
    else:
        _arg(out, "out", "f32", (G, P, Q), dev)
    lib = _lib()
    size = _call(lib.janus_packed_wgrad_workspace(rows, G, P, Q, code), "janus_packed_wgrad_workspace")
    work = torch.empty(size, dtype=torch.uint8, device=dev)
    _launch(dev, "janus_packed_wgrad", lib.janus_packed_wgrad, *at, pb, ldb, code, out.data_ptr(), row_off.data_ptr(), G,
            rows, P, Q, work.data_ptr(), size)
    return out


def upload(batch, device="cuda:0"):
    """Device copies of a synthetic batch: dict with pos, cell, species, offsets, E_ref, F_ref, W."""
    import torch
    t = lambda a, dt: torch.as_tensor(np.ascontiguousarray(a)).to(device=device, dtype=dt)
    return {
        "pos": t(batch.pos, torch.float32),
        "cell": t(batch.cell, torch.float32),
        "species": t(batch.species, torch.int32),
        "offsets": t(batch.offsets, torch.int32),
        "E_ref": t(batch.E_ref, torch.float32),
        "F_ref": t(batch.F_ref, torch.float32),
        "S_ref": None if batch.S_ref is None else t(batch.S_ref, torch.float32),
        "labels": None if batch.task is None else tuple(t(getattr(batch, k), torch.int32)
                                                        for k in ("task", "charge", "spin")),
        "W": t(pack_weights(batch.weights, batch.model), torch.float32),
    }
