"""Python binding of libmgn (argument marshalling only).

Every entry point of ``include/mgn.h`` is wrapped with the same name.  Host
arrays are NumPy; device buffers are torch tensors (torch supplies device
memory and the current HIP stream, nothing else).  All computation runs in
the HIP library; if ``libmgn.so`` is missing the import of any entry point
raises, there is no fallback.
"""
from __future__ import annotations

import collections
import ctypes as C
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
# MGN_LIB selects another build of the same library (the host-sanitizer
# build of build_sanitized.py); by default the in-tree libmgn.so
LIB_PATH = os.environ.get("MGN_LIB") or os.path.join(HERE, "libmgn.so")

OK, ERR_ARG, ERR_RANGE, ERR_SHAPE, ERR_WORKSPACE, ERR_STATE, ERR_DEVICE, ERR_NOMEM = 0, -1, -2, -3, -4, -5, -6, -7
FP32, BF16, E4M3, E5M2 = 0, 1, 2, 3
FORMATS = {"e4m3": E4M3, "e5m2": E5M2}
ACTS = {"none": 0, "relu": 1, "relu_grad": 2}
NORMS = {"none": 0, "layer": 1, "rms": 2}
GROUP_ACTS = {"none": 0, "relu": 1, "silu": 3}
NORM_MAX_COLS = 16384  # MGN_NORM_MAX_COLS of include/mgn.h
EULER, HEUN2, MIDPOINT, HEUN3, RK4, RALSTON2, RALSTON3 = 0, 1, 2, 3, 4, 5, 6
SCHEMES = {"euler": EULER, "heun2": HEUN2, "midpoint": MIDPOINT, "heun3": HEUN3, "rk4": RK4,
           "ralston2": RALSTON2, "ralston3": RALSTON3}
PRECISIONS = {"fp32": FP32, "bf16": BF16}


class MgnError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libmgn error {code}: {msg}")
        self.code = code


class Config(C.Structure):
    _fields_ = [("node_in", C.c_int32), ("edge_in", C.c_int32), ("latent", C.c_int32),
                ("out", C.c_int32), ("mp_steps", C.c_int32), ("mlp_layers", C.c_int32),
                ("ln_eps", C.c_float), ("precision", C.c_int32)]


class DGraph(C.Structure):
    _fields_ = [("n_nodes", C.c_int64), ("n_edges", C.c_int64), ("rowptr", C.c_void_p),
                ("senders", C.c_void_p), ("receivers", C.c_void_p), ("rev", C.c_void_p),
                ("tiles", C.c_void_p),
                ("n_tiles", C.c_int64), ("long_nodes", C.c_void_p), ("n_long", C.c_int64)]


class DPatch(C.Structure):
    _fields_ = [("g", DGraph), ("efeat", C.c_void_p), ("node_l2g", C.c_void_p), ("interior", C.c_void_p)]


class Adam(C.Structure):
    """mgn_adam: the paper's schedule (App. C) by default."""
    _fields_ = [("lr_start", C.c_double), ("lr_end", C.c_double), ("decay_steps", C.c_int64),
                ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double)]

    def __init__(self, lr_start=1e-3, lr_end=1e-7, decay_steps=4_000_000, beta1=0.9, beta2=0.999, eps=1e-8):
        super().__init__(lr_start, lr_end, decay_steps, beta1, beta2, eps)


class CMat8(C.Structure):
    _fields_ = [("q", C.c_void_p), ("scale", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64),
                ("ld", C.c_int64), ("format", C.c_int32), ("block_rows", C.c_int32)]


class Epilogue(C.Structure):
    _fields_ = [("bias", C.c_void_p), ("act", C.c_int32), ("aux_type", C.c_int32), ("aux", C.c_void_p),
                ("ldaux", C.c_int64), ("accumulate", C.c_int32)]


class CNormGate(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int32), ("x_type", C.c_int32), ("b_type", C.c_int32),
                ("post", C.c_int32), ("pre", C.c_int32), ("eps", C.c_float), ("skip", C.c_float),
                ("scale", C.c_float), ("post_gamma", C.c_void_p), ("post_beta", C.c_void_p),
                ("pre_gamma", C.c_void_p), ("pre_beta", C.c_void_p), ("gate", C.c_void_p),
                ("gate_ptr", C.c_void_p), ("n_gates", C.c_int64)]


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("ld", C.c_int64)]


class CNormGateGrads(C.Structure):
    _fields_ = [("post_gamma", C.c_void_p), ("post_beta", C.c_void_p), ("pre_gamma", C.c_void_p),
                ("pre_beta", C.c_void_p), ("gate", C.c_void_p), ("accumulate", C.c_int32)]


class CMat4(C.Structure):
    _fields_ = [("q", C.c_void_p), ("scale", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64)]


class CGroupNorm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int32), ("groups", C.c_int32), ("type", C.c_int32), ("act", C.c_int32),
                ("eps", C.c_float), ("gamma", C.c_void_p), ("beta", C.c_void_p), ("sample_ptr", C.c_void_p),
                ("n_samples", C.c_int64)]


class CTensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("in_type", C.c_int32),
                ("out_type", C.c_int32)]


class CPiece(C.Structure):
    _fields_ = [("data", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int32), ("types", C.c_int32)]


_lib = None

EXPORTS = [
    "mgn_param_count", "mgn_build_graph", "mgn_graph_info", "mgn_graph_copy",
    "mgn_graph_schedule", "mgn_tile_edges", "mgn_tile_nodes", "mgn_graph_destroy",
    "mgn_partition", "mgn_extract_patch", "mgn_patch_union", "mgn_patch_copy_maps", "mgn_ctx_create",
    "mgn_ctx_destroy", "mgn_forward", "mgn_forward_noalloc", "mgn_backward", "mgn_integrate_step",
    "mgn_pec_step", "mgn_patch_step", "mgn_adam_lr", "mgn_adam_step", "mgn_train_step", "mgn_scheme_stages", "mgn_version", "mgn_last_error", "mgn_profile_enable",
    "mgn_profile_collect", "mgn_quant8_workspace", "mgn_quant8", "mgn_matmul8_workspace", "mgn_matmul8",
    "mgn_norm_gate_forward", "mgn_norm_gate_workspace", "mgn_norm_gate_backward",
    "mgn_quant4_workspace", "mgn_quant4", "mgn_dequant4", "mgn_matmul4_workspace", "mgn_matmul4",
    "mgn_group_norm_workspace", "mgn_group_norm_forward", "mgn_group_norm_backward", "mgn_grad_piece",
    "mgn_grad_pieces", "mgn_grad_norm_workspace", "mgn_grad_norm", "mgn_grad_clip",
]


def lib():
    """Load libmgn.so (built in-tree); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"HIP library {LIB_PATH} is not built; run __graft_entry__.build()")
    L = C.CDLL(LIB_PATH)
    P, i32, i64, vp = C.POINTER, C.c_int32, C.c_int64, C.c_void_p
    sig = {
        "mgn_param_count": (i64, [P(Config)]),
        "mgn_build_graph": (C.c_int, [vp, i64, i32, vp, i64, i32, P(vp)]),
        "mgn_graph_info": (C.c_int, [vp, P(i64), P(i64)]),
        "mgn_graph_copy": (C.c_int, [vp, vp, vp, vp, vp, vp]),
        "mgn_graph_schedule": (C.c_int, [vp, vp, P(i64), vp, P(i64)]),
        "mgn_tile_edges": (i32, []),
        "mgn_tile_nodes": (i32, []),
        "mgn_graph_destroy": (None, [vp]),
        "mgn_partition": (C.c_int, [vp, i64, i32, vp, vp]),
        "mgn_extract_patch": (C.c_int, [vp, vp, i32, i32, P(vp)]),
        "mgn_patch_union": (C.c_int, [vp, i32, P(vp)]),
        "mgn_patch_copy_maps": (C.c_int, [vp, vp, vp, vp, vp, P(i64)]),
        "mgn_ctx_create": (C.c_int, [P(Config), i64, i64, i32, i32, P(C.c_size_t), P(vp)]),
        "mgn_ctx_destroy": (None, [vp]),
        "mgn_forward": (C.c_int, [vp, P(DGraph), vp, vp, vp, vp, i32, vp, C.c_size_t, vp]),
        "mgn_forward_noalloc": (C.c_int, [vp, P(DGraph), vp, vp, vp, vp, vp]),
        "mgn_backward": (C.c_int, [vp, vp, vp, vp, vp]),
        "mgn_integrate_step": (C.c_int, [vp, P(DGraph), vp, i32, vp, vp, vp, vp, i32, vp, C.c_size_t, vp]),
        "mgn_pec_step": (C.c_int, [vp, P(DGraph), vp, vp, vp, vp, vp, vp, i32, vp, C.c_size_t, vp]),
        "mgn_patch_step": (C.c_int, [vp, i32, P(DPatch), vp, i32, vp, vp, vp, i64, vp, C.c_size_t, vp]),
        "mgn_adam_lr": (C.c_double, [P(Adam), i64]),
        "mgn_adam_step": (C.c_int, [P(Adam), i64, vp, vp, vp, vp, i64, vp]),
        "mgn_train_step": (C.c_int, [vp, i32, P(DPatch), vp, i32, vp, vp, vp, vp, vp, i64, vp, vp, vp, P(Adam), i64,
                                     vp, i64, vp, C.c_size_t, vp]),
        "mgn_scheme_stages": (C.c_int, [i32]),
        "mgn_version": (C.c_char_p, []),
        "mgn_last_error": (C.c_char_p, []),
        "mgn_profile_enable": (C.c_int, [vp, i32]),
        "mgn_profile_collect": (C.c_int, [vp, i32, vp, vp, vp, P(i32)]),
        "mgn_quant8_workspace": (C.c_int, [i64, i64, P(C.c_size_t)]),
        "mgn_quant8": (C.c_int, [vp, i32, i64, i64, i64, i32, i32, vp, i64, vp, vp, i64, vp, vp, i32, vp, C.c_size_t,
                                 vp]),
        "mgn_matmul8_workspace": (C.c_int, [i64, i64, i64, P(C.c_size_t)]),
        "mgn_matmul8": (C.c_int, [P(CMat8), P(CMat8), P(Epilogue), i32, vp, i64, vp, C.c_size_t, vp]),
        "mgn_norm_gate_forward": (C.c_int, [P(CNormGate), Rows, Rows, Rows, Rows, vp, vp]),
        "mgn_norm_gate_workspace": (C.c_int, [i64, i32, P(C.c_size_t)]),
        "mgn_norm_gate_backward": (C.c_int, [P(CNormGate), Rows, Rows, vp, Rows, Rows, Rows, Rows, P(CNormGateGrads),
                                             vp, C.c_size_t, vp]),
        "mgn_quant4_workspace": (C.c_int, [i64, i64, P(C.c_size_t)]),
        "mgn_quant4": (C.c_int, [vp, i32, i64, i64, i64, vp, i64, vp, vp, i64, vp, vp, i32, vp, C.c_size_t, vp]),
        "mgn_dequant4": (C.c_int, [P(CMat4), i32, vp, i64, vp]),
        "mgn_matmul4_workspace": (C.c_int, [i64, i64, i64, P(C.c_size_t)]),
        "mgn_matmul4": (C.c_int, [P(CMat4), P(CMat4), P(Epilogue), i32, vp, i64, vp, C.c_size_t, vp]),
        "mgn_group_norm_workspace": (C.c_int, [P(CGroupNorm), i32, P(C.c_size_t)]),
        "mgn_group_norm_forward": (C.c_int, [P(CGroupNorm), Rows, Rows, vp, vp, C.c_size_t, vp]),
        "mgn_group_norm_backward": (C.c_int, [P(CGroupNorm), Rows, vp, Rows, Rows, vp, vp, i32, vp, C.c_size_t, vp]),
        "mgn_grad_piece": (i32, []),
        "mgn_grad_pieces": (C.c_int, [P(CTensor), i64, P(CPiece), P(i64)]),
        "mgn_grad_norm_workspace": (C.c_int, [i64, P(C.c_size_t)]),
        "mgn_grad_norm": (C.c_int, [vp, i64, vp, vp, C.c_size_t, vp]),
        "mgn_grad_clip": (C.c_int, [vp, i64, C.c_double, vp, i32, vp, C.c_size_t, vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def _check(rc):
    if rc != OK:
        raise MgnError(rc, lib().mgn_last_error().decode())
    return rc


def version():
    return lib().mgn_version().decode()


def last_error():
    return lib().mgn_last_error().decode()


def tile_edges():
    return lib().mgn_tile_edges()


def config(mp_steps, precision="fp32", ln_eps=1e-5, latent=128):
    prec = PRECISIONS[precision] if isinstance(precision, str) else int(precision)
    return Config(8, 4, latent, 4, int(mp_steps), 2, float(ln_eps), prec)


def param_count(mp_steps, latent=128):
    cfg = config(mp_steps, latent=latent)
    n = lib().mgn_param_count(C.byref(cfg))
    if n < 0:
        raise MgnError(ERR_SHAPE, last_error())
    return n


def _np(a, dtype):
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.ctypes.data_as(C.c_void_p)


# ------------------------------------------------------------ host graphs
class Graph:
    """Host mesh graph or patch (owns an mgn_graph handle)."""

    def __init__(self, handle, is_patch=False):
        self._h = C.c_void_p(handle)
        self.is_patch = is_patch
        n, e = C.c_int64(), C.c_int64()
        _check(lib().mgn_graph_info(self._h, C.byref(n), C.byref(e)))
        self.n_nodes, self.n_edges = n.value, e.value

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.mgn_graph_destroy(self._h)
            self._h = None

    def arrays(self):
        N, E = self.n_nodes, self.n_edges
        rowptr = np.empty(N + 1, np.int32)
        s = np.empty(E, np.int32)
        r = np.empty(E, np.int32)
        rev = np.empty(E, np.int32)
        f = np.empty((E, 4), np.float32)
        _check(lib().mgn_graph_copy(self._h, rowptr.ctypes.data, s.ctypes.data, r.ctypes.data,
                                    rev.ctypes.data, f.ctypes.data))
        return {"rowptr": rowptr, "senders": s, "receivers": r, "rev": rev, "efeat": f}

    def schedule(self):
        nt, nl = C.c_int64(), C.c_int64()
        _check(lib().mgn_graph_schedule(self._h, None, C.byref(nt), None, C.byref(nl)))
        tiles = np.empty((nt.value, 4), np.int32)
        longn = np.empty((nl.value, 4), np.int32)
        _check(lib().mgn_graph_schedule(self._h, tiles.ctypes.data, C.byref(nt),
                                        longn.ctypes.data, C.byref(nl)))
        return tiles, longn

    def patch_maps(self):
        N, E = self.n_nodes, self.n_edges
        l2g = np.empty(N, np.int32)
        hop = np.empty(N, np.int32)
        it = np.empty(N, np.uint8)
        el2g = np.empty(E, np.int64)
        ni = C.c_int64()
        _check(lib().mgn_patch_copy_maps(self._h, l2g.ctypes.data, hop.ctypes.data, it.ctypes.data,
                                         el2g.ctypes.data, C.byref(ni)))
        return {"node_l2g": l2g, "hop": hop, "interior": it, "edge_l2g": el2g,
                "n_interior": ni.value}


def build_graph(cells, pos):
    cells, pc = _np(cells, np.int32)
    pos, pp = _np(pos, np.float32)
    if cells.ndim != 2 or pos.ndim != 2:
        raise MgnError(ERR_ARG, "cells and pos must be 2-D")
    out = C.c_void_p()
    _check(lib().mgn_build_graph(pc, cells.shape[0], cells.shape[1], pp, pos.shape[0], pos.shape[1],
                                 C.byref(out)))
    return Graph(out.value)


def partition(pos, splits):
    pos, pp = _np(pos, np.float32)
    sp, spp = _np(splits, np.int32)
    part = np.empty(pos.shape[0], np.int32)
    _check(lib().mgn_partition(pp, pos.shape[0], pos.shape[1], spp, part.ctypes.data))
    return part


def extract_patch(g: Graph, part, p, k):
    part, pp = _np(part, np.int32)
    if part.shape != (g.n_nodes,):
        raise MgnError(ERR_ARG, "part must have one id per node")
    out = C.c_void_p()
    _check(lib().mgn_extract_patch(g._h, pp, int(p), int(k), C.byref(out)))
    return Graph(out.value, is_patch=True)


def patch_union(patches):
    """Disjoint union of patches as one patch-like graph (see include/mgn.h)."""
    arr = (C.c_void_p * max(1, len(patches)))(*[p._h.value for p in patches])
    out = C.c_void_p()
    _check(lib().mgn_patch_union(arr, len(patches), C.byref(out)))
    return Graph(out.value, is_patch=True)


# --------------------------------------------------------- device side
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dptr(t, dtype=None, shape=None, name="tensor"):
    torch = _torch()
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise MgnError(ERR_ARG, f"{name} must be a device tensor")
    if dtype is not None and t.dtype != dtype:
        raise MgnError(ERR_ARG, f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise MgnError(ERR_ARG, f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise MgnError(ERR_ARG, f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return C.c_void_p(t.data_ptr())


def _stream(stream):
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


class DeviceGraph:
    """Device copies of a graph's CSR arrays and tile schedule."""

    def __init__(self, g: Graph, device="cuda"):
        torch = _torch()
        a = g.arrays()
        tiles, longn = g.schedule()
        dev = torch.device(device)
        self.n_nodes, self.n_edges = g.n_nodes, g.n_edges
        self.rowptr = torch.from_numpy(a["rowptr"]).to(dev)
        self.senders = torch.from_numpy(a["senders"]).to(dev)
        self.receivers = torch.from_numpy(a["receivers"]).to(dev)
        self.rev = torch.from_numpy(a["rev"]).to(dev)
        self.tiles = torch.from_numpy(tiles.reshape(-1)).to(dev)
        self.long_nodes = torch.from_numpy(longn.reshape(-1)).to(dev)
        self.efeat = torch.from_numpy(a["efeat"]).to(dev)
        self.n_tiles, self.n_long = tiles.shape[0], longn.shape[0]
        self.struct = DGraph(self.n_nodes, self.n_edges, self.rowptr.data_ptr(),
                             self.senders.data_ptr(), self.receivers.data_ptr(),
                             self.rev.data_ptr(), self.tiles.data_ptr(),
                             self.n_tiles,
                             self.long_nodes.data_ptr() if self.n_long else None, self.n_long)


class DevicePatch:
    """A patch on the device: its local graph (DeviceGraph) and the maps
    node_l2g / interior of mgn_patch_copy_maps."""

    def __init__(self, patch: Graph, device="cuda"):
        torch = _torch()
        mp = patch.patch_maps()
        self.dg = DeviceGraph(patch, device)
        self.node_l2g = torch.from_numpy(mp["node_l2g"]).to(device)
        self.interior = torch.from_numpy(mp["interior"]).to(device)
        self.n_nodes, self.n_edges, self.n_interior = patch.n_nodes, patch.n_edges, mp["n_interior"]
        self.struct = DPatch(self.dg.struct, self.dg.efeat.data_ptr(), self.node_l2g.data_ptr(),
                             self.interior.data_ptr())


class Context:
    """mgn_ctx plus a workspace tensor of the size the library asks for."""

    def __init__(self, mp_steps, max_nodes, max_edges, precision="fp32", max_stages=1,
                 save=False, ln_eps=1e-5, device="cuda", allocate=True, latent=128):
        self.cfg = config(mp_steps, precision, ln_eps, latent)
        self.mp_steps = int(mp_steps)
        self.latent = int(latent)
        ws = C.c_size_t()
        h = C.c_void_p()
        _check(lib().mgn_ctx_create(C.byref(self.cfg), int(max_nodes), int(max_edges),
                                    int(max_stages), 1 if save else 0, C.byref(ws), C.byref(h)))
        self._h = h
        self.ws_bytes = ws.value
        self.ws = None
        if allocate:
            torch = _torch()
            self.ws = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=device)

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.mgn_ctx_destroy(self._h)
            self._h = None


def mgn_forward(ctx: Context, g: DeviceGraph, params, node_in, efeat, out=None, save=False,
                stream=None):
    torch = _torch()
    N, E = g.n_nodes, g.n_edges
    if out is None:
        out = torch.empty((N, 4), dtype=torch.float32, device=node_in.device)
    _check(lib().mgn_forward(ctx._h, C.byref(g.struct), _dptr(params, torch.float32, name="params"),
                             _dptr(node_in, torch.float32, (N, 8), "node_in"),
                             _dptr(efeat, torch.float32, (E, 4), "efeat"),
                             _dptr(out, torch.float32, (N, 4), "out"), 1 if save else 0,
                             _dptr(ctx.ws, name="workspace"), ctx.ws_bytes, _stream(stream)))
    return out


NOALLOC_SCRATCH_BYTES = 128 << 20  # MGN_NOALLOC_SCRATCH_BYTES of include/mgn.h


def mgn_forward_noalloc(ctx: Context, g: DeviceGraph, params, node_in, efeat, out, stream=None):
    """mgn_forward (no saved activations) on the library's static device
    scratch instead of ctx's workspace: the context may be created with
    allocate=False; `out` must be given (nothing is allocated)."""
    torch = _torch()
    N, E = g.n_nodes, g.n_edges
    _check(lib().mgn_forward_noalloc(ctx._h, C.byref(g.struct), _dptr(params, torch.float32, name="params"),
                                     _dptr(node_in, torch.float32, (N, 8), "node_in"),
                                     _dptr(efeat, torch.float32, (E, 4), "efeat"),
                                     _dptr(out, torch.float32, (N, 4), "out"), _stream(stream)))
    return out


def mgn_backward(ctx: Context, grad_out, grad_params, grad_in=None, stream=None):
    torch = _torch()
    _check(lib().mgn_backward(ctx._h, _dptr(grad_out, torch.float32, name="grad_out"),
                              _dptr(grad_params, torch.float32, name="grad_params"),
                              _dptr(grad_in, torch.float32, name="grad_in") if grad_in is not None else None,
                              _stream(stream)))
    return grad_params


def mgn_integrate_step(ctx: Context, g: DeviceGraph, params, scheme, static, y, efeat,
                       y_next=None, save=False, stream=None):
    torch = _torch()
    N, E = g.n_nodes, g.n_edges
    sc = SCHEMES[scheme] if isinstance(scheme, str) else int(scheme)
    if y_next is None:
        y_next = torch.empty((N, 4), dtype=torch.float32, device=y.device)
    _check(lib().mgn_integrate_step(ctx._h, C.byref(g.struct), _dptr(params, torch.float32, name="params"),
                                    sc, _dptr(static, torch.float32, (N, 4), "static"),
                                    _dptr(y, torch.float32, (N, 4), "y"),
                                    _dptr(efeat, torch.float32, (E, 4), "efeat"),
                                    _dptr(y_next, torch.float32, (N, 4), "y_next"), 1 if save else 0,
                                    _dptr(ctx.ws, name="workspace"), ctx.ws_bytes, _stream(stream)))
    return y_next


def mgn_patch_step(ctx: Context, patches, params, scheme, static, y, y_next=None, stream=None):
    """One integration step of the whole mesh computed patch by patch with
    ghost refresh (see include/mgn.h); patches: list of DevicePatch."""
    torch = _torch()
    n = y.shape[0]
    sc = SCHEMES[scheme] if isinstance(scheme, str) else int(scheme)
    if y_next is None:
        y_next = torch.empty((n, 4), dtype=torch.float32, device=y.device)
    arr = (DPatch * max(1, len(patches)))(*[p.struct for p in patches])
    _check(lib().mgn_patch_step(ctx._h, len(patches), arr, _dptr(params, torch.float32, name="params"), sc,
                                _dptr(static, torch.float32, (n, 4), "static"), _dptr(y, torch.float32, (n, 4), "y"),
                                _dptr(y_next, torch.float32, (n, 4), "y_next"), n,
                                _dptr(ctx.ws, name="workspace"), ctx.ws_bytes, _stream(stream)))
    return y_next


def mgn_adam_lr(adam, k):
    return lib().mgn_adam_lr(C.byref(adam), int(k))


def mgn_adam_step(adam, k, params, grad, m, v, stream=None):
    """The k-th Adam update of params in place (see include/mgn.h)."""
    torch = _torch()
    n = params.numel()
    _check(lib().mgn_adam_step(C.byref(adam), int(k), _dptr(params, torch.float32, name="params"),
                               _dptr(grad, torch.float32, (n,), "grad"), _dptr(m, torch.float32, (n,), "m"),
                               _dptr(v, torch.float32, (n,), "v"), n, _stream(stream)))


def mgn_train_step(ctx: Context, patches, params, scheme, static, y, y_target, noise, grad, m, v, adam, k,
                   n_loss_nodes=None, noise_std=None, loss=None, stream=None):
    """One patch-training step (see include/mgn.h); returns the device loss
    (a 1-element tensor)."""
    torch = _torch()
    n = y.shape[0]
    sc = SCHEMES[scheme] if isinstance(scheme, str) else int(scheme)
    if loss is None:
        loss = torch.zeros(1, dtype=torch.float32, device=y.device)
    if n_loss_nodes is None:
        n_loss_nodes = sum(int(p.n_interior) for p in patches)
    sd = None if noise_std is None else (C.c_float * 4)(*[float(x) for x in noise_std])
    arr = (DPatch * max(1, len(patches)))(*[p.struct for p in patches])
    npar = params.numel()
    _check(lib().mgn_train_step(ctx._h, len(patches), arr, _dptr(params, torch.float32, name="params"), sc,
                                _dptr(static, torch.float32, (n, 4), "static"), _dptr(y, torch.float32, (n, 4), "y"),
                                _dptr(y_target, torch.float32, (n, 4), "y_target"),
                                _dptr(noise, torch.float32, (n, 4), "noise") if noise is not None else None,
                                C.cast(sd, C.c_void_p) if sd is not None else None, int(n_loss_nodes),
                                _dptr(grad, torch.float32, (npar,), "grad"), _dptr(m, torch.float32, (npar,), "m"),
                                _dptr(v, torch.float32, (npar,), "v"), C.byref(adam), int(k),
                                _dptr(loss, torch.float32, (1,), "loss"), n,
                                _dptr(ctx.ws, name="workspace"), ctx.ws_bytes, _stream(stream)))
    return loss


def mgn_pec_step(ctx: Context, g: DeviceGraph, params, static, y, khist, efeat, first=False,
                 y_next=None, stream=None):
    """One predict-evaluate-correct inference step; khist [2][N][4] is the
    derivative history, updated in place (see include/mgn.h)."""
    torch = _torch()
    N, E = g.n_nodes, g.n_edges
    if y_next is None:
        y_next = torch.empty((N, 4), dtype=torch.float32, device=y.device)
    _check(lib().mgn_pec_step(ctx._h, C.byref(g.struct), _dptr(params, torch.float32, name="params"),
                              _dptr(static, torch.float32, (N, 4), "static"),
                              _dptr(y, torch.float32, (N, 4), "y"),
                              _dptr(khist, torch.float32, (2, N, 4), "khist"),
                              _dptr(efeat, torch.float32, (E, 4), "efeat"),
                              _dptr(y_next, torch.float32, (N, 4), "y_next"), 1 if first else 0,
                              _dptr(ctx.ws, name="workspace"), ctx.ws_bytes, _stream(stream)))
    return y_next


def mgn_profile_enable(ctx: Context, enable=True):
    _check(lib().mgn_profile_enable(ctx._h, 1 if enable else 0))


def mgn_profile_collect(ctx: Context, max_kernels=32):
    """{kernel kind: (total_ms, launches)} since the last collect."""
    names = C.create_string_buffer(32 * max_kernels)
    ms = np.zeros(max_kernels, np.float64)
    cnt = np.zeros(max_kernels, np.int64)
    n = C.c_int32()
    _check(lib().mgn_profile_collect(ctx._h, max_kernels, names, ms.ctypes.data, cnt.ctypes.data,
                                     C.byref(n)))
    out = {}
    for k in range(min(n.value, max_kernels)):
        nm = names.raw[32 * k:32 * k + 32].split(b"\0")[0].decode()
        out[nm] = (float(ms[k]), int(cnt[k]))
    return out


def scheme_stages(scheme):
    sc = SCHEMES[scheme] if isinstance(scheme, str) else int(scheme)
    n = lib().mgn_scheme_stages(sc)
    if n < 0:
        raise MgnError(n, last_error())
    return n


# ------------------------------------------------------- row operators
# Inputs of these may be slices of wider tensors: any row stride, columns next
# to each other.  Outputs that are not given are allocated, and scratch is
# taken from torch's allocator for the call.
def _row_type(t, name):
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 2:
        raise MgnError(ERR_ARG, f"{name} must be a two-dimensional device tensor")
    dt = t.dtype
    if dt is torch.float32:
        return FP32
    if dt is torch.bfloat16:
        return BF16
    raise MgnError(ERR_ARG, f"{name} must be float32 or bfloat16, got {dt}")


def _row_ld(t, name, shape=None):
    """Leading dimension of a row tensor (its columns have to be adjacent)."""
    r, c = t.shape
    if shape is not None and (r, c) != shape:
        raise MgnError(ERR_ARG, f"{name} has shape {(r, c)}, expected {shape}")
    sr, sc = t.stride()
    if c > 1 and sc != 1:
        raise MgnError(ERR_ARG, f"{name}: the columns of a row must be adjacent")
    if r <= 1:
        return c
    if sr < c:
        raise MgnError(ERR_ARG, f"{name}: rows overlap (stride {sr} for {c} columns)")
    return sr


def _vector(t, name, n, device):
    torch = _torch()
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.device != device or t.numel() != n \
            or not t.is_contiguous():
        raise MgnError(ERR_ARG, f"{name} must be {n} contiguous float32 values on {device}")
    return t.data_ptr()


_raw_stream = None  # device index -> the current stream's handle


def _current_stream(device):
    global _raw_stream
    if _raw_stream is None:
        torch = _torch()
        # torch.cuda.current_stream builds an object: 1.9 us a call instead of 0.1
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _raw_stream(device.index)


def _run(device, fn, args):
    """fn(*args, current stream) with the tensors' device current."""
    torch = _torch()
    if device.index == torch.cuda.current_device():
        rc = fn(*args, _current_stream(device))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _current_stream(device))
    if rc != OK:
        _check(rc)


def _elsewhere(fn, args):
    """fn(**args) on args["stream"]: what it allocates belongs to that stream,
    and the tensors it is given are kept from reuse until it is done with them."""
    torch = _torch()
    stream = args.pop("stream")
    given = []
    for v in args.values():
        given += [v] if isinstance(v, torch.Tensor) else [v.q, v.scale] if isinstance(v, (Mat8, Mat4)) else \
            v.tensors() if isinstance(v, TensorList) else \
            [t for t in v if isinstance(t, torch.Tensor)] if isinstance(v, tuple) else []
    for t in given:
        if t.is_cuda and t.device != stream.device:
            raise MgnError(ERR_ARG, f"the stream is of {stream.device}, a tensor on {t.device}")
    with torch.cuda.stream(stream):
        out = fn(**args)
    for t in given:
        if t.is_cuda:
            t.record_stream(stream)
    return out


def _scratch(nbytes, device):
    torch = _torch()
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _at(t):
    return None if t is None else t.data_ptr()


def _matrix_ld(q):
    """Leading dimension of a matrix's numbers, whose columns have to be adjacent: of one
    row, whose stride means nothing, its columns rounded up to a multiple of 16."""
    r, c = q.shape
    ld = _row_ld(q, "q") if r > 0 else c
    return ld if r > 1 else -(-c // 16) * 16


class Mat8:
    """An mgn_mat8 of include/mgn.h: q, a float8_e4m3fn or float8_e5m2 tensor
    [rows][ld >= cols] whose bytes from cols to the next multiple of 16 are
    zero, and its scales [ceil(cols / 128)][ceil(rows / block_rows)] in float32."""
    __slots__ = ("q", "scale", "rows", "cols", "block_rows", "struct")

    def __init__(self, q, scale, cols=None, block_rows=1):
        torch = _torch()
        if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 2:
            raise MgnError(ERR_ARG, "q must be a two-dimensional device tensor")
        if q.dtype == torch.float8_e4m3fn:
            fmt = E4M3
        elif q.dtype == torch.float8_e5m2:
            fmt = E5M2
        else:
            raise MgnError(ERR_ARG, f"q must be float8_e4m3fn or float8_e5m2, got {q.dtype}")
        rows, width = q.shape
        cols = width if cols is None else int(cols)
        if block_rows not in (1, 128):
            raise MgnError(ERR_ARG, f"blocks of {block_rows} rows (1 or 128)")
        ld = _matrix_ld(q)
        if not 0 <= cols <= width or (width < -(-cols // 16) * 16 and rows > 0):
            raise MgnError(ERR_ARG, f"q has {width} columns for {cols}: rows are padded to multiples of 16")
        want = (-(-cols // 128), -(-rows // block_rows))
        if not isinstance(scale, torch.Tensor) or scale.dtype != torch.float32 or tuple(scale.shape) != want \
                or scale.device != q.device or not scale.is_contiguous():
            raise MgnError(ERR_ARG, f"scale must be a contiguous float32 tensor of shape {want} on {q.device}")
        self._set(q, scale, rows, cols, ld, fmt, block_rows)

    def _set(self, q, scale, rows, cols, ld, fmt, block_rows):
        self.q, self.scale, self.rows, self.cols, self.block_rows = q, scale, rows, cols, block_rows
        self.struct = CMat8(q.data_ptr(), scale.data_ptr(), rows, cols, ld, fmt, block_rows)
        return self


Quantised = collections.namedtuple("Quantised", "rows columns colsum")


def mgn_quant8(x, format="e4m3", block_rows=1, rowwise=True, transposed=False, colsum=False, accumulate=False,
               stream=None):
    """Quantises x [rows][cols] to 8 bits with a scale for each block of
    block_rows x 128 (see include/mgn.h).  Returns (rows, columns, colsum): x
    and its transpose as Mat8, or None, and the sums over x's rows: a new
    tensor with colsum=True, or the given one (added to with accumulate)."""
    if stream is not None:
        return _elsewhere(mgn_quant8, dict(locals()))
    torch = _torch()
    xt = _row_type(x, "x")
    fmt = FORMATS.get(format)
    if fmt is None:
        raise MgnError(ERR_ARG, f"unknown 8-bit format {format!r}")
    if block_rows != 1 and block_rows != 128:
        raise MgnError(ERR_ARG, f"blocks of {block_rows} rows (1 or 128)")
    r, c = x.shape
    ldx = _row_ld(x, "x")
    dev, f8 = x.device, torch.float8_e4m3fn if fmt == E4M3 else torch.float8_e5m2
    q = s = qt = st = sums = ws = None
    rb, cb, ldq, ldqt, need = -(-r // 128), -(-c // 128), -(-c // 16) * 16, -(-r // 16) * 16, 0
    if rowwise:
        q = torch.empty((r, ldq), dtype=f8, device=dev)
        s = torch.empty((cb, r if block_rows == 1 else rb), dtype=torch.float32, device=dev)
    if transposed:
        qt = torch.empty((c, ldqt), dtype=f8, device=dev)
        st = torch.empty((rb, c if block_rows == 1 else cb), dtype=torch.float32, device=dev)
    if isinstance(colsum, torch.Tensor):
        sums = colsum
        _vector(sums, "colsum", c, dev)
    elif accumulate:
        raise MgnError(ERR_ARG, "accumulate needs the sums to add to")
    elif colsum:
        sums = torch.empty(c, dtype=torch.float32, device=dev)
    if sums is not None:
        need = rb * c * 4
        ws = _scratch(need, dev)
    if r > 0 and c > 0 or sums is not None:
        _run(dev, lib().mgn_quant8,
             (x.data_ptr(), xt, r, c, ldx, fmt, block_rows, _at(q) or None, ldq, _at(s) or None, _at(qt) or None, ldqt,
              _at(st) or None, _at(sums), 1 if accumulate else 0, _at(ws), need))
    return Quantised(Mat8.__new__(Mat8)._set(q, s, r, c, ldq, fmt, block_rows) if rowwise else None,
                     Mat8.__new__(Mat8)._set(qt, st, c, r, ldqt, fmt, block_rows) if transposed else None, sums)


def mgn_matmul8(a, b, bias=None, act="none", aux=None, out=None, dtype=None, accumulate=False, stream=None):
    """act(a b^T + bias) of two Mat8 (see include/mgn.h): [a.rows][b.rows] in
    float32 or bfloat16 (dtype, default float32; out: written, or added to
    with accumulate)."""
    if stream is not None:
        return _elsewhere(mgn_matmul8, dict(locals()))
    torch = _torch()
    if not isinstance(a, Mat8) or not isinstance(b, Mat8):
        raise MgnError(ERR_ARG, "a and b must be Mat8")
    if a.cols != b.cols:
        raise MgnError(ERR_SHAPE, f"a has {a.cols} columns, b {b.cols}")
    if act not in ACTS:
        raise MgnError(ERR_ARG, f"unknown act {act!r}")
    dev, m, n = a.q.device, a.rows, b.rows
    if b.q.device != dev:
        raise MgnError(ERR_ARG, f"b is on {b.q.device}, expected {dev}")
    if out is None:
        if accumulate:
            raise MgnError(ERR_ARG, "accumulate needs an out to add to")
        if dtype is None or dtype == torch.float32:
            ct, out = FP32, torch.empty((m, n), dtype=torch.float32, device=dev)
        elif dtype == torch.bfloat16:
            ct, out = BF16, torch.empty((m, n), dtype=torch.bfloat16, device=dev)
        else:
            raise MgnError(ERR_ARG, f"out is float32 or bfloat16, not {dtype}")
        ldc = n
    else:
        ct, ldc = _row_type(out, "out"), _row_ld(out, "out", (m, n))
        if dtype is not None and out.dtype != dtype:
            raise MgnError(ERR_ARG, f"out must be {dtype}, got {out.dtype}")
        if out.device != dev:
            raise MgnError(ERR_ARG, f"out is on {out.device}, expected {dev}")
    ep = None
    if bias is not None or act != "none" or accumulate:
        ep = Epilogue(bias=_vector(bias, "bias", n, dev), act=ACTS[act], accumulate=1 if accumulate else 0)
    if act == "relu_grad":
        ep.aux_type, ep.ldaux = _row_type(aux, "aux"), _row_ld(aux, "aux", (m, n))
        if aux.device != dev:
            raise MgnError(ERR_ARG, f"aux is on {aux.device}, expected {dev}")
        ep.aux = aux.data_ptr()
    elif aux is not None:
        raise MgnError(ERR_ARG, "aux is for relu_grad only")
    if m == 0 or n == 0:
        return out
    L = lib()
    need = C.c_size_t()
    _check(L.mgn_matmul8_workspace(m, n, a.cols, C.byref(need)))
    ws = _scratch(need.value, dev)
    _run(dev, L.mgn_matmul8,
         (C.byref(a.struct), C.byref(b.struct), None if ep is None else C.byref(ep), ct, out.data_ptr(), ldc, _at(ws),
          need.value))
    return out


def _norm_gate(x, b, post, pre, post_gamma, post_beta, pre_gamma, pre_beta, gate, gate_ptr, skip, scale, eps):
    torch = _torch()
    xt, bt = _row_type(x, "x"), _row_type(b, "b")
    if post not in NORMS or pre not in NORMS:
        raise MgnError(ERR_ARG, f"unknown norm {post!r} or {pre!r}")
    rows, cols = x.shape
    dev, n_gates = x.device, 0
    if b.device != dev:
        raise MgnError(ERR_ARG, f"b is on {b.device}, expected {dev}")
    if not 1 <= cols <= NORM_MAX_COLS:
        raise MgnError(ERR_SHAPE, f"{cols} columns (1 to {NORM_MAX_COLS})")
    if gate is not None:
        if not isinstance(gate, torch.Tensor) or gate.dim() != 2 or gate.shape[1] != cols:
            raise MgnError(ERR_ARG, f"gate must be a tensor of shape (gates, {cols})")
        n_gates = gate.shape[0]
        if n_gates == 0 and rows > 0:
            raise MgnError(ERR_ARG, f"no gates for {rows} rows (without a gate: None)")
        _vector(gate, "gate", n_gates * cols, dev)
    if gate_ptr is not None:
        _dptr(gate_ptr, torch.int32, (n_gates + 1,), "gate_ptr")
        if gate_ptr.device != dev:
            raise MgnError(ERR_ARG, f"gate_ptr is on {gate_ptr.device}, expected {dev}")
        if gate is not None and n_gates == 0:
            gate_ptr = None  # no groups and no rows
    return CNormGate(rows, cols, xt, bt, NORMS[post], NORMS[pre], eps, skip, scale,
                     _vector(post_gamma, "post_gamma", cols, dev), _vector(post_beta, "post_beta", cols, dev),
                     _vector(pre_gamma, "pre_gamma", cols, dev), _vector(pre_beta, "pre_beta", cols, dev), _at(gate),
                     _at(gate_ptr), n_gates)


def _as_rows(t, name, shape, dtype, device):
    if t is None:
        return Rows(None, 0)
    _row_type(t, name)
    if t.dtype != dtype:
        raise MgnError(ERR_ARG, f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise MgnError(ERR_ARG, f"{name} is on {t.device}, expected {device}")
    return Rows(t.data_ptr(), _row_ld(t, name, shape))


def _new_rows(shape, dtype, device):
    t = _torch().empty(shape, dtype=dtype, device=device)
    return t, Rows(t.data_ptr(), shape[1])


def mgn_norm_gate_forward(x, b, post="none", pre="none", post_gamma=None, post_beta=None, pre_gamma=None,
                          pre_beta=None, gate=None, gate_ptr=None, skip=1.0, scale=1.0, eps=1e-5, save=False, y=None,
                          z=None, stream=None):
    """y = skip x + scale gate post(b), z = pre(y) (see include/mgn.h).
    Returns (y, z, stats): z None with pre="none", stats None without save.
    y may be x, z may be b.  Rows outside of the groups of gate_ptr are not
    written: a y or z that is not given holds any bits there."""
    if stream is not None:
        return _elsewhere(mgn_norm_gate_forward, dict(locals()))
    torch = _torch()
    op = _norm_gate(x, b, post, pre, post_gamma, post_beta, pre_gamma, pre_beta, gate, gate_ptr, skip, scale, eps)
    shape, dev = tuple(x.shape), x.device
    y, yr = _new_rows(shape, x.dtype, dev) if y is None else (y, _as_rows(y, "y", shape, x.dtype, dev))
    if pre == "none":
        if z is not None:
            raise MgnError(ERR_ARG, "z without a norm before the next block")
        zr = Rows(None, 0)
    else:
        z, zr = _new_rows(shape, b.dtype, dev) if z is None else (z, _as_rows(z, "z", shape, b.dtype, dev))
    stats = torch.empty((shape[0], 4), dtype=torch.float32, device=dev) if save else None
    xr, br = Rows(x.data_ptr(), _row_ld(x, "x")), Rows(b.data_ptr(), _row_ld(b, "b", shape))
    _run(dev, lib().mgn_norm_gate_forward, (C.byref(op), xr, br, yr, zr, _at(stats)))
    return y, z, stats


NormGateGrads = collections.namedtuple("NormGateGrads", "dx db dgate dpost_gamma dpost_beta dpre_gamma dpre_beta")


def mgn_norm_gate_backward(x, b, stats, dy, dz, post="none", pre="none", post_gamma=None, post_beta=None,
                           pre_gamma=None, pre_beta=None, gate=None, gate_ptr=None, skip=1.0, scale=1.0, eps=1e-5,
                           dx=None, db=None, grads=None, stream=None):
    """Reverse of mgn_norm_gate_forward (see include/mgn.h) from its inputs and
    stats.  dy or dz None: zero.  Returns NormGateGrads; the gradients of the
    vectors and of the gate are those of the parameters that were given, new
    tensors, or those of grads (a NormGateGrads of an earlier call) added to.
    Rows of dx and db outside of the groups of gate_ptr are not written."""
    if stream is not None:
        return _elsewhere(mgn_norm_gate_backward, dict(locals()))
    torch = _torch()
    op = _norm_gate(x, b, post, pre, post_gamma, post_beta, pre_gamma, pre_beta, gate, gate_ptr, skip, scale, eps)
    shape, dev = tuple(x.shape), x.device
    rows, cols = shape
    dx, dxr = _new_rows(shape, x.dtype, dev) if dx is None else (dx, _as_rows(dx, "dx", shape, x.dtype, dev))
    db, dbr = _new_rows(shape, b.dtype, dev) if db is None else (db, _as_rows(db, "db", shape, b.dtype, dev))
    if not isinstance(stats, torch.Tensor) or tuple(stats.shape) != (rows, 4):
        raise MgnError(ERR_ARG, "stats must be the forward's, of shape (rows, 4)")
    _vector(stats, "stats", rows * 4, dev)
    out = {}
    for name, p, used in (("dgate", gate, True), ("dpost_gamma", post_gamma, post != "none"),
                          ("dpost_beta", post_beta, post != "none"), ("dpre_gamma", pre_gamma, pre != "none"),
                          ("dpre_beta", pre_beta, pre != "none")):
        g = getattr(grads, name) if grads is not None else None
        if p is None or not used:
            if g is not None:
                raise MgnError(ERR_ARG, f"{name} without its parameter")
        elif grads is None:
            g = torch.empty(p.shape, dtype=torch.float32, device=dev)
        elif g is not None:
            _vector(g, name, p.numel(), dev)
        out[name] = g
    cg = CNormGateGrads(_at(out["dpost_gamma"]), _at(out["dpost_beta"]), _at(out["dpre_gamma"]), _at(out["dpre_beta"]),
                        _at(out["dgate"]), 0 if grads is None else 1)
    xr, br = Rows(x.data_ptr(), _row_ld(x, "x")), Rows(b.data_ptr(), _row_ld(b, "b", shape))
    dyr, dzr = _as_rows(dy, "dy", shape, x.dtype, dev), _as_rows(dz, "dz", shape, b.dtype, dev)
    need = C.c_size_t()
    _check(lib().mgn_norm_gate_workspace(rows, cols, C.byref(need)))
    ws = _scratch(need.value, dev)
    _run(dev, lib().mgn_norm_gate_backward,
         (C.byref(op), xr, br, stats.data_ptr(), dyr, dzr, dxr, dbr, C.byref(cg), _at(ws), need.value))
    return NormGateGrads(dx, db, **out)


class Mat4:
    """An mgn_mat4 of include/mgn.h: q, a uint8 tensor [rows][ld] of 4-bit numbers,
    two a byte, those from cols to the next multiple of 32 zero, and its scales
    [ceil(cols / 128)][rows][4] in float8_e8m0fnu (or uint8), those behind the
    last 32 columns zero bytes."""
    __slots__ = ("q", "scale", "rows", "cols", "struct")

    def __init__(self, q, scale, cols):
        torch = _torch()
        if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 2 or q.dtype != torch.uint8:
            raise MgnError(ERR_ARG, "q must be a two-dimensional uint8 device tensor")
        rows, width = q.shape
        cols = int(cols)
        need = -(-cols // 32) * 16
        ld = _matrix_ld(q)
        if cols < 0 or (width < need and rows > 0):
            raise MgnError(ERR_ARG, f"q has {width} bytes a row for {cols} columns: {need} are needed")
        want = (-(-cols // 128), rows, 4)
        if not isinstance(scale, torch.Tensor) or scale.dtype not in (torch.float8_e8m0fnu, torch.uint8) \
                or tuple(scale.shape) != want or scale.device != q.device or not scale.is_contiguous():
            raise MgnError(ERR_ARG, f"scale must be a contiguous float8_e8m0fnu tensor of shape {want} on {q.device}")
        self._set(q, scale, rows, cols, ld)

    def _set(self, q, scale, rows, cols, ld):
        self.q, self.scale, self.rows, self.cols = q, scale, rows, cols
        self.struct = CMat4(q.data_ptr(), scale.data_ptr(), rows, cols, ld)
        return self


def mgn_quant4(x, rowwise=True, transposed=False, colsum=False, accumulate=False, stream=None):
    """Quantises x [rows][cols] to 4 bits with a power of two for each 32 columns
    of a row (see include/mgn.h).  Returns (rows, columns, colsum): x and its
    transpose as Mat4, or None, and the sums over x's rows: a new tensor with
    colsum=True, or the given one (added to with accumulate)."""
    if stream is not None:
        return _elsewhere(mgn_quant4, dict(locals()))
    torch = _torch()
    xt = _row_type(x, "x")
    r, c = x.shape
    ldx = _row_ld(x, "x")
    dev = x.device
    q = s = qt = st = sums = ws = None
    rb, cb, ldq, ldqt, need = -(-r // 128), -(-c // 128), -(-c // 32) * 16, -(-r // 32) * 16, 0
    if rowwise:
        q = torch.empty((r, ldq), dtype=torch.uint8, device=dev)
        s = torch.empty((cb, r, 4), dtype=torch.float8_e8m0fnu, device=dev)
    if transposed:
        qt = torch.empty((c, ldqt), dtype=torch.uint8, device=dev)
        st = torch.empty((rb, c, 4), dtype=torch.float8_e8m0fnu, device=dev)
    if isinstance(colsum, torch.Tensor):
        sums = colsum
        _vector(sums, "colsum", c, dev)
    elif accumulate:
        raise MgnError(ERR_ARG, "accumulate needs the sums to add to")
    elif colsum:
        sums = torch.empty(c, dtype=torch.float32, device=dev)
    if sums is not None:
        need = rb * c * 4
        ws = _scratch(need, dev)
    if r > 0 and c > 0 or sums is not None:
        _run(dev, lib().mgn_quant4,
             (x.data_ptr(), xt, r, c, ldx, _at(q) or None, ldq, _at(s) or None, _at(qt) or None, ldqt, _at(st) or None,
              _at(sums), 1 if accumulate else 0, _at(ws), need))
    return Quantised(Mat4.__new__(Mat4)._set(q, s, r, c, ldq) if rowwise else None,
                     Mat4.__new__(Mat4)._set(qt, st, c, r, ldqt) if transposed else None, sums)


def mgn_dequant4(a, dtype=None, out=None, stream=None):
    """The values of a Mat4 as rows in float32 or bfloat16 (dtype, default
    float32, or those of out)."""
    if stream is not None:
        return _elsewhere(mgn_dequant4, dict(locals()))
    if not isinstance(a, Mat4):
        raise MgnError(ERR_ARG, "a must be a Mat4")
    yt, ldy, out = _result(out, dtype, (a.rows, a.cols), a.q.device)
    if a.rows > 0 and a.cols > 0:
        _run(a.q.device, lib().mgn_dequant4, (C.byref(a.struct), yt, out.data_ptr(), ldy))
    return out


def _result(out, dtype, shape, device):
    """(type, leading dimension, tensor) of a result: out, or a new one of dtype."""
    torch = _torch()
    if out is None:
        if dtype is None or dtype == torch.float32:
            return FP32, shape[1], torch.empty(shape, dtype=torch.float32, device=device)
        if dtype == torch.bfloat16:
            return BF16, shape[1], torch.empty(shape, dtype=torch.bfloat16, device=device)
        raise MgnError(ERR_ARG, f"out is float32 or bfloat16, not {dtype}")
    t, ld = _row_type(out, "out"), _row_ld(out, "out", shape)
    if dtype is not None and out.dtype != dtype:
        raise MgnError(ERR_ARG, f"out must be {dtype}, got {out.dtype}")
    if out.device != device:
        raise MgnError(ERR_ARG, f"out is on {out.device}, expected {device}")
    return t, ld, out


def mgn_matmul4(a, b, bias=None, act="none", aux=None, out=None, dtype=None, accumulate=False, stream=None):
    """act(a b^T + bias) of two Mat4 (see include/mgn.h): [a.rows][b.rows] in
    float32 or bfloat16 (dtype, default float32; out: written, or added to
    with accumulate)."""
    if stream is not None:
        return _elsewhere(mgn_matmul4, dict(locals()))
    if not isinstance(a, Mat4) or not isinstance(b, Mat4):
        raise MgnError(ERR_ARG, "a and b must be Mat4")
    if a.cols != b.cols:
        raise MgnError(ERR_SHAPE, f"a has {a.cols} columns, b {b.cols}")
    if act not in ACTS:
        raise MgnError(ERR_ARG, f"unknown act {act!r}")
    dev, m, n = a.q.device, a.rows, b.rows
    if b.q.device != dev:
        raise MgnError(ERR_ARG, f"b is on {b.q.device}, expected {dev}")
    if out is None and accumulate:
        raise MgnError(ERR_ARG, "accumulate needs an out to add to")
    ct, ldc, out = _result(out, dtype, (m, n), dev)
    ep = None
    if bias is not None or act != "none" or accumulate:
        ep = Epilogue(bias=_vector(bias, "bias", n, dev), act=ACTS[act], accumulate=1 if accumulate else 0)
    if act == "relu_grad":
        ep.aux_type, ep.ldaux = _row_type(aux, "aux"), _row_ld(aux, "aux", (m, n))
        if aux.device != dev:
            raise MgnError(ERR_ARG, f"aux is on {aux.device}, expected {dev}")
        ep.aux = aux.data_ptr()
    elif aux is not None:
        raise MgnError(ERR_ARG, "aux is for relu_grad only")
    if m == 0 or n == 0:
        return out
    L = lib()
    need = C.c_size_t()
    _check(L.mgn_matmul4_workspace(m, n, a.cols, C.byref(need)))
    ws = _scratch(need.value, dev)
    _run(dev, L.mgn_matmul4,
         (C.byref(a.struct), C.byref(b.struct), None if ep is None else C.byref(ep), ct, out.data_ptr(), ldc, _at(ws),
          need.value))
    return out


def _group_norm(x, groups, gamma, beta, act, samples, sample_ptr, eps):
    xt = _row_type(x, "x")
    rows, cols = x.shape
    dev = x.device
    if act not in GROUP_ACTS:
        raise MgnError(ERR_ARG, f"unknown act {act!r}")
    if not 1 <= cols <= NORM_MAX_COLS:  # here: the struct's fields hold 32 bits of these
        raise MgnError(ERR_SHAPE, f"{cols} columns (1 to {NORM_MAX_COLS})")
    groups = int(groups)
    if groups < 1 or cols % groups != 0:
        raise MgnError(ERR_ARG, f"{groups} groups do not divide {cols} columns")
    if sample_ptr is None:
        n = 1 if samples is None else int(samples)
    else:
        torch = _torch()
        if not isinstance(sample_ptr, torch.Tensor) or sample_ptr.dim() != 1 or sample_ptr.numel() < 1:
            raise MgnError(ERR_ARG, "sample_ptr must be a tensor of one number more than there are samples")
        n = sample_ptr.numel() - 1
        if samples is not None and samples != n:
            raise MgnError(ERR_ARG, f"sample_ptr is of {n} samples, not {samples}")
        _dptr(sample_ptr, torch.int32, (n + 1,), "sample_ptr")
        if sample_ptr.device != dev:
            raise MgnError(ERR_ARG, f"sample_ptr is on {sample_ptr.device}, expected {dev}")
    return CGroupNorm(rows, cols, groups, xt, GROUP_ACTS[act], eps, _vector(gamma, "gamma", cols, dev),
                      _vector(beta, "beta", cols, dev), _at(sample_ptr), n)


def mgn_group_norm_forward(x, groups, gamma=None, beta=None, act="none", samples=None, sample_ptr=None, eps=1e-5,
                           save=False, y=None, stream=None):
    """y = act(gamma xhat + beta), xhat being x normed over each sample's rows and
    each of the groups of columns (see include/mgn.h).  Samples: as many runs of
    equal length (default 1), or the runs of sample_ptr (int32, one number more
    than there are samples).  Returns (y, stats): stats None without save.  y
    may be x.  Rows outside of sample_ptr's are not written: a y that is not given
    holds any bits there."""
    if stream is not None:
        return _elsewhere(mgn_group_norm_forward, dict(locals()))
    torch = _torch()
    op = _group_norm(x, groups, gamma, beta, act, samples, sample_ptr, eps)
    shape, dev = tuple(x.shape), x.device
    need = C.c_size_t()
    _check(lib().mgn_group_norm_workspace(C.byref(op), 0, C.byref(need)))
    y, yr = _new_rows(shape, x.dtype, dev) if y is None else (y, _as_rows(y, "y", shape, x.dtype, dev))
    stats = torch.empty((op.n_samples, op.groups, 2), dtype=torch.float32, device=dev) if save else None
    ws = _scratch(need.value, dev)
    _run(dev, lib().mgn_group_norm_forward,
         (C.byref(op), Rows(x.data_ptr(), _row_ld(x, "x")), yr, _at(stats), _at(ws), need.value))
    return y, stats


GroupNormGrads = collections.namedtuple("GroupNormGrads", "dx dgamma dbeta")


def mgn_group_norm_backward(x, stats, dy, groups, gamma=None, beta=None, act="none", samples=None, sample_ptr=None,
                            eps=1e-5, dx=None, grads=None, stream=None):
    """Reverse of mgn_group_norm_forward (see include/mgn.h) from its input and
    stats.  Returns GroupNormGrads; dgamma and dbeta are those of the parameters
    that were given, new tensors, or those of grads (a GroupNormGrads of an
    earlier call) added to.  dx may be dy or x.  Rows of dx outside of
    sample_ptr's are not written."""
    if stream is not None:
        return _elsewhere(mgn_group_norm_backward, dict(locals()))
    torch = _torch()
    op = _group_norm(x, groups, gamma, beta, act, samples, sample_ptr, eps)
    shape, dev = tuple(x.shape), x.device
    need = C.c_size_t()
    _check(lib().mgn_group_norm_workspace(C.byref(op), 1, C.byref(need)))
    dx, dxr = _new_rows(shape, x.dtype, dev) if dx is None else (dx, _as_rows(dx, "dx", shape, x.dtype, dev))
    if not isinstance(stats, torch.Tensor) or tuple(stats.shape) != (op.n_samples, op.groups, 2):
        raise MgnError(ERR_ARG, "stats must be the forward's, of shape (samples, groups, 2)")
    _vector(stats, "stats", stats.numel(), dev)
    if dy is None:
        raise MgnError(ERR_ARG, "dy is needed")
    dyr = _as_rows(dy, "dy", shape, x.dtype, dev)
    out = {}
    for name, p in (("dgamma", gamma), ("dbeta", beta)):
        g = getattr(grads, name) if grads is not None else None
        if p is None:
            if g is not None:
                raise MgnError(ERR_ARG, f"{name} without its parameter")
        elif grads is None:
            g = torch.empty(p.shape, dtype=torch.float32, device=dev)
        elif g is not None:
            _vector(g, name, p.numel(), dev)
        out[name] = g
    ws = _scratch(need.value, dev)
    _run(dev, lib().mgn_group_norm_backward,
         (C.byref(op), Rows(x.data_ptr(), _row_ld(x, "x")), stats.data_ptr(), dyr, dxr, _at(out["dgamma"]),
          _at(out["dbeta"]), 0 if grads is None else 1, _at(ws), need.value))
    return GroupNormGrads(dx, **out)


class TensorList:
    """The list of gradients that mgn_grad_norm and mgn_grad_clip take: contiguous
    float32 or bfloat16 tensors of one device and any sizes, and, for clipping,
    the places of the clipped ones, as many tensors of the same sizes (out;
    None: the gradients themselves).  A program makes it once and keeps it; it
    keeps its tensors, whose values may change but not their places.  Making it copies
    its table to the device and waits for that (75 us for 6 tensors, 1.2 ms for 290 of 300 M
    elements), so not while a graph is captured; where every step's gradients are new
    tensors, every step pays for it."""

    def __init__(self, tensors, out=None):
        torch = _torch()
        self._given, self._out = list(tensors), None if out is None else list(out)
        if not self._given:
            raise MgnError(ERR_ARG, "a list of no tensors")
        places = self._given if self._out is None else self._out
        if len(places) != len(self._given):
            raise MgnError(ERR_ARG, f"{len(places)} places for {len(self._given)} gradients")
        types = {torch.float32: FP32, torch.bfloat16: BF16}
        self.device = None
        table = (CTensor * len(places))()
        for i, (t, o) in enumerate(zip(self._given, places)):
            for v in (t, o):
                if not isinstance(v, torch.Tensor) or not v.is_cuda or v.dtype not in types or not v.is_contiguous():
                    raise MgnError(ERR_ARG, f"tensor {i} must be contiguous, float32 or bfloat16, on the device")
                if self.device is None:
                    self.device = v.device
                if v.device != self.device:
                    raise MgnError(ERR_ARG, f"tensor {i} is on {v.device}, expected {self.device}")
            if t.numel() != o.numel():
                raise MgnError(ERR_ARG, f"tensor {i}: a place of {o.numel()} elements for {t.numel()}")
            table[i] = CTensor(t.data_ptr(), o.data_ptr(), t.numel(), types[t.dtype], types[o.dtype])
        n = C.c_int64()
        _check(lib().mgn_grad_pieces(table, len(places), None, C.byref(n)))
        pieces = (CPiece * n.value)()
        _check(lib().mgn_grad_pieces(table, len(places), pieces, C.byref(n)))
        self.n = n.value
        # on the device once it is made, whatever stream uses it first
        self.pieces = torch.frombuffer(bytearray(pieces), dtype=torch.uint8).to(self.device) if self.n else None
        torch.cuda.current_stream(self.device).synchronize()
        need = C.c_size_t()
        _check(lib().mgn_grad_norm_workspace(self.n, C.byref(need)))
        self.ws_bytes = need.value

    def tensors(self):
        return self._given + (self._out or []) + ([self.pieces] if self.n else [])


def _list(tensors):
    if not isinstance(tensors, TensorList):
        raise MgnError(ERR_ARG, "a TensorList is needed")
    return tensors.device


def mgn_grad_norm(tensors, stream=None):
    """The norm over all elements of a TensorList, a float32 tensor of one."""
    if stream is not None:
        return _elsewhere(mgn_grad_norm, dict(locals()))
    dev = _list(tensors)
    norm = _torch().empty(1, dtype=_torch().float32, device=dev)
    ws = _scratch(tensors.ws_bytes, dev)
    _run(dev, lib().mgn_grad_norm, (_at(tensors.pieces), tensors.n, norm.data_ptr(), _at(ws), tensors.ws_bytes))
    return norm


def mgn_grad_clip(tensors, max_norm, norm=None, stream=None):
    """Scales a TensorList's gradients, into their places, by min(1, max_norm /
    norm) (see include/mgn.h).  norm: of all of them, or the given float32 tensor
    of one element (say of a norm over several processes).  Returns the norm.  One
    that is not finite leaves the values as they are."""
    if stream is not None:
        return _elsewhere(mgn_grad_clip, dict(locals()))
    dev = _list(tensors)
    given = norm is not None
    if given:
        _vector(norm, "norm", 1, dev)
    else:
        norm = _torch().empty(1, dtype=_torch().float32, device=dev)
    need = 0 if given else tensors.ws_bytes
    ws = _scratch(need, dev)
    _run(dev, lib().mgn_grad_clip,
         (_at(tensors.pieces), tensors.n, float(max_norm), norm.data_ptr(), 1 if given else 0, _at(ws), need))
    return norm


# short aliases
forward = mgn_forward
backward = mgn_backward
integrate_step = mgn_integrate_step
