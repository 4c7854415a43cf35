"""Python binding of libcardan.so (argument marshalling only).

Every function here checks dtypes, shapes, devices and contiguity of torch
tensors, turns them into raw device pointers and calls the C ABI declared in
``include/cardan.h``; all arithmetic runs in the library's HIP kernels.
Importing this module loads the library and raises ``ImportError`` when it is
missing: there is no fallback path.

bf16 arrays are passed as ``torch.bfloat16`` tensors (their storage is the
raw bf16 bit pattern the ABI expects).
"""

from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
# CARDAN_LIB names another build of the library (the tests' sanitizer build)
LIB_PATH = os.environ.get("CARDAN_LIB") or os.path.join(HERE, "libcardan.so")

LAYER_FIELDS = (
    "router_w", "router_bias", "cb_gate", "cb_up", "cb_down",
    "codes_gate", "codes_up", "codes_down", "U_gate", "U_up",
    "V_gate", "V_up", "A_down", "B_down",
)

DENSE_LAYER_FIELDS = ("router_w", "router_bias", "W_gate", "W_up", "W_down")

KERNEL_KINDS = ("route", "expert", "rmsnorm")

ERRORS = {-1: "NULL_PTR", -2: "BAD_SHAPE", -3: "UNSUPPORTED", -4: "WORKSPACE", -5: "HIP",
          -6: "ALIGN"}


class CardanError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"cardan error {code} ({ERRORS.get(code, '?')}): {msg}")
        self.code = code


class Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("H", "I", "E", "top_k", "d", "K", "r")]


class FfnShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("H", "I", "E", "act")]


class FfnWeightsStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("W_gate", "W_up", "W_down")]


class Routing(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("E", "top_k", "score", "renorm", "groups", "top_groups",
                                              "group_best")] + [("scale", ctypes.c_float)]


class AdamwTensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")]
    _fields_ += [("n", ctypes.c_int64)]


class Adamw(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("param_type", "grad_type", "state_bits", "step")]
    _fields_ += [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")]
    _fields_ += [(n, ctypes.c_void_p) for n in ("step_device", "lr_device", "grad_scale")]


class LayerStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in LAYER_FIELDS]


class DenseLayerStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in DENSE_LAYER_FIELDS]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing; build it with `python -m paper_2609_21137_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    sp = ctypes.POINTER(Shape)
    lp = ctypes.POINTER(LayerStruct)
    dp = ctypes.POINTER(DenseLayerStruct)
    fp = ctypes.POINTER(FfnShape)
    wp = ctypes.POINTER(FfnWeightsStruct)
    rp = ctypes.POINTER(Routing)
    i64, f32 = ctypes.c_int64, ctypes.c_float
    sig = {
        "cardan_abi_version": ([], ctypes.c_int),
        "cardan_last_error": ([], ctypes.c_char_p),
        "cardan_workspace_bytes": ([sp, i32, ctypes.POINTER(sz)], ctypes.c_int),
        "cardan_route_topk": ([sp, i32, vp, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_shared_proj": ([sp, i32, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_vq_lr_expert_ffn": ([sp, i32, vp, vp, vp, vp, lp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_moe_layer": ([sp, i32, vp, lp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_moe_layer_noalloc": ([sp, i32, vp, lp, vp, vp, vp, vp], ctypes.c_int),
        "cardan_moe_layer_relu2": ([sp, i32, vp, lp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_moe_decode_step": ([sp, i32, i32, vp, lp, ctypes.c_float, vp, vp, vp, vp, vp, sz, vp],
                                   ctypes.c_int),
        "cardan_moe_layer_dense_down": ([sp, i32, vp, lp, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_dense_moe_layer": ([sp, i32, vp, dp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_dense_moe_layer_relu2": ([sp, i32, vp, dp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_rmsnorm_bf16": ([i32, i32, vp, ctypes.c_float, vp, vp], ctypes.c_int),
        "cardan_ffn_workspace_bytes": ([fp, i32, ctypes.POINTER(sz)], ctypes.c_int),
        "cardan_ffn_forward": ([fp, i32, vp, vp, wp, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_ffn_backward": ([fp, i32, vp, vp, vp, wp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_distill_loss": ([i32, i32, i32, i32, vp, i64, vp, vp, vp, f32, f32, vp, vp, vp, i64, vp],
                                ctypes.c_int),
        "cardan_route_rows_workspace_bytes": ([rp, i32, ctypes.POINTER(sz)], ctypes.c_int),
        "cardan_route_rows": ([rp, i32, i32, vp, i64, vp, vp, vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "cardan_route_rows_backward": ([rp, i32, i32, vp, i64, vp, vp, vp, i64, vp], ctypes.c_int),
        "cardan_dispatch_rows": ([i32, i32, i32, i32, vp, vp, vp, vp], ctypes.c_int),
        "cardan_combine_rows": ([i32, i32, i32, i32, vp, vp, vp, i32, vp, vp], ctypes.c_int),
        "cardan_combine_rows_backward": ([i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp], ctypes.c_int),
        "cardan_adamw_step": ([ctypes.POINTER(Adamw), i32, vp, vp], ctypes.c_int),
        "cardan_profile_begin": ([i32], ctypes.c_int),
        "cardan_profile_end": ([ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)], ctypes.c_int),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    return lib


_lib = _load()

EXPORTED = (
    "cardan_abi_version", "cardan_last_error", "cardan_workspace_bytes", "cardan_route_topk",
    "cardan_shared_proj", "cardan_vq_lr_expert_ffn", "cardan_moe_layer", "cardan_moe_layer_noalloc",
    "cardan_moe_decode_step", "cardan_moe_layer_relu2",
    "cardan_moe_layer_dense_down", "cardan_dense_moe_layer", "cardan_dense_moe_layer_relu2",
    "cardan_rmsnorm_bf16",
    "cardan_ffn_workspace_bytes", "cardan_ffn_forward", "cardan_ffn_backward",
    "cardan_distill_loss",
    "cardan_route_rows_workspace_bytes", "cardan_route_rows", "cardan_route_rows_backward",
    "cardan_dispatch_rows", "cardan_combine_rows", "cardan_combine_rows_backward",
    "cardan_adamw_step",
    "cardan_profile_begin", "cardan_profile_end",
)


def lib():
    return _lib


def _check(rc: int):
    if rc != 0:
        raise CardanError(rc, _lib.cardan_last_error().decode())


def _fits(*counts):
    """Refuses what the library's 32-bit counts do not hold (ctypes keeps the low bits)."""
    for n in counts:
        if not -(1 << 31) <= n < 1 << 31:
            raise ValueError(f"{n} does not fit 32 bits")


def abi_version() -> int:
    return _lib.cardan_abi_version()


def make_shape(H, I, E, top_k, d, K, r) -> Shape:
    return Shape(H, I, E, top_k, d, K, r)


def shape_of(w) -> Shape:
    """Shape struct of a workload from ``configs``."""
    return Shape(w.H, w.I, w.E, w.top_k, w.d, w.K, w.r)


def workspace_bytes(shape: Shape, B: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.cardan_workspace_bytes(ctypes.byref(shape), B, ctypes.byref(out)))
    return out.value


def workspace_status(ws: torch.Tensor) -> int:
    """Number of in-kernel waits that gave up (0 unless an invariant broke)."""
    return int(ws[:4].view(torch.int32).item())


def new_workspace(shape: Shape, B: int, device="cuda") -> torch.Tensor:
    """Zero-filled workspace (the library needs zeros before the first use)."""
    return torch.zeros(workspace_bytes(shape, B), dtype=torch.uint8, device=device)


def _ptr(t, dtype, name, shape=None, optional=False):
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must live on a GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return ctypes.c_void_p(t.data_ptr())


def _stream(dev) -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)


def bf16_tensor(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """Raw bf16 bit patterns (uint16) to a bfloat16 tensor on ``device``."""
    arr = np.ascontiguousarray(bits, dtype=np.uint16).view(np.int16)
    return torch.from_numpy(arr).view(torch.bfloat16).to(device)


def bf16_bits(t: torch.Tensor) -> np.ndarray:
    """bfloat16 tensor back to raw uint16 bit patterns on the host."""
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


@dataclass
class DeviceLayer:
    """One layer's weights as device tensors (field names of ``cardan_layer``).

    ``routing``: the arguments of ``route_rows`` that the layer was trained to
    route by (the key of that name of a layer dict, ``fit.distill_layer``). Such
    a layer runs by ``route_rows(logits, top_k, **layer.routing)`` and
    ``vq_lr_expert_ffn``; calls that route by themselves, by the softmax over the
    kept logits, refuse it."""
    tensors: dict
    routing: dict | None = None

    @classmethod
    def from_numpy(cls, L: dict, device="cuda") -> "DeviceLayer":
        T, routing = {}, L.get("routing")
        if routing is not None and routing.get("bias") is not None:
            routing = {**routing, "bias": torch.as_tensor(routing["bias"], dtype=torch.float32).to(device)}
        for key in LAYER_FIELDS:
            v = L.get(key)
            if v is None:
                T[key] = None
            elif key == "U_up" and L.get("U_up") is L.get("U_gate"):
                T[key] = T["U_gate"]
            elif v.dtype == np.uint16:
                T[key] = bf16_tensor(v, device)
            elif v.dtype == np.uint8:
                T[key] = torch.from_numpy(np.ascontiguousarray(v)).to(device)
            else:
                T[key] = torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).to(device)
        return cls(T, routing)

    def struct(self, routed: bool = False) -> LayerStruct:
        """``routed``: the call is given its routing."""
        if self.routing and not routed:
            raise ValueError("this layer has a routing of its own: run it by route_rows and vq_lr_expert_ffn")
        vals = []
        for key in LAYER_FIELDS:
            t = self.tensors.get(key)
            if t is None:
                vals.append(None)
            else:
                if not t.is_contiguous() or t.device.type != "cuda":
                    raise ValueError(f"{key} must be a contiguous GPU tensor")
                vals.append(t.data_ptr())
        return LayerStruct(*vals)

    def nbytes(self) -> int:
        seen, tot = set(), 0
        for t in self.tensors.values():
            if t is not None and t.data_ptr() not in seen:
                seen.add(t.data_ptr())
                tot += t.numel() * t.element_size()
        return tot


def route_topk(shape: Shape, x, router_w, router_bias=None, ws=None):
    """Router logits, top-k (descending, ties to the lower index) and softmax
    gating. Returns ``(topk_idx int32 [B, k], topk_w float32 [B, k])``."""
    B = x.shape[0]
    dev = x.device
    idx = torch.empty((B, shape.top_k), dtype=torch.int32, device=dev)
    w = torch.empty((B, shape.top_k), dtype=torch.float32, device=dev)
    if ws is None:
        ws = new_workspace(shape, B, dev)
    _check(_lib.cardan_route_topk(
        ctypes.byref(shape), B, _ptr(x, torch.bfloat16, "x", (B, shape.H)),
        _ptr(router_w, torch.bfloat16, "router_w", (shape.H, shape.E)),
        _ptr(router_bias, torch.float32, "router_bias", (shape.E,), optional=True),
        _ptr(idx, torch.int32, "topk_idx"), _ptr(w, torch.float32, "topk_w"),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(dev)))
    return idx, w


def shared_proj(shape: Shape, x, U_gate, U_up=None, ws=None):
    """Shared projections ``z[2, B, r]`` (gate, up) of every token."""
    B = x.shape[0]
    dev = x.device
    U_up = U_gate if U_up is None else U_up
    z = torch.empty((2, B, shape.r), dtype=torch.float32, device=dev)
    if ws is None:
        ws = new_workspace(shape, B, dev)
    _check(_lib.cardan_shared_proj(
        ctypes.byref(shape), B, _ptr(x, torch.bfloat16, "x", (B, shape.H)),
        _ptr(U_gate, torch.bfloat16, "U_gate", (shape.H, shape.r)),
        _ptr(U_up, torch.bfloat16, "U_up", (shape.H, shape.r)),
        _ptr(z, torch.float32, "z"), _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(dev)))
    return z


def vq_lr_expert_ffn(shape: Shape, x, topk_idx, topk_w, z, layer: DeviceLayer, ws=None, out=None):
    """Grouped expert computation and weighted combine for a given routing."""
    B = x.shape[0]
    dev = x.device
    y = out if out is not None else torch.empty((B, shape.H), dtype=torch.float32, device=dev)
    if ws is None:
        ws = new_workspace(shape, B, dev)
    st = layer.struct(routed=True)
    _check(_lib.cardan_vq_lr_expert_ffn(
        ctypes.byref(shape), B, _ptr(x, torch.bfloat16, "x", (B, shape.H)),
        _ptr(topk_idx, torch.int32, "topk_idx", (B, shape.top_k)),
        _ptr(topk_w, torch.float32, "topk_w", (B, shape.top_k)),
        _ptr(z, torch.float32, "z", (2, B, shape.r), optional=shape.r == 0),
        ctypes.byref(st), _ptr(y, torch.float32, "y", (B, shape.H)),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(dev)))
    return y


def moe_layer(shape: Shape, x, layer: DeviceLayer, ws=None, out=None, idx=None, w=None):
    """The whole layer. Returns ``(y float32 [B, H], topk_idx, topk_w)``."""
    B = x.shape[0]
    dev = x.device
    y = out if out is not None else torch.empty((B, shape.H), dtype=torch.float32, device=dev)
    idx = idx if idx is not None else torch.empty((B, shape.top_k), dtype=torch.int32, device=dev)
    w = w if w is not None else torch.empty((B, shape.top_k), dtype=torch.float32, device=dev)
    if ws is None:
        ws = new_workspace(shape, B, dev)
    st = layer.struct()
    _check(_lib.cardan_moe_layer(
        ctypes.byref(shape), B, _ptr(x, torch.bfloat16, "x", (B, shape.H)), ctypes.byref(st),
        _ptr(y, torch.float32, "y", (B, shape.H)),
        _ptr(idx, torch.int32, "topk_idx", (B, shape.top_k)),
        _ptr(w, torch.float32, "topk_w", (B, shape.top_k)),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(dev)))
    return y, idx, w


def moe_layer_relu2(shape: Shape, x, layer: DeviceLayer, ws=None, out=None, idx=None, w=None):
    """The whole layer with up-only squared-ReLU experts (the layer's gate
    fields are not read). Returns ``(y float32 [B, H], topk_idx, topk_w)``."""
    B = x.shape[0]
    dev = x.device
    y, idx, w = _outputs(shape, x, out, idx, w)
    if ws is None:
        ws = new_workspace(shape, B, dev)
    st = layer.struct()
    _check(_lib.cardan_moe_layer_relu2(
        ctypes.byref(shape), B, _ptr(x, torch.bfloat16, "x", (B, shape.H)), ctypes.byref(st),
        _ptr(y, torch.float32, "y", (B, shape.H)),
        _ptr(idx, torch.int32, "topk_idx", (B, shape.top_k)),
        _ptr(w, torch.float32, "topk_w", (B, shape.top_k)),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(dev)))
    return y, idx, w


def moe_decode_step(shape: Shape, x0, layers, eps: float = 1e-6, ws=None, out=None, x_norm=None,
                    idx=None, w=None):
    """``len(layers)`` stacked layers, each output RMS-normalised (bf16) into
    the next layer's input. Returns ``(y [B, H] of the last layer,
    topk_idx [L, B, k], topk_w [L, B, k])``; ``x_norm`` (optional,
    ``[L - 1, B, H]`` bf16) receives the normalised inputs of layers 1..L-1."""
    B = x0.shape[0]
    L = len(layers)
    dev = x0.device
    y = out if out is not None else torch.empty((B, shape.H), dtype=torch.float32, device=dev)
    idx = idx if idx is not None else torch.empty((L, B, shape.top_k), dtype=torch.int32, device=dev)
    w = w if w is not None else torch.empty((L, B, shape.top_k), dtype=torch.float32, device=dev)
    if ws is None:
        ws = new_workspace(shape, B, dev)
    structs = (LayerStruct * L)(*[dl.struct() for dl in layers])
    xn = (_ptr(x_norm, torch.bfloat16, "x_norm", (L - 1, B, shape.H)) if x_norm is not None and L > 1
          else None)
    _check(_lib.cardan_moe_decode_step(
        ctypes.byref(shape), B, L, _ptr(x0, torch.bfloat16, "x0", (B, shape.H)), structs,
        ctypes.c_float(eps), _ptr(y, torch.float32, "y", (B, shape.H)), xn,
        _ptr(idx, torch.int32, "topk_idx", (L, B, shape.top_k)),
        _ptr(w, torch.float32, "topk_w", (L, B, shape.top_k)),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(dev)))
    return y, idx, w


def moe_layer_noalloc(shape: Shape, x, layer: DeviceLayer, out=None, idx=None, w=None):
    """The whole layer on the library's own scratch array (no workspace, no
    device allocation inside the call). Returns ``(y, topk_idx, topk_w)``."""
    B = x.shape[0]
    dev = x.device
    y, idx, w = _outputs(shape, x, out, idx, w)
    st = layer.struct()
    _check(_lib.cardan_moe_layer_noalloc(
        ctypes.byref(shape), B, _ptr(x, torch.bfloat16, "x", (B, shape.H)), ctypes.byref(st),
        _ptr(y, torch.float32, "y", (B, shape.H)),
        _ptr(idx, torch.int32, "topk_idx", (B, shape.top_k)),
        _ptr(w, torch.float32, "topk_w", (B, shape.top_k)), _stream(dev)))
    return y, idx, w


def _outputs(shape: Shape, x, out, idx, w):
    B = x.shape[0]
    dev = x.device
    y = out if out is not None else torch.empty((B, shape.H), dtype=torch.float32, device=dev)
    idx = idx if idx is not None else torch.empty((B, shape.top_k), dtype=torch.int32, device=dev)
    w = w if w is not None else torch.empty((B, shape.top_k), dtype=torch.float32, device=dev)
    return y, idx, w


def moe_layer_dense_down(shape: Shape, x, layer: DeviceLayer, W_down, ws=None, out=None, idx=None,
                         w=None):
    """The layer with compressed gate/up and a dense bf16 ``W_down [E, I, H]``
    (the layer's compressed down fields are not read). Returns
    ``(y float32 [B, H], topk_idx, topk_w)``."""
    B = x.shape[0]
    dev = x.device
    y, idx, w = _outputs(shape, x, out, idx, w)
    if ws is None:
        ws = new_workspace(shape, B, dev)
    st = layer.struct()
    _check(_lib.cardan_moe_layer_dense_down(
        ctypes.byref(shape), B, _ptr(x, torch.bfloat16, "x", (B, shape.H)), ctypes.byref(st),
        _ptr(W_down, torch.bfloat16, "W_down", (shape.E, shape.I, shape.H)),
        _ptr(y, torch.float32, "y", (B, shape.H)),
        _ptr(idx, torch.int32, "topk_idx", (B, shape.top_k)),
        _ptr(w, torch.float32, "topk_w", (B, shape.top_k)),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(dev)))
    return y, idx, w


@dataclass
class DenseLayer:
    """An uncompressed layer's device tensors (fields of ``cardan_dense_layer``):
    router_w [H, E] bf16, router_bias [E] f32 or None, W_gate / W_up [E, H, I]
    and W_down [E, I, H] bf16."""
    tensors: dict

    def struct(self, shape: Shape, up_only: bool = False) -> DenseLayerStruct:
        H, I, E = shape.H, shape.I, shape.E
        want = {"router_w": (torch.bfloat16, (H, E)), "router_bias": (torch.float32, (E,)),
                "W_gate": (torch.bfloat16, (E, H, I)), "W_up": (torch.bfloat16, (E, H, I)),
                "W_down": (torch.bfloat16, (E, I, H))}
        vals = []
        for key in DENSE_LAYER_FIELDS:
            dt, shp = want[key]
            optional = key == "router_bias" or (up_only and key == "W_gate")
            p = _ptr(self.tensors.get(key), dt, key, shp, optional=optional)
            vals.append(None if p is None else p.value)
        return DenseLayerStruct(*vals)


def dense_moe_layer(shape: Shape, x, layer: DenseLayer, ws=None, out=None, idx=None, w=None,
                    relu2: bool = False):
    """The uncompressed MoE layer (only H, I, E, top_k of ``shape`` are read);
    ``relu2``: up-only squared-ReLU experts (``W_gate`` not read).
    Returns ``(y float32 [B, H], topk_idx, topk_w)``."""
    B = x.shape[0]
    dev = x.device
    y, idx, w = _outputs(shape, x, out, idx, w)
    if ws is None:
        ws = new_workspace(shape, B, dev)
    st = layer.struct(shape, up_only=relu2)
    fn = _lib.cardan_dense_moe_layer_relu2 if relu2 else _lib.cardan_dense_moe_layer
    _check(fn(
        ctypes.byref(shape), B, _ptr(x, torch.bfloat16, "x", (B, shape.H)), ctypes.byref(st),
        _ptr(y, torch.float32, "y", (B, shape.H)),
        _ptr(idx, torch.int32, "topk_idx", (B, shape.top_k)),
        _ptr(w, torch.float32, "topk_w", (B, shape.top_k)),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(dev)))
    return y, idx, w


def rmsnorm_bf16(y, eps: float = 1e-6, out=None):
    """``bf16_rne(y / sqrt(mean(y^2) + eps))`` per row, as a bfloat16 tensor."""
    B, H = y.shape
    xn = out if out is not None else torch.empty((B, H), dtype=torch.bfloat16, device=y.device)
    _check(_lib.cardan_rmsnorm_bf16(B, H, _ptr(y, torch.float32, "y", (B, H)), eps,
                                    _ptr(xn, torch.bfloat16, "x_next", (B, H)), _stream(y.device)))
    return xn


# ---------------------------------------------------------------------------
# training: the feed-forward block and the distillation loss
# ---------------------------------------------------------------------------
FFN_ACTS = {"silu_glu": 0, "relu2_up": 1}


def _arg(t, dtype, name, shape, dev, optional=False):
    """``_ptr`` for the calls whose whole time is a few microseconds: one pass
    over a tensor's properties, with ``_ptr``'s messages where one does not fit,
    and the tensor must live on the call's device. Returns the address."""
    if t is None and optional:
        return None
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_contiguous()
            and t.device == dev and t.is_cuda):
        return t.data_ptr()
    _ptr(t, dtype, name, shape)
    raise ValueError(f"{name} is on {t.device}, expected {dev}")


class _Device:
    """The current stream of a tensor's device, which is made current for the call."""
    __slots__ = ("index", "was")

    def __init__(self, dev):
        self.index = dev.index

    def __enter__(self):
        self.was = torch.cuda.current_device()
        if self.was != self.index:
            torch.cuda.set_device(self.index)
        return torch._C._cuda_getCurrentRawStream(self.index)

    def __exit__(self, *exc):
        if self.was != self.index:
            torch.cuda.set_device(self.was)


def ffn_shape(H, I, E=1, act="silu_glu") -> FfnShape:
    if act not in FFN_ACTS:
        raise ValueError(f"unknown activation {act!r}")
    return FfnShape(H, I, E, FFN_ACTS[act])


def ffn_workspace_bytes(shape: FfnShape, N: int) -> int:
    """Bytes of workspace of a forward or backward call over up to N rows (no
    zero fill needed; nothing is kept in it between calls)."""
    _fits(N)
    out = ctypes.c_size_t(0)
    _check(_lib.cardan_ffn_workspace_bytes(ctypes.byref(shape), N, ctypes.byref(out)))
    return out.value


@functools.lru_cache(maxsize=256)
def _ffn_bytes(H, I, E, act, N):
    return ffn_workspace_bytes(ffn_shape(H, I, E, act), N)


def _ffn_call(x, W_gate, W_up, W_down, offsets, act, ws):
    """Shape, weights, offsets and workspace of a call, as the ABI takes them."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x must be a [N, H] tensor")
    if not isinstance(W_up, torch.Tensor) or W_up.dim() not in (2, 3):
        raise ValueError("W_up must be a [H, I] or [E, H, I] tensor")
    N, H = x.shape
    up_shape = W_up.shape
    I = up_shape[-1]
    many = len(up_shape) == 3
    E = up_shape[0] if many else 1
    shape = ffn_shape(H, I, E, act)
    in_shape, out_shape = ((E, H, I), (E, I, H)) if many else ((H, I), (I, H))
    up_only = act == "relu2_up"
    if up_only and W_gate is not None:
        raise ValueError("up-only experts have no W_gate")
    dev, bf = x.device, torch.bfloat16
    weights = FfnWeightsStruct(_arg(W_gate, bf, "W_gate", in_shape, dev, up_only),
                               _arg(W_up, bf, "W_up", in_shape, dev), _arg(W_down, bf, "W_down", out_shape, dev))
    off = _arg(offsets, torch.int32, "offsets", (E + 1,), dev, E == 1)
    if ws is None:
        ws = torch.empty(_ffn_bytes(H, I, E, act, N), dtype=torch.uint8, device=dev)
    elif ws.dtype is not torch.uint8 or ws.device != dev or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous uint8 tensor on {dev}")
    return shape, N, weights, off, ws


def ffn_forward(x, W_gate, W_up, W_down, offsets=None, act: str = "silu_glu", save: bool = False,
                ws=None, out=None, saved=None):
    """Feed-forward block of dense bf16 weights: ``y = h W_down`` with
    ``h = silu(x W_gate) * (x W_up)``, or ``max(x W_up, 0)^2`` for
    ``act="relu2_up"`` (``W_gate=None``).

    ``x [N, H]``; weights ``[H, I]`` / ``[I, H]``, or ``[E, H, I]`` /
    ``[E, I, H]`` with ``offsets`` (int32 ``[E + 1]``): rows
    ``offsets[e]:offsets[e + 1]`` go through expert e. Returns ``y [N, H]``
    (bf16; rows in no group are not written), and with ``save=True`` also the
    activations ``(gate, up, hidden)`` that ``ffn_backward`` reads (float32,
    float32, bf16, ``[N, I]``; ``gate`` is None for up-only experts).
    ``out`` and ``saved`` give the tensors to write.

    The outputs carry no autograd graph, also where an input requires a
    gradient: gradients come from ``ffn_backward``."""
    shape, N, weights, off, ws = _ffn_call(x, W_gate, W_up, W_down, offsets, act, ws)
    H, I, dev = shape.H, shape.I, x.device
    bf, f32 = torch.bfloat16, torch.float32
    gated = act == "silu_glu"
    y = out if out is not None else torch.empty((N, H), dtype=bf, device=dev)
    keep = save or saved is not None
    g = u = h = None
    if saved is not None:
        g, u, h = saved
    elif save:
        g = torch.empty((N, I), dtype=f32, device=dev) if gated else None
        u, h = torch.empty((N, I), dtype=f32, device=dev), torch.empty((N, I), dtype=bf, device=dev)
    xp, yp = _arg(x, bf, "x", (N, H), dev), _arg(y, bf, "out", (N, H), dev)
    gp, up, hp = (_arg(g, f32, "gate", (N, I), dev, not gated), _arg(u, f32, "up", (N, I), dev),
                  _arg(h, bf, "hidden", (N, I), dev)) if keep else (None, None, None)
    with _Device(dev) as stream:
        _check(_lib.cardan_ffn_forward(ctypes.byref(shape), N, xp, off, ctypes.byref(weights), yp, gp, up, hp,
                                       ws.data_ptr(), ws.numel(), stream))
    return (y, (g, u, h)) if keep else y


def ffn_backward(dy, x, W_gate, W_up, W_down, saved, offsets=None, act: str = "silu_glu",
                 need_dx: bool = True, need_dw: bool = True, ws=None, out=None):
    """Gradients of ``ffn_forward`` for the upstream gradient ``dy [N, H]``
    (bf16), from the activations ``saved`` by it. Returns ``(dx, dW_gate,
    dW_up, dW_down)`` in bf16, laid out as their inputs (rows in no group of
    dx are not written; weight gradients of a group without rows are zero);
    None where not asked for. ``out`` gives the four tensors to write; nothing
    is added to an input's ``.grad``."""
    shape, N, weights, off, ws = _ffn_call(x, W_gate, W_up, W_down, offsets, act, ws)
    H, I, dev = shape.H, shape.I, x.device
    bf, f32 = torch.bfloat16, torch.float32
    gated = act == "silu_glu"
    if out is not None:
        dx, dWg, dWu, dWd = out
    else:
        dx = torch.empty_like(x) if need_dx else None
        dWg = torch.empty_like(W_gate) if need_dw and gated else None
        dWu, dWd = (torch.empty_like(W_up), torch.empty_like(W_down)) if need_dw else (None, None)
    g, u, h = saved
    args = (_arg(dy, bf, "dy", (N, H), dev), _arg(x, bf, "x", (N, H), dev), off, ctypes.byref(weights),
            _arg(g, f32, "gate", (N, I), dev, not gated), _arg(u, f32, "up", (N, I), dev),
            _arg(h, bf, "hidden", (N, I), dev), _arg(dx, bf, "dx", (N, H), dev, True),
            _arg(dWg, bf, "dW_gate", W_up.shape, dev, True), _arg(dWu, bf, "dW_up", W_up.shape, dev, True),
            _arg(dWd, bf, "dW_down", W_down.shape, dev, True))
    with _Device(dev) as stream:
        _check(_lib.cardan_ffn_backward(ctypes.byref(shape), N, *args, ws.data_ptr(), ws.numel(), stream))
    return dx, dWg, dWu, dWd


def _rows_ptr(t, dtype, name, shape, dev):
    """A [N, V] tensor whose rows are contiguous, as (address, row stride)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype is not dtype or not t.is_cuda or t.device != dev or t.shape != shape:
        raise ValueError(f"{name} must be a tensor of {dtype} and shape {shape} on {dev if dev.type == 'cuda' else 'a GPU'}, "
                         f"got {t.dtype}, {tuple(t.shape)} on {t.device}")
    N, V = shape
    st = t.stride()
    if V > 1 and st[1] != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    ld = st[0] if N > 1 else V
    if ld < V:
        raise ValueError(f"the rows of {name} overlap")
    return t.data_ptr(), ld


_ANY_START = 16  # CARDAN_LOGITS_ANY_START


def distill_loss(logits, teacher, ids, labels=None, temperature: float = 1.0, ce_weight: float = 0.0,
                 row_weight=None, grad: bool = True, out=None, dlogits=None):
    """Distillation loss of student ``logits [N, V]`` (bf16 or float32, rows
    may be padded and start on any element) against a teacher's kept logits ``teacher [N, K]`` (float32)
    at the vocabulary entries ``ids [N, K]`` (int32), and its gradient.

    Returns ``(loss [N, 2], dlogits)``: per row ``kd = T^2 KL(softmax(teacher
    / T) || softmax(logits / T))`` over the teacher's entries and the cross
    entropy of ``labels`` (int32, [N]); ``dlogits`` is the gradient of
    ``sum_n row_weight[n] (kd_n + ce_weight ce_n)`` in the logits' type and
    with rows padded as theirs, or None with ``grad=False``. ``dlogits=logits`` overwrites the
    logits. Ids and labels outside ``[0, V)`` mark absent entries and labels, and a
    teacher's logit of -inf an absent entry. The losses carry no autograd graph,
    also where the logits require a gradient: ``dlogits`` is it."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits must be a [N, V] tensor of bfloat16 or float32")
    N, V = logits.shape
    dev = logits.device
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
        raise ValueError("ids must be a [N, K] tensor")
    K = ids.shape[1]
    _fits(N, V, K)
    dt, f32, i32 = logits.dtype, torch.float32, torch.int32
    lp, ld = _rows_ptr(logits, dt, "logits", (N, V), dev)
    loss = out if out is not None else torch.empty((N, 2), dtype=f32, device=dev)
    if dlogits is None and grad:
        # rows that start as the logits' do (their alignment), as far apart where that is padding
        width, skip = ld if ld <= 2 * V else V, lp % 16 // logits.element_size()
        dlogits = torch.empty(skip + N * width, dtype=dt, device=dev)[skip:].view(N, width)[:, :V]
    gp, dld = _rows_ptr(dlogits, dt, "dlogits", (N, V), dev) if dlogits is not None else (None, 0)
    args = (_arg(teacher, f32, "teacher", (N, K), dev), _arg(ids, i32, "ids", (N, K), dev),
            _arg(labels, i32, "labels", (N,), dev, True), temperature, ce_weight,
            _arg(row_weight, f32, "row_weight", (N,), dev, True), _arg(loss, f32, "out", (N, 2), dev), gp, dld)
    with _Device(dev) as stream:
        _check(_lib.cardan_distill_loss(N, V, K, _ANY_START + (1 if dt is f32 else 0), lp, ld, *args, stream))
    return loss, dlogits


# ---------------------------------------------------------------------------
# training: the router, rows to their experts and back, the optimizer
# ---------------------------------------------------------------------------
SCORES = {"softmax": 0, "sigmoid": 1}
_TYPES = {torch.bfloat16: 0, torch.float32: 1, torch.float64: 2}


@functools.lru_cache(maxsize=256)
def _routing(E, top_k, score, renorm, scale, groups, top_groups, group_best) -> Routing:
    if score not in SCORES:
        raise ValueError(f"unknown score {score!r}")
    _fits(E, top_k, groups, top_groups, group_best)
    return Routing(E, top_k, SCORES[score], int(bool(renorm)), groups, top_groups, group_best, scale)


def route_rows_workspace_bytes(N: int, E: int, top_k: int, score: str = "softmax", renorm: bool = True,
                               scale: float = 1.0, groups: int = 1, top_groups: int = 1, group_best: int = 1) -> int:
    """Bytes of workspace of ``route_rows`` over up to N rows (no zero fill
    needed; nothing is kept in it between calls)."""
    _fits(N)
    out = ctypes.c_size_t(0)
    r = _routing(E, top_k, score, renorm, scale, groups, top_groups, group_best)
    _check(_lib.cardan_route_rows_workspace_bytes(ctypes.byref(r), N, ctypes.byref(out)))
    return out.value


@functools.lru_cache(maxsize=256)
def _route_bytes(E, top_k, N):
    return route_rows_workspace_bytes(N, E, top_k)


def _logit_rows(logits):
    if isinstance(logits, torch.Tensor) and logits.dim() == 2 and logits.is_cuda and logits.is_contiguous():
        kind = _TYPES.get(logits.dtype)
        if kind is not None:
            return logits.data_ptr(), logits.shape[1], kind
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or logits.dtype not in _TYPES:
        raise ValueError("logits must be a [N, E] tensor of bfloat16, float32 or float64")
    lp, ld = _rows_ptr(logits, logits.dtype, "logits", logits.shape, logits.device)
    return lp, ld, _TYPES[logits.dtype]


def route_rows(logits, top_k: int, bias=None, score: str = "softmax", renorm: bool = True, scale: float = 1.0,
               groups: int = 1, top_groups: int = 1, group_best: int = 1, places: bool = True, ws=None, out=None):
    """Routing of rows of any number by their ``logits [N, E]`` (bf16, float32
    or float64; rows may be padded): the ``top_k`` experts of each row and
    their weights.

    ``score``: ``"softmax"`` over all experts or ``"sigmoid"``; ``bias``
    (float32 ``[E]``) takes part in the selection alone; with ``groups`` a row
    chooses among the experts of its ``top_groups`` best groups, which count by
    their best expert or by their best two (``group_best``). The weights are the
    scores, divided by their sum with ``renorm``, times ``scale``. Ties go to
    the lower index; selections of equal scores are decided in float64.

    Returns ``(idx, weight, place, offsets)``: int32 and float32 ``[N, top_k]``,
    and the rows' places in an array grouped by expert (int32 ``[N, top_k]``)
    with its ``offsets`` (int32 ``[E + 1]``), as ``dispatch_rows``,
    ``ffn_forward`` and ``combine_rows`` take them (None, None with
    ``places=False``). An expert whose logit is -inf is never chosen; where a
    row has fewer than ``top_k`` others (a padding row has none) ``idx`` and
    ``place`` are -1 and the weight is 0. ``out`` gives the four tensors to
    write. The weights carry no autograd graph: their gradient goes through
    ``route_rows_backward``."""
    lp, ld, kind = _logit_rows(logits)
    N, E = logits.shape
    if N >> 31:
        _fits(N)
    dev, i32, f32 = logits.device, torch.int32, torch.float32
    r = _routing(E, top_k, score, renorm, scale, groups, top_groups, group_best)
    if out is not None:
        idx, weight, place, offsets = out
        outs = (_arg(idx, i32, "idx", (N, top_k), dev), _arg(weight, f32, "weight", (N, top_k), dev),
                _arg(place, i32, "place", (N, top_k), dev, offsets is None),
                _arg(offsets, i32, "offsets", (E + 1,), dev, place is None))
    else:
        # (each an allocation of its own: parts of one would start anywhere, which calls that take the weights on
        # 16 bytes refuse, and share a version, so that a change of idx spoils a graph that keeps the weights)
        idx = torch.empty((N, top_k), dtype=i32, device=dev)
        weight = torch.empty((N, top_k), dtype=f32, device=dev)
        place, offsets = (torch.empty_like(idx), torch.empty((E + 1,), dtype=i32, device=dev)) if places else (None, None)
        outs = (idx.data_ptr(), weight.data_ptr(), place.data_ptr() if places else None,
                offsets.data_ptr() if places else None)
    need = _route_bytes(E, top_k, N) if offsets is not None else 0
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    elif ws.dtype is not torch.uint8 or ws.device != dev or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous uint8 tensor on {dev}")
    bias = None if bias is None else _arg(bias, f32, "bias", (E,), dev)
    with _Device(dev) as stream:
        _check(_lib.cardan_route_rows(ctypes.byref(r), N, kind, lp, ld, bias, *outs, ws.data_ptr() if ws is not None else None,
                                      ws.numel() if ws is not None else 0, stream))
    return idx, weight, place, offsets


def route_rows_backward(logits, idx, dweight, top_k: int | None = None, score: str = "softmax", renorm: bool = True,
                        scale: float = 1.0, groups: int = 1, top_groups: int = 1, group_best: int = 1, out=None):
    """Gradient of ``route_rows``'s ``logits`` for the gradient ``dweight [N,
    top_k]`` (float32) of its weights, at the experts ``idx`` that it chose; the
    other arguments as there. In the logits' type, whole rows (zero at experts
    that the weights do not depend on); ``out=logits`` overwrites the logits.
    Where ``idx`` is -1 ``dweight`` is not looked at."""
    lp, ld, kind = _logit_rows(logits)
    N, E = logits.shape
    if N >> 31:
        _fits(N)
    dev = logits.device
    if not isinstance(idx, torch.Tensor) or idx.dim() != 2 or (top_k is not None and idx.shape[1] != top_k):
        raise ValueError("idx must be a [N, top_k] tensor")
    k = idx.shape[1]
    r = _routing(E, k, score, renorm, scale, groups, top_groups, group_best)
    if out is not None:
        d, (dp, dld) = out, _rows_ptr(out, logits.dtype, "out", (N, E), dev)
    else:
        d = torch.empty((N, E), dtype=logits.dtype, device=dev)
        dp, dld = d.data_ptr(), E
    args = (_arg(idx, torch.int32, "idx", (N, k), dev), _arg(dweight, torch.float32, "dweight", (N, k), dev))
    with _Device(dev) as stream:
        _check(_lib.cardan_route_rows_backward(ctypes.byref(r), N, kind, lp, ld, *args, dp, dld, stream))
    return d


def _row_types(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a two-dimensional tensor")
    return t.shape


def dispatch_rows(x, place, rows: int | None = None, out=None):
    """Copies of the rows ``x [N, H]`` (bf16) at the places ``place [N, k]``
    (int32, as ``route_rows`` gives them): ``xe[place[n, j]] = x[n]`` in an
    array of ``rows`` rows (default N k). Places outside it are none; rows that
    no place names are not written, and a row named twice is unspecified (any mix of
    the two). The gradient of x is ``combine_rows`` of
    xe's, without weights."""
    N, H = _row_types(x, "x")
    k = _row_types(place, "place")[1]
    dev, bf = x.device, torch.bfloat16
    M = _row_types(out, "out")[0] if out is not None else N * k if rows is None else rows
    if (N | k | H | M) >> 31:
        _fits(N, k, H, M)
    if out is not None:
        xe = out
        to = _arg(xe, bf, "out", (M, H), dev)
    else:
        xe = torch.empty((M, H), dtype=bf, device=dev)
        to = xe.data_ptr()
    args = (_arg(x, bf, "x", (N, H), dev), _arg(place, torch.int32, "place", (N, k), dev), to)
    with _Device(dev) as stream:
        _check(_lib.cardan_dispatch_rows(N, k, H, M, *args, stream))
    return xe


def combine_rows(ye, place, weight=None, dtype=torch.bfloat16, out=None):
    """Sums of the rows ``ye [M, H]`` (bf16) that ``place [N, k]`` names,
    weighted by ``weight [N, k]`` (float32; None: ones): ``y[n] = sum_j weight[n,
    j] ye[place[n, j]]``, in float32 in the order of j, as bf16 or float32
    (``dtype``) ``[N, H]``. Places outside ``[0, M)`` add nothing. The result
    carries no autograd graph: ``combine_rows_backward``."""
    M, H = _row_types(ye, "ye")
    N, k = _row_types(place, "place")
    if (N | k | H | M) >> 31:
        _fits(N, k, H, M)
    dev = ye.device
    if out is not None:
        y, dtype = out, getattr(out, "dtype", None)
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("y is bfloat16 or float32")
    if out is None:
        y = torch.empty((N, H), dtype=dtype, device=dev)
    args = (_arg(ye, torch.bfloat16, "ye", (M, H), dev), _arg(place, torch.int32, "place", (N, k), dev),
            _arg(weight, torch.float32, "weight", (N, k), dev, True), _TYPES[dtype],
            y.data_ptr() if out is None else _arg(y, dtype, "out", (N, H), dev))
    with _Device(dev) as stream:
        _check(_lib.cardan_combine_rows(N, k, H, M, *args, stream))
    return y


def combine_rows_backward(dy, ye, place, weight=None, need_dye: bool = True, need_dweight: bool = True, dye=None,
                          dweight=None):
    """Gradients of ``combine_rows`` for ``dy [N, H]`` (bf16 or float32):
    ``dye[place[n, j]] = weight[n, j] dy[n]`` (bf16, laid out as ye; rows that no
    place names are not written, a row named twice is unspecified) and ``dweight[n,
    j] = <dy[n], ye[place[n, j]]>`` (float32, 0 without a place). Returns ``(dye,
    dweight)``, None where not asked for; ``dye`` and ``dweight`` give the tensors to write."""
    M, H = _row_types(ye, "ye")
    N, k = _row_types(place, "place")
    if (N | k | H | M) >> 31:
        _fits(N, k, H, M)
    dev = ye.device
    if not isinstance(dy, torch.Tensor) or dy.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("dy must be a [N, H] tensor of bfloat16 or float32")
    if dye is None and need_dye:
        dye = torch.empty_like(ye)
    if dweight is None and need_dweight:
        dweight = torch.empty((N, k), dtype=torch.float32, device=dev)
    args = (_TYPES[dy.dtype], _arg(dy, dy.dtype, "dy", (N, H), dev), _arg(ye, torch.bfloat16, "ye", (M, H), dev),
            _arg(place, torch.int32, "place", (N, k), dev), _arg(weight, torch.float32, "weight", (N, k), dev, True),
            _arg(dye, torch.bfloat16, "dye", (M, H), dev, True), _arg(dweight, torch.float32, "dweight", (N, k), dev, True))
    with _Device(dev) as stream:
        _check(_lib.cardan_combine_rows_backward(N, k, H, M, *args, stream))
    return dye, dweight


ADAMW_BLOCK = 256  # values of a tensor that share a scale of 8-bit moments


def adamw_state(param, bits: int = 32):
    """Moments of ``param`` before its first ``adamw_step``: ``(m, v)`` in
    float32, or with ``bits=8`` ``(m, v, m_scale, v_scale)``: float8_e4m3fn and
    float8_e5m2 values with a float32 scale for every 256 of them (in the order
    of the tensor's elements), so that m is ``m.float() * its scale``."""
    dev, n = param.device, param.numel()
    if bits == 32:
        return tuple(torch.zeros(param.shape, dtype=torch.float32, device=dev) for _ in range(2))
    if bits != 8:
        raise ValueError("bits is 8 or 32")
    blocks = -(-n // ADAMW_BLOCK)
    return (torch.zeros(param.shape, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn),
            torch.zeros(param.shape, dtype=torch.uint8, device=dev).view(torch.float8_e5m2),
            torch.zeros(blocks, dtype=torch.float32, device=dev), torch.zeros(blocks, dtype=torch.float32, device=dev))


def _scalar(t, dtype, name, dev):
    if t.dim() > 1 or t.numel() != 1:
        raise ValueError(f"{name} must hold one value")
    return _arg(t, dtype, name, t.shape, dev)


def adamw_step(params, grads, states, step, lr, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0,
               grad_scale=None, copies=None):
    """One AdamW step over many tensors, in place and unseen by autograd: ``params`` (all float32 or
    all bf16), their ``grads`` (all float32 or all bf16; a parameter whose
    gradient is None is left out) and their ``states`` (``adamw_state``, all of one
    kind, each of one parameter alone), at ``step`` (1 for the first).

    ``m = b1 m + (1 - b1) g``, ``v = b2 v + (1 - b2) g^2``, ``p -= lr
    (weight_decay p + m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps))`` in float32.
    8-bit moments and bf16 weights are stored with dithered rounding (right in
    the mean, a function of step and place). ``step`` (int32) and ``lr`` (float32)
    may be one-element tensors on the device, which a captured call then follows;
    ``grad_scale`` (float32, one element on the device) multiplies every
    gradient. What a step writes must not overlap. ``copies``: bf16 tensors (or None) that receive float32 weights
    rounded to bf16, as ``ffn_forward`` takes them."""
    params, grads, states = list(params), list(grads), list(states)
    copies = [None] * len(params) if copies is None else list(copies)
    if not len(params) == len(grads) == len(states) == len(copies):
        raise ValueError("params, grads, states and copies must have one entry for each tensor")
    todo = [t for t in zip(params, grads, states, copies) if t[1] is not None]
    if not todo:
        return
    if not isinstance(step, torch.Tensor):
        _fits(step)
    p, g, s, _ = todo[0]
    if not isinstance(p, torch.Tensor) or not isinstance(g, torch.Tensor):
        raise TypeError("params and grads must be torch tensors")
    dev, pt, gt, kinds = p.device, p.dtype, g.dtype, len(s)
    for t, name in ((pt, "params"), (gt, "grads")):
        if t not in (torch.float32, torch.bfloat16):
            raise ValueError(f"{name} must be float32 or bfloat16")
    if kinds not in (2, 4):
        raise ValueError("a state is (m, v) or (m, v, m_scale, v_scale)")
    f32 = torch.float32
    mt, vt = (f32, f32) if kinds == 2 else (torch.float8_e4m3fn, torch.float8_e5m2)
    index, kept, rows = dev.index, torch.bfloat16, []  # of AdamwTensor
    for p, g, s, c in todo:
        if len(s) != kinds:
            raise ValueError("states must be of one kind")
        m, v = s[0], s[1]
        # (a pass over what _arg looks at, which gives the message where one does not fit)
        try:
            shape, n = p.shape, p.numel()
            fits = (p.dtype is pt and g.dtype is gt and m.dtype is mt and v.dtype is vt and p.get_device() == index == g.get_device()
                    and m.get_device() == index == v.get_device() and g.shape == shape and m.shape == shape and v.shape == shape
                    and p.is_contiguous() and g.is_contiguous() and m.is_contiguous() and v.is_contiguous())
        except AttributeError:
            shape, fits = getattr(p, "shape", None), False
        if fits and index is not None:
            rows += (p.data_ptr(), g.data_ptr(), m.data_ptr(), v.data_ptr())
        else:
            rows += (_arg(p, pt, "params", shape, dev), _arg(g, gt, "grads", shape, dev), _arg(m, mt, "m", shape, dev),
                     _arg(v, vt, "v", shape, dev))
        if kinds == 4:
            blocks = (-(-n // ADAMW_BLOCK),)
            rows += (_arg(s[2], f32, "m_scale", blocks, dev), _arg(s[3], f32, "v_scale", blocks, dev))
        else:
            rows += (0, 0)
        rows += (0 if c is None else _arg(c, kept, "copies", shape, dev), n)
    table = (ctypes.c_int64 * len(rows))(*rows)
    written = [a for i in (0, 2, 3, 4, 5, 6) for a in rows[i::8] if a]
    if len(set(written)) != len(written):
        raise ValueError("a tensor is given twice")
    conf = Adamw(_TYPES[pt], _TYPES[gt], 32 if kinds == 2 else 8, 0, 0.0, betas[0], betas[1], eps, weight_decay)
    if isinstance(step, torch.Tensor):
        conf.step_device = _scalar(step, torch.int32, "step", dev)
    else:
        conf.step = step
    if isinstance(lr, torch.Tensor):
        conf.lr_device = _scalar(lr, f32, "lr", dev)
    else:
        conf.lr = lr
    if grad_scale is not None:
        conf.grad_scale = _scalar(grad_scale, f32, "grad_scale", dev)
    with _Device(dev) as stream:
        _check(_lib.cardan_adamw_step(ctypes.byref(conf), len(todo), table, stream))


def profile_begin(max_calls: int):
    _check(_lib.cardan_profile_begin(max_calls))


def profile_end() -> dict:
    """``{kind: (total_ms, launches)}`` for the calls since ``profile_begin``."""
    n = len(KERNEL_KINDS)
    ms = (ctypes.c_float * n)()
    cnt = (ctypes.c_int32 * n)()
    _check(_lib.cardan_profile_end(ms, cnt))
    return {k: (ms[i], cnt[i]) for i, k in enumerate(KERNEL_KINDS)}
