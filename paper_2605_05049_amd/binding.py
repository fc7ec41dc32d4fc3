"""ctypes binding of libmoe_gfx950.so.  Argument marshalling only; see include/moe.h for the semantics."""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, Structure, c_char_p, c_int, c_int32, c_int64, c_size_t, c_void_p
from typing import Optional

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libmoe_gfx950.so"
_lib = None

EXPORTED_SYMBOLS = (
    "moe_status_str", "moe_workspace_bytes", "moe_grouped_ffn_small_tiles", "moe_grouped_ffn_mid_tiles", "moe_abi_version",
    "moe_profile_enable", "moe_profile_count", "moe_profile_get", "moe_profile_reset",
    "moe_route_topk", "moe_route_topk_bwd", "moe_permute", "moe_permute_noalloc", "moe_permute_bwd", "moe_permute_bwd_add",
    "moe_router_fwd", "moe_router_route_fwd", "moe_router_bwd", "moe_grouped_ffn_fwd", "moe_grouped_ffn_bwd", "moe_grouped_ffn_bwd_recompute",
    "moe_grouped_ffn_router_bwd",
    "moe_unpermute_combine", "moe_unpermute_combine_bwd", "moe_unpermute_combine_route_bwd",
    "moe_load_accumulate", "moe_load_imbalance", "moe_rebalance_experts",
    "moe_halo_pack_remote", "moe_halo_repack", "moe_halo_unpack",
    "moe_mxfp4_quantize", "moe_mxfp4_quantize_t", "moe_mxfp4_dequantize", "moe_mxfp4_grouped_gemm", "moe_mxfp4_grouped_gemm_large_tiles",
    "moe_mxfp4_grouped_ffn_fwd", "moe_mxfp4_workspace_bytes",
    "moe_layer_few_workspace_bytes", "moe_layer_few_fwd", "moe_layer_few_mxfp4_fwd",
    "moe_gate_fwd", "moe_gate_form", "moe_router_gate_fwd", "moe_gate_bwd", "moe_gate_bias_step",
    "moe_norm_fwd", "moe_norm_bwd", "moe_norm_workspace_bytes",
)
NORM_COLS_MAX = 16384   # MOE_NORM_COLS_MAX: columns of a moe_norm_* call
FEW_TOKENS_MAX = 64   # MOE_FEW_TOKENS_MAX: tokens of a moe_layer_few_* call


class MoeError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {status} ({status_str(status)})")


class _CShape(Structure):
    _fields_ = [("T", c_int32), ("d_model", c_int32), ("d_ffn", c_int32), ("E", c_int32), ("k", c_int32),
                ("E_shared", c_int32), ("renorm", c_int32)]


class Shape:
    """Problem statement of one layer: T tokens, d_model, d_ffn, E routed experts, top-k, E_shared, renorm.  E_total, K_slots
    and N follow from them (and are kept, not computed: every call reads them several times)."""

    def __init__(self, T, d_model, d_ffn, E, k, E_shared=0, renorm=1):
        T, d_model, d_ffn, E, k, E_shared, renorm = int(T), int(d_model), int(d_ffn), int(E), int(k), int(E_shared), int(renorm)
        self.__dict__.update(T=T, d_model=d_model, d_ffn=d_ffn, E=E, k=k, E_shared=E_shared, renorm=renorm,
                             E_total=E + E_shared, K_slots=k + E_shared, N=T * (k + E_shared),
                             _c=_CShape(T, d_model, d_ffn, E, k, E_shared, renorm))

    def __setattr__(self, name, value):
        if name in ("E_total", "K_slots", "N"):
            raise AttributeError(f"{name} follows from the other fields of a Shape")
        fields = {f: self.__dict__[f] for f, _ in _CShape._fields_}
        if name in fields:
            fields[name] = value
            Shape.__init__(self, **fields)
        else:
            object.__setattr__(self, name, value)

    @classmethod
    def of(cls, s) -> "Shape":
        """From any object with the same attribute names (e.g. a workloads.MoEShape)."""
        return s if isinstance(s, Shape) else cls(s.T, s.d_model, s.d_ffn, s.E, s.k, s.E_shared, s.renorm)


class _CGate(Structure):
    _fields_ = [("scores", c_int32), ("groups", c_int32), ("groups_kept", c_int32), ("group_best", c_int32), ("scale", ctypes.c_float)]


class Gate:
    """How a layer routes: scores "softmax" or "sigmoid", the experts in `groups` equal groups of which a token's best `groups_kept` stay (a group's
    score: the sum of its `group_best` best selection scores), `scale` on the weights.  top-k and renormalisation are the Shape's."""

    _SCORES = ("softmax", "sigmoid")

    def __init__(self, scores="softmax", groups=1, groups_kept=None, group_best=1, scale=1.0):
        if scores not in self._SCORES:
            raise ValueError(f"scores {scores!r}: expected one of {self._SCORES}")
        groups = int(groups)
        self.scores, self.groups, self.groups_kept = scores, groups, groups if groups_kept is None else int(groups_kept)
        self.group_best, self.scale = int(group_best), float(scale)
        self._c = _CGate(self._SCORES.index(scores), groups, self.groups_kept, self.group_best, self.scale)

    def __setattr__(self, name, value):
        if "_c" in self.__dict__:
            raise AttributeError("a Gate does not change: make another one")
        object.__setattr__(self, name, value)


def library_path() -> str:
    """The in-tree library; MOE_LIBRARY_PATH overrides it (e.g. to try another build of the same ABI)."""
    return os.environ.get("MOE_LIBRARY_PATH") or os.path.join(PKG_DIR, _LIB_NAME)


def load_library():
    """Loads the shared library (once).  Raises if it has not been built: there is no fallback path."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                           "(or python paper_2605_05049_amd/build.py) first; there is no CPU fallback")
    lib = ctypes.CDLL(path)
    sp = POINTER(_CShape)
    lib.moe_status_str.restype = c_char_p
    lib.moe_status_str.argtypes = [c_int]
    lib.moe_workspace_bytes.restype = c_size_t
    lib.moe_workspace_bytes.argtypes = [sp]
    lib.moe_grouped_ffn_small_tiles.restype = c_int
    lib.moe_grouped_ffn_small_tiles.argtypes = [sp]
    lib.moe_grouped_ffn_mid_tiles.restype = c_int
    lib.moe_grouped_ffn_mid_tiles.argtypes = [sp]
    lib.moe_abi_version.restype = c_int
    lib.moe_abi_version.argtypes = []
    lib.moe_profile_enable.restype = c_int
    lib.moe_profile_enable.argtypes = [c_int]
    lib.moe_profile_count.restype = c_int
    lib.moe_profile_count.argtypes = []
    lib.moe_profile_get.restype = c_int
    lib.moe_profile_get.argtypes = [c_int, POINTER(c_char_p), POINTER(ctypes.c_float)]
    lib.moe_profile_reset.restype = c_int
    lib.moe_profile_reset.argtypes = []
    lib.moe_mxfp4_workspace_bytes.restype = c_size_t
    lib.moe_mxfp4_workspace_bytes.argtypes = [sp]
    lib.moe_layer_few_workspace_bytes.restype = c_size_t
    lib.moe_layer_few_workspace_bytes.argtypes = [sp]
    V = c_void_p
    sigs = {
        "moe_route_topk": [sp, V, V, V, V, V],
        "moe_route_topk_bwd": [sp, V, V, V, V, V, V],
        "moe_permute": [sp, V, V, V, V, V, V, V, V, c_size_t, V],
        "moe_permute_noalloc": [sp, V, V, V, V, V, V, V, V],
        "moe_permute_bwd": [sp, V, V, V, V],
        "moe_permute_bwd_add": [sp, V, V, V, V, V],
        "moe_router_fwd": [sp, V, V, V, V, c_size_t, V],
        "moe_router_route_fwd": [sp, V, V, V, V, V, V, V, c_size_t, V],
        "moe_grouped_ffn_router_bwd": [sp] + [V] * 17 + [c_int, V, c_size_t, V],
        "moe_router_bwd": [sp, V, V, V, V, V, c_int, V, c_size_t, V],
        "moe_grouped_ffn_fwd": [sp, V, V, V, V, V, V, V, V, V, c_size_t, V],
        "moe_grouped_ffn_bwd": [sp, V, V, V, V, V, V, V, V, V, V, V, V, c_int, V, c_size_t, V],
        "moe_grouped_ffn_bwd_recompute": [sp, V, V, V, V, V, V, V, V, V, V, c_int, V, c_size_t, V],
        "moe_unpermute_combine": [sp, V, V, V, V, V],
        "moe_unpermute_combine_bwd": [sp, V, V, V, V, V, V, V],
        "moe_unpermute_combine_route_bwd": [sp, V, V, V, V, V, V, V, V, V, V],
    }
    sigs["moe_halo_pack_remote"] = [V, V, c_int, c_int, c_size_t, c_int, V]
    sigs["moe_halo_repack"] = [V, V, c_int, c_int, c_size_t, V]
    sigs["moe_halo_unpack"] = [V, V, V, c_int, c_int, c_size_t, c_int, V]
    sigs["moe_load_accumulate"] = [V, V, c_int]
    sigs["moe_load_imbalance"] = [V, c_int, c_int, V, POINTER(ctypes.c_double)]
    sigs["moe_rebalance_experts"] = [V, c_int, c_int, V, c_int, POINTER(ctypes.c_int32), V]
    sigs["moe_mxfp4_quantize"] = [V, c_int64, c_int, V, V, V]
    sigs["moe_mxfp4_quantize_t"] = [V, c_int, c_int, c_int, V, V, V]
    sigs["moe_mxfp4_dequantize"] = [V, V, c_int64, c_int, V, V]
    sigs["moe_mxfp4_grouped_gemm"] = [c_int, c_int64, c_int, c_int, V, V, V, V, V, V, V]
    sigs["moe_mxfp4_grouped_gemm_large_tiles"] = [c_int, c_int64, c_int, c_int]
    sigs["moe_mxfp4_grouped_ffn_fwd"] = [sp] + [V] * 10 + [c_size_t, V]
    sigs["moe_layer_few_fwd"] = [sp] + [V] * 9 + [c_size_t, V]
    sigs["moe_layer_few_mxfp4_fwd"] = [sp] + [V] * 12 + [c_size_t, V]
    gp, c_float = POINTER(_CGate), ctypes.c_float
    sigs["moe_gate_fwd"] = [sp, gp, V, V, V, V, V]
    sigs["moe_gate_form"] = [sp, gp, POINTER(c_int32)]
    sigs["moe_router_gate_fwd"] = [sp, gp, V, V, V, V, V, V, V, c_size_t, V]
    sigs["moe_gate_bwd"] = [sp, gp, V, V, V, V, V, c_float, V, V, V, c_size_t, V]
    sigs["moe_gate_bias_step"] = [sp, V, c_float, V, V]
    sigs["moe_norm_fwd"] = [c_int64, c_int, c_int, c_float] + [V] * 9
    sigs["moe_norm_bwd"] = [c_int64, c_int, c_int] + [V] * 9 + [c_int, V, c_size_t, V]
    lib.moe_norm_workspace_bytes.restype = c_size_t
    lib.moe_norm_workspace_bytes.argtypes = [c_int64, c_int]
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.restype = c_int
        fn.argtypes = args
    _lib = lib
    return lib


def status_str(status: int) -> str:
    return load_library().moe_status_str(int(status)).decode()


def abi_version() -> int:
    return int(load_library().moe_abi_version())


def workspace_bytes(shape) -> int:
    return int(load_library().moe_workspace_bytes(ctypes.byref(Shape.of(shape)._c)))


def mxfp4_grouped_gemm_large_tiles(experts, rows, n, k) -> bool:
    """Whether moe_mxfp4_grouped_gemm runs on tiles of 256 x 256 at these sizes."""
    return bool(load_library().moe_mxfp4_grouped_gemm_large_tiles(experts, rows, n, k))


def mxfp4_workspace_bytes(shape) -> int:
    """Bytes of workspace of a forward on 4-bit weights: the router, the permutation and moe_mxfp4_grouped_ffn_fwd (0: the shape is invalid)."""
    return int(load_library().moe_mxfp4_workspace_bytes(ctypes.byref(Shape.of(shape)._c)))


def layer_few_workspace_bytes(shape) -> int:
    """Bytes of workspace of a moe_layer_few_* call (0: the shape is invalid, or has more tokens or slots than such a call takes)."""
    return int(load_library().moe_layer_few_workspace_bytes(ctypes.byref(Shape.of(shape)._c)))


def _gemm_names(bits: int) -> tuple:
    return tuple(name for i, name in enumerate(("gate_up", "down", "dh", "dx")) if bits >> i & 1)


def grouped_ffn_small_tiles(shape) -> tuple:
    """The GEMMs of the grouped FFN that run on 64-row tiles at this shape, out of "gate_up", "down", "dh", "dx"."""
    return _gemm_names(load_library().moe_grouped_ffn_small_tiles(ctypes.byref(Shape.of(shape)._c)))


def grouped_ffn_mid_tiles(shape) -> tuple:
    """The GEMMs of the grouped FFN that run on tiles of 128 columns and up to 192 rows at this shape."""
    return _gemm_names(load_library().moe_grouped_ffn_mid_tiles(ctypes.byref(Shape.of(shape)._c)))


def profile_enable(on: bool) -> None:
    _check("moe_profile_enable", load_library().moe_profile_enable(int(bool(on))))


def profile_reset() -> None:
    _check("moe_profile_reset", load_library().moe_profile_reset())


def profile_records():
    """[(label, milliseconds)] of every launch recorded since the last reset (synchronises on each)."""
    lib = load_library()
    out = []
    for i in range(lib.moe_profile_count()):
        name = c_char_p()
        ms = ctypes.c_float()
        _check("moe_profile_get", lib.moe_profile_get(i, ctypes.byref(name), ctypes.byref(ms)))
        out.append((name.value.decode(), float(ms.value)))
    return out


# ------------------------------------------------------------------------------------------------------------
# marshalling helpers
# ------------------------------------------------------------------------------------------------------------

# torch is looked up once, not imported at the top (the build does without it) nor in every call: the dozen calls of a small
# layer's step are bound by what happens here (256 tokens: 122 us of calls around 96 us of kernels)
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _ptr(t, dtype=None, numel: Optional[int] = None, name: str = "tensor"):
    """Device pointer of a contiguous CUDA(HIP) tensor, after checking dtype (one, or a tuple of them) and element count."""
    if t is None:
        return None
    if (t.is_cuda and t.is_contiguous() and (dtype is None or t.dtype is dtype or (type(dtype) is tuple and t.dtype in dtype))
            and (numel is None or t.numel() >= numel)):
        return t.data_ptr()
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    if dtype is not None:
        ok = t.dtype in dtype if isinstance(dtype, (tuple, list)) else t.dtype == dtype
        if not ok:
            raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name}: {t.numel()} elements, need {numel}")
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(_device())
    return _find_stream()


_raw_stream = _device = None   # the current stream's handle of a device, and the current device: no Stream object is made for them


def _find_stream():
    global _raw_stream, _device
    torch = _torch_module or _torch()
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    _raw_stream, _device = raw, device   # (initialised once, it stays so)
    return raw(device())


def _check(fn: str, rc: int):
    if rc != 0:
        raise MoeError(fn, rc)


_bf16 = None


def _bf16_types():
    global _bf16
    if _bf16 is None:
        torch = _torch()
        _bf16 = (torch.bfloat16, torch.int16, torch.uint16)
    return _bf16


# ------------------------------------------------------------------------------------------------------------
# entry points (same names and argument order as include/moe.h)
# ------------------------------------------------------------------------------------------------------------

def moe_route_topk(shape, logits, topk_idx, topk_w, probs_save=None, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    rc = load_library().moe_route_topk(
        ctypes.byref(s._c), _ptr(logits, torch.float32, s.T * s.E, "logits"),
        _ptr(topk_idx, torch.int32, s.N, "topk_idx"), _ptr(topk_w, torch.float32, s.N, "topk_w"),
        _ptr(probs_save, torch.float32, s.T * s.E, "probs_save"), _stream(stream))
    _check("moe_route_topk", rc)


def moe_route_topk_bwd(shape, dtopk_w, topk_idx, topk_w, probs_save, dlogits, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    rc = load_library().moe_route_topk_bwd(
        ctypes.byref(s._c), _ptr(dtopk_w, torch.float32, s.N, "dtopk_w"), _ptr(topk_idx, torch.int32, s.N, "topk_idx"),
        _ptr(topk_w, torch.float32, s.N, "topk_w"), _ptr(probs_save, torch.float32, s.T * s.E, "probs_save"),
        _ptr(dlogits, torch.float32, s.T * s.E, "dlogits"), _stream(stream))
    _check("moe_route_topk_bwd", rc)


def moe_permute(shape, x, topk_idx, x_perm, counts, offsets, row_of_slot, slot_of_row, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_permute(
        ctypes.byref(s._c), _ptr(x, bf, s.T * s.d_model, "x"), _ptr(topk_idx, torch.int32, s.N, "topk_idx"),
        _ptr(x_perm, bf, s.N * s.d_model, "x_perm"), _ptr(counts, torch.int32, s.E_total, "counts"),
        _ptr(offsets, torch.int32, s.E_total + 1, "offsets"), _ptr(row_of_slot, torch.int32, s.N, "row_of_slot"),
        _ptr(slot_of_row, torch.int32, s.N, "slot_of_row"), _ptr(ws, None, None, "ws"),
        ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_permute", rc)


def moe_permute_noalloc(shape, x, topk_idx, x_perm, counts, offsets, row_of_slot, slot_of_row, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_permute_noalloc(
        ctypes.byref(s._c), _ptr(x, bf, s.T * s.d_model, "x"), _ptr(topk_idx, torch.int32, s.N, "topk_idx"),
        _ptr(x_perm, bf, s.N * s.d_model, "x_perm"), _ptr(counts, torch.int32, s.E_total, "counts"),
        _ptr(offsets, torch.int32, s.E_total + 1, "offsets"), _ptr(row_of_slot, torch.int32, s.N, "row_of_slot"),
        _ptr(slot_of_row, torch.int32, s.N, "slot_of_row"), _stream(stream))
    _check("moe_permute_noalloc", rc)


def moe_permute_bwd(shape, dx_perm, row_of_slot, dx, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_permute_bwd(
        ctypes.byref(s._c), _ptr(dx_perm, bf, s.N * s.d_model, "dx_perm"),
        _ptr(row_of_slot, torch.int32, s.N, "row_of_slot"), _ptr(dx, bf, s.T * s.d_model, "dx"), _stream(stream))
    _check("moe_permute_bwd", rc)


def moe_permute_bwd_add(shape, dx_perm, row_of_slot, dx_addend, dx, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_permute_bwd_add(
        ctypes.byref(s._c), _ptr(dx_perm, bf, s.N * s.d_model, "dx_perm"),
        _ptr(row_of_slot, torch.int32, s.N, "row_of_slot"), _ptr(dx_addend, bf, s.T * s.d_model, "dx_addend"),
        _ptr(dx, bf, s.T * s.d_model, "dx"), _stream(stream))
    _check("moe_permute_bwd_add", rc)


def moe_router_fwd(shape, x, w_router, logits, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_router_fwd(
        ctypes.byref(s._c), _ptr(x, bf, s.T * s.d_model, "x"), _ptr(w_router, bf, s.E * s.d_model, "w_router"),
        _ptr(logits, torch.float32, s.T * s.E, "logits"), _ptr(ws, None, None, "ws"), ws.numel() * ws.element_size(),
        _stream(stream))
    _check("moe_router_fwd", rc)


def moe_router_route_fwd(shape, x, w_router, logits, topk_idx, topk_w, probs_save, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_router_route_fwd(
        ctypes.byref(s._c), _ptr(x, bf, s.T * s.d_model, "x"), _ptr(w_router, bf, s.E * s.d_model, "w_router"),
        _ptr(logits, torch.float32, s.T * s.E, "logits"), _ptr(topk_idx, torch.int32, s.N, "topk_idx"),
        _ptr(topk_w, torch.float32, s.N, "topk_w"), _ptr(probs_save, torch.float32, s.T * s.E, "probs_save"),
        _ptr(ws, None, None, "ws"), ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_router_route_fwd", rc)


def moe_router_bwd(shape, x, w_router, dlogits, dx_router, dw_router, accumulate, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_router_bwd(
        ctypes.byref(s._c), _ptr(x, bf, s.T * s.d_model, "x"), _ptr(w_router, bf, s.E * s.d_model, "w_router"),
        _ptr(dlogits, torch.float32, s.T * s.E, "dlogits"), _ptr(dx_router, bf, s.T * s.d_model, "dx_router"),
        _ptr(dw_router, torch.float32, s.E * s.d_model, "dw_router"), int(bool(accumulate)),
        _ptr(ws, None, None, "ws"), ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_router_bwd", rc)


def moe_grouped_ffn_fwd(shape, x_perm, offsets, w_gate, w_up, w_down, y_perm, save_g, save_u, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    nw = s.E_total * s.d_model * s.d_ffn
    rc = load_library().moe_grouped_ffn_fwd(
        ctypes.byref(s._c), _ptr(x_perm, bf, s.N * s.d_model, "x_perm"), _ptr(offsets, torch.int32, s.E_total + 1, "offsets"),
        _ptr(w_gate, bf, nw, "w_gate"), _ptr(w_up, bf, nw, "w_up"), _ptr(w_down, bf, nw, "w_down"),
        _ptr(y_perm, bf, s.N * s.d_model, "y_perm"),
        None if save_g is None else _ptr(save_g, bf, s.N * s.d_ffn, "save_g"),
        None if save_u is None else _ptr(save_u, bf, s.N * s.d_ffn, "save_u"), _ptr(ws, None, None, "ws"),
        ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_grouped_ffn_fwd", rc)


def moe_grouped_ffn_bwd_recompute(shape, dy_perm, x_perm, offsets, w_gate, w_up, w_down, dx_perm, dw_gate, dw_up, dw_down,
                                  accumulate, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    nw = s.E_total * s.d_model * s.d_ffn
    rc = load_library().moe_grouped_ffn_bwd_recompute(
        ctypes.byref(s._c), _ptr(dy_perm, bf, s.N * s.d_model, "dy_perm"), _ptr(x_perm, bf, s.N * s.d_model, "x_perm"),
        _ptr(offsets, torch.int32, s.E_total + 1, "offsets"), _ptr(w_gate, bf, nw, "w_gate"), _ptr(w_up, bf, nw, "w_up"),
        _ptr(w_down, bf, nw, "w_down"), _ptr(dx_perm, bf, s.N * s.d_model, "dx_perm"),
        _ptr(dw_gate, torch.float32, nw, "dw_gate"), _ptr(dw_up, torch.float32, nw, "dw_up"),
        _ptr(dw_down, torch.float32, nw, "dw_down"), int(bool(accumulate)), _ptr(ws, None, None, "ws"),
        ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_grouped_ffn_bwd_recompute", rc)


def moe_grouped_ffn_bwd(shape, dy_perm, x_perm, offsets, w_gate, w_up, w_down, save_g, save_u, dx_perm,
                        dw_gate, dw_up, dw_down, accumulate, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    nw = s.E_total * s.d_model * s.d_ffn
    rc = load_library().moe_grouped_ffn_bwd(
        ctypes.byref(s._c), _ptr(dy_perm, bf, s.N * s.d_model, "dy_perm"), _ptr(x_perm, bf, s.N * s.d_model, "x_perm"),
        _ptr(offsets, torch.int32, s.E_total + 1, "offsets"), _ptr(w_gate, bf, nw, "w_gate"), _ptr(w_up, bf, nw, "w_up"),
        _ptr(w_down, bf, nw, "w_down"), _ptr(save_g, bf, s.N * s.d_ffn, "save_g"), _ptr(save_u, bf, s.N * s.d_ffn, "save_u"),
        _ptr(dx_perm, bf, s.N * s.d_model, "dx_perm"), _ptr(dw_gate, torch.float32, nw, "dw_gate"),
        _ptr(dw_up, torch.float32, nw, "dw_up"), _ptr(dw_down, torch.float32, nw, "dw_down"), int(bool(accumulate)),
        _ptr(ws, None, None, "ws"), ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_grouped_ffn_bwd", rc)


def moe_grouped_ffn_router_bwd(shape, dy_perm, x_perm, offsets, w_gate, w_up, w_down, save_g, save_u, dx_perm, dw_gate, dw_up, dw_down,
                               x, w_router, dlogits, dx_router, dw_router, accumulate, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    nw = s.E_total * s.d_model * s.d_ffn
    rc = load_library().moe_grouped_ffn_router_bwd(
        ctypes.byref(s._c), _ptr(dy_perm, bf, s.N * s.d_model, "dy_perm"), _ptr(x_perm, bf, s.N * s.d_model, "x_perm"),
        _ptr(offsets, torch.int32, s.E_total + 1, "offsets"), _ptr(w_gate, bf, nw, "w_gate"), _ptr(w_up, bf, nw, "w_up"),
        _ptr(w_down, bf, nw, "w_down"), _ptr(save_g, bf, s.N * s.d_ffn, "save_g"), _ptr(save_u, bf, s.N * s.d_ffn, "save_u"),
        _ptr(dx_perm, bf, s.N * s.d_model, "dx_perm"), _ptr(dw_gate, torch.float32, nw, "dw_gate"),
        _ptr(dw_up, torch.float32, nw, "dw_up"), _ptr(dw_down, torch.float32, nw, "dw_down"),
        _ptr(x, bf, s.T * s.d_model, "x"), _ptr(w_router, bf, s.E * s.d_model, "w_router"),
        _ptr(dlogits, torch.float32, s.T * s.E, "dlogits"), _ptr(dx_router, bf, s.T * s.d_model, "dx_router"),
        _ptr(dw_router, torch.float32, s.E * s.d_model, "dw_router"), int(bool(accumulate)),
        _ptr(ws, None, None, "ws"), ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_grouped_ffn_router_bwd", rc)


def moe_unpermute_combine(shape, y_perm, row_of_slot, topk_w, out, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_unpermute_combine(
        ctypes.byref(s._c), _ptr(y_perm, bf, s.N * s.d_model, "y_perm"), _ptr(row_of_slot, torch.int32, s.N, "row_of_slot"),
        _ptr(topk_w, torch.float32, s.N, "topk_w"), _ptr(out, bf, s.T * s.d_model, "out"), _stream(stream))
    _check("moe_unpermute_combine", rc)


def moe_unpermute_combine_bwd(shape, dout, y_perm, row_of_slot, topk_w, dy_perm, dtopk_w, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_unpermute_combine_bwd(
        ctypes.byref(s._c), _ptr(dout, bf, s.T * s.d_model, "dout"), _ptr(y_perm, bf, s.N * s.d_model, "y_perm"),
        _ptr(row_of_slot, torch.int32, s.N, "row_of_slot"), _ptr(topk_w, torch.float32, s.N, "topk_w"),
        _ptr(dy_perm, bf, s.N * s.d_model, "dy_perm"), _ptr(dtopk_w, torch.float32, s.N, "dtopk_w"), _stream(stream))
    _check("moe_unpermute_combine_bwd", rc)


def moe_unpermute_combine_route_bwd(shape, dout, y_perm, row_of_slot, topk_idx, topk_w, probs_save, dy_perm, dtopk_w, dlogits, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_unpermute_combine_route_bwd(
        ctypes.byref(s._c), _ptr(dout, bf, s.T * s.d_model, "dout"), _ptr(y_perm, bf, s.N * s.d_model, "y_perm"),
        _ptr(row_of_slot, torch.int32, s.N, "row_of_slot"), _ptr(topk_idx, torch.int32, s.N, "topk_idx"),
        _ptr(topk_w, torch.float32, s.N, "topk_w"), _ptr(probs_save, torch.float32, s.T * s.E, "probs_save"),
        _ptr(dy_perm, bf, s.N * s.d_model, "dy_perm"), _ptr(dtopk_w, torch.float32, s.N, "dtopk_w"),
        _ptr(dlogits, torch.float32, s.T * s.E, "dlogits"), _stream(stream))
    _check("moe_unpermute_combine_route_bwd", rc)


# ---- microscaled 4-bit floating point; the whole layer for a few tokens ------------------------------------------

def _u8(t, numel, name):
    return _ptr(t, (_torch_module or _torch()).uint8, numel, name)


def _last(t, what):
    if t.dim() < 1 or t.shape[-1] < 1:
        raise ValueError(f"{what}: expected rows of at least one element")
    return t.numel() // t.shape[-1], t.shape[-1]


def moe_mxfp4_quantize(x, q, scales, stream=None):
    """x [..., cols] bf16 -> q [..., cols / 2], scales [..., cols / 32] (uint8)."""
    rows, cols = _last(x, "x")
    rc = load_library().moe_mxfp4_quantize(_ptr(x, _bf16_types(), None, "x"), rows, cols, _u8(q, rows * cols // 2, "q"),
                                           _u8(scales, rows * cols // 32, "scales"), _stream(stream))
    _check("moe_mxfp4_quantize", rc)


def moe_mxfp4_quantize_t(w, q, scales, stream=None):
    """w [..., K, C] bf16 -> q [..., C, K / 2], scales [..., C, K / 32] (uint8): blocks along K."""
    if w.dim() < 2:
        raise ValueError("w: expected a matrix, or several")
    n, (rows, cols) = w.numel(), w.shape[-2:]
    batch = n // (rows * cols) if n else 0
    rc = load_library().moe_mxfp4_quantize_t(_ptr(w, _bf16_types(), None, "w"), batch, rows, cols, _u8(q, n // 2, "q"), _u8(scales, n // 32, "scales"),
                                             _stream(stream))
    _check("moe_mxfp4_quantize_t", rc)


def moe_mxfp4_dequantize(q, scales, x, stream=None):
    """q [..., cols / 2], scales [..., cols / 32] (uint8) -> x [..., cols] bf16."""
    rows, cols = _last(x, "x")
    rc = load_library().moe_mxfp4_dequantize(_u8(q, rows * cols // 2, "q"), _u8(scales, rows * cols // 32, "scales"), rows, cols,
                                             _ptr(x, _bf16_types(), None, "x"), _stream(stream))
    _check("moe_mxfp4_dequantize", rc)


def moe_mxfp4_grouped_gemm(xq, x_scales, offsets, wq, w_scales, y, stream=None):
    """y [rows, n] bf16 = per expert xq [rows, k / 2] times wq [experts, n, k / 2], rows grouped by `offsets` [experts + 1]."""
    torch = _torch_module or _torch()
    if xq.dim() != 2 or wq.dim() != 3 or xq.shape[1] != wq.shape[2]:
        raise ValueError("xq, wq: expected [rows, k / 2] and [experts, n, k / 2]")
    rows, (experts, n, half) = xq.shape[0], wq.shape
    rc = load_library().moe_mxfp4_grouped_gemm(
        experts, rows, n, 2 * half, _u8(xq, None, "xq"), _u8(x_scales, rows * half // 16, "x_scales"),
        _ptr(offsets, torch.int32, experts + 1, "offsets"), _u8(wq, None, "wq"), _u8(w_scales, experts * n * half // 16, "w_scales"),
        _ptr(y, _bf16_types(), rows * n, "y"), _stream(stream))
    _check("moe_mxfp4_grouped_gemm", rc)


def _mx_weights(s, wq_gate, s_gate, wq_up, s_up, wq_down, s_down):
    n = s.E_total * s.d_model * s.d_ffn
    return (_u8(wq_gate, n // 2, "wq_gate"), _u8(s_gate, n // 32, "s_gate"), _u8(wq_up, n // 2, "wq_up"), _u8(s_up, n // 32, "s_up"),
            _u8(wq_down, n // 2, "wq_down"), _u8(s_down, n // 32, "s_down"))


def moe_mxfp4_grouped_ffn_fwd(shape, x_perm, offsets, wq_gate, s_gate, wq_up, s_up, wq_down, s_down, y_perm, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_mxfp4_grouped_ffn_fwd(
        ctypes.byref(s._c), _ptr(x_perm, bf, s.N * s.d_model, "x_perm"), _ptr(offsets, torch.int32, s.E_total + 1, "offsets"),
        *_mx_weights(s, wq_gate, s_gate, wq_up, s_up, wq_down, s_down), _ptr(y_perm, bf, s.N * s.d_model, "y_perm"), _ptr(ws, None, None, "ws"),
        ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_mxfp4_grouped_ffn_fwd", rc)


def moe_layer_few_fwd(shape, x, w_router, w_gate, w_up, w_down, out, topk_idx, topk_w, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    nw = s.E_total * s.d_model * s.d_ffn
    rc = load_library().moe_layer_few_fwd(
        ctypes.byref(s._c), _ptr(x, bf, s.T * s.d_model, "x"), _ptr(w_router, bf, s.E * s.d_model, "w_router"), _ptr(w_gate, bf, nw, "w_gate"),
        _ptr(w_up, bf, nw, "w_up"), _ptr(w_down, bf, nw, "w_down"), _ptr(out, bf, s.T * s.d_model, "out"),
        _ptr(topk_idx, torch.int32, s.N, "topk_idx"), _ptr(topk_w, torch.float32, s.N, "topk_w"), _ptr(ws, None, None, "ws"),
        ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_layer_few_fwd", rc)


def moe_layer_few_mxfp4_fwd(shape, x, w_router, wq_gate, s_gate, wq_up, s_up, wq_down, s_down, out, topk_idx, topk_w, ws, stream=None):
    torch = _torch_module or _torch()
    s = Shape.of(shape)
    bf = _bf16_types()
    rc = load_library().moe_layer_few_mxfp4_fwd(
        ctypes.byref(s._c), _ptr(x, bf, s.T * s.d_model, "x"), _ptr(w_router, bf, s.E * s.d_model, "w_router"),
        *_mx_weights(s, wq_gate, s_gate, wq_up, s_up, wq_down, s_down), _ptr(out, bf, s.T * s.d_model, "out"),
        _ptr(topk_idx, torch.int32, s.N, "topk_idx"), _ptr(topk_w, torch.float32, s.N, "topk_w"), _ptr(ws, None, None, "ws"),
        ws.numel() * ws.element_size(), _stream(stream))
    _check("moe_layer_few_mxfp4_fwd", rc)


# ---- in front of the experts: routing with scores of another kind, and the norm ------------------------------------

def norm_workspace_bytes(rows, cols) -> int:
    """Bytes of workspace of moe_norm_bwd (0: sizes outside the limits)."""
    return int(load_library().moe_norm_workspace_bytes(rows, cols))


def _here():
    """The current device, where a launch goes (without one: no tensor's)."""
    return _device() if _device is not None else _find_device()


def _find_device():
    global _device
    torch = _torch_module or _torch()
    if not torch.cuda.is_initialized():
        return -2
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _device()


def _as(dtype, t, numel, name, here):
    """_ptr of one dtype on the device `here`, for the calls that are short: the checks in the order in which they cost least."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == here and t.is_contiguous() and t.numel() >= numel:
        return t.data_ptr()
    ptr = _ptr(t, _bf16_types() if dtype is _torch_module.bfloat16 else dtype, numel, name)
    _on(here, t.get_device(), name)
    return ptr


def _on(here, device, name):
    if device != here:
        raise ValueError(f"{name} on device {device}: the call belongs within torch.cuda.device({device})")


def _stream_on(here, stream):
    if stream is not None:
        _on(here, getattr(stream, "device_index", here), "stream")
    return _stream(stream)


def _workspace(ws, here):
    if ws is None:
        return None, 0
    ptr = _ptr(ws, None, None, "ws")
    _on(here, ws.get_device(), "ws")
    return ptr, ws.numel() * ws.element_size()


def moe_gate_fwd(shape, gate, logits, bias, topk_idx, topk_w, stream=None):
    torch = _torch_module or _torch()
    s, f32, here = Shape.of(shape), torch.float32, _here()
    rc = (_lib or load_library()).moe_gate_fwd(
        ctypes.byref(s._c), ctypes.byref(gate._c), _as(f32, logits, s.T * s.E, "logits", here), _as(f32, bias, s.E, "bias", here),
        _as(torch.int32, topk_idx, s.N, "topk_idx", here), _as(f32, topk_w, s.N, "topk_w", here), _stream_on(here, stream))
    if rc:
        _check("moe_gate_fwd", rc)


def gate_form(shape, gate):
    """(keys of a list, lanes of a token, experts of a lane, whether every lane has as many): the form of moe_gate_fwd that these tokens run."""
    form = (c_int32 * 4)()
    _check("moe_gate_form", load_library().moe_gate_form(ctypes.byref(Shape.of(shape)._c), ctypes.byref(gate._c), form))
    return tuple(form)


def moe_router_gate_fwd(shape, gate, x, w_router, bias, logits, topk_idx, topk_w, ws, stream=None):
    torch = _torch_module or _torch()
    s, f32, bf, here = Shape.of(shape), torch.float32, torch.bfloat16, _here()
    rc = (_lib or load_library()).moe_router_gate_fwd(
        ctypes.byref(s._c), ctypes.byref(gate._c), _as(bf, x, s.T * s.d_model, "x", here), _as(bf, w_router, s.E * s.d_model, "w_router", here),
        _as(f32, bias, s.E, "bias", here), _as(f32, logits, s.T * s.E, "logits", here),
        _as(torch.int32, topk_idx, s.N, "topk_idx", here), _as(f32, topk_w, s.N, "topk_w", here), *_workspace(ws, here), _stream_on(here, stream))
    if rc:
        _check("moe_router_gate_fwd", rc)


def moe_gate_bwd(shape, gate, dtopk_w, logits, topk_idx, topk_w, counts, balance, dlogits, loss=None, ws=None, stream=None):
    """counts None: no balance loss.  loss [1] fp32 needs counts and a workspace."""
    torch = _torch_module or _torch()
    s, f32, here = Shape.of(shape), torch.float32, _here()
    rc = (_lib or load_library()).moe_gate_bwd(
        ctypes.byref(s._c), ctypes.byref(gate._c), _as(f32, dtopk_w, s.N, "dtopk_w", here), _as(f32, logits, s.T * s.E, "logits", here),
        _as(torch.int32, topk_idx, s.N, "topk_idx", here), _as(f32, topk_w, s.N, "topk_w", here), _as(torch.int32, counts, s.E_total, "counts", here), balance,
        _as(f32, dlogits, s.T * s.E, "dlogits", here), _as(f32, loss, 1, "loss", here), *_workspace(ws, here), _stream_on(here, stream))
    if rc:
        _check("moe_gate_bwd", rc)


def moe_gate_bias_step(shape, counts, rate, bias, stream=None):
    torch = _torch_module or _torch()
    s, here = Shape.of(shape), _here()
    rc = (_lib or load_library()).moe_gate_bias_step(ctypes.byref(s._c), _as(torch.int32, counts, s.E_total, "counts", here), rate,
                                                     _as(torch.float32, bias, s.E, "bias", here), _stream_on(here, stream))
    if rc:
        _check("moe_gate_bias_step", rc)


def moe_norm_fwd(centre, eps, x, addend, gamma, beta, sum, y, mean, rstd, stream=None):
    """x [..., cols] bf16; addend, gamma, beta, sum, mean and rstd may be None."""
    torch = _torch_module or _torch()
    f32, bf, here = torch.float32, torch.bfloat16, _here()
    rows, cols = _last(x, "x")
    n = rows * cols
    rc = (_lib or load_library()).moe_norm_fwd(
        rows, cols, 1 if centre else 0, eps, _as(bf, x, n, "x", here), _as(bf, addend, n, "addend", here), _as(bf, gamma, cols, "gamma", here),
        _as(bf, beta, cols, "beta", here), _as(bf, sum, n, "sum", here), _as(bf, y, n, "y", here), _as(f32, mean, rows, "mean", here),
        _as(f32, rstd, rows, "rstd", here), _stream_on(here, stream))
    if rc:
        _check("moe_norm_fwd", rc)


def moe_norm_bwd(centre, dy, h, gamma, mean, rstd, dx_addend, dx, dgamma, dbeta, accumulate, ws, stream=None):
    """dy, h [..., cols] bf16; gamma, dx_addend, dgamma, dbeta and (without centre) mean may be None, ws without dgamma and dbeta."""
    torch = _torch_module or _torch()
    f32, bf, here = torch.float32, torch.bfloat16, _here()
    rows, cols = _last(h, "h")
    n = rows * cols
    rc = (_lib or load_library()).moe_norm_bwd(
        rows, cols, 1 if centre else 0, _as(bf, dy, n, "dy", here), _as(bf, h, n, "h", here), _as(bf, gamma, cols, "gamma", here),
        _as(f32, mean, rows, "mean", here), _as(f32, rstd, rows, "rstd", here), _as(bf, dx_addend, n, "dx_addend", here), _as(bf, dx, n, "dx", here),
        _as(f32, dgamma, cols, "dgamma", here), _as(f32, dbeta, cols, "dbeta", here), 1 if accumulate else 0, *_workspace(ws, here), _stream_on(here, stream))
    if rc:
        _check("moe_norm_bwd", rc)


# ---- single-GPU steps of the hierarchical all-to-all (device tensors; rows of any dtype, 16-byte multiples) -----

def _rows(t, n_rows, what):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous CUDA tensor")
    nbytes = t.numel() * t.element_size()
    if n_rows == 0:
        return ctypes.c_void_p(t.data_ptr()), 0
    if nbytes % n_rows:
        raise ValueError(f"{what}: {nbytes} bytes do not split into {n_rows} rows")
    return ctypes.c_void_p(t.data_ptr()), nbytes // n_rows


def moe_halo_pack_remote(S, F2s, num_nodes, R, node_id, stream=None):
    ps, rb = _rows(S, num_nodes * R, "S")
    pd, rb2 = _rows(F2s, (num_nodes - 1) * R, "F2s")
    if num_nodes > 1 and rb != rb2:
        raise ValueError("S and F2s differ in row size")
    _check("moe_halo_pack_remote", load_library().moe_halo_pack_remote(ps, pd, int(num_nodes), int(R), rb, int(node_id), _stream(stream)))


def moe_halo_repack(F2r, F3s, M, R, stream=None):
    ps, rb = _rows(F2r, M * R, "F2r")
    pd, rb2 = _rows(F3s, M * R, "F3s")
    if rb != rb2:
        raise ValueError("F2r and F3s differ in size")
    _check("moe_halo_repack", load_library().moe_halo_repack(ps, pd, int(M), int(R), rb if M else 16, _stream(stream)))


def moe_halo_unpack(P1, F3r, O, num_nodes, R, node_id, stream=None):
    p1, rb = _rows(P1, R, "P1")
    po, rb2 = _rows(O, num_nodes * R, "O")
    if rb != rb2:
        raise ValueError("P1 and O differ in row size")
    p3 = None
    if num_nodes > 1:
        p3, rb3 = _rows(F3r, R * (num_nodes - 1), "F3r")
        if rb3 != rb:
            raise ValueError("F3r and O differ in row size")
    _check("moe_halo_unpack", load_library().moe_halo_unpack(p1, p3, po, int(num_nodes), int(R), rb, int(node_id), _stream(stream)))


# ---- host-side load statistics and rebalancing (NumPy arrays; nothing here touches the GPU) ------------------

def _np(a, dtype, what):
    import numpy as np
    if not isinstance(a, np.ndarray) or a.dtype != dtype or not a.flags["C_CONTIGUOUS"]:
        raise ValueError(f"{what}: expected a C-contiguous numpy array of {np.dtype(dtype).name}")
    return a.ctypes.data_as(ctypes.c_void_p)


def load_accumulate(running, counts):
    """running[e] += counts[e] in place (running int64 [E], counts int32 [E], both on the host)."""
    import numpy as np
    if running.shape != counts.shape:
        raise ValueError("running and counts differ in shape")
    _check("moe_load_accumulate", load_library().moe_load_accumulate(_np(running, np.int64, "running"), _np(counts, np.int32, "counts"),
                                                                     int(running.size)))


def load_imbalance(load, groups) -> float:
    """max group load / mean group load for a placement `groups` (int32 [n_groups, experts per group])."""
    import numpy as np
    r = ctypes.c_double(0.0)
    _check("moe_load_imbalance", load_library().moe_load_imbalance(_np(load, np.int64, "load"), int(load.size), int(groups.shape[0]),
                                                                   _np(groups, np.int32, "groups"), ctypes.byref(r)))
    return float(r.value)


def rebalance_experts(load, groups, max_iters=100):
    """Algorithm 2 on a copy of `groups`; returns (new groups, swaps) with swaps an int32 [n, 2] array."""
    import numpy as np
    out = np.ascontiguousarray(groups, dtype=np.int32).copy()
    swaps = np.zeros((max(int(max_iters), 1), 2), dtype=np.int32)
    n = ctypes.c_int32(0)
    _check("moe_rebalance_experts", load_library().moe_rebalance_experts(
        _np(load, np.int64, "load"), int(load.size), int(out.shape[0]), _np(out, np.int32, "groups"), int(max_iters),
        ctypes.byref(n), _np(swaps, np.int32, "swaps")))
    return out, swaps[:n.value].copy()
