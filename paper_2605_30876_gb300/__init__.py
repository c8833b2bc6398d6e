"""dMoE block-routed MoE-layer forward on GB300 (sm_103a): Python binding of libdmoe.so.

The functions below carry the names of the C ABI in ``include/dmoe.h`` and only marshal
arguments: torch tensors (CUDA, contiguous, of the documented dtype) become device
pointers, ``None`` becomes NULL, and the current torch CUDA stream is used unless one is
given. Every step of the forward runs in the library's CUDA kernels; there is no other
implementation in this package, and importing it fails when the library is not built.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

__all__ = [
    "DMOE_ROUTE_TOKEN", "DMOE_ROUTE_BLOCK", "DmoeError", "LayerDesc", "make_desc",
    "dmoe_workspace_size", "dmoe_workspace_init", "dmoe_router", "dmoe_dispatch", "dmoe_moe_forward",
    "dmoe_layer_forward", "dmoe_get_device_error", "dmoe_status_string", "dmoe_abi_version",
    "dmoe_layer_forward_launches",
    "alloc_workspace", "LIB_PATH", "dmoe_set_profile_events", "KERNELS",
    "dmoe_sort_workspace_size", "alloc_sort_workspace", "dmoe_sort_tokens", "dmoe_gather_rows",
    "dmoe_gather_rows_backward", "dmoe_combine_rows", "dmoe_combine_rows_backward",
    "Q4Desc", "make_q4_desc", "dmoe_q4_size", "alloc_q4", "dmoe_q4_quantize",
    "dmoe_q4_dequantize", "dmoe_q4_linear", "dmoe_q4_swiglu",
    "dmoe_q4_device_error",
    "ExpertDesc", "dmoe_expert_ffn", "dmoe_expert_ffn_backward", "dmoe_expert_device_error",
    "NormDesc", "dmoe_norm_residual", "dmoe_norm_workspace_size", "alloc_norm_workspace",
    "dmoe_norm_residual_backward",
]

DMOE_ROUTE_TOKEN = 0
DMOE_ROUTE_BLOCK = 1

DMOE_OK = 0
STATUS_NAMES = {0: "DMOE_OK", 1: "DMOE_ERR_INVALID_ARG", 2: "DMOE_ERR_UNSUPPORTED",
                3: "DMOE_ERR_WORKSPACE", 4: "DMOE_ERR_CUDA", 5: "DMOE_ERR_DEVICE",
                6: "DMOE_ERR_TIMEOUT"}

# DMOE_LIB selects another build of the same library (for example one compiled with other
# flags); by default the in-tree libdmoe.so
LIB_PATH = os.environ.get("DMOE_LIB") or os.path.join(
    os.path.dirname(os.path.abspath(__file__)), "libdmoe.so")


class LayerDesc(ctypes.Structure):
    """dmoe_layer_desc (include/dmoe.h)."""
    _fields_ = [("d_model", ctypes.c_int32), ("n_experts", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("d_ff", ctypes.c_int32),
                ("d_ff_shared", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("n_blocks", ctypes.c_int32), ("mode", ctypes.c_int32),
                ("top_p", ctypes.c_float), ("block_top_k", ctypes.c_int32)]

    @property
    def T(self) -> int:
        return self.n_blocks * self.block_size


def make_desc(d_model, n_experts, top_k, d_ff, d_ff_shared, block_size, n_blocks,
              mode=DMOE_ROUTE_BLOCK, top_p=0.0, block_top_k=0) -> LayerDesc:
    return LayerDesc(d_model, n_experts, top_k, d_ff, d_ff_shared, block_size, n_blocks,
                     mode, float(top_p), int(block_top_k))


class Q4Desc(ctypes.Structure):
    """dmoe_q4_desc (include/dmoe.h)."""
    _fields_ = [("n_experts", ctypes.c_int32), ("n_out", ctypes.c_int32),
                ("n_in", ctypes.c_int32), ("group", ctypes.c_int32)]


def make_q4_desc(n_experts, n_out, n_in, group=64) -> Q4Desc:
    return Q4Desc(n_experts, n_out, n_in, group)


class ExpertDesc(ctypes.Structure):
    """dmoe_expert_desc (include/dmoe.h)."""
    _fields_ = [("dtype", ctypes.c_int32), ("n_experts", ctypes.c_int32),
                ("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32)]


class NormDesc(ctypes.Structure):
    """dmoe_norm_desc (include/dmoe.h)."""
    _fields_ = [("dtype", ctypes.c_int32), ("d", ctypes.c_int32), ("T", ctypes.c_int64),
                ("gate_tokens", ctypes.c_int64), ("scale", ctypes.c_float), ("eps", ctypes.c_float)]


class DmoeError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        msg = f"{where}: {STATUS_NAMES.get(status, status)}"
        if detail:
            msg += f" ({detail})"
        super().__init__(msg)


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.c_void_p
    D = ctypes.POINTER(LayerDesc)
    st = ctypes.c_int
    lib.dmoe_workspace_size.argtypes = [D, ctypes.POINTER(ctypes.c_size_t)]
    lib.dmoe_workspace_size.restype = st
    lib.dmoe_workspace_init.argtypes = [P, ctypes.c_size_t, P]
    lib.dmoe_workspace_init.restype = st
    lib.dmoe_router.argtypes = [D, P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P]
    lib.dmoe_router.restype = st
    lib.dmoe_router_prepare.argtypes = [D, P, P, ctypes.c_size_t, P]
    lib.dmoe_router_prepare.restype = st
    lib.dmoe_dispatch.argtypes = [D, P, P, P, P, P, P, P, ctypes.c_size_t, P]
    lib.dmoe_dispatch.restype = st
    lib.dmoe_moe_forward.argtypes = [D] + [P] * 14 + [P, ctypes.c_size_t, P]
    lib.dmoe_moe_forward.restype = st
    lib.dmoe_layer_forward.argtypes = [D] + [P] * 14 + [P, ctypes.c_size_t, P]
    lib.dmoe_layer_forward.restype = st
    lib.dmoe_get_device_error.argtypes = [P, P, ctypes.POINTER(ctypes.c_int32)]
    lib.dmoe_get_device_error.restype = st
    lib.dmoe_status_string.argtypes = [ctypes.c_int]
    lib.dmoe_status_string.restype = ctypes.c_char_p
    lib.dmoe_last_error_message.argtypes = []
    lib.dmoe_last_error_message.restype = ctypes.c_char_p
    lib.dmoe_abi_version.argtypes = []
    lib.dmoe_abi_version.restype = ctypes.c_int32
    lib.dmoe_layer_forward_launches.argtypes = [ctypes.POINTER(LayerDesc)]
    lib.dmoe_layer_forward_launches.restype = ctypes.c_int32
    lib.dmoe_set_profile_events.argtypes = [ctypes.c_int32, P, P]
    lib.dmoe_set_profile_events.restype = st
    lib.dmoe_set_debug_hold.argtypes = [P, ctypes.c_int32, P]
    lib.dmoe_set_debug_hold.restype = st
    lib.dmoe_router_no_alloc.argtypes = [D, P, P, P, P, P, P, P, P, P]
    lib.dmoe_router_no_alloc.restype = st
    lib.dmoe_router_no_alloc_device_error.argtypes = [P, ctypes.POINTER(ctypes.c_int32)]
    lib.dmoe_router_no_alloc_device_error.restype = st
    lib.dmoe_no_alloc_scratch.argtypes = [ctypes.POINTER(P), ctypes.POINTER(ctypes.c_size_t)]
    lib.dmoe_no_alloc_scratch.restype = st
    i32, i64, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    Q = ctypes.POINTER(Q4Desc)
    sizes = ctypes.POINTER(size)
    products = [Q, i64, i32, P, i64, i64, P, i32, P, P]
    X = ctypes.POINTER(ExpertDesc)
    N = ctypes.POINTER(NormDesc)
    for name, args in {
            "dmoe_sort_workspace_size": [i64, i32, i32, sizes],
            "dmoe_sort_tokens": [i64, i32, i32, P, P, P, P, P, size, P],
            "dmoe_gather_rows": [i32, i64, i32, i32, P, i64, P, P, i64, P],
            "dmoe_gather_rows_backward": [i32, i64, i32, i32, P, i64, P, P, i64, P],
            "dmoe_combine_rows": [i32, i64, i32, i32, P, i64, P, P, P, i64, P, i64, P],
            "dmoe_combine_rows_backward": [i32, i64, i32, i32, P, i64, P, i64, P, P, P, i64, P, P],
            "dmoe_q4_size": [Q, sizes, sizes],
            "dmoe_q4_quantize": [Q, P, P, P, P],
            "dmoe_q4_dequantize": [Q, P, P, P, P],
            "dmoe_q4_device_error": [P, ctypes.POINTER(i32)],
            "dmoe_q4_set_debug_hold": [i32],
            "dmoe_expert_ffn": [X, i64, i32, P, i64, P, P] + [P] * 5 + [P, i64, i32, P],
            "dmoe_expert_ffn_backward": [X, i64, P, i64, P, i64] + [P] * 8 + [i64] + [P] * 3 + [i32, P],
            "dmoe_expert_device_error": [P, ctypes.POINTER(i32)],
            "dmoe_expert_set_debug_hold": [i32],
            "dmoe_norm_residual": [N] + [P, i64] * 2 + [P, P, i64, P] + [P, i64] * 2 + [P, P],
            "dmoe_norm_workspace_size": [N, sizes],
            "dmoe_norm_residual_backward": [N] + [P, i64] * 2 + [P, P, i64, P, P] + [P, i64] * 5 +
                                           [P, P, P, size, P],
            "dmoe_q4_linear": products + [P] * 2 + [P, i64, i32, P],
            "dmoe_q4_swiglu": products + [P] * 4 + [P, i64, i32, P]}.items():
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, st
    return lib


_lib = _load()

_Tensor = torch.Tensor
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = torch._C._cuda_getDevice if _raw_stream is not None else None


def _check(status: int, where: str) -> None:
    if status != DMOE_OK:
        detail = _lib.dmoe_last_error_message().decode() if status == 4 else ""
        raise DmoeError(status, where, detail)


def _ptr(t, dtype=None, name="tensor"):
    """Device pointer of a contiguous CUDA tensor (None -> NULL; an int is passed through)."""
    if not isinstance(t, _Tensor):
        if t is None or isinstance(t, int):
            return t
        raise TypeError(f"{name}: expected a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is None or not torch.cuda.is_initialized():
            return torch.cuda.current_stream().cuda_stream
        # the same stream without the Python object that torch.cuda.current_stream() makes
        return _raw_stream(_current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _ws(workspace: torch.Tensor) -> Tuple[int, int]:
    if workspace is None:
        raise ValueError("workspace is required (see alloc_workspace)")
    return _ptr(workspace, torch.uint8, "workspace"), workspace.numel()


def dmoe_workspace_size(desc: LayerDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.dmoe_workspace_size(ctypes.byref(desc), ctypes.byref(n)), "dmoe_workspace_size")
    return n.value


def alloc_workspace(desc: LayerDesc, device="cuda") -> torch.Tensor:
    """A zeroed uint8 buffer of dmoe_workspace_size(desc) bytes on `device` (torch allocates)."""
    ws = torch.empty(dmoe_workspace_size(desc), dtype=torch.uint8, device=device)
    if not ws.is_cuda:   # a host image of a workspace: nothing was prepared at its address
        return ws.zero_()
    dmoe_workspace_init(ws)
    return ws


def dmoe_workspace_init(workspace, stream=None) -> None:
    """Zero-fills a workspace and forgets any preparation of an earlier one at its address."""
    ws, nb = _ws(workspace)
    with torch.cuda.device(workspace.device):
        _check(_lib.dmoe_workspace_init(ws, nb, _stream(stream)), "dmoe_workspace_init")


def dmoe_router(desc, x, w_r, bias, topk_idx, topk_gate, coreset=None, coreset_size=None,
                probs=None, workspace=None, stream=None) -> None:
    ws, nb = _ws(workspace)
    _check(_lib.dmoe_router(ctypes.byref(desc), _ptr(x, torch.bfloat16, "x"),
                            _ptr(w_r, torch.float32, "w_r"), _ptr(bias, torch.float32, "bias"),
                            _ptr(topk_idx, torch.int32, "topk_idx"),
                            _ptr(topk_gate, torch.float32, "topk_gate"),
                            _ptr(coreset, torch.int32, "coreset"),
                            _ptr(coreset_size, torch.int32, "coreset_size"),
                            _ptr(probs, torch.float32, "probs"), ws, nb, _stream(stream)),
           "dmoe_router")


def dmoe_router_prepare(desc, w_r, workspace, stream=None) -> None:
    ws, nb = _ws(workspace)
    _check(_lib.dmoe_router_prepare(ctypes.byref(desc), _ptr(w_r, torch.float32, "w_r"), ws, nb,
                                    _stream(stream)), "dmoe_router_prepare")


def dmoe_dispatch(desc, topk_idx, n_unique, unique_ids, offsets, rows, pos, workspace=None,
                  stream=None) -> None:
    ws, nb = _ws(workspace)
    i32 = torch.int32
    _check(_lib.dmoe_dispatch(ctypes.byref(desc), _ptr(topk_idx, i32, "topk_idx"),
                              _ptr(n_unique, i32, "n_unique"), _ptr(unique_ids, i32, "unique_ids"),
                              _ptr(offsets, i32, "offsets"), _ptr(rows, i32, "rows"),
                              _ptr(pos, i32, "pos"), ws, nb, _stream(stream)), "dmoe_dispatch")


def dmoe_moe_forward(desc, x, w_gate, w_up, w_down, ws_gate, ws_up, ws_down, topk_gate,
                     n_unique, unique_ids, offsets, rows, pos, y, workspace=None,
                     stream=None) -> None:
    ws, nb = _ws(workspace)
    b, i32 = torch.bfloat16, torch.int32
    _check(_lib.dmoe_moe_forward(
        ctypes.byref(desc), _ptr(x, b, "x"), _ptr(w_gate, b, "w_gate"), _ptr(w_up, b, "w_up"),
        _ptr(w_down, b, "w_down"), _ptr(ws_gate, b, "ws_gate"), _ptr(ws_up, b, "ws_up"),
        _ptr(ws_down, b, "ws_down"), _ptr(topk_gate, torch.float32, "topk_gate"),
        _ptr(n_unique, i32, "n_unique"), _ptr(unique_ids, i32, "unique_ids"),
        _ptr(offsets, i32, "offsets"), _ptr(rows, i32, "rows"), _ptr(pos, i32, "pos"),
        _ptr(y, b, "y"), ws, nb, _stream(stream)), "dmoe_moe_forward")


def dmoe_layer_forward(desc, x, w_r, bias, w_gate, w_up, w_down, ws_gate, ws_up, ws_down, y,
                       topk_idx=None, topk_gate=None, n_unique=None, unique_ids=None,
                       workspace=None, stream=None) -> None:
    ws, nb = _ws(workspace)
    b, i32 = torch.bfloat16, torch.int32
    _check(_lib.dmoe_layer_forward(
        ctypes.byref(desc), _ptr(x, b, "x"), _ptr(w_r, torch.float32, "w_r"),
        _ptr(bias, torch.float32, "bias"), _ptr(w_gate, b, "w_gate"), _ptr(w_up, b, "w_up"),
        _ptr(w_down, b, "w_down"), _ptr(ws_gate, b, "ws_gate"), _ptr(ws_up, b, "ws_up"),
        _ptr(ws_down, b, "ws_down"), _ptr(y, b, "y"), _ptr(topk_idx, i32, "topk_idx"),
        _ptr(topk_gate, torch.float32, "topk_gate"), _ptr(n_unique, i32, "n_unique"),
        _ptr(unique_ids, i32, "unique_ids"), ws, nb, _stream(stream)), "dmoe_layer_forward")


def dmoe_get_device_error(workspace, stream=None) -> Tuple[int, Tuple[int, int, int]]:
    """Synchronises the stream; returns (status, (code, where, value)) and clears the record."""
    info = (ctypes.c_int32 * 4)()
    st = _lib.dmoe_get_device_error(_ptr(workspace, torch.uint8, "workspace"), _stream(stream),
                                    info)
    return st, (info[0], info[1], info[2])


def dmoe_router_no_alloc(desc, x, w_r, bias, topk_idx, topk_gate, coreset=None,
                         coreset_size=None, probs=None, stream=None) -> None:
    """dmoe_router without a workspace (the library's static scratch array)."""
    _check(_lib.dmoe_router_no_alloc(
        ctypes.byref(desc), _ptr(x, torch.bfloat16, "x"), _ptr(w_r, torch.float32, "w_r"),
        _ptr(bias, torch.float32, "bias"), _ptr(topk_idx, torch.int32, "topk_idx"),
        _ptr(topk_gate, torch.float32, "topk_gate"), _ptr(coreset, torch.int32, "coreset"),
        _ptr(coreset_size, torch.int32, "coreset_size"), _ptr(probs, torch.float32, "probs"),
        _stream(stream)), "dmoe_router_no_alloc")


def dmoe_router_no_alloc_device_error(stream=None) -> Tuple[int, Tuple[int, int, int]]:
    """Synchronises the stream; returns (status, (code, where, value)) of the static scratch
    array's fault record and clears it."""
    info = (ctypes.c_int32 * 4)()
    st = _lib.dmoe_router_no_alloc_device_error(_stream(stream), info)
    return st, (info[0], info[1], info[2])


def dmoe_no_alloc_scratch() -> Tuple[int, int]:
    """(device address, bytes) of the static scratch array on the current device."""
    ptr, n = ctypes.c_void_p(0), ctypes.c_size_t(0)
    _check(_lib.dmoe_no_alloc_scratch(ctypes.byref(ptr), ctypes.byref(n)),
           "dmoe_no_alloc_scratch")
    return int(ptr.value or 0), n.value


def dmoe_set_debug_hold(workspace, hold: int, stream=None) -> None:
    """Diagnostic: makes the expert launch's bounded waits run out while
    `hold` is nonzero (see include/dmoe.h); cleared by dmoe_get_device_error."""
    _check(_lib.dmoe_set_debug_hold(_ptr(workspace, torch.uint8, "workspace"), int(hold),
                                    _stream(stream)), "dmoe_set_debug_hold")


# ---------------------------------------------------------------- a layer by its parts
# (include/dmoe.h has the meaning of every argument). Matrices of rows are 2-D tensors whose rows
# are contiguous; their stride may leave gaps between rows. All tensors of a call are on one device,
# which need not be the current one.

_DTYPE_IDS = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def _matrix(t, name, n, d, dtype, device) -> Tuple[int, int]:
    """(device pointer, row stride) of an [n, d] CUDA tensor of contiguous rows."""
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if device < 0 or t.get_device() != device:
        raise ValueError(f"{name}: must be a CUDA tensor on the call's device")
    if t.shape != (n, d):
        raise ValueError(f"{name}: expected shape {(n, d)}, got {tuple(t.shape)}")
    ld, step = t.stride()
    if step != 1 and d > 1:
        raise ValueError(f"{name}: its rows must be contiguous")
    return t.data_ptr(), ld if n > 1 else d   # (one row: any stride)


def _vector(t, name, numel, dtype, device) -> Optional[int]:
    """Device pointer of a contiguous CUDA tensor of `numel` elements (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if device < 0 or t.get_device() != device:
        raise ValueError(f"{name}: must be a CUDA tensor on the call's device")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if t.numel() != numel:
        raise ValueError(f"{name}: expected {numel} elements, got {t.numel()}")
    return t.data_ptr()


def _launch(fn, device, stream, *args) -> None:
    """Calls the library on the tensors' device, on its current stream unless one is given."""
    if _raw_stream is not None and device == _current_device():
        status = fn(*args, _raw_stream(device) if stream is None else _stream(stream))
    else:
        with torch.cuda.device(device):
            status = fn(*args, _stream(stream))
    if status != DMOE_OK:
        _check(status, fn.__name__)


def _slots(tokens, pos, name="pos") -> int:
    k, rest = divmod(pos.numel(), tokens) if tokens > 0 else (1, pos.numel())
    if rest or k < 1 or (pos.dim() == 2 and pos.shape[0] != tokens):
        raise ValueError(f"{name}: {pos.numel()} entries {tuple(pos.shape)} are no k slots for "
                         f"each of {tokens} tokens")
    return k


def _gates(t, name, tokens, k, device) -> Optional[int]:
    """Device pointer of fp32 gates [T, k] (None -> NULL). Their shape says how the R slots are cut: it has
    to agree with the other tensors' tokens."""
    if isinstance(t, _Tensor) and t.dim() == 2 and t.shape[0] != tokens:
        raise ValueError(f"{name}: expected shape {(tokens, k)}, got {tuple(t.shape)}")
    return _vector(t, name, tokens * k, torch.float32, device)


def _row_dtype(t, name) -> int:
    if not isinstance(t, _Tensor) or t.dtype not in _DTYPE_IDS or t.dim() != 2:
        raise TypeError(f"{name}: expected a 2-D bf16, fp16 or fp32 tensor")
    return _DTYPE_IDS[t.dtype]


def dmoe_sort_workspace_size(T: int, k: int, E: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.dmoe_sort_workspace_size(T, k, E, ctypes.byref(n)), "dmoe_sort_workspace_size")
    return n.value


def alloc_sort_workspace(T: int, k: int, E: int, device="cuda") -> torch.Tensor:
    """A zeroed workspace for dmoe_sort_tokens of these sizes."""
    ws = torch.empty(dmoe_sort_workspace_size(T, k, E), dtype=torch.uint8, device=device)
    dmoe_workspace_init(ws)
    return ws


def dmoe_sort_tokens(topk_idx, E, offsets, rows, pos, workspace=None, stream=None) -> None:
    """topk_idx int32 [T, k] (negative: no expert) -> offsets [E + 1], rows [T * k], pos [T * k]."""
    if not isinstance(topk_idx, _Tensor) or topk_idx.dim() != 2:
        raise TypeError("topk_idx: expected an int32 tensor [T, k]")
    T, k = topk_idx.shape
    dev, i32 = topk_idx.get_device(), torch.int32
    ws, nb = _ws(workspace)
    if workspace.get_device() != dev:
        raise ValueError("workspace: must be on the call's device")
    _launch(_lib.dmoe_sort_tokens, dev, stream, T, k, E, _vector(topk_idx, "topk_idx", T * k, i32, dev),
            _vector(offsets, "offsets", E + 1, i32, dev), _vector(rows, "rows", T * k, i32, dev),
            _vector(pos, "pos", T * k, i32, dev), ws, nb)


def dmoe_gather_rows(x, pos, xs, stream=None) -> None:
    """xs[pos[t, j]] = x[t]; zeros in the rows of slots without an expert."""
    dt = _row_dtype(x, "x")
    T, d = x.shape
    R, dev = pos.numel(), x.get_device()
    k = _slots(T, pos)
    px, ldx = _matrix(x, "x", T, d, x.dtype, dev)
    po, ldo = _matrix(xs, "xs", R, d, x.dtype, dev)
    _launch(_lib.dmoe_gather_rows, dev, stream, dt, T, k, d, px, ldx,
            _vector(pos, "pos", R, torch.int32, dev), po, ldo)


def dmoe_gather_rows_backward(dxs, pos, dx, stream=None) -> None:
    """dx[t] = sum over its slots of dxs[pos[t, j]]."""
    dt = _row_dtype(dxs, "dxs")
    R, d = dxs.shape
    T, dev = dx.shape[0], dxs.get_device()
    k = _slots(T, pos)
    pi, ldi = _matrix(dxs, "dxs", T * k if T else 0, d, dxs.dtype, dev)
    po, ldo = _matrix(dx, "dx", T, d, dxs.dtype, dev)
    _launch(_lib.dmoe_gather_rows_backward, dev, stream, dt, T, k, d, pi, ldi,
            _vector(pos, "pos", R, torch.int32, dev), po, ldo)


def dmoe_combine_rows(ys, pos, gates, add, y, stream=None) -> None:
    """y[t] = add[t] + sum over its slots of gates[t, j] * ys[pos[t, j]] (gates, add: or None)."""
    dt = _row_dtype(ys, "ys")
    R, d = ys.shape
    T, dev = y.shape[0], ys.get_device()
    k = _slots(T, pos)
    pi, ldi = _matrix(ys, "ys", T * k if T else 0, d, ys.dtype, dev)
    pa, lda = (None, 0) if add is None else _matrix(add, "add", T, d, ys.dtype, dev)
    po, ldo = _matrix(y, "y", T, d, ys.dtype, dev)
    _launch(_lib.dmoe_combine_rows, dev, stream, dt, T, k, d, pi, ldi,
            _vector(pos, "pos", R, torch.int32, dev),
            _gates(gates, "gates", T, k, dev), pa, lda, po, ldo)


def dmoe_combine_rows_backward(dy, ys, pos, gates, dys, dgates, stream=None) -> None:
    """dys[pos[t, j]] = gates[t, j] * dy[t] and dgates[t, j] = <dy[t], ys[pos[t, j]]> (either of
    dys and dgates may be None; ys is read for dgates only)."""
    dt = _row_dtype(dy, "dy")
    T, d = dy.shape
    R, dev = pos.numel(), dy.get_device()
    k = _slots(T, pos)
    pd, ldd = _matrix(dy, "dy", T, d, dy.dtype, dev)
    py, ldy = (None, 0) if ys is None else _matrix(ys, "ys", R, d, dy.dtype, dev)
    po, ldo = (None, 0) if dys is None else _matrix(dys, "dys", R, d, dy.dtype, dev)
    _launch(_lib.dmoe_combine_rows_backward, dev, stream, dt, T, k, d, pd, ldd, py, ldy,
            _vector(pos, "pos", R, torch.int32, dev), _gates(gates, "gates", T, k, dev), po, ldo,
            _gates(dgates, "dgates", T, k, dev))


def dmoe_q4_size(desc: Q4Desc) -> Tuple[int, int]:
    """(bytes of the codes, bytes of the scales)."""
    c, s = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(_lib.dmoe_q4_size(ctypes.byref(desc), ctypes.byref(c), ctypes.byref(s)), "dmoe_q4_size")
    return c.value, s.value


def alloc_q4(desc: Q4Desc, device="cuda") -> Tuple[torch.Tensor, torch.Tensor]:
    """Buffers (uint8) for the codes and the scales of `desc`'s matrices."""
    return tuple(torch.empty(n, dtype=torch.uint8, device=device) for n in dmoe_q4_size(desc))


def _q4_bytes(desc) -> Tuple[int, int]:
    """dmoe_q4_size without the call (a product checks it every time): tiles of 32 rows, blocks of 128
    inputs. The library refuses what is no valid desc."""
    blocks = desc.n_experts * (-(-desc.n_out // 32)) * (-(-desc.n_in // 128))
    return 2048 * blocks, 64 * (128 // max(desc.group, 1)) * blocks


def _q4(sizes, codes, scales, name, device) -> Tuple[int, int]:
    if codes is None or scales is None:
        raise TypeError(f"{name}: codes and scales are required")
    return (_vector(codes, f"{name} codes", sizes[0], torch.uint8, device),
            _vector(scales, f"{name} scales", sizes[1], torch.uint8, device))


def _q4_convert(name, desc, w, codes, scales, stream):
    if not isinstance(w, _Tensor):
        raise TypeError("w: expected a torch.Tensor")
    dev = w.get_device()
    c, s = _q4(_q4_bytes(desc), codes, scales, "w", dev)
    p = _vector(w, "w", desc.n_experts * desc.n_out * desc.n_in, torch.bfloat16, dev)
    pw = (p, c, s) if name == "dmoe_q4_quantize" else (c, s, p)
    _launch(getattr(_lib, name), dev, stream, ctypes.byref(desc), *pw)


def dmoe_q4_quantize(desc, w, codes, scales, stream=None) -> None:
    """w bf16 [n_experts, n_out, n_in] -> codes, scales (alloc_q4)."""
    _q4_convert("dmoe_q4_quantize", desc, w, codes, scales, stream)


def dmoe_q4_dequantize(desc, codes, scales, w, stream=None) -> None:
    """codes, scales -> the bf16 values they stand for, w [n_experts, n_out, n_in]."""
    _q4_convert("dmoe_q4_dequantize", desc, w, codes, scales, stream)


def _q4_products(fn, desc, x, offsets, weights, y, rows, k, expert_ids, stream):
    if not isinstance(x, _Tensor) or x.dim() != 2 or not isinstance(y, _Tensor) or y.dim() != 2:
        raise TypeError("x, y: expected 2-D tensors")
    dev, T, R = x.get_device(), x.shape[0], y.shape[0]
    px, ldx = _matrix(x, "x", T, desc.n_in, torch.bfloat16, dev)
    ydt = torch.float32 if y.dtype is torch.float32 else torch.bfloat16
    py, ldy = _matrix(y, "y", R, desc.n_out, ydt, dev)
    n = offsets.numel() - 1 if offsets is not None else 1
    i32, sizes, ptrs = torch.int32, _q4_bytes(desc), []
    for i in range(0, len(weights), 2):
        ptrs += _q4(sizes, weights[i], weights[i + 1], "weights", dev)
    _launch(fn, dev, stream, ctypes.byref(desc), R, n, px, ldx, T, _vector(rows, "rows", R, i32, dev),
            k, _vector(offsets, "offsets", n + 1, i32, dev),
            _vector(expert_ids, "expert_ids", n, i32, dev), *ptrs, py, ldy, _DTYPE_IDS[ydt])


def dmoe_q4_linear(desc, x, offsets, codes, scales, y, rows=None, k=1, expert_ids=None,
                   stream=None) -> None:
    """y[r] = W[expert of r] x[rows[r] // k] (rows None: x[r]) for the rows of every group of
    offsets (None: one group of all rows)."""
    _q4_products(_lib.dmoe_q4_linear, desc, x, offsets, (codes, scales), y, rows, k, expert_ids,
                 stream)


def dmoe_q4_swiglu(desc, x, offsets, gate_codes, gate_scales, up_codes, up_scales, y, rows=None,
                   k=1, expert_ids=None, stream=None) -> None:
    """y[r] = silu(Wg x) * (Wu x), arguments as for dmoe_q4_linear."""
    _q4_products(_lib.dmoe_q4_swiglu, desc, x, offsets, (gate_codes, gate_scales, up_codes, up_scales),
                 y, rows, k, expert_ids, stream)


def dmoe_q4_device_error(stream=None) -> Tuple[int, Tuple[int, int, int]]:
    """Synchronises the stream; returns (status, (code, where, value)) of the fault record of the
    4-bit products on the current device and clears it."""
    info = (ctypes.c_int32 * 4)()
    st = _lib.dmoe_q4_device_error(_stream(stream), info)
    return st, (info[0], info[1], info[2])


def dmoe_q4_set_debug_hold(hold: int) -> None:
    """Diagnostic: makes the 4-bit products' bounded waits run out while `hold` is nonzero (see
    include/dmoe.h); cleared by dmoe_q4_device_error."""
    _check(_lib.dmoe_q4_set_debug_hold(int(hold)), "dmoe_q4_set_debug_hold")


def _experts(x, w_gate, w_up, w_down, name="x"):
    """(desc, R, device, pointers of the three weights) of a feed-forward block's tensors."""
    for n, t in ((name, x), ("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        if not isinstance(t, _Tensor) or t.dim() != (2 if t is x else 3):
            raise TypeError(f"{n}: expected a {2 if n == name else 3}-D tensor")
    dt, dev = x.dtype, x.get_device()
    if dt is not torch.bfloat16 and dt is not torch.float16:
        raise TypeError(f"{name}: expected bf16 or fp16, got {dt}")
    E, I, d = w_gate.shape
    if w_up.shape != w_gate.shape or w_down.shape != (E, d, I):
        raise ValueError(f"expected w_gate and w_up [E, I, d] and w_down [E, d, I], got "
                         f"{tuple(w_gate.shape)}, {tuple(w_up.shape)} and {tuple(w_down.shape)}")
    n = E * I * d
    return (ExpertDesc(_DTYPE_IDS[dt], E, d, I), x.shape[0], dev, _vector(w_gate, "w_gate", n, dt, dev),
            _vector(w_up, "w_up", n, dt, dev), _vector(w_down, "w_down", n, dt, dev))


def _offsets(offsets, dev):
    """(groups, device pointer)."""
    if offsets is None:
        return 1, None
    n = offsets.numel() - 1 if isinstance(offsets, _Tensor) else 0
    if n < 1:
        raise TypeError("offsets: expected an int32 tensor [groups + 1]")
    return n, _vector(offsets, "offsets", n + 1, torch.int32, dev)


def dmoe_expert_ffn(x, offsets, w_gate, w_up, w_down, h, y, pre=None, expert_ids=None, zero_rest=False,
                    stream=None) -> None:
    """y[r] = w_down[e] (silu(w_gate[e] x[r]) * (w_up[e] x[r])) for the rows of every group of offsets
    (None: one group of all rows). h [R, I] and, for the gradients, pre [R, 2, I] are written, too."""
    desc, R, dev, wg, wu, wd = _experts(x, w_gate, w_up, w_down)
    d, I, dt = desc.d_model, desc.d_ff, x.dtype
    px, ldx = _matrix(x, "x", R, d, dt, dev)
    py, ldy = _matrix(y, "y", R, d, dt, dev)
    if h is None:
        raise TypeError("h: expected a tensor [R, I]")
    n, po = _offsets(offsets, dev)
    _launch(_lib.dmoe_expert_ffn, dev, stream, ctypes.byref(desc), R, n, px, ldx, po,
            _vector(expert_ids, "expert_ids", n, torch.int32, dev), wg, wu, wd,
            _vector(pre, "pre", 2 * R * I, dt, dev), _vector(h, "h", R * I, dt, dev), py, ldy,
            1 if zero_rest else 0)


def dmoe_expert_ffn_backward(dy, x, offsets, w_gate, w_up, w_down, pre, h, dpre, dx, dw_gate, dw_up,
                             dw_down, zero_rest=False, stream=None) -> None:
    """dmoe_expert_ffn's gradients by x and by the weights (any of dx, dw_gate with dw_up, and dw_down may
    be None); group u is expert u. dpre [R, 2, I] is scratch."""
    desc, R, dev, wg, wu, wd = _experts(dy, w_gate, w_up, w_down, "dy")
    E, d, I, dt = desc.n_experts, desc.d_model, desc.d_ff, dy.dtype
    n, po = _offsets(offsets, dev)
    if n != E:
        raise ValueError(f"offsets: expected {E + 1} entries, got {n + 1}")
    pdy, lddy = _matrix(dy, "dy", R, d, dt, dev)
    px, ldx = (None, 0) if x is None else _matrix(x, "x", R, d, dt, dev)
    pdx, lddx = (None, 0) if dx is None else _matrix(dx, "dx", R, d, dt, dev)
    _launch(_lib.dmoe_expert_ffn_backward, dev, stream, ctypes.byref(desc), R, pdy, lddy, px, ldx, po,
            wg, wu, wd, _vector(pre, "pre", 2 * R * I, dt, dev), _vector(h, "h", R * I, dt, dev),
            _vector(dpre, "dpre", 2 * R * I, dt, dev), pdx, lddx,
            _vector(dw_gate, "dw_gate", E * I * d, dt, dev), _vector(dw_up, "dw_up", E * I * d, dt, dev),
            _vector(dw_down, "dw_down", E * I * d, dt, dev), 1 if zero_rest else 0)


def dmoe_expert_device_error(stream=None) -> Tuple[int, Tuple[int, int, int]]:
    """Synchronises the stream; returns (status, (code, where, value)) of the fault record of the
    feed-forward block's calls on the current device and clears it."""
    info = (ctypes.c_int32 * 4)()
    st = _lib.dmoe_expert_device_error(_stream(stream), info)
    return st, (info[0], info[1], info[2])


def dmoe_expert_set_debug_hold(hold: int) -> None:
    """Diagnostic: makes the feed-forward block's bounded waits run out while `hold` is nonzero;
    cleared by dmoe_expert_device_error."""
    _check(_lib.dmoe_expert_set_debug_hold(int(hold)), "dmoe_expert_set_debug_hold")


def _norm_args(x, y, w_post, gate, w_pre, scale, eps, gate_tokens):
    """(desc, device, arguments of what both directions read, None where there is nothing)."""
    dt = _row_dtype(x, "x")
    T, d = x.shape
    dev, t = x.get_device(), x.dtype
    G = 0 if gate is None else int(gate_tokens) or 1
    px, ldx = _matrix(x, "x", T, d, t, dev)
    py, ldy = (None, 0) if y is None else _matrix(y, "y", T, d, t, dev)
    pg, ldg = (None, 0) if gate is None else _matrix(gate, "gate", -(-T // G) if G > 0 else 0, d, t, dev)
    return (NormDesc(dt, d, T, G, scale, eps), dev,
            (px, ldx, py, ldy, _vector(w_post, "w_post", d, torch.float32, dev), pg, ldg,
             _vector(w_pre, "w_pre", d, torch.float32, dev)))


def dmoe_norm_residual(x, y, w_post, gate, w_pre, r, n, stats=None, scale=1.0, eps=1e-6, gate_tokens=0,
                       stream=None) -> None:
    """r = scale * x + gate * norm(y) * w_post, n = norm(r) * w_pre. y, w_post, gate, w_pre (with n) and r
    may be None; gate [ceil(T / gate_tokens), d]: row t // gate_tokens holds for token t (gate_tokens 0: a row
    for each token)."""
    desc, dev, args = _norm_args(x, y, w_post, gate, w_pre, scale, eps, gate_tokens)
    T, d, t = desc.T, desc.d, x.dtype
    pr, ldr = (None, 0) if r is None else _matrix(r, "r", T, d, t, dev)
    pn, ldn = (None, 0) if n is None else _matrix(n, "n", T, d, t, dev)
    _launch(_lib.dmoe_norm_residual, dev, stream, ctypes.byref(desc), *args, pr, ldr, pn, ldn,
            _vector(stats, "stats", 2 * T, torch.float32, dev))


def dmoe_norm_workspace_size(T: int, d: int, gate_tokens: int = 0) -> int:
    n = ctypes.c_size_t(0)
    desc = NormDesc(0, d, T, gate_tokens, 1.0, 0.0)
    _check(_lib.dmoe_norm_workspace_size(ctypes.byref(desc), ctypes.byref(n)), "dmoe_norm_workspace_size")
    return n.value


def alloc_norm_workspace(T: int, d: int, gate_tokens: int = 0, device="cuda") -> torch.Tensor:
    """A workspace for dmoe_norm_residual_backward of these sizes."""
    return torch.empty(dmoe_norm_workspace_size(T, d, gate_tokens), dtype=torch.uint8, device=device)


def dmoe_norm_residual_backward(x, y, w_post, gate, w_pre, stats, dr, dn, dx, dy, dgate, dw_post, dw_pre,
                                scale=1.0, gate_tokens=0, workspace=None, stream=None) -> None:
    """dmoe_norm_residual's gradients by x, y, gate and the weights (any may be None) from those by r and
    by n (either may be None)."""
    desc, dev, args = _norm_args(x, y, w_post, gate, w_pre, scale, 0.0, gate_tokens)
    T, d, t = desc.T, desc.d, x.dtype
    more = []
    for name, m, rows in (("dr", dr, T), ("dn", dn, T), ("dx", dx, T), ("dy", dy, T),
                          ("dgate", dgate, 0 if gate is None else gate.shape[0])):
        more += (None, 0) if m is None else _matrix(m, name, rows, d, t, dev)
    f32 = torch.float32
    ws = (None, 0)
    if workspace is not None:
        ws = (_vector(workspace, "workspace", workspace.numel(), torch.uint8, dev), workspace.numel())
    _launch(_lib.dmoe_norm_residual_backward, dev, stream, ctypes.byref(desc), *args,
            _vector(stats, "stats", 2 * T, f32, dev), *more, _vector(dw_post, "dw_post", d, f32, dev),
            _vector(dw_pre, "dw_pre", d, f32, dev), *ws)


KERNELS = {"router": 0, "dispatch": 1, "gather": 2, "experts": 3, "combine": 4}


def dmoe_set_profile_events(kernel, ev_begin=None, ev_end=None) -> None:
    """Record torch.cuda.Event pairs around every launch of `kernel` (name or id) made by
    later calls on this thread; (None, None) clears."""
    kid = KERNELS[kernel] if isinstance(kernel, str) else int(kernel)
    b = ev_begin.cuda_event if ev_begin is not None else None
    e = ev_end.cuda_event if ev_end is not None else None
    _check(_lib.dmoe_set_profile_events(kid, b, e), "dmoe_set_profile_events")


def dmoe_status_string(status: int) -> str:
    return _lib.dmoe_status_string(status).decode()


def dmoe_abi_version() -> int:
    return _lib.dmoe_abi_version()


def dmoe_layer_forward_launches(desc) -> int:
    """Kernel launches of one dmoe_layer_forward call for `desc` (-1: invalid desc)."""
    return _lib.dmoe_layer_forward_launches(ctypes.byref(desc))
