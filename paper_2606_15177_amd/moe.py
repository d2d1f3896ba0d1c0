"""Python binding of the gfx950 MoE-layer library (include/moe.h).

Argument marshalling only: torch tensors are used for device memory and the
current HIP stream, their raw pointers go to the C ABI, and every step of the
layer runs in the library's kernels.  Importing this module fails loudly when
the built library is missing; there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
import re

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe_gfx950.so")
HEADER = os.path.join(os.path.dirname(_HERE), "include", "moe.h")

MOE_OK, MOE_ERR_NULL, MOE_ERR_DIMS, MOE_ERR_UNSUPPORTED = 0, -1, -2, -3
MOE_ERR_WORKSPACE, MOE_ERR_DEVICE, MOE_ERR_ALIGN = -4, -5, -6
ENTRY_PERMUTE, ENTRY_EXPERT_FFN, ENTRY_FORWARD = 1, 2, 3
ENTRY_EXPERT_FFN_I8, ENTRY_FORWARD_I8 = 4, 5
ENTRY_EXPERT_FFN_F8, ENTRY_FORWARD_F8 = 6, 7
GATE_SOFTMAX_TOPK, GATE_SOFTMAX, GATE_SIGMOID = 0, 1, 2   # moe_dims.flags
STAGES = ("route", "permute", "ffn_up", "ffn_down", "combine")


class MoeDims(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("T", "H", "E", "k", "I", "S", "E_local", "n_shared", "I_shared", "flags")]


class MoeWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_gate", "w_up", "w_down", "sh_gate", "sh_up", "sh_down")]


class MoeGating(C.Structure):
    _fields_ = [("bias", C.c_void_p), ("routed_scale", C.c_float), ("n_group", C.c_int32),
                ("topk_group", C.c_int32)]
    bias_tensor = None   # what gating() was given


class MoeTaps(C.Structure):
    _fields_ = [("topk_idx", C.c_void_p), ("topk_w", C.c_void_p), ("expert_load", C.c_void_p),
                ("offsets", C.c_void_p), ("perm_token", C.c_void_p), ("inv_pos", C.c_void_p),
                ("events", C.c_void_p * (2 * len(STAGES)))]
    tensors = {}   # by name, what make_taps was given


class MoeLinearDims(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("M", "N", "K", "G", "X")] +
                [(n, C.c_int64) for n in ("ldx", "ldw", "ldy")] + [("R", C.c_int32)])


class MoeWeightsI8(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_gate", "w_up", "w_down", "s_gate", "s_up", "s_down", "sh_gate", "sh_up",
                                          "sh_down", "sh_s_gate", "sh_s_up", "sh_s_down")]
    # of a handle that make_weights_i8 made: its device, and its experts, H, I and shared width
    device_index = sizes = None


class MoeWeightsF8(C.Structure):
    _fields_ = MoeWeightsI8._fields_
    # of a handle that make_weights_f8 made (see MoeWeightsI8)
    device_index = sizes = None


class MoeNorm(C.Structure):
    _fields_ = ([("H", C.c_int32), ("weight", C.c_void_p), ("post_weight", C.c_void_p)] +
                [(n, C.c_float) for n in ("residual_scale", "eps", "weight_add")])
    tensors = ()   # what norm() was given


class MoeNormIo(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("h", "h_out", "x", "q", "scale", "gate")] +
                [(n, C.c_int64) for n in ("ldh", "ldh_out", "ldx", "ldq", "gate_row", "gate_col")])
    tensors, shape = (), None   # what norm_io() was given, and (T, H)


class MoePlaceDims(C.Structure):
    _fields_ = [("L", C.c_int32), ("S", C.c_int32), ("E", C.c_int32), ("G", C.c_int32),
                ("alpha", C.c_double), ("beta", C.c_double), ("gamma", C.c_double),
                ("m_uniform", C.c_double)]


class MoeWindowDims(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("L", "S", "E", "G", "n_engines")]


class MoeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} ({status})")


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2606_15177_amd.build`")
    lib = C.CDLL(LIB_PATH)
    vp, i32, sz = C.c_void_p, C.c_int, C.c_size_t
    dp = C.POINTER(MoeDims)
    sig = {
        "moe_abi_version": ([], i32),
        "moe_strerror": ([i32], C.c_char_p),
        "moe_workspace_bytes": ([dp, i32], sz),
        "moe_validate": ([dp, i32, sz], i32),
        "moe_route": ([dp, C.POINTER(MoeGating), vp, vp, vp, vp], i32),
        "moe_route_stats": ([dp, vp, vp, vp, vp, vp], i32),
        "moe_permute": ([dp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp], i32),
        "moe_expert_ffn": ([dp, vp, vp, C.POINTER(MoeWeights), vp, vp, vp, vp, sz, vp], i32),
        "moe_combine": ([dp, vp, vp, vp, vp, vp, vp], i32),
        "moe_forward": ([dp, C.POINTER(MoeGating), vp, vp, vp, vp, C.POINTER(MoeWeights), vp, vp,
                         C.POINTER(MoeTaps), vp, sz, vp], i32),
        "moe_forward_noalloc": ([dp, C.POINTER(MoeGating), vp, vp, vp, vp, C.POINTER(MoeWeights), vp, vp,
                                 C.POINTER(MoeTaps), vp], i32),
        "moe_quantize_rows": ([C.c_int32, C.c_int32, vp, C.c_int64, vp, C.c_int64, vp, vp], i32),
        "moe_linear_i8": ([C.POINTER(MoeLinearDims), vp, vp, vp, vp, vp, vp], i32),
        "moe_grouped_linear_i8": ([C.POINTER(MoeLinearDims), vp, vp, vp, vp, vp, vp, vp, vp], i32),
        "moe_expert_ffn_i8": ([dp, vp, vp, C.POINTER(MoeWeightsI8), vp, vp, vp, vp, sz, vp], i32),
        "moe_forward_i8": ([dp, C.POINTER(MoeGating), vp, vp, vp, vp, C.POINTER(MoeWeightsI8), vp, vp,
                            C.POINTER(MoeTaps), vp, sz, vp], i32),
        "moe_norm_rows": ([C.POINTER(MoeNorm), C.POINTER(MoeNormIo), C.c_int32, vp, C.c_int64, vp], i32),
        "moe_quantize_rows_f8": ([C.c_int32, C.c_int32, vp, C.c_int64, vp, C.c_int64, vp, vp], i32),
        "moe_quantize_blocks_f8": ([C.c_int32, C.c_int32, C.c_int32, vp, C.c_int64, vp, C.c_int64, vp, vp], i32),
        "moe_linear_f8": ([C.POINTER(MoeLinearDims), vp, vp, vp, vp, vp, vp], i32),
        "moe_grouped_linear_f8": ([C.POINTER(MoeLinearDims), vp, vp, vp, vp, vp, vp, vp, vp], i32),
        "moe_expert_ffn_f8": ([dp, vp, vp, C.POINTER(MoeWeightsF8), vp, vp, vp, vp, sz, vp], i32),
        "moe_forward_f8": ([dp, C.POINTER(MoeGating), vp, vp, vp, vp, vp, vp, C.POINTER(MoeWeightsF8), vp, vp,
                            C.POINTER(MoeNorm), C.POINTER(MoeNormIo), C.POINTER(MoeTaps), vp, sz, vp], i32),
        "moe_place_slots": ([C.POINTER(MoePlaceDims), vp], sz),
        "moe_place_experts": ([C.POINTER(MoePlaceDims), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp], i32),
        "moe_window_stats": ([C.POINTER(MoeWindowDims), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp], i32),
    }
    for name, (args, res) in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res
    return lib


_lib = _load()


def header_functions() -> list[str]:
    """Names of the functions include/moe.h declares."""
    with open(HEADER) as f:
        text = f.read()
    return sorted(set(re.findall(r"\b(moe_[a-z0-9_]+)\s*\(", text)))


def strerror(status: int) -> str:
    return _lib.moe_strerror(status).decode()


def _check(status: int, where: str) -> None:
    if status != MOE_OK:
        raise MoeError(status, where)


def dims(T, H, E, k, I, S, E_local, n_shared=0, I_shared=0, flags=0) -> MoeDims:
    return MoeDims(T, H, E, k, I, S, E_local, n_shared, I_shared if n_shared else 0, flags)


def dims_of(cfg, **override) -> MoeDims:
    d = dict(cfg.dims)
    d["flags"] = getattr(cfg, "gate", 0)
    d.update(override)
    return dims(**d)


def workspace_bytes(d: MoeDims, entry: int) -> int:
    return int(_lib.moe_workspace_bytes(C.byref(d), entry))


def validate(d: MoeDims, entry: int = 0, ws_bytes: int = 0) -> int:
    return int(_lib.moe_validate(C.byref(d), entry, ws_bytes))


def _ptr(t, dtypes=None) -> int | None:
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch tensor")
    if not t.is_cuda:
        raise ValueError("tensor must live on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    if dtypes is not None and t.dtype not in dtypes:
        raise TypeError(f"dtype {t.dtype} not in {dtypes}")
    return t.data_ptr()


_BF16 = (torch.bfloat16, torch.int16, torch.uint16)
_I32 = (torch.int32,)
_I64 = (torch.int64,)
_F32 = (torch.float32,)
_F64 = (torch.float64,)


def _stream(stream) -> int | None:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def make_weights(w: dict) -> MoeWeights:
    return MoeWeights(_ptr(w["w_gate"], _BF16), _ptr(w["w_up"], _BF16), _ptr(w["w_down"], _BF16),
                      _ptr(w.get("sh_gate"), _BF16), _ptr(w.get("sh_up"), _BF16),
                      _ptr(w.get("sh_down"), _BF16))


def workspace(d: MoeDims, entry: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(workspace_bytes(d, entry), 1), dtype=torch.uint8, device=device)


def gating(bias=None, routed_scale=1.0, n_group=0, topk_group=0) -> MoeGating:
    """Parameters of the gate function that moe_dims.flags selects; bias is a
    device fp32 [E] tensor (sigmoid gates only)."""
    g = MoeGating(_ptr(bias, _F32), float(routed_scale), int(n_group), int(topk_group))
    g.bias_tensor = bias
    return g


def _gating_ref(g):
    return None if g is None else C.byref(g)


def route(d, logits, topk_idx, topk_w, stream=None, gating=None):
    _check(_lib.moe_route(C.byref(d), _gating_ref(gating), _ptr(logits, _F32), _ptr(topk_idx, _I32),
                          _ptr(topk_w, _F32), _stream(stream)), "moe_route")


def route_stats(d, src, topk_idx, counts, expert_load=None, stream=None):
    _check(_lib.moe_route_stats(C.byref(d), _ptr(src, _I32), _ptr(topk_idx, _I32), _ptr(counts, _I64),
                                _ptr(expert_load, _I32), _stream(stream)), "moe_route_stats")


def permute(d, topk_idx, local_experts, x, offsets, perm_token, inv_pos, x_perm, ws, stream=None):
    _check(_lib.moe_permute(C.byref(d), _ptr(topk_idx, _I32), _ptr(local_experts, _I32),
                            _ptr(x, _BF16), _ptr(offsets, _I32), _ptr(perm_token, _I32),
                            _ptr(inv_pos, _I32), _ptr(x_perm, _BF16), _ptr(ws),
                            0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)),
           "moe_permute")


def expert_ffn(d, x_perm, offsets, weights, x, y_perm, y_shared, ws, stream=None):
    w = weights if isinstance(weights, MoeWeights) else make_weights(weights)
    _check(_lib.moe_expert_ffn(C.byref(d), _ptr(x_perm, _BF16), _ptr(offsets, _I32), C.byref(w),
                               _ptr(x, _BF16), _ptr(y_perm, _BF16), _ptr(y_shared, _BF16), _ptr(ws),
                               0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)),
           "moe_expert_ffn")


def combine(d, y_perm, inv_pos, topk_w, y_shared, out, stream=None):
    _check(_lib.moe_combine(C.byref(d), _ptr(y_perm, _BF16), _ptr(inv_pos, _I32), _ptr(topk_w, _F32),
                            _ptr(y_shared, _BF16), _ptr(out, _BF16), _stream(stream)), "moe_combine")


def make_taps(topk_idx=None, topk_w=None, expert_load=None, offsets=None, perm_token=None,
              inv_pos=None, events=None) -> MoeTaps:
    t = MoeTaps(_ptr(topk_idx, _I32), _ptr(topk_w, _F32), _ptr(expert_load, _I32),
                _ptr(offsets, _I32), _ptr(perm_token, _I32), _ptr(inv_pos, _I32))
    t.tensors = {n: v for n, v in (("topk_idx", topk_idx), ("topk_w", topk_w), ("expert_load", expert_load),
                                   ("offsets", offsets), ("perm_token", perm_token), ("inv_pos", inv_pos)) if v is not None}
    if events is not None:
        for i, e in enumerate(events):
            t.events[i] = e  # None leaves the slot empty: that stage is not recorded
    return t


def forward(d, logits, src, x, local_experts, weights, counts, out, ws, taps=None, stream=None, gating=None):
    w = weights if isinstance(weights, MoeWeights) else make_weights(weights)
    _check(_lib.moe_forward(C.byref(d), _gating_ref(gating), _ptr(logits, _F32), _ptr(src, _I32), _ptr(x, _BF16),
                            _ptr(local_experts, _I32), C.byref(w), _ptr(counts, _I64),
                            _ptr(out, _BF16), None if taps is None else C.byref(taps), _ptr(ws),
                            0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)),
           "moe_forward")


def forward_noalloc(d, logits, src, x, local_experts, weights, counts, out, taps=None, stream=None, gating=None):
    """moe_forward_noalloc: the layer with the library's own scratch array as
    its workspace (no workspace argument, nothing allocated)."""
    w = weights if isinstance(weights, MoeWeights) else make_weights(weights)
    _check(_lib.moe_forward_noalloc(C.byref(d), _gating_ref(gating), _ptr(logits, _F32), _ptr(src, _I32),
                                    _ptr(x, _BF16), _ptr(local_experts, _I32), C.byref(w), _ptr(counts, _I64),
                                    _ptr(out, _BF16), None if taps is None else C.byref(taps), _stream(stream)),
           "moe_forward_noalloc")


# ---- 8-bit integer experts ----

_I8 = (torch.int8,)


# The handle of a device's current stream (torch.cuda.current_stream builds a
# Stream object each time: 2.8 us of a call that launches in 4).
_current_handle = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _on_device(stream, *tensors):
    """The tensors' device index and the stream to launch on: the given one, or
    that device's current stream.  Tensors of two devices, or a stream of another
    one, are refused."""
    dev = None
    for t in tensors:
        if t is not None:
            d = t.get_device()
            if d < 0:
                raise ValueError("tensor must live on the GPU")
            if dev is None:
                dev = d
            elif d != dev:
                raise ValueError(f"tensors live on different devices: cuda:{dev}, cuda:{d}")
    if stream is None:
        return dev, _current_handle(dev)
    if getattr(stream, "device", None) is not None and stream.device.index != dev:
        raise ValueError(f"stream of {stream.device}, tensors on cuda:{dev}")
    return dev, _stream(stream)


def _call(dev: int, where: str, *args) -> None:
    """A library call with `dev` as the current device."""
    f = getattr(_lib, where)
    if torch.cuda.current_device() == dev:
        status = f(*args)
    else:
        with torch.cuda.device(dev):
            status = f(*args)
    if status != MOE_OK:
        raise MoeError(status, where)


def _allocating_on(stream, dev: int):
    """Context in which tensors are allocated for use on `stream` of device dev,
    which may be a raw handle (0, and HIP's 1, stand for the default stream)."""
    if stream is not None and not isinstance(stream, torch.cuda.Stream):
        handle = _stream(stream)
        handle = getattr(handle, "value", handle) or 0
        stream = torch.cuda.ExternalStream(handle, device=dev) if handle > 1 else torch.cuda.default_stream(dev)
    return torch.cuda.stream(stream)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _fits(where: str, sizes: int) -> None:
    """Sizes (or'ed) of 31 bits in the C interface, which ctypes would cut to 32."""
    if sizes >> 31:
        raise MoeError(MOE_ERR_UNSUPPORTED, where)


def _pad16(n: int) -> int:
    return (n + 15) // 16 * 16


def _rows(t, dtypes, cols: int, what: str):
    """Pointer and row stride of a 2-D tensor of at least `cols` columns whose
    rows are contiguous."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a torch tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{what}: dtype {t.dtype} not in {dtypes}")
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[1] < cols:
        raise ValueError(f"{what}: expected rows of at least {cols} values, got {tuple(shape)}")
    if shape[1] != 1 and stride[1] != 1:
        raise ValueError(f"{what}: rows must be contiguous")
    # one row has no stride to speak of: 8-bit rows are asked for in whole 16s
    return t.data_ptr(), stride[0] if shape[0] > 1 else cols if t.element_size() == 1 else shape[1]


def _vec(t, dtypes, n: int, what: str):
    if not isinstance(t, torch.Tensor) or t.numel() < n:
        raise ValueError(f"{what}: expected {n} values")
    return _ptr(t, dtypes)


def _opt(t, dtypes, n: int, what: str):
    """_vec of a tensor that may be left out."""
    return None if t is None else _vec(t, dtypes, n, what)


def quantize_rows(x, q=None, scale=None, stream=None):
    """moe_quantize_rows: int8 rows and their fp32 scales of x, bf16 [rows,
    cols] (rows contiguous, any row stride).  q is int8 [rows, cols rounded up
    to a multiple of 16], padded with zeros; both are allocated when not given.
    Returns (q, scale)."""
    xp, ldx = _rows(x, _BF16, 1, "x")
    rows, cols = x.shape
    _fits("moe_quantize_rows", rows | cols)
    dev, st = _on_device(stream, x, q, scale)
    if q is None or scale is None:
        with _allocating_on(stream, dev):
            q = torch.empty((rows, _pad16(cols)), dtype=torch.int8, device=x.device) if q is None else q
            scale = torch.empty((rows,), dtype=torch.float32, device=x.device) if scale is None else scale
    qp, ldq = _rows(q, _I8, _pad16(cols), "q")
    _need(q.shape[0] == rows, "q: expected as many rows as x has")
    _call(dev, "moe_quantize_rows", rows, cols, xp, ldx, qp, ldq, _vec(scale, _F32, rows, "scale"), st)
    return q, scale


def linear_i8(K, xq, x_scale, wq, w_scale, y, stream=None):
    """moe_linear_i8: y [M, N] bf16 of xq [M, >= K padded to 16] and wq [N, the
    same] int8 with fp32 scales [M] and [N], as quantize_rows makes them.  The
    rows of xq, wq and y may lie apart."""
    yp, ldy = _rows(y, _BF16, 1, "y")
    M, N = y.shape
    xp, ldx = _rows(xq, _I8, _pad16(K), "xq")
    wp, ldw = _rows(wq, _I8, _pad16(K), "wq")
    _need(xq.shape[0] == M and wq.shape[0] == N, "expected as many rows of xq and wq as y has rows and columns")
    _fits("moe_linear_i8", M | N)
    dev, st = _on_device(stream, xq, x_scale, wq, w_scale, y)
    _call(dev, "moe_linear_i8", C.byref(MoeLinearDims(M, N, K, 1, 0, ldx, ldw, ldy)), xp, _vec(x_scale, _F32, M, "x_scale"),
          wp, _vec(w_scale, _F32, N, "w_scale"), yp, st)


def grouped_linear_i8(K, xq, x_scale, offsets, wq, w_scale, y, x_rows=None, stream=None, rows=None):
    """moe_grouped_linear_i8: rows offsets[g] .. offsets[g+1] of y [M, N] from
    those of xq (or xq[x_rows[r]]) and wq[g]; wq int8 [G, N, >= K padded to 16],
    w_scale fp32 [G, N], offsets int32 [G+1], x_rows int32 [M].  rows: how many of
    the M are expected to be in groups where y has room for more (the kernel is
    chosen by it; no result depends on it)."""
    yp, ldy = _rows(y, _BF16, 1, "y")
    M, N = y.shape
    if not isinstance(wq, torch.Tensor) or wq.dim() != 3 or wq.shape[1] != N:
        raise ValueError(f"wq: expected [groups, {N}, ...]")
    G = wq.shape[0]
    xp, ldx = _rows(xq, _I8, _pad16(K), "xq")
    wp, ldw = _rows(wq.flatten(0, 1), _I8, _pad16(K), "wq")
    _need(wp == wq.data_ptr(), "wq: the groups must lie one behind the other")
    _need(x_rows is not None or xq.shape[0] == M, "expected as many rows of xq as of y")
    _fits("moe_grouped_linear_i8", M | N | G | xq.shape[0])
    dev, st = _on_device(stream, xq, x_scale, offsets, wq, w_scale, y, x_rows)
    _call(dev, "moe_grouped_linear_i8", C.byref(MoeLinearDims(M, N, K, G, xq.shape[0], ldx, ldw, ldy, min(rows or 0, M))), xp,
          _vec(x_scale, _F32, xq.shape[0], "x_scale"), None if x_rows is None else _vec(x_rows, _I32, M, "x_rows"),
          _vec(offsets, _I32, G + 1, "offsets"), wp, _vec(w_scale, _F32, G * N, "w_scale"), yp, st)


def quantize_weights(d: MoeDims, w: dict) -> dict:
    """The int8 weights of a layer (moe_weights_i8's layout) from its bf16 ones
    (moe_weights' layout), a scale per output channel."""
    EL, H, I = d.E_local, d.H, d.I
    out = {}

    def put(name, scale_name, t, shape):
        q, s = quantize_rows(t)
        out[name], out[scale_name] = q.view(*shape, -1), s.view(*shape)

    put("w_gate", "s_gate", w["w_gate"].reshape(EL * I, H), (EL, I))
    put("w_up", "s_up", w["w_up"].reshape(EL * I, H), (EL, I))
    put("w_down", "s_down", w["w_down"].reshape(EL * H, I), (EL, H))
    if d.n_shared:
        width = d.n_shared * d.I_shared
        put("sh_gate", "sh_s_gate", w["sh_gate"].reshape(width, H), (width,))
        put("sh_up", "sh_s_up", w["sh_up"].reshape(width, H), (width,))
        down = w["sh_down"].reshape(d.n_shared, H, d.I_shared).permute(1, 0, 2).reshape(H, width)
        put("sh_down", "sh_s_down", down, (H,))
    return out


def make_weights_i8(d: MoeDims, w: dict) -> MoeWeightsI8:
    """The handle of int8 weights (see quantize_weights); it holds the tensors."""
    EL, H, I, width = d.E_local, d.H, d.I, d.n_shared * d.I_shared
    hp, ip, wp = _pad16(H), _pad16(I), _pad16(width)
    need = {"w_gate": (_I8, EL * I * hp), "w_up": (_I8, EL * I * hp), "w_down": (_I8, EL * H * ip),
            "s_gate": (_F32, EL * I), "s_up": (_F32, EL * I), "s_down": (_F32, EL * H)}
    if d.n_shared:
        need.update({"sh_gate": (_I8, width * hp), "sh_up": (_I8, width * hp), "sh_down": (_I8, H * wp),
                     "sh_s_gate": (_F32, width), "sh_s_up": (_F32, width), "sh_s_down": (_F32, H)})
    h = MoeWeightsI8(**{n: _vec(w.get(n), t, size, n) for n, (t, size) in need.items()})
    h.tensors = {n: w[n] for n in need}
    h.device_index = _on_device(None, *h.tensors.values())[0]
    h.sizes = (EL, H, I, width)
    return h


def _weights_i8(d: MoeDims, w, dev: int) -> MoeWeightsI8:
    """The handle w, or that of the dict w; refused where it was made for another
    device or other sizes (more experts, or shared ones that d does not have, are
    none)."""
    if isinstance(w, dict):
        w = make_weights_i8(d, w)
    elif not isinstance(w, MoeWeightsI8):
        raise TypeError(f"weights: expected int8 ones (make_weights_i8, quantize_weights), not a {type(w).__name__} or bf16 ones")
    return _handle_fits(d, w, dev)


def _handle_fits(d: MoeDims, w, dev: int):
    if w.sizes is not None:
        _need(w.device_index == dev, "weights live on another device")
        EL, H, I, width = w.sizes
        _need(EL >= d.E_local and H == d.H and I == d.I and (not d.n_shared or width == d.n_shared * d.I_shared),
              "weights were made for other sizes")
    return w


def _bytes(ws) -> int:
    return 0 if ws is None else ws.numel() * ws.element_size()


def expert_ffn_i8(d, x_perm, offsets, weights, x, y_perm, y_shared, ws, stream=None):
    """moe_expert_ffn_i8; weights as make_weights_i8 returns them, or its dict."""
    n, n_shared = d.T * d.k * d.H, d.T * d.H if d.n_shared else 0
    dev, st = _on_device(stream, x_perm, offsets, x, y_perm, y_shared, ws)
    weights = _weights_i8(d, weights, dev)
    _call(dev, "moe_expert_ffn_i8", C.byref(d), _vec(x_perm, _BF16, n, "x_perm"), _vec(offsets, _I32, d.E_local + 1, "offsets"),
          C.byref(weights), _opt(x, _BF16, n_shared, "x"), _vec(y_perm, _BF16, n, "y_perm"),
          _opt(y_shared, _BF16, n_shared, "y_shared"), _ptr(ws), _bytes(ws), st)


def forward_i8(d, logits, src, x, local_experts, weights, counts, out, ws, taps=None, stream=None, gating=None):
    """moe_forward_i8; weights as make_weights_i8 returns them, or its dict."""
    n = d.T * d.H
    tapped = {} if taps is None else taps.tensors
    bias = None if gating is None else gating.bias_tensor
    dev, st = _on_device(stream, logits, src, x, local_experts, counts, out, ws, bias, *tapped.values())
    for name, t in tapped.items():
        size = {"expert_load": d.E, "offsets": d.E_local + 1}.get(name, d.T * d.k)
        _need(t.numel() >= size, f"taps: {name}: expected {size} values")
    _need(bias is None or bias.numel() >= d.E, f"gating: bias: expected {d.E} values")
    weights = _weights_i8(d, weights, dev)
    _call(dev, "moe_forward_i8", C.byref(d), _gating_ref(gating), _vec(logits, _F32, d.T * d.E, "logits"),
          _opt(src, _I32, 0 if counts is None else d.T, "src"), _vec(x, _BF16, n, "x"),
          _opt(local_experts, _I32, d.E_local, "local_experts"), C.byref(weights), _opt(counts, _I64, d.S * d.E, "counts"),
          _vec(out, _BF16, n, "out"),
          None if taps is None else C.byref(taps), _ptr(ws), _bytes(ws), st)


# ---- norms around the layer ----

_F8 = (torch.float8_e4m3fn,)


def _blocks128(n: int) -> int:
    return (n + 127) // 128


def _strided_rows(t, T: int, H: int, what: str):
    """Pointer and row stride of a bf16 tensor [T, H]."""
    if isinstance(t, torch.Tensor) and t.dtype in _BF16 and t.shape == (T, H):
        row, col = t.stride()
        if (col == 1 or H == 1) and (row >= H or T == 1):
            return t.data_ptr(), row if T > 1 else H
    _rows(t, _BF16, H, what)   # (says what is wrong with its rows)
    _need(t.shape == (T, H), f"{what}: expected [{T}, {H}], got {tuple(t.shape)}")
    raise ValueError(f"{what}: rows overlap")


def norm(H, weight=None, post_weight=None, residual_scale=1.0, eps=1e-6, weight_add=0.0) -> MoeNorm:
    """The parameters of the norms around a block (moe_norm): bf16 [H] weights of
    the norm before the next block (None: without weights) and of the one after
    this block (None: no such norm).  The handle holds the tensors."""
    n = MoeNorm(H, _opt(weight, _BF16, H, "weight"), _opt(post_weight, _BF16, H, "post_weight"), float(residual_scale), float(eps),
                float(weight_add))
    n.tensors = tuple(t for t in (weight, post_weight) if t is not None)
    return n


def norm_io(h, h_out=None, x=None, q=None, scale=None, gate=None) -> MoeNormIo:
    """The rows of a call (moe_norm_io): h, h_out, x bf16 [T, H] (rows contiguous,
    any row stride), q float8_e4m3fn [T, H rounded up to 16], scale fp32 [T,
    ceil(H / 128)], gate bf16 [T or 1, H or 1].  It holds the tensors; a caller whose
    buffers stay keeps it."""
    if not isinstance(h, torch.Tensor) or h.dim() != 2:
        raise ValueError("h: expected a tensor [T, H]")
    T, H = h.shape
    _fits("moe_norm_rows", T | H)
    hp, ldh = _strided_rows(h, T, H, "h")
    tensors = [h]
    op = xp = qp = sp = gp = None
    ldo = ldx = ldq = gate_row = gate_col = 0
    if h_out is not None:
        op, ldo = _strided_rows(h_out, T, H, "h_out")
        tensors.append(h_out)
    if x is not None:
        xp, ldx = _strided_rows(x, T, H, "x")
        tensors.append(x)
    if q is not None or scale is not None:
        _need(q is not None and scale is not None, "q and scale: both or none")
        qp, ldq = _rows(q, _F8, _pad16(H), "q")
        _need(q.shape[0] == T, "q: expected as many rows as h has")
        _need(ldq >= _pad16(H), "q: rows overlap")
        if not isinstance(scale, torch.Tensor) or scale.dtype not in _F32:
            raise TypeError("scale: expected an fp32 tensor")
        _need(scale.numel() >= T * _blocks128(H) and scale.is_contiguous(), "scale: expected [T, ceil(H / 128)], contiguous")
        sp = scale.data_ptr()
        tensors += (q, scale)
    if gate is not None:
        if not isinstance(gate, torch.Tensor) or gate.dtype not in _BF16:
            raise TypeError("gate: expected a bf16 tensor")
        if gate.dim() != 2 or gate.shape[0] not in (1, T) or gate.shape[1] not in (1, H):
            raise ValueError(f"gate: expected [1 or {T}, 1 or {H}]")
        rows, cols = gate.shape
        row, col = gate.stride()
        _need(cols == 1 or col == 1, "gate: rows must be contiguous")
        _need(rows == 1 or cols == 1 or row >= H, "gate: rows overlap")
        gp, gate_row, gate_col = gate.data_ptr(), row if rows > 1 else 0, 1 if cols > 1 else 0
        tensors.append(gate)
    r = MoeNormIo(hp, op, xp, qp, sp, gp, ldh, ldo, ldx, ldq, gate_row, gate_col)
    r.tensors, r.shape = tensors, (T, H)
    return r


def norm_rows(norm: MoeNorm, rows: MoeNormIo, y=None, stream=None):
    """moe_norm_rows: the end of the block that computed y (bf16 [T, H], any row
    stride; None: a block's first norm) and the beginning of the next."""
    T, H = rows.shape
    if norm.H != H:
        raise ValueError(f"norm: made for {norm.H} columns, rows have {H}")
    yp, ldy = (None, 0) if y is None else _strided_rows(y, T, H, "y")
    dev, st = _on_device(stream, y, *rows.tensors, *norm.tensors)
    _call(dev, "moe_norm_rows", C.byref(norm), C.byref(rows), T, yp, ldy, st)


# ---- experts in 8-bit floating point ----


def quantize_rows_f8(x, q=None, scale=None, stream=None):
    """moe_quantize_rows_f8: e4m3 rows of x, bf16 [rows, cols] (rows contiguous,
    any row stride), and fp32 scales [rows, ceil(cols / 128)].  q is float8_e4m3fn
    [rows, cols rounded up to a multiple of 16], padded with zeros; both are
    allocated when not given.  Returns (q, scale)."""
    xp, ldx = _rows(x, _BF16, 1, "x")
    rows, cols = x.shape
    _fits("moe_quantize_rows_f8", rows | cols)
    dev, st = _on_device(stream, x, q, scale)
    if q is None or scale is None:
        with _allocating_on(stream, dev):
            q = torch.empty((rows, _pad16(cols)), dtype=_F8[0], device=x.device) if q is None else q
            scale = torch.empty((rows, _blocks128(cols)), dtype=torch.float32, device=x.device) if scale is None else scale
    qp, ldq = _rows(q, _F8, _pad16(cols), "q")
    _need(q.shape[0] == rows, "q: expected as many rows as x has")
    _call(dev, "moe_quantize_rows_f8", rows, cols, xp, ldx, qp, ldq, _vec(scale, _F32, rows * _blocks128(cols), "scale"), st)
    return q, scale


def _matrices(t, dtypes, G: int, rows: int, cols: int, what: str):
    """Pointer and row stride of G matrices one behind the other."""
    _need(tuple(t.shape[:2]) == (G, rows), f"{what}: expected [{G}, {rows}, ...]")
    flat = t.flatten(0, 1)
    p, ld = _rows(flat, dtypes, cols, what)
    _need(p == t.data_ptr(), f"{what}: the matrices must lie one behind the other")
    return p, ld


def quantize_blocks_f8(x, q=None, scale=None, stream=None):
    """moe_quantize_blocks_f8: e4m3 matrices of x, bf16 [rows, cols] or [G, rows,
    cols], with an fp32 scale for each 128 x 128 block: [G,] ceil(rows / 128),
    ceil(cols / 128).  q as quantize_rows_f8's.  Returns (q, scale)."""
    if not isinstance(x, torch.Tensor) or x.dim() not in (2, 3):
        raise ValueError("x: expected a tensor [rows, cols] or [G, rows, cols]")
    one = x.dim() == 2
    x3 = x.unsqueeze(0) if one else x
    G, rows, cols = x3.shape
    _fits("moe_quantize_blocks_f8", G | rows | cols)
    xp, ldx = _matrices(x3, _BF16, G, rows, 1, "x")
    dev, st = _on_device(stream, x, q, scale)
    if q is None or scale is None:
        with _allocating_on(stream, dev):
            lead = () if one else (G,)
            q = torch.empty((*lead, rows, _pad16(cols)), dtype=_F8[0], device=x.device) if q is None else q
            scale = (torch.empty((*lead, _blocks128(rows), _blocks128(cols)), dtype=torch.float32, device=x.device)
                     if scale is None else scale)
    _need(q.dim() == x.dim(), "q: expected as many dimensions as x has")
    qp, ldq = _matrices(q.unsqueeze(0) if one else q, _F8, G, rows, _pad16(cols), "q")
    _call(dev, "moe_quantize_blocks_f8", G, rows, cols, xp, ldx, qp, ldq,
          _vec(scale, _F32, G * _blocks128(rows) * _blocks128(cols), "scale"), st)
    return q, scale


def linear_f8(K, xq, x_scale, wq, w_scale, y, stream=None):
    """moe_linear_f8: y [M, N] bf16 of xq [M, >= K padded to 16] and wq [N, the
    same] e4m3 with fp32 scales [M, ceil(K / 128)] and [ceil(N / 128), ceil(K /
    128)], as quantize_rows_f8 and quantize_blocks_f8 make them.  The rows of xq,
    wq and y may lie apart."""
    yp, ldy = _rows(y, _BF16, 1, "y")
    M, N = y.shape
    xp, ldx = _rows(xq, _F8, _pad16(K), "xq")
    wp, ldw = _rows(wq, _F8, _pad16(K), "wq")
    _need(xq.shape[0] == M and wq.shape[0] == N, "expected as many rows of xq and wq as y has rows and columns")
    _fits("moe_linear_f8", M | N)
    dev, st = _on_device(stream, xq, x_scale, wq, w_scale, y)
    kb = _blocks128(K)
    _call(dev, "moe_linear_f8", C.byref(MoeLinearDims(M, N, K, 1, 0, ldx, ldw, ldy)), xp, _vec(x_scale, _F32, M * kb, "x_scale"),
          wp, _vec(w_scale, _F32, _blocks128(N) * kb, "w_scale"), yp, st)


def grouped_linear_f8(K, xq, x_scale, offsets, wq, w_scale, y, x_rows=None, stream=None, rows=None):
    """moe_grouped_linear_f8: rows offsets[g] .. offsets[g+1] of y [M, N] from those
    of xq (or xq[x_rows[r]]) and wq[g]; wq e4m3 [G, N, >= K padded to 16], w_scale
    fp32 [G, ceil(N / 128), ceil(K / 128)]; offsets, x_rows and rows as
    grouped_linear_i8's."""
    yp, ldy = _rows(y, _BF16, 1, "y")
    M, N = y.shape
    if not isinstance(wq, torch.Tensor) or wq.dim() != 3 or wq.shape[1] != N:
        raise ValueError(f"wq: expected [groups, {N}, ...]")
    G = wq.shape[0]
    xp, ldx = _rows(xq, _F8, _pad16(K), "xq")
    wp, ldw = _matrices(wq, _F8, G, N, _pad16(K), "wq")
    _need(x_rows is not None or xq.shape[0] == M, "expected as many rows of xq as of y")
    _fits("moe_grouped_linear_f8", M | N | G | xq.shape[0])
    dev, st = _on_device(stream, xq, x_scale, offsets, wq, w_scale, y, x_rows)
    kb = _blocks128(K)
    _call(dev, "moe_grouped_linear_f8", C.byref(MoeLinearDims(M, N, K, G, xq.shape[0], ldx, ldw, ldy, min(rows or 0, M))), xp,
          _vec(x_scale, _F32, xq.shape[0] * kb, "x_scale"), None if x_rows is None else _vec(x_rows, _I32, M, "x_rows"),
          _vec(offsets, _I32, G + 1, "offsets"), wp, _vec(w_scale, _F32, G * _blocks128(N) * kb, "w_scale"), yp, st)


def quantize_weights_f8(d: MoeDims, w: dict) -> dict:
    """The e4m3 weights of a layer (moe_weights_f8's layout) from its bf16 ones
    (moe_weights' layout), a scale per 128 x 128 block."""
    EL, H, I = d.E_local, d.H, d.I
    out = {}
    for n, rows, cols in (("gate", I, H), ("up", I, H), ("down", H, I)):
        out["w_" + n], out["s_" + n] = quantize_blocks_f8(w["w_" + n].reshape(EL, rows, cols))
    if d.n_shared:
        width = d.n_shared * d.I_shared
        for n in ("gate", "up"):
            out["sh_" + n], out["sh_s_" + n] = quantize_blocks_f8(w["sh_" + n].reshape(width, H))
        down = w["sh_down"].reshape(d.n_shared, H, d.I_shared).permute(1, 0, 2).reshape(H, width)
        out["sh_down"], out["sh_s_down"] = quantize_blocks_f8(down)
    return out


def make_weights_f8(d: MoeDims, w: dict) -> MoeWeightsF8:
    """The handle of e4m3 weights (see quantize_weights_f8); it holds the tensors."""
    EL, H, I, width = d.E_local, d.H, d.I, d.n_shared * d.I_shared
    hp, ip, wp = _pad16(H), _pad16(I), _pad16(width)
    hb, ib, wb = _blocks128(H), _blocks128(I), _blocks128(width)
    need = {"w_gate": (_F8, EL * I * hp), "w_up": (_F8, EL * I * hp), "w_down": (_F8, EL * H * ip),
            "s_gate": (_F32, EL * ib * hb), "s_up": (_F32, EL * ib * hb), "s_down": (_F32, EL * hb * ib)}
    if d.n_shared:
        need.update({"sh_gate": (_F8, width * hp), "sh_up": (_F8, width * hp), "sh_down": (_F8, H * wp),
                     "sh_s_gate": (_F32, wb * hb), "sh_s_up": (_F32, wb * hb), "sh_s_down": (_F32, hb * wb)})
    h = MoeWeightsF8(**{n: _vec(w.get(n), t, size, n) for n, (t, size) in need.items()})
    h.tensors = {n: w[n] for n in need}
    h.device_index = _on_device(None, *h.tensors.values())[0]
    h.sizes = (EL, H, I, width)
    return h


def _weights_f8(d: MoeDims, w, dev: int) -> MoeWeightsF8:
    """As _weights_i8."""
    if isinstance(w, dict):
        w = make_weights_f8(d, w)
    elif not isinstance(w, MoeWeightsF8):
        raise TypeError(f"weights: expected e4m3 ones (make_weights_f8, quantize_weights_f8), not a {type(w).__name__} or other ones")
    return _handle_fits(d, w, dev)


def expert_ffn_f8(d, x_perm, offsets, weights, x, y_perm, y_shared, ws, stream=None):
    """moe_expert_ffn_f8; weights as make_weights_f8 returns them, or its dict."""
    n, n_shared = d.T * d.k * d.H, d.T * d.H if d.n_shared else 0
    dev, st = _on_device(stream, x_perm, offsets, x, y_perm, y_shared, ws)
    weights = _weights_f8(d, weights, dev)
    _call(dev, "moe_expert_ffn_f8", C.byref(d), _vec(x_perm, _BF16, n, "x_perm"), _vec(offsets, _I32, d.E_local + 1, "offsets"),
          C.byref(weights), _opt(x, _BF16, n_shared, "x"), _vec(y_perm, _BF16, n, "y_perm"),
          _opt(y_shared, _BF16, n_shared, "y_shared"), _ptr(ws), _bytes(ws), st)


def forward_f8(d, logits, src, x, local_experts, weights, counts, out, ws, taps=None, stream=None, gating=None, xq=None,
               x_scale=None, norm=None, rows=None):
    """moe_forward_f8; weights as make_weights_f8 returns them, or its dict.  x is
    bf16 [T, H], or None with the same rows quantised, xq and x_scale, as
    quantize_rows_f8 and norm_rows leave them (dense).  norm and rows (see norm,
    norm_io): the layer's output goes through moe_norm_rows; out may then be
    None."""
    n = d.T * d.H
    tapped = {} if taps is None else taps.tensors
    bias = None if gating is None else gating.bias_tensor
    _need((norm is None) == (rows is None), "norm and rows: both or none")
    _need((xq is None) == (x_scale is None) and (x is None) != (xq is None), "rows to the layer: x, or xq and x_scale")
    ends = () if norm is None else (*norm.tensors, *rows.tensors)
    dev, st = _on_device(stream, logits, src, x, xq, x_scale, local_experts, counts, out, ws, bias, *tapped.values(), *ends)
    for name, t in tapped.items():
        size = {"expert_load": d.E, "offsets": d.E_local + 1}.get(name, d.T * d.k)
        _need(t.numel() >= size, f"taps: {name}: expected {size} values")
    _need(bias is None or bias.numel() >= d.E, f"gating: bias: expected {d.E} values")
    if norm is not None:
        _need(rows.shape == (d.T, d.H), f"rows: expected [{d.T}, {d.H}], got {rows.shape}")
    weights = _weights_f8(d, weights, dev)
    _call(dev, "moe_forward_f8", C.byref(d), _gating_ref(gating), _vec(logits, _F32, d.T * d.E, "logits"),
          _opt(src, _I32, 0 if counts is None else d.T, "src"), _opt(x, _BF16, n, "x"),
          _opt(xq, _F8, d.T * _pad16(d.H), "xq"), _opt(x_scale, _F32, d.T * _blocks128(d.H), "x_scale"),
          _opt(local_experts, _I32, d.E_local, "local_experts"), C.byref(weights), _opt(counts, _I64, d.S * d.E, "counts"),
          _opt(out, _BF16, n, "out"), None if norm is None else C.byref(norm), None if rows is None else C.byref(rows),
          None if taps is None else C.byref(taps), _ptr(ws), _bytes(ws), st)


PAPER_PLACE_WEIGHTS = (1.0, 0.0025, 1.0)  # (alpha, beta, gamma), Sec. 6


def place_dims(L, S, E, G, alpha=1.0, beta=0.0025, gamma=1.0, m_uniform=1.0) -> MoePlaceDims:
    return MoePlaceDims(L, S, E, G, alpha, beta, gamma, m_uniform)


def _host_i32(a):
    import numpy as np
    a = np.ascontiguousarray(a.cpu().numpy() if isinstance(a, torch.Tensor) else a, dtype=np.int32)
    return a, a.ctypes.data_as(C.c_void_p)


def place_slots(pd: MoePlaceDims, cap) -> int:
    cap_h, cap_p = _host_i32(cap)
    return int(_lib.moe_place_slots(C.byref(pd), cap_p))


def place_experts(pd: MoePlaceDims, cap, A, D, x0, x, B=None, M=None, rank_experts=None, cost=None,
                  stream=None):
    """moe_place_experts: cap is a host sequence of G ints, every tensor lives
    on the GPU (A int64 [L,S,E], D fp64 [S,G], x0/x int32 [L,E], B int64 [L,E],
    M fp64 [L,E,G], rank_experts int32 [L,G,slots], cost fp64 [L,3])."""
    cap_h, cap_p = _host_i32(cap)
    _check(_lib.moe_place_experts(C.byref(pd), cap_p, _ptr(A, _I64), _ptr(B, _I64), _ptr(D, _F64),
                                  _ptr(M, _F64), _ptr(x0, _I32), _ptr(x, _I32), _ptr(rank_experts, _I32),
                                  _ptr(cost, _F64), _stream(stream)), "moe_place_experts")


def window_stats(wd: MoeWindowDims, A, x, home, remote, total, rank_load, B=None, engine=None, pressure=None,
                 stream=None):
    """moe_window_stats: every tensor on the GPU (A int64 [L,S,E], x int32
    [L,E], home int32 [S], engine int32 [G]; outputs remote/total int64 [L,S],
    rank_load int64 [L,G], pressure fp64 [n_engines])."""
    _check(_lib.moe_window_stats(C.byref(wd), _ptr(A, _I64), _ptr(B, _I64), _ptr(x, _I32), _ptr(home, _I32),
                                 _ptr(engine, _I32), _ptr(remote, _I64), _ptr(total, _I64),
                                 _ptr(rank_load, _I64), _ptr(pressure, _F64), _stream(stream)),
           "moe_window_stats")


class MoeLayer:
    """One GPU's MoE layer with its weights resident in HBM.

    Holds the bf16 weights, the placement list and a forward workspace, and
    calls moe_forward.  ``counts`` (int64 [S, E]) is the caller's source x
    expert matrix for this layer, accumulated by every call."""

    def __init__(self, d: MoeDims, weights: dict, local_experts=None, device="cuda", gating=None):
        self.d = d
        self.gating = gating   # MoeGating for the gate function d.flags selects (None: defaults)
        self.weights = {k: v for k, v in weights.items() if v is not None}
        self.local_experts = local_experts
        self._w = make_weights(self.weights)
        self.ws = workspace(d, ENTRY_FORWARD, device)
        self.device = device

    def forward(self, logits, src, x, counts=None, out=None, taps=None, stream=None):
        if out is None:
            out = torch.empty((self.d.T, self.d.H), dtype=torch.bfloat16, device=self.device)
        forward(self.d, logits, src, x, self.local_experts, self._w, counts, out, self.ws, taps, stream,
                gating=self.gating)
        return out


class MoeLayerI8:
    """MoeLayer on int8 experts: the weights are quantised once (bf16 ones, in
    MoeLayer's layout) or taken as they are (quantize_weights' dict), and
    forward calls moe_forward_i8.  Calls that may overlap (other streams, other
    captured graphs replayed at the same time) each need a workspace of their
    own: workspace(d, ENTRY_FORWARD_I8), given to forward as `ws`."""

    def __init__(self, d: MoeDims, weights: dict, local_experts=None, device="cuda", gating=None):
        self.d = d
        self.gating = gating
        self.local_experts = local_experts
        self._w = make_weights_i8(d, weights if "s_gate" in weights else quantize_weights(d, weights))
        self.ws = workspace(d, ENTRY_FORWARD_I8, device)
        self.device = device

    def forward(self, logits, src, x, counts=None, out=None, taps=None, stream=None, ws=None):
        if out is None:
            with _allocating_on(stream, _on_device(stream, x)[0]):
                out = torch.empty((self.d.T, self.d.H), dtype=torch.bfloat16, device=x.device)
        forward_i8(self.d, logits, src, x, self.local_experts, self._w, counts, out, self.ws if ws is None else ws, taps,
                   stream, gating=self.gating)
        return out


class MoeLayerF8:
    """MoeLayer on e4m3 experts: the weights are quantised once (bf16 ones, in
    MoeLayer's layout) or taken as they are (quantize_weights_f8's dict), and
    forward calls moe_forward_f8.  With `norm` and `rows` the norms after the
    layer are its end, and it returns None unless `out` is given.  Calls that may
    overlap each need a workspace of their own: workspace(d, ENTRY_FORWARD_F8),
    given to forward as `ws`."""

    def __init__(self, d: MoeDims, weights: dict, local_experts=None, device="cuda", gating=None):
        self.d = d
        self.gating = gating
        self.local_experts = local_experts
        self._w = make_weights_f8(d, weights if "s_gate" in weights else quantize_weights_f8(d, weights))
        self.ws = workspace(d, ENTRY_FORWARD_F8, device)
        self.device = device

    def forward(self, logits, src, x=None, counts=None, out=None, taps=None, stream=None, ws=None, xq=None, x_scale=None,
                norm=None, rows=None):
        if out is None and norm is None:
            dev = _on_device(stream, x, xq)[0]
            with _allocating_on(stream, dev):
                out = torch.empty((self.d.T, self.d.H), dtype=torch.bfloat16, device=torch.device("cuda", dev))
        forward_f8(self.d, logits, src, x, self.local_experts, self._w, counts, out, self.ws if ws is None else ws, taps,
                   stream, gating=self.gating, xq=xq, x_scale=x_scale, norm=norm, rows=rows)
        return out
