"""Python binding of libimbd.so: the gfx950 hot path of integrated model/batch/domain
parallel SGD (Gholami et al., arXiv:1712.04432).

Functions carry the names of the C ABI in include/imbd.h and marshal arguments (those of the
expert layer and of AdamW also check the tensors against each other): torch tensors supply
device pointers and the current HIP stream; every step of the path runs in the library's
kernels. Missing library -> RuntimeError (no fallback).

bf16 tensors are torch.bfloat16 (the bytes are bf16 bit patterns), fp32 tensors
torch.float32. Activations are [B][d] (one sample per row, the paper's column-major
X_i); weights [d_out][d_in].
"""
from __future__ import annotations

import ctypes

from ._abi import (IMBD_BF16, IMBD_F32, IMBD_K_BIAS, IMBD_K_CAST, IMBD_K_CONV_DGRAD,  # noqa: F401
                   IMBD_K_CONV_FWD, IMBD_K_CONV_WGRAD, IMBD_K_GEMM_DW, IMBD_K_GEMM_DX,
                   IMBD_K_GEMM_FWD, IMBD_K_SGD, IMBD_K_SOFTMAX, IMBD_K_SPLITK, IMBD_K_EXPERT_FWD,
                   IMBD_K_EXPERT_DX, IMBD_K_EXPERT_DW, IMBD_K_ROUTE, IMBD_K_COMBINE, IMBD_K_ADAMW, IMBD_OK,
                   IMBD_EINVAL, IMBD_EUNSUPPORTED, IMBD_EHIP, IMBD_EWORKSPACE,
                   IMBD_WS_ACT, IMBD_WS_DY, IMBD_WS_LOGITS, IMBD_WS_ROWLOSS, AdamWTensor, ImbdError,
                   Layer, MlpDesc, check, load)
from ._abi import IMBD_STATIC_SCRATCH_BYTES  # noqa: F401
from ._abi import (IMBD_OPT_CONV_NT, IMBD_OPT_COUNT, IMBD_OPT_DW_GENERIC, IMBD_OPT_DW_STREAM,  # noqa: F401
                   IMBD_OPT_DW_WIDE_DUAL, IMBD_OPT_DW_WIDE_MIN_K, IMBD_OPT_LOCAL_PAIR, IMBD_OPT_GEMM_CFG, IMBD_OPT_GEMM_SPLITS, IMBD_OPT_SKINNY_OFF,
                   IMBD_OPT_SKINNY_NB, IMBD_OPT_SKINNY_SPLITS, IMBD_OPT_TOP_UNFUSED, IMBD_OPT_WIDE_OFF,
                   IMBD_OPT_WIDE_SPLITS, IMBD_OPT_REDUCE_TAIL)

__all__ = [
    "load", "ImbdError", "MLP", "mlp_workspace_bytes", "mlp_workspace_offset", "mlp_fwd",
    "mlp_bwd", "mlp_train_step", "mlp_train_step_static", "sgd_step", "cast_f32_bf16", "softmax_xent", "mlp_local_fwd",
    "mlp_local_bwd", "mlp_local_workspace_bytes", "conv3x3_tile_fwd", "conv3x3_tile_dgrad",
    "conv3x3_tile_wgrad", "conv3x3_tile_bwd", "conv3x3_wgrad_workspace_bytes", "timing_begin",
    "timing_end",
    "expert_route_workspace_bytes", "expert_route", "expert_route_bwd", "expert_fwd", "expert_bwd",
    "expert_combine", "expert_combine_bwd", "AdamW", "adamw_step",
    "ws_view", "dtype_code", "set_option", "get_option", "option_name", "options",
]


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def dtype_code(t_or_dtype) -> int:
    torch = _torch()
    dt = t_or_dtype.dtype if hasattr(t_or_dtype, "dtype") else t_or_dtype
    if dt == torch.bfloat16:
        return IMBD_BF16
    if dt == torch.float32:
        return IMBD_F32
    raise TypeError(f"unsupported dtype {dt}")


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    torch = _torch()
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


class MLP:
    """Shape of a network: widths d_0..d_L, batch B, operand type ('bf16' or 'f32')."""

    def __init__(self, dims, batch: int, dtype: str = "bf16"):
        self.dims = [int(d) for d in dims]
        self.batch = int(batch)
        self.dtype = dtype
        self.code = IMBD_BF16 if dtype == "bf16" else IMBD_F32
        self._dims_arr = (ctypes.c_int * len(self.dims))(*self.dims)
        self._desc = MlpDesc(len(self.dims) - 1, self._dims_arr, self.batch, self.code)

    @property
    def n_layers(self):
        return len(self.dims) - 1

    @property
    def desc(self):
        return ctypes.byref(self._desc)

    def torch_dtype(self):
        torch = _torch()
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32


def _layers(layers):
    """layers: sequence of dicts with keys w, w_lp, b, (dw, db) -> ctypes Layer array."""
    arr = (Layer * len(layers))()
    for i, l in enumerate(layers):
        arr[i].w = l["w"].data_ptr()
        arr[i].w_lp = l["w_lp"].data_ptr()
        arr[i].b = l["b"].data_ptr()
        arr[i].dw = l["dw"].data_ptr() if l.get("dw") is not None else None
        arr[i].db = l["db"].data_ptr() if l.get("db") is not None else None
    return arr


def mlp_workspace_bytes(net: MLP) -> int:
    n = load().mlp_workspace_bytes(net.desc)
    if n == 0:
        raise ImbdError(IMBD_EINVAL, "mlp_workspace_bytes")
    return n


def mlp_workspace_offset(net: MLP, kind: int, layer: int = 0) -> int:
    off = load().mlp_workspace_offset(net.desc, kind, layer)
    if off < 0:
        raise ImbdError(IMBD_EINVAL, "mlp_workspace_offset")
    return off


def ws_view(net: MLP, ws, kind: int, layer: int = 0):
    """A tensor view of one workspace region (activations, logits, Delta_Y, row losses)."""
    torch = _torch()
    off = mlp_workspace_offset(net, kind, layer)
    B = net.batch
    if kind == IMBD_WS_ACT:
        shape, dt = (B, net.dims[layer]), net.torch_dtype()
    elif kind == IMBD_WS_LOGITS:
        shape, dt = (B, net.dims[-1]), torch.float32
    elif kind == IMBD_WS_DY:
        shape, dt = (B, net.dims[layer]), net.torch_dtype()
    else:
        shape, dt = (B,), torch.float32
    esz = torch.empty((), dtype=dt).element_size()
    n = 1
    for s in shape:
        n *= s
    return ws[off:off + n * esz].view(dt).view(shape)


def mlp_fwd(net: MLP, layers, x, labels, ws, loss, stream=None):
    lib = load()
    arr = _layers(layers)
    check(lib.mlp_fwd(net.desc, arr, _ptr(x), _ptr(labels), _ptr(ws), ws.numel() * ws.element_size(),
                      _ptr(loss), _stream(stream)), "mlp_fwd")


def mlp_bwd(net: MLP, layers, x, ws, fuse_sgd: bool, lr: float, dx1=None, stream=None):
    lib = load()
    arr = _layers(layers)
    check(lib.mlp_bwd(net.desc, arr, _ptr(x), _ptr(ws), ws.numel() * ws.element_size(), int(bool(fuse_sgd)),
                      float(lr), _ptr(dx1), _stream(stream)), "mlp_bwd")


def mlp_train_step(net: MLP, layers, x, labels, ws, lr: float, loss, stream=None):
    lib = load()
    arr = _layers(layers)
    check(lib.mlp_train_step(net.desc, arr, _ptr(x), _ptr(labels), _ptr(ws), ws.numel() * ws.element_size(),
                             float(lr), _ptr(loss), _stream(stream)), "mlp_train_step")


def mlp_train_step_static(net: MLP, layers, x, labels, lr: float, loss, stream=None):
    """mlp_train_step on the library's static scratch (no workspace argument, no allocation)."""
    lib = load()
    arr = _layers(layers)
    check(lib.mlp_train_step_static(net.desc, arr, _ptr(x), _ptr(labels), float(lr), _ptr(loss), _stream(stream)),
          "mlp_train_step_static")


def sgd_step(w, grad, lr: float, grad_scale: float = 1.0, w_lp=None, stream=None):
    lib = load()
    check(lib.sgd_step(_ptr(w), _ptr(w_lp), IMBD_BF16 if w_lp is not None else IMBD_F32, _ptr(grad),
                       w.numel(), float(lr), float(grad_scale), _stream(stream)), "sgd_step")


def cast_f32_bf16(src, dst, stream=None):
    lib = load()
    check(lib.cast_f32_bf16(_ptr(src), _ptr(dst), src.numel(), _stream(stream)), "cast_f32_bf16")


def softmax_xent(logits, labels, inv_batch: float, loss, row_loss, dz=None, stream=None):
    lib = load()
    B, C = logits.shape
    check(lib.softmax_xent(B, C, _ptr(logits), logits.stride(0), _ptr(labels), float(inv_batch), _ptr(loss),
                           _ptr(row_loss), _ptr(dz), dz.stride(0) if dz is not None else C,
                           dtype_code(dz) if dz is not None else IMBD_F32, _stream(stream)), "softmax_xent")


def mlp_local_workspace_bytes(which: int, dtype_: int, d_out_blk: int, d_in: int, b_blk: int) -> int:
    return load().mlp_local_workspace_bytes(which, dtype_, d_out_blk, d_in, b_blk)


def _ld(t):
    return t.stride(0) if t is not None else 0


def mlp_local_fwd(w_blk, x_blk, y_blk, P_r: int, P_c: int, bias=None, relu: bool = False, ws=None,
                  stream=None):
    """Y_blk = W_blk X_blk (+bias, ReLU) for one process of the P_r x P_c grid."""
    lib = load()
    d_out, d_in = w_blk.shape
    b_blk = x_blk.shape[0]
    check(lib.mlp_local_fwd(dtype_code(w_blk), int(relu), P_r, P_c, d_out, d_in, b_blk, _ptr(w_blk),
                            _ld(w_blk), _ptr(bias), _ptr(x_blk), _ld(x_blk), _ptr(y_blk), _ld(y_blk),
                            dtype_code(y_blk), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                            _stream(stream)), "mlp_local_fwd")


def mlp_local_bwd(w_blk, dy_blk, x_blk, dw_part, P_r: int, P_c: int, db_part=None, dx_part=None,
                  mask_relu: bool = False, ws=None, stream=None):
    lib = load()
    d_out, d_in = w_blk.shape
    b_blk = x_blk.shape[0]
    check(lib.mlp_local_bwd(dtype_code(w_blk), P_r, P_c, d_out, d_in, b_blk, _ptr(w_blk), _ld(w_blk),
                            _ptr(dy_blk), _ld(dy_blk), _ptr(x_blk), _ld(x_blk), _ptr(dw_part), _ld(dw_part),
                            _ptr(db_part), _ptr(dx_part), _ld(dx_part), int(bool(mask_relu)), _ptr(ws),
                            0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)),
          "mlp_local_bwd")


def conv3x3_tile_fwd(x_pad, w, y, stream=None):
    lib = load()
    N, Hp, Wp, Ci = x_pad.shape
    check(lib.conv3x3_tile_fwd(N, Hp - 2, Wp - 2, Ci, w.shape[0], _ptr(x_pad), _ptr(w), _ptr(y),
                               dtype_code(y), _stream(stream)), "conv3x3_tile_fwd")


def conv3x3_tile_dgrad(dy_pad, w, dx, stream=None):
    lib = load()
    N, Hp, Wp, Co = dy_pad.shape
    check(lib.conv3x3_tile_dgrad(N, Hp - 2, Wp - 2, w.shape[3], Co, _ptr(dy_pad), _ptr(w), _ptr(dx),
                                 dtype_code(dx), _stream(stream)), "conv3x3_tile_dgrad")


def conv3x3_wgrad_workspace_bytes(N, H, W, Ci, Co) -> int:
    return load().conv3x3_wgrad_workspace_bytes(N, H, W, Ci, Co)


def conv3x3_tile_wgrad(x_pad, dy_pad, dw, ws=None, stream=None):
    lib = load()
    N, Hp, Wp, Ci = x_pad.shape
    check(lib.conv3x3_tile_wgrad(N, Hp - 2, Wp - 2, Ci, dy_pad.shape[3], _ptr(x_pad), _ptr(dy_pad), _ptr(dw),
                                 _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                 _stream(stream)), "conv3x3_tile_wgrad")


def conv3x3_tile_bwd(x_pad, w, dy_pad, dw, dx=None, ws=None, stream=None):
    """Input gradient (skipped when dx is None) and partial weight gradient of the tile."""
    lib = load()
    N, Hp, Wp, Ci = x_pad.shape
    check(lib.conv3x3_tile_bwd(N, Hp - 2, Wp - 2, Ci, dy_pad.shape[3], _ptr(x_pad), _ptr(w), _ptr(dy_pad),
                               _ptr(dx), dtype_code(dx) if dx is not None else IMBD_BF16, _ptr(dw), _ptr(ws),
                               0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)),
          "conv3x3_tile_bwd")


# ------------------------------------------------------------------- a layer of experts
# These take their sizes from several tensors at once, and the kernels trust them, so the
# tensors are checked against each other here (ValueError, TypeError); everything else is
# checked by the library (ImbdError). Sizes reach it as C ints, of which ctypes keeps the low 32 bits:
# larger ones are refused here too (ValueError).
def _sizes(t, shape, dtype, name, device, whole=False):
    """Shape, type, device (its index) and layout of one tensor: rows without gaps between elements,
    or (whole) contiguous. Returns its address."""
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, need {tuple(shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {t.dtype}, need {dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, need cuda:{device}")
    if not t.is_contiguous() and (whole or (t.shape[-1] > 1 and t.stride(-1) != 1)):
        raise ValueError(f"{name}: strides {t.stride()}")
    return t.data_ptr()


def _here(t, name):
    """The index of the tensor's device, which has to be the current one (the stream is taken from
    it)."""
    dev = t.get_device()
    if dev < 0 or dev != _torch()._C._cuda_getDevice():
        raise ValueError(f"{name}: on {t.device}, which is not the current device")
    return dev


def _too_large(*sizes):
    raise ValueError(f"sizes {sizes}: each has to be under 2^31")


def _on(stream, device):
    """The address of a stream, or of the device's current one."""
    return _torch()._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _rows_ld(t):
    """Leading dimension of a matrix, or of each matrix of a batch. (Of a single row, whose
    stride means nothing, its length.)"""
    return t.stride(-2) if t.shape[-2] > 1 else max(t.shape[-1], 1)


def _float(t, name):
    torch = _torch()
    dt = t.dtype
    if dt is torch.bfloat16:
        return dt, IMBD_BF16
    if dt is torch.float32:
        return dt, IMBD_F32
    raise TypeError(f"{name}: {dt}, need torch.bfloat16 or torch.float32")


def expert_route_workspace_bytes(T: int, E: int, k: int) -> int:
    if max(T, E, k) >> 31 > 0:
        _too_large(T, E, k)
    return load().expert_route_workspace_bytes(T, E, k)


def expert_route(logits, gates, experts, offsets, rows, slots, ws=None, renorm: bool = True, stream=None):
    """Each token's k experts (k = gates.shape[1]), their gates, and the plan in expert order."""
    torch = _torch()
    lib, dev = load(), _here(logits, "logits")
    T, E = logits.shape
    k = gates.shape[-1]
    if (T | E | k) >> 31:
        _too_large(T, E, k)
    i32, f32 = torch.int32, torch.float32
    check(lib.expert_route(T, E, k, bool(renorm), _sizes(logits, (T, E), f32, "logits", dev), _rows_ld(logits),
                           _sizes(gates, (T, k), f32, "gates", dev, True),
                           _sizes(experts, (T, k), i32, "experts", dev, True),
                           _sizes(offsets, (E + 1,), i32, "offsets", dev, True),
                           _sizes(rows, (T * k,), i32, "rows", dev, True),
                           _sizes(slots, (T, k), i32, "slots", dev, True),
                           None if ws is None else _sizes(ws, ws.shape, ws.dtype, "ws", dev, True),
                           0 if ws is None else ws.numel() * ws.element_size(), _on(stream, dev)), "expert_route")


def expert_route_bwd(logits, gates, experts, dgates, dlogits, renorm: bool = True, stream=None):
    """The logits' gradient from the gates' (logits may be None with renorm)."""
    torch = _torch()
    lib, dev = load(), _here(dlogits, "dlogits")
    T, E = dlogits.shape
    k = gates.shape[-1]
    if (T | E | k) >> 31:
        _too_large(T, E, k)
    f32, none = torch.float32, logits is None
    check(lib.expert_route_bwd(T, E, k, bool(renorm), None if none else _sizes(logits, (T, E), f32, "logits", dev),
                               0 if none else _rows_ld(logits), _sizes(gates, (T, k), f32, "gates", dev, True),
                               _sizes(experts, (T, k), torch.int32, "experts", dev, True),
                               _sizes(dgates, (T, k), f32, "dgates", dev, True),
                               _sizes(dlogits, (T, E), f32, "dlogits", dev), _rows_ld(dlogits), _on(stream, dev)),
          "expert_route_bwd")


def expert_fwd(w, x, offsets, y, bias=None, relu: bool = False, rows=None, stream=None):
    """y[s] = W_e x[rows[s]] + b_e, ReLU, for every slot s of every expert e. w [E][d_out][d_in]."""
    torch = _torch()
    lib, dev = load(), _here(w, "w")
    E, d_out, d_in = w.shape
    (dt, code), (ydt, ycode) = _float(w, "w"), _float(y, "y")
    n, n_x, i32 = y.shape[0], x.shape[0], torch.int32
    if (E | d_out | d_in | n | n_x) >> 31:
        _too_large(E, d_out, d_in, n, n_x)
    check(lib.expert_fwd(code, bool(relu), E, d_out, d_in, n, n_x, _sizes(w, (E, d_out, d_in), dt, "w", dev),
                         _rows_ld(w), w.stride(0),
                         None if bias is None else _sizes(bias, (E, d_out), torch.float32, "bias", dev, True),
                         _sizes(x, (n_x, d_in), dt, "x", dev), _rows_ld(x),
                         None if rows is None else _sizes(rows, (n,), i32, "rows", dev, True),
                         _sizes(offsets, (E + 1,), i32, "offsets", dev, True), _sizes(y, (n, d_out), ydt, "y", dev),
                         _rows_ld(y), ycode, _on(stream, dev)), "expert_fwd")


def expert_bwd(w, dy, x, offsets, dw=None, db=None, dx=None, rows=None, mask_relu: bool = False, stream=None):
    """The backward products of expert_fwd: dx in expert order, dw and db of every expert. What is
    None is skipped; w gives the sizes also where dx is None."""
    torch = _torch()
    lib, dev = load(), _here(w, "w")
    E, d_out, d_in = w.shape
    dt, code = _float(w, "w")
    n, f32, i32 = dy.shape[0], torch.float32, torch.int32
    n_x = n if x is None else x.shape[0]
    if (E | d_out | d_in | n | n_x) >> 31:
        _too_large(E, d_out, d_in, n, n_x)
    dxdt, dxcode = (None, IMBD_F32) if dx is None else _float(dx, "dx")
    check(lib.expert_bwd(code, E, d_out, d_in, n, n_x, _sizes(w, (E, d_out, d_in), dt, "w", dev), _rows_ld(w),
                         w.stride(0), _sizes(dy, (n, d_out), dt, "dy", dev), _rows_ld(dy),
                         None if x is None else _sizes(x, (n_x, d_in), dt, "x", dev), 0 if x is None else _rows_ld(x),
                         None if rows is None else _sizes(rows, (n,), i32, "rows", dev, True),
                         _sizes(offsets, (E + 1,), i32, "offsets", dev, True),
                         None if dw is None else _sizes(dw, (E, d_out, d_in), f32, "dw", dev),
                         0 if dw is None else _rows_ld(dw), 0 if dw is None else dw.stride(0),
                         None if db is None else _sizes(db, (E, d_out), f32, "db", dev, True),
                         None if dx is None else _sizes(dx, (n, d_in), dxdt, "dx", dev),
                         0 if dx is None else _rows_ld(dx), dxcode, bool(mask_relu), _on(stream, dev)), "expert_bwd")


def expert_combine(ys, slots, y, gates=None, stream=None):
    """y[t] = sum_j gates[t][j] ys[slots[t][j]] (gates None: 1)."""
    torch = _torch()
    lib, dev = load(), _here(ys, "ys")
    n, d = ys.shape
    T, k = slots.shape
    if (T | k | n | d) >> 31:
        _too_large(T, k, n, d)
    (dt, code), (ydt, ycode) = _float(ys, "ys"), _float(y, "y")
    check(lib.expert_combine(code, T, k, d, n, _sizes(ys, (n, d), dt, "ys", dev), _rows_ld(ys),
                             _sizes(slots, (T, k), torch.int32, "slots", dev, True),
                             None if gates is None else _sizes(gates, (T, k), torch.float32, "gates", dev, True),
                             _sizes(y, (T, d), ydt, "y", dev), _rows_ld(y), ycode, _on(stream, dev)),
          "expert_combine")


def expert_combine_bwd(dy, ys, slots, gates, dys, dgates=None, stream=None):
    """dys[slots[t][j]] = gates[t][j] dy[t] and dgates[t][j] = dy[t] . ys[slots[t][j]] (ys may be None
    without dgates)."""
    torch = _torch()
    lib, dev = load(), _here(dy, "dy")
    T, d = dy.shape
    n, k = dys.shape[0], slots.shape[-1]
    if (T | k | n | d) >> 31:
        _too_large(T, k, n, d)
    dt, code = _float(dy, "dy")
    f32 = torch.float32
    check(lib.expert_combine_bwd(code, T, k, d, n, _sizes(dy, (T, d), dt, "dy", dev), _rows_ld(dy),
                                 None if ys is None else _sizes(ys, (n, d), dt, "ys", dev),
                                 0 if ys is None else _rows_ld(ys),
                                 _sizes(slots, (T, k), torch.int32, "slots", dev, True),
                                 _sizes(gates, (T, k), f32, "gates", dev, True), _sizes(dys, (n, d), dt, "dys", dev),
                                 _rows_ld(dys), None if dgates is None else _sizes(dgates, (T, k), f32, "dgates", dev, True),
                                 _on(stream, dev)), "expert_combine_bwd")


# ------------------------------------------------------------------------------- AdamW
class AdamW:
    """The plan of an AdamW update over many tensors, made once and kept.

    tensors: sequence of dicts with w (fp32), grad (fp32 or bf16), m and v, and optionally w_lp
    (bf16 copy) and decay (0). 32-bit state: m and v fp32. 8-bit state: m torch.float8_e4m3fn, v
    torch.float8_e5m2, and m_scale and v_scale, fp32 [ceil(n/256)]. All contiguous, of one device,
    and kept alive by the plan; no two may share memory (gradients may). Zeros are the state before the
    first step. The plan holds addresses and is built tensor by tensor on the host: for a tensor that
    is allocated again, a gradient too, it has to be made anew.
    """

    def __init__(self, tensors):
        torch = _torch()
        lib = load()
        tensors = [dict(t) for t in tensors]
        self.tensors = tensors
        arr = (AdamWTensor * max(len(tensors), 1))()
        dev = _here(tensors[0]["w"], "w") if tensors else torch.cuda.current_device()
        f32 = torch.float32
        for a, t in zip(arr, tensors):
            w, n = t["w"], t["w"].numel()
            bits8 = t["m"].dtype is torch.float8_e4m3fn
            _sizes(w, w.shape, f32, "w", dev, True)
            _sizes(t["grad"], w.shape, _float(t["grad"], "grad")[0], "grad", dev, True)
            _sizes(t["m"], w.shape, torch.float8_e4m3fn if bits8 else f32, "m", dev, True)
            _sizes(t["v"], w.shape, torch.float8_e5m2 if bits8 else f32, "v", dev, True)
            if t.get("w_lp") is not None:
                _sizes(t["w_lp"], w.shape, torch.bfloat16, "w_lp", dev, True)
                a.w_lp = t["w_lp"].data_ptr()
            if bits8:
                blocks = ((n + 255) // 256,)
                _sizes(t["m_scale"], blocks, f32, "m_scale", dev, True)
                _sizes(t["v_scale"], blocks, f32, "v_scale", dev, True)
                a.m_scale, a.v_scale = t["m_scale"].data_ptr(), t["v_scale"].data_ptr()
            a.w, a.grad, a.m, a.v = w.data_ptr(), t["grad"].data_ptr(), t["m"].data_ptr(), t["v"].data_ptr()
            a.n, a.decay = n, float(t.get("decay", 0.0))
            a.grad_dtype, a.state_bits = dtype_code(t["grad"]), 8 if bits8 else 32
        self.device = dev
        self.n_tensors = len(tensors)
        self.bytes = lib.adamw_plan_bytes(arr, len(tensors))
        host = torch.empty(max(self.bytes, 8), dtype=torch.uint8)
        # (a plan of no bytes: nothing to update, or a bad argument, which this call reports)
        check(lib.adamw_plan(arr, len(tensors), _ptr(host), self.bytes), "adamw_plan")
        self.plan = host.to(torch.device("cuda", dev))
        self.address = self.plan.data_ptr()


def adamw_step(plan: AdamW, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, step=1,
               grad_scale: float = 1.0, stream=None):
    """One AdamW step on every tensor of a plan. step: the step's number, from 1 on, or a device int32
    tensor that holds it (read by the kernel, so a captured launch follows it)."""
    lib, torch = load(), _torch()
    dev = plan.device
    dev_step = None
    if isinstance(step, int) and step >> 31 > 0:
        raise ValueError(f"step {step}: has to be under 2^31")
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"plan: on cuda:{dev}, which is not the current device")
    if not isinstance(step, int):
        dev_step = _sizes(step, step.shape, torch.int32, "step", dev, True)
        if step.numel() != 1:
            raise ValueError(f"step: {step.numel()} elements, need 1")
        step = 1
    check(lib.adamw_step(plan.address, plan.bytes, plan.n_tensors, lr, beta1, beta2, eps, grad_scale, step, dev_step,
                         _on(stream, dev)), "adamw_step")


def timing_begin(kernel_class: int, layer: int = -1, max_launches: int = 1000):
    check(load().imbd_timing_begin(kernel_class, layer, max_launches), "imbd_timing_begin")


def timing_end():
    n = ctypes.c_int(0)
    ms = ctypes.c_double(0.0)
    check(load().imbd_timing_end(ctypes.byref(n), ctypes.byref(ms)), "imbd_timing_end")
    return n.value, ms.value


def set_option(key: int, value: int):
    check(load().imbd_set_option(int(key), int(value)), "imbd_set_option")


def get_option(key: int) -> int:
    v = ctypes.c_int(0)
    check(load().imbd_get_option(int(key), ctypes.byref(v)), "imbd_get_option")
    return v.value


def option_name(key: int) -> str:
    return load().imbd_option_name(int(key)).decode()


class options:
    """Context manager: set options (key -> value) for a block, restore them after."""

    def __init__(self, **kv):
        import sys
        mod = sys.modules[__name__]
        self.kv = {getattr(mod, "IMBD_OPT_" + k.upper()): int(v) for k, v in kv.items() if v is not None}
        self.old = {}

    def __enter__(self):
        for k, v in self.kv.items():
            self.old[k] = get_option(k)
            set_option(k, v)
        return self

    def __exit__(self, *exc):
        for k, v in self.old.items():
            set_option(k, v)
