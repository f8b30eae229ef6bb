"""Training and serving of the head that makes an index's vectors.

The binding of ``include/head.h``: softmax cross entropy over a collection's items
and its gradients, rows kept in 8 bits with the backward steps that read them,
and products with 4-bit weights.  Operands are CUDA ``torch`` tensors of one
device, whose rows may be strided; work is queued on torch's current stream of
that device, outputs and scratch come from torch's allocator on that stream,
and nothing waits for the GPU.  A tensor made on another stream is the caller's
to order, as with torch's own operators.  Autograd does not see these calls: a
result has no graph, whether its inputs require gradients or not, and the gradients are
the backward entry points' to compute.  A negative status raises ``PvsError``;
wrong shapes and types raise ``ValueError`` and ``TypeError``.
"""
from __future__ import annotations

import ctypes

PVS_BF16 = 0
PVS_F16 = 1
PVS_F32 = 2
PVS_ACT_NONE = 0
PVS_ACT_GELU = 1

_P, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
_MAX_DIM = 32767
_MAX_ROWS = (1 << 31) - (1 << 16)


class pvs_xent_args(ctypes.Structure):
    _fields_ = [("x", _P), ("w", _P), ("targets", _P), ("bias", _P), ("rows", _i64),
                ("items", _i64), ("ldx", _i64), ("ldw", _i64), ("ignore_index", _i64),
                ("dim", _i32), ("dtype", _i32), ("scale", ctypes.c_float), ("reserved", _i32)]


_SIGNATURES = {
    "pvs_head_status": (_i32, []),
    "pvs_head_set_wait_limit": (_i32, [_i64]),
    "pvs_xent_workspace": (_i32, [_P, _i32, _P]),
    "pvs_xent_forward": (_i32, [_P, _P, _P, _P, ctypes.c_size_t, _P]),
    "pvs_xent_backward": (_i32, [_P, _P, _P, _P, _i64, _P, _i64, _P, ctypes.c_size_t, _P]),
    "pvs_ckpt_store": (_i32, [_P, _i64, _i64, _i32, _i32, _i32, _P, _i64, _P, _P, _i64, _P]),
    "pvs_ckpt_load": (_i32, [_P, _i64, _P, _i64, _i32, _P, _i64, _i32, _P]),
    "pvs_ckpt_act_backward": (_i32, [_P, _i64, _P, _i64, _P, _i64, _i32, _i32, _i32, _P, _i64,
                                     _P]),
    "pvs_ckpt_grad_workspace": (_i32, [_i64, _i32, _i32, _i32, _P]),
    "pvs_ckpt_grad_weight": (_i32, [_P, _i64, _P, _i64, _P, _i64, _i32, _i32, _i32, _P, _i64, _P,
                                    ctypes.c_size_t, _P]),
    "pvs_wq_pack": (_i32, [_P, _i64, _i64, _i32, _i32, _i32, _P, _P, _P]),
    "pvs_wq_unpack": (_i32, [_P, _P, _i64, _i32, _i32, _P, _i64, _i32, _P]),
    "pvs_wq_matvec": (_i32, [_P, _i64, _i32, _P, _P, _i64, _i32, _i32, _i32, _P, _i64, _P]),
}
EXPORTED = tuple(_SIGNATURES)

_lib = None
_check = None


def _bind(lib, check) -> None:
    global _lib, _check
    _lib, _check = lib, check
    for name, (res, args) in _SIGNATURES.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args


torch = None              # bound by the first call: the package imports without it
_CODES = {}


def _bind_torch() -> None:
    global torch, _CODES
    import torch as t
    _CODES = {t.bfloat16: PVS_BF16, t.float16: PVS_F16, t.float32: PVS_F32}
    torch = t


def _dtype_code(dtype) -> int:
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"{dtype} is none of bfloat16, float16 and float32")
    return code


def _on_gpu(*tensors) -> int:
    """The index of the device that all of them are on (None entries are left out).
    The checks of a call cost as much as a small kernel: they stay plain."""
    if torch is None:
        _bind_torch()
    device = -1
    for x in tensors:
        if x is None:
            continue
        d = x.get_device() if isinstance(x, torch.Tensor) else -1
        if d < 0:
            raise TypeError("the operators take CUDA tensors")
        if device < 0:
            device = d
        elif d != device:
            raise ValueError("the tensors must be on one device")
    return device


def _elsewhere(device: int) -> bool:
    """Whether another device is current: the call is then made again with this one."""
    return torch._C._cuda_getDevice() != device


def _stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def _matrix(x, name: str, dtype=None):
    """A 2-D tensor whose rows the kernels can read: (tensor, leading dimension)."""
    if x.dim() != 2:
        raise ValueError(f"{name} must be 2-D")
    if dtype is not None and x.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    rows, cols = x.shape
    if cols < 1 or cols > _MAX_DIM:
        raise ValueError(f"{name} has {cols} columns, outside [1, {_MAX_DIM}]")
    if rows > _MAX_ROWS:
        raise ValueError(f"{name} has more than {_MAX_ROWS} rows")
    if x.is_contiguous():
        return x, cols
    if (cols > 1 and x.stride(1) != 1) or (rows > 1 and x.stride(0) < cols):
        return x.contiguous(), cols
    return x, (x.stride(0) if rows > 1 else cols)


def _vector(x, name: str, n: int, dtype):
    if x.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if x.dim() != 1 or x.shape[0] != n:
        raise ValueError(f"{name} must have {n} entries")
    return x.contiguous()


def _ptr(x):
    return x.data_ptr() if x is not None else None


def pvs_head_status() -> int:
    """PVS_OK, or raises what an earlier operator of this module left on the
    current device (PVS_ERR_TIMEOUT); ask after a synchronisation."""
    return _check(_lib.pvs_head_status(), "pvs_head_status")


def pvs_head_set_wait_limit(ns: int) -> None:
    """Limit of the device-side waits of products queued from now on on the current
    device (default and maximum 2e9; 0: a wait gives up unless it need not wait)."""
    _check(_lib.pvs_head_set_wait_limit(int(ns)), "pvs_head_set_wait_limit")


def _xent_args(x, w, targets, bias, scale, ignore_index):
    device = _on_gpu(x, w, targets, bias)
    x, ldx = _matrix(x, "x")
    w, ldw = _matrix(w, "w", x.dtype)
    if x.shape[1] != w.shape[1]:
        raise ValueError(f"x has {x.shape[1]} columns, w {w.shape[1]}")
    if w.shape[0] < 1:
        raise ValueError("w must have a row at least")
    if not (0.0 < scale < float("inf")):
        raise ValueError("scale must be positive and finite")
    targets = _vector(targets, "targets", x.shape[0], torch.int64)
    if bias is not None:
        bias = _vector(bias, "bias", w.shape[0], torch.float32)
    a = pvs_xent_args(x.data_ptr(), w.data_ptr(), targets.data_ptr(),
                      bias.data_ptr() if bias is not None else None, x.shape[0], w.shape[0], ldx,
                      ldw, int(ignore_index), x.shape[1], _dtype_code(x.dtype), float(scale), 0)
    return a, device, (x, w, targets, bias)


def _workspace(n: int, device):
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


def pvs_xent_forward(x, w, targets, bias=None, scale: float = 1.0, ignore_index: int = -100):
    """Softmax cross entropy of the rows of x [T, d] over the items w [V, d]:
    logits ``scale * x @ w.T + bias``, targets int64 [T] (``ignore_index``: no loss),
    bias float32 [V] or None (-inf: the item is not in the softmax).  Returns
    (loss float32 [T], stats float32 [T, 4]); the backward pass takes the stats.
    x and w are both bfloat16, float16 or float32.  No logit is kept."""
    a, device, keep = _xent_args(x, w, targets, bias, scale, ignore_index)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_xent_forward(x, w, targets, bias, scale, ignore_index)
    loss = torch.empty(a.rows, dtype=torch.float32, device=device)
    stats = torch.empty(a.rows, 4, dtype=torch.float32, device=device)
    n = ctypes.c_size_t()
    _check(_lib.pvs_xent_workspace(ctypes.byref(a), 0, ctypes.byref(n)), "pvs_xent_workspace")
    ws = _workspace(n.value, device)
    _check(_lib.pvs_xent_forward(ctypes.byref(a), _ptr(loss), _ptr(stats), _ptr(ws), n.value,
                                 _stream(device)), "pvs_xent_forward")
    return loss, stats


def pvs_xent_backward(x, w, targets, stats, grad_loss, bias=None, scale: float = 1.0,
                      ignore_index: int = -100, need_x: bool = True, need_w: bool = True):
    """The gradients (dx, dw) of ``(grad_loss * loss).sum()``, grad_loss float32
    [T], from the forward pass's stats; None for one that is not needed.  The
    logits are computed again, a piece of the items at a time."""
    a, device, keep = _xent_args(x, w, targets, bias, scale, ignore_index)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_xent_backward(x, w, targets, stats, grad_loss, bias, scale, ignore_index,
                                     need_x, need_w)
    _on_gpu(x, stats, grad_loss)
    if stats.dtype != torch.float32 or tuple(stats.shape) != (a.rows, 4):
        raise ValueError("stats must be the forward pass's float32 [T, 4]")
    stats = stats.contiguous()
    if stats.data_ptr() % 16:
        stats = stats.clone()
    grad_loss = _vector(grad_loss, "grad_loss", a.rows, torch.float32)
    dx = torch.empty(a.rows, a.dim, dtype=x.dtype, device=device) if need_x else None
    dw = torch.empty(a.items, a.dim, dtype=x.dtype, device=device) if need_w else None
    n = ctypes.c_size_t()
    _check(_lib.pvs_xent_workspace(ctypes.byref(a), 1, ctypes.byref(n)), "pvs_xent_workspace")
    ws = _workspace(n.value, device)
    _check(_lib.pvs_xent_backward(ctypes.byref(a), _ptr(stats), _ptr(grad_loss), _ptr(dx),
                                  a.dim, _ptr(dw), a.dim, _ptr(ws), n.value, _stream(device)),
           "pvs_xent_backward")
    return dx, dw


def _codes(codes, scales):
    codes, ld = _matrix(codes, "codes", torch.int8)
    return codes, ld, _vector(scales, "scales", codes.shape[0], torch.float32)


def pvs_ckpt_store(x, act: int = PVS_ACT_NONE):
    """Rows of x [R, K] in 8 bits: (codes int8 [R, K], scales float32 [R], y) with
    y = act(x) in x's type, None for PVS_ACT_NONE.  Row r stands for
    ``scales[r] * codes[r]``."""
    device = _on_gpu(x)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_ckpt_store(x, act)
    x, ldx = _matrix(x, "x")
    dt = _dtype_code(x.dtype)
    rows, cols = x.shape
    codes = torch.empty(rows, cols, dtype=torch.int8, device=device)
    scales = torch.empty(rows, dtype=torch.float32, device=device)
    y = torch.empty(rows, cols, dtype=x.dtype, device=device) if act != PVS_ACT_NONE else None
    _check(_lib.pvs_ckpt_store(_ptr(x), ldx, rows, cols, dt, int(act), _ptr(codes), cols,
                               _ptr(scales), _ptr(y), cols, _stream(device)),
           "pvs_ckpt_store")
    return codes, scales, y


def pvs_ckpt_load(codes, scales, dtype):
    """What rows kept by ``pvs_ckpt_store`` stand for, as a tensor of `dtype`."""
    device = _on_gpu(codes, scales)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_ckpt_load(codes, scales, dtype)
    codes, ld, scales = _codes(codes, scales)
    dt = _dtype_code(dtype)
    rows, cols = codes.shape
    out = torch.empty(rows, cols, dtype=dtype, device=device)
    _check(_lib.pvs_ckpt_load(_ptr(codes), ld, _ptr(scales), rows, cols, _ptr(out), cols, dt,
                              _stream(device)), "pvs_ckpt_load")
    return out


def pvs_ckpt_act_backward(dy, codes, scales, act: int = PVS_ACT_GELU):
    """``dy * act'(x)`` for the rows x that the codes stand for, in dy's type."""
    device = _on_gpu(dy, codes, scales)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_ckpt_act_backward(dy, codes, scales, act)
    dy, lddy = _matrix(dy, "dy")
    dt = _dtype_code(dy.dtype)
    codes, ld, scales = _codes(codes, scales)
    if dy.shape != codes.shape:
        raise ValueError("dy and codes must have one shape")
    rows, cols = codes.shape
    dx = torch.empty(rows, cols, dtype=dy.dtype, device=device)
    _check(_lib.pvs_ckpt_act_backward(_ptr(dy), lddy, _ptr(codes), ld, _ptr(scales), rows,
                                      cols, dt, int(act), _ptr(dx), cols, _stream(device)),
           "pvs_ckpt_act_backward")
    return dx


def pvs_ckpt_grad_weight(dy, codes, scales):
    """The weight gradient ``dy.T @ x`` [N, K] of a linear layer, dy [R, N], from the
    rows x [R, K] that the codes stand for, in dy's type."""
    device = _on_gpu(dy, codes, scales)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_ckpt_grad_weight(dy, codes, scales)
    dy, lddy = _matrix(dy, "dy")
    dt = _dtype_code(dy.dtype)
    codes, ld, scales = _codes(codes, scales)
    if dy.shape[0] != codes.shape[0]:
        raise ValueError("dy and codes must have as many rows")
    rows, n, k = dy.shape[0], dy.shape[1], codes.shape[1]
    dw = torch.empty(n, k, dtype=dy.dtype, device=device)
    size = ctypes.c_size_t()
    _check(_lib.pvs_ckpt_grad_workspace(rows, n, k, dt, ctypes.byref(size)),
           "pvs_ckpt_grad_workspace")
    ws = _workspace(size.value, device)
    _check(_lib.pvs_ckpt_grad_weight(_ptr(dy), lddy, _ptr(codes), ld, _ptr(scales), rows, n, k,
                                     dt, _ptr(dw), k, _ptr(ws), size.value, _stream(device)),
           "pvs_ckpt_grad_weight")
    return dw


def _wq_padded(k: int) -> int:
    return (k + 127) // 128 * 128


def _wq_weights(codes, scales, group: int):
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    if codes.dtype != torch.uint8 or scales.dtype != torch.bfloat16:
        raise TypeError("codes must be uint8 and scales bfloat16")
    if codes.dim() != 2 or scales.dim() != 2:
        raise ValueError("codes and scales must be 2-D")
    n, half = codes.shape
    if half % 64 != 0 or half == 0:
        raise ValueError("codes must be [N, padded K / 2], padded K a multiple of 128")
    ns, groups = scales.shape
    if ns != n or groups != half * 2 // group:
        raise ValueError("scales must be [N, padded K / group]")
    codes, scales = codes.contiguous(), scales.contiguous()
    # a view can start anywhere; the kernels read 16 (8) bytes at once
    if codes.data_ptr() % 16:
        codes = codes.clone()
    if scales.data_ptr() % 8:
        scales = scales.clone()
    return codes, scales, half * 2


def pvs_wq_pack(w, group: int):
    """Weights [N, K] in 4 bits with a bfloat16 scale for every `group` (32, 64 or
    128) of a row: (codes uint8 [N, Kp / 2], scales bfloat16 [N, Kp / group]), Kp
    = K padded to a multiple of 128."""
    device = _on_gpu(w)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_wq_pack(w, group)
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    w, ldw = _matrix(w, "w")
    dt = _dtype_code(w.dtype)
    n, k = w.shape
    kp = _wq_padded(k)
    codes = torch.empty(n, kp // 2, dtype=torch.uint8, device=device)
    scales = torch.empty(n, kp // group, dtype=torch.bfloat16, device=device)
    _check(_lib.pvs_wq_pack(_ptr(w), ldw, n, k, dt, int(group), _ptr(codes), _ptr(scales),
                            _stream(device)), "pvs_wq_pack")
    return codes, scales


def pvs_wq_unpack(codes, scales, group: int, cols: int, dtype):
    """The weights [N, cols] that packed ones stand for, as a tensor of `dtype`."""
    device = _on_gpu(codes, scales)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_wq_unpack(codes, scales, group, cols, dtype)
    codes, scales, kp = _wq_weights(codes, scales, group)
    dt = _dtype_code(dtype)
    if cols < 1 or _wq_padded(cols) != kp:
        raise ValueError(f"cols = {cols} does not pad to {kp}")
    n = codes.shape[0]
    out = torch.empty(n, cols, dtype=dtype, device=device)
    _check(_lib.pvs_wq_unpack(_ptr(codes), _ptr(scales), n, cols, int(group), _ptr(out), cols,
                              dt, _stream(device)), "pvs_wq_unpack")
    return out


def pvs_wq_matvec(x, codes, scales, group: int):
    """``x @ weights.T`` [B, N] in x's type, for a few rows x [B, K] (B <= 64) and
    packed weights."""
    device = _on_gpu(x, codes, scales)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_wq_matvec(x, codes, scales, group)
    codes, scales, kp = _wq_weights(codes, scales, group)
    x, ldx = _matrix(x, "x")
    dt = _dtype_code(x.dtype)
    b, k = x.shape
    if b > 64:
        raise ValueError("x has more than 64 rows")
    if _wq_padded(k) != kp:
        raise ValueError(f"x has {k} columns, the packed weights {kp} after padding")
    n = codes.shape[0]
    y = torch.empty(b, n, dtype=x.dtype, device=device)
    _check(_lib.pvs_wq_matvec(_ptr(x), ldx, b, _ptr(codes), _ptr(scales), n, k, int(group), dt,
                              _ptr(y), n, _stream(device)), "pvs_wq_matvec")
    return y
