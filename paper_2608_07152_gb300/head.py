"""Training and serving of the head that makes an index's vectors.

The binding of ``include/head.h``: softmax cross entropy over a collection's items and
distillation from a teacher's lists of them, with their gradients, table lookups and the
table's gradient, rows kept in 8 bits with the backward steps that read them, and
products with 4-bit weights and of microscaled 4-bit rows.  Operands are CUDA ``torch`` tensors of one
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
import functools

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


class pvs_distill_args(ctypes.Structure):
    _fields_ = [("student", pvs_xent_args), ("ids", _P), ("logits", _P), ("top", _i32),
                ("teacher_dtype", _i32), ("teacher_scale", ctypes.c_float), ("reserved", _i32)]


_SIGNATURES = {
    "pvs_head_status": (_i32, []),
    "pvs_head_set_wait_limit": (_i32, [_i64]),
    "pvs_xent_workspace": (_i32, [_P, _i32, _P]),
    "pvs_xent_forward": (_i32, [_P, _P, _P, _P, ctypes.c_size_t, _P]),
    "pvs_xent_backward": (_i32, [_P, _P, _P, _P, _i64, _P, _i64, _P, ctypes.c_size_t, _P]),
    "pvs_distill_workspace": (_i32, [_P, _i32, _P]),
    "pvs_distill_forward": (_i32, [_P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "pvs_distill_backward": (_i32, [_P, _P, _P, _P, _P, _i64, _P, _i64, _P, ctypes.c_size_t, _P]),
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
    "pvs_mx_pack": (_i32, [_P, _i64, _i64, _i32, _i32, _i32, _P, _P, _P, _P]),
    "pvs_mx_unpack": (_i32, [_P, _P, _P, _i64, _i32, _i32, _P, _i64, _i32, _P]),
    "pvs_mx_workspace": (_i32, [_i64, _i64, _i32, _i32, _P]),
    "pvs_mx_matmul": (_i32, [_P, _i64, _i64, _P, _P, _P, _i64, _i32, _i32, _i32, _P, _i64, _P,
                             ctypes.c_size_t, _P]),
    "pvs_embed_forward": (_i32, [_P, _i64, _i64, _i32, _i32, _P, _i64, ctypes.c_float, _i64, _P,
                                 _i64, _P]),
    "pvs_embed_workspace": (_i32, [_i64, _i64, _i32, _P]),
    "pvs_embed_backward": (_i32, [_P, _i64, _P, _i64, _i64, _i32, _i32, ctypes.c_float, _i64, _P,
                                  _i64, _P, ctypes.c_size_t, _P]),
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


_MAX_TOP = 1024


def _list(x, name: str, rows: int):
    if x.dim() != 2 or x.shape[0] != rows or not 1 <= x.shape[1] <= _MAX_TOP:
        raise ValueError(f"{name} must be [{rows}, K], K in [1, {_MAX_TOP}]")
    return x.contiguous()


# What an operator wants of scratch follows from a call's sizes and alignments alone, and asking for it
# costs a small call a tenth of its time: the last few thousand answers are kept.
def _asked(name: str, *args) -> int:
    n = ctypes.c_size_t()
    _check(getattr(_lib, name)(*args, ctypes.byref(n)), name)
    return n.value


@functools.lru_cache(maxsize=4096)
def _distill_bytes(device: int, backward: int, x_fits: bool, w_fits: bool, bias: bool, rows: int, items: int,
                   ldx: int, ldw: int, dim: int, dtype: int, top: int) -> int:
    at = 1 << 20              # a pointer that nothing reads, and one that is on its elements alone
    off = at + (4 if dtype == PVS_F32 else 2)
    s = pvs_xent_args(at if x_fits else off, at if w_fits else off, None, at if bias else None, rows, items,
                      ldx, ldw, 0, dim, dtype, 1.0, 0)
    a = pvs_distill_args(s, at, None, top, PVS_F32, 1.0, 0)
    return _asked("pvs_distill_workspace", ctypes.byref(a), backward)


def _distill_scratch(a, device: int, backward: int):
    s = a.student
    n = _distill_bytes(device, backward, s.x % 16 == 0 if s.x else True, s.w % 16 == 0, bool(s.bias), s.rows,
                       s.items, s.ldx, s.ldw, s.dim, s.dtype, a.top)
    return _workspace(n, device), n


def _distill_args(x, w, ids, logits, bias, scale, teacher_scale, ignore_index):
    device = _on_gpu(x, w, ids, logits, bias)
    x, ldx = _matrix(x, "x")
    w, ldw = _matrix(w, "w", x.dtype)
    if x.shape[1] != w.shape[1]:
        raise ValueError(f"x has {x.shape[1]} columns, w {w.shape[1]}")
    if w.shape[0] < 1:
        raise ValueError("w must have a row at least")
    for name, v in (("scale", scale), ("teacher_scale", teacher_scale)):
        if not (0.0 < v < float("inf")):
            raise ValueError(f"{name} must be positive and finite")
    ids = _list(ids, "ids", x.shape[0])
    if ids.dtype != torch.int64:
        raise TypeError("ids must be torch.int64")
    teacher = PVS_F32
    if logits is not None:
        teacher = _dtype_code(logits.dtype)
        logits = _list(logits, "logits", x.shape[0])
        if logits.shape != ids.shape:
            raise ValueError("logits and ids must have one shape")
    if bias is not None:
        bias = _vector(bias, "bias", w.shape[0], torch.float32)
    s = pvs_xent_args(x.data_ptr(), w.data_ptr(), None, _ptr(bias), x.shape[0], w.shape[0], ldx, ldw,
                      int(ignore_index), x.shape[1], _dtype_code(x.dtype), float(scale), 0)
    a = pvs_distill_args(s, ids.data_ptr(), _ptr(logits), ids.shape[1], teacher, float(teacher_scale), 0)
    return a, device, (x, w, ids, logits, bias)


def pvs_distill_forward(x, w, ids, logits, bias=None, scale: float = 1.0,
                        teacher_scale: float = 1.0, ignore_index: int = -100):
    """Distillation of a teacher's logits [T, K] of the items ids, int64 [T, K], into the softmax
    of the rows of x [T, d] over all items w [V, d] (logits ``scale * x @ w.T + bias``, bias
    float32 [V] or None): the divergence of that softmax from ``softmax(teacher_scale *
    logits)`` over each row's list.  A slot of ``ignore_index``, or of an item whose bias is -inf,
    is not in the list; a row without a list has no loss.  Returns (loss float32 [T], stats
    float32 [T, 4], hits float32 [T, K]); the backward pass takes the last two.  x and w are
    both bfloat16, float16 or float32, logits any of them."""
    if logits is None:
        raise TypeError("logits must be a tensor")
    a, device, keep = _distill_args(x, w, ids, logits, bias, scale, teacher_scale, ignore_index)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_distill_forward(x, w, ids, logits, bias, scale, teacher_scale, ignore_index)
    rows = a.student.rows
    loss = torch.empty(rows, dtype=torch.float32, device=device)
    stats = torch.empty(rows, 4, dtype=torch.float32, device=device)
    hits = torch.empty(rows, a.top, dtype=torch.float32, device=device)
    ws, n = _distill_scratch(a, device, 0)
    _check(_lib.pvs_distill_forward(ctypes.byref(a), _ptr(loss), _ptr(stats), _ptr(hits), _ptr(ws), n,
                                    _stream(device)), "pvs_distill_forward")
    return loss, stats, hits


def pvs_distill_backward(x, w, ids, stats, hits, grad_loss, bias=None, scale: float = 1.0,
                         ignore_index: int = -100, need_x: bool = True, need_w: bool = True):
    """The gradients (dx, dw) of ``(grad_loss * loss).sum()`` of ``pvs_distill_forward``,
    grad_loss float32 [T], from its stats and hits; None for one that is not needed."""
    a, device, keep = _distill_args(x, w, ids, None, bias, scale, 1.0, ignore_index)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_distill_backward(x, w, ids, stats, hits, grad_loss, bias, scale, ignore_index,
                                        need_x, need_w)
    _on_gpu(x, stats, hits, grad_loss)
    s = a.student
    if stats.dtype != torch.float32 or tuple(stats.shape) != (s.rows, 4):
        raise ValueError("stats must be the forward pass's float32 [T, 4]")
    if hits.dtype != torch.float32 or tuple(hits.shape) != (s.rows, a.top):
        raise ValueError("hits must be the forward pass's float32 [T, K]")
    stats, hits = stats.contiguous(), hits.contiguous()
    if stats.data_ptr() % 16:
        stats = stats.clone()
    grad_loss = _vector(grad_loss, "grad_loss", s.rows, torch.float32)
    dx = torch.empty(s.rows, s.dim, dtype=x.dtype, device=device) if need_x else None
    dw = torch.empty(s.items, s.dim, dtype=x.dtype, device=device) if need_w else None
    ws, n = _distill_scratch(a, device, 1)
    _check(_lib.pvs_distill_backward(ctypes.byref(a), _ptr(stats), _ptr(hits), _ptr(grad_loss),
                                     _ptr(dx), s.dim, _ptr(dw), s.dim, _ptr(ws), n, _stream(device)),
           "pvs_distill_backward")
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


def _finite(scale: float) -> float:
    if not abs(scale) < float("inf"):
        raise ValueError("scale must be finite")
    return float(scale)


def pvs_embed_forward(w, ids, scale: float = 1.0, ignore_index: int = -100):
    """Rows of the table w [V, d] by their ids, int64 [T], times `scale`: [T, d] in w's
    type.  ``ignore_index`` gives a row of zeros, another id outside the table NaN."""
    device = _on_gpu(w, ids)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_embed_forward(w, ids, scale, ignore_index)
    w, ldw = _matrix(w, "w")
    dt = _dtype_code(w.dtype)
    items, dim = w.shape
    if items < 1:
        raise ValueError("w must have a row at least")
    ids = _vector(ids, "ids", ids.shape[0] if ids.dim() == 1 else -1, torch.int64)
    if ids.shape[0] > _MAX_ROWS:
        raise ValueError(f"more than {_MAX_ROWS} ids")
    y = torch.empty(ids.shape[0], dim, dtype=w.dtype, device=device)
    _check(_lib.pvs_embed_forward(_ptr(w), ldw, items, dim, dt, _ptr(ids), ids.shape[0],
                                  _finite(scale), int(ignore_index), _ptr(y), dim, _stream(device)),
           "pvs_embed_forward")
    return y


@functools.lru_cache(maxsize=4096)
def _embed_bytes(rows: int, items: int, dim: int) -> int:
    return _asked("pvs_embed_workspace", rows, items, dim)


def pvs_embed_backward(dy, ids, items: int, scale: float = 1.0, ignore_index: int = -100):
    """The gradient [items, d] of a table from the gradient dy [T, d] of the rows that
    ``pvs_embed_forward`` took from it, in dy's type."""
    device = _on_gpu(dy, ids)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_embed_backward(dy, ids, items, scale, ignore_index)
    dy, lddy = _matrix(dy, "dy")
    dt = _dtype_code(dy.dtype)
    rows, dim = dy.shape
    ids = _vector(ids, "ids", rows, torch.int64)
    items = int(items)
    if items < 1 or items > _MAX_ROWS:
        raise ValueError(f"items must be in [1, {_MAX_ROWS}]")
    scale = _finite(scale)
    dw = torch.empty(items, dim, dtype=dy.dtype, device=device)
    n = _embed_bytes(rows, items, dim)
    ws = _workspace(n, device)
    _check(_lib.pvs_embed_backward(_ptr(dy), lddy, _ptr(ids), rows, items, dim, dt, scale,
                                   int(ignore_index), _ptr(dw), dim, _ptr(ws), n, _stream(device)),
           "pvs_embed_backward")
    return dw


def _mx_group(group: int) -> int:
    if group not in (16, 32):
        raise ValueError("group must be 16 or 32")
    return int(group)


def _mx_rows(codes, scales, row_scales, group: int):
    """Packed rows that the kernels can read, and their padded columns."""
    group = _mx_group(group)
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8:
        raise TypeError("codes and scales must be uint8")
    if codes.dim() != 2 or codes.shape[1] % 64 != 0 or codes.shape[1] == 0:
        raise ValueError("codes must be [N, padded K / 2], padded K a multiple of 128")
    n, kp = codes.shape[0], codes.shape[1] * 2
    if tuple(scales.shape) != ((n + 127) // 128, kp // (4 * group), 512):
        raise ValueError("scales must be [ceil(N / 128), padded K / (4 group), 512]")
    codes, scales = codes.contiguous(), scales.contiguous()
    # a view can start anywhere; the kernels copy 16 bytes at once
    if codes.data_ptr() % 16:
        codes = codes.clone()
    if scales.data_ptr() % 16:
        scales = scales.clone()
    if group == 16:
        if row_scales is None:
            raise ValueError("groups of 16 have row scales")
        row_scales = _vector(row_scales, "row_scales", n, torch.float32)
    elif row_scales is not None:
        raise ValueError("groups of 32 have no row scales")
    return codes, scales, row_scales, kp


def pvs_mx_pack(x, group: int):
    """Rows [N, K] in microscaled 4-bit floating point with a scale for every `group` (16 or 32)
    of a row: (codes uint8 [N, Kp / 2], scales uint8 [ceil(N / 128), Kp / (4 group), 512],
    row_scales float32 [N], None for groups of 32), Kp = K padded to a multiple of 128."""
    device = _on_gpu(x)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_mx_pack(x, group)
    group = _mx_group(group)
    x, ldx = _matrix(x, "x")
    dt = _dtype_code(x.dtype)
    n, k = x.shape
    kp = _wq_padded(k)
    codes = torch.empty(n, kp // 2, dtype=torch.uint8, device=device)
    scales = torch.empty((n + 127) // 128, kp // (4 * group), 512, dtype=torch.uint8, device=device)
    rows = torch.empty(n, dtype=torch.float32, device=device) if group == 16 else None
    _check(_lib.pvs_mx_pack(_ptr(x), ldx, n, k, dt, group, _ptr(codes), _ptr(scales), _ptr(rows),
                            _stream(device)), "pvs_mx_pack")
    return codes, scales, rows


def pvs_mx_unpack(codes, scales, row_scales, group: int, cols: int, dtype):
    """The rows [N, cols] that packed ones stand for, as a tensor of `dtype`."""
    device = _on_gpu(codes, scales, row_scales)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_mx_unpack(codes, scales, row_scales, group, cols, dtype)
    codes, scales, row_scales, kp = _mx_rows(codes, scales, row_scales, group)
    dt = _dtype_code(dtype)
    if cols < 1 or cols > _MAX_DIM or _wq_padded(cols) != kp:
        raise ValueError(f"cols = {cols} does not pad to {kp}")
    n = codes.shape[0]
    out = torch.empty(n, cols, dtype=dtype, device=device)
    _check(_lib.pvs_mx_unpack(_ptr(codes), _ptr(scales), _ptr(row_scales), n, cols, group, _ptr(out), cols,
                              dt, _stream(device)), "pvs_mx_unpack")
    return out


@functools.lru_cache(maxsize=4096)
def _mx_bytes(device: int, batch: int, rows: int, cols: int, group: int) -> int:
    return _asked("pvs_mx_workspace", batch, rows, cols, group)


def pvs_mx_matmul(x, codes, scales, row_scales, group: int):
    """``x @ weights.T`` [B, N] in x's type, for any number of rows x [B, K] and weights packed by
    ``pvs_mx_pack``; x is put into the same format first, so that both operands have 4 bits."""
    device = _on_gpu(x, codes, scales, row_scales)
    if _elsewhere(device):
        with torch.cuda.device(device):
            return pvs_mx_matmul(x, codes, scales, row_scales, group)
    codes, scales, row_scales, kp = _mx_rows(codes, scales, row_scales, group)
    x, ldx = _matrix(x, "x")
    dt = _dtype_code(x.dtype)
    b, k = x.shape
    if _wq_padded(k) != kp:
        raise ValueError(f"x has {k} columns, the packed weights {kp} after padding")
    n = codes.shape[0]
    if n > _MAX_ROWS:
        raise ValueError(f"the weights have more than {_MAX_ROWS} rows")
    y = torch.empty(b, n, dtype=x.dtype, device=device)
    size = _mx_bytes(device, b, n, k, group)
    ws = _workspace(size, device)
    _check(_lib.pvs_mx_matmul(_ptr(x), ldx, b, _ptr(codes), _ptr(scales), _ptr(row_scales), n, k, group, dt,
                              _ptr(y), n, _ptr(ws), size, _stream(device)), "pvs_mx_matmul")
    return y
