"""Python binding of the training-side operators (include/hc_train.h): embedding
lookup with scaling, its gradient by sorted token ids, and Newton-Schulz
orthogonalisation.  Argument marshalling only, like the package's other calls;
the names mirror the C ABI:

    hc_embed              out[i] = scale * table[ids[i]]
    hc_embed_grad         the gradient of the whole table (zeros where no id
                          points), or added to one
    hc_embed_grad_rows    the touched rows alone: ids, sums and their number
    hc_orthogonalise      the Newton-Schulz polynomial of a matrix, as the Muon
                          optimiser orthogonalises an update
"""
from __future__ import annotations

import ctypes

from . import _check, _lib, _ptr, _stream, _u32

HC_T_I32, HC_T_F32, HC_T_BF16, HC_T_F16 = range(4)
FIXED_POINT = 2.0**20          # fixed point of the int32 gradients
MUON = (3.4445, -4.7750, 2.0315)

TRAIN_EXPORTS = ("hc_embed", "hc_embed_grad_bytes", "hc_embed_grad", "hc_embed_grad_rows",
                 "hc_orthogonalise_bytes", "hc_orthogonalise")


class hc_embed_params(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_uint64), ("count", ctypes.c_uint64), ("dim", ctypes.c_uint64),
                ("table_ld", ctypes.c_uint64), ("x_ld", ctypes.c_uint64),
                ("padding", ctypes.c_int64), ("id_bits", ctypes.c_uint32),
                ("reserved", ctypes.c_uint32), ("scale", ctypes.c_float),
                ("fixed", ctypes.c_float)]


class hc_orthogonalise_params(ctypes.Structure):
    _fields_ = [("m", ctypes.c_uint64), ("n", ctypes.c_uint64), ("batch", ctypes.c_uint64),
                ("x_ld", ctypes.c_uint64), ("x_stride", ctypes.c_uint64),
                ("out_ld", ctypes.c_uint64), ("out_stride", ctypes.c_uint64),
                ("type", ctypes.c_uint32), ("steps", ctypes.c_uint32),
                ("coeffs", ctypes.POINTER(ctypes.c_float)),
                ("eps", ctypes.c_float), ("scale", ctypes.c_float)]


_P, _Z = ctypes.c_void_p, ctypes.c_size_t
_EP, _OP = ctypes.POINTER(hc_embed_params), ctypes.POINTER(hc_orthogonalise_params)
_lib.hc_embed.argtypes = [_EP, ctypes.c_int, _P, _P, _P, _P]
_lib.hc_embed_grad_bytes.argtypes = [_EP, ctypes.POINTER(_Z)]
_lib.hc_embed_grad.argtypes = [_EP, ctypes.c_int, _P, _P, ctypes.c_int, _P, ctypes.c_int, _P, _Z, _P]
_lib.hc_embed_grad_rows.argtypes = [_EP, ctypes.c_int, _P, _P, ctypes.c_int, _P, _P,
                                    ctypes.c_uint64, _P, _P, _Z, _P]
_lib.hc_orthogonalise_bytes.argtypes = [_OP, ctypes.POINTER(_Z)]
_lib.hc_orthogonalise.argtypes = [_OP, _P, _P, _P, _Z, _P]
for _f in TRAIN_EXPORTS:
    getattr(_lib, _f).restype = ctypes.c_int

_TYPES = {}     # torch's types, filled by the first call (importing the package needs no torch)
_ID_BITS = {}


def _code(table, dtype, message):
    if not _TYPES:
        import torch
        _ID_BITS.update({torch.int32: 32, torch.int64: 64})
        _TYPES.update({torch.int32: HC_T_I32, torch.float32: HC_T_F32, torch.bfloat16: HC_T_BF16,
                       torch.float16: HC_T_F16})
    code = table.get(dtype)
    if code is None:
        raise ValueError(f"{message} has dtype {dtype}, expected one of {tuple(table)}")
    return code


def _type(t, name):
    code = _TYPES.get(t.dtype)
    return _code(_TYPES, t.dtype, name) if code is None else code


def _rows(t, name):
    """(device pointer, rows, columns, row stride) of a tensor whose last dimension is
    contiguous and whose others are one stride apart (a matrix, or contiguous)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    dims = t.dim()
    if dims == 2:
        rows, cols = t.shape
        if t.is_contiguous():
            return t.data_ptr(), rows, cols, cols
    elif dims > 2:
        if not t.is_contiguous():
            raise ValueError(f"{name} must be a matrix or contiguous")
        cols = t.shape[-1]
        return t.data_ptr(), t.numel() // cols if cols else 0, cols, cols
    else:
        raise ValueError(f"{name} needs two dimensions or more")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    if rows > 1 and t.stride(0) < cols:
        raise ValueError(f"{name}'s rows overlap")
    return t.data_ptr(), rows, cols, t.stride(0) if rows > 1 else cols


def _ids(ids):
    bits = _ID_BITS.get(ids.dtype)
    if bits is None:
        bits = _code(_ID_BITS, ids.dtype, "ids")
    if not ids.is_cuda:
        raise ValueError("ids must be a device tensor")
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    return ids.data_ptr(), ids.numel(), bits


def _bytes(ws):
    import torch
    return _ptr(ws, "ws", (torch.uint8,))


def hc_embed(table, ids, out, scale: float = 1.0, stream=None):
    """out[i] = scale * table[ids[i]]; an id outside the table gives zeros.  table [vocab, dim]
    and out [.., dim] float32, bfloat16 or float16; ids int32 or int64, one for each row of
    out."""
    t, vocab, dim, table_ld = _rows(table, "table")
    o, rows, cols, out_ld = _rows(out, "out")
    i, count, bits = _ids(ids)
    if table.dtype != out.dtype:
        raise ValueError(f"table is {table.dtype}, out {out.dtype}")
    if cols != dim or rows != count:
        raise ValueError(f"out is {rows} x {cols}, expected {count} x {dim}")
    p = hc_embed_params(vocab, count, dim, table_ld, out_ld, -1, bits, 0, scale, 1.0)
    _check(_lib.hc_embed(ctypes.byref(p), _type(table, "table"), t, i, o, _stream(stream)),
           "hc_embed")


def hc_embed_grad_bytes(vocab: int, dim: int, count: int) -> int:
    p = hc_embed_params(vocab, count, dim, dim, dim, -1, 64, 0, 1.0, 1.0)
    b = _Z()
    _check(_lib.hc_embed_grad_bytes(ctypes.byref(p), ctypes.byref(b)), "hc_embed_grad_bytes")
    return b.value


def alloc_embed_workspace(vocab: int, dim: int, count: int, device="cuda"):
    """Workspace of hc_embed_grad and hc_embed_grad_rows for up to `count` ids."""
    import torch
    return torch.empty(max(hc_embed_grad_bytes(vocab, dim, count), 256), dtype=torch.uint8,
                       device=device)


def _grad_args(dout, ids, vocab, dst, name, scale, fixed, padding):
    """Arguments of the gradient calls; vocab None: as many rows as dst has."""
    x, rows, dim, x_ld = _rows(dout, "dout")
    d, dst_rows, cols, dst_ld = _rows(dst, name)
    i, count, bits = _ids(ids)
    if rows != count:
        raise ValueError(f"dout has {rows} rows, ids {count} elements")
    if cols != dim:
        raise ValueError(f"{name} has {cols} columns, dout {dim}")
    if vocab is None:
        vocab = dst_rows
    p = hc_embed_params(vocab, count, dim, dst_ld, x_ld, padding, bits, 0, scale, fixed)
    return p, _type(dout, "dout"), x, i, _type(dst, name), d, dst_rows


def hc_embed_grad(dout, ids, dtable, ws, scale: float = 1.0, fixed: float = FIXED_POINT,
                  padding: int = -1, accumulate: bool = False, stream=None):
    """dtable[v] = scale * sum of dout[i] over ids[i] == v (or added to dtable).  dout [.., dim]
    float32, bfloat16 or float16; dtable [vocab, dim] one of them, or int32: fixed point with
    `fixed` units per 1.0.  Ids outside the table and `padding` add nothing."""
    p, xt, x, i, gt, d, _ = _grad_args(dout, ids, None, dtable, "dtable", scale, fixed, padding)
    _check(_lib.hc_embed_grad(ctypes.byref(p), xt, x, i, gt, d, 1 if accumulate else 0,
                              _bytes(ws), ws.numel(), _stream(stream)),
           "hc_embed_grad")


def hc_embed_grad_rows(dout, ids, vocab: int, rows, values, touched, ws, scale: float = 1.0,
                       fixed: float = FIXED_POINT, padding: int = -1, stream=None):
    """The touched rows alone: rows[u] ascending distinct ids, values[u] their sums (types as
    hc_embed_grad's dtable), touched[0] how many there are.  rows and values hold `cap` entries;
    what lies past touched is not written."""
    p, xt, x, i, gt, d, cap = _grad_args(dout, ids, vocab, values, "values", scale, fixed, padding)
    _check(_lib.hc_embed_grad_rows(ctypes.byref(p), xt, x, i, gt, _ptr(rows, "rows", _u32(), cap), d,
                                   cap, _ptr(touched, "touched", _u32(), 1),
                                   _bytes(ws), ws.numel(), _stream(stream)),
           "hc_embed_grad_rows")


def _matrices(t, name):
    """(pointer, batch, m, n, row stride, matrix stride) of [m, n] or [batch, m, n]."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} must be [m, n] or [batch, m, n]")
    m, n = t.shape[-2:]
    if n > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    ld = t.stride(-2) if m > 1 else n
    if ld < n:
        raise ValueError(f"{name}'s rows overlap")
    batch = t.shape[0] if t.dim() == 3 else 1
    return t.data_ptr(), batch, m, n, ld, t.stride(0) if batch > 1 else m * ld


def _ortho_params(x, out, steps, coeffs, eps, scale):
    px, batch, m, n, x_ld, x_stride = _matrices(x, "x")
    po, out_ld, out_stride = None, n, m * n
    if out is not None:
        if out.dtype != x.dtype or out.shape != x.shape:
            raise ValueError(f"out is {out.dtype} {tuple(out.shape)}, x {x.dtype} {tuple(x.shape)}")
        po, _, _, _, out_ld, out_stride = _matrices(out, "out")
    c = None
    if coeffs is not None:
        flat = list(coeffs)
        if flat and not isinstance(flat[0], (int, float)):
            flat = [v for step in flat for v in step]
        elif len(flat) == 3:
            flat = flat * steps
        if len(flat) != 3 * steps:
            raise ValueError("coeffs must be (a, b, c), or one such triple for each step")
        c = (ctypes.c_float * max(1, len(flat)))(*flat)
    p = hc_orthogonalise_params(m, n, batch, x_ld, x_stride, out_ld, out_stride, _type(x, "x"), steps,
                                c, eps, scale)
    return p, px, po


def hc_orthogonalise_bytes(x, steps: int = 5) -> int:
    p, _, _ = _ortho_params(x, None, steps, None, 1e-7, 1.0)
    b = _Z()
    _check(_lib.hc_orthogonalise_bytes(ctypes.byref(p), ctypes.byref(b)), "hc_orthogonalise_bytes")
    return b.value


def alloc_orthogonalise_workspace(x):
    """Workspace of hc_orthogonalise for matrices of x's shape and type."""
    import torch
    return torch.empty(max(hc_orthogonalise_bytes(x), 256), dtype=torch.uint8, device=x.device)


def hc_orthogonalise(x, out, ws, steps: int = 5, coeffs=MUON, eps: float = 1e-7,
                     scale: float = 1.0, stream=None):
    """out = scale * X_steps, X_0 = x / (|x|_F + eps), X <- a X + (b A + c A^2) X with A = X X^T.
    x, out: [m, n] or [batch, m, n] float32 or bfloat16, rows contiguous; coeffs (a, b, c), or a
    triple for each step."""
    p, px, po = _ortho_params(x, out, steps, coeffs, eps, scale)
    _check(_lib.hc_orthogonalise(ctypes.byref(p), px, po, _bytes(ws), ws.numel(),
                                 _stream(stream)), "hc_orthogonalise")
