"""Python binding of the training-side operators (include/hc_train.h): embedding
lookup with scaling, its gradient by sorted token ids, Newton-Schulz
orthogonalisation, dropout, and the linear layer with its gradient.  Argument marshalling only, like the package's other calls;
the names mirror the C ABI:

    hc_embed              out[i] = scale * table[ids[i]]
    hc_embed_grad         the gradient of the whole table (zeros where no id
                          points), or added to one
    hc_embed_grad_rows    the touched rows alone: ids, sums and their number
    hc_orthogonalise      the Newton-Schulz polynomial of a matrix, as the Muon
                          optimiser orthogonalises an update
    hc_dropout            dropout or its gradient, with a residual
    hc_linear             matrix product with bias, activation, dropout, residual
    hc_linear_grad        its gradient: of the input, the weight and the bias
"""
from __future__ import annotations

import ctypes

from . import _check, _lib, _ptr, _stream, _u32

HC_T_I32, HC_T_F32, HC_T_BF16, HC_T_F16 = range(4)
FIXED_POINT = 2.0**20          # fixed point of the int32 gradients
MUON = (3.4445, -4.7750, 2.0315)

TRAIN_EXPORTS = ("hc_embed", "hc_embed_grad_bytes", "hc_embed_grad", "hc_embed_grad_rows",
                 "hc_orthogonalise_bytes", "hc_orthogonalise", "hc_dropout", "hc_linear_bytes",
                 "hc_linear", "hc_linear_grad_bytes", "hc_linear_grad")
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, "tanh": 4, "sigmoid": 5}


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


class hc_dropout_params(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_uint64), ("cols", ctypes.c_uint64), ("x_ld", ctypes.c_uint64),
                ("residual_ld", ctypes.c_uint64), ("out_ld", ctypes.c_uint64),
                ("seed", ctypes.c_uint64), ("draw", ctypes.c_uint64), ("p", ctypes.c_float),
                ("reserved", ctypes.c_uint32)]


class hc_linear_params(ctypes.Structure):
    _fields_ = [("m", ctypes.c_uint64), ("n", ctypes.c_uint64), ("k", ctypes.c_uint64),
                ("x_ld", ctypes.c_uint64), ("w_ld", ctypes.c_uint64), ("y_ld", ctypes.c_uint64),
                ("z_ld", ctypes.c_uint64), ("residual_ld", ctypes.c_uint64),
                ("dx_ld", ctypes.c_uint64), ("dw_ld", ctypes.c_uint64),
                ("seed", ctypes.c_uint64), ("draw", ctypes.c_uint64), ("p", ctypes.c_float),
                ("act", ctypes.c_uint32), ("fixed", ctypes.c_float), ("reserved", ctypes.c_uint32)]


_P, _Z = ctypes.c_void_p, ctypes.c_size_t
_EP, _OP = ctypes.POINTER(hc_embed_params), ctypes.POINTER(hc_orthogonalise_params)
_lib.hc_embed.argtypes = [_EP, ctypes.c_int, _P, _P, _P, _P]
_lib.hc_embed_grad_bytes.argtypes = [_EP, ctypes.POINTER(_Z)]
_lib.hc_embed_grad.argtypes = [_EP, ctypes.c_int, _P, _P, ctypes.c_int, _P, ctypes.c_int, _P, _Z, _P]
_lib.hc_embed_grad_rows.argtypes = [_EP, ctypes.c_int, _P, _P, ctypes.c_int, _P, _P,
                                    ctypes.c_uint64, _P, _P, _Z, _P]
_lib.hc_orthogonalise_bytes.argtypes = [_OP, ctypes.POINTER(_Z)]
_lib.hc_orthogonalise.argtypes = [_OP, _P, _P, _P, _Z, _P]
_DP, _LP = ctypes.POINTER(hc_dropout_params), ctypes.POINTER(hc_linear_params)
_lib.hc_dropout.argtypes = [_DP, ctypes.c_int, _P, _P, _P, _P, _P]
_lib.hc_linear_bytes.argtypes = [_LP, ctypes.c_int, ctypes.POINTER(_Z)]
_lib.hc_linear.argtypes = [_LP, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P, _Z, _P]
_lib.hc_linear_grad_bytes.argtypes = [_LP, ctypes.c_int, ctypes.POINTER(_Z)]
_lib.hc_linear_grad.argtypes = [_LP, ctypes.c_int, _P, _P, _P, _P, _P, ctypes.c_int, _P, _P,
                                ctypes.c_int, _P, _P, _Z, _P]
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


_device = _UINT8 = None     # the current device's number, torch's byte; filled by the first call


def _current():
    """The current device, whose stream the layer operators use and whose tensors they take."""
    global _device, _UINT8
    if _device is None:
        import torch
        _UINT8 = torch.uint8
        if not torch.cuda.is_available():
            return None             # no tensor is on it
        _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _device()


def _here(t, name, device):
    if t.get_device() != device:    # -1: not a device tensor
        raise ValueError(f"{name} must be a device tensor of the current device ({device}), not of {t.device}")


def _matrix(t, name, device):
    """(device pointer, rows, columns, row stride), as _rows'."""
    if t.get_device() != device:
        _here(t, name, device)
    shape = t.shape
    if len(shape) == 2 and t.is_contiguous():
        rows, cols = shape
        return t.data_ptr(), rows, cols, cols
    return _rows(t, name)


def _like(t, name, x, rows, cols, device):
    """(pointer, row stride) of a [rows, cols] tensor of x's type; None: none."""
    if t is None:
        return None, 0
    if t.dtype != x.dtype:
        raise ValueError(f"{name} is {t.dtype}, expected {x.dtype}")
    p, r, c, ld = _matrix(t, name, device)
    if r != rows or c != cols:
        raise ValueError(f"{name} is {r} x {c}, expected {rows} x {cols}")
    return p, ld


def _vector(t, name, dtype, n, device):
    """Pointer of n contiguous elements; None: none."""
    if t is None:
        return None
    if t.get_device() != device:
        _here(t, name, device)
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be {n} contiguous elements of {dtype}, not {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _workspace(ws, device):
    """(pointer, bytes)"""
    n = ws.numel()
    return _vector(ws, "ws", _UINT8, n, device), n


def _counter(t, device):
    """Pointer of the counter, the first element where there are more."""
    if t is None:
        return None
    import torch
    dtype = torch.uint64 if t.dtype == getattr(torch, "uint64", None) else torch.int64
    return _vector(t, "counter", dtype, max(1, t.numel()), device)


_LOW = 2**64 - 1


def hc_dropout(x, out, p: float, seed: int, draw: int = 0, residual=None, counter=None, stream=None):
    """out = residual + mask * x, or mask * x: an element is dropped with probability p (a multiple
    of 2^-16), the others are scaled by 1 / (1 - p).  x, out and residual [.., cols] float32,
    bfloat16 or float16; out may be x or residual.  The mask depends on seed, draw and an
    element's row and column alone: the same call on an output gradient is the backward pass.
    counter (int64, one element, on the device) is added to draw when the kernel runs."""
    device = _current()
    px, rows, cols, x_ld = _matrix(x, "x", device)
    po, out_ld = _like(out, "out", x, rows, cols, device)
    pr, r_ld = _like(residual, "residual", x, rows, cols, device)
    q = hc_dropout_params(rows, cols, x_ld, r_ld, out_ld, seed & _LOW, draw & _LOW, p, 0)
    _check(_lib.hc_dropout(ctypes.byref(q), _type(x, "x"), px, pr, po, _counter(counter, device),
                           _stream(stream)), "hc_dropout")


def _act(act):
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError(f"act is {act!r}, expected one of {tuple(ACTIVATIONS)}")
    return code


def _layer(m, n, k, x_ld, w_ld, y_ld, z_ld=0, residual_ld=0, dx_ld=0, dw_ld=0, seed=0, draw=0, p=0.0,
           act="none", fixed=1.0):
    return hc_linear_params(m, n, k, x_ld, w_ld, y_ld, z_ld, residual_ld, dx_ld, dw_ld, seed & _LOW,
                            draw & _LOW, p, _act(act), fixed, 0)


def _layer_bytes(call, where, x, w):
    px, m, k, x_ld = _rows(x, "x")
    pw, n, kw, w_ld = _rows(w, "w")
    if kw != k:
        raise ValueError(f"w has {kw} columns, x {k}")
    b = _Z()
    _check(call(ctypes.byref(_layer(m, n, k, x_ld, w_ld, n)), _type(x, "x"), ctypes.byref(b)), where)
    return b.value


def hc_linear_bytes(x, w) -> int:
    return _layer_bytes(_lib.hc_linear_bytes, "hc_linear_bytes", x, w)


def alloc_linear_workspace(x, w):
    """Workspace of hc_linear for x [.., k] and w [n, k] (and for fewer rows of x)."""
    import torch
    return torch.empty(max(hc_linear_bytes(x, w), 256), dtype=torch.uint8, device=x.device)


def hc_linear(x, w, y, ws, bias=None, residual=None, z=None, act: str = "none", p: float = 0.0,
              seed: int = 0, draw: int = 0, counter=None, stream=None):
    """y = residual + mask * act(x w^T + bias), with hc_dropout's mask of y's rows and columns where
    p > 0.  x [.., k], w [n, k], bias [n], residual, y and z [.., n], all float32, bfloat16 or
    float16; act "none", "relu", "gelu" (by erf), "silu", "tanh" or "sigmoid".  z, where given,
    gets x w^T + bias: hc_linear_grad reads it.  y may be residual."""
    device = _current()
    px, m, k, x_ld = _matrix(x, "x", device)
    pw, n, kw, w_ld = _matrix(w, "w", device)
    dtype = x.dtype
    if kw != k or w.dtype != dtype:
        raise ValueError(f"w is {w.dtype} with {kw} columns, x {dtype} with {k}")
    py, y_ld = _like(y, "y", x, m, n, device)
    pz, z_ld = _like(z, "z", x, m, n, device)
    pr, r_ld = _like(residual, "residual", x, m, n, device)
    pws, ws_bytes = _workspace(ws, device)
    q = _layer(m, n, k, x_ld, w_ld, y_ld, z_ld, r_ld, 0, 0, seed, draw, p, act)
    _check(_lib.hc_linear(ctypes.byref(q), _type(x, "x"), px, pw, _vector(bias, "bias", dtype, n, device),
                          pr, py, pz, _counter(counter, device), pws, ws_bytes, _stream(stream)),
           "hc_linear")


def hc_linear_grad_bytes(x, w) -> int:
    return _layer_bytes(_lib.hc_linear_grad_bytes, "hc_linear_grad_bytes", x, w)


def alloc_linear_grad_workspace(x, w):
    """Workspace of hc_linear_grad for x [.., k] and w [n, k] (and for fewer rows of x)."""
    import torch
    return torch.empty(max(hc_linear_grad_bytes(x, w), 256), dtype=torch.uint8, device=x.device)


def hc_linear_grad(dy, ws, x=None, w=None, z=None, dx=None, dw=None, db=None, act: str = "none",
                   p: float = 0.0, seed: int = 0, draw: int = 0, fixed: float = FIXED_POINT,
                   accumulate: bool = False, counter=None, stream=None):
    """The gradient of hc_linear for the output gradient dy [.., n]: dz = act'(z) * mask * dy, then
    dx = dz w, dw = dz^T x and db = dz's rows summed, those of them that are given.  dx needs w, dw
    needs x, an activation needs z; dy, x, w, z and dx are of one type.  dw [n, k] and db [n] are
    both float32, bfloat16, float16, or int32: fixed point with `fixed` units per 1.0; accumulate
    adds to them.  The residual's gradient is dy itself."""
    device = _current()
    py, m, n, y_ld = _matrix(dy, "dy", device)
    if dx is not None and w is None:
        raise ValueError("dx needs w")
    if dw is not None and x is None:
        raise ValueError("dw needs x")
    if act != "none" and z is None:
        raise ValueError(f"the gradient of {act} needs z")
    k = 1
    for t in (x, w, dx, dw):
        if t is not None:
            k = t.shape[-1]
            break
    px, x_ld = _like(x, "x", dy, m, k, device)
    pw, w_ld = _like(w, "w", dy, n, k, device)
    pz, z_ld = _like(z, "z", dy, m, n, device)
    pdx, dx_ld = _like(dx, "dx", dy, m, k, device)
    pdw, dw_ld, g_type, pdb = None, 0, HC_T_F32, None
    if dw is not None:
        pdw, rows, cols, dw_ld = _matrix(dw, "dw", device)
        g_type = _type(dw, "dw")
        if rows != n or cols != k:
            raise ValueError(f"dw is {rows} x {cols}, expected {n} x {k}")
    if db is not None:
        pdb = _vector(db, "db", db.dtype if dw is None else dw.dtype, n, device)
        g_type = _type(db, "db")
    pws, ws_bytes = _workspace(ws, device)
    q = _layer(m, n, k, x_ld or k, w_ld or k, y_ld, z_ld, 0, dx_ld, dw_ld, seed, draw, p, act, fixed)
    _check(_lib.hc_linear_grad(ctypes.byref(q), _type(dy, "dy"), py, px, pw, pz, pdx, g_type, pdw,
                               pdb, 1 if accumulate else 0, _counter(counter, device), pws, ws_bytes,
                               _stream(stream)), "hc_linear_grad")
