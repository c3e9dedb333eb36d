"""A learner's operators (the C ABI in include/ps_learner.h) for torch device tensors.

What a learner computes between a pull and a push with the layers that hold most
of the server's parameters: embedding tables and fully connected layers, the latter
in 8-bit floating point with a scale per block of 128, dropout, and the norms around
a residual block of layers; the AdamW step that it makes of a gradient (`AdamW`); and
layers in 8-bit integers, with which a replica answers. Weights are
read where they lie in a replica (any view with unit column stride), weight
gradients are written where they belong in a gradient row.

Native calls make their results past torch's dispatcher: its modes, and the deterministic fill of new
memory, do not see them.

No call records anything for autograd: a result does not require a gradient, whatever its
arguments do. The backward pass is a call of its own (`embedding_grad`, `linear_fp8_grad`,
`residual_norm_grad`, `dropout` again).

Every call enqueues its kernels on torch's current stream and returns without
waiting; as with torch's own operators, a tensor last used on another stream is
for the caller to order and to record. Refused arguments raise `TypeError` or
`ValueError` (shapes, types, devices) or `PSError` (what the library refuses). There
is no CPU fallback: if the library is not built, the first call raises.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import NamedTuple, Optional, Sequence, Tuple, Union

import torch

from .ps import PS_BF16, PS_EINVAL, PS_F32, PS_OK, PSError

PL_I32 = 0
PL_I64 = 1

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgadeilearner.so")


class pl_drop(ctypes.Structure):
    _fields_ = [("p", ctypes.c_float), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64)]


class pl_fp8(ctypes.Structure):
    _fields_ = [("values", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


class pl_int8(ctypes.Structure):
    _fields_ = [("values", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


class pl_adamw_tensor(ctypes.Structure):
    _fields_ = [("weight", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("count", ctypes.c_int64),
                ("decay", ctypes.c_float)]


_VP, _INT, _I64, _SIZE = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
_F32, _F64, _U64 = ctypes.c_float, ctypes.c_double, ctypes.c_uint64
_DROP, _FP8 = ctypes.POINTER(pl_drop), ctypes.POINTER(pl_fp8)
_INT8, _ADAMW = ctypes.POINTER(pl_int8), ctypes.POINTER(pl_adamw_tensor)
_SIGS = {
    "pl_embedding": (_INT, [_VP, _INT, _I64, _VP, _INT, _I64, _I64, _I64, ctypes.c_float, _DROP,
                            _VP, _INT, _I64, _VP]),
    "pl_embedding_grad": (_INT, [_VP, _INT, _I64, _VP, _INT, _I64, _I64, ctypes.c_float, _DROP, _VP,
                                 _INT, _I64, _I64, _INT, _VP, _SIZE, _VP]),
    "pl_embedding_grad_workspace": (_SIZE, [_I64, _I64, _I64]),
    "pl_dropout": (_INT, [_VP, _INT, _I64, _I64, _I64, _DROP, _VP, _I64, _VP]),
    "pl_fp8_ld": (_I64, [_I64]),
    "pl_fp8_values_bytes": (_SIZE, [_I64, _I64]),
    "pl_fp8_scales_bytes": (_SIZE, [_I64, _I64]),
    "pl_quantize_fp8": (_INT, [_VP, _INT, _I64, _I64, _I64, _INT, _FP8, _FP8, _VP]),
    "pl_matmul_fp8": (_INT, [_I64, _I64, _I64, _FP8, _FP8, _VP, _INT, _INT, _VP, _INT, _I64, _INT,
                             _VP, _SIZE, _VP]),
    "pl_matmul_fp8_workspace": (_SIZE, [_I64, _I64, _I64, _INT]),
    "pl_linear_fp8": (_INT, [_VP, _INT, _I64, _I64, _I64, _I64, _FP8, _VP, _INT, _INT, _VP, _INT, _I64,
                             _VP, _SIZE, _VP]),
    "pl_linear_fp8_workspace": (_SIZE, [_I64, _I64, _I64, _INT, _INT]),
    "pl_linear_fp8_grad": (_INT, [_VP, _INT, _I64, _VP, _INT, _I64, _I64, _I64, _I64, _FP8, _VP, _INT,
                                  _I64, _VP, _INT, _I64, _INT, _VP, _SIZE, _VP]),
    "pl_linear_fp8_grad_workspace": (_SIZE, [_I64, _I64, _I64, _INT, _INT]),
    "pl_norm": (_INT, [_VP, _INT, _I64, _VP, _INT, _I64, _I64, _I64, _VP, _INT, _I64, _I64, _VP, _VP, _INT,
                       _F32, _F32, _VP, _I64, _VP, _I64, _VP]),
    "pl_norm_grad": (_INT, [_VP, _INT, _I64, _VP, _INT, _I64, _VP, _I64, _VP, _I64, _I64, _I64, _VP, _INT, _I64,
                            _I64, _VP, _VP, _INT, _F32, _F32, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _VP, _INT,
                            _INT, _VP, _SIZE, _VP]),
    "pl_norm_grad_workspace": (_SIZE, [_I64, _I64]),
    "pl_int8_ld": (_I64, [_I64]),
    "pl_int8_values_bytes": (_SIZE, [_I64, _I64]),
    "pl_quantize_int8": (_INT, [_VP, _INT, _I64, _I64, _I64, _INT8, _VP]),
    "pl_matmul_int8": (_INT, [_I64, _I64, _I64, _INT8, _INT8, _VP, _INT, _INT, _VP, _INT, _I64, _VP, _SIZE, _VP]),
    "pl_matmul_int8_workspace": (_SIZE, [_I64, _I64, _I64]),
    "pl_linear_int8": (_INT, [_VP, _INT, _I64, _I64, _I64, _I64, _INT8, _VP, _INT, _INT, _VP, _INT, _I64, _VP,
                              _SIZE, _VP]),
    "pl_linear_int8_workspace": (_SIZE, [_I64, _I64, _I64]),
    "pl_adamw_room": (_I64, [_ADAMW, _I64]),
    "pl_adamw_parts": (_I64, [_ADAMW, _I64]),
    "pl_adamw_plan_bytes": (_SIZE, [_I64]),
    "pl_adamw_plan": (_INT, [_ADAMW, _I64, _INT, _INT, _INT, _I64, _VP, _SIZE]),
    "pl_adamw_steps": (_I64, [_VP]),
    "pl_adamw_step": (_INT, [_VP, _I64, _INT, _INT, _INT, _INT, _I64, _VP, _VP, _VP, _VP, _F64, _F64, _F32, _F32,
                             _VP, _F32, _VP, _U64, _VP]),
    "pl_adamw_moments": (_INT, [_I64, _VP, _VP, _VP, _VP, _VP, _VP, _INT, _VP]),
    "pl_last_error": (ctypes.c_char_p, []),
}

_lib = None


def load_library(path: Optional[str] = None):
    """Load the built library (once). Raises if it is missing."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(
            f"{p} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
            "(a learner's operators have no CPU fallback)")
    L = ctypes.CDLL(p)
    for name, (res, args) in _SIGS.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    if path is None:
        _lib = L
    return L


def _check(rc: int) -> None:
    if rc != PS_OK:
        raise PSError(rc, load_library().pl_last_error().decode())


_native = None   # the native calls' module; False: not built


def _native_calls():
    """The native side of the calls below, or False where it is not built (or built for
    another torch): they then go through ctypes, which is slower."""
    global _native
    if _native is None:
        load_library()
        try:
            from . import _learner
            _native = _learner
        except ImportError as e:
            warnings.warn(f"a learner's calls go through ctypes, which is slower: {e}", RuntimeWarning,
                          stacklevel=3)
            _native = False
    return _native


def _done(result) -> bool:
    """Whether a native call has made the call: it returns None for arguments that it does not
    take, and the status of a call that was refused."""
    if result is None:
        return False
    if type(result) is int:
        _check(result)
    return True


_CODES = {torch.float32: PS_F32, torch.bfloat16: PS_BF16}
_ID_CODES = {torch.int32: PL_I32, torch.int64: PL_I64}


def _code(dtype) -> int:
    code = _CODES.get(dtype)
    if code is None:
        raise TypeError(f"float32 or bfloat16 expected, not {dtype}")
    return code


def _on_device(name: str, t) -> None:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: a tensor expected, not {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{name}: a device tensor expected")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, the current device is "
                         f"cuda:{torch.cuda.current_device()}")


def _matrix(name: str, t, rows: Optional[int] = None, cols: Optional[int] = None):
    """(pointer, dtype code, row stride) of a matrix with unit column stride."""
    _on_device(name, t)
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or \
            (cols is not None and t.shape[1] != cols):
        want = f"{'any' if rows is None else rows} x {'any' if cols is None else cols}"
        raise ValueError(f"{name}: a matrix of {want} expected, not {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: neighbouring columns are {t.stride(1)} elements apart")
    # a row stride of 0, of rows that share their memory, is refused by the library
    return t.data_ptr(), _code(t.dtype), t.stride(0)


def _flat(name: str, t, rows: int, cols: int):
    try:
        return t.view(rows, cols)
    except RuntimeError as e:
        raise ValueError(f"{name}: its rows, of shape {tuple(t.shape)} with strides {t.stride()}, are not those "
                         "of a matrix") from e


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


class Dropout(NamedTuple):
    """Which elements a call drops: each with probability `p` (to the nearest 2^-16),
    by its row and column, `seed` and `offset` alone. A backward pass names the same
    three; a layer that is to drop other elements at its next call takes another
    offset."""
    p: float
    seed: int
    offset: int = 0


def _drop(drop: Optional[Dropout]):
    if drop is None:
        return None
    if not isinstance(drop, tuple) or len(drop) != 3:
        raise TypeError(f"drop: a Dropout expected, not {type(drop).__name__}")
    drop = Dropout(*drop)
    if not 0 <= drop.seed < 1 << 64 or not 0 <= drop.offset < 1 << 64:
        raise ValueError("dropout: seed and offset are 64-bit")
    return ctypes.byref(pl_drop(drop.p, drop.seed, drop.offset))


def _ids(ids):
    _on_device("ids", ids)
    code = _ID_CODES.get(ids.dtype)
    if code is None:
        raise TypeError(f"ids: int32 or int64 expected, not {ids.dtype}")
    return ids if ids.is_contiguous() else ids.contiguous(), code


def embedding(ids, table, scale: float = 1.0, drop: Optional[Dropout] = None, dtype=None, out=None):
    """scale * table[ids], then dropout with the token's position in `ids` as the row.
    An id outside the table (padding) gives zeros. Shape: that of `ids`, then the table's
    columns; of `dtype` (the table's by default), or written to `out`, a matrix of one row
    per id."""
    if out is not None and dtype is not None and getattr(out, "dtype", dtype) != dtype:
        raise TypeError(f"out is {out.dtype}, not {dtype}")
    native = _native or _native_calls()
    if native:
        done = native.embedding(ids, table, scale, drop, dtype or getattr(table, "dtype", None), out)
        if _done(done):
            return done
    ids, id_code = _ids(ids)
    src, src_code, src_ld = _matrix("table", table)
    tokens, (vocab, dim) = ids.numel(), table.shape
    result = out
    if out is None:
        result = torch.empty((*ids.shape, dim), dtype=dtype or table.dtype, device=table.device)
        out = result.view(tokens, dim)
    dst, dst_code, dst_ld = _matrix("out", out, tokens, dim)
    _check(load_library().pl_embedding(ids.data_ptr(), id_code, tokens, src, src_code, vocab, dim,
                                       src_ld, scale, _drop(drop), dst, dst_code, dst_ld, _stream()))
    return result


def embedding_grad(ids, grad, rows: int, scale: float = 1.0, drop: Optional[Dropout] = None,
                   dtype=torch.float32, out=None, accumulate: bool = False):
    """The gradient of `embedding` for its table of `rows` rows, from `grad`, that of its
    result (the shape of `ids`, then the columns): every row of it, of `dtype` or written to
    `out`; with `accumulate` added to what `out` holds. Equal calls give equal bits."""
    native = _native or _native_calls()
    if native:
        done = native.embedding_grad(ids, grad, rows, scale, drop, dtype, out, accumulate)
        if _done(done):
            return done
    ids, id_code = _ids(ids)
    _on_device("grad", grad)
    tokens = ids.numel()
    if grad.dim() != 2:
        if tuple(grad.shape[:-1]) != tuple(ids.shape):
            raise ValueError(f"grad of shape {tuple(grad.shape)} for ids of {tuple(ids.shape)}")
        grad = grad.reshape(tokens, grad.shape[-1])
    src, src_code, src_ld = _matrix("grad", grad, rows=tokens)
    dim = grad.shape[1]
    if rows < 0:
        raise ValueError(f"{rows} rows")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((rows, dim), dtype=dtype, device=grad.device)
    dst, dst_code, dst_ld = _matrix("out", out, rows, dim)
    L = load_library()
    need = L.pl_embedding_grad_workspace(tokens, rows, dim)
    work = torch.empty(need, dtype=torch.uint8, device=grad.device)
    _check(L.pl_embedding_grad(ids.data_ptr(), id_code, tokens, src, src_code, src_ld, dim, scale,
                               _drop(drop), dst, dst_code, dst_ld, rows, int(bool(accumulate)),
                               work.data_ptr(), need, _stream()))
    return out


def dropout(x, drop: Dropout, out=None):
    """x with dropout, and of a gradient the backward pass. x is a matrix, or anything
    contiguous: then its last dimension is the columns and the others together the rows.
    `out` may be x."""
    native = _native or _native_calls()
    if native:
        done = native.dropout(x, drop, out)
        if _done(done):
            return done
    _on_device("x", x)
    if out is not None:
        _on_device("out", out)
    if out is not None and (out.shape != x.shape or out.dtype != x.dtype):
        raise ValueError(f"out of {tuple(out.shape)} {out.dtype} for x of {tuple(x.shape)} {x.dtype}")
    result = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
    if x.dim() != 2:
        cols = x.shape[-1] if x.dim() else 1
        rows = x.numel() // cols if cols else 0
        x, out = _flat("x", x, rows, cols), _flat("out", result, rows, cols)
    else:
        out = result
    rows, cols = x.shape
    src, code, src_ld = _matrix("x", x)
    dst, _, dst_ld = _matrix("out", out)
    _check(load_library().pl_dropout(src, code, rows, cols, src_ld, _drop(drop), dst, dst_ld,
                                     _stream()))
    return result


class Fp8Matrix:
    """A matrix in 8-bit floating point with a power-of-two scale per block of 128 columns
    of a row. `values` (rows x columns padded to whole blocks, torch.float8_e4m3fn) and
    `scales` (int32; the bytes are the exponents, plus 127, of four blocks) hold it as the
    library does."""

    def __init__(self, rows: int, cols: int, device):
        self.shape = (rows, cols)
        blocks = -(-cols // 128)
        self.values = torch.empty((rows, 128 * blocks), dtype=torch.float8_e4m3fn, device=device)
        self.scales = torch.empty((-(-blocks // 4), rows), dtype=torch.int32, device=device)

    @property
    def parts(self):
        """What the native calls take."""
        return (self.values, self.scales, *self.shape)

    def exponents(self):
        """The exponent of every block: rows x blocks, int32."""
        rows, cols = self.shape
        words, blocks = self.scales.shape[0], -(-cols // 128)
        per_byte = self.scales.view(torch.uint8).view(words, rows, 4)
        return per_byte.permute(1, 0, 2).reshape(rows, 4 * words)[:, :blocks].int() - 127

    def dequantize(self):
        """The values that it stands for, in fp32 (exact; 2^128, to which numbers next to fp32's
        largest round, is infinity)."""
        rows, cols = self.shape
        blocks = -(-cols // 128)
        two = ((self.exponents() + 127) << 23).view(torch.float32)
        values = self.values.float().view(rows, blocks, 128) * two[:, :, None]
        return values.view(rows, 128 * blocks)[:, :cols]


def _parts(name: str, q):
    if not isinstance(q, Fp8Matrix):
        raise TypeError(f"{name}: an Fp8Matrix expected, not {type(q).__name__}")
    return q.parts


def _ref(q: Optional[Fp8Matrix]):
    return None if q is None else ctypes.byref(pl_fp8(q.values.data_ptr(), q.scales.data_ptr()))


def _fp8(name: str, q: Fp8Matrix):
    """_ref(q) of a caller's matrix, whose tensors may have been exchanged for others."""
    rows, cols = q.shape
    blocks = -(-cols // 128)
    for part, t, dtype, shape in (("values", q.values, torch.float8_e4m3fn, (rows, 128 * blocks)),
                                  ("scales", q.scales, torch.int32, (-(-blocks // 4), rows))):
        _on_device(f"{name}.{part}", t)
        if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name}.{part}: contiguous {dtype} of {shape} expected, not {t.dtype} of "
                             f"{tuple(t.shape)}, {t.stride()} elements apart")
    return _ref(q)


def _quantize(x, square: bool, plain: bool, transposed: bool):
    src, code, ld = _matrix("x", x)
    rows, cols = x.shape
    out = Fp8Matrix(rows, cols, x.device) if plain else None
    out_t = Fp8Matrix(cols, rows, x.device) if transposed else None
    _check(load_library().pl_quantize_fp8(src, code, rows, cols, ld, int(bool(square)), _ref(out),
                                          _ref(out_t), _stream()))
    return out, out_t


def quantize_fp8(x, square: bool = False, transpose: bool = False) -> Fp8Matrix:
    """x, or its transpose, as an `Fp8Matrix`: one scale per 128 columns of a row of the
    result, or (square) per 128 x 128 tile, in which case x and its transpose hold the same
    values."""
    out, out_t = _quantize(x, square, not transpose, transpose)
    return out_t if transpose else out


def quantize_fp8_both(x, square: bool = False) -> Tuple[Fp8Matrix, Fp8Matrix]:
    """x and its transpose, read once."""
    return _quantize(x, square, True, True)


def _bias(bias, n: int):
    """(pointer, dtype code) of a bias of n values; none: (None, any code)."""
    if bias is None:
        return None, PS_F32
    _on_device("bias", bias)
    if bias.shape != (n,) or not bias.is_contiguous():
        raise ValueError(f"bias: {n} contiguous values expected, not {tuple(bias.shape)}")
    return bias.data_ptr(), _code(bias.dtype)


def matmul_fp8(a: Fp8Matrix, b: Fp8Matrix, bias=None, relu: bool = False, dtype=torch.bfloat16,
               out=None, accumulate: bool = False):
    """a b^T (+ bias, then max(., 0) with relu), of `dtype` or written to `out`; with
    `accumulate` added to what `out` holds.

    Results in fp32 have fp32 sums. Those in bf16 are summed by the 8-bit matrix instructions,
    twice as fast: of eight neighbouring products they keep 13 bits below the largest, which
    bf16's rounding covers unless large products cancel."""
    a_parts, b_parts = _parts("a", a), _parts("b", b)
    native = _native or _native_calls()
    if native:
        done = native.product(a_parts, b_parts, bias, relu, dtype, out, accumulate)
        if _done(done):
            return done
    (m, k), (n, k2) = a.shape, b.shape
    if k != k2:
        raise ValueError(f"rows of {k} and of {k2} columns")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((m, n), dtype=dtype, device=a.values.device)
    dst, code, ld = _matrix("out", out, m, n)
    a_ref, b_ref = _fp8("a", a), _fp8("b", b)
    bias_ptr, bias_code = _bias(bias, n)
    L = load_library()
    need = L.pl_matmul_fp8_workspace(m, n, k, code)
    work = torch.empty(need, dtype=torch.uint8, device=out.device) if need else None
    _check(L.pl_matmul_fp8(m, n, k, a_ref, b_ref, bias_ptr, bias_code, int(bool(relu)), dst, code, ld,
                           int(bool(accumulate)), work.data_ptr() if need else None, need, _stream()))
    return out


def linear_fp8(x, w: Fp8Matrix, bias=None, relu: bool = False, dtype=torch.bfloat16, out=None):
    """A fully connected layer: x w^T (+ bias, relu). x is quantised along its rows; w is the
    layer's weight (outputs x inputs), quantised (square) once per pull. Sums are those of
    `matmul_fp8` for the result's type."""
    w_parts = _parts("w", w)
    native = _native or _native_calls()
    if native:
        done = native.linear(x, w_parts, bias, relu, dtype, out)
        if _done(done):
            return done
    src, code, src_ld = _matrix("x", x, cols=w.shape[1])
    m, (n, k) = x.shape[0], w.shape
    w_ref = _fp8("w", w)
    if out is None:
        out = torch.empty((m, n), dtype=dtype, device=x.device)
    dst, dst_code, dst_ld = _matrix("out", out, m, n)
    bias_ptr, bias_code = _bias(bias, n)
    L = load_library()
    need = L.pl_linear_fp8_workspace(m, n, k, code, dst_code)
    work = torch.empty(need, dtype=torch.uint8, device=x.device)
    _check(L.pl_linear_fp8(src, code, m, k, src_ld, n, w_ref, bias_ptr, bias_code, int(bool(relu)), dst,
                           dst_code, dst_ld, work.data_ptr(), need, _stream()))
    return out


def linear_fp8_grad(x, grad, w_t: Fp8Matrix, dtype=torch.bfloat16, weight_dtype=torch.float32,
                    x_out=None, weight_out=None, accumulate: bool = False):
    """Gradients of x w^T from `grad`, that of the result: (for x, for w). w_t is the
    transposed weight, quantised (square); grad is quantised along its rows for the first
    product and along its columns, as x, for the second. `weight_out`, a view into the
    learner's gradient row, is written, or with `accumulate` added to. Sums are those of
    `matmul_fp8` for each result's type."""
    w_parts = _parts("w_t", w_t)
    native = _native or _native_calls()
    if native:
        done = native.linear_grad(x, grad, w_parts, dtype, weight_dtype, x_out, weight_out, accumulate)
        if _done(done):
            return done
    k, n = w_t.shape
    src, code, src_ld = _matrix("x", x, cols=k)
    m = x.shape[0]
    grd, grd_code, grd_ld = _matrix("grad", grad, m, n)
    w_ref = _fp8("w_t", w_t)
    if x_out is None:
        x_out = torch.empty((m, k), dtype=dtype, device=x.device)
    if weight_out is None:
        if accumulate:
            raise ValueError("accumulate needs weight_out")
        weight_out = torch.empty((n, k), dtype=weight_dtype, device=x.device)
    dst, dst_code, dst_ld = _matrix("x_out", x_out, m, k)
    wgt, wgt_code, wgt_ld = _matrix("weight_out", weight_out, n, k)
    L = load_library()
    need = L.pl_linear_fp8_grad_workspace(m, n, k, dst_code, wgt_code)
    work = torch.empty(need, dtype=torch.uint8, device=x.device)
    _check(L.pl_linear_fp8_grad(src, code, src_ld, grd, grd_code, grd_ld, m, n, k, w_ref, dst,
                                dst_code, dst_ld, wgt, wgt_code, wgt_ld, int(bool(accumulate)),
                                work.data_ptr(), need, _stream()))
    return x_out, weight_out


# ------------------------------------------------- norms around a block

def _vector(name: str, t, cols: int):
    """(pointer, dtype code) of `cols` contiguous values; none: (None, None)."""
    if t is None:
        return None, None
    _on_device(name, t)
    if t.shape != (cols,) or not t.is_contiguous():
        raise ValueError(f"{name}: {cols} contiguous values expected, not {tuple(t.shape)}")
    return t.data_ptr(), _code(t.dtype)


def _one_type(what: str, *codes) -> int:
    """The dtype code of tensors of one type, some of which may be missing (all: any)."""
    there = {c for c in codes if c is not None}
    if len(there) > 1:
        raise TypeError(f"{what} are of different types")
    return there.pop() if there else PS_F32


def _gate(name: str, gate, rows: int, cols: int):
    """(pointer, dtype code, rows, row stride) of a gate: `cols` values for all rows, or a matrix. The library refuses
    one of no rows that has an address; of a stream of no rows either it may be none at all."""
    if gate is None:
        return None, PS_F32, 0, 0
    _on_device(name, gate)
    m = gate[None] if gate.dim() == 1 else gate
    ptr, code, ld = _matrix(name, m, cols=cols)
    return _there(ptr) if rows or m.shape[0] else None, code, m.shape[0], ld


def _like(name: str, out, rows: int, cols: int, dtype, device):
    """`out`, of `dtype`, or a new matrix."""
    if out is None:
        return torch.empty((rows, cols), dtype=dtype, device=device)
    _matrix(name, out, rows, cols)
    if out.dtype != dtype:
        raise TypeError(f"{name} is {out.dtype}, not {dtype}")
    return out


def _there(ptr) -> int:
    """An empty tensor has no address, which stands for a tensor that is not given: any other does."""
    return ptr or 256


def rms_norm(x, weight=None, eps: float = 1e-6, dtype=None, out=None):
    """weight * x / sqrt(mean(x^2) + eps) over each row of x, a matrix: of `dtype` (that of x by default), or
    written to `out`."""
    native = _native or _native_calls()
    if native:
        done = native.norm(x, None, None, None, weight, 1.0, eps, dtype, None, out)
        if _done(done):
            return done
    src, code, ld = _matrix("x", x)
    rows, cols = x.shape
    w, w_code = _vector("weight", weight, cols)
    if out is not None:
        _on_device("out", out)
    out = _like("out", out, rows, cols, dtype or (x if out is None else out).dtype, x.device)
    dst, dst_code, dst_ld = _matrix("out", out)
    _check(load_library().pl_norm(src, code, ld, None, dst_code, 0, rows, cols, None, PS_F32, 0, 0, None, w,
                                  _one_type("weights", w_code), 1.0, eps, None, 0, _there(dst), dst_ld,
                                  _stream()))
    return out


def residual_norm(x, y, gate=None, after=None, before=None, scale: float = 1.0, eps: float = 1e-6, out=None,
                  normed_out=None):
    """What a block's output y leaves in the stream x, and the next block's input:

        h = scale * x + gate * after * N(y)        z = before * N(h),   N(v) = v / sqrt(mean(v^2) + eps)

    over rows; without `after` the block's output is not normed, without `gate` not gated. Returns (h, z), or
    (h, None) without `before`. h is of x's type, z, of the h that is not yet rounded, of y's. `gate` has a value
    for each column, or is a matrix whose rows (one at least, if x has any) are each for as many neighbouring rows of
    x."""
    native = _native or _native_calls()
    if native:
        done = native.norm(x, y, gate, after, before, scale, eps, None, out, normed_out)
        if _done(done):
            return done
    src, code, ld = _matrix("x", x)
    rows, cols = x.shape
    blk, blk_code, blk_ld = _matrix("y", y, rows, cols)
    gt, gt_code, gates, gt_ld = _gate("gate", gate, rows, cols)
    (aft, aft_code), (bef, bef_code) = _vector("after", after, cols), _vector("before", before, cols)
    if before is None and normed_out is not None:
        raise ValueError("normed_out without before")
    out = _like("out", out, rows, cols, x.dtype, x.device)
    dst, _, dst_ld = _matrix("out", out)
    normed, nrm, nrm_ld = None, None, 0
    if before is not None:
        normed = _like("normed_out", normed_out, rows, cols, y.dtype, x.device)
        nrm, _, nrm_ld = _matrix("normed_out", normed)
    _check(load_library().pl_norm(
        src, code, ld, _there(blk), blk_code, blk_ld, rows, cols, gt, gt_code, gates, gt_ld, aft, bef,
        _one_type("after and before", aft_code, bef_code), scale, eps, dst, dst_ld, nrm, nrm_ld, _stream()))
    return out, normed


class NormGrads(NamedTuple):
    """Gradients of `residual_norm` for what they are named after; None for what was not given."""
    x: torch.Tensor
    y: torch.Tensor
    gate: Optional[torch.Tensor]
    after: Optional[torch.Tensor]
    before: Optional[torch.Tensor]


def _weight_out(name: str, out, like, dtype, accumulate: bool):
    """Where the gradient of `like` (a vector or a matrix, or None) goes: a matrix, and what is returned."""
    if like is None:
        if out is not None:
            raise ValueError(f"{name} for what is not given")
        return None, None
    if out is None:
        if accumulate:
            raise ValueError(f"accumulate needs {name}")
        out = torch.empty(like.shape, dtype=dtype, device=like.device)
    _on_device(name, out)
    if out.shape != like.shape or (out.dim() == 1 and not out.is_contiguous()):
        raise ValueError(f"{name} of {tuple(out.shape)} for {tuple(like.shape)}")
    return out[None] if out.dim() == 1 else out, out


def _norm_grad(h, y, grad, normed_grad, gate, after, before, scale, eps, weight_dtype, x_out, y_out, gate_out,
               after_out, before_out, accumulate):
    native = _native or _native_calls()
    if native:
        done = native.norm_grad(h, y, grad, normed_grad, gate, after, before, scale, eps, weight_dtype, x_out, y_out,
                                gate_out, after_out, before_out, accumulate)
        if _done(done):
            return done
    src, code, ld = _matrix("h", h)
    rows, cols = h.shape
    blk, blk_code, blk_ld = (None, None, 0) if y is None else _matrix("y", y, rows, cols)
    grd, grd_ld, nrm, nrm_ld = None, 0, None, 0
    if grad is not None:
        grd, grd_code, grd_ld = _matrix("grad", grad, rows, cols)
        if grd_code != code:
            raise TypeError(f"grad is {grad.dtype}, h {h.dtype}")
    if normed_grad is not None:
        nrm, nrm_code, nrm_ld = _matrix("normed_grad", normed_grad, rows, cols)
        if blk_code is not None and nrm_code != blk_code:
            raise TypeError(f"normed_grad is {normed_grad.dtype}, y {y.dtype}")
        blk_code = nrm_code
    gt, gt_code, gates, gt_ld = _gate("gate", gate, rows, cols)
    (aft, aft_code), (bef, bef_code) = _vector("after", after, cols), _vector("before", before, cols)
    if before is not None and normed_grad is None:
        raise ValueError("before without normed_grad")
    x_out = _like("x_out", x_out, rows, cols, h.dtype, h.device)
    y_out = None if y is None else _like("y_out", y_out, rows, cols, y.dtype, h.device)
    outs = [_weight_out(f"{name}_out", out, like, weight_dtype, accumulate) for name, out, like in (
        ("gate", gate_out, gate), ("after", after_out, after), ("before", before_out, before))]
    ptrs = [(None, None, 0) if m is None else _matrix("a gradient of weights", m) for m, _ in outs]
    out_code = _one_type("gate_out, after_out and before_out", *(p[1] for p in ptrs))
    L = load_library()
    need = L.pl_norm_grad_workspace(rows, cols)
    work = torch.empty(need, dtype=torch.uint8, device=h.device)
    _check(L.pl_norm_grad(
        src, code, ld, None if y is None else _there(blk), code if blk_code is None else blk_code, blk_ld,
        None if grad is None else _there(grd), grd_ld, None if normed_grad is None else _there(nrm), nrm_ld, rows, cols,
        gt, gt_code, gates, gt_ld, aft, bef, _one_type("after and before", aft_code, bef_code), scale, eps,
        x_out.data_ptr(), x_out.stride(0), None if y is None else y_out.data_ptr(), 0 if y is None else y_out.stride(0),
        ptrs[0][0], ptrs[0][2], ptrs[1][0], ptrs[2][0], out_code, int(bool(accumulate)), work.data_ptr(), need,
        _stream()))
    return NormGrads(x_out, y_out, *(out for _, out in outs))


def residual_norm_grad(h, y, grad, normed_grad=None, gate=None, after=None, before=None, scale: float = 1.0,
                       eps: float = 1e-6, weight_dtype=torch.float32, x_out=None, y_out=None, gate_out=None,
                       after_out=None, before_out=None, accumulate: bool = False) -> NormGrads:
    """The gradients of `residual_norm` for x, y, gate, after and before, from `grad`, that of h (which is what the
    call returned), and `normed_grad`, that of z; one of them may be None (zeros). Those of gate, after and before are
    of `weight_dtype`, or written to views into the learner's gradient row, with `accumulate` added to what they
    hold. Equal calls give equal bits."""
    if y is None:
        raise TypeError("y: a tensor expected, not NoneType")
    got = _norm_grad(h, y, grad, normed_grad, gate, after, before, scale, eps, weight_dtype, x_out, y_out, gate_out,
                     after_out, before_out, accumulate)
    return got if type(got) is NormGrads else NormGrads(*got)


def rms_norm_grad(x, weight, grad, eps: float = 1e-6, stream_grad=None, weight_dtype=torch.float32, x_out=None,
                  weight_out=None, accumulate: bool = False):
    """Gradients of `rms_norm` from `grad`, that of its result: (for x, for weight; None without one). `stream_grad`,
    what else is known of x's gradient (of a residual stream that goes on beside the norm), is added to x's."""
    got = _norm_grad(x, None, stream_grad, grad, None, None, weight, 1.0, eps, weight_dtype, x_out, None, None, None,
                     weight_out, accumulate)
    return got[0], got[4]


# ---------------------------------------------------- 8-bit integers

class Int8Matrix:
    """A matrix in 8-bit integers with a scale for each row. `values` (rows x columns padded to multiples of 128,
    torch.int8) and `scales` (torch.float32) hold it as the library does."""

    def __init__(self, rows: int, cols: int, device):
        self.shape = (rows, cols)
        self.values = torch.empty((rows, -(-cols // 128) * 128), dtype=torch.int8, device=device)
        self.scales = torch.empty(rows, dtype=torch.float32, device=device)

    @property
    def parts(self):
        """What the native calls take."""
        return (self.values, self.scales, *self.shape)

    def dequantize(self):
        """The values that it stands for, each rounded to fp32 once."""
        return self.values[:, :self.shape[1]].float() * self.scales[:, None]


def _int8_parts(name: str, q):
    if not isinstance(q, Int8Matrix):
        raise TypeError(f"{name}: an Int8Matrix expected, not {type(q).__name__}")
    return q.parts


def _int8(name: str, q: Int8Matrix):
    """The library's form of a caller's matrix, whose tensors may have been exchanged for others."""
    rows, cols = q.shape
    for part, t, dtype, shape in (("values", q.values, torch.int8, (rows, -(-cols // 128) * 128)),
                                  ("scales", q.scales, torch.float32, (rows,))):
        _on_device(f"{name}.{part}", t)
        if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name}.{part}: contiguous {dtype} of {shape} expected, not {t.dtype} of "
                             f"{tuple(t.shape)}, {t.stride()} elements apart")
    return ctypes.byref(pl_int8(q.values.data_ptr(), q.scales.data_ptr()))


def quantize_int8(x) -> Int8Matrix:
    """x as an `Int8Matrix`: a scale for each row (a layer's weights, outputs x inputs: for each output)."""
    src, code, ld = _matrix("x", x)
    rows, cols = x.shape
    out = Int8Matrix(rows, cols, x.device)
    _check(load_library().pl_quantize_int8(src, code, rows, cols, ld, _int8("out", out), _stream()))
    return out


def matmul_int8(a: Int8Matrix, b: Int8Matrix, bias=None, relu: bool = False, dtype=torch.bfloat16, out=None):
    """a b^T (+ bias, then max(., 0) with relu), of `dtype` or written to `out`. The products' sums are exact, so an
    element depends on its rows of a and b alone: a token's answer is the same in any batch."""
    a_parts, b_parts = _int8_parts("a", a), _int8_parts("b", b)
    native = _native or _native_calls()
    if native:
        done = native.product_int8(a_parts, b_parts, bias, relu, dtype, out)
        if _done(done):
            return done
    (m, k), (n, k2) = a.shape, b.shape
    if k != k2:
        raise ValueError(f"rows of {k} and of {k2} columns")
    if out is None:
        out = torch.empty((m, n), dtype=dtype, device=a.values.device)
    dst, code, ld = _matrix("out", out, m, n)
    a_ref, b_ref = _int8("a", a), _int8("b", b)
    bias_ptr, bias_code = _bias(bias, n)
    L = load_library()
    need = L.pl_matmul_int8_workspace(m, n, k)
    work = torch.empty(need, dtype=torch.uint8, device=out.device) if need else None
    _check(L.pl_matmul_int8(m, n, k, a_ref, b_ref, bias_ptr, bias_code, int(bool(relu)), dst, code, ld,
                            work.data_ptr() if need else None, need, _stream()))
    return out


def linear_int8(x, w: Int8Matrix, bias=None, relu: bool = False, dtype=torch.bfloat16, out=None):
    """A fully connected layer that answers: x w^T (+ bias, relu), x as integers with a scale for each row (token),
    w the layer's weight (outputs x inputs), quantised once per pull."""
    w_parts = _int8_parts("w", w)
    native = _native or _native_calls()
    if native:
        done = native.linear_int8(x, w_parts, bias, relu, dtype, out)
        if _done(done):
            return done
    src, code, src_ld = _matrix("x", x, cols=w.shape[1])
    m, (n, k) = x.shape[0], w.shape
    w_ref = _int8("w", w)
    if out is None:
        out = torch.empty((m, n), dtype=dtype, device=x.device)
    dst, dst_code, dst_ld = _matrix("out", out, m, n)
    bias_ptr, bias_code = _bias(bias, n)
    L = load_library()
    need = L.pl_linear_int8_workspace(m, n, k)
    work = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    _check(L.pl_linear_int8(src, code, m, k, src_ld, n, w_ref, bias_ptr, bias_code, int(bool(relu)), dst, dst_code,
                            dst_ld, work.data_ptr() if need else None, need, _stream()))
    return out


# ------------------------------------------------------------ AdamW

class AdamW:
    """AdamW over many tensors, each step one launch:

        m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  t = steps made
        step = lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay * weight);  weight -= step

    `weights` and `grads`: tensors of equal sizes, contiguous (views into a replica and a gradient row are), all
    weights of a type and all gradients of a type. A step reads the gradients where they lie. `decay`: a number, or
    one for each tensor. With `push` a step is written in the gradients' place and the weights (fp32 or bf16) are only
    read: a learner pushes the row to a server with lr 1 and momentum 0, which then makes the step.

    The states are fp32 (`bits` 32) or a byte an element with a byte per 128 (`bits` 8), rounded at random, so that
    what is kept is right on average; `seed` names the random numbers, and equal calls give equal bits. `m`, `v`
    (`m_scales`, `v_scales`) hold tensor after tensor, each from a multiple of 128 elements on.

    Steps are made one after another, on torch's current stream. A step can be captured in a graph; replayed it goes
    on counting. The memory that the tensors have when the optimizer is made is what it reads and writes. Autograd
    does not see that weights change."""

    def __init__(self, weights: Sequence[torch.Tensor], grads: Sequence[torch.Tensor],
                 decay: Union[float, Sequence[float]] = 0.01, betas: Tuple[float, float] = (0.9, 0.999),
                 eps: float = 1e-8, bits: int = 32, push: bool = False, seed: int = 0):
        self.weights, self.grads = tuple(weights), tuple(grads)
        count = len(self.weights)
        if count == 0 or len(self.grads) != count:
            raise ValueError(f"{count} weights and {len(self.grads)} gradients")
        if bits not in (8, 32):
            raise ValueError(f"states of {bits} bits")
        if not 0 <= seed < 1 << 64:
            raise ValueError("seed: 64 bits")
        decays = [float(decay)] * count if isinstance(decay, (int, float)) else [float(d) for d in decay]
        if len(decays) != count:
            raise ValueError(f"{len(decays)} decays for {count} weights")
        here = torch.cuda.current_device() if torch.cuda.is_available() else None
        for name, ts in (("weights", self.weights), ("grads", self.grads)):
            for i, t in enumerate(ts):
                if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device.index != here:
                    _on_device(f"{name}[{i}]", t)   # raises
                if t.dtype != ts[0].dtype:
                    raise TypeError(f"{name}: {ts[0].dtype} and {t.dtype}")
                if not t.is_contiguous() or t.numel() != self.weights[i].numel():
                    raise ValueError(f"{name}[{i}]: {self.weights[i].numel()} contiguous elements expected, not "
                                     f"{tuple(t.shape)}, {t.stride()} elements apart")
        # the plan names their memory, which so lives as long as the optimizer, whatever becomes of the tensors
        self._memory = [t.untyped_storage() for t in (*self.weights, *self.grads)]
        self.bits, self.push, self.seed = bits, bool(push), seed
        self.betas, self.eps = (float(betas[0]), float(betas[1])), float(eps)
        self._codes = _code(self.weights[0].dtype), _code(self.grads[0].dtype)
        self._tensors = (pl_adamw_tensor * count)(*(
            pl_adamw_tensor(w.data_ptr(), g.data_ptr(), w.numel(), d)
            for w, g, d in zip(self.weights, self.grads, decays)))
        L = load_library()
        self._parts = L.pl_adamw_parts(self._tensors, count)
        self._room = L.pl_adamw_room(self._tensors, count)
        if self._parts < 0:
            _check(PS_EINVAL)
        self.device = self.weights[0].device
        plan = self._plan(0)
        kind = torch.float32 if bits == 32 else torch.uint8
        self.m, self.v = (torch.zeros(self._room, dtype=kind, device=self.device) for _ in range(2))
        self.m_scales = self.v_scales = None
        if bits == 8:
            self.m_scales, self.v_scales = (torch.zeros(self._room // 128, dtype=torch.uint8, device=self.device)
                                            for _ in range(2))
        self.plan = plan.to(self.device)
        # what does not change, as the native call takes it
        self._fixed = (self._parts, self._room, *self._codes, int(self.push), bits, seed)

    def _plan(self, steps: int):
        L = load_library()
        plan = torch.empty(L.pl_adamw_plan_bytes(self._parts), dtype=torch.uint8)
        _check(L.pl_adamw_plan(self._tensors, len(self._tensors), *self._codes, int(self.push), steps,
                               plan.data_ptr(), plan.numel()))
        return plan

    def _here(self) -> None:
        if self.device.index != torch.cuda.current_device():
            raise ValueError(f"the optimizer is on {self.device}, the current device is "
                             f"cuda:{torch.cuda.current_device()}")

    def _states(self):
        """Their addresses, as the library takes them; a caller may have exchanged the tensors for others."""
        kind, out = torch.float32 if self.bits == 32 else torch.uint8, []
        for name, n in (("m", self._room), ("v", self._room), ("m_scales", self._room // 128),
                        ("v_scales", self._room // 128))[:2 if self.bits == 32 else 4]:
            t = getattr(self, name)
            _on_device(name, t)
            if t.dtype != kind or t.numel() != n or not t.is_contiguous():
                raise ValueError(f"{name}: {n} contiguous elements of {kind} expected, not {t.dtype} of "
                                 f"{tuple(t.shape)}")
            out.append(t.data_ptr())
        return out if self.bits == 8 else out + [None, None]

    def step(self, lr, factor=1.0) -> None:
        """One step. `lr`, and `factor`, by which gradients are multiplied first (of a clipped norm, or of a scaled
        loss): numbers, or fp32 tensors of one element on the device, read when the step is made."""
        native = _native or _native_calls()
        if native:
            done = native.adamw_step(self.m, self.v, self.m_scales, self.v_scales, self.plan, self._fixed, *self.betas,
                                     self.eps, lr, factor)
            if _done(done):
                return
        self._here()
        numbers = []
        for name, x in (("lr", lr), ("factor", factor)):
            if isinstance(x, torch.Tensor):
                _on_device(name, x)
                if x.dtype != torch.float32 or x.numel() != 1:
                    raise TypeError(f"{name}: a number or one float32 expected, not {x.dtype} of {tuple(x.shape)}")
                numbers += [0.0, x.data_ptr()]
            else:
                numbers += [x, None]
        _on_device("plan", self.plan)
        if self.plan.numel() != load_library().pl_adamw_plan_bytes(self._parts) or self.plan.dtype != torch.uint8 or \
                not self.plan.is_contiguous():
            raise ValueError(f"plan: not this optimizer's, but {self.plan.dtype} of {tuple(self.plan.shape)}")
        _check(load_library().pl_adamw_step(
            self.plan.data_ptr(), self._parts, *self._codes, int(self.push), self.bits, self._room, *self._states(),
            *self.betas, self.eps, *numbers, self.seed, _stream()))

    @property
    def steps(self) -> int:
        """The steps made (waits for them)."""
        if self._parts == 0:
            return 0
        plan = self.plan[:load_library().pl_adamw_plan_bytes(1)].cpu()
        return load_library().pl_adamw_steps(plan.data_ptr())

    def moments(self, dtype=torch.float32):
        """(m, v) as numbers of `dtype`, laid out as the states: in 32 bits the states themselves where that is
        their type."""
        self._here()
        if self.bits == 32:
            return self.m.to(dtype), self.v.to(dtype)
        native = _native or _native_calls()
        if native:
            done = native.adamw_moments(self.m, self.v, self.m_scales, self.v_scales, self._room, dtype)
            if _done(done):
                return done
        m, v = (torch.empty(self._room, dtype=dtype, device=self.device) for _ in range(2))
        _check(load_library().pl_adamw_moments(self._room, *self._states(), m.data_ptr(), v.data_ptr(), _code(dtype),
                                               _stream()))
        return m, v

    def views(self, states):
        """A vector laid out as the states are, as a view for each weight, of its shape."""
        out, at = [], 0
        for w in self.weights:
            out.append(states[at:at + w.numel()].view(w.shape))
            at += -(-w.numel() // 128) * 128
        return out

    def state(self) -> dict:
        """What `load` takes: the steps made and the states (the tensors themselves)."""
        names = ("m", "v") if self.bits == 32 else ("m", "v", "m_scales", "v_scales")
        return {"steps": self.steps, **{k: getattr(self, k) for k in names}}

    def load(self, state: dict) -> None:
        """Goes on from `state()` of an optimizer of the same sizes and bits; its tensors are copied."""
        own = self.state()
        if set(state) != set(own):
            raise ValueError(f"{sorted(own)} expected, not {sorted(state)}")
        for k, t in own.items():
            if k != "steps" and (state[k].shape != t.shape or state[k].dtype != t.dtype):
                raise ValueError(f"{k}: {t.dtype} of {tuple(t.shape)} expected, not {state[k].dtype} of "
                                 f"{tuple(state[k].shape)}")
        plan = self._plan(state["steps"])
        for k, t in own.items():
            if k != "steps":
                t.copy_(state[k])
        self.plan.copy_(plan)
