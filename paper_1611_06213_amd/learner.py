"""A learner's operators (the C ABI in include/ps_learner.h) for torch device tensors.

What a learner computes between a pull and a push with the layers that hold most
of the server's parameters: embedding tables and fully connected layers, the latter
in 8-bit floating point with a scale per block of 128, and dropout. Weights are
read where they lie in a replica (any view with unit column stride), weight
gradients are written where they belong in a gradient row.

No call records anything for autograd: a result does not require a gradient, whatever its
arguments do. The backward pass is a call of its own (`embedding_grad`, `linear_fp8_grad`,
`dropout` again).

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
from typing import NamedTuple, Optional, Tuple

import torch

from .ps import PS_BF16, PS_F32, PS_OK, PSError

PL_I32 = 0
PL_I64 = 1

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgadeilearner.so")


class pl_drop(ctypes.Structure):
    _fields_ = [("p", ctypes.c_float), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64)]


class pl_fp8(ctypes.Structure):
    _fields_ = [("values", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


_VP, _INT, _I64, _SIZE = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
_DROP, _FP8 = ctypes.POINTER(pl_drop), ctypes.POINTER(pl_fp8)
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
