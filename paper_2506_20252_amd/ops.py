"""Binding of include/pat_ops.h: operators on gathered and scattered tensors.

4-bit block quantisation and products, embedding lookup and its gradient, and
dropout from a counter-based generator.  The ``pat_*`` functions are the C
calls with the same arguments (buffers as addresses or objects with
``data_ptr()``); the others read sizes, strides and types from torch tensors,
allocate outputs and workspaces, and raise.  Marshalling only: all work is done
by the HIP kernels of ``libpat.so``, and there is no fallback.

Tensors are 2-D with unit stride along rows; rows may be strided.  Calls run on
`stream`, by default torch's current stream of the tensors' device; what they
allocate belongs to that stream.

Nothing here is recorded for autograd: a result carries no graph, also where an
input requires grad.  A training step calls the gradients by name, or from an
autograd function of its own.
"""

import ctypes
from typing import NamedTuple

import torch

from . import pat

PAT_MX_GROUP = 128

# Every function include/pat_ops.h declares.
EXPORTS = (
    "pat_mx_quantize", "pat_mx_dequantize", "pat_mx_matmul", "pat_mx_linear", "pat_mx_linear_workspace",
    "pat_mx_matmul_grad", "pat_mx_matmul_grad_workspace", "pat_embedding", "pat_embedding_grad",
    "pat_embedding_grad_workspace", "pat_dropout",
)

_P, _N, _S, _I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64, ctypes.c_int
_SIGNATURES = {
    "pat_mx_quantize": ([_P, _S, _N, _N, _I, _P, _P, _P], _I),
    "pat_mx_dequantize": ([_P, _P, _N, _N, _P, _S, _I, _P], _I),
    "pat_mx_matmul": ([_P, _P, _P, _P, _N, _N, _N, _P, _S, _I, _P], _I),
    "pat_mx_linear": ([_P, _S, _I, _P, _P, _N, _N, _N, _P, _S, _I, _P, _N, _P], _I),
    "pat_mx_linear_workspace": ([_N, _N, _N], _N),
    "pat_mx_matmul_grad": ([_P, _S, _I, _P, _P, _N, _N, _N, _P, _S, _I, _P, _N, _P], _I),
    "pat_mx_matmul_grad_workspace": ([_N, _N, _N], _N),
    "pat_embedding": ([_P, _I, _N, _P, _S, _I, _S, _N, _N, ctypes.c_float, _P, _S, _I, _P], _I),
    "pat_embedding_grad": ([_P, _I, _N, _P, _S, _I, _S, _N, _N, ctypes.c_float, _P, _S, _I, _P, _N, _P], _I),
    "pat_embedding_grad_workspace": ([_N, _N, _N], _N),
    "pat_dropout": ([_P, _S, _P, _S, _P, _S, _N, _N, _I, ctypes.c_double, ctypes.c_uint64, ctypes.c_uint64,
                     ctypes.c_uint64, _P], _I),
}

class _Calls:
    """The library's functions, each looked up and given its signature at its first use."""

    def __getattr__(self, name):
        if name not in _SIGNATURES:
            raise AttributeError(name)
        fn = getattr(pat.lib(), name)
        fn.argtypes, fn.restype = _SIGNATURES[name]
        setattr(self, name, fn)
        return fn


_c = _Calls()


def _address(b):
    if b is None:
        return None
    return b.data_ptr() if hasattr(b, "data_ptr") else int(b)


# ---------------------------------------------------------------------------
# The C calls
# ---------------------------------------------------------------------------


def pat_mx_quantize(x, x_stride, rows, cols, dtype, codes, scales, stream=None):
    return _c.pat_mx_quantize(_address(x), x_stride, rows, cols, pat._dtype(dtype), _address(codes),
                              _address(scales), pat._stream(stream))


def pat_mx_dequantize(codes, scales, rows, cols, out, out_stride, dtype, stream=None):
    return _c.pat_mx_dequantize(_address(codes), _address(scales), rows, cols, _address(out), out_stride,
                                pat._dtype(dtype), pat._stream(stream))


def pat_mx_matmul(a_codes, a_scales, b_codes, b_scales, m, n, k, out, out_stride, dtype, stream=None):
    return _c.pat_mx_matmul(_address(a_codes), _address(a_scales), _address(b_codes), _address(b_scales), m, n, k,
                            _address(out), out_stride, pat._dtype(dtype), pat._stream(stream))


def pat_mx_linear(x, x_stride, x_dtype, w_codes, w_scales, m, n, k, out, out_stride, dtype, workspace, workspace_bytes,
                  stream=None):
    return _c.pat_mx_linear(_address(x), x_stride, pat._dtype(x_dtype), _address(w_codes), _address(w_scales), m, n, k,
                            _address(out), out_stride, pat._dtype(dtype), _address(workspace), workspace_bytes,
                            pat._stream(stream))


def pat_mx_linear_workspace(m, n, k):
    return _c.pat_mx_linear_workspace(m, n, k)


def pat_mx_matmul_grad(g, g_stride, transposed, q_codes, q_scales, rows, inner, cols, out, out_stride, dtype, workspace,
                       workspace_bytes, stream=None):
    return _c.pat_mx_matmul_grad(_address(g), g_stride, int(transposed), _address(q_codes), _address(q_scales), rows,
                                 inner, cols, _address(out), out_stride, pat._dtype(dtype), _address(workspace),
                                 workspace_bytes, pat._stream(stream))


def pat_mx_matmul_grad_workspace(rows, inner, cols):
    return _c.pat_mx_matmul_grad_workspace(rows, inner, cols)


def pat_embedding(tokens, token_bytes, ntokens, table, table_stride, table_dtype, first, rows, cols, scale, out,
                  out_stride, dtype, stream=None):
    return _c.pat_embedding(_address(tokens), token_bytes, ntokens, _address(table), table_stride,
                            pat._dtype(table_dtype), first, rows, cols, scale, _address(out), out_stride,
                            pat._dtype(dtype), pat._stream(stream))


def pat_embedding_grad(tokens, token_bytes, ntokens, g, g_stride, g_dtype, first, rows, cols, scale, out, out_stride,
                       dtype, workspace, workspace_bytes, stream=None):
    return _c.pat_embedding_grad(_address(tokens), token_bytes, ntokens, _address(g), g_stride, pat._dtype(g_dtype),
                                 first, rows, cols, scale, _address(out), out_stride, pat._dtype(dtype),
                                 _address(workspace), workspace_bytes, pat._stream(stream))


def pat_embedding_grad_workspace(ntokens, rows, cols):
    return _c.pat_embedding_grad_workspace(ntokens, rows, cols)


def pat_dropout(x, x_stride, residual, residual_stride, out, out_stride, rows, cols, dtype, p, seed, index, index_stride,
                stream=None):
    return _c.pat_dropout(_address(x), x_stride, _address(residual), residual_stride, _address(out), out_stride, rows,
                          cols, pat._dtype(dtype), p, seed, index, index_stride, pat._stream(stream))


# ---------------------------------------------------------------------------
# Tensor-level calls
# ---------------------------------------------------------------------------

_CODE = {torch.float32: pat.PAT_FLOAT32, torch.bfloat16: pat.PAT_BFLOAT16}


class Mx(NamedTuple):
    """A matrix in 4-bit blocks: codes [rows, 64 * G] and scales [rows, 4 * G], uint8 and contiguous, with
    G = ceil(cols / 128).  The rows of several ranks' shards, gathered, are the whole matrix's."""

    codes: torch.Tensor
    scales: torch.Tensor
    cols: int


def mx_empty(rows, cols, device="cuda"):
    """An Mx to quantise or gather into (uninitialised)."""
    groups = -(-cols // PAT_MX_GROUP)
    return Mx(torch.empty((rows, 64 * groups), dtype=torch.uint8, device=device),
              torch.empty((rows, 4 * groups), dtype=torch.uint8, device=device), cols)


def _float(dtype, what):
    code = _CODE.get(dtype)
    if code is None:
        raise ValueError(f"{what}: float32 or bfloat16, got {dtype}")
    return code


def _matrix(t, what):
    """Checks a float matrix; returns its rows, columns, row stride and type."""
    size = t.shape
    if len(size) != 2 or not t.is_cuda:
        raise ValueError(f"{what}: a 2-D GPU tensor")
    code = _CODE.get(t.dtype)
    if code is None:
        _float(t.dtype, what)
    rows, cols = size
    stride, unit = t.stride()
    if stride == cols and unit == 1:
        return rows, cols, stride, code
    if rows and cols > 1 and unit != 1:
        raise ValueError(f"{what}: the elements of a row must be consecutive in memory")
    if rows > 1 and cols and stride < cols:
        raise ValueError(f"{what}: rows overlap")
    return rows, cols, max(stride, cols), code


def _stored(q, what):
    """Checks an Mx; returns its codes, scales, rows and columns."""
    codes, scales, cols = q
    groups = -(-cols // PAT_MX_GROUP)
    rows = codes.shape[0] if codes.dim() == 2 else -1
    if (codes.shape == (rows, 64 * groups) and scales.shape == (rows, 4 * groups) and codes.dtype is scales.dtype is torch.uint8
            and codes.is_cuda and scales.is_cuda and codes.is_contiguous() and scales.is_contiguous()):
        return codes, scales, rows, cols
    raise ValueError(f"{what}: codes (rows, {64 * groups}) and scales (rows, {4 * groups}) must be contiguous uint8 GPU tensors, "
                     f"got {codes.dtype} {tuple(codes.shape)} and {scales.dtype} {tuple(scales.shape)}")


def _indices(t, what):
    if t.dim() != 1 or not t.is_cuda or t.dtype not in (torch.int32, torch.int64) or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous 1-D int32 or int64 GPU tensor")
    return t.element_size()


def _on(stream, *tensors):
    """The stream of a call, as an integer; all tensors must be on the current device."""
    device = _current_device()
    for t in tensors:
        if t.get_device() != device:
            raise ValueError(f"all tensors must be on the current device, cuda:{device}, got {t.device}")
    if stream is None:
        return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(device)
    return pat._stream(stream)


# The current stream's handle without a Stream object and the current device, where this torch has them: two microseconds
# less per call, which takes six to eight and the GPU three.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _empty(shape, dtype, like, stream):
    """New memory for a call on `stream`: that stream's own (torch hands memory out again in the order of the stream
    that it was allocated on), so that neither earlier nor later work on the current stream meets it."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(pat._stream(stream), device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _output(out, rows, cols, dtype, what):
    """Checks a given output; returns its row stride."""
    if out.dtype != dtype:
        raise ValueError(f"{what}: out is {out.dtype}, not {dtype}")
    r, c, stride, _ = _matrix(out, "out")
    if r != rows or c != cols:
        raise ValueError(f"out: shape {(rows, cols)} is needed, got {(r, c)}")
    return stride


def _work(nbytes, like, stream):
    """Address of a workspace and the tensor that holds it."""
    if not nbytes:
        return None, None
    w = _empty(nbytes, torch.uint8, like, stream)
    return w.data_ptr(), w


def mx_quantize(x, out=None, stream=None):
    """4-bit blocks of a float32 or bfloat16 matrix, as an Mx."""
    rows, cols, stride, code = _matrix(x, "x")
    if out is None:
        groups = -(-cols // PAT_MX_GROUP)
        codes, scales = _empty((rows, 64 * groups), torch.uint8, x, stream), _empty((rows, 4 * groups), torch.uint8, x, stream)
        on, out = _on(stream, x), Mx(codes, scales, cols)
    else:
        codes, scales, out_rows, out_cols = _stored(out, "out")
        if out_rows != rows or out_cols != cols:
            raise ValueError(f"out: an Mx of {rows} x {cols} is needed")
        on = _on(stream, x, codes, scales)
    status = _c.pat_mx_quantize(x.data_ptr(), stride, rows, cols, code, codes.data_ptr(), scales.data_ptr(), on)
    if status:
        pat.check(status, "pat_mx_quantize")
    return out


def mx_dequantize(q, dtype=torch.bfloat16, out=None, stream=None):
    """The matrix that an Mx stands for, in `dtype` (exact)."""
    codes, scales, rows, cols = _stored(q, "q")
    code = _float(dtype, "dtype")
    if out is None:
        out, stride, on = _empty((rows, cols), dtype, codes, stream), cols, _on(stream, codes, scales)
    else:
        stride, on = _output(out, rows, cols, dtype, "mx_dequantize"), _on(stream, codes, scales, out)
    status = _c.pat_mx_dequantize(codes.data_ptr(), scales.data_ptr(), rows, cols, out.data_ptr(), stride, code, on)
    if status:
        pat.check(status, "pat_mx_dequantize")
    return out


def mx_matmul(a, b, dtype=torch.bfloat16, out=None, stream=None):
    """a b^T of two Mx with the same number of columns."""
    a_codes, a_scales, m, k = _stored(a, "a")
    b_codes, b_scales, n, b_cols = _stored(b, "b")
    if b_cols != k:
        raise ValueError(f"a has {k} columns, b has {b_cols}")
    code = _float(dtype, "dtype")
    if out is None:
        out, stride, on = _empty((m, n), dtype, a_codes, stream), n, _on(stream, a_codes, a_scales, b_codes, b_scales)
    else:
        stride, on = _output(out, m, n, dtype, "mx_matmul"), _on(stream, a_codes, a_scales, b_codes, b_scales, out)
    status = _c.pat_mx_matmul(a_codes.data_ptr(), a_scales.data_ptr(), b_codes.data_ptr(), b_scales.data_ptr(), m, n, k,
                              out.data_ptr(), stride, code, on)
    if status:
        pat.check(status, "pat_mx_matmul")
    return out


def mx_linear(x, w, dtype=None, out=None, stream=None):
    """Q(x) w^T: the rows of x, quantised on the way, times an Mx; `dtype` is x's by default."""
    m, k, x_stride, x_code = _matrix(x, "x")
    codes, scales, n, cols = _stored(w, "w")
    if cols != k:
        raise ValueError(f"x has {k} columns, w has {cols}")
    if dtype is None:
        dtype, code = x.dtype, x_code
    else:
        code = _float(dtype, "dtype")
    if out is None:
        out, stride, on = _empty((m, n), dtype, x, stream), n, _on(stream, x, codes, scales)
    else:
        stride, on = _output(out, m, n, dtype, "mx_linear"), _on(stream, x, codes, scales, out)
    need = _c.pat_mx_linear_workspace(m, n, k)
    work, hold = _work(need, x, stream)
    status = _c.pat_mx_linear(x.data_ptr(), x_stride, x_code, codes.data_ptr(), scales.data_ptr(), m, n, k, out.data_ptr(),
                              stride, code, work, need, on)
    if status:
        pat.check(status, "pat_mx_linear")
    return out


def mx_matmul_grad(g, q, dtype=torch.bfloat16, transposed=False, out=None, stream=None):
    """g q, or g^T q where `transposed`: with g the bfloat16 gradient of a b^T, the gradient of a is
    ``mx_matmul_grad(g, b)`` and that of b is ``mx_matmul_grad(g, a, transposed=True)``."""
    rows, terms, g_stride, _ = _matrix(g, "g")
    codes, scales, inner, cols = _stored(q, "q")
    if g.dtype != torch.bfloat16:
        raise ValueError(f"g: bfloat16, got {g.dtype}")
    if transposed:
        rows, terms = terms, rows
    if terms != inner:
        raise ValueError(f"g: {tuple(g.shape)} does not match q's {inner} rows")
    code = _float(dtype, "dtype")
    if out is None:
        out, stride, on = _empty((rows, cols), dtype, g, stream), cols, _on(stream, g, codes, scales)
    else:
        stride, on = _output(out, rows, cols, dtype, "mx_matmul_grad"), _on(stream, g, codes, scales, out)
    need = _c.pat_mx_matmul_grad_workspace(rows, inner, cols)
    work, hold = _work(need, g, stream)
    status = _c.pat_mx_matmul_grad(g.data_ptr(), g_stride, bool(transposed), codes.data_ptr(), scales.data_ptr(), rows, inner,
                                   cols, out.data_ptr(), stride, code, work, need, on)
    if status:
        pat.check(status, "pat_mx_matmul_grad")
    return out


def embedding(tokens, table, scale=1.0, first=0, dtype=None, out=None, stream=None):
    """out[t] = scale * table[tokens[t] - first], zero for a token that the table's rows do not hold; `dtype` is
    the table's by default."""
    size = _indices(tokens, "tokens")
    rows, cols, table_stride, table_code = _matrix(table, "table")
    n = tokens.shape[0]
    if dtype is None:
        dtype, code = table.dtype, table_code
    else:
        code = _float(dtype, "dtype")
    if out is None:
        out, stride, on = _empty((n, cols), dtype, table, stream), cols, _on(stream, tokens, table)
    else:
        stride, on = _output(out, n, cols, dtype, "embedding"), _on(stream, tokens, table, out)
    status = _c.pat_embedding(tokens.data_ptr(), size, n, table.data_ptr(), table_stride, table_code, first, rows, cols, scale,
                              out.data_ptr(), stride, code, on)
    if status:
        pat.check(status, "pat_embedding")
    return out


def embedding_grad(tokens, g, rows, scale=1.0, first=0, dtype=None, out=None, stream=None):
    """The gradient of ``embedding`` with respect to a table of `rows` rows, dense; `dtype` is g's by default."""
    size = _indices(tokens, "tokens")
    n, cols, g_stride, g_code = _matrix(g, "g")
    if tokens.shape[0] != n:
        raise ValueError(f"g has {n} rows for {tokens.shape[0]} tokens")
    if dtype is None:
        dtype, code = g.dtype, g_code
    else:
        code = _float(dtype, "dtype")
    if out is None:
        out, stride, on = _empty((rows, cols), dtype, g, stream), cols, _on(stream, tokens, g)
    else:
        stride, on = _output(out, rows, cols, dtype, "embedding_grad"), _on(stream, tokens, g, out)
    need = _c.pat_embedding_grad_workspace(n, rows, cols)
    work, hold = _work(need, g, stream)
    status = _c.pat_embedding_grad(tokens.data_ptr(), size, n, g.data_ptr(), g_stride, g_code, first, rows, cols, scale,
                                   out.data_ptr(), stride, code, work, need, on)
    if status:
        pat.check(status, "pat_embedding_grad")
    return out


def dropout(x, p, seed, index=0, index_stride=None, residual=None, out=None, stream=None):
    """x with each element dropped with probability p or scaled, plus `residual`.  The mask is a function of `seed`
    and the element's place: element (r, c) has number index + r * index_stride + c in the whole tensor
    (`index_stride`: x's columns by default, the whole's for a shard of its columns).  The gradient is the same
    call on the output's gradient.  `out` may be x or the residual."""
    rows, cols, x_stride, code = _matrix(x, "x")
    if out is None:
        out, stride, on = _empty((rows, cols), x.dtype, x, stream), cols, _on(stream, x)
    else:
        stride, on = _output(out, rows, cols, x.dtype, "dropout"), _on(stream, x, out)
    address, residual_stride = None, 0
    if residual is not None:
        r, c, residual_stride, residual_code = _matrix(residual, "residual")
        if r != rows or c != cols:
            raise ValueError(f"residual: shape {(rows, cols)} is needed, got {(r, c)}")
        if residual_code != code:
            raise ValueError(f"residual is {residual.dtype}, x is {x.dtype}")
        _on(stream, residual)
        address = residual.data_ptr()
    status = _c.pat_dropout(x.data_ptr(), x_stride, address, residual_stride, out.data_ptr(), stride, rows, cols, code, p, seed,
                            index, cols if index_stride is None else index_stride, on)
    if status:
        pat.check(status, "pat_dropout")
    return out
