"""Binding of include/pat_ops.h: operators on gathered and scattered tensors.

4-bit block quantisation and products, embedding lookup and its gradient, and
dropout from a counter-based generator.  The ``pat_*`` functions are the C
calls with the same arguments (buffers as addresses or objects with
``data_ptr()``); the others read sizes, strides and types from torch tensors,
allocate outputs and workspaces, and raise.  Marshalling only: all work is done
by the HIP kernels of ``libpat.so``, and there is no fallback.

Tensors are 2-D with unit stride along rows; rows may be strided.  Calls run on
`stream`, by default torch's current stream of the tensors' device.
"""

import ctypes
from typing import NamedTuple

import torch

from . import pat

PAT_MX_GROUP = 128

# Every function include/pat_ops.h declares.
EXPORTS = (
    "pat_mx_quantize", "pat_mx_dequantize", "pat_mx_matmul", "pat_mx_matmul_workspace", "pat_mx_linear",
    "pat_mx_linear_workspace", "pat_mx_matmul_grad", "pat_mx_matmul_grad_workspace", "pat_embedding",
    "pat_embedding_grad", "pat_embedding_grad_workspace", "pat_dropout",
)

_P, _N, _S, _I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64, ctypes.c_int
_SIGNATURES = {
    "pat_mx_quantize": ([_P, _S, _N, _N, _I, _P, _P, _P], _I),
    "pat_mx_dequantize": ([_P, _P, _N, _N, _P, _S, _I, _P], _I),
    "pat_mx_matmul": ([_P, _P, _P, _P, _N, _N, _N, _P, _S, _I, _P, _N, _P], _I),
    "pat_mx_matmul_workspace": ([_N, _N, _N], _N),
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

_fns = {}


def _fn(name):
    fn = _fns.get(name)
    if fn is None:
        fn = getattr(pat.lib(), name)
        fn.argtypes, fn.restype = _SIGNATURES[name]
        _fns[name] = fn
    return fn


def _address(b):
    if b is None:
        return None
    return b.data_ptr() if hasattr(b, "data_ptr") else int(b)


# ---------------------------------------------------------------------------
# The C calls
# ---------------------------------------------------------------------------


def pat_mx_quantize(x, x_stride, rows, cols, dtype, codes, scales, stream=None):
    return _fn("pat_mx_quantize")(_address(x), x_stride, rows, cols, pat._dtype(dtype), _address(codes),
                                  _address(scales), pat._stream(stream))


def pat_mx_dequantize(codes, scales, rows, cols, out, out_stride, dtype, stream=None):
    return _fn("pat_mx_dequantize")(_address(codes), _address(scales), rows, cols, _address(out), out_stride,
                                    pat._dtype(dtype), pat._stream(stream))


def pat_mx_matmul(a_codes, a_scales, b_codes, b_scales, m, n, k, out, out_stride, dtype, workspace, workspace_bytes,
                  stream=None):
    return _fn("pat_mx_matmul")(_address(a_codes), _address(a_scales), _address(b_codes), _address(b_scales), m, n, k,
                                _address(out), out_stride, pat._dtype(dtype), _address(workspace), workspace_bytes,
                                pat._stream(stream))


def pat_mx_matmul_workspace(m, n, k):
    return _fn("pat_mx_matmul_workspace")(m, n, k)


def pat_mx_linear(x, x_stride, x_dtype, w_codes, w_scales, m, n, k, out, out_stride, dtype, workspace, workspace_bytes,
                  stream=None):
    return _fn("pat_mx_linear")(_address(x), x_stride, pat._dtype(x_dtype), _address(w_codes), _address(w_scales), m, n, k,
                                _address(out), out_stride, pat._dtype(dtype), _address(workspace), workspace_bytes,
                                pat._stream(stream))


def pat_mx_linear_workspace(m, n, k):
    return _fn("pat_mx_linear_workspace")(m, n, k)


def pat_mx_matmul_grad(g, g_stride, transposed, q_codes, q_scales, rows, inner, cols, out, out_stride, dtype, workspace,
                       workspace_bytes, stream=None):
    return _fn("pat_mx_matmul_grad")(_address(g), g_stride, int(transposed), _address(q_codes), _address(q_scales), rows,
                                     inner, cols, _address(out), out_stride, pat._dtype(dtype), _address(workspace),
                                     workspace_bytes, pat._stream(stream))


def pat_mx_matmul_grad_workspace(rows, inner, cols):
    return _fn("pat_mx_matmul_grad_workspace")(rows, inner, cols)


def pat_embedding(tokens, token_bytes, ntokens, table, table_stride, table_dtype, first, rows, cols, scale, out,
                  out_stride, dtype, stream=None):
    return _fn("pat_embedding")(_address(tokens), token_bytes, ntokens, _address(table), table_stride,
                                pat._dtype(table_dtype), first, rows, cols, scale, _address(out), out_stride,
                                pat._dtype(dtype), pat._stream(stream))


def pat_embedding_grad(tokens, token_bytes, ntokens, g, g_stride, g_dtype, first, rows, cols, scale, out, out_stride,
                       dtype, workspace, workspace_bytes, stream=None):
    return _fn("pat_embedding_grad")(_address(tokens), token_bytes, ntokens, _address(g), g_stride, pat._dtype(g_dtype),
                                     first, rows, cols, scale, _address(out), out_stride, pat._dtype(dtype),
                                     _address(workspace), workspace_bytes, pat._stream(stream))


def pat_embedding_grad_workspace(ntokens, rows, cols):
    return _fn("pat_embedding_grad_workspace")(ntokens, rows, cols)


def pat_dropout(x, x_stride, residual, residual_stride, out, out_stride, rows, cols, dtype, p, seed, index, index_stride,
                stream=None):
    return _fn("pat_dropout")(_address(x), x_stride, _address(residual), residual_stride, _address(out), out_stride, rows,
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
    if dtype not in _CODE:
        raise ValueError(f"{what}: float32 or bfloat16, got {dtype}")
    return _CODE[dtype]


def _matrix(t, what, shape=None):
    """Checks a float matrix and returns its row stride."""
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{what}: a 2-D GPU tensor")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(shape)} is needed, got {tuple(t.shape)}")
    _float(t.dtype, what)
    rows, cols = t.shape
    stride, unit = t.stride()
    if rows and cols > 1 and unit != 1:
        raise ValueError(f"{what}: the elements of a row must be consecutive in memory")
    if rows > 1 and cols and stride < cols:
        raise ValueError(f"{what}: rows overlap")
    return max(stride, cols)


def _stored(q, what):
    """Checks an Mx and returns its row count."""
    codes, scales, cols = q
    groups = -(-cols // PAT_MX_GROUP)
    rows = codes.shape[0] if codes.dim() == 2 else -1
    for t, width, name in ((codes, 64 * groups, "codes"), (scales, 4 * groups, "scales")):
        if not t.is_cuda or t.dtype != torch.uint8 or not t.is_contiguous() or tuple(t.shape) != (rows, width):
            raise ValueError(f"{what}: {name} must be a contiguous uint8 GPU tensor of shape (rows, {width})")
    return rows


def _indices(t, what):
    if t.dim() != 1 or not t.is_cuda or t.dtype not in (torch.int32, torch.int64) or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous 1-D int32 or int64 GPU tensor")
    return t.element_size()


def _on(stream, *tensors):
    """The stream of a call whose tensors must all be on the current device."""
    device = tensors[0].device
    for t in tensors[1:]:
        if t.device != device:
            raise ValueError(f"all tensors must be on one device, got {device} and {t.device}")
    return pat._tensor_call_stream(device, stream)


def _output(out, shape, dtype, device, what):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if out.dtype != dtype:
        raise ValueError(f"{what}: out is {out.dtype}, not {dtype}")
    return out


def _work(nbytes, device, stream):
    """A workspace, or None.  On another stream than torch's current one, the caching allocator is told, so that
    the memory is not handed out again before the call has run."""
    if not nbytes:
        return None
    w = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if isinstance(stream, torch.cuda.Stream) and stream != torch.cuda.current_stream(device):
        w.record_stream(stream)
    return w


def mx_quantize(x, out=None, stream=None):
    """4-bit blocks of a float32 or bfloat16 matrix, as an Mx."""
    stride = _matrix(x, "x")
    rows, cols = x.shape
    q = mx_empty(rows, cols, x.device) if out is None else out
    if _stored(q, "out") != rows or q.cols != cols:
        raise ValueError(f"out: an Mx of {rows} x {cols} is needed")
    stream = _on(stream, x, q.codes, q.scales)
    pat.check(pat_mx_quantize(x, stride, rows, cols, _CODE[x.dtype], q.codes, q.scales, stream), "pat_mx_quantize")
    return q


def mx_dequantize(q, dtype=torch.bfloat16, out=None, stream=None):
    """The matrix that an Mx stands for, in `dtype` (exact)."""
    rows = _stored(q, "q")
    _float(dtype, "dtype")
    out = _output(out, (rows, q.cols), dtype, q.codes.device, "mx_dequantize")
    stride = _matrix(out, "out", (rows, q.cols))
    stream = _on(stream, q.codes, q.scales, out)
    pat.check(pat_mx_dequantize(q.codes, q.scales, rows, q.cols, out, stride, _CODE[dtype], stream), "pat_mx_dequantize")
    return out


def mx_matmul(a, b, dtype=torch.bfloat16, out=None, stream=None):
    """a b^T of two Mx with the same number of columns."""
    m, n, k = _stored(a, "a"), _stored(b, "b"), a.cols
    if b.cols != k:
        raise ValueError(f"a has {k} columns, b has {b.cols}")
    _float(dtype, "dtype")
    out = _output(out, (m, n), dtype, a.codes.device, "mx_matmul")
    stride = _matrix(out, "out", (m, n))
    stream = _on(stream, a.codes, a.scales, b.codes, b.scales, out)
    need = pat_mx_matmul_workspace(m, n, k)
    pat.check(pat_mx_matmul(a.codes, a.scales, b.codes, b.scales, m, n, k, out, stride, _CODE[dtype],
                            _work(need, out.device, stream), need, stream), "pat_mx_matmul")
    return out


def mx_linear(x, w, dtype=None, out=None, stream=None):
    """Q(x) w^T: the rows of x, quantised on the way, times an Mx; `dtype` is x's by default."""
    stride, n = _matrix(x, "x"), _stored(w, "w")
    m, k = x.shape
    if w.cols != k:
        raise ValueError(f"x has {k} columns, w has {w.cols}")
    dtype = x.dtype if dtype is None else dtype
    _float(dtype, "dtype")
    out = _output(out, (m, n), dtype, x.device, "mx_linear")
    out_stride = _matrix(out, "out", (m, n))
    stream = _on(stream, x, w.codes, w.scales, out)
    need = pat_mx_linear_workspace(m, n, k)
    pat.check(pat_mx_linear(x, stride, _CODE[x.dtype], w.codes, w.scales, m, n, k, out, out_stride, _CODE[dtype],
                            _work(need, out.device, stream), need, stream), "pat_mx_linear")
    return out


def mx_matmul_grad(g, q, dtype=torch.bfloat16, transposed=False, out=None, stream=None):
    """g q, or g^T q where `transposed`: with g the bfloat16 gradient of a b^T, the gradient of a is
    ``mx_matmul_grad(g, b)`` and that of b is ``mx_matmul_grad(g, a, transposed=True)``."""
    stride, inner = _matrix(g, "g"), _stored(q, "q")
    if g.dtype != torch.bfloat16:
        raise ValueError(f"g: bfloat16, got {g.dtype}")
    rows = g.shape[1 if transposed else 0]
    if g.shape[0 if transposed else 1] != inner:
        raise ValueError(f"g: {tuple(g.shape)} does not match q's {inner} rows")
    _float(dtype, "dtype")
    out = _output(out, (rows, q.cols), dtype, g.device, "mx_matmul_grad")
    out_stride = _matrix(out, "out", (rows, q.cols))
    stream = _on(stream, g, q.codes, q.scales, out)
    need = pat_mx_matmul_grad_workspace(rows, inner, q.cols)
    pat.check(pat_mx_matmul_grad(g, stride, transposed, q.codes, q.scales, rows, inner, q.cols, out, out_stride,
                                 _CODE[dtype], _work(need, out.device, stream), need, stream), "pat_mx_matmul_grad")
    return out


def embedding(tokens, table, scale=1.0, first=0, dtype=None, out=None, stream=None):
    """out[t] = scale * table[tokens[t] - first], zero for a token that the table's rows do not hold; `dtype` is
    the table's by default."""
    size, stride = _indices(tokens, "tokens"), _matrix(table, "table")
    rows, cols = table.shape
    dtype = table.dtype if dtype is None else dtype
    _float(dtype, "dtype")
    n = tokens.numel()
    out = _output(out, (n, cols), dtype, table.device, "embedding")
    out_stride = _matrix(out, "out", (n, cols))
    stream = _on(stream, tokens, table, out)
    pat.check(pat_embedding(tokens, size, n, table, stride, _CODE[table.dtype], first, rows, cols, scale, out, out_stride,
                            _CODE[dtype], stream), "pat_embedding")
    return out


def embedding_grad(tokens, g, rows, scale=1.0, first=0, dtype=None, out=None, stream=None):
    """The gradient of ``embedding`` with respect to a table of `rows` rows, dense; `dtype` is g's by default."""
    size, stride = _indices(tokens, "tokens"), _matrix(g, "g")
    n, cols = g.shape
    if tokens.numel() != n:
        raise ValueError(f"g has {n} rows for {tokens.numel()} tokens")
    dtype = g.dtype if dtype is None else dtype
    _float(dtype, "dtype")
    out = _output(out, (rows, cols), dtype, g.device, "embedding_grad")
    out_stride = _matrix(out, "out", (rows, cols))
    stream = _on(stream, tokens, g, out)
    need = pat_embedding_grad_workspace(n, rows, cols)
    pat.check(pat_embedding_grad(tokens, size, n, g, stride, _CODE[g.dtype], first, rows, cols, scale, out, out_stride,
                                 _CODE[dtype], _work(need, out.device, stream), need, stream), "pat_embedding_grad")
    return out


def dropout(x, p, seed, index=0, index_stride=None, residual=None, out=None, stream=None):
    """x with each element dropped with probability p or scaled, plus `residual`.  The mask is a function of `seed`
    and the element's place: element (r, c) has number index + r * index_stride + c in the whole tensor
    (`index_stride`: x's columns by default, the whole's for a shard of its columns).  The gradient is the same
    call on the output's gradient.  `out` may be x or the residual."""
    stride = _matrix(x, "x")
    rows, cols = x.shape
    out = _output(out, x.shape, x.dtype, x.device, "dropout")
    out_stride = _matrix(out, "out", x.shape)
    tensors, residual_stride = [x, out], 0
    if residual is not None:
        residual_stride = _matrix(residual, "residual", x.shape)
        if residual.dtype != x.dtype:
            raise ValueError(f"residual is {residual.dtype}, x is {x.dtype}")
        tensors.append(residual)
    stream = _on(stream, *tensors)
    pat.check(pat_dropout(x, stride, residual, residual_stride, out, out_stride, rows, cols, _CODE[x.dtype], p, seed, index,
                          cols if index_stride is None else index_stride, stream), "pat_dropout")
    return out
