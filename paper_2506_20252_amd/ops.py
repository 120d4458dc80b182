"""Binding of include/pat_ops.h: operators on gathered and scattered tensors.

4-bit block quantisation and products, embedding lookup and its gradient,
dropout from a counter-based generator; 8-bit blocks for activations and
checkpoints, root-mean-square norm and the gated feed-forward block, with their
gradients.  The ``pat_*`` functions are the C
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
    "pat_embedding_grad_workspace", "pat_dropout", "pat_mxb_quantize", "pat_mxb_dequantize", "pat_mxb_linear",
    "pat_mxb_weight_grad", "pat_mxb_weight_grad_workspace", "pat_gated", "pat_gated_grad", "pat_rms_norm",
    "pat_rms_norm_grad", "pat_rms_norm_grad_workspace",
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
    "pat_mxb_quantize": ([_P, _S, _N, _N, _I, _P, _P, _P], _I),
    "pat_mxb_dequantize": ([_P, _P, _N, _N, _P, _S, _I, _P], _I),
    "pat_mxb_linear": ([_P, _P, _P, _P, _N, _N, _N, _P, _S, _P, _S, _I, _P], _I),
    "pat_mxb_weight_grad": ([_P, _S, _P, _P, _N, _N, _N, _P, _S, _I, _P, _N, _P], _I),
    "pat_mxb_weight_grad_workspace": ([_N, _N, _N], _N),
    "pat_gated": ([_P, _P, _P, _P, _N, _N, _N, _I, _P, _S, _I, _P, _P, _P, _P, _P], _I),
    "pat_gated_grad": ([_P, _S, _I, _P, _P, _N, _N, _I, _P, _S, _P], _I),
    "pat_rms_norm": ([_P, _S, _P, _S, _I, _P, _I, _N, _N, ctypes.c_float, _P, _S, _P, _S, _I, _P, _P, _P], _I),
    "pat_rms_norm_grad": ([_P, _S, _I, _P, _S, _I, _P, _I, _P, _S, _N, _N, ctypes.c_float, _P, _S, _P, _P, _N, _P], _I),
    "pat_rms_norm_grad_workspace": ([_N, _N], _N),
}

PAT_SILU, PAT_GELU = 0, 1
_ACT = {"silu": PAT_SILU, "gelu": PAT_GELU}


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


def pat_mxb_quantize(x, x_stride, rows, cols, dtype, codes, scales, stream=None):
    return _c.pat_mxb_quantize(_address(x), x_stride, rows, cols, pat._dtype(dtype), _address(codes), _address(scales),
                               pat._stream(stream))


def pat_mxb_dequantize(codes, scales, rows, cols, out, out_stride, dtype, stream=None):
    return _c.pat_mxb_dequantize(_address(codes), _address(scales), rows, cols, _address(out), out_stride,
                                 pat._dtype(dtype), pat._stream(stream))


def pat_mxb_linear(x_codes, x_scales, w_codes, w_scales, m, n, k, residual, residual_stride, out, out_stride, dtype,
                   stream=None):
    return _c.pat_mxb_linear(_address(x_codes), _address(x_scales), _address(w_codes), _address(w_scales), m, n, k,
                             _address(residual), residual_stride, _address(out), out_stride, pat._dtype(dtype),
                             pat._stream(stream))


def pat_mxb_weight_grad(g, g_stride, x_codes, x_scales, rows, inner, cols, out, out_stride, dtype, workspace,
                        workspace_bytes, stream=None):
    return _c.pat_mxb_weight_grad(_address(g), g_stride, _address(x_codes), _address(x_scales), rows, inner, cols,
                                  _address(out), out_stride, pat._dtype(dtype), _address(workspace), workspace_bytes,
                                  pat._stream(stream))


def pat_mxb_weight_grad_workspace(rows, inner, cols):
    return _c.pat_mxb_weight_grad_workspace(rows, inner, cols)


def pat_gated(x_codes, x_scales, w_codes, w_scales, m, n, k, act, out, out_stride, dtype, out_codes, out_scales,
              saved_codes, saved_scales, stream=None):
    return _c.pat_gated(_address(x_codes), _address(x_scales), _address(w_codes), _address(w_scales), m, n, k,
                        _ACT.get(act, act), _address(out), out_stride, pat._dtype(dtype), _address(out_codes),
                        _address(out_scales), _address(saved_codes), _address(saved_scales), pat._stream(stream))


def pat_gated_grad(g, g_stride, g_dtype, saved_codes, saved_scales, m, n, act, out, out_stride, stream=None):
    return _c.pat_gated_grad(_address(g), g_stride, pat._dtype(g_dtype), _address(saved_codes), _address(saved_scales), m,
                             n, _ACT.get(act, act), _address(out), out_stride, pat._stream(stream))


def pat_rms_norm(x, x_stride, residual, residual_stride, dtype, weight, weight_dtype, rows, cols, eps, total, total_stride,
                 out, out_stride, out_dtype, out_codes, out_scales, stream=None):
    return _c.pat_rms_norm(_address(x), x_stride, _address(residual), residual_stride, pat._dtype(dtype), _address(weight),
                           pat._dtype(weight_dtype), rows, cols, eps, _address(total), total_stride, _address(out),
                           out_stride, pat._dtype(out_dtype), _address(out_codes), _address(out_scales),
                           pat._stream(stream))


def pat_rms_norm_grad(g, g_stride, dtype, x, x_stride, x_dtype, weight, weight_dtype, total_grad, total_grad_stride, rows,
                      cols, eps, out, out_stride, dweight, workspace, workspace_bytes, stream=None):
    return _c.pat_rms_norm_grad(_address(g), g_stride, pat._dtype(dtype), _address(x), x_stride, pat._dtype(x_dtype),
                                _address(weight), pat._dtype(weight_dtype), _address(total_grad), total_grad_stride, rows,
                                cols, eps, _address(out), out_stride, _address(dweight), _address(workspace),
                                workspace_bytes, pat._stream(stream))


def pat_rms_norm_grad_workspace(rows, cols):
    return _c.pat_rms_norm_grad_workspace(rows, cols)


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


class Mxb(NamedTuple):
    """A matrix in 8-bit blocks: codes [rows, 128 * G] and scales [rows, 4 * G], uint8 and contiguous, with
    G = ceil(cols / 128).  As a `dtype` it asks for a result in this form."""

    codes: torch.Tensor
    scales: torch.Tensor
    cols: int


def mxb_empty(rows, cols, device="cuda"):
    """An Mxb to write into (uninitialised)."""
    groups = -(-cols // PAT_MX_GROUP)
    return Mxb(torch.empty((rows, 128 * groups), dtype=torch.uint8, device=device),
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


def _blocks(q, what):
    """Checks an Mxb; returns its codes, scales, rows and columns."""
    if type(q) is Mxb:
        codes, scales, cols = q
        groups, size = -(-cols // PAT_MX_GROUP), codes.shape
        if (len(size) == 2 and size[1] == 128 * groups and scales.shape == (size[0], 4 * groups)
                and codes.dtype is scales.dtype is torch.uint8 and codes.is_cuda and scales.is_cuda and codes.is_contiguous()
                and scales.is_contiguous()):
            return codes, scales, size[0], cols
    raise ValueError(f"{what}: an Mxb is needed, codes (rows, 128 * G) and scales (rows, 4 * G) contiguous uint8 GPU tensors "
                     f"with G = ceil(cols / {PAT_MX_GROUP})")


def _weight(w, what):
    """Checks an Mx that stands beside an Mxb; returns its codes, scales, rows and columns."""
    if type(w) is not Mx:
        raise ValueError(f"{what}: an Mx is needed")
    return _stored(w, what)


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
# A new tensor of given strides on the current device and stream, where this torch has it: 0.8 us instead of 1.5.
_strided = getattr(getattr(getattr(torch._C, "_dynamo", None), "guards", None), "_empty_strided_cuda", None)


def _empty(shape, dtype, like, stream):
    """New memory for a call on `stream`: that stream's own (torch hands memory out again in the order of the stream
    that it was allocated on), so that neither earlier nor later work on the current stream meets it."""
    if stream is None:
        if _strided is None or like.get_device() != _current_device():
            return like.new_empty(shape, dtype=dtype)
        return _strided(shape, (shape[1] or 1, 1) if len(shape) == 2 else (1,), dtype)
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


def _blocks_out(out, rows, cols, like, what, stream):
    """An Mxb to write into, given or new."""
    if out is None:
        groups = -(-cols // PAT_MX_GROUP)
        return Mxb(_empty((rows, 128 * groups), torch.uint8, like, stream), _empty((rows, 4 * groups), torch.uint8, like, stream), cols)
    _, _, out_rows, out_cols = _blocks(out, what)
    if out_rows != rows or out_cols != cols:
        raise ValueError(f"{what}: an Mxb of {rows} x {cols} is needed")
    return out


def _result(out, rows, cols, dtype, like, what, stream):
    """A result's place, a matrix of `dtype` or an Mxb: (what is returned, address, row stride, type's number, codes' and scales'
    addresses, the tensors that were given)."""
    if dtype is Mxb:
        given, out = out, _blocks_out(out, rows, cols, like, "out", stream)
        return out, None, 0, pat.PAT_FLOAT32, out.codes.data_ptr(), out.scales.data_ptr(), () if given is None else out[:2]
    code = _CODE.get(dtype)
    if code is None:
        _float(dtype, "dtype")
    if out is None:
        out = _empty((rows, cols), dtype, like, stream)
        return out, out.data_ptr(), cols, code, None, None, ()
    if type(out) is Mxb:
        raise ValueError(f"{what}: out is an Mxb, not {dtype}")
    return out, out.data_ptr(), _output(out, rows, cols, dtype, what), code, None, None, (out,)


def _beside(t, rows, cols, code, what):
    """Checks a matrix of the same shape and type as another; returns its address and row stride."""
    r, c, stride, own = _matrix(t, what)
    if r != rows or c != cols or own != code:
        raise ValueError(f"{what}: shape {(rows, cols)} and the same type are needed, got {(r, c)} of {t.dtype}")
    return t.data_ptr(), stride


def _activation(name):
    act = _ACT.get(name)
    if act is None:
        raise ValueError(f"activation: one of {sorted(_ACT)}, got {name!r}")
    return act


def _work(nbytes, like, stream):
    """Address of a workspace and the tensor that holds it."""
    if not nbytes:
        return None, None
    w = _empty((nbytes,), torch.uint8, like, stream)
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


def mxb_quantize(x, out=None, stream=None):
    """8-bit blocks of a float32 or bfloat16 matrix, as an Mxb."""
    rows, cols, stride, code = _matrix(x, "x")
    out = _blocks_out(out, rows, cols, x, "out", stream)
    on = _on(stream, x, out.codes, out.scales)
    status = _c.pat_mxb_quantize(x.data_ptr(), stride, rows, cols, code, out.codes.data_ptr(), out.scales.data_ptr(), on)
    if status:
        pat.check(status, "pat_mxb_quantize")
    return out


def mxb_dequantize(q, dtype=torch.bfloat16, out=None, stream=None):
    """The matrix that an Mxb stands for, in `dtype` (exact but for bfloat16 below 2^-126; values of 2^128 are infinite)."""
    codes, scales, rows, cols = _blocks(q, "q")
    code = _float(dtype, "dtype")
    if out is None:
        out, stride, on = _empty((rows, cols), dtype, codes, stream), cols, _on(stream, codes, scales)
    else:
        stride, on = _output(out, rows, cols, dtype, "mxb_dequantize"), _on(stream, codes, scales, out)
    status = _c.pat_mxb_dequantize(codes.data_ptr(), scales.data_ptr(), rows, cols, out.data_ptr(), stride, code, on)
    if status:
        pat.check(status, "pat_mxb_dequantize")
    return out


def mxb_linear(x, w, dtype=torch.bfloat16, residual=None, out=None, stream=None):
    """x w^T, plus `residual` where one is given: x an Mxb, w an Mx with as many columns.  `out` may be the residual."""
    x_codes, x_scales, m, k = _blocks(x, "x")
    w_codes, w_scales, n, cols = _weight(w, "w")
    if cols != k:
        raise ValueError(f"x has {k} columns, w has {cols}")
    code = _float(dtype, "dtype")
    if out is None:
        out, stride, on = _empty((m, n), dtype, x_codes, stream), n, _on(stream, x_codes, x_scales, w_codes, w_scales)
    else:
        stride, on = _output(out, m, n, dtype, "mxb_linear"), _on(stream, x_codes, x_scales, w_codes, w_scales, out)
    address, residual_stride = None, 0
    if residual is not None:
        address, residual_stride = _beside(residual, m, n, code, "residual")
        _on(stream, residual)
    status = _c.pat_mxb_linear(x_codes.data_ptr(), x_scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), m, n, k, address,
                               residual_stride, out.data_ptr(), stride, code, on)
    if status:
        pat.check(status, "pat_mxb_linear")
    return out


def mxb_weight_grad(g, x, dtype=torch.bfloat16, out=None, stream=None):
    """g^T x: the gradient of w in ``x w^T`` from its output's gradient g, bfloat16, and the Mxb of its input that was kept."""
    inner, rows, g_stride, _ = _matrix(g, "g")
    codes, scales, terms, cols = _blocks(x, "x")
    if g.dtype != torch.bfloat16:
        raise ValueError(f"g: bfloat16, got {g.dtype}")
    if terms != inner:
        raise ValueError(f"g: {tuple(g.shape)} does not match x's {terms} rows")
    code = _float(dtype, "dtype")
    if out is None:
        out, stride, on = _empty((rows, cols), dtype, g, stream), cols, _on(stream, g, codes, scales)
    else:
        stride, on = _output(out, rows, cols, dtype, "mxb_weight_grad"), _on(stream, g, codes, scales, out)
    need = _c.pat_mxb_weight_grad_workspace(rows, inner, cols)
    work, hold = _work(need, g, stream)
    status = _c.pat_mxb_weight_grad(g.data_ptr(), g_stride, codes.data_ptr(), scales.data_ptr(), rows, inner, cols, out.data_ptr(),
                                    stride, code, work, need, on)
    if status:
        pat.check(status, "pat_mxb_weight_grad")
    return out


def gated(x, w, activation="silu", dtype=torch.bfloat16, checkpoint=False, out=None, stream=None):
    """act(a) * b with a and b the halves of x w^T: x an Mxb, w an Mx whose first half of rows gives a ("silu": a / (1 + e^-a),
    "gelu": a (1 + erf(a / sqrt 2)) / 2).  `dtype` may be Mxb, for a next product.  With `checkpoint` (True, or an Mxb of
    twice x's rows to write into) the result is (out, checkpoint), from which ``gated_grad`` forms the gradients."""
    x_codes, x_scales, m, k = _blocks(x, "x")
    w_codes, w_scales, rows, cols = _weight(w, "w")
    if cols != k:
        raise ValueError(f"x has {k} columns, w has {cols}")
    if rows % 2:
        raise ValueError(f"w: an even number of rows is needed, got {rows}")
    n, act = rows // 2, _activation(activation)
    out, address, stride, code, codes, scales, tensors = _result(out, m, n, dtype, x_codes, "gated", stream)
    saved = saved_codes = saved_scales = None
    if checkpoint is not False and checkpoint is not None:
        saved = _blocks_out(None if checkpoint is True else checkpoint, 2 * m, n, x_codes, "checkpoint", stream)
        saved_codes, saved_scales = saved.codes.data_ptr(), saved.scales.data_ptr()
        if checkpoint is not True:
            tensors += saved[:2]
    on = _on(stream, x_codes, x_scales, w_codes, w_scales, *tensors)
    status = _c.pat_gated(x_codes.data_ptr(), x_scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), m, n, k, act, address,
                          stride, code, codes, scales, saved_codes, saved_scales, on)
    if status:
        pat.check(status, "pat_gated")
    return out if saved is None else (out, saved)


def gated_grad(g, checkpoint, activation="silu", out=None, stream=None):
    """The gradients of a and b of ``gated``, beside each other, bfloat16 [m, 2 n]: with d this result,
    ``mx_matmul_grad(d, w)`` is the gradient of x and ``mxb_weight_grad(d, x)`` that of w."""
    m, n, g_stride, g_code = _matrix(g, "g")
    codes, scales, rows, cols = _blocks(checkpoint, "checkpoint")
    if rows != 2 * m or cols != n:
        raise ValueError(f"checkpoint: an Mxb of {2 * m} x {n} is needed, got {rows} x {cols}")
    act = _activation(activation)
    if out is None:
        out, stride, on = _empty((m, 2 * n), torch.bfloat16, g, stream), 2 * n, _on(stream, g, codes, scales)
    else:
        stride, on = _output(out, m, 2 * n, torch.bfloat16, "gated_grad"), _on(stream, g, codes, scales, out)
    status = _c.pat_gated_grad(g.data_ptr(), g_stride, g_code, codes.data_ptr(), scales.data_ptr(), m, n, act, out.data_ptr(),
                               stride, on)
    if status:
        pat.check(status, "pat_gated_grad")
    return out


def _vector(t, n, what):
    """Checks a weight vector; returns its type's number."""
    if t.shape != (n,) or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous 1-D GPU tensor of {n} elements")
    code = _CODE.get(t.dtype)
    return _float(t.dtype, what) if code is None else code


def rms_norm(x, weight, eps, residual=None, dtype=None, total=None, out=None, stream=None):
    """t * weight / sqrt(mean(t^2) + eps) of every row, t = x; `dtype` is x's by default and may be Mxb, for a next product.
    With a `residual`, t = x + residual rounded to x's type, and the result is (out, t); `total` is where t goes, new by
    default.  `total` or `out` may be x or the residual.  Sums of squares are float32's: full precision up to 2^127 a row, and
    zeros from 2^128 on."""
    rows, cols, x_stride, x_code = _matrix(x, "x")
    weight_code = _vector(weight, cols, "weight")
    out, address, stride, code, codes, scales, tensors = _result(out, rows, cols, x.dtype if dtype is None else dtype, x, "rms_norm",
                                                                 stream)
    res = res_stride = tot = tot_stride = 0
    if residual is not None:
        res, res_stride = _beside(residual, rows, cols, x_code, "residual")
        if total is None:
            total, tot_stride = _empty((rows, cols), x.dtype, x, stream), cols
            tot = total.data_ptr()
            tensors += (residual,)
        else:
            tot, tot_stride = _beside(total, rows, cols, x_code, "total")
            tensors += (residual, total)
    elif total is not None:
        raise ValueError("total: without a residual it is x")
    on = _on(stream, x, weight, *tensors)
    status = _c.pat_rms_norm(x.data_ptr(), x_stride, res, res_stride, x_code, weight.data_ptr(), weight_code, rows, cols, eps, tot,
                             tot_stride, address, stride, code, codes, scales, on)
    if status:
        pat.check(status, "pat_rms_norm")
    return out if residual is None else (out, total)


def rms_norm_grad(g, x, weight, eps, total_grad=None, out=None, stream=None):
    """The gradients of ``rms_norm`` from its output's, g: (dx, dweight), dx of g's type and dweight float32.  x is what was
    normed (the total where there was a residual, whose gradient dx is too); `total_grad`, of g's type, is what reaches
    the total from elsewhere and is added.  `out`, for dx, may be g or `total_grad`."""
    rows, cols, g_stride, g_code = _matrix(g, "g")
    x_rows, x_cols, x_stride, x_code = _matrix(x, "x")
    if x_rows != rows or x_cols != cols:
        raise ValueError(f"g is {tuple(g.shape)}, x is {tuple(x.shape)}")
    weight_code = _vector(weight, cols, "weight")
    if out is None:
        out, stride, on = _empty((rows, cols), g.dtype, g, stream), cols, _on(stream, g, x, weight)
    else:
        stride, on = _output(out, rows, cols, g.dtype, "rms_norm_grad"), _on(stream, g, x, weight, out)
    dweight = _empty((cols,), torch.float32, g, stream)
    tot = tot_stride = 0
    if total_grad is not None:
        tot, tot_stride = _beside(total_grad, rows, cols, g_code, "total_grad")
        _on(stream, total_grad)
    need = _c.pat_rms_norm_grad_workspace(rows, cols)
    work, hold = _work(need, g, stream)
    status = _c.pat_rms_norm_grad(g.data_ptr(), g_stride, g_code, x.data_ptr(), x_stride, x_code, weight.data_ptr(), weight_code, tot,
                                  tot_stride, rows, cols, eps, out.data_ptr(), stride, dweight.data_ptr(), work, need, on)
    if status:
        pat.check(status, "pat_rms_norm_grad")
    return out, dweight
