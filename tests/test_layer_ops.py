"""A layer's operators of include/pat_ops.h: 8-bit blocks, products of them with 4-bit weights, the gated block,
root-mean-square norm, and their gradients.  On the CPU the refusals and the oracle's own pins; on the GPU every operator
against its plain form in 64 bits (oracle/layer.py).

Tolerances, with u = 2^-24 (float32) and e = 2^-8 (bfloat16), half a step of either: as for the operators of
tests/test_ops.py, sums of n terms are off by at most (n + 2) roundings of the sum of magnitudes, doubled for matrix
instructions.  Further ones are derived at their functions.  What leaves in 8-bit blocks is a rounding of a value that is
off by at most some `err`: rounding keeps order, so the code lies between those of the value less and plus `err`, under a
scale that lies between those of the block's largest magnitude less and plus `err`.
"""

import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import layer as L
from oracle import operators as O
from paper_2506_20252_amd import build as B
from paper_2506_20252_amd import ops, pat
from test_ops import E, F32, B16, U, f64, guarded, random_mx, strided, values, within

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
gpu = pytest.mark.gpu


def random_mxb(rows, cols, seed, low=115, high=135, top=0x47):
    """A stored form of random codes up to `top` and scales, on the GPU, and its values in float64."""
    g = np.random.default_rng(seed)
    groups = -(-cols // 128)
    codes = (g.integers(0, top + 1, size=(rows, 128 * groups)) + 128 * g.integers(0, 2, size=(rows, 128 * groups))).astype(np.uint8)
    codes[:, cols:] = 0
    scales = g.integers(low, high, size=(rows, 4 * groups)).astype(np.uint8)
    scales[:, -(-cols // 32):] = 0
    return ops.Mxb(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), cols), L.mxb_values(codes, scales, cols)


def guarded_mxb(rows, cols):
    """An Mxb inside larger buffers of one value, and a check that nothing around it was written."""
    groups = -(-cols // 128)
    codes = torch.full((rows + 2, 128 * groups), 0xEE, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows + 8, 4 * groups), 0xEE, dtype=torch.uint8, device="cuda")

    def untouched():
        return bool((codes[0] == 0xEE).all() and (codes[-1] == 0xEE).all() and (scales[:4] == 0xEE).all() and (scales[-4:] == 0xEE).all())

    return ops.Mxb(codes[1:rows + 1], scales[4:rows + 4], cols), untouched


def blocks_within(q, want, err):
    """The codes and scales of a rounding of values within `err` of `want`; what fills rows up is zero."""
    codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    rows, cols = want.shape
    pad = scales.shape[1] * 32 - cols
    v, err = (np.pad(a, ((0, 0), (0, pad))) for a in (want, np.broadcast_to(err, want.shape)))
    lo, hi = np.maximum(np.abs(v) - err, 0), np.abs(v) + err
    low, high = (L.scale_of(a.reshape(rows, -1, 32).max(axis=2)) for a in (lo, hi))
    assert np.all((low <= scales) & (scales <= high))
    s = np.repeat(scales, 32, axis=1)
    top = 3.75 * np.exp2(s.astype(np.float64) - 127)
    got = L.CODES[codes] * np.exp2(s.astype(np.float64) - 127)
    below, above = (L.CODES[L.code_of(np.clip(a, -top, top), s)] * np.exp2(s.astype(np.float64) - 127) for a in (v - err, v + err))
    assert np.all((below <= got) & (got <= above))
    assert np.all(codes[:, cols:] == 0)


# ---------------------------------------------------------------------------
# On the CPU
# ---------------------------------------------------------------------------


def test_oracle_codes_by_hand():
    assert L.CODES[[0, 1, 7, 8, 0x38, 0x7E, 0xB8, 0xFE]].tolist() == [0, 2.0**-9, 7 * 2.0**-9, 2.0**-6, 1, 448, -1, -448]
    row = np.zeros((1, 160))
    row[0, :9] = [3.75, 1.0625, 1.1875, -1.0625, 2.0**-10, 3 * 2.0**-10, 3.625, 3.375, -0.0]
    row[0, 32] = 3.8125
    row[0, 64], row[0, 65] = np.nan, 1
    row[0, 96] = 2.0**-149
    row[0, 128] = -3.5 * 2.0**100
    codes, scales = L.mxb_quantize(row)
    assert scales[0].tolist() == [127, 128, 255, 0, 227, 0, 0, 0]
    assert codes[0, :9].tolist() == [0x47, 0x38, 0x3A, 0xB8, 0, 2, 0x46, 0x46, 0x80]  # all ties, to the even code
    assert codes[0, 32] == 0x3F and not codes[0, 64:96].any() and codes[0, 96] == 0 and codes[0, 128] == 0xC6
    v = L.mxb_values(codes, scales, 160)
    assert np.isnan(v[0, 64:96]).all() and v[0, 32] == 3.75 and v[0, 128] == -3.5 * 2.0**100


def test_oracle_gradients_against_differences():
    g = np.random.default_rng(1)
    t, w, dy = g.standard_normal((3, 7)), g.standard_normal(7), g.standard_normal((3, 7))
    dx, dw = L.rms_norm_grad(dy, t, w, 1e-3)
    h = 1e-5
    for r, c in ((0, 0), (1, 3), (2, 6)):
        step = np.zeros((3, 7))
        step[r, c] = h
        diff = np.sum(dy * (L.rms_norm(t + step, w, 1e-3) - L.rms_norm(t - step, w, 1e-3))) / (2 * h)
        assert abs(diff - dx[r, c]) < 1e-8
        diff = np.sum(dy * (L.rms_norm(t, w + step[r], 1e-3) - L.rms_norm(t, w - step[r], 1e-3))) / (2 * h)
        assert abs(diff - dw[c]) < 1e-8
    a, b = g.standard_normal((2, 50)) * 4, g.standard_normal((2, 50))
    dy = g.standard_normal((2, 50))
    for name in ("silu", "gelu"):
        d = L.gated_grad(dy, a, b, name)
        assert np.allclose(d[:, :50], dy * (L.gated(a + h, b, name) - L.gated(a - h, b, name)) / (2 * h), atol=1e-8)
        assert np.allclose(d[:, 50:], dy * (L.gated(a, b + h, name) - L.gated(a, b - h, name)) / (2 * h), atol=1e-8)


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include/hip"),
                    reason="no g++ or no HIP headers")
def test_host_side_under_asan_ubsan(tmp_path):
    """How sizes are cut into workgroups, what the entry points take and hand on."""
    exe = tmp_path / "layer_check"
    csrc = os.path.join(ROOT, "paper_2506_20252_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", csrc, os.path.join(csrc, "layer.cpp"),
           os.path.join(ROOT, "tests", "host", "layer_check.cpp"), "-o", str(exe)]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, (res.stdout[-2000:], res.stderr[-2000:])
    assert " 0 failures" in res.stdout


@pytest.mark.parametrize("source", ["mxb.hip", "mxb_product.hip", "gated.hip", "norm.hip"])
def test_kernels_as_compiled(source, tmp_path):
    """No scratch memory, no packed fp32; a workgroup of eight waves leaves two waves a SIMD their registers."""
    if shutil.which(B.hipcc()) is None:
        pytest.skip("hipcc not available")
    out = tmp_path / "kernels.s"
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    subprocess.run([B.hipcc(), *flags, "--cuda-device-only", "-S", "-I", os.path.join(ROOT, "include"),
                    os.path.join(B.CSRC, source), "-o", str(out)], check=True, capture_output=True, timeout=600)
    asm = out.read_text()
    names, private, vgprs = (re.findall(rf"^\s+\.{field}:\s+(\S+)$", asm, re.M)
                             for field in ("name", "private_segment_fixed_size", "vgpr_count"))
    assert names and len(names) == len(private) == len(vgprs)
    assert not [(n, p) for n, p in zip(names, private) if p != "0"]
    assert not [(n, v) for n, v in zip(names, vgprs) if int(v) > 256]
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm)


BASE = 1 << 32  # addresses that no call below may reach


def args_of(**defaults):
    def make(**kw):
        assert not set(kw) - set(defaults)
        return list({**defaults, **kw}.values())

    make.defaults = defaults
    return make


quantize_args = args_of(x=BASE, x_stride=200, rows=3, cols=200, dtype="float32", codes=BASE + 0x10000, scales=BASE + 0x20000)
dequantize_args = args_of(codes=BASE, scales=BASE + 0x1000, rows=3, cols=200, out=BASE + 0x2000, out_stride=200, dtype="bfloat16")
linear_args = args_of(x_codes=BASE, x_scales=BASE + 0x1000, w_codes=BASE + 0x2000, w_scales=BASE + 0x4000, m=3, n=5, k=200,
                      residual=BASE + 0x6000, residual_stride=5, out=BASE + 0x5000, out_stride=5, dtype="float32")
weight_grad_args = args_of(g=BASE, g_stride=40, x_codes=BASE + 0x1000000, x_scales=BASE + 0x2000000, rows=40, inner=8449, cols=200,
                           out=BASE + 0x4000000, out_stride=200, dtype="float32", workspace=BASE + 0x5000000,
                           workspace_bytes=1 << 24)
gated_args = args_of(x_codes=BASE, x_scales=BASE + 0x1000, w_codes=BASE + 0x2000, w_scales=BASE + 0x4000, m=3, n=5, k=200, act=0,
                     out=BASE + 0x5000, out_stride=5, dtype="float32", out_codes=0, out_scales=0, saved_codes=BASE + 0x6000,
                     saved_scales=BASE + 0x7000)
gated_grad_args = args_of(g=BASE, g_stride=200, g_dtype="float32", saved_codes=BASE + 0x2000, saved_scales=BASE + 0x3000, m=3, n=200,
                          act=1, out=BASE + 0x4000, out_stride=400)
norm_args = args_of(x=BASE, x_stride=200, residual=BASE + 0x1000, residual_stride=200, dtype="float32", weight=BASE + 0x2000,
                    weight_dtype="bfloat16", rows=3, cols=200, eps=1e-5, total=BASE + 0x3000, total_stride=200, out=BASE + 0x4000,
                    out_stride=200, out_dtype="bfloat16", out_codes=0, out_scales=0)
norm_grad_args = args_of(g=BASE, g_stride=200, dtype="float32", x=BASE + 0x10000, x_stride=200, x_dtype="bfloat16",
                         weight=BASE + 0x20000, weight_dtype="float32", total_grad=BASE + 0x30000, total_grad_stride=200, rows=30,
                         cols=200, eps=1e-5, out=BASE + 0x40000, out_stride=200, dweight=BASE + 0x50000, workspace=BASE + 0x60000,
                         workspace_bytes=1 << 20)

INVALID, UNSUPPORTED, TOO_LARGE = pat.PAT_ERR_INVALID_ARGUMENT, pat.PAT_ERR_UNSUPPORTED, pat.PAT_ERR_TOO_LARGE
REFUSED = [
    (ops.pat_mxb_quantize, quantize_args, [
        (dict(x=0), INVALID), (dict(x=BASE + 2), INVALID), (dict(x_stride=199), INVALID), (dict(codes=BASE + 0x10008), INVALID),
        (dict(scales=BASE + 0x20002), INVALID), (dict(codes=BASE), INVALID), (dict(scales=BASE + 0x10000), INVALID),
        (dict(dtype="int32"), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED),
        (dict(rows=1 << 30, cols=1 << 10, x_stride=1 << 10), UNSUPPORTED)]),
    (ops.pat_mxb_dequantize, dequantize_args, [
        (dict(codes=0), INVALID), (dict(scales=0), INVALID), (dict(out=BASE + 0x2001), INVALID), (dict(out=BASE + 64), INVALID),
        (dict(out_stride=100), INVALID), (dict(dtype="int32"), UNSUPPORTED)]),
    (ops.pat_mxb_linear, linear_args, [
        (dict(x_codes=0), INVALID), (dict(x_scales=BASE + 0x1002), INVALID), (dict(w_codes=BASE + 0x2008), INVALID),
        (dict(w_scales=0), INVALID), (dict(out=0), INVALID), (dict(out=BASE), INVALID), (dict(out=BASE + 0x2000), INVALID),
        (dict(out_stride=4), INVALID), (dict(residual_stride=4), INVALID), (dict(residual=BASE + 0x6002), INVALID),
        (dict(residual=BASE + 0x5004), INVALID), (dict(residual=BASE + 0x5000, residual_stride=6), INVALID),
        (dict(dtype="int32"), UNSUPPORTED), (dict(n=1 << 31), UNSUPPORTED), (dict(k=1 << 24), UNSUPPORTED)]),
    (ops.pat_mxb_weight_grad, weight_grad_args, [
        (dict(g=0), INVALID), (dict(g=BASE + 1), INVALID), (dict(g_stride=39), INVALID), (dict(x_codes=0), INVALID),
        (dict(out=BASE + 0x1000000), INVALID), (dict(dtype="int32"), UNSUPPORTED), (dict(workspace_bytes=64), TOO_LARGE),
        (dict(workspace=BASE + 0x5000008), INVALID), (dict(workspace=BASE + 0x4000000), INVALID), (dict(workspace=0), INVALID),
        (dict(workspace=BASE), INVALID), (dict(workspace=BASE + 0x2000000), INVALID)]),
    (ops.pat_gated, gated_args, [
        (dict(x_codes=0), INVALID), (dict(w_scales=0), INVALID), (dict(act=2), UNSUPPORTED), (dict(act=-1), UNSUPPORTED),
        (dict(out=0), INVALID), (dict(out_codes=BASE + 0x8000, out_scales=BASE + 0x9000), INVALID),
        (dict(out=0, out_codes=BASE + 0x8000), INVALID), (dict(out=0, out_codes=BASE + 0x8008, out_scales=BASE + 0x9000), INVALID),
        (dict(out=0, out_codes=BASE + 0x6000, out_scales=BASE + 0x9000), INVALID),
        (dict(out=0, out_codes=BASE + 0x8000, out_scales=BASE + 0x8010), INVALID),
        (dict(out=BASE), INVALID), (dict(out=BASE + 0x6000), INVALID), (dict(out_stride=4), INVALID), (dict(saved_codes=0), INVALID),
        (dict(saved_scales=0), INVALID), (dict(saved_codes=BASE + 0x2000), INVALID), (dict(saved_scales=BASE + 0x6000), INVALID),
        (dict(saved_scales=BASE + 0x1000), INVALID), (dict(dtype="int32"), UNSUPPORTED), (dict(n=1 << 25), UNSUPPORTED),
        (dict(m=1 << 26), UNSUPPORTED)]),
    (ops.pat_gated_grad, gated_grad_args, [
        (dict(g=0), INVALID), (dict(g_stride=199), INVALID), (dict(saved_codes=0), INVALID), (dict(saved_scales=BASE + 0x3001), INVALID),
        (dict(out=0), INVALID), (dict(out_stride=399), INVALID), (dict(out=BASE), INVALID), (dict(out=BASE + 0x2000), INVALID),
        (dict(act=7), UNSUPPORTED), (dict(g_dtype="int32"), UNSUPPORTED), (dict(m=1 << 30), UNSUPPORTED)]),
    (ops.pat_rms_norm, norm_args, [
        (dict(x=0), INVALID), (dict(x_stride=199), INVALID), (dict(weight=0), INVALID), (dict(weight=BASE + 0x2001), INVALID),
        (dict(residual=0), INVALID), (dict(residual=BASE + 0x1001), INVALID), (dict(eps=-1e-9), INVALID), (dict(eps=math.nan), INVALID),
        (dict(eps=math.inf), INVALID), (dict(total=BASE + 4), INVALID), (dict(total=BASE, total_stride=201), INVALID),
        (dict(total=BASE + 0x2000), INVALID), (dict(out=BASE + 0x3000), INVALID), (dict(out=BASE), INVALID), (dict(out=0), INVALID),
        (dict(out_codes=BASE + 0x8000, out_scales=BASE + 0x9000), INVALID),
        (dict(out=0, out_codes=BASE + 0x1000, out_scales=BASE + 0x9000), INVALID),
        (dict(out=0, out_codes=BASE + 0x8000, out_scales=BASE + 0x2000), INVALID), (dict(dtype="int32"), UNSUPPORTED),
        (dict(weight_dtype="int32"), UNSUPPORTED), (dict(out_dtype="int32"), UNSUPPORTED), (dict(cols=1 << 31), UNSUPPORTED)]),
    (ops.pat_rms_norm_grad, norm_grad_args, [
        (dict(g=0), INVALID), (dict(x=0), INVALID), (dict(weight=0), INVALID), (dict(dweight=0), INVALID),
        (dict(dweight=BASE + 0x50002), INVALID), (dict(g_stride=3), INVALID), (dict(total_grad=BASE + 0x30002), INVALID),
        (dict(out=BASE + 4), INVALID), (dict(out=BASE + 0x30000, out_stride=201), INVALID), (dict(out=BASE + 0x10000), INVALID),
        (dict(dweight=BASE + 0x40000), INVALID), (dict(dweight=BASE), INVALID), (dict(eps=-1.0), INVALID),
        (dict(workspace_bytes=16), TOO_LARGE), (dict(workspace=0), INVALID), (dict(workspace=BASE + 0x60008), INVALID),
        (dict(workspace=BASE + 0x40000), INVALID), (dict(workspace=BASE + 0x50000), INVALID), (dict(dtype="int32"), UNSUPPORTED),
        (dict(rows=1 << 28), UNSUPPORTED), (dict(cols=1 << 26), UNSUPPORTED)]),
]


@pytest.mark.parametrize("call,args,change,status", [(c, a, d, s) for c, a, cases in REFUSED for d, s in cases],
                         ids=lambda v: getattr(v, "__name__", str(v)) if not isinstance(v, dict) else str(v))
def test_bad_arguments_are_refused_before_any_device_call(call, args, change, status):
    assert call(*args(**change)) == status


def test_calls_without_elements_launch_nothing():
    assert ops.pat_mxb_quantize(*quantize_args(rows=0, x=0, codes=0, scales=0)) == pat.PAT_OK
    assert ops.pat_mxb_dequantize(*dequantize_args(cols=0, out=0, codes=0, scales=0)) == pat.PAT_OK
    assert ops.pat_mxb_linear(*linear_args(m=0, out=0, residual=0)) == pat.PAT_OK
    assert ops.pat_mxb_weight_grad(*weight_grad_args(rows=0, out=0, workspace=0)) == pat.PAT_OK
    assert ops.pat_gated(*gated_args(n=0, out=0)) == pat.PAT_OK
    assert ops.pat_gated_grad(*gated_grad_args(m=0, g=0, out=0)) == pat.PAT_OK
    assert ops.pat_rms_norm(*norm_args(rows=0, x=0, residual=0, total=0, out=0)) == pat.PAT_OK
    assert ops.pat_rms_norm_grad(*norm_grad_args(cols=0, g=0, x=0, out=0, dweight=0, weight=0)) == pat.PAT_OK


def test_tensor_calls_refuse_what_the_kernels_do_not_take():
    x, w = torch.zeros(4, 8), torch.zeros(8)
    q = ops.Mxb(torch.zeros(4, 128).byte(), torch.zeros(4, 4).byte(), 8)
    m = ops.Mx(torch.zeros(6, 64).byte(), torch.zeros(6, 4).byte(), 8)
    for call in (lambda: ops.mxb_quantize(x), lambda: ops.mxb_dequantize(q), lambda: ops.mxb_dequantize(m), lambda: ops.mxb_linear(q, m),
                 lambda: ops.mxb_linear(x, m), lambda: ops.mxb_weight_grad(x.bfloat16(), q), lambda: ops.gated(q, m),
                 lambda: ops.gated_grad(x, q), lambda: ops.rms_norm(x, w, 1e-5), lambda: ops.rms_norm_grad(x, x, w, 1e-5)):
        with pytest.raises(ValueError):
            call()


@gpu
def test_tensor_calls_refuse_what_does_not_match():
    x, w = values((4, 40), 1), torch.ones(40, device="cuda")
    q, m = ops.mxb_quantize(x), ops.mx_quantize(values((6, 40), 2))
    odd, other = ops.mx_quantize(values((7, 40), 3)), ops.mxb_quantize(values((4, 41), 4))
    for call in (lambda: ops.mxb_linear(other, m), lambda: ops.mxb_linear(q, q), lambda: ops.mxb_linear(m, m),
                 lambda: ops.mxb_linear(q, m, F32, residual=values((4, 6), 5, B16)), lambda: ops.mxb_linear(q, m, F32, residual=x),
                 lambda: ops.gated(q, odd), lambda: ops.gated(q, m, "tanh"), lambda: ops.gated(q, m, checkpoint=q),
                 lambda: ops.gated(q, m, dtype=torch.float16), lambda: ops.gated(q, m, dtype=ops.Mx),
                 lambda: ops.gated(q, m, dtype=F32, out=ops.mxb_empty(4, 3)), lambda: ops.gated(q, m, dtype=ops.Mxb, out=x),
                 lambda: ops.gated_grad(x, q), lambda: ops.mxb_weight_grad(x, q), lambda: ops.mxb_weight_grad(x[:3].bfloat16(), q),
                 lambda: ops.rms_norm(x, w[:39], 1e-5), lambda: ops.rms_norm(x, w, 1e-5, total=x),
                 lambda: ops.rms_norm(x, w, 1e-5, residual=x.bfloat16()), lambda: ops.rms_norm(x, w.half(), 1e-5),
                 lambda: ops.rms_norm_grad(x, x[:3], w, 1e-5), lambda: ops.rms_norm_grad(x, x, w, 1e-5, total_grad=x.bfloat16()),
                 lambda: ops.mxb_quantize(x, out=other)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError):
        ops.rms_norm(x, w, -1.0)


# ---------------------------------------------------------------------------
# 8-bit blocks
# ---------------------------------------------------------------------------

SHAPES = [(1, 1), (1, 31), (2, 32), (3, 33), (5, 127), (4, 128), (7, 129), (1, 255), (33, 100), (16, 640), (3, 1111), (2, 4)]


@gpu
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 0), (9, 1)])
def test_quantize(rows, cols, dtype, pad, shift):
    x = values((rows, cols), rows * 1000 + cols, dtype)
    x.view(-1)[::7] = 0
    q, untouched = guarded_mxb(rows, cols)
    ops.mxb_quantize(strided(x, pad, shift) if pad else x, out=q)
    assert untouched()
    codes, scales = L.mxb_quantize(f64(x))
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    for dtype_out in (F32, B16):
        out, untouched = guarded((rows, cols), dtype_out, pad, shift)
        assert np.array_equal(f64(ops.mxb_dequantize(q, dtype_out, out)), L.mxb_values(codes, scales, cols))
        assert untouched()


@gpu
@pytest.mark.parametrize("dtype", [F32, B16])
def test_quantize_edges(dtype):
    """Every tie, both ends of the scales, subnormals, the largest values, infinities, NaN, negative zero, a block of zeros."""
    x = torch.zeros((16, 160), dtype=torch.float64)
    ties = torch.from_numpy((L.CODES[:71] + L.CODES[1:72]) / 2)
    for r, e in enumerate((0, -100, 100, -117, -127, 126)):
        x[r, :71] = ties * 2.0**e
        for block in range(4):
            x[r, 32 * block + 31] = 3.75 * 2.0**e  # the scale is known
    x[6, 0], x[6, 1], x[6, 64] = 2.0**-133, -0.0, -0.0
    x[7, 3], x[7, 40] = float("inf"), float("-inf")
    x[8, 31], x[8, 95] = float("nan"), 1.0
    big = 3.3895313892515355e38  # the largest bfloat16
    x[9, 0], x[9, 1], x[9, 2], x[9, 33] = big, -big, 1e38, big / 3
    x[10, :32] = 2.0**-126
    x[11, 0], x[11, 1] = 1.0, 1e-30
    for block, top in enumerate((3.75, 3.765625, 1.875, 1.8828125, 4.0)):  # either side of where the scale goes up
        x[12, 32 * block] = top
    x = x.to(dtype).cuda()
    q = ops.mxb_quantize(x)
    codes, scales = L.mxb_quantize(f64(x))
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    # the largest values are nearest to 2^128, which neither type holds
    want = torch.from_numpy(L.mxb_values(codes, scales, 160)).float()
    assert bool(torch.isinf(want[9, :2]).all()) and int(torch.isinf(want).sum()) == 2
    assert np.array_equal(f64(ops.mxb_dequantize(q, F32)), f64(want), equal_nan=True)
    assert np.array_equal(f64(ops.mxb_dequantize(q, B16)), f64(want.to(B16)), equal_nan=True)


@gpu
def test_dequantize_every_code_and_scale():
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.tile(np.arange(256, dtype=np.uint8)[:, None], (1, 8))
    q = ops.Mxb(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 256)
    want = torch.from_numpy(L.mxb_values(codes, scales, 256)).float()
    assert np.array_equal(f64(ops.mxb_dequantize(q, F32)), f64(want), equal_nan=True)
    assert np.array_equal(f64(ops.mxb_dequantize(q, B16)), f64(want.to(B16)), equal_nan=True)


# ---------------------------------------------------------------------------
# Products
# ---------------------------------------------------------------------------

PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 300, 128), (2, 17, 129), (3, 33, 500), (16, 16, 512), (17, 100, 640), (24, 70, 1001),
            (40, 65, 300), (48, 8300, 130), (33, 4200, 300), (64, 64, 256), (65, 130, 96), (100, 129, 777), (128, 128, 1024),
            (130, 257, 384), (256, 256, 512), (300, 270, 1300), (520, 260, 130), (5, 2000, 64), (2000, 3, 200), (1, 64, 20000),
            (48, 40, 8200), (49, 49, 500), (1500, 1500, 250), (2900, 2900, 140), (60, 100, 7), (700, 5, 640)]


@gpu
@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", [F32, B16])
def test_linear(m, n, k, dtype):
    x, vx = random_mxb(m, k, m + n)
    w, vw = random_mx(n, k, n + k)
    want, size = vx @ vw.T, np.abs(vx) @ np.abs(vw).T
    out, untouched = guarded((m, n), dtype, pad=n % 3, shift=k % 2)
    ops.mxb_linear(x, w, dtype, out=out)
    assert untouched()
    within(out, want, size, k, dtype)
    res = values((m, n), m * n, dtype, 2.0**10)
    for view in (res, strided(res, 5, 1)):
        out, untouched = guarded((m, n), dtype)
        ops.mxb_linear(x, w, dtype, view, out)
        assert untouched()
        within(out, want + f64(res), size + np.abs(f64(res)), k + 1, dtype)
    view = strided(res, 3)
    ops.mxb_linear(x, w, dtype, view, view)  # in place
    assert torch.equal(view, out)


@gpu
@pytest.mark.parametrize("m,n,k", [(3, 70, 1000), (300, 270, 1300), (33, 50, 128)])
def test_linear_of_codes_up_to_448(m, n, k):
    """Products that are added in eights keep 13 bits below the exponent of the largest: each loses less than 2^-13 of that,
    eight of them 2^-10 of it, and no more of the sum of magnitudes."""
    x, vx = random_mxb(m, k, m + n, top=0x7E)
    w, vw = random_mx(n, k, n + k)
    size = np.abs(vx) @ np.abs(vw).T
    off = np.abs(f64(ops.mxb_linear(x, w, F32)) - vx @ vw.T)
    assert np.all(off <= (2.0**-10 + 2 * (k + 2) * U) * size)


def act_error(a, name, ea):
    """An activation's error at a value that is off by `ea`: slopes are below 1.13; the exponential is off by (|a| + 2) u and the
    quotient and the product by 3 u more; P(a) = (1 + erf(a / sqrt 2)) / 2 is off by 4 u at most."""
    return 1.13 * ea + U * ((np.abs(a) + 8) * np.abs(L.act(a, name)[0]) + 4 * np.abs(a))


def gated_error(vx, vw, n, k, name):
    """h, a, b and their errors."""
    y, size = vx @ vw.T, 2 * (k + 2) * U * (np.abs(vx) @ np.abs(vw).T)
    a, b, ea, eb = y[:, :n], y[:, n:], size[:, :n], size[:, n:]
    value, ev = L.act(a, name)[0], act_error(a, name, ea)
    return value * b, a, b, ev * np.abs(b) + (np.abs(value) + ev) * eb + 2 * U * np.abs(value * b), ea, eb


@gpu
@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_gated(m, n, k, name):
    x, vx = random_mxb(m, k, m + n, 118, 124)
    w, vw = random_mx(2 * n, k, n + k, 115, 124)
    h, a, b, eh, ea, eb = gated_error(vx, vw, n, k, name)
    for dtype in (F32, B16):
        out, untouched = guarded((m, n), dtype, pad=n % 3, shift=k % 2)
        ops.gated(x, w, name, dtype, out=out)
        assert untouched()
        off = np.abs(f64(out) - h)
        assert np.all(off <= eh + (E if dtype == B16 else 2 * U) * np.abs(h) + 1e-300)
    plain = out
    q, untouched = guarded_mxb(m, n)
    saved, saved_untouched = guarded_mxb(2 * m, n)
    got, kept = ops.gated(x, w, name, ops.Mxb, saved, q)
    assert got is q and kept is saved and untouched() and saved_untouched()
    blocks_within(q, h, eh)
    blocks_within(ops.Mxb(saved.codes[:m], saved.scales[:m], n), a, ea)
    blocks_within(ops.Mxb(saved.codes[m:], saved.scales[m:], n), b, eb)
    # the same with the other outputs, to the bit
    other, kept = ops.gated(x, w, name, B16, True)
    assert torch.equal(other, plain) and torch.equal(kept.codes, saved.codes) and torch.equal(kept.scales, saved.scales)
    alone = ops.gated(x, w, name, ops.Mxb)
    assert torch.equal(alone.codes, q.codes) and torch.equal(alone.scales, q.scales)


@gpu
def test_gated_without_a_checkpoint():
    q, m = ops.mxb_quantize(values((4, 40), 1)), ops.mx_quantize(values((6, 40), 2))
    want, kept = ops.gated(q, m, checkpoint=True)
    assert type(kept) is ops.Mxb
    for none in (False, None):
        assert torch.equal(ops.gated(q, m, checkpoint=none), want)


@gpu
@pytest.mark.parametrize("m,n", [(1500, 1501), (2900, 2899), (700, 300)])  # every size of tile
@pytest.mark.parametrize("k", [1030, 1160, 1290, 1420, 2430])  # 9, 10, 11, 12 and 19 groups: every rest of the loop by four
def test_products_through_many_columns_of_tiles(m, n, k):
    """The reference in 64 bits by the GPU's library.  Twice: a race would hardly give the same bits."""
    x, vx = random_mxb(m, k, m + k)
    w, vw = random_mx(n, k, n + k)
    tx, tw = torch.from_numpy(vx).cuda(), torch.from_numpy(vw).cuda().t().contiguous()
    want, size = f64(torch.mm(tx, tw)), f64(torch.mm(tx.abs(), tw.abs()))
    for dtype in (F32, B16):
        out, untouched = guarded((m, n), dtype, pad=1)
        ops.mxb_linear(x, w, dtype, out=out)
        assert untouched()
        within(out, want, size, k, dtype)
        assert torch.equal(out, ops.mxb_linear(x, w, dtype))
    if n % 2 == 0 or n == 1501:
        half = (n // 2)
        w2 = ops.Mx(w.codes[:2 * half], w.scales[:2 * half], k)
        h, saved = ops.gated(x, w2, "silu", ops.Mxb, True)
        ea = 2 * (k + 2) * U * size[:, :2 * half]
        blocks_within(ops.Mxb(saved.codes[:m], saved.scales[:m], half), want[:, :half], ea[:, :half])
        blocks_within(ops.Mxb(saved.codes[m:], saved.scales[m:], half), want[:, half:2 * half], ea[:, half:])
        again = ops.gated(x, w2, "silu", ops.Mxb, True)
        assert torch.equal(h.codes, again[0].codes) and torch.equal(saved.codes, again[1].codes)


@gpu
@pytest.mark.parametrize("m,n,k", [(3, 20, 0), (300, 300, 0)])
def test_products_of_no_columns(m, n, k):
    x, w = ops.mxb_empty(m, k), ops.mx_empty(2 * n, k)
    out, res = torch.full((m, 2 * n), 5.0, device="cuda"), values((m, 2 * n), 1)
    assert bool((ops.mxb_linear(x, w, F32, out=out) == 0).all()) and torch.equal(ops.mxb_linear(x, w, F32, res), res)
    assert bool((ops.gated(x, w, dtype=F32) == 0).all())
    h, saved = ops.gated(x, w, "gelu", ops.Mxb, True)
    assert not any(bool(t.any()) for t in (*h[:2], *saved[:2]))
    assert bool((ops.mxb_weight_grad(torch.empty((0, 9), dtype=B16, device="cuda"), ops.mxb_empty(0, 40), F32) == 0).all())


@gpu
def test_product_of_no_columns_and_more_tiles_than_a_launch_holds():
    m, n = 1 << 17, 1 << 16
    res = values((m, 1), 1, B16).expand(m, n).contiguous()
    assert torch.equal(ops.mxb_linear(ops.mxb_empty(m, 0), ops.mx_empty(n, 0), B16, res, res.clone()), res)


@gpu
@pytest.mark.parametrize("m,n,k", [(2, 40, 256), (70, 40, 300), (300, 300, 256)])
def test_products_carry_what_is_not_finite(m, n, k):
    """A NaN block makes its token's results NaN and no other's, and blocks of them NaN in whole; so does a NaN code; sums that
    are too large are infinite, and their blocks NaN."""
    v = values((m, k), 5, F32)
    v[1, 7] = float("inf")
    w, _ = random_mx(2 * n, k, 6)
    x = ops.mxb_quantize(v)
    x.codes[0, k - 1] = 0x7F
    x.scales[0, (k - 1) // 32] = 127
    got = f64(ops.mxb_linear(x, w, F32))
    assert np.isnan(got[:2]).all() and np.isfinite(got[2:]).all()
    h, saved = ops.gated(x, w, dtype=ops.Mxb, checkpoint=True)
    blocks = -(-n // 32)
    for q, rows in ((h, [0, 1]), (saved, [0, 1, m, m + 1])):
        nan = q.scales[:, :blocks] == 255
        assert bool(nan[rows].all()) and int(nan.sum()) == len(rows) * blocks and not bool(q.codes[rows].any())
    big, _ = random_mxb(m, k, 7, 250, 253)
    heavy, _ = random_mx(2 * n, k, 8, 250, 253)
    assert not np.isfinite(f64(ops.mxb_linear(big, heavy, F32))).any()
    q = ops.gated(big, heavy, dtype=ops.Mxb)
    assert bool((q.scales[:, :blocks] == 255).all())
    x.scales[1] = 127
    g = torch.ones((m, n), dtype=B16, device="cuda")
    got = f64(ops.mxb_weight_grad(g, x, F32))
    assert np.isnan(got[:, k - 1]).all() and np.isfinite(got[:, :k - 1]).all()


WEIGHT_GRADS = [(1, 1, 1), (1, 16, 32), (3, 40, 33), (16, 32, 128), (33, 65, 100), (64, 64, 64), (70, 129, 257), (130, 70, 300),
                (256, 128, 256), (300, 200, 520), (20, 3000, 40), (257, 1000, 129), (1000, 5, 130), (64, 31, 640), (100, 4096, 90),
                (64, 5761, 33), (40, 8449, 200), (130, 8, 64), (9, 7, 300), (7, 500, 40), (1500, 330, 1490), (1537, 70, 1501),
                (2901, 390, 2900), (2896, 261, 2950)]


@gpu
@pytest.mark.parametrize("rows,inner,cols", WEIGHT_GRADS)
@pytest.mark.parametrize("dtype", [F32, B16])
def test_weight_grad(rows, inner, cols, dtype):
    g = values((inner, rows), rows + inner, B16)
    x, vx = random_mxb(inner, cols, cols)
    vg = f64(g).T
    for view in (g, strided(g, 3, 1)):
        out, untouched = guarded((rows, cols), dtype)
        ops.mxb_weight_grad(view, x, dtype, out)
        assert untouched()
        within(out, vg @ vx, np.abs(vg) @ np.abs(vx), inner, dtype)


@gpu
def test_linear_gradients_against_differences():
    """The product is linear in each value, so a changed code changes sum(g * out) by the change times that value's gradient,
    up to the sums' rounding."""
    m, n, k = 24, 40, 130
    x, vx = random_mxb(m, k, 1, 120, 126)
    w, vw = random_mx(n, k, 2, 120, 130)
    g = values((m, n), 3, B16)
    vg, base = f64(g), f64(ops.mxb_linear(x, w, F32))
    dw = f64(ops.mxb_weight_grad(g, x, F32))
    for r, c in ((0, 0), (5, 31), (11, 77), (39, 129)):
        moved = ops.Mx(w.codes.clone(), w.scales, k)
        moved.codes[r, c // 2] ^= 1 << (4 * (c % 2) + 2)
        step = O.mx_values(moved.codes.cpu().numpy(), w.scales.cpu().numpy(), k)[r, c] - vw[r, c]
        after = f64(ops.mxb_linear(x, moved, F32))
        size = np.abs(vg) * (np.abs(vx) @ np.abs(vw).T + np.abs(after))
        assert abs(np.sum(vg * (after - base)) - step * dw[r, c]) <= 8 * (k + n + m) * U * np.sum(size)


# ---------------------------------------------------------------------------
# The gated block's gradient
# ---------------------------------------------------------------------------


def slope_error(a, name):
    """silu' = s (1 + a (1 - s)): s is off by (|a| + 6) u s; 1 - s by that and u, times s |a|; products and sums 4 u more.
    gelu' = P + a p: P by 4 u, p by (a^2 + 8) u, and as much for products."""
    if name == "silu":
        s = 0.5 * (1 + np.tanh(0.5 * a))
        return U * ((np.abs(a) + 10) * s * (1 + 2 * np.abs(a)) + np.abs(a))
    return U * (8 + np.abs(a) * np.exp(-0.5 * a * a) * (a * a + 12))


def check_gated_grad(d, g, a, b, name):
    want = L.gated_grad(g, a, b, name)
    err = np.concatenate((np.abs(g * b) * slope_error(a, name), np.abs(g) * act_error(a, name, 0.0)), axis=1)
    assert np.all(np.abs(f64(d) - want) <= 1.01 * err + (E + 4 * U) * np.abs(want) + 2.0**-133)


@gpu
@pytest.mark.parametrize("m,n", SHAPES + [(70, 3000), (1, 20000), (300, 7)])
@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [F32, B16])
def test_gated_grad(m, n, name, dtype):
    g = values((m, n), m + n, dtype)
    saved, v = random_mxb(2 * m, n, n, 110, 124)
    for view in (g, strided(g, 3, 1)):
        out, untouched = guarded((m, 2 * n), B16, pad=n % 5)
        ops.gated_grad(view, saved, name, out)
        assert untouched()
        check_gated_grad(out, f64(g), v[:m], v[m:], name)


@gpu
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_gated_grad_of_far_values_and_differences(name):
    """Values where the exponential overflows or vanishes; a gradient against the definition's differences."""
    a = torch.tensor([[0.0, -0.0, 1e-30, -1e-30, 88.0, -88.0, 104.0, -104.0, 1000.0, -1000.0, 1e30, -1e30, 3.0, -3.0, 0.5, -0.5]]).cuda()
    q = [ops.mxb_quantize(a.t().contiguous().repeat_interleave(32, 1).view(1, -1)), ops.mxb_quantize(torch.full((1, 512), 1.5).cuda())]
    saved = ops.Mxb(torch.cat([p.codes for p in q]), torch.cat([p.scales for p in q]), 512)
    g = torch.ones((1, 512), device="cuda")
    d = ops.gated_grad(g, saved, name)
    va = f64(ops.mxb_dequantize(q[0], F32))
    with np.errstate(over="ignore", under="ignore"):
        check_gated_grad(d, f64(g), va, np.full((1, 512), 1.5), name)
    near = np.abs(va) < 200
    h = 1e-4
    diff = (L.gated(va + h, 1.5, name) - L.gated(va - h, 1.5, name)) / (2 * h)
    assert np.all(np.abs(f64(d)[:, :512] - diff)[near] <= (E * np.abs(diff) + 1e-6)[near])


# ---------------------------------------------------------------------------
# Norm
# ---------------------------------------------------------------------------


def depth(cols):
    """Roundings that a term of a row's sum goes through: 8 in a lane's vector, 4 vectors, 6 exchanges, 15 waves, and a turn for
    every 2048 columns of long rows."""
    return 33 + cols / 2048


NORMS = [(1, 1), (3, 2), (2, 3), (5, 4), (3, 5), (1, 8), (300, 7), (70, 31), (9, 33), (4, 127), (65, 128), (7, 129), (2, 1000), (3, 2048),
         (1, 2049), (5, 4096), (3, 4100), (2, 8192), (1, 8200), (2, 16384), (2, 16385), (3, 32768), (1, 40001), (2049, 130), (2100, 4096), (2050, 1000),
         (2048, 515), (5000, 16), (600, 2129), (513, 3000), (300, 9795), (270, 16383)]


@gpu
@pytest.mark.parametrize("rows,cols", NORMS)
@pytest.mark.parametrize("dtype,out_dtype,weight_dtype", [(F32, F32, F32), (B16, B16, F32), (B16, F32, B16), (F32, B16, B16),
                                                          (B16, ops.Mxb, F32), (F32, ops.Mxb, B16)])
def test_rms_norm(rows, cols, dtype, out_dtype, weight_dtype):
    x, res = values((rows, cols), rows + cols, dtype), values((rows, cols), cols, dtype)
    weight = 1 + values((cols,), 5, weight_dtype)
    x[0, ::3] = 0
    eps = 2.0**-7
    for a, r in ((x, None), (strided(x, 3, 1), None), (x, res), (strided(x, 1), strided(res, 2, 1))):
        t = x if r is None else (x.float() + res.float()).to(dtype)
        want = L.rms_norm(f64(t), f64(weight), eps)
        err = (depth(cols) / 2 + 8) * U * np.abs(want)
        if out_dtype is ops.Mxb:
            out, untouched = guarded_mxb(rows, cols)
        else:
            out, untouched = guarded((rows, cols), out_dtype, pad=cols % 3)
        if r is None:
            got = ops.rms_norm(a, weight, eps, dtype=out_dtype, out=out)
        else:
            total, total_untouched = guarded((rows, cols), dtype, pad=1)
            got, kept = ops.rms_norm(a, weight, eps, r, out_dtype, total, out)
            assert kept is total and total_untouched() and torch.equal(total, t)
        assert got is out and untouched()
        if out_dtype is ops.Mxb:
            blocks_within(out, want, err)
        else:
            assert np.all(np.abs(f64(out) - want) <= err + (E if out_dtype == B16 else 2 * U) * np.abs(want) + 2.0**-133)


@gpu
@pytest.mark.parametrize("rows,cols", NORMS)
@pytest.mark.parametrize("dtype,x_dtype,weight_dtype", [(F32, F32, F32), (B16, B16, F32), (F32, B16, B16), (B16, F32, B16)])
def test_rms_norm_grad(rows, cols, dtype, x_dtype, weight_dtype):
    x, g, more = values((rows, cols), rows + cols, x_dtype), values((rows, cols), cols, dtype), values((rows, cols), rows, dtype)
    weight = 1 + values((cols,), 5, weight_dtype)
    eps = 2.0**-7
    vx, vg, vw = f64(x), f64(g), f64(weight)
    r = 1 / np.sqrt(np.mean(vx * vx, axis=1, keepdims=True) + eps)
    size = r * (np.abs(vg * vw) + np.abs(vx) * r**2 * np.mean(np.abs(vg * vw * vx), axis=1, keepdims=True))
    first = None
    for a, b, t in ((x, g, None), (x, g, more), (strided(x, 3, 1), strided(g, 1), strided(more, 2, 1))):
        dx, dw = L.rms_norm_grad(vg, vx, vw, eps, None if t is None else f64(more))
        out, untouched = guarded((rows, cols), dtype, pad=cols % 3)
        got, dweight = ops.rms_norm_grad(b, a, weight, eps, t, out)
        assert got is out and untouched()
        extra = 0 if t is None else np.abs(f64(more))
        assert np.all(np.abs(f64(out) - dx) <= 2 * (depth(cols) + 12) * U * size + 2 * U * extra + (E if dtype == B16 else 2 * U) * np.abs(dx) + 2.0**-133)
        within(dweight, dw, np.sum(np.abs(vg * vx * r), axis=0), rows + depth(cols), F32)
        first = dweight if first is None else first
        assert torch.equal(first, dweight)  # to the bit, whatever the strides


@gpu
def test_rms_norm_gradient_against_differences():
    rows, cols, eps = 5, 300, 1e-3
    x, g, weight = values((rows, cols), 1), values((rows, cols), 2), values((cols,), 3)
    dx, dw = (f64(t) for t in ops.rms_norm_grad(g, x, weight, eps))
    vx, vg, vw = f64(x), f64(g), f64(weight)

    def loss(t, w):
        return np.sum(vg * L.rms_norm(t, w, eps))

    for r, c in ((0, 0), (2, 150), (4, 299)):
        h = 1e-4 * max(1.0, abs(vx[r, c]))
        step = np.zeros((rows, cols))
        step[r, c] = h
        diff = (loss(vx + step, vw) - loss(vx - step, vw)) / (2 * h)
        size = np.abs(vg[r] * vw).max() / np.sqrt(np.mean(vx[r]**2))
        assert abs(diff - dx[r, c]) <= 1e-4 * size  # differences are good to h^2, sums to 42 u
        diff = (loss(vx, vw + step[r]) - loss(vx, vw - step[r])) / (2 * h)
        assert abs(diff - dw[c]) <= 1e-5 * np.sum(np.abs(vg[:, c] * vx[:, c]) / np.sqrt(np.mean(vx**2, axis=1)))


@gpu
@pytest.mark.parametrize("cols", [100, 4096, 20000])
@pytest.mark.parametrize("dtype", [F32, B16])
def test_norm_in_place(cols, dtype):
    rows = 9
    x, res, weight = values((rows, cols), 1, dtype), values((rows, cols), 2, dtype), values((cols,), 3)
    want, total = ops.rms_norm(x, weight, 1e-5, res)
    for target in ("x", "residual"):
        a, r = x.clone(), res.clone()
        to = a if target == "x" else r
        got, kept = ops.rms_norm(a, weight, 1e-5, r, total=to)
        assert kept is to and torch.equal(got, want) and torch.equal(to, total)
        a, r = x.clone(), res.clone()
        to = a if target == "x" else r
        got, kept = ops.rms_norm(a, weight, 1e-5, r, out=to)
        assert torch.equal(to, want) and torch.equal(kept, total)
    a = x.clone()
    assert torch.equal(ops.rms_norm(a, weight, 1e-5, out=a), ops.rms_norm(x, weight, 1e-5))
    g, more = values((rows, cols), 4, dtype), values((rows, cols), 5, dtype)
    dx, dw = ops.rms_norm_grad(g, x, weight, 1e-5, more)
    for target in ("g", "more"):
        a, b = g.clone(), more.clone()
        got, dweight = ops.rms_norm_grad(a, x, weight, 1e-5, b, out=a if target == "g" else b)
        assert torch.equal(got, dx) and torch.equal(dweight, dw)


@gpu
@pytest.mark.parametrize("rows,cols", [(9000, 7), (5000, 333), (1500, 2129), (700, 16383), (600, 16391)])
@pytest.mark.parametrize("dtype", [F32, B16])
def test_norm_in_place_through_many_rows(rows, cols, dtype):
    """More rows than go through at once, with ends that vectors are moved down from: the next row is read before this one is written."""
    x, res, weight = values((rows, cols), 1, dtype), values((rows, cols), 2, dtype), values((cols,), 3)
    want, total = ops.rms_norm(x, weight, 1e-5, res)
    a, r = x.clone(), res.clone()
    got, kept = ops.rms_norm(a, weight, 1e-5, r, total=a, out=r)
    assert got is r and kept is a and torch.equal(got, want) and torch.equal(kept, total)
    a = x.clone()
    assert torch.equal(ops.rms_norm(a, weight, 1e-5, out=a), ops.rms_norm(x, weight, 1e-5))
    dx, dw = ops.rms_norm_grad(res, x, weight, 1e-5, total)
    for target in ("g", "more"):
        g, more = res.clone(), total.clone()
        got, dweight = ops.rms_norm_grad(g, x, weight, 1e-5, more, out=g if target == "g" else more)
        assert torch.equal(got, dx) and torch.equal(dweight, dw)


@gpu
@pytest.mark.parametrize("cols", [33, 4096, 20001])
def test_norm_of_one_tensor_in_two_places(cols):
    """x its own residual, g the total's gradient too, a weight that starts inside another vector."""
    x, g = values((70, cols), 1, B16), values((70, cols), 2, B16)
    weight = values((cols + 1,), 3, B16)[1:]
    out, total = ops.rms_norm(x, weight, 1e-5, x)
    other = ops.rms_norm(x.clone(), weight.clone(), 1e-5, x.clone())
    assert torch.equal(out, other[0]) and torch.equal(total, other[1])
    both = x.clone()
    out, total = ops.rms_norm(both, weight, 1e-5, both, total=both)
    assert total is both and torch.equal(out, other[0]) and torch.equal(both, other[1])
    want = ops.rms_norm_grad(g.clone(), x, weight.clone(), 1e-5, g.clone())
    both = g.clone()
    got = ops.rms_norm_grad(both, x, weight, 1e-5, both, out=both)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@gpu
@pytest.mark.parametrize("m,n,k", [(5, 70, 300), (60, 140, 300), (300, 1500, 700), (1500, 1500, 300)])
def test_rows_of_stored_matrices(m, n, k):
    """Rows of a larger stored matrix are a stored matrix: as input, as weight and as output."""
    x, w = ops.mxb_quantize(values((m + 7, k), 1)), ops.mx_quantize(values((2 * n + 5, k), 2))
    part = ops.Mxb(x.codes[3:m + 3], x.scales[3:m + 3], k)
    rows = ops.Mx(w.codes[5:], w.scales[5:], k)
    own = ops.Mxb(part.codes.clone(), part.scales.clone(), k), ops.Mx(rows.codes.clone(), rows.scales.clone(), k)
    assert torch.equal(ops.mxb_linear(part, rows), ops.mxb_linear(*own))
    out = ops.Mxb(*(t.fill_(0x55) for t in ops.mxb_empty(m + 2, n)[:2]), n)
    ops.gated(part, rows, "silu", ops.Mxb, out=ops.Mxb(out.codes[1:-1], out.scales[1:-1], n))
    want = ops.gated(*own, "silu", ops.Mxb)
    assert torch.equal(out.codes[1:-1], want.codes) and torch.equal(out.scales[1:-1], want.scales)
    for t in out[:2]:
        assert bool((t[0] == 0x55).all()) and bool((t[-1] == 0x55).all())
    g = values((m, n), 3, B16)
    assert torch.equal(ops.mxb_weight_grad(g, part), ops.mxb_weight_grad(g, own[0]))


@gpu
@pytest.mark.parametrize("cols", [40, 300, 20000])
def test_norm_of_zero_rows_infinities_and_nan(cols):
    """A row of zeros gives zeros (NaN where eps is 0, as the formula does), what is not finite stays in its row, and blocks of
    such a row are NaN with zeros behind its end."""
    x, weight = values((5, cols), 1), torch.ones(cols, device="cuda")
    x[0], x[1, 3], x[2, 5] = 0, float("nan"), float("inf")
    got = f64(ops.rms_norm(x, weight, 1e-5))
    assert (got[0] == 0).all() and np.isnan(got[1]).all() and np.isnan(got[2, 5]) and np.isfinite(got[3:]).all()
    assert (np.delete(got[2], 5) == 0).all()
    assert np.isnan(f64(ops.rms_norm(x, weight, 0.0))[0]).all()
    blocks = -(-cols // 32)
    q = ops.rms_norm(x, weight, 0.0, dtype=ops.Mxb)
    assert bool((q.scales[:2, :blocks] == 255).all()) and not bool(q.scales[:, blocks:].any()) and bool((q.scales[3:, :blocks] < 255).all())
    assert not bool(q.codes[:2].any()) and int((q.scales[2] == 255).sum()) == 1
    g = values((5, cols), 2)
    dx, dw = ops.rms_norm_grad(g, x, weight, 1e-5)
    assert np.isnan(f64(dx)[1]).all() and np.isfinite(f64(dx)[[0, 3, 4]]).all() and np.isnan(f64(dw)).any()


@gpu
def test_norm_of_no_rows():
    g, weight = torch.empty((0, 70), device="cuda"), torch.ones(70, device="cuda")
    dx, dw = ops.rms_norm_grad(g, g, weight, 1e-5)
    assert dx.shape == (0, 70) and dw.shape == (70,) and not bool(dw.any())
    assert ops.rms_norm(g, weight, 1e-5).shape == (0, 70)


# ---------------------------------------------------------------------------
# Streams, graphs, large offsets
# ---------------------------------------------------------------------------


def flat(v):
    return [v] if isinstance(v, torch.Tensor) else [t for p in v if not isinstance(p, int) for t in flat(p)]


def every_operator():
    """Name -> call of a stream, on inputs of its own."""
    x, w = values((60, 300), 1, B16), torch.ones(300, device="cuda")
    res, g = values((60, 300), 2, B16), values((60, 70), 3, B16)
    q, m = ops.mxb_quantize(x), ops.mx_quantize(values((140, 300), 4))
    few = ops.mxb_quantize(x[:5])
    saved = ops.mxb_quantize(values((120, 70), 5))
    tall, tall_g = ops.mxb_quantize(values((8449, 200), 6)), values((8449, 40), 7, B16)
    long, long_w = values((30, 20000), 8), torch.ones(20000, device="cuda")
    return {
        "quantize": lambda s=None: ops.mxb_quantize(x, stream=s), "dequantize": lambda s=None: ops.mxb_dequantize(q, F32, stream=s),
        "linear": lambda s=None: ops.mxb_linear(q, m, F32, stream=s), "linear_few": lambda s=None: ops.mxb_linear(few, m, B16, stream=s),
        "gated": lambda s=None: ops.gated(q, m, "silu", ops.Mxb, True, stream=s), "gated_few": lambda s=None: ops.gated(few, m, "gelu", F32, stream=s),
        "gated_grad": lambda s=None: ops.gated_grad(g, saved, stream=s),
        "weight_grad": lambda s=None: ops.mxb_weight_grad(tall_g, tall, F32, stream=s),
        "norm": lambda s=None: ops.rms_norm(x, w, 1e-5, res, ops.Mxb, stream=s),
        "norm_grad": lambda s=None: ops.rms_norm_grad(res, x, w, 1e-5, x, stream=s),
        "norm_grad_long": lambda s=None: ops.rms_norm_grad(long, long, long_w, 1e-5, stream=s),
    }


EVERY = ["quantize", "dequantize", "linear", "linear_few", "gated", "gated_few", "gated_grad", "weight_grad", "norm", "norm_grad",
         "norm_grad_long"]


@gpu
@pytest.mark.parametrize("name", EVERY)
def test_graph_replays(name):
    """Captured once, in a pool of its own, and replayed with eager work between: every replay gives the eager result."""
    call = every_operator()[name]
    want = [t.clone() for t in flat(call())]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = flat(call())
    for _ in range(4):
        for t in got:
            t.zero_()
        junk = torch.full((1 << 22,), 0x77, dtype=torch.uint8, device="cuda")
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(flat(call()), want))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool((junk == 0x77).all())


@gpu
def test_two_streams_at_once():
    """Calls that run beside each other share nothing: each gives what it gives alone."""
    calls = every_operator()
    want = {name: [t.clone() for t in flat(call())] for name, call in calls.items()}
    x, w = ops.mxb_quantize(values((1500, 1300), 1)), ops.mx_quantize(values((3000, 1300), 2))
    calls["tiles"] = lambda s=None: ops.gated(x, w, "gelu", ops.Mxb, True, stream=s)
    want["tiles"] = [t.clone() for t in flat(calls["tiles"]())]
    torch.cuda.synchronize()
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    names = list(calls)
    for shift in range(len(names)):
        got = []
        for i, name in enumerate(names):
            other = names[(i + shift) % len(names)]
            got += [(name, calls[name](first)), (other, calls[other](second))]
        torch.cuda.synchronize()
        for name, out in got:
            assert all(torch.equal(a, b) for a, b in zip(flat(out), want[name])), (name, shift)


@gpu
@pytest.mark.parametrize("name", EVERY)
def test_results_and_workspaces_belong_to_the_stream_of_the_call(name):
    """The result is right while the current stream writes over memory that it has just freed, and its memory is the other
    stream's."""
    call, side = every_operator()[name], torch.cuda.Stream()
    want = [t.clone() for t in flat(call())]
    torch.cuda.synchronize()
    for handle in (side, side.cuda_stream):
        for _ in range(3):
            torch.cuda._sleep(2_000_000)
            late = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (512, 4480, 15600, 24000, 84000, 200000, 1 << 21)]
            for t in late:
                t.fill_(0x77)
            del late, t
            got = flat(call(handle))
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        torch.cuda.synchronize()
        segments = torch.cuda.memory_snapshot()
        for t in got:
            where = [s["stream"] for s in segments if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]
            assert where == [side.cuda_stream]


@gpu
def test_offsets_beyond_32_bits():
    """Rows spread over 10 GiB: byte and element offsets pass 2^32."""
    pitch, rows, cols = 1 << 30, 5, 40
    room = torch.zeros((rows, pitch), dtype=B16, device="cuda")
    far, out, third = room[:, :cols], room[:, 128:128 + cols], room[:, 256:256 + 2 * cols]
    small, res, weight = values((rows, cols), 1, B16), values((rows, cols), 2, B16), values((cols,), 3)
    far.copy_(small)
    q, want = ops.mxb_quantize(far), ops.mxb_quantize(small)
    assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
    assert torch.equal(ops.mxb_dequantize(want, B16, out), ops.mxb_dequantize(want, B16))
    w = ops.mx_quantize(values((2 * cols, cols), 4))
    half = ops.Mx(w.codes[:cols], w.scales[:cols], cols)
    assert torch.equal(ops.mxb_linear(want, half, B16, far, out), ops.mxb_linear(want, half, B16, small))
    assert torch.equal(ops.gated(want, w, dtype=B16, out=out), ops.gated(want, w, dtype=B16))
    saved = ops.mxb_quantize(values((2 * rows, cols), 5))
    assert torch.equal(ops.gated_grad(far, saved, out=third), ops.gated_grad(small, saved))
    assert torch.equal(ops.mxb_weight_grad(far, want, F32), ops.mxb_weight_grad(small, want, F32))
    a, b = ops.rms_norm(far, weight, 1e-5, res, out=out), ops.rms_norm(small, weight, 1e-5, res)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    a, b = ops.rms_norm_grad(far, res, weight, 1e-5, out=out), ops.rms_norm_grad(small, res, weight, 1e-5)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert bool((room[:, cols:128] == 0).all()) and bool((room[:, 400:4096] == 0).all())


@gpu
@pytest.mark.parametrize("name", ["quantize", "gated_grad", "norm", "norm_grad"])
def test_more_work_than_a_launch_has_workgroups(name):
    """Workgroups that go round several times: every part of a large result is that of a small call on the same values."""
    parts = 4099
    if name == "quantize":  # more than 2^26 groups
        x = values((4096, 600), 1, B16)
        q, got = ops.mxb_quantize(x), ops.mxb_quantize(x.repeat(parts, 1)[:-5])
        assert got.codes.shape[0] * 5 > 1 << 26
        for big, small in zip(got[:2], q[:2]):
            assert all(torch.equal(part, small[:len(part)]) for part in big.split(4096))
        back = ops.mxb_dequantize(got, B16)
        small = ops.mxb_dequantize(q, B16)
        assert all(torch.equal(part, small[:len(part)]) for part in back.split(4096))
    elif name == "gated_grad":  # more than 2^25 groups
        rows = (1 << 25) + 4097
        g = values((4096, 6), 1, B16)
        a, b = ops.mxb_quantize(values((4096, 6), 2)), ops.mxb_quantize(values((4096, 6), 3))
        n = -(-rows // 4096)
        big = [torch.cat((p.repeat(n, 1)[:rows], q.repeat(n, 1)[:rows])) for p, q in zip(a[:2], b[:2])]
        want = ops.gated_grad(g, ops.Mxb(torch.cat((a.codes, b.codes)), torch.cat((a.scales, b.scales)), 6))
        got = ops.gated_grad(g.repeat(n, 1)[:rows], ops.Mxb(*big, 6))
        assert all(torch.equal(part, want[:len(part)]) for part in got.split(4096))
    elif name == "norm":  # 256 rows a workgroup
        rows = (1 << 28) + 70001
        x, weight = values((1 << 20, 3), 1, B16), values((3,), 2)
        want, got = ops.rms_norm(x, weight, 1e-5), ops.rms_norm(x.repeat(257, 1)[:rows], weight, 1e-5)
        assert all(torch.equal(part, want[:len(part)]) for part in got.split(1 << 20))
    else:  # the most rows
        rows = (1 << 28) - 1
        x = values((1 << 20, 2), 1, B16).repeat(256, 1)[:rows]
        g, weight = torch.ones((rows, 2), dtype=B16, device="cuda"), values((2,), 2)
        dx, dw = ops.rms_norm_grad(g, x, weight, 1e-5)
        want, dw_part = ops.rms_norm_grad(g[:1 << 20], x[:1 << 20], weight, 1e-5)
        assert all(torch.equal(part, want[:len(part)]) for part in dx.split(1 << 20))
        # parts of 2^28 / (512 * 256) rows a lane, then sums of their sums
        size = (x[:1 << 20].double().abs() * torch.rsqrt(x[:1 << 20].double().square().mean(1, keepdim=True) + 1e-5)).sum(0)
        assert bool(((dw.double() - 256 * dw_part.double()).abs() <= (2048 + 1024) * 2 * U * 256 * size).all())


# ---------------------------------------------------------------------------
# The operators together
# ---------------------------------------------------------------------------


@gpu
@pytest.mark.parametrize("m,n,k", [(1, 96, 64), (7, 200, 130), (70, 333, 256), (300, 640, 384)])
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_a_layer_forward_and_backward(m, n, k, name):
    """Norm, gated block and projection back with the residual, and their gradients from what the forward pass keeps in 8 bits:
    every step against the definitions, from what the step before it gave."""
    eps = 1e-5
    x, res, weight = values((m, k), 1, B16), values((m, k), 2, B16), 1 + values((k,), 3, F32, 0.1)
    w, vw = random_mx(2 * n, k, 4, 118, 122)
    back, vback = random_mx(k, n, 5, 118, 122)
    y, total = ops.rms_norm(x, weight, eps, res, ops.Mxb)
    h, saved = ops.gated(y, w, name, ops.Mxb, True)
    out = ops.mxb_linear(h, back, B16, total)
    dout = values((m, k), 6, B16)
    dh = ops.mx_matmul_grad(dout, back, B16)
    d = ops.gated_grad(dh, saved, name)
    dy = ops.mx_matmul_grad(d, w, B16)
    dx, dweight = ops.rms_norm_grad(dy, total, weight, eps, dout)
    dback, dw = ops.mxb_weight_grad(dout, h, F32), ops.mxb_weight_grad(d, y, F32)

    t = f64(total)
    assert torch.equal(total, (x.float() + res.float()).to(B16))
    norm = L.rms_norm(t, f64(weight), eps)
    blocks_within(y, norm, (depth(k) / 2 + 8) * U * np.abs(norm))
    vy, vh = (L.mxb_values(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.cols) for q in (y, h))
    want, a, b, eh, ea, eb = gated_error(vy, vw, n, k, name)
    blocks_within(h, want, eh)
    vs = L.mxb_values(saved.codes.cpu().numpy(), saved.scales.cpu().numpy(), n)
    blocks_within(ops.Mxb(saved.codes[:m], saved.scales[:m], n), a, ea)
    blocks_within(ops.Mxb(saved.codes[m:], saved.scales[m:], n), b, eb)
    within(out, vh @ vback.T + t, np.abs(vh) @ np.abs(vback).T + np.abs(t), n + 1, B16)
    vo, vdh, vd, vdy = f64(dout), f64(dh), f64(d), f64(dy)
    within(dh, vo @ vback, np.abs(vo) @ np.abs(vback), k, B16)
    check_gated_grad(d, vdh, vs[:m], vs[m:], name)
    within(dy, vd @ vw, np.abs(vd) @ np.abs(vw), 2 * n, B16)
    want, want_w = L.rms_norm_grad(vdy, t, f64(weight), eps, vo)
    r = 1 / np.sqrt(np.mean(t * t, axis=1, keepdims=True) + eps)
    u = np.abs(vdy * f64(weight))
    size = r * (u + np.abs(t) * r**2 * np.mean(u * np.abs(t), axis=1, keepdims=True))
    assert np.all(np.abs(f64(dx) - want) <= 2 * (depth(k) + 12) * U * size + 2 * U * np.abs(vo) + E * np.abs(want) + 2.0**-133)
    within(dweight, want_w, np.sum(np.abs(vdy * t * r), axis=0), m + depth(k), F32)
    within(dback, vo.T @ vh, np.abs(vo).T @ np.abs(vh), m, F32)
    within(dw, vd.T @ vy, np.abs(vd).T @ np.abs(vy), m, F32)
