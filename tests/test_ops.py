"""Operators of include/pat_ops.h: the binding's and the C calls' refusals and
the oracle's own pins on the CPU; on the GPU every operator against its plain
form in 64 bits (oracle/operators.py).

Tolerances, with u = 2^-24 (float32) and e = 2^-8 (bfloat16, twice its
rounding): results that are one product are off by one rounding; sums of n
terms by at most (n + 2) roundings of the sum of magnitudes (Higham, Accuracy
and Stability of Numerical Algorithms, 2002, chapter 3), doubled for matrix
instructions, which may cut where float32 adds round; an output in bfloat16
adds e times its value.  Codes, scales, widened values and masks are exact.
"""

import ctypes
import importlib.util
import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2506_20252_amd import build as B
from paper_2506_20252_amd import ops, pat

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U, E = 2.0**-24, 2.0**-8
F32, B16 = torch.float32, torch.bfloat16
gpu = pytest.mark.gpu


def f64(t):
    return t.detach().double().cpu().numpy()


def values(shape, seed, dtype=F32, scale=1.0):
    """Normal values of widely different row and column sizes, as a tensor on the GPU."""
    g = np.random.default_rng(seed)
    x = g.standard_normal(shape) * scale
    if len(shape) == 2:
        x *= np.exp2(g.integers(-6, 7, size=(shape[0], 1))) * np.where(g.random((1, shape[1])) < 0.05, 16.0, 1.0)
    return torch.from_numpy(x).to(dtype).cuda()


def strided(t, pad, shift=0):
    """The same values as rows of a wider matrix, `shift` elements off its start."""
    wide = torch.full((t.shape[0], t.shape[1] + pad + shift), float("nan"), dtype=t.dtype, device=t.device)
    view = wide[:, shift:shift + t.shape[1]]
    view.copy_(t)
    return view


def guarded(shape, dtype, pad=0, shift=0):
    """An output view inside a larger buffer of one value, and a check that nothing around it was written."""
    rows, cols = shape
    wide = torch.full((rows + 2, cols + pad + shift + 2), -77.0, dtype=dtype, device="cuda")
    view = wide[1:rows + 1, shift + 1:shift + 1 + cols]

    def untouched():
        around = wide.clone()
        around[1:rows + 1, shift + 1:shift + 1 + cols] = -77.0
        return bool((around == -77.0).all())

    return view, untouched


def random_mx(rows, cols, seed, low=110, high=140):
    """A stored form of random codes and scales, on the GPU, and its values in float64."""
    g = np.random.default_rng(seed)
    groups = -(-cols // 128)
    codes = g.integers(0, 16, size=(rows, 128 * groups))
    codes[:, cols:] = 0
    scales = g.integers(low, high, size=(rows, 4 * groups))
    scales[:, -(-cols // 32):] = 0
    c, s = O.mx_pack(codes, scales)
    return ops.Mx(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), cols), O.mx_values(c, s, cols)


def within(got, want, magnitude, terms, dtype):
    """|got - want| at most what (terms + 2) doubled roundings of the magnitude and the output's type allow."""
    bound = 2 * (terms + 2) * U * magnitude + (E if dtype == B16 else 2 * U) * np.abs(want) + 1e-300
    off = np.abs(f64(got) - want)
    assert np.all(off <= bound), (off.max(), (off / bound).max(), np.argmax(off / bound))


# ---------------------------------------------------------------------------
# On the CPU
# ---------------------------------------------------------------------------


def test_library_exports_every_operator():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "pat_ops.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(pat_[a-z_]+)\s*\(", text)))
    lib = ctypes.CDLL(pat.LIB_PATH)
    assert names == sorted(ops.EXPORTS) and all(hasattr(lib, n) for n in names)


def test_philox_known_answers():
    """The three vectors published with the generator."""
    assert O.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert O.philox([ones] * 4, [ones] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert O.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_oracle_quantisation_by_hand():
    """Ties, the clamp, both ends of the scales and a block that is not finite."""
    row = np.zeros((1, 160))
    row[0, :12] = [7.9, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, 0.26, 4.99]
    row[0, 32] = np.inf
    row[0, 64] = 2.0**-149
    row[0, 96] = 2.0**127
    row[0, 128] = -2.0**-100
    codes, scales = O.mx_quantize(row)
    assert codes[0, :12].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 10, 1, 6]
    assert scales[0].tolist() == [127, 255, 0, 252, 25, 0, 0, 0]
    assert codes[0, 32:64].tolist() == [0] * 32 and codes[0, 64] == 0 and codes[0, 96] == 6 and codes[0, 128] == 14
    v = O.mx_values(*O.mx_pack(codes, scales), 160)
    assert np.isnan(v[0, 32:64]).all() and v[0, 96] == 2.0**127 and v[0, 128] == -2.0**-100


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include/hip"),
                    reason="no g++ or no HIP headers")
def test_host_side_under_asan_ubsan(tmp_path):
    """How sizes are cut into workgroups, slices and pieces, and what the entry points hand on."""
    exe = tmp_path / "ops_check"
    csrc = os.path.join(ROOT, "paper_2506_20252_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", csrc, os.path.join(csrc, "ops.cpp"),
           os.path.join(ROOT, "tests", "host", "ops_check.cpp"), "-o", str(exe)]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, (res.stdout[-2000:], res.stderr[-2000:])
    assert " 0 failures" in res.stdout


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include/hip"),
                    reason="no g++ or no HIP headers")
def test_launches_hold_their_lanes(tmp_path):
    """Every size that is accepted gives a launch of fewer than 2^32 lanes that reaches all of its work."""
    exe = tmp_path / "ops_grid_check"
    csrc = os.path.join(ROOT, "paper_2506_20252_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", csrc, os.path.join(csrc, "ops.cpp"),
           os.path.join(ROOT, "tests", "host", "ops_grid_check.cpp"), "-o", str(exe)]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, (res.stdout[-2000:], res.stderr[-2000:])
    assert " 0 failures" in res.stdout


@pytest.mark.parametrize("source", ["mx.hip", "mx_product.hip", "mx_grad.hip", "embedding.hip", "dropout.hip"])
def test_kernels_as_compiled(source, tmp_path):
    """No scratch memory, no packed fp32; a workgroup of eight waves and more leaves two waves a SIMD their registers."""
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


def quantize_args(**kw):
    a = dict(x=BASE, x_stride=200, rows=3, cols=200, dtype="float32", codes=BASE + 0x10000, scales=BASE + 0x20000)
    return list({**a, **kw}.values())


def matmul_args(**kw):
    a = dict(a_codes=BASE, a_scales=BASE + 0x1000, b_codes=BASE + 0x2000, b_scales=BASE + 0x4000, m=3, n=5, k=200,
             out=BASE + 0x5000, out_stride=5, dtype="float32")
    return list({**a, **kw}.values())


def linear_args(**kw):
    a = dict(x=BASE, x_stride=200, x_dtype="bfloat16", w_codes=BASE + 0x2000, w_scales=BASE + 0x4000, m=3, n=5, k=200,
             out=BASE + 0x5000, out_stride=5, dtype="float32", workspace=BASE + 0x8000, workspace_bytes=1 << 20)
    return list({**a, **kw}.values())


def grad_args(**kw):
    a = dict(g=BASE, g_stride=5, transposed=0, q_codes=BASE + 0x2000, q_scales=BASE + 0x4000, rows=3, inner=5, cols=200,
             out=BASE + 0x5000, out_stride=200, dtype="float32", workspace=BASE + 0x8000, workspace_bytes=1 << 20)
    return list({**a, **kw}.values())


def embedding_args(**kw):
    a = dict(tokens=BASE, token_bytes=4, ntokens=7, table=BASE + 0x1000, table_stride=200, table_dtype="float32", first=0,
             rows=5, cols=200, scale=1.0, out=BASE + 0x5000, out_stride=200, dtype="float32")
    return list({**a, **kw}.values())


def embedding_grad_args(**kw):
    a = dict(tokens=BASE, token_bytes=4, ntokens=5000, g=BASE + 0x10000, g_stride=200, g_dtype="float32", first=0, rows=5,
             cols=200, scale=1.0, out=BASE + 0x1000000, out_stride=200, dtype="float32", workspace=BASE + 0x2000000,
             workspace_bytes=1 << 24)
    return list({**a, **kw}.values())


def dropout_args(**kw):
    a = dict(x=BASE, x_stride=200, residual=BASE + 0x10000, residual_stride=200, out=BASE + 0x20000, out_stride=200, rows=3,
             cols=200, dtype="float32", p=0.1, seed=1, index=0, index_stride=200)
    return list({**a, **kw}.values())


INVALID, UNSUPPORTED, TOO_LARGE = pat.PAT_ERR_INVALID_ARGUMENT, pat.PAT_ERR_UNSUPPORTED, pat.PAT_ERR_TOO_LARGE
REFUSED = [
    (ops.pat_mx_quantize, quantize_args, [
        (dict(x=0), INVALID), (dict(x=BASE + 2), INVALID), (dict(x_stride=199), INVALID), (dict(x_stride=-200), INVALID),
        (dict(codes=BASE + 0x10008), INVALID), (dict(scales=BASE + 0x20002), INVALID), (dict(codes=BASE), INVALID),
        (dict(scales=BASE + 0x10000), INVALID), (dict(dtype="int32"), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED),
        (dict(rows=1 << 30, cols=1 << 10, x_stride=1 << 10), UNSUPPORTED), (dict(x_stride=1 << 62), INVALID)]),
    (ops.pat_mx_dequantize, lambda **kw: (lambda d: list({**d, **kw}.values()))(
        dict(codes=BASE, scales=BASE + 0x1000, rows=3, cols=200, out=BASE + 0x2000, out_stride=200, dtype="bfloat16")), [
        (dict(codes=0), INVALID), (dict(scales=0), INVALID), (dict(out=BASE + 0x2001), INVALID), (dict(out=BASE + 64), INVALID),
        (dict(out_stride=100), INVALID), (dict(dtype="int32"), UNSUPPORTED)]),
    (ops.pat_mx_matmul, matmul_args, [
        (dict(a_codes=0), INVALID), (dict(b_scales=0), INVALID), (dict(b_codes=BASE + 0x2004), INVALID), (dict(out=0), INVALID),
        (dict(out=BASE + 0x2000), INVALID), (dict(out_stride=4), INVALID), (dict(dtype="int32"), UNSUPPORTED),
        (dict(n=1 << 31), UNSUPPORTED), (dict(m=1 << 30, n=1 << 30, k=1), UNSUPPORTED)]),
    (ops.pat_mx_linear, linear_args, [
        (dict(x=0), INVALID), (dict(x_dtype="int32"), UNSUPPORTED), (dict(w_codes=0), INVALID), (dict(x_stride=100), INVALID),
        (dict(out=BASE + 0x4000), INVALID), (dict(out=BASE), INVALID), (dict(dtype="int32"), UNSUPPORTED)]),
    (ops.pat_mx_matmul_grad, grad_args, [
        (dict(g=0), INVALID), (dict(g=BASE + 1), INVALID), (dict(g_stride=4), INVALID), (dict(transposed=1, g_stride=2), INVALID),
        (dict(q_scales=0), INVALID), (dict(out=BASE + 0x2000), INVALID), (dict(dtype="int32"), UNSUPPORTED)]),
    (ops.pat_embedding, embedding_args, [
        (dict(tokens=0), INVALID), (dict(tokens=BASE + 2), INVALID), (dict(token_bytes=2), UNSUPPORTED),
        (dict(token_bytes=8, tokens=BASE + 4), INVALID), (dict(table=0), INVALID), (dict(table_dtype="int32"), UNSUPPORTED),
        (dict(out=BASE + 0x1000), INVALID), (dict(out_stride=1), INVALID), (dict(ntokens=1 << 31), UNSUPPORTED)]),
    (ops.pat_embedding_grad, embedding_grad_args, [
        (dict(tokens=0), INVALID), (dict(token_bytes=1), UNSUPPORTED), (dict(g=0), INVALID), (dict(out=BASE + 0x10000), INVALID),
        (dict(workspace=BASE + 0x1000000), INVALID), (dict(workspace=BASE + 0x10000), INVALID), (dict(workspace=0), INVALID),
        (dict(workspace=BASE + 0x2000008), INVALID), (dict(workspace_bytes=16), TOO_LARGE), (dict(g_dtype="int32"), UNSUPPORTED)]),
    (ops.pat_dropout, dropout_args, [
        (dict(p=-0.01), INVALID), (dict(p=1.01), INVALID), (dict(p=math.nan), INVALID), (dict(x=0), INVALID),
        (dict(out=BASE + 4), INVALID), (dict(out=BASE, out_stride=201), INVALID), (dict(out=BASE + 0x10004), INVALID),
        (dict(residual_stride=3), INVALID), (dict(dtype="int32"), UNSUPPORTED)]),
]


@pytest.mark.parametrize("call,args,change,status", [(c, a, d, s) for c, a, cases in REFUSED for d, s in cases],
                         ids=lambda v: getattr(v, "__name__", str(v)))
def test_bad_arguments_are_refused_before_any_device_call(call, args, change, status):
    assert call(*args(**change)) == status


LARGE_LINEAR = dict(m=60, x=BASE + 0x100000, out=BASE + 0x200000, workspace=BASE + 0x300000)
LARGE_GRAD = dict(rows=40, inner=8449, g=BASE + 0x1000000, g_stride=8449, q_codes=BASE + 0x2000000, q_scales=BASE + 0x3000000,
                  out=BASE + 0x4000000, workspace=BASE + 0x5000000)


@pytest.mark.parametrize("call,args,size,need", [
    (ops.pat_mx_linear, lambda **kw: linear_args(**{**LARGE_LINEAR, **kw}), LARGE_LINEAR, lambda: ops.pat_mx_linear_workspace(60, 5, 200)),
    (ops.pat_mx_matmul_grad, lambda **kw: grad_args(**{**LARGE_GRAD, **kw}), LARGE_GRAD,
     lambda: ops.pat_mx_matmul_grad_workspace(40, 8449, 200))], ids=["linear", "grad"])
def test_bad_workspaces_are_refused_before_any_device_call(call, args, size, need):
    """Too small, absent, misaligned, or over the output, an input, or a stored form."""
    need = need()
    assert need > 0
    assert call(*args(workspace_bytes=need - 1)) == TOO_LARGE and call(*args(workspace_bytes=0)) == TOO_LARGE
    stored = [size.get(name, BASE + place) for name, place in (("q_codes", 0x2000), ("q_scales", 0x4000))]
    for place in (0, size["workspace"] + 8, size["out"], size["out"] - need + 16, size.get("g", size.get("x")), *stored):
        assert call(*args(workspace=place, workspace_bytes=need)) == INVALID, hex(place)


def test_calls_without_elements_launch_nothing():
    none = dict(x=0, codes=0, scales=0)
    assert ops.pat_mx_quantize(*quantize_args(rows=0, **none)) == pat.PAT_OK
    assert ops.pat_mx_quantize(*quantize_args(cols=0, **none)) == pat.PAT_OK
    assert ops.pat_mx_matmul(*matmul_args(m=0, out=0)) == pat.PAT_OK
    assert ops.pat_mx_linear(*linear_args(n=0, out=0)) == pat.PAT_OK
    assert ops.pat_mx_matmul_grad(*grad_args(rows=0, out=0)) == pat.PAT_OK
    assert ops.pat_embedding(*embedding_args(ntokens=0, tokens=0, out=0)) == pat.PAT_OK
    assert ops.pat_embedding_grad(*embedding_grad_args(rows=0, out=0)) == pat.PAT_OK
    assert ops.pat_dropout(*dropout_args(rows=0, x=0, residual=0, out=0)) == pat.PAT_OK


def test_tensor_calls_refuse_what_the_kernels_do_not_take():
    x = torch.zeros(4, 8)
    for call in (lambda: ops.mx_quantize(x), lambda: ops.dropout(x, 0.1, 1), lambda: ops.embedding(torch.zeros(3).int(), x),
                 lambda: ops.embedding_grad(torch.zeros(4).int(), x, 5),
                 lambda: ops.mx_dequantize(ops.Mx(torch.zeros(2, 64).byte(), torch.zeros(2, 4).byte(), 8)),
                 lambda: ops.mx_linear(x, ops.Mx(torch.zeros(2, 64).byte(), torch.zeros(2, 4).byte(), 8))):
        with pytest.raises(ValueError):
            call()


# ---------------------------------------------------------------------------
# 4-bit blocks
# ---------------------------------------------------------------------------

SHAPES = [(1, 1), (1, 31), (2, 32), (3, 33), (5, 127), (4, 128), (7, 129), (1, 255), (33, 100), (16, 640), (3, 1111)]


@gpu
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 0), (9, 1)])
def test_quantize(rows, cols, dtype, pad, shift):
    x = values((rows, cols), rows * 1000 + cols, dtype)
    x.view(-1)[:: 7] = 0
    q = ops.mx_empty(rows, cols)
    q.codes.fill_(0xEE), q.scales.fill_(0xEE)
    ops.mx_quantize(strided(x, pad, shift) if pad else x, out=q)
    codes, scales = O.mx_pack(*O.mx_quantize(f64(x)))
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    for dtype_out in (F32, B16):
        out, untouched = guarded((rows, cols), dtype_out, pad, shift)
        assert np.array_equal(f64(ops.mx_dequantize(q, dtype_out, out)), O.mx_values(codes, scales, cols))
        assert untouched()


@gpu
@pytest.mark.parametrize("dtype", [F32, B16])
def test_quantize_edges(dtype):
    """Every tie, both clamps, subnormals, the largest values, infinities, NaN, negative zero, a block of zeros."""
    x = torch.zeros((12, 96), dtype=torch.float64)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.875], dtype=torch.float64)
    for r, e in enumerate((0, -100, 100, -126, -124, 120)):
        x[r, :9], x[r, 9:18] = ties * 2.0**e, -ties * 2.0**e
        x[r, 32:50] = x[r, :18] * 0.5
    x[6, 0], x[6, 1], x[6, 64] = 2.0**-133, -0.0, -0.0
    x[7, 3], x[7, 40] = float("inf"), float("-inf")
    x[8, 31], x[8, 95] = float("nan"), 1.0
    big = 3.3895313892515355e38  # the largest bfloat16
    x[9, 0], x[9, 1], x[9, 2], x[9, 33] = big, -big, 1e38, big / 3
    x[10, :32] = 2.0**-126
    x[11, 0], x[11, 1] = 1.0, 1e-30
    x = x.to(dtype).cuda()
    q = ops.mx_quantize(x)
    codes, scales = O.mx_pack(*O.mx_quantize(f64(x)))
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    for dtype_out in (F32, B16):
        assert np.array_equal(f64(ops.mx_dequantize(q, dtype_out)), O.mx_values(codes, scales, 96), equal_nan=True)


@gpu
def test_dequantize_every_code_and_scale():
    codes = np.tile(np.arange(16), (256, 8))
    scales = np.tile(np.arange(256)[:, None], (1, 4))
    c, s = O.mx_pack(codes, scales)
    q = ops.Mx(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), 128)
    want = O.mx_values(c, s, 128)
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)  # 4 and 6 times 2^127 and 2^126 * 4 are infinite
    for dtype in (F32, B16):
        assert np.array_equal(f64(ops.mx_dequantize(q, dtype)), want, equal_nan=True)


PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 300, 128), (2, 17, 129), (3, 33, 500), (16, 16, 512), (17, 100, 640), (24, 70, 1001),
            (40, 65, 300), (64, 64, 256), (65, 130, 96), (100, 129, 777), (128, 128, 1024), (130, 257, 384), (256, 256, 512),
            (300, 270, 1300), (520, 260, 130), (5, 2000, 64), (2000, 3, 200), (1, 64, 20000), (48, 40, 8200),
            (3, 8000, 40), (20, 4200, 300), (40, 8300, 130), (49, 49, 500), (1500, 1500, 250), (2900, 2900, 140), (60, 100, 7)]


@gpu
@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", [F32, B16])
def test_matmul(m, n, k, dtype):
    a, va = random_mx(m, k, m + n)
    b, vb = random_mx(n, k, n + k)
    out, untouched = guarded((m, n), dtype, pad=n % 3, shift=k % 2)
    ops.mx_matmul(a, b, dtype, out)
    assert untouched()
    within(out, va @ vb.T, np.abs(va) @ np.abs(vb).T, k, dtype)


@gpu
@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (B16, B16), (B16, F32)])
def test_linear(m, n, k, dtype, out_dtype):
    """Against the plain form, and to the bit against quantising first."""
    x = values((m, k), m * n + k, dtype)
    w, vw = random_mx(n, k, k + n)
    vx = O.mx_values(*O.mx_pack(*O.mx_quantize(f64(x))), k)
    for view in (x, strided(x, 5, 1)):
        out, untouched = guarded((m, n), out_dtype)
        ops.mx_linear(view, w, out_dtype, out)
        assert untouched()
        within(out, vx @ vw.T, np.abs(vx) @ np.abs(vw).T, k, out_dtype)
        assert torch.equal(out, ops.mx_matmul(ops.mx_quantize(view), w, out_dtype))


@gpu
@pytest.mark.parametrize("m,n", [(1500, 1501), (2900, 2899)])  # tiles of 128 and of 256
@pytest.mark.parametrize("k", [1030, 1160, 1290, 1420, 2430])  # 9, 10, 11, 12 and 19 groups: every rest of the loop by four
@pytest.mark.parametrize("dtype", [F32, B16])
def test_matmul_goes_through_many_columns_of_large_tiles(m, n, k, dtype):
    """The reference in 64 bits by the GPU's library.  Twice: a race would hardly give the same bits."""
    a, va = random_mx(m, k, m + k)
    b, vb = random_mx(n, k, n + k)
    out, untouched = guarded((m, n), dtype, pad=1)
    ops.mx_matmul(a, b, dtype, out)
    assert untouched()
    ta, tb = torch.from_numpy(va).cuda(), torch.from_numpy(vb).cuda().t().contiguous()
    within(out, f64(torch.mm(ta, tb)), f64(torch.mm(ta.abs(), tb.abs())), k, dtype)
    assert torch.equal(out, ops.mx_matmul(a, b, dtype))


@gpu
@pytest.mark.parametrize("m,n,k", [(3, 20, 0), (300, 300, 0)])
def test_products_of_no_columns_are_zero(m, n, k):
    a, b = ops.mx_empty(m, k), ops.mx_empty(n, k)
    out = torch.full((m, n), 5.0, device="cuda")
    assert bool((ops.mx_matmul(a, b, F32, out) == 0).all())
    out.fill_(5.0)
    assert bool((ops.mx_linear(torch.empty((m, k), device="cuda"), b, F32, out) == 0).all())
    out = torch.full((m, 40), 5.0, device="cuda")  # a gradient of no rows
    empty = torch.empty((m, 0), dtype=B16, device="cuda")
    assert bool((ops.mx_matmul_grad(empty, ops.mx_empty(0, 40), F32, out=out) == 0).all())


@gpu
def test_product_of_no_columns_and_many_values_is_zero():
    """2^35 values, of more tiles of any size than one launch holds."""
    m = n = 1 << 17
    out = torch.full((2 * m, n), 5.0, dtype=B16, device="cuda")
    ops.mx_matmul(ops.mx_empty(2 * m, 0), ops.mx_empty(n, 0), B16, out)
    assert not any(bool(part.any()) for part in out.split(8192))


@gpu
@pytest.mark.parametrize("m,n,k", [(2, 40, 256), (70, 40, 300), (300, 300, 256)])
def test_products_carry_what_is_not_finite(m, n, k):
    """A NaN block makes its row's products NaN and no other; values too large for the sum give infinities."""
    x = values((m, k), 5, F32)
    x[1, 7] = float("inf")
    w, vw = random_mx(n, k, 6)
    got = f64(ops.mx_linear(x, w, F32))
    assert np.isnan(got[1]).all() and np.isfinite(np.delete(got, 1, axis=0)).all()
    a, _ = random_mx(m, k, 7, 250, 253)
    b, _ = random_mx(n, k, 8, 250, 253)
    assert not np.isfinite(f64(ops.mx_matmul(a, b, F32))).any()
    w.scales[3, 1] = 255
    got = f64(ops.mx_matmul_grad(torch.ones((m, n), dtype=B16, device="cuda"), w, F32))
    assert np.isnan(got[:, 32:64]).all() and np.isfinite(got[:, :32]).all() and np.isfinite(got[:, 64:]).all()


GRADS = [(1, 1, 1), (1, 16, 32), (3, 40, 33), (16, 32, 128), (33, 65, 100), (64, 64, 64), (70, 129, 257), (128, 128, 128),
         (130, 70, 300), (256, 128, 256), (300, 200, 520), (20, 3000, 40), (257, 1000, 129), (1000, 5, 130), (64, 31, 640), (100, 4096, 90), (64, 5761, 33), (40, 8449, 200), (130, 8, 64),
         (9, 7, 300), (7, 500, 40), (520, 700, 600), (1500, 330, 1490), (1537, 70, 1501), (2901, 390, 2900), (2896, 261, 2950)]


@gpu
@pytest.mark.parametrize("rows,inner,cols", GRADS)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", [F32, B16])
def test_matmul_grad(rows, inner, cols, transposed, dtype):
    g = values((inner, rows) if transposed else (rows, inner), rows + inner, B16)
    q, vq = random_mx(inner, cols, cols)
    vg = f64(g).T if transposed else f64(g)
    for view in (g, strided(g, 3, 1)):
        out, untouched = guarded((rows, cols), dtype)
        ops.mx_matmul_grad(view, q, dtype, transposed, out)
        assert untouched()
        within(out, vg @ vq, np.abs(vg) @ np.abs(vq), inner, dtype)


@gpu
@pytest.mark.parametrize("rows,cols", [(131075, 131072), (40001, 40003)])
def test_matmul_grad_of_more_tiles_than_workgroups(rows, cols):
    """Outer products, the first of more 16 x 16 tiles than one launch holds (2^34 values and more): each value is
    one product, exact in float32 and rounded once."""
    g = values((1, rows), 1, B16)
    q, vq = random_mx(1, cols, 2)
    row = torch.from_numpy(vq[0]).float().cuda()
    out = torch.full((rows, cols), 5.0, dtype=B16, device="cuda")
    ops.mx_matmul_grad(g, q, B16, True, out)
    for r0 in range(0, rows, 4096):
        part = slice(r0, min(r0 + 4096, rows))
        assert torch.equal(out[part], (g[0, part, None].float() * row).to(B16)), r0


@gpu
def test_matmul_gradients_against_differences():
    """The product is linear in each value of its factors, so a changed code changes sum(g * out) by the change
    times that value's gradient, up to the sums' rounding."""
    m, n, k = 24, 40, 130
    a, va = random_mx(m, k, 1, 120, 130)
    b, vb = random_mx(n, k, 2, 120, 130)
    g = values((m, n), 3, B16)
    vg, base = f64(g), f64(ops.mx_matmul(a, b, F32))
    da, db = f64(ops.mx_matmul_grad(g, b, F32)), f64(ops.mx_matmul_grad(g, a, F32, transposed=True))
    for q, v, grad, first in ((a, va, da, True), (b, vb, db, False)):
        for r, c in ((0, 0), (5, 31), (11, 77), (23, 129)):
            moved = ops.Mx(q.codes.clone(), q.scales, k)
            moved.codes[r, c // 2] ^= 1 << (4 * (c % 2) + 2)
            step = O.mx_values(moved.codes.cpu().numpy(), q.scales.cpu().numpy(), k)[r, c] - v[r, c]
            after = f64(ops.mx_matmul(moved, b, F32) if first else ops.mx_matmul(a, moved, F32))
            size = np.abs(vg) * (np.abs(va) @ np.abs(vb).T + np.abs(after))
            assert abs(np.sum(vg * (after - base)) - step * grad[r, c]) <= 8 * (k + n + m) * U * np.sum(size)


# ---------------------------------------------------------------------------
# Embedding
# ---------------------------------------------------------------------------


@gpu
@pytest.mark.parametrize("ntokens,rows,cols,first", [(1, 1, 1, 0), (3, 10, 8, 0), (100, 7, 33, 5), (65, 300, 129, 100),
                                                     (17, 50, 1000, 0), (5, 3, 2050, 1), (1000, 4, 5, -2)])
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (B16, B16), (B16, F32), (F32, B16)])
@pytest.mark.parametrize("wide", [False, True])
def test_embedding(ntokens, rows, cols, first, dtype, out_dtype, wide):
    """Tokens below, inside and above the table's rows."""
    tokens = np.random.default_rng(ntokens).integers(first - rows, first + 2 * rows, size=ntokens)
    if wide and ntokens > 2:
        tokens[0], tokens[1], tokens[2] = -2**63, 2**63 - 1, 2**32 + first  # and not their low 32 bits
    t = torch.from_numpy(tokens).to(torch.int64 if wide else torch.int32).cuda()
    table = values((rows, cols), rows, dtype)
    want = O.embedding(tokens, f64(table), 1.75, first)
    for view in (table, strided(table, 2, 1)):
        out, untouched = guarded((ntokens, cols), out_dtype)
        ops.embedding(t, view, 1.75, first, out_dtype, out)
        assert untouched()
        within(out, want, 0.0, 0, out_dtype)


@gpu
@pytest.mark.parametrize("ntokens,rows,cols", [(2051, 37, 1031), (2047, 9, 4100), (66001, 300, 40), (524001, 50, 5)])
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (B16, B16), (B16, F32), (F32, B16)])
def test_embedding_of_many_tokens(ntokens, rows, cols, dtype, out_dtype):
    """Two tokens a lane in turn; a workgroup's last ones may not exist, a third of all is outside the table."""
    tokens = np.random.default_rng(ntokens).integers(3 - rows, 3 + 2 * rows, size=ntokens)
    table = values((rows, cols), rows, dtype)
    inside = (tokens >= 3) & (tokens < 3 + rows)
    want = np.where(inside[:, None], 1.75 * f64(table)[np.where(inside, tokens - 3, 0)], 0.0)
    for token_dtype, view in ((torch.int32, table), (torch.int64, strided(table, 2, 1))):
        out, untouched = guarded((ntokens, cols), out_dtype)
        ops.embedding(torch.from_numpy(tokens).to(token_dtype).cuda(), view, 1.75, 3, out_dtype, out)
        assert untouched()
        within(out, want, 0.0, 0, out_dtype)


@gpu
def test_embedding_in_a_table_without_rows():
    out = torch.full((9, 40), 5.0, device="cuda")
    ops.embedding(torch.arange(9, device="cuda"), torch.empty((0, 40), device="cuda"), dtype=F32, out=out)
    assert bool((out == 0).all())


def token_sets():
    g = np.random.default_rng(9)
    yield "one", np.array([3]), 10, 0
    yield "all the same", np.full(700, 4), 9, 0
    yield "none inside", np.arange(50) + 100, 20, 0
    yield "each once, falling", np.arange(300)[::-1].copy(), 300, 0
    yield "one row", g.integers(-1, 2, size=200), 1, 0
    yield "shard", g.integers(0, 1000, size=3000), 250, 500
    yield "frequent and rare", np.minimum(np.exp(g.random(5000) * 8).astype(np.int64), 1999), 2000, 0
    yield "more rows than one pass sorts", g.integers(0, 5000, size=2500), 5000, 0
    yield "few, and a frequent row", np.where(g.random(1024) < 0.7, 3, g.integers(0, 400, size=1024)), 400, 0
    yield "few, and two frequent rows", np.where(g.random(1000) < 0.8, 9 + 4 * g.integers(0, 2, 1000), 1), 70, 0
    yield "few, of many rows", g.integers(0, 30000, size=600), 30000, 0
    yield "many, all the same", np.full(6000, 4), 9, 0
    yield "many, none inside", np.arange(5000) + 100, 20, 0
    yield "many, each once, falling", np.arange(4500)[::-1].copy(), 4500, 0
    yield "many, one row", g.integers(-1, 2, size=4097), 1, 0
    yield "many, shard", g.integers(0, 2000, size=7000), 250, 500
    yield "two passes and a frequent row", np.where(g.random(9000) < 0.4, 4000, g.integers(0, 70000, size=9000)), 70000, 0


@gpu
@pytest.mark.parametrize("name,tokens,rows,first", list(token_sets()), ids=lambda v: v if isinstance(v, str) else "")
@pytest.mark.parametrize("cols,dtype,out_dtype", [(1, F32, F32), (33, F32, F32), (16, B16, F32), (40, B16, B16), (24, F32, B16)])
def test_embedding_grad(name, tokens, rows, first, cols, dtype, out_dtype):
    g = values((len(tokens), cols), rows + cols, dtype)
    inside = tokens[(tokens >= first) & (tokens < first + rows)]
    terms = np.bincount(inside - first, minlength=rows).max() if len(inside) else 0
    want = O.embedding_grad(tokens, f64(g), rows, 0.5, first)
    size = O.embedding_grad(tokens, np.abs(f64(g)), rows, 0.5, first)
    first_out = None
    for token_dtype, view in ((torch.int32, g), (torch.int64, strided(g, 3, 1))):
        out, untouched = guarded((rows, cols), out_dtype)
        ops.embedding_grad(torch.from_numpy(tokens).to(token_dtype).cuda(), view, rows, 0.5, first, out_dtype, out)
        assert untouched()
        within(out, want, size, terms, out_dtype)
        if first_out is None:
            first_out = out.clone()
        assert torch.equal(first_out, out)  # to the bit, whatever ran beside it


@gpu
@pytest.mark.parametrize("ntokens,cols", [(0, 5), (2000, 2100), (20, 4100), (600, 1500)])
def test_embedding_grad_of_wide_rows_and_none(ntokens, cols):
    tokens = np.random.default_rng(3).integers(0, 40, size=ntokens)
    tokens[: ntokens // 2] = 7
    g = values((ntokens, cols), 4, B16)
    out = ops.embedding_grad(torch.from_numpy(tokens).cuda(), g, 41, dtype=F32)
    within(out, O.embedding_grad(tokens, f64(g), 41, 1.0, 0), O.embedding_grad(tokens, np.abs(f64(g)), 41, 1.0, 0), ntokens,
           F32)


@gpu
@pytest.mark.parametrize("ntokens,rows,cols,share", [
    (9001, 500, 1030, 0.3),         # whole waves a piece, sorted by several workgroups; pieces of 16 entries
    (70001, 3000, 1031, 0.4),       # pieces of 32
    (140001, 3000, 1030, 0.5),      # pieces of 64, sorting workgroups of more than 1024 entries
    (140001, 1, 260, 0.0),          # one row of all
    (30001, 70000, 2057, 0.2),      # two column parts, most rows without an entry
    (150001, 1100000, 5, 0.1),      # three sorting passes
])
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (B16, F32), (B16, B16)])
def test_embedding_grad_of_many_tokens(ntokens, rows, cols, share, dtype, out_dtype):
    """A frequent row (`share` of the tokens), rare ones, some outside; the sums in 64 bits on the GPU."""
    r = np.random.default_rng(ntokens + cols)
    tokens = np.where(r.random(ntokens) < share, rows // 3, r.integers(-rows // 8 - 1, rows + rows // 8 + 1, size=ntokens))
    t = torch.from_numpy(tokens).cuda()
    g = torch.randn((ntokens, cols), device="cuda", generator=torch.Generator("cuda").manual_seed(ntokens)).to(dtype)
    inside = ((t >= 0) & (t < rows)).nonzero()[:, 0]
    terms = int(torch.bincount(t[inside]).max())
    want, size = (torch.zeros((rows, cols), dtype=torch.float64, device="cuda") for _ in range(2))
    for part in inside.split(20000):
        want.index_add_(0, t[part], 0.5 * g[part].double())
        size.index_add_(0, t[part], 0.5 * g[part].double().abs())
    out, untouched = guarded((rows, cols), out_dtype)
    ops.embedding_grad(t, g, rows, 0.5, 0, out_dtype, out)
    assert untouched()
    bound = 2 * (terms + 2) * U * size + (E if out_dtype == B16 else 2 * U) * want.abs() + 1e-300  # as within()
    assert bool(((out.double() - want).abs() <= bound).all())
    wide = strided(g, 3, 1)
    assert torch.equal(ops.embedding_grad(t.int(), wide, rows, 0.5, 0, out_dtype), out)


@gpu
def test_embedding_gradient_against_differences():
    """sum(g * out) is linear in the table."""
    tokens = torch.tensor([4, 1, 4, 9, 0, 4], dtype=torch.int32, device="cuda")
    table, g = values((8, 20), 1), values((6, 20), 2)
    grad = f64(ops.embedding_grad(tokens, g, 8, 3.0))
    base = f64(ops.embedding(tokens, table, 3.0))
    for r, c in ((4, 3), (1, 19), (0, 0), (7, 5)):
        moved = table.clone()
        moved[r, c] += 0.5
        step = float(moved[r, c].double() - table[r, c].double())
        after = f64(ops.embedding(tokens, moved, 3.0))
        size = np.sum(np.abs(f64(g)) * (np.abs(base) + np.abs(after)))
        assert abs(np.sum(f64(g) * (after - base)) - step * grad[r, c]) <= 8 * U * size


# ---------------------------------------------------------------------------
# Dropout
# ---------------------------------------------------------------------------


@gpu
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (1, 64), (3, 8), (5, 333), (64, 31), (9, 2100)])
@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("index,index_stride", [(0, None), (5, None), (8, 4096), (3, 4099), (2**35 + 1, 2**33 + 3),
                                                (2**64 - 9, 17)])
def test_dropout(rows, cols, dtype, index, index_stride):
    x, res = values((rows, cols), rows, dtype), values((rows, cols), cols, dtype)
    seed = 2**63 + 12345 + rows
    keep, factor = O.dropout_keep(rows, cols, 0.3, seed, index, cols if index_stride is None else index_stride)
    want = np.where(keep, f64(x) * factor, 0.0)
    for a, r in ((x, None), (strided(x, 3, 1), None), (x, res), (strided(x, 1), strided(res, 2, 1))):
        out, untouched = guarded((rows, cols), dtype)
        ops.dropout(a, 0.3, seed, index, index_stride, r, out)
        assert untouched()
        full = want if r is None else want + f64(res)
        within(out, full, np.abs(want) + (0 if r is None else np.abs(f64(res))), 0, dtype)
        if r is None:
            assert np.array_equal(f64(out) == 0, ~keep | (f64(x) == 0))


@gpu
@pytest.mark.parametrize("dtype", [F32, B16])
def test_dropout_shards_have_the_masks_of_the_whole(dtype):
    """Rows, columns and both: each shard's call gives its part of the whole's result, to the bit."""
    x = values((24, 100), 7, dtype)
    whole = ops.dropout(x, 0.4, 99, index=1000)
    for r0, r1, c0, c1 in ((0, 12, 0, 100), (12, 24, 0, 100), (0, 24, 33, 67), (5, 6, 99, 100), (7, 23, 8, 80)):
        part = ops.dropout(x[r0:r1, c0:c1], 0.4, 99, index=1000 + 100 * r0 + c0, index_stride=100)
        assert torch.equal(part, whole[r0:r1, c0:c1])


@gpu
@pytest.mark.parametrize("dtype", [F32, B16])
def test_dropout_ends_and_in_place(dtype):
    x, res = values((20, 77), 1, dtype), values((20, 77), 2, dtype)
    assert torch.equal(ops.dropout(x, 0.0, 5), x)
    assert bool((ops.dropout(x, 1.0, 5) == 0).all())
    assert torch.equal(ops.dropout(x, 1.0, 5, residual=res), res)
    want, want_res = ops.dropout(x, 0.5, 5), ops.dropout(x, 0.5, 5, residual=res)
    y, z = x.clone(), res.clone()
    assert torch.equal(ops.dropout(y, 0.5, 5, out=y), want)
    assert torch.equal(ops.dropout(x, 0.5, 5, residual=z, out=z), want_res)
    bad = x.clone()
    bad[:, ::2] = float("nan")
    bad[:, 1::2] = float("inf")
    assert torch.equal(torch.isfinite(ops.dropout(bad, 0.5, 5)), want == 0)
    # the share that is dropped: 1000 x 1000 elements, six standard deviations
    y = ops.dropout(torch.ones((1000, 1000), dtype=dtype, device="cuda"), 0.1, 6)
    assert abs(float((y == 0).double().mean()) - 6554 / 65536) < 6 * math.sqrt(0.1 * 0.9 / 1e6)


@gpu
def test_dropout_gradient_against_differences():
    x, g = values((6, 40), 1), values((6, 40), 2)
    grad, base = f64(ops.dropout(g, 0.25, 11)), f64(ops.dropout(x, 0.25, 11))
    for r, c in ((0, 0), (3, 17), (5, 39), (2, 8)):
        moved = x.clone()
        moved[r, c] += 2.0
        step = float(moved[r, c].double() - x[r, c].double())
        after = f64(ops.dropout(moved, 0.25, 11))
        size = np.sum(np.abs(f64(g)) * (np.abs(base) + np.abs(after)))
        assert abs(np.sum(f64(g) * (after - base)) - step * grad[r, c]) <= 8 * U * size


# ---------------------------------------------------------------------------
# Streams, graphs, large offsets
# ---------------------------------------------------------------------------


def every_operator():
    """Calls of each operator on inputs of their own: name, call, expected result from a first call."""
    x, w = values((20, 300), 1, B16), values((70, 300), 2)
    g, tokens = values((20, 70), 3, B16), torch.arange(20, device="cuda") * 7 % 13
    q = ops.mx_quantize(w)
    xq = ops.mx_quantize(x)
    return {
        "quantize": lambda out: ops.mx_quantize(w, out=out), "dequantize": lambda out: ops.mx_dequantize(q, F32, out),
        "matmul": lambda out: ops.mx_matmul(xq, q, F32, out), "linear": lambda out: ops.mx_linear(x, q, F32, out),
        "grad": lambda out: ops.mx_matmul_grad(g, q, F32, out=out),
        "grad_t": lambda out: ops.mx_matmul_grad(g, xq, F32, True, out),
        "embedding": lambda out: ops.embedding(tokens, w, 2.0, dtype=F32, out=out),
        "embedding_grad": lambda out: ops.embedding_grad(tokens, x, 13, dtype=F32, out=out),
        "dropout": lambda out: ops.dropout(w, 0.2, 3, out=out),
    }


@gpu
@pytest.mark.parametrize("name", ["quantize", "dequantize", "matmul", "linear", "grad", "grad_t", "embedding",
                                  "embedding_grad", "dropout"])
def test_graph_replays_and_other_streams(name):
    """Captured once and replayed with eager work between: every replay gives the eager result."""
    call = every_operator()[name]
    want = call(None)
    parts = want[:2] if name == "quantize" else (want,)
    out = ops.Mx(*(torch.zeros_like(p) for p in parts), want.cols) if name == "quantize" else torch.zeros_like(want)
    got = out[:2] if name == "quantize" else (out,)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, parts))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for _ in range(4):
        for p in got:
            p.zero_()
        graph.replay()
        call(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, parts))


@gpu
@pytest.mark.parametrize("name", ["quantize", "dequantize", "linear", "grad", "embedding_grad", "dropout"])
def test_memory_of_a_call_on_another_stream(name):
    """Outputs and workspaces of a call on a given stream are not memory that work queued on the current stream still
    writes: a tensor that a delayed fill goes to is freed before the call."""
    x, w = values((20, 300), 1, B16), values((70, 300), 2)
    g, tokens, q = values((20, 70), 3, B16), torch.arange(20, device="cuda") * 7 % 13, ops.mx_quantize(w)
    call = {"quantize": lambda s: ops.mx_quantize(w, stream=s).codes, "dequantize": lambda s: ops.mx_dequantize(q, F32, stream=s),
            "linear": lambda s: ops.mx_linear(x, q, F32, stream=s),
            "grad": lambda s: ops.mx_matmul_grad(g, q, F32, stream=s),
            "embedding_grad": lambda s: ops.embedding_grad(tokens, x, 13, dtype=F32, stream=s),
            "dropout": lambda s: ops.dropout(w, 0.2, 3, stream=s)}[name]
    want, side = call(None), torch.cuda.Stream()
    torch.cuda.synchronize()
    for handle in (side, side.cuda_stream):
        torch.cuda._sleep(20_000_000)
        late = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (512, 4480, 6000, 15600, 24000, 84000, 200000)]
        for t in late:
            t.fill_(0x77)
        del late, t
        got = call(handle)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def with_workspaces():
    """Calls that need memory between their launches: name -> (call of an output and a stream, bytes of workspace)."""
    x, w = values((60, 300), 1, B16), values((70, 300), 2)
    q = ops.mx_quantize(w)
    g, tall = values((40, 8449), 3, B16), ops.mx_quantize(values((8449, 200), 4))
    by_terms = g.t().contiguous()
    rows = {n: (values((n, 24), n, B16), torch.from_numpy(np.random.default_rng(n).integers(-3, 300, size=n) // 2).cuda())
            for n in (2000, 6000)}
    return {
        "linear": (lambda out, s=None: ops.mx_linear(x, q, F32, out, s), ops.pat_mx_linear_workspace(60, 70, 300)),
        "grad": (lambda out, s=None: ops.mx_matmul_grad(g, tall, F32, False, out, s),
                 ops.pat_mx_matmul_grad_workspace(40, 8449, 200)),
        "grad_t": (lambda out, s=None: ops.mx_matmul_grad(by_terms, tall, F32, True, out, s),
                   ops.pat_mx_matmul_grad_workspace(40, 8449, 200)),
        **{f"embedding_grad_{n}": (lambda out, s=None, n=n: ops.embedding_grad(rows[n][1], rows[n][0], 140, dtype=F32, out=out, stream=s),
                                   ops.pat_embedding_grad_workspace(n, 140, 24)) for n in rows},
    }


WITH_WORKSPACES = ["linear", "grad", "grad_t", "embedding_grad_2000", "embedding_grad_6000"]


@gpu
@pytest.mark.parametrize("name", WITH_WORKSPACES)
def test_graph_replays_of_calls_with_workspaces(name):
    call, need = with_workspaces()[name]
    assert need > 0
    want = call(None)
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for _ in range(4):
        out.zero_()
        junk = torch.full((max(need, 1 << 20),), 0x77, dtype=torch.uint8, device="cuda")  # the pool's memory is not the graph's
        graph.replay()
        assert torch.equal(call(None), want)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and bool((junk == 0x77).all())


@gpu
@pytest.mark.parametrize("name", WITH_WORKSPACES)
def test_workspaces_belong_to_the_stream_of_the_call(name, monkeypatch):
    """Output and workspace of a call on a given stream are that stream's memory, and the result is right while the current
    stream writes over blocks of the same sizes that it has just freed."""
    call, need = with_workspaces()[name]
    assert need > 0
    want, side, held = call(None), torch.cuda.Stream(), []
    take = ops._work

    def work(*args):
        address, tensor = take(*args)
        held.append((address, tensor.numel()))
        return address, tensor

    monkeypatch.setattr(ops, "_work", work)
    torch.cuda.synchronize()
    for handle in (side, side.cuda_stream):
        for _ in range(20):
            late = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in 2 * (need, want.numel() * 4)]
            for t in late:
                t.fill_(0x77)
            del late, t
            got = call(None, handle)
            side.synchronize()
            assert torch.equal(got, want)
        torch.cuda.synchronize()
        segments = torch.cuda.memory_snapshot()

        def stream_of(address):
            return [s["stream"] for s in segments if s["address"] <= address < s["address"] + s["total_size"]]

        assert len(held) == 20 and all(size == need and stream_of(at) == [side.cuda_stream] for at, size in held)
        assert stream_of(got.data_ptr()) == [side.cuda_stream]
        held.clear()


@gpu
@pytest.mark.parametrize("name", ["quantize", "dequantize", "embedding", "embedding_grad", "dropout"])
def test_more_work_than_a_launch_has_workgroups(name):
    """Workgroups that go round several times: every part of a large result is that of a small call on the same values."""
    parts = 4099  # of 4096 rows each, the last one short
    if name in ("quantize", "dequantize"):  # more than 2^26 groups of 128 values
        x = values((4096, 600), 1, B16)
        q = ops.mx_quantize(x)
        if name == "quantize":
            got = ops.mx_quantize(x.repeat(parts, 1)[:-5])
            wanted = q[:2]
        else:
            got = (ops.mx_dequantize(ops.Mx(q.codes.repeat(parts, 1)[:-5], q.scales.repeat(parts, 1)[:-5], 600), B16),)
            wanted = (ops.mx_dequantize(q, B16),)
        assert got[0].shape[0] * 5 > 1 << 26
        for big, small in zip(got, wanted):
            assert all(torch.equal(part, small[:len(part)]) for part in big.split(4096))
    elif name == "embedding":  # two tokens a lane, 256 lanes, 2^20 workgroups
        n, table = (1 << 29) + 70001, values((1 << 20, 2), 2, B16)
        tokens = torch.randint(-9, 1 << 20, (n,), dtype=torch.int32, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        out = torch.full((n, 2), 5.0, dtype=B16, device="cuda")
        ops.embedding(tokens, table, out=out)
        for r0 in range(0, n, 1 << 24):
            t = tokens[r0:r0 + (1 << 24)].long()
            assert torch.equal(out[r0:r0 + (1 << 24)], torch.where((t >= 0)[:, None], table[t.clamp_min(0)], 0.0)), r0
    elif name == "embedding_grad":  # 128 rows a workgroup
        rows, n = (1 << 27) + 9001, 1000
        tokens = torch.randint(0, rows, (n,), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
        tokens[1:5], tokens[5] = tokens[0], rows - 1
        g = torch.randint(-8, 9, (n, 3), device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(F32)  # exact sums
        out = torch.full((rows, 3), 5.0, dtype=F32, device="cuda")
        ops.embedding_grad(tokens, g, rows, out=out)
        assert torch.equal(out, torch.zeros((rows, 3), device="cuda").index_add_(0, tokens, g))
    else:  # one lane and one element a row
        rows = (1 << 30) + 5001
        x = torch.ones((rows, 1), dtype=B16, device="cuda")
        out = ops.dropout(x, 0.25, 3, index=2**64 - 77, index_stride=3)
        assert abs(float((out[:1 << 26] == 0).double().mean()) - 0.25) < 6 * math.sqrt(0.25 * 0.75 / 2**26)
        for r0 in (0, 1 << 29, (1 << 30) - 100, 1 << 30, rows - 3000):
            part = x[r0:r0 + 3000]
            assert torch.equal(out[r0:r0 + 3000], ops.dropout(part, 0.25, 3, index=3 * r0 - 77, index_stride=3))


@gpu
def test_offsets_beyond_32_bits():
    """Tables, gradients and outputs whose byte and element offsets pass 2^32: rows spread over 10 GiB."""
    pitch, rows, cols = 1 << 30, 5, 40
    room = torch.zeros((rows, pitch), dtype=B16, device="cuda")
    table = room[:, :cols]
    small = values((rows, cols), 1, B16)
    table.copy_(small)
    tokens = torch.tensor([4, 0, 3, 4, 1], dtype=torch.int32, device="cuda")
    assert torch.equal(ops.embedding(tokens, table, 2.0), ops.embedding(tokens, small, 2.0))
    assert torch.equal(ops.embedding_grad(tokens, table, 5, dtype=F32), ops.embedding_grad(tokens, small, 5, dtype=F32))
    assert torch.equal(ops.dropout(table, 0.5, 1), ops.dropout(small, 0.5, 1))
    q, want = ops.mx_quantize(table), ops.mx_quantize(small)
    assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
    assert torch.equal(ops.mx_linear(table, want, F32), ops.mx_linear(small, want, F32))
    g, q = values((rows, 8), 2, B16), ops.mx_quantize(values((8, cols), 3))
    far = room[:, 64:72]
    far.copy_(g)
    assert torch.equal(ops.mx_matmul_grad(far, q, F32), ops.mx_matmul_grad(g, q, F32))
    out = room[:, 128:128 + cols]
    assert torch.equal(ops.mx_dequantize(want, B16, out), ops.mx_dequantize(want, B16))
    assert torch.equal(ops.mx_matmul_grad(g, q, B16, out=out), ops.mx_matmul_grad(g, q, B16))
    assert torch.equal(ops.embedding(tokens, small, 2.0, out=out), ops.embedding(tokens, small, 2.0))
    assert bool((room[:, cols:64] == 0).all()) and bool((room[:, 200:4096] == 0).all())


@gpu
@pytest.mark.parametrize("dtype", [F32, B16])
def test_input_and_output_in_columns_of_one_buffer(dtype):
    """Whatever stands in the columns beside an output is read as it was and left so."""
    x, tokens = values((40, 96), 1, dtype), torch.arange(40, device="cuda") * 7 % 40
    q = ops.mx_quantize(values((70, 96), 3))
    calls = {"dropout": lambda a, out: ops.dropout(a, 0.3, 5, out=out),
             "residual": lambda a, out: ops.dropout(x, 0.3, 5, residual=a, out=out),
             "embedding": lambda a, out: ops.embedding(tokens, a, 2.0, out=out),
             "embedding_grad": lambda a, out: ops.embedding_grad(tokens, a, 40, 2.0, out=out)}
    if dtype == B16:
        calls["grad"] = lambda a, out: ops.mx_matmul_grad(a, ops.mx_quantize(values((96, 96), 4)), out=out)
    calls["linear"] = lambda a, out: ops.mx_linear(a, q, out=out)
    for name, call in calls.items():
        want = call(x, None)
        for left, right in ((0, 0), (3, 5)):
            for first in (False, True):
                room = torch.full((40, 96 + want.shape[1] + left + right), -77.0, dtype=dtype, device="cuda")
                at = left if first else left + want.shape[1]
                to = left + 96 if first else left
                a, out = room[:, at:at + 96], room[:, to:to + want.shape[1]]
                a.copy_(x)
                call(a, out)
                assert torch.equal(out, want) and torch.equal(a, x), name
                assert bool((room[:, :left] == -77.0).all()) and bool((room[:, left + 96 + want.shape[1]:] == -77.0).all()), name


# ---- the operators together, between the collectives

def example():
    spec = importlib.util.spec_from_file_location("sharded_step", os.path.join(ROOT, "examples", "sharded_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.gpu
@pytest.mark.parametrize("ranks", [1, 2, 4])
def test_sharded_step(ranks):
    """One step's loss and weights against the definitions, for the whole batch at once.

    The embedding's scale (16) and the dropout's factor (2) are powers of two, so everything up to the 4-bit rows of
    the layer's input is exact; after it the bounds follow each rounding: 32-bit sums of k or fewer terms, the
    gradient's rounding to bfloat16 before the products and after the one for the input."""
    vocabulary, width, outputs, batch, p, rate = 64, 256, 96, 128, 0.5, 2.0
    step = example()
    start = step.problem(vocabulary, width, outputs, batch)
    losses, layer, table = step.train(ranks, 1, *start, p=p, rate=rate)

    w, e, tokens, targets = f64(start[0]), f64(start[1].bfloat16()), start[2].cpu().numpy(), f64(start[3])
    keep, factor = O.dropout_keep(batch, width, p, 1000, 0, width)
    h = O.embedding(tokens, e, 16.0, 0) * keep * factor
    hv, wv = (O.mx_values(*O.mx_pack(*O.mx_quantize(v)), width) for v in (h, w))
    y = hv @ wv.T
    y_err = (width + 3) * 2.0**-24 * (np.abs(hv) @ np.abs(wv).T + np.abs(targets))
    err = y - targets
    loss = np.sum(err**2) / (2 * batch * outputs)
    assert abs(losses[0] - loss) <= 2.0**-11 * loss + np.sum(np.abs(err) * y_err) / (batch * outputs)

    g = err / batch
    g_err = 2.0**-8 * np.abs(g) + y_err / batch
    sums = (batch + outputs) * 2.0**-24
    dl, dl_err = g.T @ hv, g_err.T @ np.abs(hv) + sums * (np.abs(g).T @ np.abs(hv))
    dh, dh_err = g @ wv, g_err @ np.abs(wv) + (sums + 2.0**-8) * (np.abs(g) @ np.abs(wv))
    dt = O.embedding_grad(tokens, dh * keep * factor, vocabulary, 16.0, 0)
    dt_err = O.embedding_grad(tokens, dh_err * keep * factor, vocabulary, 16.0, 0)
    dt_err += sums * O.embedding_grad(tokens, np.abs(dh) * keep * factor, vocabulary, 16.0, 0)
    for got, old, d, d_err in ((layer, w, dl, dl_err), (table, f64(start[1]), dt, dt_err)):
        want, bound = old - rate / outputs * d, rate / outputs * d_err + 2.0**-22 * (np.abs(old) + np.abs(d))
        assert np.all(np.abs(f64(got) - want) <= bound)


@pytest.mark.gpu
def test_sharded_steps_learn():
    step = example()
    losses, _, _ = step.train(8, 5, *step.problem())
    assert all(b < a for a, b in zip(losses, losses[1:]))
