"""What the documents and comments of a layer's operators promise beyond single results: bounds, workspaces, places, and the
rules of how the kernels' sources are written.  Tolerances as in tests/test_layer_ops.py; others are derived at their tests.
"""

import glob
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import layer as L
from paper_2506_20252_amd import build as B
from paper_2506_20252_amd import ops, pat
from test_layer_ops import EVERY, act_error, blocks_within, depth, every_operator, flat, gated_error, random_mxb
from test_ops import E, F32, B16, U, f64, guarded, random_mx, values, within

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
gpu = pytest.mark.gpu
NAME = {F32: "float32", B16: "bfloat16"}


def header():
    """include/pat_ops.h as one line."""
    with open(os.path.join(ROOT, "include", "pat_ops.h")) as f:
        return re.sub(r"[\s*]+", " ", f.read())


def stated(pattern):
    """A number that the header states."""
    found = re.search(pattern, header())
    assert found, pattern
    return float(found[1])


# ---------------------------------------------------------------------------
# On the CPU
# ---------------------------------------------------------------------------


def test_inline_assembly_names_the_m0_that_it_uses():
    """Loads into LDS take their place from m0.  The compiler keeps values of its own there, so an asm statement either takes m0
    as an operand or says that it writes it."""
    found = 0
    for path in glob.glob(os.path.join(B.CSRC, "*.h*")):
        with open(path) as f:
            text = f.read()
        for statement in re.findall(r"\basm(?:\s+volatile)?\s*\((.*?)\);", text, re.S):
            code, _, operands = statement.partition("::")
            if re.search(r"\bm0\b", code):
                assert re.search(r':\s*"(?:.*,\s*")?m0"', operands), (path, statement)
            elif "load_lds" in code:
                assert '"{m0}"(' in operands, (path, statement)
            else:
                continue
            found += 1
    assert found >= 3


def rows_of_blocks():
    """Blocks whose largest value is just above, between and at the ends of where a scale holds, other values down to 2^-12 of it,
    and of each sign; at several scales."""
    g = np.random.default_rng(5)
    x = np.exp2(-12 * g.random((7 * 64, 32))) * g.choice([-1.0, 1.0], size=(7 * 64, 32))
    x = x.reshape(7, 64, 32)
    for i, top in enumerate((1.8750001, 1.876, 2.0, 2.5, 3.0, 3.7, 3.75)):
        x[i] *= top
        x[i, :, 0] = top
        x[i, :, 1] = 1.2 * 2.0**-8 * top
    x[:, :16] *= 2.0**-100
    x[:, 16:32] *= 2.0**90
    return x.reshape(7, -1).astype(np.float32).astype(np.float64)


def check_rounding(x, got, scales):
    """Half a step at most, as the header says it."""
    part = stated(r"down to 1/(\d+) of the block's largest")
    unit = np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, axis=1)[:, :x.shape[1]]
    largest = np.repeat(np.abs(x).reshape(x.shape[0], -1, 32).max(axis=2), 32, axis=1)
    off = np.abs(got - x)
    near = np.abs(x) >= 2.0**-6 * unit
    assert np.all(off[near] <= 2.0**-4 * np.abs(x)[near]) and np.all(off[~near] <= 2.0**-10 * unit[~near])
    assert np.all(near[np.abs(x) >= largest / part])
    assert not np.all(near[np.abs(x) >= largest / (1.01 * part)])  # no smaller part would be true


def test_oracle_rounding_is_what_the_header_says():
    x = rows_of_blocks()
    codes, scales = L.mxb_quantize(x)
    check_rounding(x, L.mxb_values(codes, scales, x.shape[1]), scales)
    row = np.full((1, 32), 1.2 * 2.0**-8 * 1.876)
    row[0, 0] = 1.876
    got = L.mxb_values(*L.mxb_quantize(row), 32)
    assert abs(got[0, 1] / row[0, 1] - 1) > 0.11  # 2^-8 of the largest is below where 2^-4 of a value holds


def source_of(name, function):
    with open(os.path.join(B.CSRC, name)) as f:
        return re.search(rf"\n[^\n]*\b{function}\(.*?\n}}\n", f.read(), re.S)[0]


def comment_of(name, function):
    with open(os.path.join(B.CSRC, name)) as f:
        return re.search(rf"((?://[^\n]*\n)+)[^\n]*\b{function}\(", f.read())[1].replace("\n// ", " ")


def normal_below(a, rcp_off=0, exp_off=0):
    """The kernels' P(a) = (1 + erf(a / sqrt 2)) / 2 in float32 step by step, with the source's coefficients; 1 / x and 2^x right or
    a unit off.  Fused multiply-adds through float64, whose own rounding is 2^-29 of float32's."""
    f = np.float32
    text = source_of("layer_device.hpp", "normal_below")
    slope = f(re.search(r"1\.0f \+ ([\d.]+)f \* fabsf", text)[1])
    c = [f(v) for v in [re.search(r"float p = (-?[\d.]+)f;", text)[1], *re.findall(r"fmaf\(p, t, (-?[\d.]+)f\)", text)]]
    assert len(c) == 7

    def unit(v, off):
        return np.nextafter(v, f(np.inf) * off) if off else v

    t = unit((1 / (1 + slope.astype(np.float64) * np.abs(a)).astype(f).astype(np.float64)).astype(f), rcp_off)
    p = np.full_like(t, c[0])
    for v in c[1:]:
        p = (p.astype(np.float64) * t + np.float64(v)).astype(f)
    log2e = f(1.44269504088896341)
    bell = unit(np.exp2((f(-0.5) * log2e * a * a).astype(np.float64)).astype(f), exp_off)
    q = f(0.5) * (p * t) * bell
    assert q.dtype == f
    return np.where(a >= 0, f(1) - q, q)


def normal(a):
    return 0.5 * torch.erfc(torch.from_numpy(-a / np.sqrt(2))).numpy()


def normal_grid():
    near = np.exp(np.linspace(np.log(1e-9), 0, 200001))
    a = np.concatenate((near, np.linspace(0, 13, 1000001))).astype(np.float32)
    return np.concatenate((a, -a))


def test_the_normal_distribution_is_as_close_as_its_comment_says():
    text = comment_of("layer_device.hpp", "normal_below")
    exact, off = (float(re.search(p, text)[1]) for p in (r"by ([\d.]+) \* 2\^-24 with float32's", r"([\d.]+) \* 2\^-24 where the"))
    near, tail = (float(re.search(rf"([\d.e-]+) down to -{e}\b", text)[1]) for e in (5, 13))
    a = normal_grid()
    want = normal(a.astype(np.float64))
    for r in (-1, 0, 1):
        for e in (-1, 0, 1):
            error = np.abs(normal_below(a, r, e) - want)
            assert error.max() <= (off if r or e else exact) * U
            assert np.all(error[a < 0] <= (tail * want)[a < 0]) and np.all(error[(a < 0) & (a >= -5)] <= (near * want)[(a < 0) & (a >= -5)])


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include/hip"),
                    reason="no g++ or no HIP headers")
def test_launches_and_workspaces_under_asan_ubsan(tmp_path):
    """By the functions that the launches use."""
    exe = tmp_path / "layer_plan_check"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", B.CSRC,
           os.path.join(ROOT, "tests", "host", "layer_plan_check.cpp"), "-o", str(exe)]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, (res.stdout[-2000:], res.stderr[-2000:])
    assert " 0 failures" in res.stdout


def test_launches_take_their_sizes_from_what_is_checked():
    """The kernels' sources cut nothing themselves: products are launched by product_plan, workspaces laid out by norm_grad_space."""
    with open(os.path.join(B.CSRC, "mxb_product.hip")) as f:
        product = f.read()
    assert product.count("product_plan(m, n, k,") == 2 and product.count("hipLaunchKernelGGL") == 2
    assert not re.search(r"\b(layer_tile|few_band|few_columns_sixteens|few_product|kFewGated|kFewLinear)\b", product)
    with open(os.path.join(B.CSRC, "norm.hip")) as f:
        norm = f.read()
    assert norm.count("norm_grad_space(") == 2


# ---------------------------------------------------------------------------
# On the GPU
# ---------------------------------------------------------------------------


@gpu
def test_rounding_is_what_the_header_says():
    x = rows_of_blocks()
    q = ops.mxb_quantize(torch.from_numpy(x).float().cuda())
    check_rounding(x, f64(ops.mxb_dequantize(q, F32)), q.scales.cpu().numpy())


NORMS = [(3, 1), (5, 7), (4, 333), (3, 4096), (2, 9795), (2, 16384), (2, 20001)]


@gpu
@pytest.mark.parametrize("rows,cols", NORMS)
@pytest.mark.parametrize("dtype", [F32, B16])
def test_norm_at_the_ends_of_its_range(rows, cols, dtype):
    """Rows whose sum of squares is just below the largest that the header names, and rows whose mean of squares is just above the
    smallest, eps zero: as exact as any.  The gradients' tolerance is that of the layer's tests; g is of a size that keeps
    g * weight * x in range."""
    high, low = stated(r"sum of squares is at most 2\^(\d+)"), stated(r"mean of squares plus eps is at least 2\^-(\d+)")
    x, g = f64(values((rows, cols), 1)), values((rows, cols), 2, dtype)
    weight = 1 + values((cols,), 3)
    x[:, 0] = 1.0  # no row of zeros
    for top in (True, False):
        size = np.sqrt(0.98 * 2.0**high / np.sum(x * x, axis=1)) if top else np.sqrt(1.02 * 2.0**-low / np.mean(x * x, axis=1))
        t = torch.from_numpy(x * size[:, None]).to(dtype).cuda()  # rounding moves a square by 2^-7 at most, both ends by less
        vt, vg, vw = f64(t), f64(g), f64(weight)
        sums = np.sum(vt * vt, axis=1)
        assert np.all(sums <= 2.0**high) if top else np.all(sums / cols >= 2.0**-low)
        want = L.rms_norm(vt, vw, 0.0)
        err = (depth(cols) / 2 + 8) * U * np.abs(want)
        off = np.abs(f64(ops.rms_norm(t, weight, 0.0, dtype=F32)) - want)
        assert np.all(off <= err + 2 * U * np.abs(want))
        blocks_within(ops.rms_norm(t, weight, 0.0, dtype=ops.Mxb), want, err)
        dx, dw = L.rms_norm_grad(vg, vt, vw, 0.0)
        r = 1 / np.sqrt(np.mean(vt * vt, axis=1, keepdims=True))
        size = r * (np.abs(vg * vw) + np.abs(vt) * r**2 * np.mean(np.abs(vg * vw * vt), axis=1, keepdims=True))
        got, dweight = ops.rms_norm_grad(g, t, weight, 0.0)
        bound = 2 * (depth(cols) + 12) * U * size + (E if dtype == B16 else 2 * U) * np.abs(dx) + 2.0**-133
        assert np.all(np.abs(f64(got) - dx) <= bound)
        within(dweight, dw, np.sum(np.abs(vg * vt * r), axis=0), rows + depth(cols), F32)


@gpu
@pytest.mark.parametrize("cols", [300, 16384, 20000])
def test_norm_beyond_its_range(cols):
    """As the header says it: an overflowing sum gives zeros, squares that vanish count as zero."""
    x = torch.full((2, cols), 2.0**64, device="cuda")
    x[1] = 2.0**-76
    one = torch.ones(cols, device="cuda")
    assert not bool(ops.rms_norm(x, one, 0.0)[0].any())
    assert not bool(torch.isfinite(ops.rms_norm(x, one, 0.0)[1]).any())
    small = f64(ops.rms_norm(x, one, 2.0**-20)[1])
    want = L.rms_norm(f64(x), 1.0, 2.0**-20)[1]
    assert np.all(np.abs(small - want) <= 8 * U * want)


@gpu
@pytest.mark.parametrize("m", [8, 40])  # few tokens; tiles
@pytest.mark.parametrize("low,high", [(112, 115), (115, 119), (119, 122)])
def test_gelu_is_as_close_as_its_distribution(m, low, high):
    """Projections that are exact (products are multiples of 2^-10 of the scales, and fewer than 2^24 of these in a sum) and b = 1, so
    that the output is a P(a) alone, rounded once.  P is off by 6.6 u at most: t by 2 u (its denominator's rounding and 1 / x), of
    which 1.57 times; the polynomial by 2.5 u (u, u/2, u/2, u/4, u/4, u/32) and p t, the bell, the two products by u each at
    most, of which half; 1 - q by u/2; the fit by 0.15 u.  Below -1 it is also off by 1.1e-4 of itself at most, down to -13."""
    n, k = 3000, 128
    g = np.random.default_rng(low)
    x, w = np.zeros((m, k)), np.zeros((2 * n, k))
    x[:, :96] = L.CODES[g.integers(0, 0x48, size=(m, 96))] * g.choice([-1, 1], size=(m, 96))
    x[:, [0, 32, 64]] = 3.75  # every block's scale is one
    x[:, 96] = 1.0
    size = np.exp2(g.integers(low, high, size=(n, 1)) - 122.0)
    w[:n, :96] = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])[g.integers(0, 8, size=(n, 96))] * g.choice([-1, 1], size=(n, 96)) * size
    w[n:, 96] = 1.0
    x8, w4 = (f(torch.from_numpy(v).float().cuda()) for f, v in ((ops.mxb_quantize, x), (ops.mx_quantize, w)))
    assert np.array_equal(f64(ops.mxb_dequantize(x8, F32)), x) and np.array_equal(f64(ops.mx_dequantize(w4, F32)), w)
    a = x @ w[:n].T
    h = f64(ops.gated(x8, w4, "gelu", F32))
    p = normal(a)
    off = np.abs(h - a * p)
    assert np.all(off <= np.abs(a) * (6.6 + 1) * U + 2.0**-149)
    tail = (a > -13) & (a < -1)
    assert np.all(off[tail] <= 1.1e-4 * np.abs(a * p)[tail] + 2.0**-149)
    assert low < 119 or np.count_nonzero(tail & (a < -5)) > 1000
    silu = f64(ops.gated(x8, w4, "silu", F32))
    want = a / (1 + np.exp(-a))  # the oracle's tanh has no relative exactness far out
    # e^-a: its argument a log2 e is off by 0.23 u for the constant and u for the product, relatively, so e^-a by 1.23 |a| u; 2^x,
    # 1 + e, 1 / x and a s by 8 u together.  From e^-a = 2^126 on, a = -87.4, its reciprocal is no normal number, and zero from
    # 2^128 on: off by 87.4 * 2^-126 < 2^-119 at most.
    assert np.all(np.abs(silu - want) <= U * (1.23 * np.abs(a) + 8) * np.abs(want) + 2.0**-119)


def guarded_workspace(nbytes, value):
    """`nbytes` inside a buffer of one value, and a check that nothing around them was written."""
    room = torch.full((nbytes + 8192,), value, dtype=torch.uint8, device="cuda")
    assert room.data_ptr() % 16 == 0

    def untouched():
        return bool((room[:4096] == value).all() and (room[4096 + nbytes:] == value).all())

    return room.data_ptr() + 4096, untouched


@gpu
@pytest.mark.parametrize("rows,cols", [(2, 3), (9, 5), (300, 7), (257, 129), (513, 1000), (1001, 1333), (70, 4097), (300, 8200), (270, 16383),
                                       (1, 16385), (2, 16391), (7, 20001), (300, 17000), (1030, 40001)])
@pytest.mark.parametrize("dtype,x_dtype", [(F32, F32), (B16, B16)])
def test_norm_gradients_in_a_workspace_of_exactly_their_bytes(rows, cols, dtype, x_dtype):
    """Nothing is written beside it and nothing read that was not written: whatever it held before, the result is the same."""
    x, g, weight = values((rows, cols), 1, x_dtype), values((rows, cols), 2, dtype), 1 + values((cols,), 3)
    want, want_weight = ops.rms_norm_grad(g, x, weight, 1e-5)
    nbytes = ops.pat_rms_norm_grad_workspace(rows, cols)
    for value in (0xFF, 0x7B):
        work, untouched = guarded_workspace(nbytes, value)
        out, dweight = torch.empty_like(g), torch.empty(cols, device="cuda")
        status = ops.pat_rms_norm_grad(g, cols, NAME[dtype], x, cols, NAME[x_dtype], weight, "float32", None, 0, rows, cols, 1e-5, out, cols, dweight, work,
                                       nbytes, torch.cuda.current_stream())
        assert status == pat.PAT_OK and untouched()
        assert torch.equal(out, want) and torch.equal(dweight, want_weight)


@gpu
@pytest.mark.parametrize("rows,inner,cols", [(40, 8449, 200), (64, 5761, 33), (100, 4096, 90), (33, 9000, 129), (512, 8200, 512), (8, 30001, 1000)])
def test_weight_gradients_in_a_workspace_of_exactly_their_bytes(rows, inner, cols):
    g, x = values((inner, rows), 1, B16), ops.mxb_quantize(values((inner, cols), 2))
    nbytes = ops.pat_mxb_weight_grad_workspace(rows, inner, cols)
    assert nbytes > 0  # sums in slices
    for dtype in (F32, B16):
        want = ops.mxb_weight_grad(g, x, dtype)
        for value in (0xFF, 0x7B):
            work, untouched = guarded_workspace(nbytes, value)
            out = torch.empty((rows, cols), dtype=dtype, device="cuda")
            status = ops.pat_mxb_weight_grad(g, rows, x.codes, x.scales, rows, inner, cols, out, cols, NAME[dtype], work, nbytes,
                                             torch.cuda.current_stream())
            assert status == pat.PAT_OK and untouched() and torch.equal(out, want)


@gpu
@pytest.mark.parametrize("m,n,k", [(16, 60, 1700), (17, 60, 1537), (24, 100, 2000), (32, 33, 4100), (32, 2048, 1664), (32, 2049, 1664),
                                   (17, 2048, 1536), (33, 40, 1700)])
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_gated_products_on_either_side_of_the_kernels_rule(m, n, k, name):
    x, vx = random_mxb(m, k, m + n, 118, 124)
    w, vw = random_mx(2 * n, k, n + k, 113, 122)
    h, a, b, eh, ea, eb = gated_error(vx, vw, n, k, name)
    for dtype in (F32, B16):
        out, untouched = guarded((m, n), dtype, pad=n % 3, shift=1)
        ops.gated(x, w, name, dtype, out=out)
        assert untouched()
        assert np.all(np.abs(f64(out) - h) <= eh + (E if dtype == B16 else 2 * U) * np.abs(h) + 1e-300)
    plain = out
    other, saved = ops.gated(x, w, name, B16, True)
    q = ops.gated(x, w, name, ops.Mxb)
    assert torch.equal(other, plain)
    blocks_within(q, h, eh)
    blocks_within(ops.Mxb(saved.codes[:m], saved.scales[:m], n), a, ea)
    blocks_within(ops.Mxb(saved.codes[m:], saved.scales[m:], n), b, eb)


# ---------------------------------------------------------------------------
# New tensors
# ---------------------------------------------------------------------------


@gpu
@pytest.mark.parametrize("shape", [(3, 5), (1, 1), (7, 0), (0, 7), (0, 0), (9,), (0,)])
@pytest.mark.parametrize("dtype", [F32, B16, torch.uint8])
def test_new_tensors_are_as_torch_makes_them(shape, dtype, monkeypatch):
    """By torch's own short way, where it has one, or by the public call: the same kind of tensor."""
    like = torch.empty(1, device="cuda")
    made = [ops._empty(shape, dtype, like, None)]
    monkeypatch.setattr(ops, "_strided", None)
    made.append(ops._empty(shape, dtype, like, None))
    want = like.new_empty(shape, dtype=dtype)
    for t in made:
        assert type(t) is torch.Tensor and not t.requires_grad and t.is_contiguous()
        assert (t.shape, t.stride(), t.dtype, t.device) == (want.shape, want.stride(), want.dtype, want.device)


@gpu
@pytest.mark.parametrize("name", EVERY)
def test_without_torchs_short_ways(name, monkeypatch):
    """Where this torch has no private functions for streams and new tensors: the same results, on the current stream."""
    call = every_operator()[name]
    want = [t.clone() for t in flat(call())]
    monkeypatch.setattr(ops, "_strided", None)
    monkeypatch.setattr(ops, "_raw_stream", None)
    monkeypatch.setattr(ops, "_current_device", torch.cuda.current_device)
    assert all(torch.equal(a, b) for a, b in zip(flat(call()), want))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = flat(call())
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
@pytest.mark.parametrize("name", EVERY)
def test_every_element_of_a_result_is_written(name, monkeypatch):
    """Whatever new memory holds: results and workspaces are filled before the call here, as torch does it to new tensors in its
    deterministic mode."""
    call, empty = every_operator()[name], ops._empty
    want = [t.clone() for t in flat(call())]
    for value in (0xFF, 0x5A):
        def filled(shape, dtype, like, stream):
            t = empty(shape, dtype, like, stream)
            t.view(torch.uint8).fill_(value)
            return t

        monkeypatch.setattr(ops, "_empty", filled)
        assert all(torch.equal(a, b) for a, b in zip(flat(call()), want))


# ---------------------------------------------------------------------------
# Stored matrices beyond 4 GiB
# ---------------------------------------------------------------------------


def repeated(q, parts, rows):
    """The rows of a stored matrix again and again, `rows` of them."""
    return type(q)(*(t.repeat(parts, 1)[:rows].contiguous() for t in q[:2]), q.cols)


def parts_agree(t, each):
    """Rows `each` apart hold the same."""
    return all(torch.equal(part, t[:len(part)]) for part in t.split(each))


@gpu
@pytest.mark.parametrize("n", [40, 300])
def test_products_of_more_than_4_gib_of_tokens(n):
    """Every part of the result is that of the same tokens elsewhere, and the first is right."""
    each, k = 4096, 8200
    m = 128 * each + 77
    some, v = random_mxb(each, k, 1, 118, 124)
    w, vw = random_mx(2 * n, k, 2, 112, 118)
    x = repeated(some, 129, m)
    assert x.codes.numel() > 1 << 32
    out = ops.mxb_linear(x, w, F32)
    assert parts_agree(out, each)
    within(out[:300], v[:300] @ vw.T, np.abs(v[:300]) @ np.abs(vw).T, k, F32)
    h, saved = ops.gated(x, w, "silu", ops.Mxb, True)
    _, a, b, _, ea, eb = gated_error(v[:300], vw, n, k, "silu")
    for codes, scales in ((saved.codes[:m], saved.scales[:m]), (saved.codes[m:], saved.scales[m:]), h[:2]):
        assert parts_agree(codes, each) and parts_agree(scales, each)
    blocks_within(ops.Mxb(saved.codes[:300], saved.scales[:300], n), a, ea)
    blocks_within(ops.Mxb(saved.codes[m:m + 300], saved.scales[m:m + 300], n), b, eb)
    # each row counts as often as it is there
    g = values((each, n), 3, B16)
    dw = ops.mxb_weight_grad(g.repeat(129, 1)[:m], x, F32)
    times = np.where(np.arange(each) < 77, 129.0, 128.0)[:, None]
    vg = f64(g) * times
    within(dw, vg.T @ v, np.abs(vg).T @ np.abs(v), m, F32)


@gpu
@pytest.mark.parametrize("m", [1, 33, 70])
def test_products_of_more_than_4_gib_of_weights(m):
    each, k = 4096, 8200
    n = 128 * each + 77
    x, vx = random_mxb(m, k, 1, 118, 124)
    some, v = random_mx(each, k, 2, 112, 118)
    half = repeated(some, 129, n)
    w = ops.Mx(torch.cat((half.codes, half.codes)), torch.cat((half.scales, half.scales)), k)
    assert half.codes.numel() > 1 << 31 and w.codes.numel() > 1 << 32
    a, size = vx @ v.T, np.abs(vx) @ np.abs(v).T
    out = ops.mxb_linear(x, w, F32)
    assert parts_agree(out[:, :n].t(), each) and torch.equal(out[:, :n], out[:, n:])
    within(out[:, :each], a, size, k, F32)
    h = ops.gated(x, w, "silu", F32)
    assert parts_agree(h.t(), each)
    err = 2 * (k + 2) * U * size
    want = L.act(a, "silu")[0]
    off = np.abs(f64(h[:, :each]) - want * a)
    assert np.all(off <= 1.01 * (act_error(a, "silu", err) * np.abs(a) + (np.abs(want) + err) * err + 4 * U * np.abs(want * a)))


@gpu
def test_products_of_the_most_terms():
    """2^24 - 1 terms in the largest tiles, whose rows lie up to 2^32 bytes apart: values of 0 and 1, so that every sum is a whole
    number below 2^24 and exact."""
    m, n, k, part = 2900, 2898, (1 << 24) - 1, 8192
    g = torch.Generator(device="cuda").manual_seed(1)
    bits_x, bits_w = (torch.randint(0, 2, (rows, part), device="cuda", generator=g, dtype=torch.uint8) for rows in (m, n))
    want = torch.mm(bits_x.double(), bits_w.double().t().contiguous()) * 2048
    want -= torch.outer(bits_x[:, -1].double(), bits_w[:, -1].double())
    assert float(want.max()) < 1 << 24
    codes = (bits_x * 0x38).repeat(1, 2048)
    codes[:, -1] = 0
    x = ops.Mxb(codes, torch.full((m, 1 << 19), 127, dtype=torch.uint8, device="cuda"), k)
    codes = (2 * bits_w[:, 0::2] + 32 * bits_w[:, 1::2]).repeat(1, 2048)
    codes[:, -1] &= 15
    w = ops.Mx(codes, torch.full((n, 1 << 19), 127, dtype=torch.uint8, device="cuda"), k)
    del codes
    assert torch.equal(ops.mxb_linear(x, w, F32).double(), want)
    a, b = want[:, :n // 2], want[:, n // 2:]
    h = ops.gated(x, w, "silu", F32).double()
    assert bool(((h - a * b).abs() <= 8 * U * a * b).all())  # e^-a is 0 against 1; a quotient and two products
    assert torch.equal(ops.mxb_linear(ops.Mxb(x.codes[:70], x.scales[:70], k), w, F32).double(), want[:70])
    assert torch.equal(ops.mxb_linear(ops.Mxb(x.codes[:5], x.scales[:5], k), w, F32).double(), want[:5])
    del x, w
    torch.cuda.empty_cache()
