"""What the documents and comments of a layer's operators promise beyond single results: bounds, workspaces, places, and the
rules of how the kernels' sources are written.  Tolerances as in tests/test_layer_ops.py; others are derived at their tests.
"""

import glob
import os
import re

import numpy as np
import pytest
import torch

from oracle import layer as L
from paper_2506_20252_amd import build as B
from paper_2506_20252_amd import ops
from test_layer_ops import blocks_within, depth
from test_ops import E, F32, B16, U, f64, values, within

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
gpu = pytest.mark.gpu


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
