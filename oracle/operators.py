"""Plain definitions of the operators of include/pat_ops.h, in numpy and 64 bits.

Every function states the operator element by element or in one matrix
expression; nothing is shared with the kernels.  Matrices are float64 arrays of
values that the tensors hold exactly (bfloat16 and float32 widen exactly).
"""

import numpy as np

FP4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx_quantize(x):
    """(codes, scales): one int per value (0..15) and per block of 32, rows filled up to groups of 128 with 0."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    width = -(-cols // 128) * 128
    full = np.zeros((rows, width))
    full[:, :cols] = x
    codes = np.zeros((rows, width), dtype=np.int64)
    scales = np.zeros((rows, width // 32), dtype=np.int64)
    for r in range(rows):
        for b in range(width // 32):
            v = full[r, 32 * b:32 * b + 32]
            if not np.all(np.isfinite(v)):
                scales[r, b] = 255
                continue
            high = np.max(np.abs(v))
            s = max(int(np.floor(np.log2(high))) + 127 - 2, 0) if high >= 2.0**-126 else 0
            scales[r, b] = s
            a = np.abs(v) / 2.0**(s - 127)
            # nearest value; of two equally near ones the even code
            far = np.abs(a[:, None] - FP4[None, :])
            near = far.min(axis=1, keepdims=True)
            tie = far == near
            pick = np.where(tie[:, 0::2].any(axis=1), 2 * tie[:, 0::2].argmax(axis=1), 1 + 2 * tie[:, 1::2].argmax(axis=1))
            codes[r, 32 * b:32 * b + 32] = pick + 8 * np.signbit(v)
    return codes, scales


def mx_pack(codes, scales):
    """The stored form's bytes."""
    return (codes[:, 0::2] + 16 * codes[:, 1::2]).astype(np.uint8), scales.astype(np.uint8)


def mx_values(code_bytes, scale_bytes, cols):
    """What a stored form stands for, float64 [rows, cols]."""
    c = np.stack([code_bytes % 16, code_bytes // 16], axis=2).reshape(code_bytes.shape[0], -1).astype(np.int64)
    v = FP4[c % 8] * np.where(c >= 8, -1.0, 1.0)
    s = np.repeat(scale_bytes.astype(np.float64), 32, axis=1)
    return np.where(s == 255, np.nan, v * 2.0**(s - 127))[:, :cols]


def embedding(tokens, table, scale, first):
    out = np.zeros((len(tokens), table.shape[1]))
    for t, token in enumerate(tokens):
        if 0 <= int(token) - first < table.shape[0]:
            out[t] = scale * table[int(token) - first]
    return out


def embedding_grad(tokens, g, rows, scale, first):
    out = np.zeros((rows, g.shape[1]))
    for t, token in enumerate(tokens):
        if 0 <= int(token) - first < rows:
            out[int(token) - first] += scale * g[t]
    return out


def philox(c, k):
    """Philox4x32-10 of four counter words under two key words, in Python integers."""
    c, k = list(c), list(k)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_keep(rows, cols, p, seed, index, index_stride):
    """The mask, bool [rows, cols], and the factor of what is kept."""
    drop = int(np.floor(p * 65536 + 0.5))
    seed, words, keep = seed % 2**64, {}, np.zeros((rows, cols), dtype=bool)
    for r in range(rows):
        for c in range(cols):
            i = (index + r * index_stride + c) % 2**64
            b = i // 8
            if b not in words:
                words[b] = philox([b % 2**32, b // 2**32, 0, 0], [seed % 2**32, seed // 2**32])
            keep[r, c] = (words[b][i % 8 // 2] >> (16 * (i % 2))) % 65536 >= drop
    return keep, 65536.0 / (65536 - drop) if drop < 65536 else 0.0


def dropout(x, p, seed, index, index_stride, residual=None):
    keep, factor = dropout_keep(*x.shape, p, seed, index, index_stride)
    y = np.where(keep, x * factor, 0.0)
    return y if residual is None else y + residual
