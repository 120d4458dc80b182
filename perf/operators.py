"""The calls that the operators on gathered and scattered tensors are timed on: 4-bit block quantisation and
products, embedding lookup and its gradient, dropout, through the tensor-level functions of
``paper_2506_20252_amd.ops``; beside each call its plain form in float32 torch operations.

A case is {"op", sizes, types}; what each op's sizes mean is said at its plain form.
"""

import math

import numpy as np
import torch

own = False

TORCH = {"float32": torch.float32, "bfloat16": torch.bfloat16}
SIZE = {"float32": 4, "bfloat16": 2}
BLOCK, GROUP = 32, 128  # values that share a scale; values that a row of codes is padded to


def listed():
    return [
        # A rank's float32 shard with an odd shape, quantised before an all-gather and widened after it.
        dict(name="cast_f32_odd", op="cast", rows=1001, cols=1000, dtype="float32", out="float32"),
        # A large bf16 weight shard, both ways.
        dict(name="cast_bf16_64m", op="cast", rows=8192, cols=8192, dtype="bfloat16", out="bfloat16"),
        # One token against a gathered 4-bit weight: reading the weight is all there is.
        dict(name="linear_token", op="linear", m=1, n=8192, k=8192, dtype="bfloat16", out="bfloat16"),
        # A small serving batch, sizes that no tile divides.
        dict(name="linear_batch_odd", op="linear", m=24, n=5000, k=4001, dtype="float32", out="float32"),
        # A long prompt or a training forward pass: the matrix units' work.
        dict(name="linear_prompt", op="linear", m=8192, n=8192, k=8192, dtype="bfloat16", out="bfloat16"),
        # A small training step with odd sizes: forward, gradient of the input, gradient of the weight.
        dict(name="linear_train_odd", op="linear_train", m=1001, n=1000, k=1333, dtype="bfloat16", out="float32"),
        # The two gradients of a large layer; the weight's goes into a reduce-scatter in float32.
        dict(name="linear_grads", op="linear_grads", m=8192, n=4096, k=4096, dtype="bfloat16", out="float32"),
        # Lookup for a large training batch.
        dict(name="embed_lookup", op="embed", tokens=65536, cols=4096, rows=32768, first=0, vocab=32768,
             dtype="bfloat16", out="bfloat16", scale=64.0),
        # A vocabulary shard (most tokens belong to other ranks), odd sizes, both directions.
        dict(name="embed_train_odd", op="embed_train", tokens=1001, cols=333, rows=1251, first=1251, vocab=5003,
             dtype="float32", out="float32", scale=18.25),
        # The dense gradient of a whole table from a large batch, for a float32 reduce-scatter.
        dict(name="embed_grad", op="embed_grad", tokens=131072, cols=2048, rows=65536, first=0, vocab=65536,
             dtype="bfloat16", out="float32", scale=1.0),
        # Dropout on the residual stream of a large batch.
        dict(name="dropout_residual", op="dropout", rows=16384, cols=4096, dtype="bfloat16", p=0.1),
        # A small step's dropout and its gradient, odd sizes: launches are what costs.
        dict(name="dropout_train_odd", op="dropout_train", rows=1001, cols=333, dtype="float32", p=0.25),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """Casts of up to 2^26 values; products from one row and 2^12 multiplications to 2^39, gradients to 2^37; lookups and
    gradients of 1 to 131072 tokens on tables of up to 2^27 values; dropout of up to 2^26 values."""
    while True:
        op = rng.choice(["cast", "linear", "linear", "linear", "linear_train", "linear_grads",
                         "embed", "embed_train", "embed_grad", "dropout", "dropout_train"])
        dtype, out = rng.choice(sorted(TORCH)), rng.choice(sorted(TORCH))
        if op == "cast":
            case = dict(rows=_log_int(rng, 1, 16384), cols=_log_int(rng, 1, 16384))
            if case["rows"] * case["cols"] > 1 << 26:
                continue
        elif op.startswith("linear"):
            few = op == "linear" and rng.random() < 0.5
            case = dict(m=_log_int(rng, 1, 64 if few else 8192), n=_log_int(rng, 16, 16384), k=_log_int(rng, 32, 16384))
            if case["m"] * case["n"] * case["k"] > (1 << 39 if op == "linear" else 1 << 37):
                continue
            if rng.random() < 0.4:  # about what a model's own widths are
                case["n"], case["k"] = max(16, case["n"] // 128 * 128), max(32, case["k"] // 128 * 128)
            if op != "linear" and max(case["m"], case["n"]) * case["k"] > 1 << 26:
                continue
        elif op.startswith("embed"):
            case = dict(tokens=_log_int(rng, 1, 131072), cols=_log_int(rng, 1, 8192), rows=_log_int(rng, 16, 131072))
            if rng.random() < 0.5:
                case["cols"] = max(8, case["cols"] // 8 * 8)
            if max(case["tokens"], case["rows"]) * case["cols"] > 1 << 27:
                continue
            shards = rng.choice([1, 1, 2, 8])
            case.update(first=case["rows"] * rng.randrange(shards), vocab=case["rows"] * shards,
                        scale=rng.choice([1.0, math.sqrt(case["cols"])]))
        else:
            case = dict(rows=_log_int(rng, 1, 32768), cols=_log_int(rng, 1, 16384), p=round(rng.uniform(0.0, 0.5), 3))
            if case["rows"] * case["cols"] > 1 << 26:
                continue
            return dict(op=op, dtype=dtype, **case)
        return dict(op=op, dtype=dtype, out=out, **case)


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------


def _pow2(byte):
    """2^(byte - 127) of an int32 scale byte, as float32 bits; 255 is NaN."""
    bits = torch.where(byte == 0, 0x00400000, byte << 23)
    return torch.where(byte == 255, 0x7FC00000, bits).to(torch.int32).view(torch.float32)


def _plain_quantize(x):
    """Codes (0..7 and a sign in bit 3) and scale bytes of rows cut into blocks of 32, both int32, [rows, blocks, 32]
    and [rows, blocks]; the last block of a row is filled up with zeros."""
    x = x.float()
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    high = x.abs().amax(2)
    field = high.view(torch.int32) >> 23
    byte = torch.where(field == 255, 255, (field - 2).clamp_min(0)).to(torch.int32)
    up = ((254 - byte.clamp_max(252)) << 23).view(torch.float32)
    v = x * up[..., None]
    a = v.abs()
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int()
            + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())
    code = code + 8 * torch.signbit(v).int()
    return torch.where(byte[..., None] == 255, 0, code).to(torch.int32), byte


def _plain_values(code, byte, cols):
    """What codes and scales stand for: float32 [rows, cols]."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    return (table[code] * _pow2(byte)[..., None]).flatten(1)[:, :cols].contiguous()


def _pack(code, byte):
    """The stored form: two codes a byte, the even one low; rows filled up to whole groups of 128 values."""
    rows, blocks = byte.shape
    groups = -(-blocks // 4)
    code, byte = code.to(torch.uint8), byte.to(torch.uint8)
    codes = torch.zeros((rows, 64 * groups), dtype=torch.uint8, device=code.device)
    codes[:, :16 * blocks] = (code[..., 0::2] | (code[..., 1::2] << 4)).view(rows, -1)
    scales = torch.zeros((rows, 4 * groups), dtype=torch.uint8, device=code.device)
    scales[:, :blocks] = byte
    return codes, scales


def _unpack(codes, scales, cols):
    """The values of the stored form."""
    code = torch.stack((codes & 15, codes >> 4), dim=2).view(codes.shape[0], -1, BLOCK).int()
    return _plain_values(code, scales.int(), cols)


def _plain_embed(s):
    row = s["tokens"] - s["first"]
    inside = (row >= 0) & (row < s["rows"])
    out = s["table"][row.clamp(0, s["rows"] - 1).long()].float() * s["scale"]
    return torch.where(inside[:, None], out, 0.0).to(s["out"])


def _plain_embed_grad(s):
    row = s["tokens"] - s["first"]
    inside = (row >= 0) & (row < s["rows"])
    g = torch.where(inside[:, None], s["g"].float(), 0.0)
    total = torch.zeros((s["rows"], s["cols"]), dtype=torch.float32, device=g.device)
    total.index_add_(0, row.clamp(0, s["rows"] - 1).long(), g)
    return (total * s["scale"]).to(s["out"])


def _philox(block, seed):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) of counters (block, 0) under key `seed`: [n, 4], each word 32 bits
    in an int64."""
    mask = 0xFFFFFFFF
    c0, c1 = block & mask, (block >> 32) & mask
    c2, c3 = torch.zeros_like(c0), torch.zeros_like(c0)
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64-bit products, kept modulo 2^64
        c0, c1, c2, c3 = ((b >> 32) & mask) ^ c1 ^ k0, b & mask, ((a >> 32) & mask) ^ c3 ^ k1, a & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return torch.stack((c0, c1, c2, c3), dim=1)


def _plain_dropout(s, x, residual):
    """Element i (row-major) is kept where the 16 bits of its half word reach p * 65536."""
    n = x.numel()
    words = _philox(torch.arange(-(-n // 8), device=x.device), s["seed"])
    u16 = torch.stack((words & 0xFFFF, words >> 16), dim=2).view(-1)[:n].view(x.shape)
    drop = int(s["p"] * 65536 + 0.5)
    y = torch.where(u16 >= drop, x.float() * (65536 / max(1, 65536 - drop)), 0.0)
    return (y if residual is None else y + residual.float()).to(x.dtype)


# ---------------------------------------------------------------------------
# Inputs and passes
# ---------------------------------------------------------------------------


def _activations(shape, gen):
    """Normal values, a few columns some ten times larger, as activations have them."""
    x = torch.empty(shape, device="cuda").normal_(generator=gen)
    big = torch.rand((1, shape[1]), device="cuda", generator=gen) < 0.01
    return torch.where(big, 10.0 * x, x)


def _tokens(case, gen):
    """Log-uniform token numbers: a few are very frequent, most are rare."""
    u = torch.rand(case["tokens"], device="cuda", generator=gen, dtype=torch.float64)
    ids = (torch.exp(u * math.log(case["vocab"] + 1)).long() - 1).clamp(0, case["vocab"] - 1)
    # a fixed spread of the frequent ones over the whole range
    return ((ids * 2654435761 + 12345) % case["vocab"]).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, s = case["op"], dict(case)
    dtype = TORCH[case["dtype"]]
    if "out" in case:
        s["out"] = TORCH[case["out"]]
    if op == "cast":
        s["x"] = _activations((case["rows"], case["cols"]), gen).to(dtype)
    elif op.startswith("linear"):
        m, n, k = case["m"], case["n"], case["k"]
        s["x"] = _activations((m, k), gen).to(dtype)
        w = torch.empty((n, k), device="cuda").normal_(0.0, 1.0 / math.sqrt(k), generator=gen)
        s["w"] = _pack(*_plain_quantize(w))
        if op != "linear":
            s["g"] = torch.empty((m, n), device="cuda").normal_(0.0, 1.0 / math.sqrt(n), generator=gen).bfloat16()
        if op == "linear_grads":  # what the forward pass has saved for them
            s["xq"] = _pack(*_plain_quantize(s.pop("x")))
    elif op.startswith("embed"):
        s["tokens"] = _tokens(case, gen)
        if op != "embed_grad":
            s["table"] = torch.empty((case["rows"], case["cols"]), device="cuda").normal_(0.0, 0.02, generator=gen).to(dtype)
        if op != "embed":
            s["g"] = torch.empty((case["tokens"], case["cols"]), device="cuda").normal_(generator=gen).to(dtype)
    else:
        shape = (case["rows"], case["cols"])
        s["seed"] = 0x5041541 + seed
        s["x"] = _activations(shape, gen).to(dtype)
        second = torch.empty(shape, device="cuda").normal_(generator=gen).to(dtype)
        s["residual" if op == "dropout" else "g"] = second
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    op = s["op"]
    if op == "cast":
        return _plain_values(*_plain_quantize(s["x"]), s["cols"]).to(s["out"])
    if op.startswith("linear"):
        k, out = s["k"], {}
        w = _unpack(*s["w"], k)
        x = _unpack(*s["xq"], k) if "xq" in s else _plain_values(*_plain_quantize(s["x"]), k)
        if op != "linear_grads":
            out["y"] = (x @ w.t()).to(s["out"])
        if op != "linear":
            g = s["g"].float()
            out["dx"], out["dw"] = (g @ w).bfloat16(), (g.t() @ x).to(s["out"])
        return out
    if op == "embed":
        return _plain_embed(s)
    if op == "embed_train":
        return {"out": _plain_embed(s), "grad": _plain_embed_grad(s)}
    if op == "embed_grad":
        return _plain_embed_grad(s)
    if op == "dropout":
        return _plain_dropout(s, s["x"], s["residual"])
    return {"y": _plain_dropout(s, s["x"], None), "dx": _plain_dropout(s, s["g"], None)}


def _run_own(s):
    from paper_2506_20252_amd import ops

    op = s["op"]
    if op == "cast":
        return ops.mx_dequantize(ops.mx_quantize(s["x"]), s["out"])
    if op.startswith("linear"):
        out, w = {}, ops.Mx(*s["w"], s["k"])
        if op == "linear":
            return {"y": ops.mx_linear(s["x"], w, s["out"])}
        if op == "linear_train":  # the quantised input is kept for the weight's gradient
            xq = ops.mx_quantize(s["x"])
            out["y"] = ops.mx_matmul(xq, w, s["out"])
        else:
            xq = ops.Mx(*s["xq"], s["k"])
        out["dx"] = ops.mx_matmul_grad(s["g"], w, torch.bfloat16)
        out["dw"] = ops.mx_matmul_grad(s["g"], xq, s["out"], transposed=True)
        return out
    if op.startswith("embed"):
        out = {}
        if op != "embed_grad":
            out["out"] = ops.embedding(s["tokens"], s["table"], s["scale"], s["first"], s["out"])
        if op != "embed":
            out["grad"] = ops.embedding_grad(s["tokens"], s["g"], s["rows"], s["scale"], s["first"], s["out"])
        return out if op == "embed_train" else next(iter(out.values()))
    if op == "dropout":
        return ops.dropout(s["x"], s["p"], s["seed"], residual=s["residual"])
    return {"y": ops.dropout(s["x"], s["p"], s["seed"]), "dx": ops.dropout(s["g"], s["p"], s["seed"])}


def work(case):
    """Inputs read once and outputs written once; 4-bit tensors at 17/32 byte a value.  A lookup reads the rows that its
    tokens are expected to touch (the tokens' distribution is known)."""
    op, size = case["op"], SIZE[case["dtype"]]
    out, q = SIZE.get(case.get("out"), 0), 17 / 32
    if op == "cast":  # the stored form is written by one call and read by the other
        return {"bytes": case["rows"] * case["cols"] * (size + 2 * q + out), "flops": 0}
    if op.startswith("linear"):
        m, n, k = case["m"], case["n"], case["k"]
        if op == "linear":
            return {"bytes": m * k * size + n * k * q + m * n * out, "flops": 2 * m * n * k}
        grads = m * n * 2 + n * k * q + m * k * q + m * k * 2 + n * k * out
        if op == "linear_grads":
            return {"bytes": grads, "flops": 4 * m * n * k}
        return {"bytes": grads + m * k * (size + q) + m * n * out, "flops": 6 * m * n * k}
    if op.startswith("embed"):
        tokens, cols, rows, vocab = case["tokens"], case["cols"], case["rows"], case["vocab"]
        share = rows / vocab
        v = np.arange(1, vocab + 1)
        touched = share * float(np.sum(1 - np.exp(-tokens * np.log1p(1 / v) / math.log(vocab + 1))))
        lookup = tokens * 4 + touched * cols * size + tokens * cols * out
        grad = tokens * 4 + share * tokens * cols * size + rows * cols * out
        return {"bytes": {"embed": lookup, "embed_grad": grad, "embed_train": lookup + grad}[op], "flops": 0}
    values = case["rows"] * case["cols"] * size
    return {"bytes": values * (3 if op == "dropout" else 4), "flops": 0}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------


def _exact_mx(x):
    """x in float64 -> the nearest multiples that a 4-bit block can hold: the exponent of the block's largest value less
    two is the scale's; steps of 1/2 below 2, of 1 below 4, of 2 above, ties to the even multiple, 6 at most."""
    rows, cols = x.shape
    full = torch.zeros((rows, -(-cols // BLOCK) * BLOCK), dtype=torch.float64, device=x.device)
    full[:, :cols] = x
    blocks = full.view(rows, -1, BLOCK)
    _, e = torch.frexp(blocks.abs().amax(2, keepdim=True))  # largest = f 2^e, f in [1/2, 1)
    unit = torch.exp2((e - 3).clamp_min(-127).double())
    a = blocks.abs() / unit
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    q = (torch.round(a / step) * step).clamp_max(6.0)
    return (torch.sign(blocks) * q * unit).view(rows, -1)[:, :cols]


def _exact_stored(q, cols):
    codes, scales = (t.cpu().numpy() for t in q)
    nibble = np.empty((codes.shape[0], codes.shape[1] * 2), dtype=np.int8)
    nibble[:, 0::2], nibble[:, 1::2] = codes % 16, codes // 16
    mag, sign = nibble % 8, 1 - 2 * (nibble // 8)
    value = sign * np.where(mag < 2, mag * 0.5, (1 + 0.5 * (mag % 2)) * np.exp2(mag // 2 - 1.0))
    value *= np.repeat(np.exp2(scales.astype(np.float64) - 127), BLOCK, axis=1)
    return torch.from_numpy(value[:, :cols].copy()).cuda()


def _exact_drop(s, x):
    """numpy's unsigned 64-bit integers, block by block."""
    n = x.numel()
    c = np.zeros((4, -(-n // 8)), dtype=np.uint64)
    c[0] = np.arange(c.shape[1], dtype=np.uint64)  # fewer than 2^32 blocks
    low, key = np.uint64(0xFFFFFFFF), [s["seed"] % 2**32, s["seed"] // 2**32]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = np.stack([(q >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), q & low,
                      (p >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), p & low])
        key = [(key[0] + 0x9E3779B9) % 2**32, (key[1] + 0xBB67AE85) % 2**32]
    half = c.T.astype("<u4").copy().view("<u2").reshape(-1)[:n].reshape(tuple(x.shape))
    threshold = math.floor(s["p"] * 65536 + 0.5)
    keep = torch.from_numpy((half >= threshold).astype(np.float64)).cuda()
    return x.double() * keep * (65536.0 / (65536.0 - threshold))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "cast":
        return _exact_mx(s["x"].double())
    if op.startswith("linear"):
        k, out = case["k"], {}
        w = _exact_stored(s["w"], k)
        x = _exact_stored(s["xq"], k) if "xq" in s else _exact_mx(s["x"].double())
        if op != "linear_grads":
            out["y"] = torch.mm(x, w.t().contiguous())
        if op != "linear":
            g = s["g"].double()
            out["dx"], out["dw"] = torch.mm(g, w), torch.mm(g.t().contiguous(), x)
        return out
    if op.startswith("embed"):
        out = {}
        row = s["tokens"].long() - case["first"]
        inside = ((row >= 0) & (row < case["rows"])).nonzero()[:, 0]
        if op != "embed_grad":
            out["out"] = torch.zeros((case["tokens"], case["cols"]), dtype=torch.float64, device="cuda")
            out["out"][inside] = case["scale"] * s["table"].double()[row[inside]]
        if op != "embed":
            out["grad"] = torch.zeros((case["rows"], case["cols"]), dtype=torch.float64, device="cuda")
            for part in inside.split(16384):
                out["grad"].index_add_(0, row[part], case["scale"] * s["g"][part].double())
        return out if op == "embed_train" else next(iter(out.values()))
    if op == "dropout":
        return _exact_drop(s, s["x"]) + s["residual"].double()
    return {"y": _exact_drop(s, s["x"]), "dx": _exact_drop(s, s["g"])}
