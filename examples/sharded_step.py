"""A sharded data-parallel training step of virtual ranks on one GPU, with everything between its collectives.

N ranks share a token embedding (vocabulary x width, bfloat16) and a linear layer (outputs x width): each rank owns
1/N of the rows of both and one part of the batch.  A step, on every rank:

  1. quantise the own rows of the layer to 4-bit blocks, all-gather codes and scales (4.25 bits a value instead of
     the 32 of the master weights); all-gather the embedding's rows;
  2. look the tokens up, scaled; dropout, numbered over the whole batch; multiply by the gathered 4-bit weight;
  3. a squared-error loss against given targets; both gradients of the product, the dropout's, the embedding's;
  4. reduce-scatter both weight gradients; update the own rows.

Since the dropout's mask belongs to an element's place in the whole batch, any number of ranks computes the same step, up to
the order of its sums.

    python examples/sharded_step.py [--ranks 8] [--steps 20]
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2506_20252_amd import ops, pat  # noqa: E402


def gather(shards):
    """Every rank's copy of the concatenation of the ranks' rows: [N, N * rows, width] of [N, rows, width]."""
    n, rows, width = shards.shape
    words = shards.view(n, -1).view(torch.int32)  # 4-bit codes, scales and pairs of bfloat16 are 32-bit words
    out = torch.empty((n, n * words.shape[1]), dtype=torch.int32, device=shards.device)
    pat.allgather(words, out)
    return out.view(shards.dtype).view(n, n * rows, width)


def scatter_sum(parts):
    """Each rank's rows of the sum over ranks: [N, rows / N, width] of [N, rows, width]."""
    n, rows, width = parts.shape
    out = torch.empty((n, rows // n * width), dtype=parts.dtype, device=parts.device)
    pat.reducescatter(parts.view(n, -1), out)
    return out.view(n, rows // n, width)


def problem(vocabulary=4096, width=512, outputs=1024, batch=2048, seed=7):
    """Random weights (layer, embedding), tokens and targets."""
    draw = dict(device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
    layer = torch.randn(outputs, width, **draw) / math.sqrt(width)
    table = torch.randn(vocabulary, width, **draw) / math.sqrt(width)
    tokens = torch.randint(0, vocabulary, (batch,), **draw)
    return layer, table, tokens, torch.randn(batch, outputs, **draw)


def train(ranks, steps, layer, table, tokens, targets, p=0.1, rate=2.0):
    """`steps` steps on `ranks` ranks; returns their losses and the weights after the last one."""
    (outputs, width), vocabulary, batch = layer.shape, table.shape[0], tokens.numel()
    layer, table = layer.clone().view(ranks, -1, width), table.clone().view(ranks, -1, width)
    tokens, targets = tokens.view(ranks, -1), targets.view(ranks, -1, outputs)
    scale, part = math.sqrt(width), batch // ranks

    groups = -(-width // ops.PAT_MX_GROUP)
    codes = torch.empty((ranks, outputs // ranks, 64 * groups), dtype=torch.uint8, device="cuda")
    scales = torch.empty((ranks, outputs // ranks, 4 * groups), dtype=torch.uint8, device="cuda")

    losses = []
    for step in range(steps):
        for r in range(ranks):
            ops.mx_quantize(layer[r], out=ops.Mx(codes[r], scales[r], width))
        all_codes, all_scales, all_tables = gather(codes), gather(scales), gather(table.bfloat16())

        d_layer = torch.empty((ranks, outputs, width), device="cuda")
        d_table = torch.empty((ranks, vocabulary, width), device="cuda")
        loss = torch.zeros((), device="cuda")
        for r in range(ranks):
            weight = ops.Mx(all_codes[r], all_scales[r], width)
            mask = dict(p=p, seed=1000 + step, index=r * part * width)
            h = ops.embedding(tokens[r], all_tables[r], scale)
            h = ops.dropout(h, out=h, **mask)
            hq = ops.mx_quantize(h)
            y = ops.mx_matmul(hq, weight, torch.float32)

            error = (y - targets[r]) / batch
            loss += (error * (y - targets[r])).sum() / (2 * outputs)
            g = error.bfloat16()

            ops.mx_matmul_grad(g, hq, torch.float32, transposed=True, out=d_layer[r])
            dh = ops.mx_matmul_grad(g, weight)
            dh = ops.dropout(dh, out=dh, **mask)
            ops.embedding_grad(tokens[r], dh, vocabulary, scale, dtype=torch.float32, out=d_table[r])
        layer -= rate / outputs * scatter_sum(d_layer)
        table -= rate / outputs * scatter_sum(d_table)
        losses.append(float(loss))
    return losses, layer.view(outputs, width), table.view(vocabulary, width)


def main():
    args = argparse.ArgumentParser(description=__doc__.split("\n", 1)[0])
    args.add_argument("--ranks", type=int, default=8)
    args.add_argument("--steps", type=int, default=20)
    args = args.parse_args()
    losses, _, _ = train(args.ranks, args.steps, *problem())
    for step, loss in enumerate(losses):
        print(f"step {step}: loss {loss:.6f}")


if __name__ == "__main__":
    main()
