"""Serving one attention layer from the block-scaled 8-bit cache: prompts in chunks, then decode steps.

    python examples/block_cache.py [--prompts 5000 700 64] [--steps 32] [--code int8|e4m3] [--dtype fp16|bf16]

Each prompt chunk is appended (keys and queries rotated on the way) and attends causally to everything before it; then every
sequence decodes one token per step, the steps replayed from a CUDA graph.  Random weights stand in for a model; the last
step's output is checked against attention in float64 over the keys and values as they were before quantization.
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_28699_gb300 as wc  # noqa: E402

HEADS, KV_HEADS, DIM, CHUNK, PAGE = 28, 4, 128, 2048, 16


def rope_tables(n, base=1e4):
    angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * base ** (
        -torch.arange(DIM // 2, device="cuda", dtype=torch.float64) * 2 / DIM)
    return angle.cos().float(), angle.sin().float()


def rotate(x, cos, sin):
    """x [n, heads, 128] float64, half layout."""
    a, b = x[..., :DIM // 2], x[..., DIM // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--prompts", type=int, nargs="+", default=[5000, 700, 64])
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--code", choices=["int8", "e4m3"], default="int8")
    ap.add_argument("--dtype", choices=["fp16", "bf16"], default="bf16")
    a = ap.parse_args(argv)
    dtype = torch.float16 if a.dtype == "fp16" else torch.bfloat16
    B, total = len(a.prompts), [n + a.steps for n in a.prompts]
    pages = [(n + PAGE - 1) // PAGE for n in total]
    desc = wc.BlockDesc(num_q_heads=HEADS, num_kv_heads=KV_HEADS, num_pages=sum(pages),
                        code=wc.CODE_INT8 if a.code == "int8" else wc.CODE_E4M3)
    cache = wc.BlockCache.empty(desc)
    table = torch.full((B, max(pages)), -1, dtype=torch.int32)
    order = torch.randperm(sum(pages)).int()
    for b, n in enumerate(pages):
        table[b, :n], order = order[:n], order[n:]
    table = table.cuda()
    cos, sin = rope_tables(max(total))
    g = torch.Generator(device="cuda").manual_seed(1)
    # a projection's output: queries, keys and values of a token side by side
    packed = [torch.randn(n, HEADS + 2 * KV_HEADS, DIM, generator=g, device="cuda").to(dtype) for n in total]
    split = lambda x: (x[:, :HEADS], x[:, HEADS:HEADS + KV_HEADS], x[:, HEADS + KV_HEADS:])  # noqa: E731
    word = torch.zeros(1, dtype=torch.int32, device="cuda")

    # prompts, a chunk of each at a time
    done = [0] * B
    ws = wc.BlockWorkspace(desc, B, B * CHUNK, max(pages))
    while any(d < n for d, n in zip(done, a.prompts)):
        new = [min(CHUNK, n - d) for d, n in zip(done, a.prompts)]
        x = torch.cat([packed[b][done[b]:done[b] + new[b]] for b in range(B)])
        done = [d + n for d, n in zip(done, new)]
        cu = torch.tensor([0] + new, dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
        ctx = torch.tensor(done, dtype=torch.int32).cuda()
        q, k, v = split(x)
        q = wc.block_append(desc, k, v, ctx, table, cache, cu_new=cu, cos=cos, sin=sin, q=q, dev_status=word)
        wc.block_extend_attention(desc, q, cu, table, ctx, cache, ws)      # the chunk's output; a model goes on from here

    # decode steps: fixed buffers, captured once, replayed
    x, ctx = torch.empty(B, HEADS + 2 * KV_HEADS, DIM, dtype=dtype, device="cuda"), torch.tensor(a.prompts, dtype=torch.int32).cuda()
    q, k, v = split(x)
    rotated, out = (torch.empty(B, HEADS, DIM, dtype=dtype, device="cuda") for _ in range(2))

    def step():
        ctx.add_(1)
        wc.block_append(desc, k, v, ctx, table, cache, cos=cos, sin=sin, q=q, q_out=rotated, dev_status=word)
        wc.block_decode_attention(desc, rotated, table, ctx, cache, ws, out=out)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(a.steps):
        x.copy_(torch.stack([packed[b][a.prompts[b] + i] for b in range(B)]))
        graph.replay()
    assert wc.read_status(word) == 0 and wc.read_status(ws) == 0

    worst = 0.0
    for b, n in enumerate(total):
        q, k, v = (t.double() for t in split(packed[b]))
        q = rotate(q[-1:], cos[n - 1:n, None].double(), sin[n - 1:n, None].double())[0].view(KV_HEADS, -1, DIM)
        k = rotate(k, cos[:n, None].double(), sin[:n, None].double())
        p = torch.softmax(torch.einsum("hgd,thd->hgt", q, k) / math.sqrt(DIM), -1)
        want = torch.einsum("hgt,thd->hgd", p, v).reshape(HEADS, DIM)
        worst = max(worst, float((out[b].double() - want).norm() / want.norm()))
    print(f"{B} sequences, {sum(a.prompts)} prompt tokens in chunks of {CHUNK}, {a.steps} steps; {cache.nbytes() / 2 ** 20:.1f} MiB of "
          f"{a.code} cache; output against unquantized float64 attention: relative error {worst:.4f}")
    return worst


if __name__ == "__main__":
    main()
