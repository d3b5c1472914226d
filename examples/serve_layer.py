"""Serves the attention block of one merged layer: quantized q / k / v products, paged cache plan, rotary positions with
the cache's append, attention over the cache, quantized o product.

    python examples/serve_layer.py [--heads 32] [--kv-heads 8] [--prompts 700,33,1500] [--steps 32]

Prompts of uneven length are read in one step, then every request decodes one token per step; the decode step is captured in
a CUDA graph once (lengths and tables live on the device, so the same graph serves every step).  Weights and activations are
random: what it shows is the order of the calls, who owns which buffer, and the time of a step.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2407_17029_b200 import binding as qb  # noqa: E402

DEV = "cuda"


class Block:
    """Four merged min-max weights and the rotary table; buffers for steps of up to `tokens` rows."""

    def __init__(self, hidden, heads, kv_heads, dim, cache, tokens, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        make = lambda o, i: qb.quantize_blockwise(torch.randn(o, i, generator=g, device=DEV) * 0.02, 64, 1,  # noqa: E731
                                                  qb.FMT_AFFINE_MINMAX)
        adapter = qb.Adapter(64, 8, 16, 1.0, (torch.randn(hidden // 64, 16, generator=g, device=DEV) * 0.02).bfloat16(),
                             (torch.randn(16, heads * dim // 8, generator=g, device=DEV) * 0.02).bfloat16())
        self.wq = qb.merge(make(heads * dim, hidden), adapter)                 # a trained adapter folded into the offsets
        self.wk, self.wv, self.wo = make(kv_heads * dim, hidden), make(kv_heads * dim, hidden), make(hidden, heads * dim)
        self.rope = qb.Rope(dim, dim, qb.ROPE_HALF, qb.rope_table(dim))
        self.cache, self.dim = cache, dim
        self.ws = qb.alloc_attention_workspace(cache, torch.empty(tokens, heads, dim, dtype=torch.bfloat16, device=DEV))

    def __call__(self, x, table, plan):
        q, k, v = (qb.lowbit_gemm(w, x).view(x.shape[0], -1, self.dim) for w in (self.wq, self.wk, self.wv))
        q = qb.rope_append(self.rope, plan.positions, plan.slots, q, k, v, self.cache, out_q=q)
        o, _ = qb.paged_attention(q, self.cache, table, plan.cu_new, plan.kv_len, ws=self.ws)
        return qb.lowbit_gemm(self.wo, o.view(x.shape[0], -1))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--page", type=int, default=16)
    ap.add_argument("--prompts", default="700,33,1500,256")
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args()
    prompts = [int(n) for n in a.prompts.split(",")]
    B = len(prompts)
    width = -(-(max(prompts) + a.steps) // a.page)
    n_pages = B * width
    cache = qb.KVCache.empty(n_pages, a.page, a.kv_heads, a.dim)
    block = Block(a.hidden, a.heads, a.kv_heads, a.dim, cache, sum(prompts))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    free, count = torch.arange(n_pages, dtype=torch.int32, device=DEV), i32([n_pages])

    # prompts: one step with all their rows
    x = torch.randn(sum(prompts), a.hidden, device=DEV).bfloat16()
    plan = qb.kv_plan(i32([0] * B), i32(prompts), table, free, count, a.page, sum(prompts))
    y = block(x, table, plan)
    ctx, count = plan.kv_len.clone(), plan.free_count.clone()

    # decode: one row per request; the plan's lengths feed the next step's
    one = i32([1] * B)
    x = torch.randn(B, a.hidden, device=DEV).bfloat16()
    outs = tuple(torch.empty(n, dtype=torch.int32, device=DEV) for n in (B + 1, B, B, B, B, 1))

    def step():
        p = qb.kv_plan(ctx, one, table, free, count, a.page, B, outs=outs)
        out = block(x, table, p)
        ctx.copy_(p.kv_len)
        count.copy_(p.free_count)
        return out

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = step()
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        for _ in range(a.steps - 2):
            graph.replay()
        stop.record()
    side.synchronize()
    assert qb.device_status(block.ws) == qb.OK
    lengths = ctx.tolist()
    assert lengths == [n + a.steps - 1 for n in prompts], lengths
    assert bool(torch.isfinite(y).all())
    print(f"{B} requests, {lengths} cached tokens, {count.item()} pages free, "
          f"{start.elapsed_time(stop) / (a.steps - 2) * 1e3:.1f} us a decode step of one attention block")


if __name__ == "__main__":
    main()
