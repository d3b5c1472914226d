"""Trains a bank of adapters beside two frozen quantized layers, then serves them from the same bank.

    python examples/train_adapters.py [--hidden 1024] [--inner 2816] [--adapters 4] [--rank 64] [--rows 300,1,77,500] [--steps 8] [--bits 8]

Every sequence of a training step belongs to one adapter (some to none); a step is the plan, both layers forward and backward with the
shared weight's calls and the adapters' calls one after the other, and one AdamW step over all A and B, which writes the banks' bf16
copies itself.  The whole step is captured in a CUDA graph: lengths, adapters and the learning rate live on the device.  Serving replays a
second graph for one token per request, whatever adapters the requests name.  Weights and data are random: what it shows is the
order of the calls, who owns which buffer, and the time of a step.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2407_17029_b200 import binding as qb  # noqa: E402

DEV = "cuda"


class Layer:
    """A frozen weight, its bank of adapters and the buffers of steps of up to `tokens` rows.  The fp32 parameters belong to the
    optimizer; the bank is its bf16 copies."""

    def __init__(self, d_out, d_in, n, rank, tokens, gen, lambda_in=4, lambda_out=4):
        make = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
        self.weight = qb.quantize_blockwise(make(d_out, d_in) / d_in ** 0.5, 64, 1, qb.FMT_AFFINE_MINMAX)
        self.params = [make(n, d_in // lambda_in, rank) / rank, make(n, rank, d_out // lambda_out) * 0.1]
        copies = [p.bfloat16() for p in self.params]
        self.bank = qb.AdapterBank(d_in, d_out, lambda_in, lambda_out, *copies, torch.ones(n, device=DEV))
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.ws = qb.alloc_adapters_workspace(self.bank, tokens)
        self.ws_bwd = qb.alloc_adapters_workspace(self.bank, tokens, backward=True)

    def forward(self, x, plan):
        return qb.adapters_fwd(self.bank, plan, x, qb.linear_fwd(self.weight, None, x), ws=self.ws)

    def backward(self, x, dy, plan, need_dx=True):
        """dX, with the gradients of A and B in self.grads."""
        dx = qb.linear_bwd(self.weight, None, None, dy)[0] if need_dx else None
        return qb.adapters_bwd(self.bank, plan, x, dy, dx, outs=self.grads, ws=self.ws_bwd)[0]

    def serve(self, x, plan):
        return qb.adapters_fwd(self.bank, plan, x, qb.lowbit_gemm(self.weight, x), ws=self.ws)


class Net:
    """x -> silu(first(x)) -> second, with its gradients for the loss sum((y - target)^2) / (2 rows)."""

    def __init__(self, hidden, inner, n, rank, tokens, seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.n, self.tokens = n, tokens
        self.layers = Layer(inner, hidden, n, rank, tokens, gen), Layer(hidden, inner, n, rank, tokens, gen)

    def gradients(self, x, target, plan):
        first, second = self.layers
        h = first.forward(x, plan)
        a = torch.nn.functional.silu(h)
        y = second.forward(a, plan)
        dy = ((y.float() - target.float()) / x.shape[0]).bfloat16()
        da = second.backward(a, dy, plan)
        s = torch.sigmoid(h.float())
        dh = (da.float() * s * (1 + h.float() * (1 - s))).bfloat16()
        first.backward(x, dh, plan, need_dx=False)
        return y

    def serve(self, x, plan):
        return self.layers[1].serve(torch.nn.functional.silu(self.layers[0].serve(x, plan)), plan)


def captured(step):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    side.synchronize()
    return graph


def timed(graph, n):
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(n):
        graph.replay()
    stop.record()
    stop.synchronize()
    return start.elapsed_time(stop) / n * 1e3


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--inner", type=int, default=2816)
    ap.add_argument("--adapters", type=int, default=4)
    ap.add_argument("--rank", type=int, default=64)
    ap.add_argument("--rows", default="300,1,77,500")
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--bits", type=int, default=8)
    a = ap.parse_args()
    rows = [int(n) for n in a.rows.split(",")]
    T, B = sum(rows), len(rows)
    net = Net(a.hidden, a.inner, a.adapters, a.rank, T)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731

    # training
    cu = i32([sum(rows[:b]) for b in range(B + 1)])
    ids = i32([b % (a.adapters + 1) - 1 for b in range(B)])                  # -1: the shared weight alone
    x, target = torch.randn(T, a.hidden, device=DEV).bfloat16(), torch.randn(T, a.hidden, device=DEV).bfloat16()
    lr = torch.full((1,), 1e-3, device=DEV)
    opt = qb.AdamW([p for la in net.layers for p in la.params], [g for la in net.layers for g in la.grads],
                   [c for la in net.layers for c in (la.bank.A, la.bank.B)], state_bits=a.bits, lr=lr, max_norm=1.0)

    def step():
        net.gradients(x, target, qb.adapter_plan(cu, ids, a.adapters, T))
        opt.step()

    graph = captured(step)
    for k in range(a.steps):
        lr.fill_(1e-3 * (1 - k / a.steps))
        graph.replay()
    train = timed(graph, a.steps)
    assert bool(torch.isfinite(opt.norm).all()) and int(opt.steps) == 1 + 2 * a.steps
    assert all(torch.equal(c, p.bfloat16()) for p, c in zip(opt.params, opt.copies))

    # serving: one token per request, any adapters
    cu1, ids1 = i32(list(range(B + 1))), ids.clone()
    x1 = torch.randn(B, a.hidden, device=DEV).bfloat16()
    out = {}

    def decode():
        out["y"] = net.serve(x1, qb.adapter_plan(cu1, ids1, a.adapters, B))

    graph = captured(decode)
    for b in range(B):
        ids1.copy_(ids.roll(b))
        graph.replay()
    serve = timed(graph, a.steps)
    assert bool(torch.isfinite(out["y"]).all())
    assert all(qb.device_status(ws) == qb.OK for la in net.layers for ws in (la.ws, la.ws_bwd))
    print(f"{a.adapters} adapters of rank {a.rank}: {train:.0f} us a training step of {T} rows (gradient norm {float(opt.norm):.3g}), "
          f"{serve:.1f} us a decode step of {B} requests")


if __name__ == "__main__":
    main()
