"""The operators for many adapters in one run: training steps (plan, forward, backward, AdamW) and decoding from the same bank."""
import importlib.util
import os
import random
import subprocess
import sys

import pytest
import torch

from tests import _adapters as ra
from tests._adapters import DEV

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_b200 import binding
    return binding


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_adapters", os.path.join(ROOT, "examples", "train_adapters.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _weight(qb, layer):
    """The dequantized weight, [d_out][d_in]: the product with the unit matrix."""
    d_in = layer.bank.d_in
    return qb.linear_fwd(layer.weight, None, torch.eye(d_in, device=DEV).bfloat16(), torch.float32).double().T


@pytest.mark.parametrize("args", [[], ["--hidden", "512", "--inner", "768", "--adapters", "2", "--rank", "8", "--rows", "1", "--bits", "32"],
                                  ["--rows", "1500,1,0,33,700,16", "--adapters", "9", "--rank", "256", "--steps", "3"]], ids=["default", "small", "uneven"])
def test_example_runs(args):
    done = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "train_adapters.py")] + args, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stdout + done.stderr
    assert "us a training step" in done.stdout


@pytest.mark.parametrize("rows", [[70, 1, 0, 33], [600, 900, 130, 1, 40]], ids=["few", "many"])
def test_example_gradients(qb, example, rows):
    # against automatic differentiation in 64 bits of the same formulas on the dequantized weights
    n, T = 3, sum(rows) + 5                                  # five rows that belong to no sequence
    net = example.Net(256, 512, n, 32, T, seed=4)
    ids = [b % (n + 1) - 1 for b in range(len(rows))]
    cu, di, _ = ra.requests(rows, ids)
    g = torch.Generator(device=DEV).manual_seed(7)
    x, target = (torch.randn(T, 256, generator=g, device=DEV).bfloat16() for _ in range(2))
    y = net.gradients(x, target, qb.adapter_plan(cu, di, n, T))
    leaves = [t.double().requires_grad_() for la in net.layers for t in (la.bank.A, la.bank.B)]
    cu = cu.tolist()

    def layer(la, A, B, x):
        out = x @ _weight(qb, la).T
        term = torch.zeros_like(out)
        for b, a in enumerate(ids):
            if a >= 0:
                t = slice(cu[b], cu[b + 1])
                z = x[t].reshape(-1, A.shape[1], la.bank.lambda_in).mean(-1) @ A[a] @ B[a] * float(la.bank.scaling[a])
                term[t] = z.repeat_interleave(la.bank.lambda_out, 1)
        return out + term

    want = layer(net.layers[1], leaves[2], leaves[3], torch.nn.functional.silu(layer(net.layers[0], leaves[0], leaves[1], x.double())))
    (0.5 * (want - target.double()).square().sum() / T).backward()
    # Between the calls h, a, y, dy, da, dh are bf16, each within 2^-8 of itself, and so is the shared projection's output before the
    # adapter's term: eight roundings on the longest way, which pass through products that keep the size of what they get: 8 2^-8 = 2^-5.
    for got, ref in [(y, want.detach())] + [(got, leaf.grad) for got, leaf in zip([g for la in net.layers for g in la.grads], leaves)]:
        assert float((got.double() - ref).norm()) <= 2.0 ** -5 * float(ref.norm())


def test_captured_training_is_the_uncaptured_one(qb, example):
    # three steps of other batches each, by one graph and call by call: the same bits in every parameter, state and copy
    n, T, B = 4, 640, 6

    def run(graphed):
        net = example.Net(256, 384, n, 64, T, seed=2)
        gen = torch.Generator(device=DEV).manual_seed(3)
        x, target = (torch.randn(T, 256, generator=gen, device=DEV).bfloat16() for _ in range(2))
        cu, ids = torch.zeros(B + 1, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
        lr = torch.zeros(1, device=DEV)
        opt = qb.AdamW([p for la in net.layers for p in la.params], [g for la in net.layers for g in la.grads],
                       [c for la in net.layers for c in (la.bank.A, la.bank.B)], state_bits=[8, 32, 32, 8], lr=lr, max_norm=0.5, seed=11)

        def step():
            net.gradients(x, target, qb.adapter_plan(cu, ids, n, T))
            opt.step()

        if graphed:
            kept = [[t.clone() for t in ts] for ts in (opt.params, opt.copies)]
            graph = example.captured(step)                   # runs one step with a learning rate of 0 and no rows
            for ts, ks in zip((opt.params, opt.copies), kept):
                assert all(torch.equal(t, k) for t, k in zip(ts, ks))
            opt.steps.zero_()
            for t in opt.m + opt.v:
                t.view(torch.uint8).zero_()
        r = random.Random(5)
        for k in range(3):
            lens = [r.randrange(0, T // B) for _ in range(B)]
            cu.copy_(torch.tensor([sum(lens[:b]) for b in range(B + 1)], dtype=torch.int32))
            ids.copy_(torch.tensor([r.randrange(-1, n) for _ in range(B)], dtype=torch.int32))
            lr.fill_(1e-2 / (k + 1))
            graph.replay() if graphed else step()
        torch.cuda.synchronize()
        assert int(opt.steps) == 3
        return [t.view(torch.uint8) for ts in (opt.params, opt.copies, opt.m, opt.v) for t in ts] + [opt.norm]

    assert all(torch.equal(a, b) for a, b in zip(run(False), run(True)))


def test_served_bank_against_the_layer_with_one_adapter(qb):
    # every request's rows as the layer with that adapter alone gives them
    n, d_in, d_out = 5, 512, 768
    bank = ra.make_bank(qb, n, d_in, d_out, 4, 8, 32, seed=6, gain=0.3)
    g = torch.Generator(device=DEV).manual_seed(1)
    qw = qb.quantize_blockwise(torch.randn(d_out, d_in, generator=g, device=DEV) / d_in ** 0.5, 64, 1, qb.FMT_AFFINE_MINMAX)
    for lens, ids in (([1] * 9, [0, 4, -1, 2, 2, 1, 3, -1, 0]), ([1, 200, 7, 1, 390], [3, 1, -1, 1, 4])):
        cu, di, T = ra.requests(lens, ids)
        X = torch.randn(T, d_in, generator=g, device=DEV).bfloat16()
        Y = qb.adapters_fwd(bank, qb.adapter_plan(cu, di, n, T), X, qb.lowbit_gemm(qw, X))
        for b, a in enumerate(ids):
            t = slice(int(cu[b]), int(cu[b + 1]))
            one = None if a < 0 else qb.Adapter(4, 8, 32, float(bank.scaling[a]), bank.A[a], bank.B[a])
            want = qb.linear_fwd(qw, one, X[t]).double()
            # both within 1e-2 of the formula in root mean square (linear_fwd's and lowbit_gemm's bound); one rounding more here
            assert float((Y[t].double() - want).norm()) <= (2e-2 + 2.0 ** -8) * float(want.norm())


def test_two_host_threads_on_their_own_streams(qb):
    # sizes of both forward paths, gradients in parts, a step each time: the bits of the calls alone
    import threading
    problems, alone, errors = [], [], []
    for k, (size, lens, ids) in enumerate((((512, 768, 4, 4, 64), [700, 1, 30], [0, 1, 1]), ((1024, 512, 8, 2, 128), [1] * 40, [b % 3 for b in range(40)]))):
        bank = ra.make_bank(qb, 3, *size, seed=40 + k)
        cu, di, T = ra.requests(lens, ids)
        g = torch.Generator(device=DEV).manual_seed(k)
        X, Y, dY = (torch.randn(T, w, generator=g, device=DEV).bfloat16() for w in (size[0], size[1], size[1]))
        problems.append((bank, cu, di, T, X, Y, dY, torch.randn(bank.A.shape, generator=g, device=DEV)))

    def once(bank, cu, di, T, X, Y, dY, param):
        plan = qb.adapter_plan(cu, di, 3, T)
        y = qb.adapters_fwd(bank, plan, X, Y.clone())
        dx, dA, dB = qb.adapters_bwd(bank, plan, X, dY, torch.zeros(X.shape, device=DEV))
        p = param.clone()
        qb.AdamW([p], [dA], state_bits=8, lr=1e-2, max_norm=1.0).step()
        return y, dx, dA, dB, p

    alone = [once(*problem) for problem in problems]
    torch.cuda.synchronize()
    start = threading.Barrier(2)

    def worker(k):
        try:
            stream = torch.cuda.Stream()
            start.wait()
            with torch.cuda.stream(stream):
                for _ in range(25):
                    got = once(*problems[k])
                    stream.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, alone[k])):
                        errors.append(k)
        except Exception as ex:      # surface in the main thread
            errors.append(repr(ex))

    threads = [threading.Thread(target=worker, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
