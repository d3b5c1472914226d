"""AdamW's constructor, set_grads and step on several streams: the results of one stream."""
import pytest
import torch

DEV = "cuda"
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_b200 import binding
    return binding


SIZES = [3000, 256, 70001, 1, 500000]


def _made(qb, **kw):
    g = torch.Generator(device=DEV).manual_seed(3)
    ps = [torch.randn(n, generator=g, device=DEV) for n in SIZES]
    sets = [[torch.randn(n, generator=g, device=DEV) for n in SIZES] for _ in range(3)]
    return qb.AdamW(ps, sets[0], state_bits=8, lr=1e-2, max_norm=1.0, seed=5, **kw), ps, sets


def _state(opt):
    return [t.clone() for ts in (opt.params, opt.m_scale, opt.v_scale) for t in ts] + [t.view(torch.uint8).clone() for t in opt.m + opt.v] + [opt.steps.clone()]


def test_set_grads_and_steps_on_other_streams(qb):
    ref, _, sets = _made(qb)
    for k in range(12):
        ref.set_grads(sets[k % 3])
        ref.step()
    want = _state(ref)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    opt, _, sets = _made(qb)
    torch.cuda.synchronize()
    for k in range(12):
        # the step before may still be in front of this table on its stream: the table waits for it, and the step for the table
        with torch.cuda.stream(streams[k % 2]):
            torch.cuda._sleep(200000)
        opt.set_grads(sets[k % 3], stream=streams[(k // 2) % 2] if k % 3 else None)
        opt.step(stream=streams[k % 2])
    torch.cuda.synchronize()
    assert opt.steps.item() == 12
    assert all(torch.equal(a, b) for a, b in zip(_state(opt), want))


def test_first_step_on_another_stream_than_the_constructor(qb):
    ref, _, _ = _made(qb)
    ref.step()
    want = _state(ref)
    torch.cuda.synchronize()
    side, step = torch.cuda.Stream(), torch.cuda.Stream()
    g = torch.Generator(device=DEV).manual_seed(3)
    ps = [torch.randn(n, generator=g, device=DEV) for n in SIZES]
    gs = [torch.randn(n, generator=g, device=DEV) for n in SIZES]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(3000000)          # the table comes late
    opt = qb.AdamW(ps, gs, state_bits=8, lr=1e-2, max_norm=1.0, seed=5, stream=side)
    opt.step(stream=step)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(_state(opt), want))


def test_a_captured_step_beside_others(qb):
    # captured on a stream of its own, replayed behind set_grads; steps call by call go on as before
    ref, _, sets = _made(qb)
    for k in range(6):
        ref.set_grads(sets[k % 3])
        ref.step()
    want = _state(ref)
    opt, _, sets = _made(qb)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            opt.step()
    torch.cuda.current_stream().wait_stream(side)
    for k in range(6):
        opt.set_grads(sets[k % 3])
        graph.replay() if k % 2 else opt.step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(_state(opt), want))


def test_the_table_outlives_an_optimizer_that_is_dropped(qb):
    # memory of one stream used on another is not handed out again before that one is done
    side = torch.cuda.Stream()
    opt, ps, sets = _made(qb)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100000000)
    opt.step(stream=side)
    made = {t.data_ptr(): t.numel() for t in (opt.ws, opt.steps, opt.lr, opt.norm, *opt.m, *opt.v, *opt.m_scale, *opt.v_scale)}
    del opt
    new = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in made.values() for _ in range(2)]
    assert not side.query() and not any(t.data_ptr() in made for t in new)
    torch.cuda.synchronize()
