"""The AdamW step over many tensors on the GPU against the formulas in 64 bits: states in 32 and in 8 bits, clipping, graphs."""
import math

import pytest
import torch

DEV = "cuda"
pytestmark = pytest.mark.gpu
M32 = 0xffffffff
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_b200 import binding
    return binding


def _randn(seed, *shape, dtype=torch.float32, gain=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * gain).to(dtype)


def _wide(codes, scale):
    n = codes.numel()
    return codes.float().double().view(-1) * scale.double().repeat_interleave(256)[:n]


def _states(opt, k, bits):
    """m and v of tensor k in 64 bits."""
    if bits == 32:
        return opt.m[k].double().view(-1), opt.v[k].double().view(-1)
    return _wide(opt.m[k], opt.m_scale[k]), _wide(opt.v[k], opt.v_scale[k]) ** 2


def _formula(p, g, m, v, t, lr, b1=0.9, b2=0.999, eps=1e-8, wd=0.0):
    """p, m, v after the step, and the update with the two terms of m added up by their absolute values: m is off by 2^-22 of
    that sum, which is more than 2^-22 of m where b1 m and (1 - b1) g cancel, and the update by m's error over the same root."""
    size = b1 * m.abs() + (1 - b1) * g.abs()
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    up = (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
    return p - lr * (up + wd * p), m, v, (size / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)


SIZES = [1, 0, 255, 256, 257, 1000, 4096, 65536 + 3, 7, 0, 300000]


def _make(qb, bits, grad=torch.float32, offset=0, copies=True, seed=0, sizes=SIZES, **kw):
    """Tensors of all sizes; `offset` elements into their storage."""
    take = lambda k, n, dtype, gain: _randn(seed + k, n + offset, dtype=dtype, gain=gain)[offset:]  # noqa: E731
    ps = [take(k, n, torch.float32, 0.05) for k, n in enumerate(sizes)]
    gs = [take(100 + k, n, grad, 10.0 ** (k % 5 - 3)) for k, n in enumerate(sizes)]
    cs = [torch.zeros(n + offset, dtype=torch.bfloat16, device=DEV)[offset:] if k % 2 == 0 else None for k, n in enumerate(sizes)] if copies else None
    return qb.AdamW(ps, gs, copies=cs, state_bits=bits, **kw), ps, gs, cs


@pytest.mark.parametrize("offset", [0, 1], ids=["aligned", "offset"])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_against_the_formula(qb, bits, grad, offset):
    # every step is held to the formula on the states that were stored before it
    opt, ps, gs, cs = _make(qb, bits, grad, offset, lr=1e-3, weight_decay=0.1, seed=3)
    for t in range(1, 5):
        before = [(p.double(), *_states(opt, k, bits)) for k, p in enumerate(ps)]
        for k, g in enumerate(gs):
            g.copy_(_randn(1000 * t + k, g.numel(), gain=10.0 ** (k % 5 - 3)))
        opt.step()
        assert opt.steps.item() == t
        for k, (p, m, v) in enumerate(before):
            if p.numel() == 0:
                continue
            want, wm, wv, up = _formula(p, gs[k].double(), m, v, t, float(opt.lr), wd=float(torch.tensor(0.1)))
            assert bool(((ps[k].double() - want).abs() <= 2.0 ** -20 * (float(opt.lr) * up.abs() + p.abs())).all()), (t, k)
            if cs[k] is not None:
                assert torch.equal(cs[k], ps[k].bfloat16())
            gm, gv = _states(opt, k, bits)
            if bits == 32:
                assert bool(((gm - wm).abs() <= 2.0 ** -22 * (m.abs() + gs[k].double().abs())).all())
                assert bool(((gv - wv).abs() <= 2.0 ** -22 * (v + gs[k].double() ** 2)).all())
                continue
            # m is off by 2^-22 of its terms' absolute sum (which matters where they cancel), the root of v by 2^-22 of itself
            for got, want8, off, scale in ((gm, wm, 2.0 ** -22 * (m.abs() + gs[k].double().abs()), opt.m_scale[k]),
                                           (gv.sqrt(), wv.sqrt(), 2.0 ** -22 * wv.sqrt(), opt.v_scale[k])):
                n = got.numel()
                pad = torch.zeros(-n % 256, dtype=torch.float64, device=DEV)
                block = lambda x: torch.cat([x, pad]).view(-1, 256).amax(-1)  # noqa: E731
                top = block(want8.abs())
                assert bool(((scale.double() - top / 448).abs() <= (2.0 ** -22 * top + block(off)) / 448).all())
                s = scale.double().repeat_interleave(256)[:n]
                y = want8.abs() / s.clamp(min=1e-300)
                step = torch.where(y < 2.0 ** -6, torch.full_like(y, 2.0 ** -9), 2.0 ** (torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3))
                # one of the two neighbours: less than a step away (and the rounding of y)
                assert bool(((got.abs() - want8.abs()).abs() <= (step + y * 2.0 ** -20) * s + off).all()), (t, k)


def _mix(x):
    x = ((x ^ (x >> 16)) * 0xA3C59AC3) & M32
    x = ((x ^ (x >> 15)) * 0x5D8E3B97) & M32
    return x ^ (x >> 16)


def test_the_chance_is_the_documented_hash(qb):
    # codes from the documented rule on whole numbers.  beta = 0: m = g and r = |g|, so nothing is rounded in front of it; the gradients'
    # largest magnitude is 448 * 2^-10 in every block, so dividing by the scale is exact too
    sizes = [700, 256, 3, 5000]
    gs = []
    for k, n in enumerate(sizes):
        g = _randn(k, n, gain=0.02).clamp(-0.43, 0.43)
        g[::256] = 448 * 2.0 ** -10
        gs.append(g)
    opt = qb.AdamW([torch.zeros(n, device=DEV) for n in sizes], gs, state_bits=8, betas=(0.0, 0.0), seed=99, steps=torch.tensor([41], dtype=torch.int32, device=DEV))
    opt.step()
    key = (_mix((_mix(torch.tensor(99)) + 42) & M32)).item()
    first = 0
    for k, n in enumerate(sizes):
        e = torch.arange(n, device=DEV) + 256 * first
        first += (n + 255) // 256
        h = _mix((e * 0x9E3779B1 + key) & M32)
        y = gs[k].abs() * 1024
        for codes, scale, bits, signed in ((opt.m[k], opt.m_scale[k], h & 0xffff, True), (opt.v[k], opt.v_scale[k], h >> 16, False)):
            assert bool((scale == 2.0 ** -10).all())
            step = torch.where(y < 2.0 ** -6, torch.full_like(y, 2.0 ** -9), 2.0 ** (torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)).double()
            q = y.double() / step
            low = torch.floor(q)
            want = (low + ((q - low) + bits.double() / 65536 >= 1)) * step
            if signed:
                want = want * gs[k].sign().double()
            got = codes.float().double()
            # r is the square root of a rounded square: a few of its values move by an ulp, and with them hardly a neighbour
            assert torch.equal(got, want) if signed else float((got != want).double().mean()) <= 1e-2


def test_rounding_keeps_the_expected_value(qb):
    # 2^20 equal values between two neighbours: their mean is the value, within five standard deviations of a fair choice
    n = 1 << 20
    g = torch.full((n,), 0.3337, device=DEV)
    g[::256] = 1.0
    opt = qb.AdamW([torch.zeros(n, device=DEV)], [g], state_bits=8, betas=(0.0, 0.0))
    opt.step()
    y = 0.3337 * 448
    step = 2.0 ** (math.floor(math.log2(y)) - 3) / 448
    frac = y / (step * 448) % 1
    inner = torch.ones(n, dtype=torch.bool, device=DEV)
    inner[::256] = False
    for codes, scale in ((opt.m[0], opt.m_scale[0]), (opt.v[0], opt.v_scale[0])):
        got = _wide(codes, scale)[inner]
        assert len(torch.unique(got)) == 2
        assert abs(float(got.mean()) - 0.3337) <= 5 * step * math.sqrt(frac * (1 - frac) / inner.sum().item()) + 1e-6
    # and the two averages' choices, and neighbours', are independent: correlation within five standard deviations
    a, b = ((_wide(c, s) > 0.3337).double() - frac for c, s in ((opt.m[0], opt.m_scale[0]), (opt.v[0], opt.v_scale[0])))
    for x, y in ((a, b), (a[1:], a[:-1]), (a[256:], a[:-256])):
        assert abs(float((x * y).mean())) / (frac * (1 - frac)) <= 5 / math.sqrt(n) + 1.5 / 128    # every 256th is not one of them


def test_slow_averages_keep_moving_in_8_bits(qb):
    # without gradients v decays by beta2 a step: 0.99^200 = 0.134; a single element's way is a walk around that, its mean over 8192 is near it
    n = 8192
    g = _randn(1, n).abs() + 0.5
    g[::256] = 1000.0                                     # keeps the scale large, so that the others decay through the codes
    opt = qb.AdamW([torch.zeros(n, device=DEV)], [g], state_bits=8, betas=(0.9, 0.99), lr=0.0)
    opt.step()
    first = _states(opt, 0, 8)[1]
    g.zero_()
    for k in range(200):
        g[::256] = 1000.0
        opt.step()
    last = _states(opt, 0, 8)[1]
    inner = torch.ones(n, dtype=torch.bool, device=DEV)
    inner[::256] = False
    # codes step by an eighth of themselves at most: E[r'] = r sqrt(0.99) exactly, and the spread of r adds up over 200 steps to
    # at most (1 + 0.125^2 / 4)^200 - 1 = 118 % of r^2 if every step chose evenly; the mean over 8000 is then within 5 * 1.1 / 89 = 6 % of r
    ratio = float(last[inner].sqrt().mean() / first[inner].sqrt().mean())
    assert abs(ratio - 0.99 ** 100) <= 0.08 * 0.99 ** 100


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [1e-4, 1.0], ids=["below", "above"])
def test_clipping_by_the_global_norm(qb, bits, scale):
    opt, ps, gs, _ = _make(qb, bits, seed=5, lr=1e-2, max_norm=0.7, weight_decay=[0.01 * k for k in range(len(SIZES))],
                           lr_mult=[1.0 + k for k in range(len(SIZES))])
    for g in gs:
        g.mul_(scale * 1e-2)
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in gs))
    assert (norm > 0.7) == (scale == 1.0)
    before = [p.double() for p in ps]
    got = opt.step()
    assert got is opt.norm and abs(float(got) - norm) <= 2.0 ** -20 * norm
    factor = min(1.0, 0.7 / norm)
    for k, p in enumerate(before):
        zero = torch.zeros_like(p)
        wd, mult = float(torch.tensor(0.01 * k)), float(1 + k)
        want, _, _, up = _formula(p, gs[k].double() * factor, zero, zero, 1, float(opt.lr) * mult, wd=wd)
        # eps is of the size of nothing here; the factor's rounding cancels in the update
        assert bool(((ps[k].double() - want).abs() <= 2.0 ** -19 * (mult * float(opt.lr) * (up.abs() + wd * p.abs()) + p.abs())).all()), k


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")], ids=["nan", "inf", "-inf"])
def test_gradients_that_are_not_finite(qb, bits, bad):
    # with a norm the step is left out; without one the element alone is lost
    for need in (True, False):
        opt, ps, gs, cs = _make(qb, bits, seed=7, need_norm=need, lr=1e-2)
        opt.step()
        held = [t.clone() for t in (*ps, *opt.m, *opt.v, opt.steps, *(s for s in opt.m_scale if s is not None), *(c for c in cs if c is not None))]
        gs[5][700] = bad
        opt.step()
        now = [t for t in (*ps, *opt.m, *opt.v, opt.steps, *(s for s in opt.m_scale if s is not None), *(c for c in cs if c is not None))]
        if need:
            assert not math.isfinite(float(opt.norm))
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(held, now) if a.numel())
            gs[5][700] = 0.5
            opt.step()
            assert opt.steps.item() == 2 and bool(torch.isfinite(ps[5]).all())
            continue
        assert opt.steps.item() == 2
        other = torch.arange(1000, device=DEV) != 700
        assert bool(torch.isfinite(ps[5][other]).all()) and not bool(torch.isfinite(ps[5][700]))
        m, v = _states(opt, 5, bits)
        assert bool(torch.isfinite(m[other]).all()) and bool(torch.isfinite(v[other]).all())
        if bits == 8:
            assert bool(m[700].isnan()) and bool(v[700].isnan()) and bool(torch.isfinite(opt.m_scale[5]).all())


def test_zero_and_tiny_blocks_in_8_bits(qb):
    # a block of zeros, one below 2^-118, one whose values span more than the codes hold
    g = torch.zeros(768, device=DEV)
    g[256:512] = 2.0 ** -120
    g[512:] = torch.logspace(-12, 0, 256, device=DEV)
    opt = qb.AdamW([torch.ones(768, device=DEV)], [g], state_bits=8, betas=(0.0, 0.0), eps=1.0, lr=1e-3)
    opt.step()
    assert not bool(opt.m[0][:512].view(torch.uint8).any()) and opt.m_scale[0][:2].tolist() == [0.0, 0.0]
    assert bool(torch.isfinite(opt.params[0]).all()) and bool((opt.params[0][:256] == 1.0).all())
    m, _ = _states(opt, 0, 8)
    assert bool(((m[512:] - g[512:].double()).abs() <= torch.maximum(g[512:].double() / 8, torch.tensor(2.0 ** -9 / 448, device=DEV)) * 1.0001).all())
    opt.step()                                            # from zeros: 0 / (0 + eps)
    assert bool(torch.isfinite(opt.params[0]).all())


@pytest.mark.parametrize("size", [1e-16, 1e-8, 1e6, 1e15])
def test_gradients_of_any_size_in_8_bits(qb, size):
    # beta = 0: m = g and r = |g|, each a neighbour of the number itself.  v = g^2 is held in fp32, whose numbers below 2^-126 are 2^-149
    # apart: off by 2^-150 at most, and with it r by 2^-150 / (2 |g|) and the update, g / r, by 2^-150 / (2 g^2) of itself
    g = _randn(3, 5000, gain=size)
    off = 2.0 ** -150 / (2 * g.double().abs())
    opt = qb.AdamW([torch.zeros(5000, device=DEV)], [g], state_bits=8, betas=(0.0, 0.0), eps=0.0, lr=1.0)
    opt.step()
    assert bool(((opt.params[0] + g.sign()).abs() <= 2.0 ** -20 + off / g.double().abs()).all())      # 0 - 1 g / |g|
    for got, want, scale in ((_wide(opt.m[0], opt.m_scale[0]), g.double(), opt.m_scale[0]), (_wide(opt.v[0], opt.v_scale[0]), g.double().abs(), opt.v_scale[0])):
        s = scale.double().repeat_interleave(256)[:5000]
        y = want.abs() / s
        step = torch.where(y < 2.0 ** -6, torch.full_like(y, 2.0 ** -9), 2.0 ** (torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3))
        assert bool(((got - want).abs() <= (step + y * 2.0 ** -20) * s + off).all())


def test_mixed_states_many_tensors_equal_bits(qb):
    # 700 tensors, 8 and 32 bits side by side, equal inputs twice, the same tensors one by one in 32 bits
    sizes = [(37 * k) % 1200 for k in range(700)]
    bits = [8 if k % 3 == 0 else 32 for k in range(700)]
    runs = [_make(qb, bits, sizes=sizes, seed=50, copies=False, lr=1e-2)
            for _ in range(2)]
    for opt, *_ in runs:
        for _ in range(3):
            opt.step()
    same = lambda a, b: a.numel() == 0 or torch.equal(a.view(torch.uint8), b.view(torch.uint8))  # noqa: E731
    (a, *_), (b, *_) = runs
    assert all(same(x, y) for k in ("params", "m", "v") for x, y in zip(getattr(a, k), getattr(b, k)))
    for k in (1, 2, 4, 697):
        one = qb.AdamW([_randn(50 + k, sizes[k], gain=0.05)], [b.grads[k]], lr=1e-2)
        for _ in range(3):
            one.step()
        assert same(one.params[0], a.params[k]) and same(one.v[0], a.v[k])


def test_captured_steps_follow_the_schedule(qb):
    opt, ps, gs, cs = _make(qb, [8 if k % 2 else 32 for k in range(len(SIZES))], seed=11, max_norm=1.0, lr=1e-3)
    ref, ps2, gs2, _ = _make(qb, [8 if k % 2 else 32 for k in range(len(SIZES))], seed=11, max_norm=1.0, lr=1e-3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            opt.step()
    side.synchronize()
    assert opt.steps.item() == 0                          # captured, not run
    for t in range(5):
        for o, grads in ((opt, gs), (ref, gs2)):
            o.lr.fill_(1e-3 / (t + 1))
            for k, g in enumerate(grads):
                g.copy_(_randn(t * 100 + k, g.numel()))
        torch.cuda.synchronize()
        graph.replay()
        ref.step()
    torch.cuda.synchronize()
    assert opt.steps.item() == ref.steps.item() == 5
    assert all(torch.equal(a, b) for a, b in zip(ps, ps2)) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(opt.v, ref.v) if a.numel())


def test_other_gradients_and_kept_states(qb):
    opt, ps, gs, _ = _make(qb, 8, seed=13, lr=1e-3)
    opt.step()
    kept = dict(m=[t.clone() for t in opt.m], v=[t.clone() for t in opt.v], m_scale=[t.clone() for t in opt.m_scale], v_scale=[t.clone() for t in opt.v_scale])
    again = qb.AdamW([p.clone() for p in ps], [g.bfloat16() for g in gs], state_bits=8, states=kept, steps=opt.steps.clone(), lr=opt.lr.clone())
    opt.set_grads([g.bfloat16() for g in gs])
    opt.step()
    again.step()
    assert all(torch.equal(a, b) for a, b in zip(opt.params, again.params)) and opt.steps.item() == again.steps.item() == 2


def test_two_streams_step_side_by_side(qb):
    made = [_make(qb, 8, seed=20 + k, lr=1e-3, max_norm=0.5) for k in range(2)]
    alone = [_make(qb, 8, seed=20 + k, lr=1e-3, max_norm=0.5) for k in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for (opt, *_), s in zip(made, streams):
            opt.step(stream=s)
    torch.cuda.synchronize()
    for opt, *_ in alone:
        for _ in range(10):
            opt.step()
    assert all(torch.equal(a, b) for (o, *_), (p, *_) in zip(made, alone) for a, b in zip(o.params, p.params))


def test_refusals(qb):
    p, g = torch.zeros(10, device=DEV), torch.zeros(10, device=DEV)
    for bad in (lambda: qb.AdamW([], []), lambda: qb.AdamW([p], [g, g]), lambda: qb.AdamW([p], [g[:5]]), lambda: qb.AdamW([p.bfloat16()], [g]),
                lambda: qb.AdamW([p], [g.half()]), lambda: qb.AdamW([p], [g], copies=[p]), lambda: qb.AdamW([p], [g], state_bits=4),
                lambda: qb.AdamW([p], [g.cpu()]), lambda: qb.AdamW([p.view(5, 2).T], [g]), lambda: qb.AdamW([p], [g], states=dict(m=[g.bfloat16()])),
                lambda: qb.AdamW([p], [g], states=dict(x=[g])), lambda: qb.AdamW([p], [g], steps=torch.zeros(1, device=DEV)),
                lambda: qb.AdamW([p], [g], lr=torch.zeros(2, device=DEV)), lambda: qb.AdamW([p], [g]).set_grads([g[:3]])):
        with pytest.raises(ValueError):
            bad()
    for kw in (dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(max_norm=-1.0)):
        with pytest.raises(qb.QbloraError) as e:
            qb.AdamW([p], [g], **kw).step()
        assert e.value.status == qb.ERR_INVALID_ARG
