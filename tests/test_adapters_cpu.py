"""Host-side checks of the calls for many adapters and of the AdamW step: struct layouts, refusals before any launch."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_b200 import build
    build.build()
    from paper_2407_17029_b200 import binding
    return binding


def test_struct_layouts_match_the_header(qb, tmp_path):
    mirrors = {"qblora_adapter_bank": qb._CAdapterBank, "qblora_adamw_tensor": qb._CAdamWTensor, "qblora_adamw_cfg": qb._CAdamWCfg}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "qblora.h"', 'int main(void) {']
    for s, m in mirrors.items():
        lines.append(f'  printf("{s} %zu\\n", sizeof({s}));')
        lines += [f'  printf("{s}.{f[0]} %zu\\n", offsetof({s}, {f[0]}));' for f in m._fields_]
    lines += ['  return 0;', '}']
    src, exe = tmp_path / "probe.c", tmp_path / "probe"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(l.split(" ", 1) for l in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for s, m in mirrors.items():
        assert int(out[s]) == ctypes.sizeof(m)
        for f in m._fields_:
            assert int(out[f"{s}.{f[0]}"]) == getattr(m, f[0]).offset


def _bank(qb, **kw):
    b = dict(d_in=256, d_out=512, lambda_in=4, lambda_out=8, n_adapters=3, rank=16, A=0x1000, B=0x2000, scaling=0x3000, ranks=None)
    b.update(kw)
    return qb._CAdapterBank(**b)


def _fwd(qb, bank, **kw):
    a = dict(rows=0x4000, start=0x5000, X=0x6000, xs=256, T=5, Y=0x7000, ys=512, dtype=1, ws=0x8000, bytes=1 << 30)
    a.update(kw)
    return qb._lib.qblora_adapters_fwd(ctypes.byref(bank) if bank is not None else None, a["rows"], a["start"], a["X"], a["xs"], a["T"], a["Y"],
                                       a["ys"], a["dtype"], a["ws"], a["bytes"], None)


def _bwd(qb, bank, **kw):
    a = dict(rows=0x4000, start=0x5000, X=0x6000, xs=256, dY=0x7000, ys=512, T=5, dX=0x9000, gs=256, dtype=1, dA=0xa000, dB=0xb000, ws=0x8000,
             bytes=1 << 30)
    a.update(kw)
    return qb._lib.qblora_adapters_bwd(ctypes.byref(bank), a["rows"], a["start"], a["X"], a["xs"], a["dY"], a["ys"], a["T"], a["dX"], a["gs"],
                                       a["dtype"], a["dA"], a["dB"], a["ws"], a["bytes"], None)


def test_adapter_calls_refuse_on_the_host(qb):
    for kw in (dict(d_in=0), dict(lambda_in=0), dict(lambda_in=3), dict(lambda_out=5), dict(n_adapters=0), dict(rank=0), dict(A=None),
               dict(B=None), dict(scaling=None), dict(A=0x1001), dict(scaling=0x3002), dict(ranks=0x3001)):
        assert _fwd(qb, _bank(qb, **kw)) == qb.ERR_INVALID_ARG, kw
        assert _bwd(qb, _bank(qb, **kw)) == qb.ERR_INVALID_ARG, kw
    assert _fwd(qb, None) == qb.ERR_INVALID_ARG
    for kw in (dict(rows=None), dict(start=0x5002), dict(X=None), dict(X=0x6001), dict(xs=255), dict(T=0), dict(T=-1), dict(Y=None),
               dict(ys=511), dict(dtype=2), dict(Y=0x7002, dtype=0), dict(Y=0x6000)):
        assert _fwd(qb, _bank(qb), **kw) == qb.ERR_INVALID_ARG, kw
    for kw in (dict(ws=None), dict(ws=0x8008), dict(bytes=16)):
        assert _fwd(qb, _bank(qb), **kw) == qb.ERR_WORKSPACE, kw
        assert _bwd(qb, _bank(qb), **kw) == qb.ERR_WORKSPACE, kw
    for kw in (dict(dY=None), dict(ys=511), dict(X=None), dict(xs=3), dict(gs=255), dict(dtype=3), dict(dA=0xa002), dict(dB=0xa000),
               dict(dX=0x6000), dict(dX=0x7000), dict(T=0)):
        assert _bwd(qb, _bank(qb), **kw) == qb.ERR_INVALID_ARG, kw
    assert _fwd(qb, _bank(qb), T=1 << 31) == qb.ERR_UNSUPPORTED
    assert _fwd(qb, _bank(qb, n_adapters=4097)) == qb.ERR_UNSUPPORTED
    assert _bwd(qb, _bank(qb), dX=None, dA=None, dB=None) == qb.OK          # nothing wanted


def test_workspace_sizes_grow_with_the_call(qb):
    size = lambda b, T, back: qb._lib.qblora_adapters_workspace_bytes(ctypes.byref(b), T, back)  # noqa: E731
    b = _bank(qb, A=None, B=None, scaling=None)                             # sizes alone decide
    assert 0 < size(b, 1, 0) <= size(b, 100, 0) <= size(b, 100, 1)
    assert size(b, 0, 0) == 0 and size(_bank(qb, lambda_in=3), 5, 0) == 0


def _plan(qb, **kw):
    a = dict(cu=0x1000, ids=0x2000, R=4, n=3, T=9, rows=0x3000, start=0x4000)
    a.update(kw)
    return qb._lib.qblora_adapter_plan(a["cu"], a["ids"], a["R"], a["n"], a["T"], a["rows"], a["start"], None)


def test_plan_refuses_on_the_host(qb):
    for kw in (dict(cu=None), dict(ids=0x2001), dict(rows=None), dict(start=0x4003), dict(R=0), dict(n=0), dict(T=0),
               dict(rows=0x1004), dict(start=0x1010), dict(rows=0x2000), dict(start=0x3020)):
        assert _plan(qb, **kw) == qb.ERR_INVALID_ARG, kw
    for kw in (dict(R=8193, ids=0x100000), dict(n=4097, start=0x200000), dict(T=1 << 31, rows=1 << 40)):
        assert _plan(qb, **kw) == qb.ERR_UNSUPPORTED, kw


def _tensor(qb, **kw):
    t = dict(p=0x1000, g=0x2000, copy=None, m=0x3000, v=0x4000, m_scale=0x5000, v_scale=0x6000, n=10, g_dtype=0, state_bits=32, lr_mult=1.0,
             weight_decay=0.0)
    t.update(kw)
    return qb._CAdamWTensor(**t)


def test_adamw_refuses_on_the_host(qb):
    blocks = ctypes.c_int64()
    prep = lambda t, n=1, ws=0x10000, size=1 << 20, out=ctypes.byref(blocks): qb._lib.qblora_adamw_prepare(  # noqa: E731
        ctypes.byref(t) if t is not None else None, n, ws, size, out, None)
    inf = float("inf")
    for kw in (dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(p=0x1002), dict(g=0x2002), dict(g=0x2001, g_dtype=1),
               dict(copy=0x7001), dict(m=0x3001), dict(n=-1), dict(g_dtype=2), dict(state_bits=16), dict(state_bits=8, m_scale=None),
               dict(state_bits=8, v_scale=0x6001), dict(lr_mult=inf), dict(weight_decay=float("nan"))):
        assert prep(_tensor(qb, **kw)) == qb.ERR_INVALID_ARG, kw
    assert prep(None) == qb.ERR_INVALID_ARG and prep(_tensor(qb), out=None) == qb.ERR_INVALID_ARG
    assert prep(_tensor(qb), ws=None) == qb.ERR_WORKSPACE and prep(_tensor(qb), size=16) == qb.ERR_WORKSPACE
    assert prep(_tensor(qb, n=1 << 40)) == qb.ERR_UNSUPPORTED
    assert qb._lib.qblora_adamw_workspace_bytes(0) == 0 and qb._lib.qblora_adamw_workspace_bytes(65537) == 0
    assert 0 < qb._lib.qblora_adamw_workspace_bytes(1) < qb._lib.qblora_adamw_workspace_bytes(600)

    def step(n=1, blocks=1, ws=0x10000, size=1 << 20, **kw):
        c = dict(lr=0x1000, steps=0x2000, beta1=0.9, beta2=0.999, eps=1e-8, max_norm=0.0, seed=0, norm=None)
        c.update(kw)
        return qb._lib.qblora_adamw_step(ctypes.byref(qb._CAdamWCfg(**c)), n, blocks, ws, size, None)

    for kw in (dict(n=0), dict(n=65537), dict(blocks=-1), dict(blocks=1 << 31), dict(lr=None), dict(steps=0x2002), dict(norm=0x3001), dict(beta1=1.0),
               dict(beta1=-0.1), dict(beta2=float("nan")), dict(eps=-1.0), dict(eps=inf), dict(max_norm=-1.0), dict(max_norm=inf)):
        assert step(**kw) == qb.ERR_INVALID_ARG, kw
    assert step(ws=None) == qb.ERR_WORKSPACE and step(size=16) == qb.ERR_WORKSPACE


@pytest.mark.parametrize("backward", [0, 1])
def test_a_workspace_for_more_rows_serves_fewer(qb, backward):
    # alloc_adapters_workspace(bank, tokens) promises "up to `tokens` rows": the size never falls as the rows grow
    for P, Q, rank, n in ((1000, 32, 128, 50), (1024, 1024, 256, 3), (216, 640, 256, 6), (4096, 2752, 64, 1), (16, 8, 8, 4096), (4096, 4096, 1024, 2), (7, 9, 5, 3)):
        bank = qb._CAdapterBank(2 * P, 4 * Q, 2, 4, n, rank, None, None, None, None)
        sizes = [qb._lib.qblora_adapters_workspace_bytes(ctypes.byref(bank), T, backward) for T in list(range(1, 1500)) + list(range(1500, 40000, 97))]
        assert all(s > 0 for s in sizes) and sizes == sorted(sizes)


def test_gradients_that_overlap_are_refused(qb):
    # dA: 3 x 64 x 16, dB: 3 x 16 x 64 numbers of four bytes
    for dA, dB in ((0x60000, 0x60000), (0x60000, 0x60000 + 3 * 64 * 16 * 4 - 4), (0x60000 + 4, 0x60000)):
        assert _bwd(qb, _bank(qb), dA=dA, dB=dB) == qb.ERR_INVALID_ARG
