"""Host-side checks of the serving calls: struct layouts, the rotation table, refusals that come before any launch."""
import ctypes
import math
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
    mirrors = {"qblora_heads": qb._CHeads, "qblora_kv_cache": qb._CKVCache, "qblora_rope_cfg": qb._CRope}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "qblora.h"', 'int main(void) {']
    for s, m in mirrors.items():
        lines.append(f'  printf("{s} %zu\\n", sizeof({s}));')
        lines += [f'  printf("{s}.{f[0]} %zu\\n", offsetof({s}, {f[0]}));' for f in m._fields_]
    lines += ['  printf("enum %d %d %d %d %d\\n", QBLORA_ROPE_HALF, QBLORA_ROPE_PAIRS, QBLORA_ROPE_SCALE_LINEAR, '
              'QBLORA_ROPE_SCALE_BASE, QBLORA_ROPE_SCALE_BANDED);', '  return 0;', '}']
    src, exe = tmp_path / "probe.c", tmp_path / "probe"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(l.split(" ", 1) for l in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for s, m in mirrors.items():
        assert int(out[s]) == ctypes.sizeof(m)
        for f in m._fields_:
            assert int(out[f"{s}.{f[0]}"]) == getattr(m, f[0]).offset
    assert out["enum"].split() == [str(x) for x in (qb.ROPE_HALF, qb.ROPE_PAIRS, qb.ROPE_SCALE_LINEAR, qb.ROPE_SCALE_BASE,
                                                    qb.ROPE_SCALE_BANDED)]


def _turns(t):
    return [(v % (1 << 64)) / 2.0 ** 64 for v in t.tolist()]


def test_rope_table_values(qb):
    # double arithmetic: a few ulp of 2^-53 relative
    close = lambda a, b: all(abs(x - y) <= 1e-14 * y for x, y in zip(a, b))  # noqa: E731
    d, two_pi = 96, 2 * math.pi
    plain = [10000.0 ** (-2 * j / d) / two_pi for j in range(d // 2)]
    assert close(_turns(qb.rope_table(d, device="cpu")), plain)
    assert close(_turns(qb.rope_table(d, scale=qb.ROPE_SCALE_LINEAR, factor=4, device="cpu")), [f / 4 for f in plain])
    b = 10000.0 * 8 ** (d / (d - 2))
    base = _turns(qb.rope_table(d, scale=qb.ROPE_SCALE_BASE, factor=8, device="cpu"))
    assert close(base, [b ** (-2 * j / d) / two_pi for j in range(d // 2)])
    assert close(base[:1], plain[:1]) and abs(base[-1] * 8 / plain[-1] - 1) < 1e-12
    band = _turns(qb.rope_table(d, scale=qb.ROPE_SCALE_BANDED, factor=8, trained_len=4096, slow=1, fast=32, device="cpu"))
    for f, g in zip(plain, band):
        w = min(1.0, max(0.0, (4096 * f - 1) / 31))
        assert abs(g - (f * w + f / 8 * (1 - w))) <= 1e-14 * f
    assert band[0] == plain[0] and abs(band[-1] * 8 / plain[-1] - 1) < 1e-12


@pytest.mark.parametrize("kw", [dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=64, base=1.0), dict(rotary_dim=64, scale=7),
                                dict(rotary_dim=64, scale=1, factor=0.0), dict(rotary_dim=64, scale=1, factor=float("nan")),
                                dict(rotary_dim=2, scale=2, factor=2.0), dict(rotary_dim=64, scale=3, factor=2.0),
                                dict(rotary_dim=64, scale=3, factor=2.0, trained_len=4096, slow=3.0, fast=3.0)])
def test_rope_table_refusals(qb, kw):
    with pytest.raises(qb.QbloraError):
        qb.rope_table(device="cpu", **kw)


P = 0x10000      # an address that is never read: every check below fails on the host first


def _heads(qb, heads=8, dtype=1, data=P, ts=1024, hs=128):
    h = qb._CHeads()
    h.data, h.token_stride, h.head_stride, h.heads, h.dtype = data, ts, hs, heads, dtype
    return h


def _cache(qb, **kw):
    c = qb._CKVCache()
    v = dict(k=P, v=P, page_stride=16 * 256, token_stride=256, head_stride=128, n_pages=4, page_size=16, kv_heads=2, head_dim=128)
    for k, x in {**v, **kw}.items():
        setattr(c, k, x)
    return c


def test_attention_refusals(qb):
    def call(cache=None, q=None, out=None, width=4, B=1, T=3, scale=1.0, window=0, table=P, cu=P, kv=P, lse=None, ws=P, n=1 << 30):
        r = lambda x: ctypes.byref(x)  # noqa: E731
        return qb._lib.qblora_paged_attention(r(cache or _cache(qb)), table, width, cu, kv, B, r(q or _heads(qb)), T, scale, 1,
                                              window, r(out or _heads(qb)), lse, ws, n, None)
    bad = [dict(q=_heads(qb, heads=7)), dict(q=_heads(qb, dtype=0)), dict(out=_heads(qb, dtype=0)), dict(q=_heads(qb, data=P + 2)),
           dict(q=_heads(qb, ts=1023)), dict(out=_heads(qb, hs=129)), dict(out=_heads(qb, heads=16)), dict(q=_heads(qb, data=None)),
           dict(cache=_cache(qb, k=None)), dict(cache=_cache(qb, v=P + 8)), dict(cache=_cache(qb, page_size=0)),
           dict(cache=_cache(qb, head_dim=100)), dict(cache=_cache(qb, n_pages=1 << 28)), dict(cache=_cache(qb, token_stride=260)),
           dict(width=0), dict(B=0), dict(T=0), dict(T=1 << 31), dict(scale=float("nan")), dict(window=-1), dict(table=None),
           dict(cu=P + 1), dict(kv=None), dict(lse=P + 2), dict(width=1 << 28)]
    for kw in bad:
        assert call(**kw) == qb.ERR_INVALID_ARG, kw
    assert call(cache=_cache(qb, head_dim=264)) == qb.ERR_UNSUPPORTED
    assert call(ws=None) == qb.ERR_WORKSPACE and call(n=0) == qb.ERR_WORKSPACE and call(ws=P + 4) == qb.ERR_WORKSPACE
    c = _cache(qb)
    assert qb._lib.qblora_attention_workspace_bytes(ctypes.byref(c), 7, 5) == 0
    assert qb._lib.qblora_attention_workspace_bytes(ctypes.byref(c), 8, 5) >= 256


def test_rope_and_append_refusals(qb):
    cfg = qb._CRope()
    cfg.head_dim, cfg.rotary_dim, cfg.layout, cfg.amplitude, cfg.turns = 128, 64, 0, 1.0, P
    r = ctypes.byref
    def rope(x=None, y=None, x2=None, y2=None, pos=P, T=3):  # noqa: E306
        return qb._lib.qblora_rope(r(cfg), 0, pos, T, r(x or _heads(qb)), r(y or _heads(qb)), r(x2) if x2 else None,
                                   r(y2) if y2 else None, None)
    for kw in [dict(pos=None), dict(T=0), dict(y=_heads(qb, heads=4)), dict(x2=_heads(qb)), dict(x=_heads(qb, dtype=5)),
               dict(x2=_heads(qb, dtype=0), y2=_heads(qb)), dict(x2=_heads(qb), y2=_heads(qb, heads=2)), dict(x=_heads(qb, ts=-1))]:
        assert rope(**kw) == qb.ERR_INVALID_ARG, kw
    for field, value in [("rotary_dim", 63), ("rotary_dim", 130), ("layout", 2), ("amplitude", float("inf")), ("turns", None)]:
        keep = getattr(cfg, field)
        setattr(cfg, field, value)
        assert rope() == qb.ERR_INVALID_ARG, field
        setattr(cfg, field, keep)
    def app(q=None, k=None, v=None, o=None, c=None, slots=P):  # noqa: E306
        return qb._lib.qblora_rope_append(r(cfg), P, slots, 3, r(q or _heads(qb)), r(k or _heads(qb, 2)), r(v or _heads(qb, 2)),
                                          r(o or _heads(qb)), r(c or _cache(qb)), None)
    for kw in [dict(k=_heads(qb, 3)), dict(v=_heads(qb, 2, dtype=0)), dict(o=_heads(qb, dtype=0)), dict(o=_heads(qb, 4)),
               dict(c=_cache(qb, head_dim=64)), dict(slots=None), dict(c=_cache(qb, n_pages=0))]:
        assert app(**kw) == qb.ERR_INVALID_ARG, kw


def test_plan_refusals(qb):
    base = dict(ctx=P, new=P, rel=None, B=4, table=P, width=8, stack=P, cap=64, cnt=P, cnt_out=P + 64, page=16, T=9, cu=P, kv=P,
                pos=P, slots=P, adm=P)
    call = lambda **kw: qb._lib.qblora_kv_plan(*{**base, **kw}.values(), None)  # noqa: E731
    for kw in [dict(ctx=None), dict(new=P + 2), dict(rel=P + 1), dict(B=0), dict(table=None), dict(width=0), dict(cap=0), dict(page=0),
               dict(T=0), dict(cnt_out=P), dict(cu=None), dict(adm=None), dict(cap=1 << 28), dict(width=1 << 28)]:
        assert call(**kw) == qb.ERR_INVALID_ARG, kw
    assert call(B=8193) == qb.ERR_UNSUPPORTED


def test_plan_refuses_arrays_that_overlap():
    # every CTA reads the lengths for itself, so an output over an input (kv_len over ctx_len, the in-place step) is a race.  The
    # check stands before the launch; the call without overlap is not made.
    from paper_2407_17029_b200 import binding as qb
    B, width, cap, T = 4, 8, 64, 9
    sizes = dict(ctx=B, new=B, rel=B, table=B * width, stack=cap, cnt=1, cnt_out=1, cu=B + 1, kv=B, pos=T, slots=T, adm=B)
    addr, at = {}, P
    for name, n in sizes.items():
        addr[name] = at
        at += n * 4
    order = ["ctx", "new", "rel", B, "table", width, "stack", cap, "cnt", "cnt_out", 16, T, "cu", "kv", "pos", "slots", "adm"]
    call = lambda a: qb._lib.qblora_kv_plan(*[a[x] if isinstance(x, str) else x for x in order], None)  # noqa: E731
    read_only = {"ctx", "new", "rel", "cnt"}
    for out in sizes.keys() - read_only:
        for other in sizes.keys() - {out}:
            # the same start, and the output's first word over the other's last one
            for where in (addr[other], addr[other] + (sizes[other] - 1) * 4):
                assert call({**addr, out: where}) == qb.ERR_INVALID_ARG, (out, other)


def test_tables_and_caches_in_host_memory_are_refused(qb):
    import torch
    table = qb.rope_table(64, device="cpu")
    with pytest.raises(ValueError):
        qb.Rope(64, 64, qb.ROPE_HALF, table).c_struct()
    with pytest.raises(ValueError):
        qb.KVCache.empty(4, 16, 2, 64, device="cpu").c_struct()
    assert qb.attention_workspace_bytes(qb.KVCache.empty(4, 16, 2, 64, device="cpu"), 2, 1) >= 256      # sizes can be asked for
    x, pos = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        qb.rope(qb.Rope(64, 64, qb.ROPE_HALF, table), pos, x)


def test_rope_refuses_its_input_in_another_type_or_order(qb):
    # in place means the same elements at the same places; the check stands before the launch, and no call without overlap is made
    cfg = qb._CRope()
    cfg.head_dim, cfg.rotary_dim, cfg.layout, cfg.amplitude, cfg.turns = 128, 64, 0, 1.0, P
    r = ctypes.byref
    Q, K, R = 1 << 20, 2 << 20, 3 << 20
    h = lambda data, heads=2, **kw: _heads(qb, heads, data=data, **kw)  # noqa: E731
    for x, y in [(h(Q, dtype=0), h(Q, dtype=1)), (h(Q), h(Q, ts=2048)), (h(Q), h(Q, hs=256))]:
        assert qb._lib.qblora_rope(r(cfg), 0, P, 3, r(x), r(y), None, None, None) == qb.ERR_INVALID_ARG
        assert qb._lib.qblora_rope(r(cfg), 0, P, 3, r(h(K, dtype=x.dtype)), r(h(R, dtype=y.dtype)), r(x), r(y), None) == qb.ERR_INVALID_ARG
    for y, y2 in [(K, R), (R, Q), (R, R)]:                    # q' over k, k' over q, both to one place
        assert qb._lib.qblora_rope(r(cfg), 0, P, 3, r(h(Q)), r(h(y)), r(h(K)), r(h(y2)), None) == qb.ERR_INVALID_ARG
    for q, o in [(h(Q, dtype=0), h(Q)), (h(Q), h(Q, ts=2048)), (h(Q), h(K)), (h(Q), h(R))]:
        k, v = h(K, dtype=q.dtype), h(R, dtype=q.dtype)
        assert qb._lib.qblora_rope_append(r(cfg), P, P, 3, r(q), r(k), r(v), r(o), r(_cache(qb)), None) == qb.ERR_INVALID_ARG


@pytest.mark.parametrize("page", [1, 8, 16, 64, 256])
def test_attention_refuses_tables_whose_last_tile_passes_31_bits(qb, page):
    # lengths are clamped to width * page_size; rounded up to a tile they still have to be a 32-bit number
    r = lambda x: ctypes.byref(x)  # noqa: E731
    for keys, want in (((1 << 31) - page, qb.ERR_WORKSPACE if page == 256 else qb.ERR_INVALID_ARG), ((1 << 31) - 256, qb.ERR_WORKSPACE)):
        got = qb._lib.qblora_paged_attention(r(_cache(qb, page_size=page, page_stride=page * 256)), P, keys // page, P, P, 1, r(_heads(qb)), 3,
                                             1.0, 1, 0, r(_heads(qb)), None, None, 0, None)
        assert got == want, (page, keys)
