"""Argument checks of the calls for several tokens per sequence, on the host (fake addresses, never dereferenced): every refused call fails
before anything is launched."""
import ctypes as C
import os

import pytest
import torch


@pytest.fixture(scope="module")
def kvq():
    from paper_2502_15075_amd import build, kvq as m
    if not os.path.exists(m.LIB_PATH) or not os.path.exists(build.BINDING):
        build.build_lib()
    m.load()
    return m


def _good(kvq):
    return kvq._CCache(0x10000, 0x20000, 0x30000, 0x40000, v_scale_exp=0x48000)


def test_workspace_sizes(kvq):
    L = kvq.Layout(2, 8, 40000)
    one = kvq.chunk_workspace_bytes(L, 64, 1, 40000)
    counters = 2 * 8 * 8                                             # one word per (sequence, kv head) behind
    assert one > counters and (one - counters) % (2 * 64 * 132 * 4) == 0       # whole records of every row
    assert kvq.window_workspace_bytes(L, 64, 40000, 0, 0) == one
    assert kvq.chunk_workspace_bytes(L, 64, 8192, 40000) == 0         # enough row tiles: nothing to cut
    assert kvq.chunk_workspace_bytes(L, 64, 0, 40000) == 0 and kvq.chunk_workspace_bytes(L, 64, 1, 0) == 0
    for args, code in (((63, 1, 100), kvq.ERR_INVALID_ARG), ((0, 1, 100), kvq.ERR_INVALID_ARG), ((64, -1, 100), kvq.ERR_INVALID_ARG),
                       ((64, 1, -1), kvq.ERR_INVALID_ARG), ((64, 1, 100, -1), kvq.ERR_INVALID_ARG), ((64, 1, 100, 0, -1), kvq.ERR_INVALID_ARG),
                       ((64, 1, 40001), kvq.ERR_CAPACITY), ((72, 1, 100), kvq.ERR_UNSUPPORTED), ((64, 1 << 20, 100), kvq.ERR_UNSUPPORTED)):
        with pytest.raises(kvq.KvqError) as e:
            kvq.chunk_workspace_bytes(L, *args)
        assert e.value.status == code, args
    out = C.c_size_t()
    assert kvq.load().kvq_chunk_workspace_bytes(None, 64, 1, 100, 0, 0, C.byref(out)) == kvq.ERR_INVALID_ARG
    assert kvq.load().kvq_chunk_workspace_bytes(L.c(), 64, 1, 100, 0, 0, None) == kvq.ERR_INVALID_ARG
    assert kvq.load().kvq_window_workspace_bytes(None, 64, 100, 0, 0, C.byref(out)) == kvq.ERR_INVALID_ARG


def test_chunk_attention_refusals(kvq):
    lib, p = kvq.load(), C.c_void_p
    L = kvq.Layout(2, 2, 100)
    good = dict(L=L, cache=_good(kvq), q=0x50000, dt=0, heads=8, sb=8192, st=1024, sh=128, n=8, ql=0, sl=0, bound=100, w=0, s=0,
                scale=0.1, out=0x60000, odt=2, ws=0x70000, wsb=1 << 20)

    def call(**kw):
        a = {**good, **kw}
        return lib.kvq_chunk_attention(a["L"].c() if a["L"] else None, a["cache"], p(a["q"]), a["dt"], a["heads"], a["sb"], a["st"], a["sh"], a["n"],
                                       p(a["ql"]), p(a["sl"]), a["bound"], a["w"], a["s"], C.c_float(a["scale"]), p(a["out"]), a["odt"], p(a["ws"]),
                                       a["wsb"], None)
    bad = [dict(L=None), dict(cache=None), dict(q=0), dict(out=0), dict(q=0x50008), dict(out=0x60004), dict(dt=2), dict(dt=3), dict(odt=3), dict(heads=7),
           dict(heads=0), dict(sb=4), dict(st=1020), dict(sh=120), dict(sh=129), dict(n=-1), dict(bound=-1), dict(w=-1), dict(s=-1), dict(scale=0.0),
           dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(ql=0x80002), dict(sl=0x80001),
           dict(cache=kvq._CCache(0x10000, 0, 0x30000, 0x40000, v_scale_exp=0x48000)), dict(cache=kvq._CCache(0x10008, 0x20000, 0x30000, 0x40000, v_scale_exp=0x48000)),
           dict(L=kvq.Layout(2, 2, 100, page_tokens=64, n_pages=8)), dict(L=kvq.Layout(2, 2, 100, bits_k=5))]
    for kw in bad:
        assert call(**kw) == kvq.ERR_INVALID_ARG, kw
    assert call(bound=101) == kvq.ERR_CAPACITY
    assert call(heads=18) == kvq.ERR_UNSUPPORTED
    assert call(ws=0x70004) == kvq.ERR_WORKSPACE
    resid = kvq._CCache(0x10000, 0x20000, 0x30000, 0x40000, 0x90000, 0xA0000, v_scale_exp=0x48000)
    assert call(L=kvq.Layout(2, 2, 128, axis_k=kvq.AXIS_SEQ), cache=resid) == kvq.ERR_UNSUPPORTED       # channel-wise keys
    assert call(L=kvq.Layout(2, 2, 128, resid_len=64), cache=resid) == kvq.ERR_UNSUPPORTED              # a residual buffer
    assert call(n=0) == kvq.OK and call(n=0, q=0, out=0) == kvq.OK                                       # nothing to do: no launch

    def window(**kw):
        a = {**good, **kw}
        return lib.kvq_window_attention(a["L"].c() if a["L"] else None, a["cache"], p(a["q"]), a["dt"], a["heads"], p(a["sl"]), a["bound"], a["w"], a["s"],
                                        C.c_float(a["scale"]), p(a["out"]), a["odt"], p(a["ws"]), a["wsb"], None)
    for kw in (dict(L=None), dict(cache=None), dict(q=0), dict(out=0x60008), dict(dt=2), dict(odt=-1), dict(heads=3), dict(w=-1), dict(s=-5), dict(scale=0.0),
               dict(sl=0x80002)):
        assert window(**kw) == kvq.ERR_INVALID_ARG, kw
    assert window(bound=101) == kvq.ERR_CAPACITY and window(heads=34) == kvq.ERR_UNSUPPORTED and window(ws=0x70001) == kvq.ERR_WORKSPACE


def test_rope_append_refusals(kvq):
    lib, p = kvq.load(), C.c_void_p
    L = kvq.Layout(2, 2, 100)
    rope = dict(cos=0x100000, sin=0x200000, rows=100, dim=128, inter=0)
    good = dict(L=L, cache=_good(kvq), q=0x50000, qb=8192, qt=1024, qh=128, heads=8, q_out=0x58000, k=0x60000, v=0x68000, dt=0, sb=2048, sh=1024, st=128,
                pos=0x80000, counts=0, n=8, rope=True, **rope)

    def call(**kw):
        a = {**good, **kw}
        r = C.byref(kvq._CRope(a["cos"], a["sin"], a["rows"], a["dim"], a["inter"])) if a["rope"] else None
        return lib.kvq_rope_append(a["L"].c() if a["L"] else None, a["cache"], p(a["q"]), a["qb"], a["qt"], a["qh"], a["heads"], p(a["q_out"]), p(a["k"]),
                                   p(a["v"]), a["dt"], a["sb"], a["sh"], a["st"], p(a["pos"]), p(a["counts"]), a["n"], r, None)
    bad = [dict(L=None), dict(cache=None), dict(rope=False), dict(cos=0), dict(sin=0), dict(cos=0x100008), dict(sin=0x200004), dict(rows=0), dict(dim=8),
           dict(dim=0), dict(dim=144), dict(dim=72), dict(inter=2), dict(q_out=0), dict(q=0x50008), dict(q_out=0x58002), dict(heads=7), dict(heads=0),
           dict(qb=4), dict(qt=1020), dict(qh=64), dict(q=0), dict(q=0, heads=0), dict(k=0), dict(v=0), dict(k=0x60008), dict(v=0x68004), dict(dt=2),
           dict(sb=4), dict(sh=1020), dict(st=120), dict(pos=0), dict(pos=0x80002), dict(counts=0x80001), dict(n=-1),
           dict(L=kvq.Layout(2, 2, 100, bits_k=16, raw_dtype=kvq.KVQ_BF16)), dict(L=kvq.Layout(2, 2, 100, page_tokens=64, n_pages=8))]
    for kw in bad:
        assert call(**kw) == kvq.ERR_INVALID_ARG, kw
    assert call(n=101) == kvq.ERR_CAPACITY
    assert call(heads=18) == kvq.ERR_UNSUPPORTED
    resid = kvq._CCache(0x10000, 0x20000, 0x30000, 0x40000, 0x90000, 0xA0000, v_scale_exp=0x48000)
    assert call(L=kvq.Layout(2, 2, 128, axis_k=kvq.AXIS_SEQ), cache=resid) == kvq.ERR_UNSUPPORTED
    assert call(L=kvq.Layout(2, 2, 128, resid_len=64), cache=resid) == kvq.ERR_UNSUPPORTED
    assert call(n=0) == kvq.OK and call(n=0, k=0, v=0) == kvq.OK                                           # nothing to do: no launch


def test_python_checks(kvq):
    """Shapes and types that the binding itself turns away (CPU tensors: nothing of this reaches the library)."""
    L = kvq.Layout(2, 2, 100)
    t = lambda *s, dtype=torch.float16: torch.zeros(*s, dtype=dtype)
    lens = t(2, dtype=torch.int32)
    with pytest.raises(AssertionError):
        kvq.Rope(t(10, 64, dtype=torch.float32), t(10, 32, dtype=torch.float32))
    with pytest.raises(AssertionError):
        kvq.Rope(t(10, 64), t(10, 64))
    rope = kvq.Rope(t(10, 64, dtype=torch.float32), t(10, 64, dtype=torch.float32))
    k = t(2, 2, 3, 128)
    for args in ((t(2, 3, 8, 128), k, t(2, 2, 4, 128), lens), (t(2, 4, 8, 128), k, k, lens), (t(2, 3, 8, 64), k, k, lens), (None, t(3, 2, 3, 128), t(3, 2, 3, 128), lens),
                 (None, k, k, lens.long()), (None, k, k, None), (t(2, 3, 8, 128, dtype=torch.bfloat16), k, k, lens)):
        with pytest.raises(AssertionError):
            kvq.rope_append(L, None, *args, rope)
    q, out = t(2, 3, 8, 128), t(2, 3, 8, 128)
    for args in ((t(3, 3, 8, 128), None, None, out), (q, lens.long(), None, out), (q, None, t(3, dtype=torch.int32), out), (q, None, None, t(2, 3, 8, 128).transpose(1, 2)),
                 (q, None, None, t(2, 3, 4, 128)), (t(2, 3, 8, 64), None, None, t(2, 3, 8, 64))):
        with pytest.raises(AssertionError):
            kvq.chunk_attention(L, None, args[0], args[1], args[2], 100, 0, 0, 0.1, args[3], None)
    with pytest.raises(AssertionError):
        kvq.window_attention(L, None, q[:, :, 0], None, 100, 0, 0, 0.1, out[:, :, 0], None)
