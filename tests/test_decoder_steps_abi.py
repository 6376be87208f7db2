"""Refusals of the steps between the quantised linears, at the C entry and without a GPU: shapes, pointers and sizes are checked before the
device is touched (the pointers below are made-up numbers and nothing is launched)."""
import ctypes

import pytest

from paper_2608_12932_b200 import binding as B
from paper_2608_12932_b200 import build as libbuild


@pytest.fixture(scope="module", autouse=True)
def built():
    libbuild.build()


def vp(n):
    return ctypes.c_void_p(n)


def cache(codes=0x100000, v=0x200000, ks=0x300000, vs=0x400000, num_blocks=8, heads=2, dim=64, block=16):
    c = B._KV8Struct(codes, v, ks, vs, num_blocks, heads, dim, block)
    return ctypes.byref(c)


def test_norm_refusals():
    f = B.lib().w4a8_add_rmsnorm_quantize
    good = dict(x=vp(0x1000), r=None, w=vp(0x2000), eps=1e-6, M=4, K=256, group=128, s=None, h=None, qa=vp(0x3000), sa=vp(0x4000), asum=vp(0x5000), st=None)

    def code(**k):
        a = {**good, **k}
        return f(a["x"], a["r"], a["w"], a["eps"], a["M"], a["K"], a["group"], a["s"], a["h"], a["qa"], a["sa"], a["asum"], a["st"])
    for bad in (dict(K=200), dict(K=0), dict(K=-128), dict(M=-1), dict(group=64), dict(eps=-1e-6), dict(eps=float("nan"))):
        assert code(**bad) == B.ERR_SHAPE, bad
    assert code(M=0, x=None) == B.OK
    for bad in (dict(x=None), dict(w=None), dict(qa=None), dict(sa=None), dict(asum=None), dict(r=vp(0x6000))):
        assert code(**bad) == B.ERR_NULL, bad
    for bad in (dict(x=vp(0x1008)), dict(w=vp(0x2002)), dict(h=vp(0x7004)), dict(qa=vp(0x3001)), dict(sa=vp(0x4001)), dict(asum=vp(0x5002)),
                dict(r=vp(0x6008), s=vp(0x8000)), dict(r=vp(0x6000), s=vp(0x8008))):
        assert code(**bad) == B.ERR_ALIGN, bad


def test_append_refusals():
    f = B.lib().w4a8_kv8_append
    good = dict(c=cache(), k=vp(0x10000), v=vp(0x20000), ks=128, vs=128, B=3, T=5, table=vp(0x30000), width=4, start=vp(0x40000), count=None,
                ws=vp(0x50000), n=B.WORKSPACE_HEADER_BYTES)

    def code(**k):
        a = {**good, **k}
        return f(a["c"], a["k"], a["v"], a["ks"], a["vs"], a["B"], a["T"], a["table"], a["width"], a["start"], a["count"], a["ws"], a["n"], None)
    for bad in (dict(c=cache(dim=96)), dict(c=cache(block=48)), dict(c=cache(block=256)), dict(c=cache(heads=0)), dict(c=cache(num_blocks=0)),
                dict(c=cache(heads=32768)), dict(B=-1), dict(T=-1), dict(width=0), dict(ks=127), dict(vs=132), dict(ks=64), dict(B=40000), dict(B=30000, T=100000)):
        assert code(**bad) == B.ERR_SHAPE, bad
    assert code(B=0) == B.OK and code(T=0) == B.OK
    for bad in (dict(c=None), dict(k=None), dict(v=None), dict(table=None), dict(start=None), dict(ws=None), dict(c=cache(codes=None)), dict(c=cache(vs=None))):
        assert code(**bad) == B.ERR_NULL, bad
    for bad in (dict(k=vp(0x10008)), dict(v=vp(0x20002)), dict(table=vp(0x30002)), dict(start=vp(0x40001)), dict(count=vp(0x60002)), dict(ws=vp(0x50010)),
                dict(c=cache(codes=0x100008)), dict(c=cache(ks=0x300001))):
        assert code(**bad) == B.ERR_ALIGN, bad
    assert code(n=B.WORKSPACE_HEADER_BYTES - 1) == B.ERR_WORKSPACE


def test_attention_refusals():
    f = B.lib().w4a8_kv8_attention
    need = B.w4a8_kv8_workspace_bytes(64)
    assert need > B.WORKSPACE_ZEROED_BYTES and B.w4a8_kv8_workspace_bytes(128) > need
    assert B.w4a8_kv8_workspace_bytes(96) == 0 and B.w4a8_kv8_workspace_bytes(0) == 0
    good = dict(c=cache(), q=vp(0x10000), qs=384, B=3, T=5, qh=6, table=vp(0x30000), width=4, limits=vp(0x40000), out=vp(0x20000), ws=vp(0x50000), n=need)

    def code(**k):
        a = {**good, **k}
        return f(a["c"], a["q"], a["qs"], a["B"], a["T"], a["qh"], a["table"], a["width"], a["limits"], 0.125, a["out"], a["ws"], a["n"], None)
    for bad in (dict(c=cache(dim=256)), dict(c=cache(block=8)), dict(qh=5), dict(qh=0), dict(qs=380), dict(qs=376), dict(B=-1), dict(T=-2), dict(width=-4),
                dict(B=1, T=2 ** 31 - 1, qh=6), dict(B=1, T=2 ** 30, qh=4), dict(c=cache(heads=1), B=60000, T=30000, qh=1024, qs=65536)):
        assert code(**bad) == B.ERR_SHAPE, bad
    assert code(B=0) == B.OK and code(T=0) == B.OK
    for bad in (dict(c=None), dict(q=None), dict(table=None), dict(limits=None), dict(out=None), dict(ws=None), dict(c=cache(v=None))):
        assert code(**bad) == B.ERR_NULL, bad
    for bad in (dict(q=vp(0x10004)), dict(out=vp(0x20008)), dict(table=vp(0x30001)), dict(limits=vp(0x40002)), dict(ws=vp(0x50080)), dict(c=cache(v=0x200004))):
        assert code(**bad) == B.ERR_ALIGN, bad
    assert code(n=need - 1) == B.ERR_WORKSPACE
    assert B.status_string(B.ERR_INDEX) not in (B.status_string(c) for c in range(8))
