"""Refusals of the selection, grouping and adapter entry points, without device work."""
import ctypes as C

import pytest
import torch

import paper_2606_15453_b200 as P

BAD = -1
X = C.c_void_p(1 << 20)      # an aligned address that no refused call may touch
Y, Z = C.c_void_p(1 << 24), C.c_void_p(1 << 28)
ODD, TWO = C.c_void_p((1 << 20) + 1), C.c_void_p((1 << 20) + 2)


def _select(**kw):
    a = dict(z=X, dt=0, st=8, bias=None, mask=None, T=4, E=8, K=2, G=1, top=1, best=1, flags=0, scale=1.0, ids=X, w=X)
    a.update(kw)
    return P.lib().stmoe_router_select(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(z=None), dict(ids=None), dict(w=None), dict(dt=2), dict(dt=3), dict(dt=5), dict(st=7), dict(T=-1), dict(T=1 << 30), dict(E=0),
                                dict(E=257, st=300), dict(K=0), dict(K=9), dict(E=64, st=64, K=33), dict(G=0), dict(G=3), dict(E=64, st=64, G=64), dict(top=0),
                                dict(top=2), dict(G=2, top=3), dict(best=0), dict(best=3), dict(flags=4), dict(flags=-1), dict(scale=float("inf")),
                                dict(scale=float("nan")), dict(z=ODD), dict(z=TWO), dict(ids=TWO), dict(w=TWO), dict(bias=TWO)])
def test_router_select_refusals(kw):
    assert _select(**kw) == BAD


def _selectb(**kw):
    a = dict(z=X, dt=0, st=8, T=4, E=8, K=2, flags=0, scale=1.0, ids=X, w=X, g=X, d=Y, ds=8)
    a.update(kw)
    return P.lib().stmoe_router_select_backward(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(z=None), dict(ids=None), dict(w=None), dict(g=None), dict(d=None), dict(ds=7), dict(st=7), dict(K=9), dict(flags=4),
                                dict(scale=float("nan")), dict(d=X), dict(d=C.c_void_p((1 << 20) + 64)), dict(d=C.c_void_p((1 << 20) - 64)), dict(g=TWO)])
def test_router_select_backward_refusals(kw):
    assert _selectb(**kw) == BAD


def test_calls_without_rows_do_nothing():
    assert _select(T=0) == 0 and _selectb(T=0) == 0 and _dispatch(T=0) == 0 and _combine(T=0) == 0 and _combineb(T=0) == 0 and _lora(T=0) == 0


def _group(**kw):
    a = dict(ids=X, T=4, K=2, n=8, counts=X, starts=X, order=X, slots=X, scratch=X, size=1 << 20)
    a.update(kw)
    return P.lib().stmoe_group_rows(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(ids=None), dict(counts=None), dict(starts=None), dict(order=None), dict(slots=None), dict(T=-1), dict(T=1 << 30), dict(T=(1 << 29) + 1), dict(K=0),
                                dict(n=0), dict(n=1025), dict(T=1 << 20, scratch=None), dict(T=1 << 20, size=64), dict(T=1 << 20, scratch=TWO), dict(ids=TWO),
                                dict(counts=ODD), dict(starts=TWO), dict(order=TWO), dict(slots=TWO)])
def test_group_rows_refusals(kw):
    assert _group(**kw) == BAD


def test_scratch_sizes_do_not_fall():
    f = P.lib().stmoe_group_rows_scratch_bytes
    sizes = [f(1 << i, 8, 256) for i in range(28)]
    assert sizes == sorted(sizes) and sizes[0] == 0 and f(4, 2, 0) == f(4, 2, 1025) == f(-1, 2, 4) == 0
    for f in (P.lib().stmoe_lora_scratch_bytes, P.lib().stmoe_lora_backward_scratch_bytes):
        assert f(4, 0, 16, 64, 64) == f(4, 4, 257, 64, 64) == f(4, 4, 16, 0, 64) == f(4, 1025, 16, 64, 64) == f(-1, 4, 16, 64, 64) == 0
        assert f(4, 4, 16, 4096, 4096) >= 4 * 16 * 4
        for n in (1, 7, 200):
            sizes = [f(tokens, n, 24, 1000, 300) for tokens in sorted({1 << i for i in range(18)} | set(range(1, 9000, 37)))]
            assert sizes == sorted(sizes)


def _dispatch(**kw):
    a = dict(x=X, bytes=64, xs=64, T=4, K=2, slots=X, n=None, out=Y, rows=8, os=64)
    a.update(kw)
    return P.lib().stmoe_dispatch_rows(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(out=None), dict(slots=None), dict(bytes=0), dict(xs=63), dict(os=63), dict(T=-1), dict(T=1 << 30), dict(K=0),
                                dict(rows=-1), dict(rows=1 << 31), dict(slots=TWO), dict(n=TWO), dict(out=X), dict(out=C.c_void_p((1 << 20) + 128)),
                                dict(bytes=1 << 31, xs=1 << 31, os=1 << 31)])
def test_dispatch_rows_refusals(kw):
    assert _dispatch(**kw) == BAD


def _combine(**kw):
    a = dict(y=X, ydt=1, ys=64, yrows=8, slots=X, w=X, res=None, rs=64, scale=1.0, T=4, K=2, cols=64, out=Y, odt=1, os=64)
    a.update(kw)
    return P.lib().stmoe_combine_rows(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(y=None), dict(slots=None), dict(out=None), dict(ydt=2), dict(odt=4), dict(ydt=0), dict(ys=63), dict(os=63), dict(yrows=-1),
                                dict(cols=0), dict(T=-1), dict(K=0), dict(res=Z, rs=63), dict(res=C.c_void_p((1 << 24) + 128)), dict(out=X), dict(y=ODD),
                                dict(w=TWO), dict(slots=TWO), dict(res=ODD), dict(out=C.c_void_p((1 << 24) + 2), odt=0)])
def test_combine_rows_refusals(kw):
    assert _combine(**kw) == BAD


def _combineb(**kw):
    a = dict(g=Z, gdt=1, gs=64, y=X, ydt=1, ys=64, yrows=8, slots=X, w=X, scale=1.0, T=4, K=2, cols=64, n=None, dy=Y, dys=64, dw=X)
    a.update(kw)
    return P.lib().stmoe_combine_rows_backward(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(g=None), dict(y=None), dict(dy=None), dict(slots=None), dict(gdt=4), dict(gdt=2), dict(gs=63), dict(ys=63), dict(dys=63),
                                dict(cols=0), dict(dy=X), dict(dy=Z), dict(dw=TWO), dict(n=TWO), dict(w=ODD)])
def test_combine_rows_backward_refusals(kw):
    assert _combineb(**kw) == BAD


def _lora(**kw):
    a = dict(x=X, dt=1, xs=64, T=4, a=X, ag=1024, ar=64, b=X, bg=1024, br=16, n=2, r=16, I=64, O=64, ids=X, order=X, counts=X, starts=X, scale=None, alpha=1.0, base=None, bs=64,
             out=Y, odt=1, os=64, hidden=None, scratch=X, size=1 << 20)
    a.update(kw)
    return P.lib().stmoe_lora(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(a=None), dict(b=None), dict(ids=None), dict(order=None), dict(counts=None), dict(starts=None), dict(out=None), dict(scratch=None), dict(size=64),
                                dict(dt=0), dict(dt=2), dict(odt=4), dict(xs=63), dict(ar=63), dict(br=15), dict(os=63), dict(base=Z, bs=63), dict(T=-1), dict(n=0),
                                dict(n=1025), dict(r=0), dict(r=257, br=300), dict(I=0), dict(O=0), dict(I=1 << 25, xs=1 << 25, ar=1 << 25), dict(ag=-1), dict(out=X),
                                dict(base=C.c_void_p((1 << 24) + 128)), dict(x=ODD), dict(a=ODD), dict(b=ODD), dict(ids=TWO), dict(order=TWO), dict(scale=TWO),
                                dict(hidden=TWO), dict(scratch=C.c_void_p((1 << 20) + 8))])
def test_lora_refusals(kw):
    assert _lora(**kw) == BAD


def _lorab(**kw):
    a = dict(g=Z, dt=1, gs=64, x=X, xs=64, T=4, a=X, ag=1024, ar=64, b=X, bg=1024, br=16, n=2, r=16, I=64, O=64, ids=X, order=X, counts=X, starts=X, scale=None,
             alpha=1.0, hidden=X, dx=Y, dxs=64, da=X, db=X, scratch=X, size=1 << 24)
    a.update(kw)
    return P.lib().stmoe_lora_backward(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(g=None), dict(x=None), dict(a=None), dict(b=None), dict(ids=None), dict(order=None), dict(counts=None), dict(starts=None),
                                dict(hidden=None), dict(dx=None), dict(scratch=None), dict(size=1024), dict(dt=0), dict(gs=63), dict(dxs=63), dict(dx=X), dict(dx=Z),
                                dict(da=ODD), dict(db=ODD), dict(hidden=TWO), dict(scratch=C.c_void_p((1 << 20) + 16)), dict(r=300, br=300)])
def test_lora_backward_refusals(kw):
    assert _lorab(**kw) == BAD


def test_binding_refuses_before_the_library():
    x, i = torch.zeros(4, 64), torch.zeros(4, 2, dtype=torch.int32)
    plan = {"slots": i, "starts": i, "counts": i, "order": i, "ids": i, "groups": 2}
    w = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    for call in (lambda: P.router_select(x, 2), lambda: P.router_select_backward(x, {}, x), lambda: P.group_rows(i, 4), lambda: P.dispatch_rows(x, plan),
                 lambda: P.combine_rows(x, plan), lambda: P.combine_rows_backward(x, x, plan), lambda: P.lora(x.bfloat16(), w, w, plan),
                 lambda: P.lora_backward(x.bfloat16(), x.bfloat16(), w, w, plan, x)):
        with pytest.raises(P.StmoeError):
            call()


def test_constants_match_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(P.__file__))), "include", "stmoe.h")).read()
    for name, value in (("SIGMOID", P.binding.SELECT_SIGMOID), ("RENORM", P.binding.SELECT_RENORM)):
        assert int(re.search(rf"#define STMOE_SELECT_{name} (\d+)", text).group(1)) == value
