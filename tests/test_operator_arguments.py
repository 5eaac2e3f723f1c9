"""Refusals of the MX4 and router-statistics entry points, without device work."""
import ctypes as C

import pytest
import torch

import paper_2606_15453_b200 as P

BAD, TOO_LARGE = -1, -7
X = C.c_void_p(1 << 20)      # an aligned address that no refused call may touch
ODD = C.c_void_p((1 << 20) + 1)


def _quant(**kw):
    a = dict(x=X, dtype=0, rows=4, cols=64, xs=64, c=X, cs=32, s=X, ss=2)
    a.update(kw)
    return P.lib().stmoe_mx4_quantize(a["x"], a["dtype"], a["rows"], a["cols"], a["xs"], a["c"], a["cs"], a["s"], a["ss"], None)


def _dequant(**kw):
    a = dict(x=X, dtype=0, rows=4, cols=64, xs=64, c=X, cs=32, s=X, ss=2)
    a.update(kw)
    return P.lib().stmoe_mx4_dequantize(a["c"], a["cs"], a["s"], a["ss"], a["rows"], a["cols"], a["x"], a["dtype"], a["xs"], None)


@pytest.mark.parametrize("call", [_quant, _dequant])
@pytest.mark.parametrize("kw", [dict(x=None), dict(c=None), dict(s=None), dict(dtype=2), dict(dtype=3), dict(dtype=5), dict(rows=-1),
                                dict(cols=0), dict(xs=63), dict(cs=28), dict(cs=33), dict(ss=1), dict(c=ODD), dict(x=ODD)])
def test_mx4_rows_refusals(call, kw):
    assert call(**kw) == BAD


def test_mx4_rows_accept_no_rows():
    assert _quant(rows=0) == 0 and _dequant(rows=0) == 0


def _mm(**kw):
    a = dict(ac=X, acs=32, as_=X, ass=2, m=4, bc=X, bcs=32, bs=X, bss=2, groups=1, n=8, kb=2, counts=None, out=X, dt=1, os=8)
    a.update(kw)
    return P.lib().stmoe_mx4_matmul(a["ac"], a["acs"], a["as_"], a["ass"], a["m"], a["bc"], a["bcs"], a["bs"], a["bss"], a["groups"],
                                    a["n"], a["kb"], a["counts"], a["out"], a["dt"], a["os"], None, None)


@pytest.mark.parametrize("kw", [dict(ac=None), dict(as_=None), dict(bc=None), dict(bs=None), dict(out=None), dict(m=-1), dict(m=1 << 32),
                                dict(n=0), dict(kb=0), dict(groups=0), dict(groups=257, counts=X), dict(groups=2), dict(ac=C.c_void_p((1 << 20) + 8)),
                                dict(bc=C.c_void_p((1 << 20) + 8)), dict(acs=40), dict(acs=16), dict(bcs=24), dict(bcs=16), dict(ass=1),
                                dict(bss=1), dict(dt=2), dict(dt=3), dict(os=7), dict(out=ODD), dict(n=1 << 25, os=1 << 25),
                                dict(groups=256, counts=X, n=1 << 24, os=1 << 24)])
def test_mx4_matmul_refusals(kw):
    assert _mm(**kw) == BAD


def test_mx4_matmul_accepts_no_rows_and_refuses_more_tiles_than_an_index_holds():
    assert _mm(m=0) == 0
    assert P.lib().stmoe_mx4_matmul(X, 32, X, 2, 1 << 30, X, 32, X, 2, 1, 1 << 24, 2, None, X, 1, 1 << 24, None, None) in (TOO_LARGE, -3)


def _bal(**kw):
    a = dict(z=X, dt=0, st=8, ids=X, mask=None, T=1 << 20, E=8, K=2, loss=X, counts=X, rows=X, scratch=X, n=1 << 24)
    a.update(kw)
    return P.lib().stmoe_router_balance(a["z"], a["dt"], a["st"], a["ids"], a["mask"], a["T"], a["E"], a["K"], a["loss"], a["counts"],
                                        a["rows"], a["scratch"], a["n"], None)


@pytest.mark.parametrize("kw", [dict(z=None), dict(ids=None), dict(loss=None), dict(counts=None), dict(rows=None), dict(scratch=None),
                                dict(dt=2), dict(dt=3), dict(st=7), dict(T=-1), dict(T=1 << 31), dict(E=0), dict(E=257, st=300), dict(K=0),
                                dict(K=9), dict(n=64), dict(scratch=ODD), dict(z=ODD), dict(z=C.c_void_p((1 << 20) + 2))])
def test_router_balance_refusals(kw):
    assert _bal(**kw) == BAD


@pytest.mark.parametrize("name", ["ids", "loss", "counts", "rows"])
@pytest.mark.parametrize("off", [1, 2])
def test_router_balance_refuses_addresses_off_their_type(name, off):
    assert _bal(**{name: C.c_void_p((1 << 20) + off)}) == BAD


def _balb(**kw):
    a = dict(z=X, dt=0, st=8, mask=None, T=4, E=8, K=2, counts=X, rows=X, g=X, d=C.c_void_p(1 << 21), ds=8)
    a.update(kw)
    return P.lib().stmoe_router_balance_backward(a["z"], a["dt"], a["st"], a["mask"], a["T"], a["E"], a["K"], a["counts"], a["rows"],
                                                 a["g"], a["d"], a["ds"], None)


@pytest.mark.parametrize("kw", [dict(z=None), dict(counts=None), dict(rows=None), dict(g=None), dict(d=None), dict(ds=7), dict(st=7),
                                dict(K=0), dict(E=0), dict(d=X), dict(d=C.c_void_p((1 << 20) + 64)), dict(d=C.c_void_p((1 << 20) - 64))])
def test_router_balance_backward_refusals(kw):
    assert _balb(**kw) == BAD


def test_scratch_sizes():
    f = P.lib().stmoe_router_balance_scratch_bytes
    assert f(1 << 20, 0) == 0 and f(1 << 20, 257) == 0 and f(1 << 20, 256) >= 2 * 257 * 4 * 148
    assert f(0, 8) == 0 and f(16, 256) == 0           # one CTA alone


def test_binding_refuses_before_the_library():
    x = torch.zeros(4, 64)
    for call in (lambda: P.mx4_quantize(x), lambda: P.mx4_dequantize(x, x, 64), lambda: P.mx4_matmul((x, x), (x, x)),
                 lambda: P.router_balance(x, torch.zeros(4, 2, dtype=torch.int32))):
        with pytest.raises(P.StmoeError):
            call()


def test_mx4_poll_limit_is_set_without_a_stack():
    hook = P.lib().stmoe_test_hook
    assert hook(None, 7, -1) == BAD and hook(X, 7, 4) == BAD and hook(None, 6, 4) == BAD
    assert hook(None, 7, 16) == 0 and hook(None, 7, 1 << 40) == 0      # the second: back to the default


def test_balance_scratch_grows_with_the_tokens_and_never_falls():
    f = P.lib().stmoe_router_balance_scratch_bytes
    for E in (2, 8, 9, 64, 100, 256):
        sizes = [f(t, E) for t in sorted({1 << i for i in range(31)} | {(1 << i) + 7 for i in range(30)})]
        assert sizes == sorted(sizes)
        # one row of sums, 2 E + 3 words, to every 256 rows of a lane at most: 256 lanes' worth of rows a CTA
        lanes = next(l for l in (1, 2, 4, 8, 16) if 16 * l >= E)
        assert sizes[-1] >= 4 * (2 * E + 3) * ((1 << 30) // (256 * 256 // lanes))


@pytest.mark.parametrize("name", ["counts", "rows", "g"])
def test_router_balance_backward_refuses_addresses_off_their_type(name):
    assert _balb(**{name: C.c_void_p((1 << 20) + 2)}) == BAD


def test_mx4_matmul_refuses_addresses_off_their_type():
    off = C.c_void_p((1 << 20) + 2)
    assert _mm(counts=off) == BAD
    assert P.lib().stmoe_mx4_matmul(X, 32, X, 2, 4, X, 32, X, 2, 1, 8, 2, None, X, 1, 8, off, None) == BAD


@pytest.mark.parametrize("name", ["h", "inv", "ids", "w", "out", "experts", "scratch"])
def test_mx4_ffn_refuses_addresses_off_their_type(name):
    a = dict(h=X, inv=X, ids=X, w=X, experts=X, out=X, scratch=X)
    a[name] = C.c_void_p((1 << 20) + (8 if name == "experts" else 128 if name == "scratch" else 2))
    rc = P.lib().stmoe_moe_ffn(a["h"], a["inv"], a["ids"], a["w"], a["experts"], 3, 2, 4, 2, 64, 64, 0.1, a["out"], a["scratch"],
                               1 << 24, None)
    assert rc == BAD
