"""Refusals of the C entry points of a layer of routed experts: found on the host, before anything is launched (no GPU needed)."""
import ctypes

import paper_1912_02057_b200 as rtn

vp = ctypes.c_void_p
P, ODD = vp(0x1000), vp(0x1001)          # never dereferenced
NULL, SHAPE, ALIGN, VALUE = 1, 2, 3, 4
NAN = float("nan")


def route(T=4, E=8, k=2, x=P, xs=8, dtype=0, score=0, bias=None, groups=1, kept=1, top=1, experts=P, weights=P, start=P, tokens=P, place=P):
    return rtn.lib().rtn_route_experts(x, xs, T, E, dtype, score, bias, groups, kept, top, k, 1, 1.0, experts, weights, start, tokens, place, None)


def test_route():
    assert route(x=None) == NULL and route(experts=None) == NULL and route(weights=None) == NULL and route(tokens=None) == NULL and route(place=None) == NULL
    assert route(start=None) == NULL and route(start=None, tokens=None) == NULL
    assert route(T=-1) == SHAPE and route(E=0) == SHAPE and route(E=1025) == SHAPE and route(k=0) == SHAPE and route(k=9) == SHAPE and route(E=64, k=33) == SHAPE
    assert route(groups=3) == SHAPE and route(groups=0) == SHAPE and route(E=64, groups=64) == SHAPE and route(groups=4, kept=5) == SHAPE
    assert route(groups=4, top=3) == SHAPE and route(groups=4, kept=0) == SHAPE and route(groups=4, k=3) == SHAPE and route(xs=-1) == SHAPE
    assert route(T=1 << 30) == SHAPE and route(T=1 << 62) == SHAPE and route(T=(1 << 62) + 1, k=4) == SHAPE
    assert route(dtype=3) == VALUE and route(score=2) == VALUE and route(score=-1) == VALUE
    assert route(x=ODD) == ALIGN and route(bias=ODD) == ALIGN and route(place=ODD) == ALIGN
    assert route(T=0, start=None, tokens=None, place=None, x=None, experts=None, weights=None) == 0


def experts(T=4, R=6, E=2, N=8, K=16, na=1, nw=1, act=0, gated=0, a=P, w=P, tokens=P, start=P, out=P, os=8, dtype=0, bias=None, lo=None, hi=None, nt=1,
            packed=None, sums=None, scale=P):
    return rtn.lib().rtn_ternary_experts(a, P, T, tokens, start, R, w, P, E, N, K, scale, P, na, P, P, nw, bias, act, gated, out, os, dtype, lo, hi, nt,
                                         packed, sums, None)


def test_experts():
    assert experts(a=None) == NULL and experts(w=None) == NULL and experts(start=None) == NULL and experts(out=None) == NULL and experts(scale=None) == NULL
    codes = dict(out=None, packed=P, sums=P, lo=P, hi=P)
    assert experts(**{**codes, "sums": None}) == NULL and experts(**{**codes, "lo": None}) == NULL and experts(sums=P) == NULL
    assert experts(T=-1) == SHAPE and experts(R=-1) == SHAPE and experts(E=0) == SHAPE and experts(E=1025) == SHAPE and experts(N=0) == SHAPE and experts(K=0) == SHAPE
    assert experts(K=(1 << 24) + 1) == SHAPE and experts(N=7, gated=1) == SHAPE and experts(na=3) == SHAPE and experts(nw=8) == SHAPE and experts(os=7) == SHAPE
    assert experts(N=1 << 31) == SHAPE and experts(N=1 << 61, E=8) == SHAPE and experts(tokens=None) == SHAPE and experts(os=3, gated=1) == SHAPE
    assert experts(**{**codes, "nt": 3}) == SHAPE and experts(T=0, a=None, scale=None, na=1) == SHAPE
    assert experts(act=5) == VALUE and experts(dtype=3) == VALUE
    assert experts(a=ODD) == ALIGN and experts(w=vp(0x1008)) == ALIGN and experts(tokens=ODD) == ALIGN and experts(out=ODD) == ALIGN
    assert experts(**{**codes, "packed": vp(0x1004)}) == ALIGN
    assert experts(R=0, out=None) == 0


def norm(T=4, W=8, R=8, k=2, branch=P, place=P, weights=P, post=P, gate=P, kind=0, scale=P, ns=8, res=P, pre=P, eps=1e-6, h=vp(0x9000), n=vp(0xa000), bs=8, gs=8,
         rs=8, hs=8, no=8, lo=None, hi=None, nt=1, packed=None, sums=None, dtype=0, sdtype=0):
    return rtn.lib().rtn_block_norm(branch, bs, R, place, weights, k, post, gate, gs, kind, scale, ns, res, rs, pre, eps, T, W, h, hs, n, no, lo, hi, nt, packed,
                                    sums, dtype, sdtype, None)


def test_block_norm():
    bare = dict(branch=None, place=None, weights=None, k=0, post=None, gate=None, scale=None)
    assert norm(branch=None) == NULL and norm(**bare, res=None) == NULL and norm(**{**bare, "post": P}) == NULL and norm(h=None, n=None) == NULL
    assert norm(place=None, k=0) == NULL and norm(sums=P) == NULL and norm(packed=P, lo=P, hi=P) == NULL and norm(packed=P, sums=P) == NULL
    assert norm(T=-1) == SHAPE and norm(W=0) == SHAPE and norm(W=16385) == SHAPE and norm(k=33) == SHAPE and norm(k=0) == SHAPE and norm(place=None) == SHAPE
    assert norm(R=-1) == SHAPE and norm(place=None, weights=None, k=0, R=3) == SHAPE and norm(T=1 << 31) == SHAPE and norm(ns=3) == SHAPE
    assert norm(bs=-1) == SHAPE and norm(hs=7) == SHAPE and norm(no=7) == SHAPE and norm(h=P, rs=16) == SHAPE
    assert norm(packed=P, sums=P, lo=P, hi=P, nt=4) == SHAPE
    assert norm(kind=3) == VALUE and norm(eps=-1.0) == VALUE and norm(eps=NAN) == VALUE and norm(dtype=3) == VALUE and norm(sdtype=-1) == VALUE
    assert norm(branch=ODD) == ALIGN and norm(place=ODD) == ALIGN and norm(h=vp(0x9002)) == ALIGN and norm(packed=vp(0x1008), sums=P, lo=P, hi=P) == ALIGN
    assert norm(T=0, branch=None, place=None, weights=None, res=None, h=None, n=None) == 0
