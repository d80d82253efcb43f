"""Refusals of the layer operators' C entry points: found on the host, before anything is launched (no GPU needed)."""
import ctypes

import paper_1912_02057_b200 as rtn

vp = ctypes.c_void_p
P, ODD = vp(0x1000), vp(0x1001)          # never dereferenced
NULL, SHAPE, ALIGN, VALUE = 1, 2, 3, 4
NAN = float("nan")


def linear(M=4, N=8, K=16, na=1, nw=1, act=0, a=P, res=None, rs=8, out=P, os=8, dtype=0, bias=None, w=P):
    return rtn.lib().rtn_ternary_linear(a, P, w, P, M, N, K, P, P, na, P, P, nw, bias, act, res, rs, out, os, dtype, None)


def test_linear():
    assert linear(w=None) == NULL and linear(a=None) == NULL and linear(out=None) == NULL
    assert linear(M=-1) == SHAPE and linear(N=0) == SHAPE and linear(K=0) == SHAPE and linear(K=(1 << 24) + 1) == SHAPE
    assert linear(na=3) == SHAPE and linear(nw=3) == SHAPE and linear(os=7) == SHAPE
    assert linear(res=P, rs=9) == SHAPE                       # in place with another stride
    assert linear(act=5) == VALUE and linear(act=-1) == VALUE and linear(dtype=3) == VALUE
    assert linear(w=ODD) == ALIGN and linear(out=ODD) == ALIGN and linear(bias=ODD) == ALIGN and linear(out=vp(0x1002)) == ALIGN
    assert linear(M=0, na=0, a=None, out=None) == 0


def table(rows=8, R=8, base=1e4, kind=0, factor=2.0, context=100.0, low=1.0, high=4.0, amplitude=1.0, t=P):
    return rtn.lib().rtn_rotary_table(t, rows, R, base, kind, factor, context, low, high, amplitude, None)


def test_table():
    assert table(t=None) == NULL and table(rows=0) == SHAPE and table(R=7) == SHAPE and table(R=0) == SHAPE and table(t=ODD) == ALIGN
    assert table(base=0.0) == VALUE and table(base=NAN) == VALUE and table(kind=4) == VALUE and table(amplitude=NAN) == VALUE
    assert table(kind=1, factor=0.0) == VALUE and table(kind=2, R=2) == VALUE
    assert table(kind=3, low=4.0) == VALUE and table(kind=3, context=0.0) == VALUE and table(kind=3, factor=NAN) == VALUE


def rotary(T=4, Hq=2, Hk=2, D=8, R=8, layout=0, q=P, k=P, oq=P, ok=P, qs=(16, 8), oqs=(16, 8), ks=(16, 8), oks=(16, 8), qw=None, kw=None,
           eps=1e-6, tab=P, rows=4, pos=None, dtype=0):
    return rtn.lib().rtn_qk_norm_rotary(q, *qs, k, *ks, oq, *oqs, ok, *oks, T, Hq, Hk, D, R, layout, qw, kw, eps, tab, rows, pos, dtype, None)


def test_rotary():
    assert rotary(q=None) == NULL and rotary(k=None) == NULL and rotary(ok=None) == NULL and rotary(tab=None) == NULL
    assert rotary(qw=P) == NULL and rotary(kw=P) == NULL
    assert rotary(T=-1) == SHAPE and rotary(Hq=0) == SHAPE and rotary(R=7) == SHAPE and rotary(R=10) == SHAPE and rotary(D=1025) == SHAPE
    assert rotary(oqs=(16, 7)) == SHAPE and rotary(oqs=(15, 8)) == SHAPE and rotary(qs=(-1, 8)) == SHAPE and rotary(oqs=(0, 8)) == SHAPE
    assert rotary(qs=(32, 8)) == SHAPE                        # in place with other strides
    assert rotary(layout=2) == VALUE and rotary(dtype=7) == VALUE and rotary(qw=P, kw=P, eps=-1.0) == VALUE and rotary(qw=P, kw=P, eps=NAN) == VALUE
    assert rotary(q=ODD) == ALIGN and rotary(pos=vp(0x1004)) == ALIGN and rotary(tab=ODD) == ALIGN
    assert rotary(T=0, q=None, k=None, oq=None, ok=None) == 0


def decay(B=2, total=4, max_len=3, H=2, Hk=1, Dk=8, Dv=8, q=P, k=P, v=P, out=vp(0x9000), start=P, g=P, state=P, state_out=P, slots=None, n_slots=2,
          dtype=0, os=(16, 8), ks=(8, 8)):
    return rtn.lib().rtn_decay_attention(q, 16, 8, k, *ks, v, 8, 8, out, *os, total, B, start, max_len, H, Hk, Dk, Dv, g, 1.0, state, state_out,
                                         slots, n_slots, dtype, None)


def step(B=2, H=2, Hk=1, Dk=8, Dv=8, q=P, k=P, v=P, out=vp(0x9000), g=P, state=P, state_out=P, slots=None, n_slots=2, dtype=0, os=(16, 8)):
    return rtn.lib().rtn_decay_attention_step(q, 16, 8, k, 8, 8, v, 8, 8, out, *os, B, H, Hk, Dk, Dv, g, 1.0, state, state_out, slots,
                                              n_slots, dtype, None)


def test_decay_attention():
    assert decay(start=None) == NULL and decay(total=-1) == SHAPE and decay(B=-1) == SHAPE and decay(max_len=-1) == SHAPE
    assert decay(start=ODD) == ALIGN and decay(total=1 << 31) == SHAPE and decay(ks=(-8, 8)) == SHAPE
    assert decay(B=0, n_slots=0, total=0, q=None, k=None, v=None, out=None) == 0
    for call in (decay, step):
        assert call(q=None) == NULL and call(v=None) == NULL and call(out=None) == NULL and call(g=None) == NULL and call(state_out=None) == NULL
        assert call(H=3, Hk=2) == SHAPE and call(Dk=0) == SHAPE and call(Dk=257) == SHAPE and call(Dv=300) == SHAPE and call(n_slots=1) == SHAPE
        assert call(os=(15, 8)) == SHAPE and call(os=(16, 7)) == SHAPE
        assert call(dtype=3) == VALUE and call(q=ODD) == ALIGN and call(state=vp(0x1002)) == ALIGN and call(slots=vp(0x1002)) == ALIGN
    assert step(B=-1) == SHAPE and step(B=0, q=None, k=None, v=None, out=None) == 0


def test_status_text():
    f = rtn.lib().rtn_status_string
    assert f(8).startswith(b"RTN_ERR_DEVICE_INDEX") and f(9).startswith(b"unknown")


def test_sizes_whose_products_pass_64_bits():
    """Refused, whatever their products are modulo 2^64."""
    assert rotary(T=1 << 62) == SHAPE and rotary(T=(1 << 62) + 1) == SHAPE and rotary(T=1 << 31) == SHAPE
    assert table(rows=1 << 62) == SHAPE and table(rows=(1 << 62) + 2) == SHAPE and table(rows=1 << 39, R=2) == SHAPE
    many = dict(H=1 << 15, Hk=1 << 15, slots=P, os=(8 << 15, 8))
    assert step(B=1 << 49, **many) == SHAPE and step(B=(1 << 49) + 1, **many) == SHAPE
    assert step(H=1 << 62, Hk=1, B=4) == SHAPE and step(H=-(1 << 62), B=2) == SHAPE
    # rows of out that meet: 2^31 - 2 tokens 2^33 elements apart are not between two heads 2^34 apart
    assert decay(total=(1 << 31) - 1, os=(1 << 33, 1 << 34)) == SHAPE
    assert rotary(T=(1 << 29) - 1, oqs=(1 << 35, 1 << 36)) == SHAPE
