"""The head norm's and the gated delta rule's entry points refuse what they cannot take, before anything is launched (no GPU
needed: the C ABI sees fake addresses that are never dereferenced, the binding sees host tensors)."""
import ctypes

import pytest
import torch

from test_layer_host import NULL, ODD, at, b, call  # noqa: F401  (b: a fixture)

f = ctypes.c_float


def test_qk_refusals(b):  # noqa: F811
    lib = b.raw()
    ok = dict(q=at(0), ldq=128, k=at(1), ldk=64, wq=at(2), wk=at(3), freq=at(4), pos=at(5), lengths=at(6), yq=at(7), yk=at(8), B=2, N=8, H=4, Hk=2, D=32, R=16,
              flags=1, eps=f(1e-6), t=0, stream=NULL)
    fwd = lambda **c: call(lib.la_qk_fwd, ok, **c)
    assert fwd(t=2) == b.LA_ERR_UNSUPPORTED and fwd(flags=3) == b.LA_ERR_UNSUPPORTED and fwd(flags=8) == b.LA_ERR_UNSUPPORTED
    for name in ("q", "k", "freq", "yq", "yk"):
        assert fwd(**{name: NULL}) == b.LA_ERR_NULL, name
    for name in ("B", "N", "H", "D"):
        assert fwd(**{name: 0}) == b.LA_ERR_SHAPE, name
    assert fwd(R=40) == b.LA_ERR_SHAPE and fwd(R=-8) == b.LA_ERR_SHAPE and fwd(Hk=-1) == b.LA_ERR_SHAPE
    assert fwd(D=36, R=0) == b.LA_ERR_UNSUPPORTED and fwd(R=12) == b.LA_ERR_UNSUPPORTED and fwd(D=520, ldq=4 * 520, ldk=2 * 520) == b.LA_ERR_UNSUPPORTED
    assert fwd(ldq=127) == b.LA_ERR_SHAPE and fwd(ldk=63) == b.LA_ERR_SHAPE and fwd(N=(1 << 30) + 1) == b.LA_ERR_SHAPE and fwd(B=1 << 20, N=1 << 20) == b.LA_ERR_SHAPE
    for eps in (-1.0, float("nan"), float("inf")):
        assert fwd(eps=f(eps)) == b.LA_ERR_SHAPE
    for name in ("q", "k", "wq", "wk", "freq", "pos", "lengths", "yq", "yk"):
        assert fwd(**{name: ODD}) == b.LA_ERR_ALIGN, name
    assert fwd(yq=at(0)) == b.LA_ERR_ALIAS and fwd(yk=at(7)) == b.LA_ERR_ALIAS and fwd(yk=at(5)) == b.LA_ERR_ALIAS
    ok2 = dict(q=at(0), ldq=128, k=at(1), ldk=64, wq=at(2), wk=at(3), freq=at(4), pos=at(5), lengths=at(6), dyq=at(7), dyk=at(8), dq=at(9), dk=at(10), dwq=at(11),
               dwk=at(12), B=2, N=8, H=4, Hk=2, D=32, R=16, flags=2, eps=f(1e-6), t=1, ws=at(13), ws_bytes=0, stream=NULL)
    bwd = lambda **c: call(lib.la_qk_bwd, ok2, **c)
    need = lib.la_qk_bwd_workspace(2, 8, 4, 2, 32, 1)
    assert need >= 2 * 32 * 4 and lib.la_qk_bwd_workspace(2, 8, 4, 2, 33, 1) == 0
    assert bwd() == b.LA_ERR_WORKSPACE and bwd(ws=NULL, ws_bytes=need) == b.LA_ERR_WORKSPACE and bwd(ws_bytes=need - 1) == b.LA_ERR_WORKSPACE
    for name in ("q", "k", "dyq", "dyk", "dq", "dk", "freq"):
        assert bwd(**{name: NULL}) == b.LA_ERR_NULL, name
    assert bwd(ws_bytes=need, Hk=0, k=NULL, dyk=NULL, dk=NULL) == b.LA_ERR_SHAPE          # a gradient of no weight
    assert bwd(ws_bytes=need, dq=at(7)) == b.LA_ERR_ALIAS and bwd(ws_bytes=need, dwk=at(11)) == b.LA_ERR_ALIAS and bwd(ws_bytes=need, ws=at(9)) == b.LA_ERR_ALIAS
    assert bwd(ws_bytes=need, ws=ODD) == b.LA_ERR_ALIGN


def test_delta_refusals(b):  # noqa: F811
    lib = b.raw()
    need = lib.la_delta_fwd_workspace(2, 40, 4, 2, 32, 48, 0, 0)
    kept = lib.la_delta_fwd_workspace(2, 40, 4, 2, 32, 48, 0, 1)
    assert 0 < need < kept
    ok = dict(q=at(0), ldq=64, k=at(1), ldk=64, v=at(2), ldv=192, g=at(3), beta=at(4), h0=at(5), lengths=at(6), o=at(7), h1=at(8), B=2, N=40, H=4, Hk=2, D=32, M=48,
              scale=f(1.0), flags=0, t=0, ws=at(9), ws_bytes=need, stream=NULL)
    fwd = lambda **c: call(lib.la_delta_fwd, ok, **c)
    assert fwd(t=4) == b.LA_ERR_UNSUPPORTED and fwd(flags=2) == b.LA_ERR_UNSUPPORTED
    for D in (16, 48, 96, 256):
        assert fwd(D=D) == b.LA_ERR_UNSUPPORTED and lib.la_delta_fwd_workspace(2, 40, 4, 2, D, 48, 0, 0) == 0
    for M in (8, 24, 528):
        assert fwd(M=M) == b.LA_ERR_UNSUPPORTED
    for name in ("q", "k", "v", "beta", "o"):
        assert fwd(**{name: NULL}) == b.LA_ERR_NULL, name
    for name in ("B", "N", "H", "Hk", "D", "M"):
        assert fwd(**{name: 0}) == b.LA_ERR_SHAPE, name
    assert fwd(Hk=3) == b.LA_ERR_SHAPE and fwd(ldq=56) == b.LA_ERR_SHAPE and fwd(ldv=184) == b.LA_ERR_SHAPE and fwd(ldk=(1 << 23) + 8) == b.LA_ERR_SHAPE
    assert fwd(N=1 << 28, B=8) == b.LA_ERR_SHAPE and fwd(N=(1 << 30) + 1) == b.LA_ERR_SHAPE
    assert fwd(scale=f(float("inf"))) == b.LA_ERR_SHAPE and fwd(scale=f(float("nan"))) == b.LA_ERR_SHAPE
    assert fwd(ldq=68) == b.LA_ERR_ALIGN and fwd(ldv=196) == b.LA_ERR_ALIGN
    for name in ("q", "k", "v", "g", "beta", "h0", "lengths", "o", "h1", "ws"):
        assert fwd(**{name: ODD}) == b.LA_ERR_ALIGN, name
    assert fwd(ws_bytes=need - 1) == b.LA_ERR_WORKSPACE and fwd(ws=NULL) == b.LA_ERR_WORKSPACE and fwd(flags=1) == b.LA_ERR_WORKSPACE
    assert fwd(o=at(2)) == b.LA_ERR_ALIAS and fwd(h1=at(5)) == b.LA_ERR_ALIAS and fwd(ws=at(7)) == b.LA_ERR_ALIAS
    need = lib.la_delta_bwd_workspace(2, 40, 4, 2, 32, 48, 0, 0)
    given = lib.la_delta_bwd_workspace(2, 40, 4, 2, 32, 48, 0, 1)
    assert 0 < given < need
    ok = dict(q=at(0), ldq=64, k=at(1), ldk=64, v=at(2), ldv=192, g=at(3), beta=at(4), h0=at(5), lengths=at(6), fwd_ws=NULL, dO=at(7), dh1=at(8), dq=at(9), dk=at(10),
              dv=at(11), dg=at(12), dbeta=at(13), dh0=at(14), B=2, N=40, H=4, Hk=2, D=32, M=48, scale=f(1.0), flags=0, t=0, ws=at(15), ws_bytes=need, stream=NULL)
    bwd = lambda **c: call(lib.la_delta_bwd, ok, **c)
    for name in ("q", "k", "v", "beta", "dO", "dq", "dk", "dv", "dbeta", "g", "dg"):
        assert bwd(**{name: NULL}) == b.LA_ERR_NULL, name
    assert bwd(flags=1) == b.LA_ERR_SHAPE and bwd(fwd_ws=at(16)) == b.LA_ERR_SHAPE         # the flag goes with the workspace
    assert bwd(ws_bytes=need - 1) == b.LA_ERR_WORKSPACE and bwd(ldk=68) == b.LA_ERR_ALIGN
    for name in ("dq", "dk", "dv", "dg", "dbeta", "dh0"):
        assert bwd(**{name: ODD}) == b.LA_ERR_ALIGN, name
        assert bwd(**{name: at(0)}) == b.LA_ERR_ALIAS, name
    assert bwd(flags=1, fwd_ws=at(15), ws_bytes=given) == b.LA_ERR_ALIAS
    ok = dict(q=at(0), k=at(1), v=at(2), g=at(3), beta=at(4), h=at(5), o=at(6), B=2, H=4, Hk=2, D=32, M=48, scale=f(1.0), t=1, stream=NULL)
    step = lambda **c: call(lib.la_delta_step, ok, **c)
    for name in ("q", "k", "v", "beta", "h", "o"):
        assert step(**{name: NULL}) == b.LA_ERR_NULL, name
        assert step(**{name: ODD}) == b.LA_ERR_ALIGN, name
    assert step(D=40) == b.LA_ERR_UNSUPPORTED and step(Hk=3) == b.LA_ERR_SHAPE and step(o=at(2)) == b.LA_ERR_ALIAS and step(h=at(0)) == b.LA_ERR_ALIAS


def test_the_binding_names_what_is_wrong():
    import paper_2006_16236_amd as la
    B, N, H, Hk, D, M = 2, 5, 4, 2, 32, 16
    z = torch.zeros
    q, k, v, g, beta, o = z(B, N, Hk, D), z(B, N, Hk, D), z(B, N, H, M), z(B, N, H), z(B, N, H), z(B, N, H, M)
    bad = [(dict(q=z(B, N, D)), "q must have 4"), (dict(k=z(B, N, Hk, 64)), "k: shape"), (dict(v=z(B, N, 3, M)), "do not divide"), (dict(g=z(B, N, Hk)), "g: shape"),
           (dict(beta=beta.double()), "beta"), (dict(beta=None), "beta"), (dict(o=o.bfloat16()), "o: dtype"), (dict(h0=z(B, H, M, D)), "h0: shape"),
           (dict(lengths=z(B)), "lengths"), (dict(q=q.half()), "unsupported dtype"), (dict(k=k.bfloat16()), "k: dtype"), (dict(v=5), "v must be")]
    for change, words in bad:
        args = {**dict(q=q, k=k, v=v, g=g, beta=beta, o=o), **change}
        with pytest.raises((ValueError, TypeError), match=words):
            la.la_delta_fwd(**args)
    with pytest.raises(ValueError, match="device"):
        la.la_delta_fwd(q, k, v, g, beta, o)
    d = dict(dq=z(B, N, Hk, D), dk=z(B, N, Hk, D), dv=z(B, N, H, M), dg=z(B, N, H), dbeta=z(B, N, H))
    for change, words in ((dict(dg=None), "dg goes with g"), (dict(dq=z(B, N, H, D)), "dq: shape"), (dict(dh0=z(1)), "dh0: shape"),
                          (dict(fwd_ws=z(4)), "fwd_ws: 16 bytes")):
        with pytest.raises(ValueError, match=words):
            la.la_delta_bwd(q, k, v, g, beta, o, **{**d, **change})
    with pytest.raises(ValueError, match="h: shape"):
        la.la_delta_step(*(t[:, 0].contiguous() for t in (q, k, v, g, beta)), z(B, H, D, 8), o[:, 0].contiguous())
    x, y = z(B, N, H, 24), z(B, N, H, 24)
    for change, words in ((dict(norm="both"), "norm must be"), (dict(yk=y), "yk goes with k"), (dict(wq=z(12)), "wq: shape"), (dict(freq=z(2, 2)), "freq must be"),
                          (dict(pos=z(B, N)), "pos: dtype"), (dict(k=z(B, N, 2, 16), yk=y), "k: shape"), (dict(k=z(B, N, 2, 24)), "yk goes with k")):
        with pytest.raises(ValueError, match=words):
            la.la_qk_fwd(**{**dict(q=x, yq=y), **change})
    with pytest.raises(ValueError, match="dwk goes with k"):
        la.la_qk_bwd(x, y, y.clone(), dwk=z(24))
