"""The norm, convolution and scan entry points refuse what they cannot take, before anything is launched (no GPU needed:
the C ABI sees fake addresses that are never dereferenced, the binding sees host tensors)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2006_16236_amd import binding
    return binding


P, ODD, NULL = 0x100000, 0x100004, None
f = ctypes.c_float
STEP = 0x1000000                                                   # between fake buffers, larger than any of them


def at(i):
    return P + i * STEP


def call(fn, args, **changes):
    """fn with the named arguments of `args` (a dict in the C order), some of them changed."""
    return fn(*{**args, **changes}.values())


def test_norm_refusals(b):
    lib = b.raw()
    ok = dict(x=at(0), r=at(1), gamma=at(2), beta=at(3), y=at(4), s=at(5), mean=at(6), rstd=at(7), rows=4, E=64, eps=f(1e-5), t=7, stream=NULL)
    fwd = lambda **c: call(lib.la_norm_fwd, ok, **c)
    assert fwd() == b.LA_ERR_UNSUPPORTED                           # no such element type: everything else is in order
    assert fwd(t=2) == b.LA_ERR_UNSUPPORTED and fwd(t=4) == b.LA_ERR_UNSUPPORTED
    assert fwd(t=0, x=NULL) == b.LA_ERR_NULL and fwd(t=0, y=NULL) == b.LA_ERR_NULL
    assert fwd(t=0, r=NULL) == b.LA_ERR_NULL                       # a sum of nothing
    assert fwd(t=0, rows=0) == b.LA_ERR_SHAPE and fwd(t=0, E=0) == b.LA_ERR_SHAPE and fwd(t=0, rows=-1) == b.LA_ERR_SHAPE
    assert fwd(t=0, E=16385) == b.LA_ERR_UNSUPPORTED
    for eps in (-1.0, float("nan"), float("inf")):
        assert fwd(t=0, eps=f(eps)) == b.LA_ERR_SHAPE
    for name in ("x", "r", "gamma", "beta", "y", "s", "mean", "rstd"):
        assert fwd(t=0, **{name: ODD}) == b.LA_ERR_ALIGN, name
    assert fwd(t=0, y=at(0)) == b.LA_ERR_ALIAS and fwd(t=0, s=at(4) + 4 * 64 * 4 - 16) == b.LA_ERR_ALIAS
    assert fwd(t=0, rstd=at(6)) == b.LA_ERR_ALIAS
    ok = dict(s=at(0), gamma=at(1), mean=at(2), rstd=at(3), dy=at(4), ds=at(5), dx=at(6), dgamma=at(7), dbeta=at(8), rows=4, E=64, t=0, ws=at(9),
              ws_bytes=0, stream=NULL)
    bwd = lambda **c: call(lib.la_norm_bwd, ok, **c)
    need = b.raw().la_norm_bwd_workspace(4, 64, 0)
    assert need >= 2 * 64 * 4 and b.raw().la_norm_bwd_workspace(0, 64, 0) == 0
    assert bwd() == b.LA_ERR_WORKSPACE and bwd(ws=NULL, ws_bytes=1 << 20) == b.LA_ERR_WORKSPACE and bwd(ws_bytes=need - 1) == b.LA_ERR_WORKSPACE
    for name in ("s", "mean", "rstd", "dy", "dx"):
        assert bwd(**{name: NULL}) == b.LA_ERR_NULL, name
    assert bwd(ws_bytes=need, dx=at(4)) == b.LA_ERR_ALIAS and bwd(ws_bytes=need, ws=at(8)) == b.LA_ERR_ALIAS
    assert bwd(ws_bytes=need, ws=ODD) == b.LA_ERR_ALIGN


def test_conv_refusals(b):
    lib = b.raw()
    ok = dict(x=at(0), ldx=64, w=at(1), bias=at(2), x0=at(3), lengths=at(4), y=at(5), x1=at(6), B=2, N=8, E=64, W=4, silu=1, t=0, stream=NULL)
    fwd = lambda **c: call(lib.la_conv_fwd, ok, **c)
    assert fwd(t=3) == b.LA_ERR_UNSUPPORTED and fwd(W=1) == b.LA_ERR_UNSUPPORTED and fwd(W=5) == b.LA_ERR_UNSUPPORTED
    for name in ("x", "w", "y"):
        assert fwd(**{name: NULL}) == b.LA_ERR_NULL, name
    for name in ("B", "N", "E"):
        assert fwd(**{name: 0}) == b.LA_ERR_SHAPE, name
    assert fwd(ldx=63) == b.LA_ERR_SHAPE and fwd(B=1 << 20, N=1 << 16) == b.LA_ERR_SHAPE and fwd(B=1 << 30, N=1, E=32) == b.LA_ERR_SHAPE
    for name in ("x", "w", "bias", "x0", "lengths", "y", "x1"):
        assert fwd(**{name: ODD}) == b.LA_ERR_ALIGN, name
    assert fwd(y=at(0)) == b.LA_ERR_ALIAS and fwd(x1=at(3)) == b.LA_ERR_ALIAS
    # a part of wider rows: y right behind the last element is fine, inside the last row is not
    inside = at(0) + (15 * 128 + 64) * 4 - 16
    assert fwd(ldx=128, y=inside) == b.LA_ERR_ALIAS
    ok2 = dict(x=at(0), ldx=64, w=at(1), bias=at(2), x0=at(3), lengths=NULL, dy=at(4), dx1=at(5), dx=at(6), dw=at(7), db=at(8), dx0=at(9), B=2, N=8, E=64,
               W=4, silu=1, t=0, ws=at(10), ws_bytes=0, stream=NULL)
    bwd = lambda **c: call(lib.la_conv_bwd, ok2, **c)
    need = lib.la_conv_bwd_workspace(2, 8, 64, 4, 0)
    assert need >= 5 * 64 * 4 and lib.la_conv_bwd_workspace(2, 8, 64, 9, 0) == 0
    assert bwd() == b.LA_ERR_WORKSPACE and bwd(ws_bytes=need - 1) == b.LA_ERR_WORKSPACE
    assert bwd(dy=NULL) == b.LA_ERR_NULL and bwd(dx=NULL) == b.LA_ERR_NULL
    assert bwd(ws_bytes=need, dx0=at(3)) == b.LA_ERR_ALIAS and bwd(ws_bytes=need, dw=at(1)) == b.LA_ERR_ALIAS
    st = dict(x=at(0), w=at(1), bias=at(2), state=at(3), y=at(4), B=2, E=64, W=4, silu=1, t=0, stream=NULL)
    step = lambda **c: call(lib.la_conv_step, st, **c)
    assert step(state=NULL) == b.LA_ERR_NULL and step(W=5) == b.LA_ERR_UNSUPPORTED and step(B=0) == b.LA_ERR_SHAPE
    assert step(y=at(3)) == b.LA_ERR_ALIAS and step(state=at(0)) == b.LA_ERR_ALIAS and step(y=ODD) == b.LA_ERR_ALIGN


def test_scan_refusals(b):
    lib = b.raw()
    ok = dict(x=at(0), ldx=64, dt=at(1), lddt=64, z=at(2), ldz=64, Bt=at(3), ldb=32, Ct=at(4), ldc=32, A=at(5), D=at(6), dt_bias=at(7), h0=at(8),
              lengths=at(9), y=at(10), h1=at(11), B=2, N=8, E=64, G=2, S=16, flags=1, t=0, ws=NULL, ws_bytes=0, stream=NULL)
    fwd = lambda **c: call(lib.la_scan_fwd, ok, **c)
    assert fwd(S=4) == b.LA_ERR_UNSUPPORTED and fwd(S=64) == b.LA_ERR_UNSUPPORTED and fwd(t=2) == b.LA_ERR_UNSUPPORTED and fwd(flags=4) == b.LA_ERR_UNSUPPORTED
    for name in ("x", "dt", "Bt", "Ct", "A", "y"):
        assert fwd(**{name: NULL}) == b.LA_ERR_NULL, name
    for name in ("B", "N", "E", "G"):
        assert fwd(**{name: 0}) == b.LA_ERR_SHAPE, name
    assert fwd(G=3) == b.LA_ERR_SHAPE and fwd(B=1 << 23) == b.LA_ERR_SHAPE
    for name in ("ldx", "lddt", "ldz"):
        assert fwd(**{name: 63}) == b.LA_ERR_SHAPE, name
    for name in ("ldb", "ldc"):
        assert fwd(**{name: 31}) == b.LA_ERR_SHAPE, name
    for name in ("x", "dt", "z", "Bt", "Ct", "A", "D", "dt_bias", "h0", "lengths", "y", "h1"):
        assert fwd(**{name: ODD}) == b.LA_ERR_ALIGN, name
    for name in ("x", "dt", "z", "Bt", "Ct", "A", "D", "dt_bias", "h0", "lengths", "h1"):
        assert fwd(y=ok[name]) == b.LA_ERR_ALIAS, name
    keep = lib.la_scan_fwd_workspace(2, 8, 64, 2, 16, 0, 3)
    assert lib.la_scan_fwd_workspace(2, 8, 64, 2, 16, 0, 1) == 0 and keep == 2 * 64 * 16 * 4
    assert fwd(flags=3) == b.LA_ERR_WORKSPACE and fwd(flags=3, ws=at(12), ws_bytes=keep - 1) == b.LA_ERR_WORKSPACE
    assert fwd(flags=3, ws=at(11), ws_bytes=keep) == b.LA_ERR_ALIAS
    # a long sequence is cut, and its pieces' states need room
    assert lib.la_scan_fwd_workspace(1, 4096, 64, 1, 16, 0, 1) > 0 and fwd(B=1, N=4096, E=64, G=1) == b.LA_ERR_WORKSPACE
    assert lib.la_scan_fwd_workspace(1, 4096, 64, 1, 12, 0, 1) == 0

    ok2 = dict(x=at(0), ldx=64, dt=at(1), lddt=64, z=at(2), ldz=64, Bt=at(3), ldb=32, Ct=at(4), ldc=32, A=at(5), D=at(6), dt_bias=at(7), h0=at(8),
               lengths=NULL, fwd_ws=at(9), dy=at(10), dh1=at(11), dx=at(12), ddt=at(13), dz=at(14), dB=at(15), dC=at(16), dA=at(17), dD=at(18),
               ddt_bias=at(19), dh0=at(20), B=2, N=8, E=64, G=2, S=16, flags=1, t=0, ws=at(21), ws_bytes=1 << 22, stream=NULL)
    bwd = lambda **c: call(lib.la_scan_bwd, ok2, **c)
    with_states, without = (lib.la_scan_bwd_workspace(2, 8, 64, 2, 16, 0, flags) for flags in (3, 1))
    assert without == with_states + keep
    assert bwd(ws_bytes=with_states - 1) == b.LA_ERR_WORKSPACE and bwd(fwd_ws=NULL, ws_bytes=with_states) == b.LA_ERR_WORKSPACE
    for name in ("dy", "dx", "ddt", "dB", "dC", "dA", "dz", "z"):
        assert bwd(**{name: NULL}) == b.LA_ERR_NULL, name
    for name in ("dx", "ddt", "dz", "dB", "dC", "dA", "dD", "ddt_bias", "dh0"):
        assert bwd(**{name: ok2["dy"]}) == b.LA_ERR_ALIAS and bwd(**{name: ODD}) == b.LA_ERR_ALIGN, name
    assert bwd(ws=at(9)) == b.LA_ERR_ALIAS

    st = dict(x=at(0), dt=at(1), z=at(2), Bt=at(3), Ct=at(4), A=at(5), D=at(6), dt_bias=at(7), h=at(8), y=at(9), B=2, E=64, G=2, S=16, flags=1, t=0, stream=NULL)
    step = lambda **c: call(lib.la_scan_step, st, **c)
    assert step(h=NULL) == b.LA_ERR_NULL and step(S=24) == b.LA_ERR_UNSUPPORTED and step(flags=3) == b.LA_ERR_UNSUPPORTED
    assert step(G=5) == b.LA_ERR_SHAPE and step(y=at(8)) == b.LA_ERR_ALIAS and step(h=at(5)) == b.LA_ERR_ALIAS and step(z=ODD) == b.LA_ERR_ALIGN


def test_binding_checks_every_tensor(b):
    import paper_2006_16236_amd as la

    def refused(fn, *args, match, error=ValueError, **kw):
        with pytest.raises(error, match=match):
            fn(*args, **kw)

    B, N, E, S, W = 2, 6, 64, 16, 4
    x, w, y, v = torch.zeros(B, N, E), torch.zeros(E, W), torch.zeros(B, N, E), torch.zeros(E)
    refused(la.la_norm_fwd, x.half(), v, v, y, match="dtype", error=TypeError)
    refused(la.la_norm_fwd, x, v[:-1], v, y, match="gamma: shape")
    refused(la.la_norm_fwd, x, v.bfloat16(), v, y, match="gamma: dtype")
    refused(la.la_norm_fwd, x, v, v, y[:, 1:], match="y: shape")
    refused(la.la_norm_fwd, x.transpose(0, 1), v, v, y.transpose(0, 1), match="x must be contiguous")
    refused(la.la_norm_fwd, x, v, v, y, torch.zeros(B), match="mean: shape")
    refused(la.la_norm_fwd, x, v, v, y, match="device tensors")
    refused(la.la_norm_bwd, x, v, torch.zeros(B, N), torch.zeros(B, N), x.bfloat16(), y, match="dy: dtype")
    refused(la.la_norm_bwd, x, v, None, torch.zeros(B, N), x, y, match="mean is required")
    refused(la.la_conv_fwd, x, w.t(), v, y, match="w: shape")
    refused(la.la_conv_fwd, x, w, v, y, x0=torch.zeros(B, W, E), match="x0: shape")
    refused(la.la_conv_fwd, x, w, v, y, lengths=torch.zeros(B, dtype=torch.int64), match="lengths: dtype")
    refused(la.la_conv_fwd, x[..., ::2], w[::2].contiguous(), v[::2].contiguous(), y[..., ::2].contiguous(), match="rows must be dense")
    refused(la.la_conv_fwd, torch.zeros(B, 2 * N, E)[:, :N], w, v, y, match="one distance")
    refused(la.la_conv_fwd, x, w, v, y, match="device tensors")
    refused(la.la_conv_bwd, x, w, v, y, torch.zeros(B, N, 2 * E)[..., :E], match="dx must be contiguous")
    refused(la.la_conv_step, x[:, 0].contiguous(), w, v, torch.zeros(B, W, E), y[:, 0].contiguous(), match="state: shape")
    dt, A, Bt, h = torch.zeros(B, N, E), torch.zeros(E, S), torch.zeros(B, N, 1, S), torch.zeros(B, E, S)
    refused(la.la_scan_fwd, x, dt, A, Bt[:, :, 0], Bt, y, match="Bt must be")
    refused(la.la_scan_fwd, x, dt, A, torch.zeros(B, N, 3, S), torch.zeros(B, N, 3, S), y, match="do not divide")
    refused(la.la_scan_fwd, x, dt.bfloat16(), A, Bt, Bt, y, match="dt: dtype")
    refused(la.la_scan_fwd, x, dt, A.t().contiguous(), Bt, Bt, y, match="A: shape")
    refused(la.la_scan_fwd, x, dt, A, Bt, Bt, y, h0=h[:, :-1], match="h0: shape")
    refused(la.la_scan_fwd, x, dt, A, Bt, Bt, y, match="device|CPU", error=(ValueError, RuntimeError))
    refused(la.la_scan_bwd, x, dt, A, Bt, Bt, y, y, y, A, Bt, Bt, z=x, match="dz goes with z")
    refused(la.la_scan_bwd, x, dt, A, Bt, Bt, y, y, y, A, Bt, Bt, fwd_ws=torch.zeros(8), match="fwd_ws: 32 bytes")
    refused(la.la_scan_step, x[:, 0].contiguous(), dt[:, 0].contiguous(), A, Bt[:, 0].contiguous(), Bt[:, 0].contiguous(), h[:1], y[:, 0].contiguous(),
            match="h: shape")


def test_the_cut_covers_every_token_once(b):
    """pieces x tiles of a piece, as the workspace query shows them: at least 4 tiles a piece, and never more room than
    the longest allowed cut needs."""
    lib = b.raw()
    for S in (8, 16, 32):
        for E in (1, 64, 100, 1000, 4096):
            for N in (1, 16, 63, 64, 65, 127, 128, 1000, 4096, 32768):
                room = lib.la_scan_fwd_workspace(1, N, E, 1, S, 0, 1)
                tiles = (N + 15) // 16
                if tiles < 8:
                    assert room == 0
                assert room <= (tiles // 4) * (E * S * 4 + E * 4) + 512


def test_sizes_beyond_int_are_refused(b):
    """int holds a size, and int what is counted beyond it; ctypes would take the lower 32 bits of any number."""
    import paper_2006_16236_amd as la
    lib = b.raw()
    args = (at(1), None, None, None, at(2), None)
    for n in ((1 << 30) + 1, (1 << 31) - 1):
        assert lib.la_conv_fwd(at(0), 4, *args, 1, n, 4, 4, 1, 0, NULL) == b.LA_ERR_SHAPE
        assert lib.la_conv_fwd(at(0), n, *args, 1, 1, n, 4, 1, 0, NULL) == b.LA_ERR_SHAPE
        assert lib.la_conv_bwd_workspace(1, n, 1, 4, 0) == 0 and lib.la_conv_bwd_workspace(1, 1, n, 4, 0) == 0
        assert lib.la_scan_fwd_workspace(1, n, 1, 1, 8, 0, 1) == 0 and lib.la_scan_bwd_workspace(1, n, 1, 1, 8, 0, 1) == 0
    assert lib.la_conv_bwd_workspace(1, 1 << 30, 1, 4, 0) > 0 and lib.la_scan_fwd_workspace(1, 1 << 30, 1, 1, 8, 0, 3) > 0
    # tensors that are all strides: nothing is allocated
    far = torch.empty((1 << 32) + 128, device="meta").as_strided((2, 1, 4), ((1 << 32) + 64, 4, 1))
    w, v, y = (torch.empty(s, device="meta") for s in ((4, 4), (4,), (2, 1, 4)))
    with pytest.raises(ValueError, match="x: the distance between tokens is 4294967360"):
        la.la_conv_fwd(far, w, v, y)
    long = torch.empty((1 << 32) + 4, 1, device="meta")
    with pytest.raises(ValueError, match="number of rows"):
        la.la_norm_fwd(long, None, None, long)
    stat = torch.empty((1 << 32) + 4, device="meta")
    with pytest.raises(ValueError, match="number of rows"):
        la.la_norm_bwd(long, None, stat, stat, long, long)
    many = torch.empty(1, (1 << 32) + 4, 1, device="meta")
    with pytest.raises(ValueError, match="a size of x"):
        la.la_conv_fwd(many, torch.empty(1, 4, device="meta"), None, many)
