"""The operators around the attention on torch tensors: layer norm with the residual sum, the short causal
convolution and the selective state space scan of include/la.h.

As in binding.py this is argument checking and marshalling only.  Inputs called rows [B, N, E] may be parts of a
wider tensor (the half of a projection's output): their last dimension dense, their tokens at one distance.
Everything else is dense.  A call runs on its tensors' device, on `stream` or that device's current stream.  What it
writes counts as changed in place: a backward that has saved such a tensor (a state that has been stepped on) is refused.

Each function first offers the call to its native counterpart (csrc/la_call.cpp), which takes it where all is as
expected and the tensors are on the current device; otherwise it goes through the checks here, which name what is wrong.
"""
from __future__ import annotations

import torch

from . import binding as _b
from .binding import LA_SCAN_KEEP, LA_SCAN_SOFTPLUS, _bytes, _call, _check, _lib, _like

_F32 = torch.float32
_CODES = {torch.float32: _b.LA_F32, torch.bfloat16: _b.LA_BF16}


def _code(name, t):
    try:
        return _CODES[t.dtype]
    except AttributeError:
        raise TypeError(f"{name} must be a torch.Tensor") from None
    except KeyError:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}: float32 or bfloat16") from None


def _dims(name, t, n):
    if t.dim() != n:
        raise ValueError(f"{name} must have {n} dimensions, not {t.dim()}")
    return _ints(f"a size of {name}", *t.shape)


def _ints(what, *sizes):
    """The sizes, each one that the C ABI's int holds (ctypes would cut off the rest)."""
    for n in sizes:
        if n > 0x7FFFFFFF:
            raise ValueError(f"{what} is {n}, at most {0x7FFFFFFF} is possible")
    return sizes


def _rows(name, t, shape, dtype, device, optional=False):
    """The distance between tokens of `t` [B, N, ...], whose rows are dense and equally far apart (0 without it)."""
    if t is None:
        if optional:
            return 0
        raise ValueError(f"{name} is required")
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if t.device != device:
        raise ValueError(f"{name}: device {t.device}, expected {device}")
    B, N, stride = shape[0], shape[1], t.stride()
    width = 1
    for n, s in zip(reversed(shape[2:]), reversed(stride[2:])):
        if n != 1 and s != width:
            raise ValueError(f"{name}: the rows must be dense")
        width *= n
    ld = stride[1] if N > 1 else stride[0] if B > 1 else width
    if ld < width or (B > 1 and stride[0] != N * ld):
        raise ValueError(f"{name}: the tokens of all sequences must lie at one distance")
    return _ints(f"{name}: the distance between tokens", ld)[0]


def _run(where, device, stream, call, written):
    """call(stream handle) with `device` current: launches go to the current device, whose stream it must be.
    written: the tensors it writes (None: not asked for)."""
    if device.type != "cuda":
        raise ValueError("tensors must be contiguous device tensors")
    if stream is None:
        stream = torch.cuda.current_stream(device)
    handle = (stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)) or None
    if device.index == torch.cuda.current_device():
        _check(call(handle), where)
    else:
        with torch.cuda.device(device):
            _check(call(handle), where)
    torch.autograd.graph.increment_version([t for t in written if t is not None])


def _p(t):
    return None if t is None else t.data_ptr()


def _workspace(ws, need, device, stream):
    """The caller's workspace, or a new one of the memory of the stream that uses it."""
    if ws is None:
        if stream is None or device.type != "cuda":
            return torch.empty(max(need, 16), dtype=torch.uint8, device=device)
        if not isinstance(stream, torch.cuda.Stream):
            handle = int(getattr(stream, "cuda_stream", stream))
            stream = torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)
        with torch.cuda.stream(stream):
            return torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    _bytes("ws", ws, device)
    return ws


def _size(ws):
    return ws.numel() * ws.element_size()


# ---- layer norm ----------------------------------------------------------------------------------

def la_norm_bwd_workspace(rows, E, dtype_code=_b.LA_F32) -> int:
    return int(_lib.la_norm_bwd_workspace(rows, E, dtype_code))


def la_norm_fwd(x, gamma, beta, y, mean=None, rstd=None, r=None, s=None, eps=1e-5, stream=None):
    """y = layer norm of s = x + r over the last dimension of x [..., E]; gamma, beta [E] fp32 or None.  s: where
    the sum goes (only with r); mean, rstd [...] fp32: what la_norm_bwd needs."""
    took = _call.norm_fwd(x, gamma, beta, y, mean, rstd, r, s, eps) if stream is None else None
    if took is not None:
        return _check(took, "la_norm_fwd")
    t, shape, dt, dev = _code("x", x), x.shape, x.dtype, x.device
    if len(shape) < 1:
        raise ValueError("x must have at least one dimension")
    E, lead = shape[-1], shape[:-1]
    _ints("the number of rows or their width", lead.numel(), E)
    _like("x", x, shape, dt, dev)
    _like("y", y, shape, dt, dev)
    _like("r", r, shape, dt, dev, optional=True)
    _like("s", s, shape, dt, dev, optional=True)
    for name, v in (("gamma", gamma), ("beta", beta)):
        _like(name, v, (E,), _F32, dev, optional=True)
    for name, v in (("mean", mean), ("rstd", rstd)):
        _like(name, v, lead, _F32, dev, optional=True)
    if x.numel() == 0:
        raise ValueError(f"x: shape {tuple(shape)} is empty")
    _run("la_norm_fwd", dev, stream,
         lambda q: _lib.la_norm_fwd(_p(x), _p(r), _p(gamma), _p(beta), _p(y), _p(s), _p(mean), _p(rstd), lead.numel(), E,
                                    float(eps), t, q), (y, mean, rstd, s))


def la_norm_bwd(s, gamma, mean, rstd, dy, dx, dgamma=None, dbeta=None, ds=None, ws=None, stream=None):
    """dx (the gradient of x and of r), dgamma, dbeta from dy; s: what was normalised; ds: the gradient of the
    sum from elsewhere.  Returns the workspace it used (None if it needed none)."""
    took = _call.norm_bwd(s, gamma, mean, rstd, dy, dx, dgamma, dbeta, ds, ws) if stream is None else None
    if took is not None:
        if type(took) is int:
            _check(took, "la_norm_bwd")
        return took
    t, shape, dt, dev = _code("s", s), s.shape, s.dtype, s.device
    if len(shape) < 1:
        raise ValueError("s must have at least one dimension")
    E, lead = shape[-1], shape[:-1]
    _ints("the number of rows or their width", lead.numel(), E)
    for name, v in (("s", s), ("dy", dy), ("dx", dx)):
        _like(name, v, shape, dt, dev)
    _like("ds", ds, shape, dt, dev, optional=True)
    for name, v in (("gamma", gamma), ("dgamma", dgamma), ("dbeta", dbeta)):
        _like(name, v, (E,), _F32, dev, optional=True)
    for name, v in (("mean", mean), ("rstd", rstd)):
        _like(name, v, lead, _F32, dev)
    if s.numel() == 0:
        raise ValueError(f"s: shape {tuple(shape)} is empty")
    rows = lead.numel()
    if dgamma is not None or dbeta is not None:
        ws = _workspace(ws, la_norm_bwd_workspace(rows, E, t), dev, stream)
    _run("la_norm_bwd", dev, stream,
         lambda q: _lib.la_norm_bwd(_p(s), _p(gamma), _p(mean), _p(rstd), _p(dy), _p(ds), _p(dx), _p(dgamma), _p(dbeta),
                                    rows, E, t, _p(ws), 0 if ws is None else _size(ws), q), (dx, dgamma, dbeta))
    return ws


# ---- short causal convolution --------------------------------------------------------------------

def la_conv_bwd_workspace(B, N, E, W, dtype_code=_b.LA_F32) -> int:
    return int(_lib.la_conv_bwd_workspace(B, N, E, W, dtype_code))


def _conv_checks(x, w, bias, n):
    t, dt, dev = _code("x", x), x.dtype, x.device
    shape = _dims("x", x, n)
    if not isinstance(w, torch.Tensor) or w.dim() != 2:
        raise ValueError("w must be a tensor [E, W]")
    E, W = shape[-1], _dims("w", w, 2)[1]
    _like("w", w, (E, W), _F32, dev)
    _like("bias", bias, (E,), _F32, dev, optional=True)
    return t, dt, dev, shape, W


def la_conv_fwd(x, w, bias, y, x0=None, x1=None, lengths=None, silu=True, stream=None):
    """Causal convolution of x [B, N, E] with w [E, W] fp32 and bias [E] or None into y; x0, x1 [B, W-1, E]: the rows
    before the first token and the last ones; lengths [B] int32."""
    took = _call.conv_fwd(x, w, bias, y, x0, x1, lengths, silu) if stream is None else None
    if took is not None:
        return _check(took, "la_conv_fwd")
    t, dt, dev, (B, N, E), W = _conv_checks(x, w, bias, 3)
    ldx = _rows("x", x, (B, N, E), dt, dev)
    _like("y", y, (B, N, E), dt, dev)
    _like("x0", x0, (B, W - 1, E), dt, dev, optional=True)
    _like("x1", x1, (B, W - 1, E), dt, dev, optional=True)
    _like("lengths", lengths, (B,), torch.int32, dev, optional=True)
    _run("la_conv_fwd", dev, stream,
         lambda q: _lib.la_conv_fwd(_p(x), ldx, _p(w), _p(bias), _p(x0), _p(lengths), _p(y), _p(x1), B, N, E, W, int(silu), t, q), (y, x1))


def la_conv_bwd(x, w, bias, dy, dx, dw=None, db=None, x0=None, dx1=None, dx0=None, lengths=None, silu=True, ws=None,
                stream=None):
    """dx, dw, db, dx0 of la_conv_fwd from dy and dx1, the gradient of the rows handed on.  Returns the workspace
    it used (None if it needed none)."""
    took = _call.conv_bwd(x, w, bias, dy, dx, dw, db, x0, dx1, dx0, lengths, silu, ws) if stream is None else None
    if took is not None:
        if type(took) is int:
            _check(took, "la_conv_bwd")
        return took
    t, dt, dev, (B, N, E), W = _conv_checks(x, w, bias, 3)
    ldx = _rows("x", x, (B, N, E), dt, dev)
    _like("dy", dy, (B, N, E), dt, dev)
    _like("dx", dx, (B, N, E), dt, dev)
    for name, v in (("x0", x0), ("dx1", dx1), ("dx0", dx0)):
        _like(name, v, (B, W - 1, E), dt, dev, optional=True)
    _like("dw", dw, (E, W), _F32, dev, optional=True)
    _like("db", db, (E,), _F32, dev, optional=True)
    _like("lengths", lengths, (B,), torch.int32, dev, optional=True)
    if dw is not None or db is not None:
        ws = _workspace(ws, la_conv_bwd_workspace(B, N, E, W, t), dev, stream)
    _run("la_conv_bwd", dev, stream,
         lambda q: _lib.la_conv_bwd(_p(x), ldx, _p(w), _p(bias), _p(x0), _p(lengths), _p(dy), _p(dx1), _p(dx), _p(dw), _p(db),
                                    _p(dx0), B, N, E, W, int(silu), t, _p(ws), 0 if ws is None else _size(ws), q), (dx, dw, db, dx0))
    return ws


def la_conv_step(x, w, bias, state, y, silu=True, stream=None):
    """One token of every sequence: x, y [B, E]; state [B, W-1, E] holds the rows before it and is moved on."""
    took = _call.conv_step(x, w, bias, state, y, silu) if stream is None else None
    if took is not None:
        return _check(took, "la_conv_step")
    t, dt, dev, (B, E), W = _conv_checks(x, w, bias, 2)
    _like("x", x, (B, E), dt, dev)
    _like("y", y, (B, E), dt, dev)
    _like("state", state, (B, W - 1, E), dt, dev)
    _run("la_conv_step", dev, stream,
         lambda q: _lib.la_conv_step(_p(x), _p(w), _p(bias), _p(state), _p(y), B, E, W, int(silu), t, q), (state, y))


# ---- selective scan ------------------------------------------------------------------------------

def la_scan_fwd_workspace(B, N, E, G, S, dtype_code=_b.LA_F32, flags=LA_SCAN_SOFTPLUS) -> int:
    return int(_lib.la_scan_fwd_workspace(B, N, E, G, S, dtype_code, flags))


def la_scan_bwd_workspace(B, N, E, G, S, dtype_code=_b.LA_F32, flags=LA_SCAN_SOFTPLUS) -> int:
    """flags with LA_SCAN_KEEP: for a call that is given the forward's workspace."""
    return int(_lib.la_scan_bwd_workspace(B, N, E, G, S, dtype_code, flags))


class _Scan:
    """Checks the inputs of a scan: sizes from x and Bt, distances between tokens."""

    def __init__(self, x, dt, A, Bt, Ct, D, z, dt_bias, lengths):
        self.t, self.dtype, self.dev = _code("x", x), x.dtype, x.device
        self.B, self.N, self.E = B, N, E = _dims("x", x, 3)
        if not isinstance(Bt, torch.Tensor) or Bt.dim() != 4:
            raise ValueError("Bt must be a tensor [B, N, G, S]")
        self.G, self.S = G, S = _dims("Bt", Bt, 4)[2:]
        if G < 1 or E % G:
            raise ValueError(f"Bt: {G} groups do not divide {E} channels")
        rows, bc = (B, N, E), (B, N, G, S)
        self.rows, self.bc, self.state = rows, bc, (B, E, S)
        self.ld = [_rows("x", x, rows, self.dtype, self.dev), _rows("dt", dt, rows, self.dtype, self.dev),
                   _rows("z", z, rows, self.dtype, self.dev, optional=True), _rows("Bt", Bt, bc, self.dtype, self.dev),
                   _rows("Ct", Ct, bc, self.dtype, self.dev)]
        _like("A", A, (E, S), _F32, self.dev)
        _like("D", D, (E,), _F32, self.dev, optional=True)
        _like("dt_bias", dt_bias, (E,), _F32, self.dev, optional=True)
        _like("lengths", lengths, (B,), torch.int32, self.dev, optional=True)
        self.dims = (B, N, E, G, S)

    def states(self, **named):
        for name, t in named.items():
            _like(name, t, self.state, _F32, self.dev, optional=True)

    def inputs(self, x, dt, z, Bt, Ct):
        ld = self.ld
        return _p(x), ld[0], _p(dt), ld[1], _p(z), ld[2], _p(Bt), ld[3], _p(Ct), ld[4]


def la_scan_fwd(x, dt, A, Bt, Ct, y, D=None, z=None, dt_bias=None, h0=None, h1=None, lengths=None, softplus=True,
                keep=False, ws=None, stream=None):
    """Selective scan of x, dt, z [B, N, E] with Bt, Ct [B, N, G, S], A [E, S], D and dt_bias [E] fp32 into y; h0, h1
    [B, E, S] fp32: the states before and after; lengths [B] int32.  Returns the workspace it used; with
    keep=True it holds what la_scan_bwd starts from (fwd_ws)."""
    took = _call.scan_fwd(x, dt, A, Bt, Ct, y, D, z, dt_bias, h0, h1, lengths, softplus, keep, ws) if stream is None else None
    if took is not None:
        if type(took) is int:
            _check(took, "la_scan_fwd")
        return took
    k = _Scan(x, dt, A, Bt, Ct, D, z, dt_bias, lengths)
    _like("y", y, k.rows, k.dtype, k.dev)
    k.states(h0=h0, h1=h1)
    flags = (LA_SCAN_SOFTPLUS if softplus else 0) | (LA_SCAN_KEEP if keep else 0)
    ws = _workspace(ws, la_scan_fwd_workspace(*k.dims, k.t, flags), k.dev, stream)
    _run("la_scan_fwd", k.dev, stream,
         lambda q: _lib.la_scan_fwd(*k.inputs(x, dt, z, Bt, Ct), _p(A), _p(D), _p(dt_bias), _p(h0), _p(lengths), _p(y), _p(h1),
                                    *k.dims, flags, k.t, _p(ws), _size(ws), q), (y, h1))
    return ws


def la_scan_bwd(x, dt, A, Bt, Ct, dy, dx, ddt, dA, dB, dC, D=None, z=None, dt_bias=None, dD=None, dz=None,
                ddt_bias=None, h0=None, dh1=None, dh0=None, lengths=None, softplus=True, fwd_ws=None, ws=None, stream=None):
    """The gradients of la_scan_fwd from dy [B, N, E] and dh1 [B, E, S], the gradient of the state handed on.  fwd_ws: the
    workspace of la_scan_fwd(keep=True) on the same inputs (None: its states are formed again).  Returns the
    workspace it used."""
    took = _call.scan_bwd(x, dt, A, Bt, Ct, dy, dx, ddt, dA, dB, dC, D, z, dt_bias, dD, dz, ddt_bias, h0, dh1, dh0, lengths, softplus, fwd_ws, ws) if stream is None else None
    if took is not None:
        if type(took) is int:
            _check(took, "la_scan_bwd")
        return took
    k = _Scan(x, dt, A, Bt, Ct, D, z, dt_bias, lengths)
    for name, v in (("dy", dy), ("dx", dx), ("ddt", ddt)):
        _like(name, v, k.rows, k.dtype, k.dev)
    if (z is None) != (dz is None):
        raise ValueError("dz goes with z")
    _like("dz", dz, k.rows, k.dtype, k.dev, optional=True)
    _like("dB", dB, k.bc, k.dtype, k.dev)
    _like("dC", dC, k.bc, k.dtype, k.dev)
    _like("dA", dA, (k.E, k.S), _F32, k.dev)
    _like("dD", dD, (k.E,), _F32, k.dev, optional=True)
    _like("ddt_bias", ddt_bias, (k.E,), _F32, k.dev, optional=True)
    k.states(h0=h0, dh1=dh1, dh0=dh0)
    flags = LA_SCAN_SOFTPLUS if softplus else 0
    kept = 0
    if fwd_ws is not None:
        _bytes("fwd_ws", fwd_ws, k.dev)
        kept = LA_SCAN_KEEP
        need = la_scan_fwd_workspace(*k.dims, k.t, flags | kept)
        if _size(fwd_ws) < need:
            raise ValueError(f"fwd_ws: {_size(fwd_ws)} bytes, {need} expected: not a workspace of la_scan_fwd(keep=True) on these sizes")
    ws = _workspace(ws, la_scan_bwd_workspace(*k.dims, k.t, flags | kept), k.dev, stream)
    _run("la_scan_bwd", k.dev, stream,
         lambda q: _lib.la_scan_bwd(*k.inputs(x, dt, z, Bt, Ct), _p(A), _p(D), _p(dt_bias), _p(h0), _p(lengths), _p(fwd_ws),
                                    _p(dy), _p(dh1), _p(dx), _p(ddt), _p(dz), _p(dB), _p(dC), _p(dA), _p(dD), _p(ddt_bias),
                                    _p(dh0), *k.dims, flags, k.t, _p(ws), _size(ws), q), (dx, ddt, dA, dB, dC, dD, dz, ddt_bias, dh0))
    return ws


def la_scan_step(x, dt, A, Bt, Ct, h, y, D=None, z=None, dt_bias=None, softplus=True, stream=None):
    """One token of every sequence: x, dt, z, y [B, E]; Bt, Ct [B, G, S]; h [B, E, S] fp32, updated in place."""
    took = _call.scan_step(x, dt, A, Bt, Ct, h, y, D, z, dt_bias, softplus) if stream is None else None
    if took is not None:
        return _check(took, "la_scan_step")
    t, dtype, dev = _code("x", x), x.dtype, x.device
    B, E = _dims("x", x, 2)
    if not isinstance(Bt, torch.Tensor) or Bt.dim() != 3:
        raise ValueError("Bt must be a tensor [B, G, S]")
    G, S = _dims("Bt", Bt, 3)[1:]
    if G < 1 or E % G:
        raise ValueError(f"Bt: {G} groups do not divide {E} channels")
    for name, v in (("x", x), ("dt", dt), ("y", y)):
        _like(name, v, (B, E), dtype, dev)
    _like("z", z, (B, E), dtype, dev, optional=True)
    _like("Bt", Bt, (B, G, S), dtype, dev)
    _like("Ct", Ct, (B, G, S), dtype, dev)
    _like("A", A, (E, S), _F32, dev)
    _like("h", h, (B, E, S), _F32, dev)
    _like("D", D, (E,), _F32, dev, optional=True)
    _like("dt_bias", dt_bias, (E,), _F32, dev, optional=True)
    _run("la_scan_step", dev, stream,
         lambda q: _lib.la_scan_step(_p(x), _p(dt), _p(z), _p(Bt), _p(Ct), _p(A), _p(D), _p(dt_bias), _p(h), _p(y), B, E, G, S,
                                     LA_SCAN_SOFTPLUS if softplus else 0, t, q), (h, y))


# ---- norm of queries and keys for each head, with the rotation -----------------------------------

_NORMS = {None: 0, "rms": _b.LA_QK_RMS, "l2": _b.LA_QK_L2}


def la_qk_bwd_workspace(B, N, H, Hk, D, dtype_code=_b.LA_F32) -> int:
    return int(_lib.la_qk_bwd_workspace(B, N, H, Hk, D, dtype_code))


class _Qk:
    """Checks the inputs of a head norm: sizes from q and k, distances between tokens."""

    def __init__(self, q, k, wq, wk, freq, pos, lengths, norm, adjacent):
        self.t, self.dtype, self.dev = _code("q", q), q.dtype, q.device
        self.B, self.N, self.H, self.D = B, N, H, D = _dims("q", q, 4)
        if norm not in _NORMS:
            raise ValueError("norm must be 'rms', 'l2' or None")
        self.flags = _NORMS[norm] | (_b.LA_QK_ADJACENT if adjacent else 0)
        self.ldq = _rows("q", q, (B, N, H, D), self.dtype, self.dev)
        self.Hk, self.ldk = 0, 0
        if k is not None:
            _code("k", k)
            self.Hk = _dims("k", k, 4)[2]
            self.ldk = _rows("k", k, (B, N, self.Hk, D), self.dtype, self.dev)
        self.qs, self.ks = (B, N, H, D), (B, N, self.Hk, D)
        for name, w in (("wq", wq), ("wk", wk)):
            _like(name, w, (D,), _F32, self.dev, optional=True)
        self.R = 0
        if freq is not None:
            if not isinstance(freq, torch.Tensor) or freq.dim() != 1:
                raise ValueError("freq must be a tensor [R / 2]")
            _like("freq", freq, freq.shape, _F32, self.dev)
            self.R = 2 * freq.shape[0]
        _like("pos", pos, (B, N), torch.int32, self.dev, optional=True)
        _like("lengths", lengths, (B,), torch.int32, self.dev, optional=True)
        self.dims = (B, N, H, self.Hk, D, self.R, self.flags)

    def of_keys(self, k, **named):
        for name, t in named.items():
            if (k is None) != (t is None):
                raise ValueError(f"{name} goes with k")
            _like(name, t, self.ks, self.dtype, self.dev, optional=True)


def la_qk_fwd(q, yq, k=None, yk=None, wq=None, wk=None, freq=None, pos=None, lengths=None, norm="rms", adjacent=False, eps=1e-6, stream=None):
    """Norm of each head of q [B, N, H, D] and k [B, N, Hk, D] or None ("rms", "l2" or None) with weights wq, wk [D] fp32, and the
    rotation of its first 2 len(freq) elements by pos * freq (pos [B, N] int32; None: 0 .. N - 1), into yq, yk; pairs are i and
    i + len(freq), or with adjacent=True neighbours; lengths [B] int32."""
    took = _call.qk_fwd(q, yq, k, yk, wq, wk, freq, pos, lengths, norm, adjacent, eps) if stream is None else None
    if took is not None:
        return _check(took, "la_qk_fwd")
    c = _Qk(q, k, wq, wk, freq, pos, lengths, norm, adjacent)
    _like("yq", yq, c.qs, c.dtype, c.dev)
    c.of_keys(k, yk=yk)
    _run("la_qk_fwd", c.dev, stream,
         lambda s: _lib.la_qk_fwd(_p(q), c.ldq, _p(k), c.ldk, _p(wq), _p(wk), _p(freq), _p(pos), _p(lengths), _p(yq), _p(yk), *c.dims,
                                  float(eps), c.t, s), (yq, yk))


def la_qk_bwd(q, dyq, dq, k=None, dyk=None, dk=None, wq=None, wk=None, freq=None, pos=None, lengths=None, norm="rms", adjacent=False,
              eps=1e-6, dwq=None, dwk=None, ws=None, stream=None):
    """dq, dk, dwq, dwk of la_qk_fwd from dyq, dyk.  Returns the workspace it used (None if it needed none)."""
    c = _Qk(q, k, wq, wk, freq, pos, lengths, norm, adjacent)
    for name, t in (("dyq", dyq), ("dq", dq)):
        _like(name, t, c.qs, c.dtype, c.dev)
    c.of_keys(k, dyk=dyk, dk=dk)
    for name, t in (("dwq", dwq), ("dwk", dwk)):
        _like(name, t, (c.D,), _F32, c.dev, optional=True)
    if k is None and dwk is not None:
        raise ValueError("dwk goes with k")
    if dwq is not None or dwk is not None:
        ws = _workspace(ws, la_qk_bwd_workspace(c.B, c.N, c.H, c.Hk, c.D, c.t), c.dev, stream)
    _run("la_qk_bwd", c.dev, stream,
         lambda s: _lib.la_qk_bwd(_p(q), c.ldq, _p(k), c.ldk, _p(wq), _p(wk), _p(freq), _p(pos), _p(lengths), _p(dyq), _p(dyk), _p(dq),
                                  _p(dk), _p(dwq), _p(dwk), *c.dims, float(eps), c.t, _p(ws), 0 if ws is None else _size(ws), s),
         (dq, dk, dwq, dwk))
    return ws


# ---- gated delta rule ------------------------------------------------------------------------------

def la_delta_fwd_workspace(B, N, H, Hk, D, M, dtype_code=_b.LA_F32, flags=0) -> int:
    return int(_lib.la_delta_fwd_workspace(B, N, H, Hk, D, M, dtype_code, flags))


def la_delta_bwd_workspace(B, N, H, Hk, D, M, dtype_code=_b.LA_F32, flags=0) -> int:
    """flags = LA_DELTA_KEEP: for a call that is given the forward's workspace."""
    return int(_lib.la_delta_bwd_workspace(B, N, H, Hk, D, M, dtype_code, flags))


class _Delta:
    """Checks the inputs of a delta rule: sizes from q and v, distances between tokens."""

    def __init__(self, q, k, v, g, beta, lengths, scale):
        self.t, self.dtype, self.dev = _code("q", q), q.dtype, q.device
        B, N, Hk, D = _dims("q", q, 4)
        if not isinstance(v, torch.Tensor) or v.dim() != 4:
            raise ValueError("v must be a tensor [B, N, H, M]")
        H, M = _dims("v", v, 4)[2:]
        if Hk < 1 or H % Hk:
            raise ValueError(f"q: {Hk} heads do not divide the {H} of v")
        self.keys, self.rows, self.per, self.state = (B, N, Hk, D), (B, N, H, M), (B, N, H), (B, H, D, M)
        self.ld = [_rows("q", q, self.keys, self.dtype, self.dev), _rows("k", k, self.keys, self.dtype, self.dev),
                   _rows("v", v, self.rows, self.dtype, self.dev)]
        _like("g", g, self.per, _F32, self.dev, optional=True)
        _like("beta", beta, self.per, _F32, self.dev)
        _like("lengths", lengths, (B,), torch.int32, self.dev, optional=True)
        self.scale = float(D) ** -0.5 if scale is None else float(scale)
        self.dims = (B, N, H, Hk, D, M)

    def states(self, **named):
        for name, t in named.items():
            _like(name, t, self.state, _F32, self.dev, optional=True)

    def inputs(self, q, k, v, g, beta, h0, lengths):
        return _p(q), self.ld[0], _p(k), self.ld[1], _p(v), self.ld[2], _p(g), _p(beta), _p(h0), _p(lengths)


def la_delta_fwd(q, k, v, g, beta, o, h0=None, h1=None, lengths=None, scale=None, keep=False, ws=None, stream=None):
    """Gated delta rule of q, k [B, N, Hk, D], v [B, N, H, M] with logarithms of the decay g (or None) and strengths beta
    [B, N, H] fp32 into o [B, N, H, M]; h0, h1 [B, H, D, M] fp32: the states before and after; lengths [B] int32; scale (None:
    D ** -0.5) is that of the outputs.  Returns the workspace it used; with keep=True it holds what la_delta_bwd starts
    from (fwd_ws)."""
    took = _call.delta_fwd(q, k, v, g, beta, o, h0, h1, lengths, scale, keep, ws) if stream is None else None
    if took is not None:
        if type(took) is int:
            _check(took, "la_delta_fwd")
        return took
    c = _Delta(q, k, v, g, beta, lengths, scale)
    _like("o", o, c.rows, c.dtype, c.dev)
    c.states(h0=h0, h1=h1)
    flags = _b.LA_DELTA_KEEP if keep else 0
    ws = _workspace(ws, la_delta_fwd_workspace(*c.dims, c.t, flags), c.dev, stream)
    _run("la_delta_fwd", c.dev, stream,
         lambda s: _lib.la_delta_fwd(*c.inputs(q, k, v, g, beta, h0, lengths), _p(o), _p(h1), *c.dims, c.scale, flags, c.t, _p(ws),
                                     _size(ws), s), (o, h1))
    return ws


def la_delta_bwd(q, k, v, g, beta, do, dq, dk, dv, dg, dbeta, h0=None, dh1=None, dh0=None, lengths=None, scale=None, fwd_ws=None,
                 ws=None, stream=None):
    """The gradients of la_delta_fwd from do [B, N, H, M] and dh1 [B, H, D, M], the gradient of the state handed on.  fwd_ws: the
    workspace of la_delta_fwd(keep=True) on the same inputs (None: it is formed again).  Returns the workspace it used."""
    c = _Delta(q, k, v, g, beta, lengths, scale)
    _like("do", do, c.rows, c.dtype, c.dev)
    _like("dv", dv, c.rows, c.dtype, c.dev)
    for name, t in (("dq", dq), ("dk", dk)):
        _like(name, t, c.keys, c.dtype, c.dev)
    if (g is None) != (dg is None):
        raise ValueError("dg goes with g")
    _like("dg", dg, c.per, _F32, c.dev, optional=True)
    _like("dbeta", dbeta, c.per, _F32, c.dev)
    c.states(h0=h0, dh1=dh1, dh0=dh0)
    flags = 0
    if fwd_ws is not None:
        _bytes("fwd_ws", fwd_ws, c.dev)
        flags = _b.LA_DELTA_KEEP
        need = la_delta_fwd_workspace(*c.dims, c.t, flags)
        if _size(fwd_ws) < need:
            raise ValueError(f"fwd_ws: {_size(fwd_ws)} bytes, {need} expected: not a workspace of la_delta_fwd(keep=True) on these sizes")
    ws = _workspace(ws, la_delta_bwd_workspace(*c.dims, c.t, flags), c.dev, stream)
    _run("la_delta_bwd", c.dev, stream,
         lambda s: _lib.la_delta_bwd(*c.inputs(q, k, v, g, beta, h0, lengths), _p(fwd_ws), _p(do), _p(dh1), _p(dq), _p(dk), _p(dv),
                                     _p(dg), _p(dbeta), _p(dh0), *c.dims, c.scale, flags, c.t, _p(ws), _size(ws), s),
         (dq, dk, dv, dg, dbeta, dh0))
    return ws


def la_delta_step(q, k, v, g, beta, h, o, scale=None, stream=None):
    """One token of every sequence: q, k [B, Hk, D]; v, o [B, H, M]; g (or None), beta [B, H] fp32; h [B, H, D, M] fp32, updated in
    place."""
    took = _call.delta_step(q, k, v, g, beta, h, o, scale) if stream is None else None
    if took is not None:
        return _check(took, "la_delta_step")
    t, dtype, dev = _code("q", q), q.dtype, q.device
    B, Hk, D = _dims("q", q, 3)
    if not isinstance(v, torch.Tensor) or v.dim() != 3:
        raise ValueError("v must be a tensor [B, H, M]")
    H, M = _dims("v", v, 3)[1:]
    if Hk < 1 or H % Hk:
        raise ValueError(f"q: {Hk} heads do not divide the {H} of v")
    for name, x, shape in (("q", q, (B, Hk, D)), ("k", k, (B, Hk, D)), ("v", v, (B, H, M)), ("o", o, (B, H, M))):
        _like(name, x, shape, dtype, dev)
    _like("g", g, (B, H), _F32, dev, optional=True)
    _like("beta", beta, (B, H), _F32, dev)
    _like("h", h, (B, H, D, M), _F32, dev)
    _run("la_delta_step", dev, stream,
         lambda s: _lib.la_delta_step(_p(q), _p(k), _p(v), _p(g), _p(beta), _p(h), _p(o), B, H, Hk, D, M,
                                      float(D) ** -0.5 if scale is None else float(scale), t, s), (h, o))
