"""torch.autograd front end of the C ABI: differentiable functions.

Marshalling only: forward and backward are the library's kernels (la_causal_fwd / la_causal_bwd,
la_global_fwd / la_global_bwd, and those of layer.py); this file allocates the outputs and tells autograd what to keep.
What is kept for the backward is Q, K, V, the denominators [B, H, N] and the forward's workspace
(the running sums at the segment borders): the attention output itself is not needed, and no
per-position state is stored (the constant-memory backward of section 3.3.1).
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as _b
from . import layer as _l


class _CausalLinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, eps, token_major):
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
        O = torch.empty_like(V)
        if token_major:     # [B, N, H, .]
            B, N, H = Q.shape[:3]
            den = torch.empty((B, H, N), dtype=torch.float32, device=Q.device)
            ws = _b.la_causal_fwd_bnhd(Q, K, V, O, den, eps)
        else:
            den = torch.empty(Q.shape[:-1], dtype=torch.float32, device=Q.device)
            ws = _b.la_causal_fwd(Q, K, V, O, den, eps)
        ctx.save_for_backward(Q, K, V, den, ws)
        ctx.eps, ctx.token_major = eps, token_major
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, den, ws = ctx.saved_tensors
        dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
        bwd = _b.la_causal_bwd_bnhd if ctx.token_major else _b.la_causal_bwd
        bwd(Q, K, V, None, den, dO.contiguous(), dQ, dK, dV, ctx.eps, fwd_ws=ws)
        return dQ, dK, dV, None, None


class _LinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, eps, token_major):
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
        O = torch.empty_like(V)
        if token_major:     # [B, N, H, .]
            B, N, H = Q.shape[:3]
            den = torch.empty((B, H, N), dtype=torch.float32, device=Q.device)
            ws = _b.la_global_fwd_bnhd(Q, K, V, O, eps, den=den)
        else:
            den = torch.empty(Q.shape[:-1], dtype=torch.float32, device=Q.device)
            ws = _b.la_global_fwd(Q, K, V, O, eps, den=den)
        ctx.save_for_backward(Q, K, V, den, ws)
        ctx.eps, ctx.token_major = eps, token_major
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, den, ws = ctx.saved_tensors
        dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
        bwd = _b.la_global_bwd_bnhd if ctx.token_major else _b.la_global_bwd
        bwd(Q, K, V, None, den, dO.contiguous(), dQ, dK, dV, ctx.eps, fwd_ws=ws)
        return dQ, dK, dV, None, None


def causal_linear_attention(Q, K, V, eps: float = 1e-6, layout: str = "bhnd"):
    """Causal linear attention (eq. 9-12) of Q, K [B, H, N, D], V [B, H, N, M] with
    phi(x) = elu(x) + 1; differentiable with respect to Q, K, V.  layout="bnhd": the tensors
    (and the result) are [B, N, H, .], as a fused projection produces them; nothing is transposed."""
    if layout not in ("bhnd", "bnhd"):
        raise ValueError("layout must be 'bhnd' or 'bnhd'")
    return _CausalLinearAttention.apply(Q, K, V, float(eps), layout == "bnhd")


def linear_attention(Q, K, V, eps: float = 1e-6, layout: str = "bhnd"):
    """Non-causal linear attention (eq. 4-6); differentiable with respect to Q, K, V.
    layout as for causal_linear_attention."""
    if layout not in ("bhnd", "bnhd"):
        raise ValueError("layout must be 'bhnd' or 'bnhd'")
    return _LinearAttention.apply(Q, K, V, float(eps), layout == "bnhd")


# ---- the operators around the attention ------------------------------------------------------------

def _dense(t):
    """t as the kernels take it: dense, at 16 bytes (a slice of one row can be dense anywhere)."""
    if t is None:
        return None
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _rows(t):
    """t [B, N, ...] itself where its tokens lie at one distance (a part of a projection's output), else a dense copy."""
    if t is None:
        return None
    B, N, width = t.shape[0], t.shape[1], 1
    for n, s in zip(reversed(t.shape[2:]), reversed(t.stride()[2:])):
        if n != 1 and s != width:
            return _dense(t)
        width *= n
    ld = t.stride(1) if N > 1 else t.stride(0) if B > 1 else width
    if ld < width or (B > 1 and t.stride(0) != N * ld) or t.data_ptr() % 16 != 0:
        return t.clone(memory_format=torch.contiguous_format)
    return t


def _new(t):
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _wanted(flag, t):
    return _new(t) if flag and t is not None else None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gamma, beta, residual, eps):
        ctx.set_materialize_grads(False)
        x, residual, gamma, beta = _dense(x), _dense(residual), _dense(gamma), _dense(beta)
        y, s = _new(x), _new(x) if residual is not None else None
        mean, rstd = (torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) for _ in range(2))
        _l.la_norm_fwd(x, gamma, beta, y, mean, rstd, r=residual, s=s, eps=eps)
        ctx.save_for_backward(x if s is None else s, gamma, mean, rstd)
        ctx.has = gamma is not None, beta is not None, residual is not None
        return y if s is None else (y, s)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, ds=None):
        s, gamma, mean, rstd = ctx.saved_tensors
        has_gamma, has_beta, has_residual = ctx.has
        if dy is None:                                   # only the sum was used
            dgamma = torch.zeros_like(gamma) if has_gamma else None
            dbeta = torch.zeros(s.shape[-1], dtype=torch.float32, device=s.device) if has_beta else None
            return ds, dgamma, dbeta, ds if has_residual else None, None
        dx = _new(s)
        dgamma = _wanted(ctx.needs_input_grad[1], gamma)
        dbeta = torch.empty(s.shape[-1], dtype=torch.float32, device=s.device) if has_beta and ctx.needs_input_grad[2] else None
        _l.la_norm_bwd(s, gamma, mean, rstd, _dense(dy), dx, dgamma, dbeta, ds=_dense(ds))
        return dx, dgamma, dbeta, dx if has_residual else None, None


def layer_norm(x, gamma=None, beta=None, residual=None, eps: float = 1e-5):
    """Layer norm over the last dimension of x (fp32 or bf16), weight gamma and offset beta fp32 or None.  With a
    residual the sum s = x + residual (rounded to their type) is normalised, and (y, s) returned."""
    return _LayerNorm.apply(x, gamma, beta, residual, float(eps))


class _CausalConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, state, lengths, silu):
        ctx.set_materialize_grads(False)
        x, w, bias, state, lengths = _rows(x), _dense(w), _dense(bias), _dense(state), _dense(lengths)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        x1 = torch.empty((x.shape[0], w.shape[1] - 1, x.shape[2]), dtype=x.dtype, device=x.device)
        _l.la_conv_fwd(x, w, bias, y, x0=state, x1=x1, lengths=lengths, silu=silu)
        ctx.save_for_backward(x, w, bias, state, lengths)
        ctx.silu = silu
        return y, x1

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dx1):
        x, w, bias, state, lengths = ctx.saved_tensors
        if dy is None and dx1 is None:
            return (None,) * 6
        dy = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dy is None else _dense(dy)
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        need = ctx.needs_input_grad
        dw, db, dx0 = _wanted(need[1], w), _wanted(need[2], bias), _wanted(need[3], state)
        _l.la_conv_bwd(x, w, bias, dy, dx, dw, db, x0=state, dx1=_dense(dx1), dx0=dx0, lengths=lengths, silu=ctx.silu)
        return dx, dw, db, dx0, None, None


def causal_conv(x, w, bias=None, state=None, lengths=None, silu: bool = True):
    """(y, next state): causal convolution of x [B, N, E] along N with w [E, W] and bias [E] fp32, through silu or not.
    state [B, W-1, E]: the rows before the first token (None: zeros); the next state is the last W - 1 rows, for the next
    piece or la_conv_step.  lengths [B] int32: tokens from lengths[b] on are no part of sequence b."""
    return _CausalConv.apply(x, w, bias, state, lengths, bool(silu))


class _SelectiveScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, A, Bt, Ct, D, z, dt_bias, state, lengths, softplus, keep):
        ctx.set_materialize_grads(False)
        x, dt, z, Bt, Ct = (_rows(t) for t in (x, dt, z, Bt, Ct))
        A, D, dt_bias, state, lengths = (_dense(t) for t in (A, D, dt_bias, state, lengths))
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        h1 = torch.empty((x.shape[0], *A.shape), dtype=torch.float32, device=x.device)
        ws = _l.la_scan_fwd(x, dt, A, Bt, Ct, y, D=D, z=z, dt_bias=dt_bias, h0=state, h1=h1, lengths=lengths, softplus=softplus,
                            keep=keep)
        ctx.save_for_backward(x, dt, A, Bt, Ct, D, z, dt_bias, state, lengths, ws)
        ctx.softplus = softplus
        return y, h1

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh1):
        x, dt, A, Bt, Ct, D, z, dt_bias, state, lengths, ws = ctx.saved_tensors
        if dy is None and dh1 is None:
            return (None,) * 12
        dy = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dy is None else _dense(dy)
        need = ctx.needs_input_grad
        dx, ddt, dB, dC = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (x, dt, Bt, Ct))
        dz = None if z is None else torch.empty(z.shape, dtype=z.dtype, device=z.device)
        dA, dD, db, dh0 = _new(A), _wanted(need[5], D), _wanted(need[7], dt_bias), _wanted(need[8], state)
        _l.la_scan_bwd(x, dt, A, Bt, Ct, dy, dx, ddt, dA, dB, dC, D=D, z=z, dt_bias=dt_bias, dD=dD, dz=dz, ddt_bias=db, h0=state,
                       dh1=_dense(dh1), dh0=dh0, lengths=lengths, softplus=ctx.softplus, fwd_ws=ws)
        return dx, ddt, dA, dB, dC, dD, dz, db, dh0, None, None, None


def selective_scan(x, dt, A, Bt, Ct, D=None, z=None, dt_bias=None, state=None, lengths=None, softplus: bool = True):
    """(y, next state): selective state space scan of x [B, N, E] with steps dt [B, N, E], Bt, Ct [B, N, G, S] (G groups of
    channels), decay rates A [E, S], D and dt_bias [E] fp32, gate z [B, N, E].  state [B, E, S] fp32: the states before the
    first token (None: zero); the next state continues the sequence here or in la_scan_step.  lengths as in causal_conv."""
    inputs = (x, dt, A, Bt, Ct, D, z, dt_bias, state)
    keep = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs)   # the states a backward needs
    return _SelectiveScan.apply(*inputs, lengths, bool(softplus), keep)


# ---- the gated delta rule and what stands before it --------------------------------------------------

class _QkNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, freq, pos, lengths, norm, adjacent, eps):
        ctx.set_materialize_grads(False)
        q, k = _rows(q), _rows(k)
        wq, wk, freq, pos, lengths = (_dense(t) for t in (wq, wk, freq, pos, lengths))
        yq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        yk = None if k is None else torch.empty(k.shape, dtype=k.dtype, device=k.device)
        _l.la_qk_fwd(q, yq, k=k, yk=yk, wq=wq, wk=wk, freq=freq, pos=pos, lengths=lengths, norm=norm, adjacent=adjacent, eps=eps)
        ctx.save_for_backward(q, k, wq, wk, freq, pos, lengths)
        ctx.how = dict(norm=norm, adjacent=adjacent, eps=eps)
        return yq if k is None else (yq, yk)

    @staticmethod
    @once_differentiable
    def backward(ctx, dyq, dyk=None):
        q, k, wq, wk, freq, pos, lengths = ctx.saved_tensors
        if dyq is None and dyk is None:
            return (None,) * 10
        need = ctx.needs_input_grad
        dyq = torch.zeros(q.shape, dtype=q.dtype, device=q.device) if dyq is None else _dense(dyq)
        dq, dk = torch.empty(q.shape, dtype=q.dtype, device=q.device), None
        if k is not None:
            dyk = torch.zeros(k.shape, dtype=k.dtype, device=k.device) if dyk is None else _dense(dyk)
            dk = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        dwq, dwk = _wanted(need[2], wq), _wanted(need[3] and k is not None, wk)
        _l.la_qk_bwd(q, dyq, dq, k=k, dyk=dyk, dk=dk, wq=wq, wk=wk, freq=freq, pos=pos, lengths=lengths, dwq=dwq, dwk=dwk, **ctx.how)
        return dq, dk, dwq, dwk, None, None, None, None, None, None


def qk_norm(q, k=None, wq=None, wk=None, freq=None, pos=None, lengths=None, norm="rms", adjacent: bool = False, eps: float = 1e-6):
    """(q, k) with each head of q [B, N, H, D] and k [B, N, Hk, D] normed ("rms", "l2" for unit length, or None) and weighted with wq, wk
    [D] fp32, and its first 2 len(freq) elements turned by pos * freq: pairs i and i + len(freq), or neighbours.  pos [B, N] int32 (None:
    0 .. N - 1), lengths [B] int32: rows behind it are zero.  Without k, q alone; wk then takes no part.  Differentiable in q, k, wq, wk."""
    return _QkNorm.apply(q, k, wq, wk, freq, pos, lengths, norm, bool(adjacent), float(eps))


def _rows8(t):
    """As _rows, the tokens a multiple of eight elements apart."""
    t = _rows(t)
    return t if t.shape[1] == 1 and t.shape[0] == 1 or t.stride(1 if t.shape[1] > 1 else 0) % 8 == 0 else _dense(t.clone(memory_format=torch.contiguous_format))


class _GatedDelta(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, g, beta, state, lengths, scale, keep):
        ctx.set_materialize_grads(False)
        q, k, v = (_rows8(t) for t in (q, k, v))
        g, beta, state, lengths = (_dense(t) for t in (g, beta, state, lengths))
        o = torch.empty(v.shape, dtype=v.dtype, device=v.device)
        h1 = torch.empty((v.shape[0], v.shape[2], q.shape[3], v.shape[3]), dtype=torch.float32, device=v.device)
        ws = _l.la_delta_fwd(q, k, v, g, beta, o, h0=state, h1=h1, lengths=lengths, scale=scale, keep=keep)
        ctx.save_for_backward(q, k, v, g, beta, state, lengths, ws if keep else None)
        ctx.scale = scale
        return o, h1

    @staticmethod
    @once_differentiable
    def backward(ctx, do, dh1):
        q, k, v, g, beta, state, lengths, ws = ctx.saved_tensors
        if do is None and dh1 is None:
            return (None,) * 9
        do = torch.zeros(v.shape, dtype=v.dtype, device=v.device) if do is None else _dense(do)
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        dg, dbeta, dh0 = None if g is None else _new(g), _new(beta), _wanted(ctx.needs_input_grad[5], state)
        _l.la_delta_bwd(q, k, v, g, beta, do, dq, dk, dv, dg, dbeta, h0=state, dh1=_dense(dh1), dh0=dh0, lengths=lengths, scale=ctx.scale,
                        fwd_ws=ws)
        return dq, dk, dv, dg, dbeta, dh0, None, None, None


def gated_delta(q, k, v, g, beta, state=None, lengths=None, scale=None):
    """(o, next state): gated delta rule of q, k [B, N, Hk, D] (keys of about unit length, see qk_norm), v [B, N, H, M] with logarithms of
    the decay g (or None) and strengths beta [B, N, H] fp32; H / Hk neighbouring states share a head of q, k.  state [B, H, D, M] fp32:
    that before the first token (None: zero); the next one continues the sequence here or in la_delta_step.  scale (None: D ** -0.5) is
    that of the outputs.  lengths as in causal_conv."""
    inputs = (q, k, v, g, beta, state)
    keep = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs)      # what a backward starts from
    return _GatedDelta.apply(*inputs, lengths, None if scale is None else float(scale), keep)
