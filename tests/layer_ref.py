"""Layer norm, short causal convolution and selective scan with their gradients in fp64 (numpy), token by token
from the formulas, and the bounds the GPU's results are held to.

Every function takes mag=True: all factors and terms then enter with their absolute values, so that a result is
the sum of the magnitudes of what is added up.  An fp32 evaluation that rounds k times along each path from an
input to a result is off by at most about k 2^-24 of that sum, whatever cancels."""
import numpy as np

U32 = 2.0 ** -24                                   # half a step of fp32
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def check(name, got, ref, mag, dtype, k):
    """|got - ref| <= k 2^-24 mag + half a step of the type for the rounding of what is stored (of the computed
    value, which differs from ref by the first term: hence the factor 1 + 2^-7 on it)."""
    got, ref, mag = (np.asarray(t, dtype=np.float64) for t in (got, ref, mag))
    assert got.shape == ref.shape == mag.shape, (name, got.shape, ref.shape, mag.shape)
    assert np.isfinite(got).all(), f"{name}: not finite"
    room = k * U32 * mag * (1 + 2.0 ** -7) + HALF_STEP[dtype] * np.abs(ref) + 1e-37
    bad = np.abs(got - ref) / room
    assert bad.size == 0 or bad.max() <= 1.0, f"{name}: {bad.max():.3g} times the bound at {np.unravel_index(bad.argmax(), bad.shape)}"


def _abs(mag):
    return np.abs if mag else (lambda v: v)


def sigmoid(v):
    e = np.exp(-np.abs(v))                         # both branches without cancellation
    return np.where(v >= 0, 1.0, e) / (1.0 + e)


def to_bf16(a):
    """Rounded to the nearest bf16, ties to even."""
    u = np.asarray(a, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7fff + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)


# ---- layer norm: s [R, E] -----------------------------------------------------------------------------

def norm(s, gamma, beta, eps, dy=None, ds=None, mag=False):
    f = _abs(mag)
    s = s.astype(np.float64)
    E = s.shape[1]
    mean = s.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((s - mean) ** 2).mean(1, keepdims=True) + eps)
    # magnitude of s - mean: what the two are made of
    xhat = (np.abs(s) + np.abs(s).mean(1, keepdims=True)) * rstd if mag else (s - mean) * rstd
    gamma = np.ones(E) if gamma is None else gamma.astype(np.float64)
    beta = np.zeros(E) if beta is None else beta.astype(np.float64)
    # the mean of squares carries the errors of s - mean: their share in rstd, relative, is at most max xhat's excess
    out = {"y": f(xhat * gamma) + f(beta), "mean": np.abs(s).mean(1) if mag else mean[:, 0], "rstd": rstd[:, 0]}
    if mag:
        grow = (xhat ** 2).mean(1)                 # >= 1: how much the variance's terms exceed the variance
        out["rstd"] = out["rstd"] * grow
        out["y"] = out["y"] * (1 + grow[:, None])
    if dy is not None:
        dy = dy.astype(np.float64)
        g = f(dy * gamma)
        m1, m2 = g.mean(1, keepdims=True), (f(g * xhat)).mean(1, keepdims=True)
        dx = rstd * (g + m1 + xhat * m2) if mag else rstd * (g - m1 - xhat * m2)
        out["dx"] = dx + (0 if ds is None else f(ds.astype(np.float64)))
        out["dgamma"], out["dbeta"] = f(dy * xhat).sum(0), f(dy).sum(0)
        if mag:
            out["dx"] = out["dx"] * (1 + grow[:, None])
            out["dgamma"] = (f(dy * xhat) * (1 + grow[:, None])).sum(0)
    return out


# ---- convolution: x [B, N, E] -------------------------------------------------------------------------

def conv(x, w, bias, x0, lengths, silu, dy=None, dx1=None, mag=False):
    f = _abs(mag)
    B, N, E = x.shape
    W = w.shape[1]
    ends = np.full(B, N) if lengths is None else np.clip(lengths, 0, N)
    w = w.astype(np.float64)
    bias = np.zeros(E) if bias is None else bias.astype(np.float64)
    out = {"y": np.zeros((B, N, E)), "x1": np.zeros((B, W - 1, E))}
    if dy is not None:
        out.update(dx=np.zeros((B, N, E)), dw=np.zeros((E, W)), db=np.zeros(E), dx0=np.zeros((B, W - 1, E)))
    for b, n in enumerate(ends):
        line = np.zeros((n + W - 1, E))
        if x0 is not None:
            line[:W - 1] = x0[b]
        line[W - 1:] = x[b, :n]
        out["x1"][b] = line[n:]
        dline = np.zeros_like(line)
        if dx1 is not None:
            dline[n:] += f(dx1[b].astype(np.float64))
        for t in range(n):
            p = bias + (w.T * line[t:t + W]).sum(0)
            pm = f(bias) + f(w.T * line[t:t + W]).sum(0)
            q = sigmoid(p)
            # silu's slope is at most 1.1, so an error of p is one of y
            out["y"][b, t] = ((pm * 1.1 + np.abs(p)) if mag else p * q) if silu else pm
            if dy is None:
                continue
            slope = q * (1 + p * (1 - q)) if silu else np.ones(E)
            # |slope'| <= 0.5: an error of p enters the slope with that factor; its own terms are at most 1 + |p|
            slope = (1.0 + np.abs(p) * q + 0.5 * pm if silu else slope) if mag else slope
            d = f(dy[b, t].astype(np.float64)) * slope
            dline[t:t + W] += d * f(w.T)
            out["dw"] += (d * f(line[t:t + W])).T
            out["db"] += d
        if dy is not None:
            out["dx"][b, :n] = dline[W - 1:]
            out["dx0"][b] = dline[:W - 1]
    return out


# ---- scan ---------------------------------------------------------------------------------------------

def scan(x, dt, A, Bt, Ct, D=None, z=None, dt_bias=None, h0=None, lengths=None, softplus=True, dy=None, dh1=None, mag=False):
    f = _abs(mag)
    B, N, E = x.shape
    G, S = Bt.shape[2:]
    x, dt, Bt, Ct = (t.astype(np.float64) for t in (x, dt, Bt, Ct))
    A = A.astype(np.float64)
    D = np.zeros(E) if D is None else D.astype(np.float64)
    bias = np.zeros(E) if dt_bias is None else dt_bias.astype(np.float64)
    ends = np.full(B, N) if lengths is None else np.clip(lengths, 0, N)
    group = np.arange(E) // (E // G)
    shape = (B, N, E)
    out = {"y": np.zeros(shape), "h1": np.zeros((B, E, S))}
    train = dy is not None
    if train:
        out.update(dx=np.zeros(shape), ddt=np.zeros(shape), dz=np.zeros(shape), dB=np.zeros(Bt.shape), dC=np.zeros(Bt.shape),
                   dA=np.zeros((E, S)), dD=np.zeros(E), ddt_bias=np.zeros(E), dh0=np.zeros((B, E, S)))
    for b, n in enumerate(ends):
        h = np.zeros((E, S)) if h0 is None else f(h0[b].astype(np.float64))
        before, saved = [], []
        for t in range(n):
            raw = dt[b, t] + bias
            d = np.logaddexp(raw, 0.0) if softplus else raw
            a = np.exp(d[:, None] * A)
            Bc, Cc = f(Bt[b, t][group]), f(Ct[b, t][group])
            before.append(h)
            h = a * h + f(d * x[b, t])[:, None] * Bc
            v = (Cc * h).sum(1) + f(D * x[b, t])
            gate = np.ones(E) if z is None else f(z[b, t].astype(np.float64)) * sigmoid(z[b, t].astype(np.float64))
            out["y"][b, t] = v * gate
            saved.append((raw, d, a, Bc, Cc, h, v, gate))
        out["h1"][b] = h
        if not train:
            continue
        g = np.zeros((E, S)) if dh1 is None else f(dh1[b].astype(np.float64))
        for t in range(n - 1, -1, -1):
            raw, d, a, Bc, Cc, h, v, gate = saved[t]
            dyt, xt, da = f(dy[b, t].astype(np.float64)), f(x[b, t]), f(d)
            dv = dyt * gate
            if z is not None:
                zt = z[b, t].astype(np.float64)
                q = sigmoid(zt)
                out["dz"][b, t] = dyt * v * q * (1 + (np.abs(zt) if mag else zt) * (1 - q))
            g = g + dv[:, None] * Cc
            gB = (g * Bc).sum(1)
            pB, pC = g * (da * xt)[:, None], dv[:, None] * h
            for e in range(G):
                out["dB"][b, t, e], out["dC"][b, t, e] = pB[group == e].sum(0), pC[group == e].sum(0)
            g = g * a
            through = g * before[t]
            out["dx"][b, t] = da * gB + f(D) * dv
            dd = (xt * gB + (through * f(A)).sum(1)) * (sigmoid(raw) if softplus else 1.0)
            out["ddt"][b, t] = dd
            out["ddt_bias"] += dd
            out["dA"] += through * da[:, None]
            out["dD"] += dv * xt
        out["dh0"][b] = g
    return out


def roundings(N, S, A, d_max):
    """Roundings on a path of the scan: per token those of exp(d A) (of d, of A log2(e), of their product and of the exp2
    itself: the first three are errors of the exponent, times its size) and of the two operations of the state; sums
    over states and tokens; the functions of dt, z."""
    return N * (4 + 4 * float(np.abs(A).max()) * d_max) + 8 * S + 64
