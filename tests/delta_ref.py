"""The gated delta rule and the head norm with rotation, with their gradients, in fp64 (numpy) token by token from the
definitions, and the bounds that the GPU's results are held to.

Bounds.  A rounding of fp32 is off by a value spread over +-2^-24 of its result.  n of them that do not depend on each other
add up to a standard deviation of sqrt(n / 3) 2^-24; K = 5 of these are allowed, of the 2-norm of a row (a head's vector of one
token) or of a state.  n = D + 2 * 64 + 32: a sum over D elements, two over the tokens of a chunk, and what is done to single values.
An error of the state goes on through S -> e^g (1 - beta k k^T) S, which lengthens nothing while beta |k|^2 <= 2: so
  e_t^2 = e^{2 g_t} e_{t-1}^2 + (n / 3) 2^-48 size_t^2,
where size_t adds up the norms of all that S_t is made of since the start of the token's 64 (the state then, and what each token
wrote).  The same holds for the state's gradient, backwards.  What is read off the states has the product rule's errors."""
import numpy as np

U32 = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
K = 5.0
CHUNK = 64


def norm(v):
    return np.sqrt((v * v).sum(-1))


def delta(q, k, v, g, beta, h0=None, lengths=None, scale=1.0, do=None, dh1=None):
    """q, k [B, N, Hk, D], v [B, N, H, M], g, beta [B, N, H] -> results, and under "e_" + name their bounds, one for each head's
    vector (or state)."""
    B, N, Hk, D = q.shape
    H, M = v.shape[2:]
    per = H // Hk
    real = np.arange(N)[None] < (np.full(B, N) if lengths is None else np.clip(lengths, 0, N))[:, None]      # [B, N]

    def clean(t):
        return np.where(real.reshape(B, N, *(1,) * (t.ndim - 2)), t.astype(np.float64), 0.0)

    q, k, v, beta = np.repeat(clean(q), per, 2), np.repeat(clean(k), per, 2), clean(v), clean(beta)
    a = np.exp(clean(g)) if g is not None else np.ones((B, N, H))
    n = D + 2 * CHUNK + 32
    u2 = n / 3 * U32 ** 2
    u1 = np.sqrt(u2)
    S = np.zeros((B, H, D, M)) if h0 is None else h0.astype(np.float64)
    e2, size = np.zeros((B, H)), np.sqrt((S * S).sum((2, 3)))
    states, misses, errs, sizes = [S], [], [np.sqrt(e2)], []
    o, e_o = np.zeros((B, N, H, M)), np.zeros((B, N, H))
    nk, nq = norm(k), norm(q)
    e_miss = np.zeros((B, N, H))
    for t in range(N):
        if t % CHUNK == 0:
            size = np.sqrt((S * S).sum((2, 3)))
        before = S * a[:, t, :, None, None]
        miss = v[:, t] - (before * k[:, t, ..., None]).sum(2)
        S = before + k[:, t, ..., None] * (beta[:, t, :, None] * miss)[:, :, None]
        fresh = norm(v[:, t]) + nk[:, t] * a[:, t] * size            # what the missing part is the difference of
        e_miss[:, t] = nk[:, t] * a[:, t] * errs[-1] + u1 * fresh
        size = a[:, t] * size + nk[:, t] * np.abs(beta[:, t]) * norm(miss)
        e2 = a[:, t] ** 2 * e2 + u2 * (size ** 2 + (nk[:, t] * beta[:, t] * fresh) ** 2)
        o[:, t] = scale * (S * q[:, t, ..., None]).sum(2)
        e_o[:, t] = abs(scale) * nq[:, t] * (np.sqrt(e2) + u1 * size)
        states.append(S)
        misses.append(miss)
        errs.append(np.sqrt(e2))
        sizes.append(size)
    out = {"o": np.where(real[..., None, None], o, 0.0), "h1": S, "e_o": K * e_o, "e_h1": K * (errs[-1] + u1 * size)}
    if do is None:
        return out
    do = scale * clean(do)
    G = np.zeros_like(S) if dh1 is None else dh1.astype(np.float64)
    f2 = np.zeros((B, H))
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    dg, dbeta = np.zeros((B, N, H)), np.zeros((B, N, H))
    e = {x: np.zeros((B, N, H)) for x in ("dq", "dk", "dv", "dg", "dbeta")}
    sizeG = np.sqrt((G * G).sum((2, 3)))
    for t in range(N - 1, -1, -1):
        if t == N - 1 or t % CHUNK == CHUNK - 1:
            sizeG, inchunk = np.sqrt((G * G).sum((2, 3))), np.zeros((B, H))
            inchunk += (u1 * sizeG * sizes[t] + np.sqrt(f2) * sizes[t] + sizeG * errs[t + 1]) ** 2         # <dS', S'>
        S, before, miss, b = states[t + 1], states[t] * a[:, t, :, None, None], misses[t], beta[:, t]
        nd, size, es = norm(do[:, t]), sizes[t], errs[t + 1]
        dq[:, t] = (S * do[:, t, :, None]).sum(3)
        e["dq"][:, t] = nd * (es + u1 * size)
        G = G + q[:, t, ..., None] * do[:, t, :, None]
        sizeG = sizeG + nq[:, t] * nd
        along = (G * k[:, t, ..., None]).sum(2)
        ef = np.sqrt(f2)
        e_along = nk[:, t] * (ef + u1 * sizeG)
        dbeta[:, t] = (along * miss).sum(-1)
        e["dbeta"][:, t] = e_along * norm(miss) + norm(along) * e_miss[:, t] + u1 * norm(along) * norm(miss)
        dv[:, t] = b[..., None] * along
        e["dv"][:, t] = np.abs(b) * e_along
        dk[:, t] = (G * (b[..., None] * miss)[:, :, None]).sum(3) - (before * dv[:, t, :, None]).sum(3)
        e["dk"][:, t] = (ef + u1 * sizeG) * np.abs(b) * norm(miss) + sizeG * np.abs(b) * e_miss[:, t] \
            + (a[:, t] * errs[t] + u1 * size) * norm(dv[:, t]) + size * e["dv"][:, t]
        G = G - k[:, t, ..., None] * dv[:, t, :, None]
        sizeG = sizeG + nk[:, t] * norm(dv[:, t])
        dg[:, t] = (G * before).sum((2, 3))
        # formed as a sum over the later tokens of the chunk of what their vectors give
        inchunk = inchunk + (nq[:, t] * (e["dq"][:, t] + u1 * norm(dq[:, t])) + nk[:, t] * (e["dk"][:, t] + u1 * norm(dk[:, t]))
                             + 2 * e["dv"][:, t] * norm(v[:, t] - miss) + 2 * norm(dv[:, t]) * (e_miss[:, t] + u1 * (norm(v[:, t]) + norm(miss)))) ** 2
        e["dg"][:, t] = np.sqrt(inchunk)
        f2 = a[:, t] ** 2 * (f2 + u2 * sizeG ** 2 * (1 + (nk[:, t] ** 2 * b) ** 2))
        G = G * a[:, t, :, None, None]
        sizeG = sizeG * a[:, t]
    shared = lambda x: x.reshape(B, N, Hk, per, *x.shape[3:]).sum(3)  # noqa: E731
    out.update(dq=shared(dq), dk=shared(dk), dv=dv, dg=np.where(real[..., None], dg, 0.0), dbeta=np.where(real[..., None], dbeta, 0.0), dh0=G)
    out.update(e_dq=K * shared(e["dq"]), e_dk=K * shared(e["dk"]), e_dh0=K * (np.sqrt(f2) + u1 * sizeG), **{"e_" + x: K * e[x] for x in ("dv", "dg", "dbeta")})
    return out


def check(name, got, want, dtype):
    """2-norms: of a head's vectors, of states; single values of dg and dbeta."""
    got, ref, room = np.asarray(got, dtype=np.float64), want[name], want["e_" + name]
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert np.isfinite(got).all(), f"{name}: not finite"
    size = np.sqrt if name in ("h1", "dh0") else None
    off, ref = ((d * d).sum((2, 3)) if size else d * d if d.ndim == 3 else (d * d).sum(-1) for d in (got - ref, ref))
    off, ref = np.sqrt(off), np.sqrt(ref)
    kind = "f32" if name in ("h1", "dh0", "dg", "dbeta") else dtype
    bad = off / (room * (1 + 2.0 ** -7) + HALF_STEP[kind] * ref + 1e-37)
    assert bad.size == 0 or bad.max() <= 1.0, f"{name}: {bad.max():.3g} times the bound at {np.unravel_index(bad.argmax(), bad.shape)}"
    return bad.max() if bad.size else 0.0


# ---- head norm and rotation ---------------------------------------------------------------------------

def qk(x, w, freq, pos, lengths, kind, adjacent, eps, dy=None, mag=False):
    """One of q, k [B, N, H, D].  mag=True: the magnitudes of what is added up, for layer_ref.check."""
    f = np.abs if mag else (lambda v: v)
    B, N, H, D = x.shape
    ends = np.full(B, N) if lengths is None else np.clip(lengths, 0, N)
    real = (np.arange(N)[None] < ends[:, None])[..., None, None]
    x = np.where(real, x.astype(np.float64), 0.0)
    squares = (x * x).sum(-1, keepdims=True) / (D if kind == "rms" else 1)
    r = np.ones_like(squares) if kind is None else 1.0 / np.sqrt(squares + eps)
    w = np.ones(D) if w is None else w.astype(np.float64)
    R = 0 if freq is None else 2 * len(freq)
    first, second = (np.arange(0, R, 2), np.arange(1, R, 2)) if adjacent else (np.arange(R // 2), np.arange(R // 2, R))
    if R:
        at = np.broadcast_to(np.arange(N), (B, N)) if pos is None else pos
        angle = (at.astype(np.float64)[..., None] * freq.astype(np.float64))[:, :, None]
        c, s = np.cos(angle), np.sin(angle)

    def turn(t, sign):
        t = t.copy()
        if R:
            u, v = t[..., first], t[..., second]
            if mag:
                t[..., first] = t[..., second] = np.abs(u) + np.abs(v)      # cosines and sines are off by a share of 1, not of themselves
            else:
                t[..., first], t[..., second] = u * c - sign * v * s, v * c + sign * u * s
        return t

    unit = f(x * r)
    out = {"y": np.where(real, turn(f(unit * w), 1), 0.0)}
    if dy is not None:
        dn = turn(f(np.where(real, dy.astype(np.float64), 0.0)), -1)
        out["dw"] = f(dn * unit).sum((0, 1, 2))
        gw = f(dn * w)
        along = f(gw * unit).sum(-1, keepdims=True) / (D if kind == "rms" else 1)
        back = 0.0 if kind is None else unit * along
        out["dx"] = np.where(real, r * (gw + back) if mag else r * (gw - back), 0.0)
    return out
