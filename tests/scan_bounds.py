"""The selective scan and its gradients in 64 bits with a bound for every element: how far an fp32 evaluation may be off,
in units of u = 2^-24, followed along the recurrence.  An error of a state decays with the state, so the bound of a long
sequence is hardly above that of a short one, and states held in fewer bits exceed it.

Counted to first order, each rounding as u of the magnitude of its result (that of its terms' absolute values):
  products, sums, fused operations 1, the exponential and logarithm of the hardware 6 (3 ulp), its reciprocal 2
  v = dt + bias: |v|, and through softplus at most |v| of d for v < 0, 1 above
  d = max(v, 0) + log1p(e), e = exp(-|v|): e to 2 |v| + 6 (the exponent's product and constant), its logarithm to 6, its product,
    the remainder that makes it log1p to 1.5, the sum 1; together at most 3 max(-v, 0) + 18 of d (for v >= 0 log1p(e) 2 v <= d)
  a = exp(d A): the exponent is off by |d A| times that of d, of A log2(e) (its constant and product) and of d times it, the power by 6
  a piece of n tokens decays as exp(A sum d) in two powers: n more of the exponent, and 14 for at least two tokens' 7 each
  sigmoid(z): 2 z^- + 10 (for z >= 0, e / (1 + e) (2 z + 6) + 3 < 10), with v^- = max(-v, 0); of v, which is itself off by |v|:
    3 v^- + 11
Sums of m terms count m of the sum of magnitudes (of a tree, its depth)."""
import numpy as np
import torch


def _t(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).double()


def scan(x, dt, A, Bt, Ct, dy=None, D=None, z=None, dt_bias=None, h0=None, dh1=None, lengths=None, softplus=True, pieces=(1, 1),
         touch=None, touch_grad=None):
    """{name: (value, bound)}.  pieces: how many a sequence is cut into, forwards and backwards.  touch(h, t), touch_grad(g, t):
    what becomes of the state behind token t and of the gradient before it (a tensor [B, E, S]), for wrong evaluations."""
    B, N, E = x.shape
    G, S = Bt.shape[2:]
    x, dt, A, Bt, Ct, dy, z = (_t(v) for v in (x, dt, A, Bt, Ct, dy, z))
    D, bias = (torch.zeros(E, dtype=torch.float64) if v is None else _t(v) for v in (D, dt_bias))
    ends = torch.full((B,), N) if lengths is None else torch.tensor(lengths).clamp(0, N)
    tiles = -(-N // 16)
    tokens = [0 if p == 1 else 16 * -(-tiles // p) for p in pieces]
    blocks, train = -(-(E // G) // 64), dy is not None
    zero = torch.zeros(B, E, S, dtype=torch.float64)
    per_channel = lambda v, t: v[:, t].repeat_interleave(E // G, 1)
    over_channels = lambda v: v.unflatten(1, (G, E // G)).sum(2)
    real = (torch.arange(N)[None] < ends[:, None])[..., None]                     # [B, N, 1]

    raw = dt + bias
    below = (-raw).clamp(min=0)
    d = torch.where(real, torch.logaddexp(raw, torch.zeros_like(raw)) if softplus else raw, 0.0)
    kd = 3 * below + 18 if softplus else torch.ones_like(raw)
    w, mw = d * x, (d * x).abs()
    if z is None:
        gate, kg = torch.ones_like(x), torch.zeros_like(x)
    else:
        zb = (-z).clamp(min=0)
        q, kq = torch.sigmoid(z), 2 * zb + 10
        gate, kg = z * q, kq + 1
    dA = d[..., None] * A                                                          # [B, N, E, S]

    def decay(t, way):
        return torch.exp(dA[:, t]), dA[:, t].abs() * (kd[:, t, :, None] + 3 + tokens[way]) + 7

    out, H, er = {}, zero if h0 is None else _t(h0).abs(), zero.clone()
    h = zero if h0 is None else _t(h0)
    before, after = [], []
    V, mV, eV = (torch.zeros_like(x) for _ in range(3))
    for t in range(N):
        on = real[:, t, :, None]
        a, ka = decay(t, 0)
        b, c = per_channel(Bt, t), per_channel(Ct, t)
        before.append((h, H, er))
        push = mw[:, t, :, None] * b.abs()
        er = torch.where(on, a * er + a * H * ka + push * (kd[:, t, :, None] + 3), er)
        H = torch.where(on, a * H + push, H)
        h = torch.where(on, a * h + w[:, t, :, None] * b, h)
        if touch is not None:
            h = touch(h, t)
        after.append((h, H, er))
        V[:, t] = (c * h).sum(-1) + D * x[:, t]
        mV[:, t] = (c.abs() * H).sum(-1) + (D * x[:, t]).abs()
        eV[:, t] = (c.abs() * er).sum(-1) + mV[:, t] * (S + 3)
    out["y"] = torch.where(real, V * gate, 0.0), torch.where(real, gate.abs() * (eV + mV * (kg + 1)), 0.0)
    out["h1"] = h, er
    if not train:
        return {n: tuple(v.numpy() for v in p) for n, p in out.items()}

    dy = torch.where(real, dy, 0.0)
    dv, kv = dy * gate, (torch.zeros_like(x) if z is None else kg + 1)
    mv = dv.abs()
    if z is not None:
        slope = 1 + z.abs() * (1 - q)
        md = dy.abs() * q * slope
        ed = dy.abs() * q * (slope * (kq + 3) + z.abs() * (q * kq + 2))
        out["dz"] = dy * q * (1 + z * (1 - q)) * V, md * eV + mV * (ed + md)
    sg = torch.sigmoid(raw) if softplus else torch.ones_like(raw)
    ks = 3 * below + 11 if softplus else torch.zeros_like(raw)
    dx, ex, dd, edd = (torch.zeros_like(x) for _ in range(4))
    dB, eB, dC, eC = (torch.zeros_like(Bt) for _ in range(4))
    sA, eA, mA = (torch.zeros(E, S, dtype=torch.float64) for _ in range(3))
    g = zero if dh1 is None else _t(dh1)
    M, eg = g.abs(), zero.clone()
    for t in range(N - 1, -1, -1):
        on = real[:, t, :, None]
        a, ka = decay(t, 1)
        b, c = per_channel(Bt, t), per_channel(Ct, t)
        hb, Hb, eb = before[t]
        ha, Ha, ea = after[t]
        dvt, mvt, kvt, kdt = (v[:, t, :, None] for v in (dv, mv, kv, kd))
        mg = M + mvt * c.abs()
        ge, gn = torch.where(on, eg + mvt * c.abs() * kvt + mg, eg), torch.where(on, g + dvt * c, g)
        mg = torch.where(on, mg, M)
        fold = 7 + blocks
        live = on.double()
        dB[:, t], eB[:, t] = over_channels(live * gn * w[:, t, :, None]), over_channels(live * mw[:, t, :, None] * (ge + mg * (kdt + 2 + fold)))
        dC[:, t], eC[:, t] = over_channels(live * ha * dvt), over_channels(live * mvt * (ea + Ha * (kvt + 1 + fold)))
        gB, mB = (gn * b).sum(-1), (mg * b.abs()).sum(-1)
        eBg = (ge * b.abs()).sum(-1) + mB * S
        eg, M, g = torch.where(on, a * ge + a * mg * ka, ge), torch.where(on, a * mg, mg), torch.where(on, a * gn, gn)
        if touch_grad is not None:
            g = touch_grad(g, t)
        through, mt, et = g * hb, M * Hb, eg * Hb + M * eb + M * Hb
        gA, mgA = (through * A).sum(-1), (mt * A.abs()).sum(-1)
        eGA = (et * A.abs()).sum(-1) + mgA * (S + 5)
        dt_, dm = d[:, t], d[:, t].abs()
        mD = (D * dv[:, t]).abs()
        dx[:, t], ex[:, t] = dt_ * gB + D * dv[:, t], dm * (eBg + mB * (kd[:, t] + 1)) + mD * (kv[:, t] + 2)
        mdd = x[:, t].abs() * mB + mgA
        dd[:, t] = (x[:, t] * gB + gA) * sg[:, t]
        edd[:, t] = sg[:, t] * (x[:, t].abs() * eBg + eGA + mdd * (ks[:, t] + 2))
        sA += (live * through * dt_[..., None]).sum(0)
        eA += (live * dm[..., None] * (et + mt * (kdt + 1))).sum(0)
        mA += (live * dm[..., None] * mt).sum(0)
    for n, v, e in (("dx", dx, ex), ("ddt", dd, edd)):
        out[n] = torch.where(real, v, 0.0), torch.where(real, e, 0.0)
    rows = B * pieces[1]
    last = -(-rows // 16) + 18                                                     # sums over the pieces' partial sums
    in_piece = -(-tiles // pieces[1])
    out["dA"] = sA, eA + mA * (16 + in_piece + last)
    out["dD"] = (dv * x).sum((0, 1)), ((mv * x.abs()) * (kv + 4 * in_piece + 8 + last)).sum((0, 1))
    out["ddt_bias"] = out["ddt"][0].sum((0, 1)), (out["ddt"][1] + out["ddt"][0].abs() * (4 * in_piece + 8 + last)).sum((0, 1))
    out["dB"], out["dC"], out["dh0"] = (dB, eB), (dC, eC), (g, eg)
    return {n: tuple(v.numpy() for v in p) for n, p in out.items()}
