"""What a layer with a gated delta rule needs, and how it is timed: the norm of queries and keys for each head with the
position rotation in the same pass (`la_qk_*`), and the gated delta rule itself (`la_delta_*`), the recurrence on the
attention's state that writes a value in the place of what the state holds for a key.  Each forward, forward + backward,
and for one new token of every sequence.

`run` makes a user's calls of the library where `own` is true, and computes the same from elementary torch
operations in fp32 where it is false.

qk     n = x w / sqrt(mean(x^2) + eps) of each head (l2: the sum instead of the mean), then the pairs (n_i, n_j) of the
       first R elements are turned by pos * freq_i: i and j = i + R/2, or neighbours (adjacent)
delta  S_t = exp(g_t) S_{t-1} + beta_t k_t (v_t - exp(g_t) S_{t-1}^T k_t)^T,  o_t = scale S_t^T q_t;  H heads of D x M
       states, Hk heads of queries and keys, each for H / Hk neighbouring states; h0 and h1 are the states before and after

Sequences of different lengths: tokens from lengths[b] on are not part of sequence b, their output rows are 0.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
CHUNK = 64                             # tokens that the plain delta rule takes together
MAX_QK = 8 * 2048 * 32 * 128           # B * N * (H + Hk) * D of the largest listed norm with rotation
MAX_DELTA = 8 * 2048 * 16 * 128 * 128  # B * N * H * D * M of the largest listed training step
MAX_PROMPT = 32768 * 16 * 128 * 128    # ... of the largest listed prompt
MAX_ROWS = 8 * 2048 * 16 * 256         # B * N * H * (D + M) of either
MAX_STATE = 512 * 16 * 128 * 128       # B * H * D * M of the largest listed step


def _qk(kind, B, N, H, Hk, D, dtype="bf16", R=None, norm="rms", weight=True, adjacent=False, ragged=False, strided=False, name=None):
    c = {"op": "qk", "kind": kind, "B": B, "N": N, "H": H, "Hk": Hk, "D": D, "R": D if R is None else R, "dtype": dtype, "norm": norm,
         "weight": weight, "adjacent": adjacent, "ragged": ragged, "strided": strided}
    return c if name is None else {"name": name, **c}


def _delta(kind, B, N, H, Hk, D, M, dtype="bf16", ragged=False, state=False, strided=False, name=None):
    c = {"op": "delta", "kind": kind, "B": B, "N": N, "H": H, "Hk": Hk, "D": D, "M": M, "dtype": dtype, "ragged": ragged, "state": state,
         "strided": strided}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # queries and keys of 64 sequences that decode a token each (8 heads of 64), at far positions: latency
        _qk("forward", 64, 1, 8, 8, 64, name="qk_decode_B64"),
        # prompts of different lengths, shared keys, a head that no power of two divides, half of it turned
        _qk("forward", 3, 2531, 6, 2, 96, "f32", R=48, adjacent=True, ragged=True, name="qk_prefill_ragged_f32"),
        # training step before a delta rule: unit length without weights, nothing turned
        _qk("train", 4, 1531, 4, 4, 64, "f32", R=0, norm="l2", weight=False, name="qk_train_l2_f32"),
        # training step of a wide model; queries and keys are parts of one projection's output
        _qk("train", 8, 2048, 16, 16, 128, strided=True, name="qk_train_D128"),
        # one token of 64 sequences through the delta rule
        _delta("step", 64, 1, 8, 8, 64, 64, state=True, name="delta_step_B64"),
        # the same for a batch whose states fill the memory system
        _delta("step", 512, 1, 16, 8, 128, 128, "f32", state=True, name="delta_step_B512_f32"),
        # a few tokens more for each of many sequences in flight
        _delta("prefill", 64, 33, 8, 4, 64, 64, ragged=True, state=True, name="delta_append_B64"),
        # prompts of different lengths from a state, values of another width than the keys
        _delta("prefill", 5, 1531, 6, 3, 64, 80, "f32", ragged=True, state=True, name="delta_prefill_ragged_f32"),
        # one long prompt: few heads, many tokens
        _delta("prefill", 1, 32768, 16, 8, 128, 128, state=True, strided=True, name="delta_prefill_N32768"),
        # training step on two sequences of odd length, shared queries and keys, from a state
        _delta("train", 2, 4095, 8, 4, 64, 64, "f32", state=True, name="delta_train_N4095_f32"),
        # training step on 28 x 28 pixels as tokens, 8 heads of 32
        _delta("train", 8, 784, 8, 8, 32, 32, name="delta_train_N784"),
        # training step on a batch of sequences; queries, keys and values are parts of one projection's output
        _delta("train", 8, 2048, 16, 16, 128, 128, strided=True, name="delta_train_D128"),
    ]


def _log_int(rng, lo, hi):
    hi = max(lo, hi)
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = rng.choice(("f32", "bf16", "bf16"))
    ragged, strided = rng.random() < 0.4, rng.random() < 0.4
    Hk = rng.choice((1, 2, 3, 4, 6, 8, 8, 12, 16))
    if rng.random() < 0.4:
        kind = rng.choice(("decode", "forward", "train", "train"))
        D = rng.choice((32, 48, 64, 64, 80, 96, 128, 128, 192, 256))
        R = rng.choice((0, D, D, D, D // 16 * 8))
        H = Hk * rng.choice((1, 1, 2, 4))
        most = MAX_QK // 2 // ((H + Hk) * D)
        N = 1 if kind == "decode" else min(_log_int(rng, 1, 16384) | (rng.random() < 0.7), most)
        B = _log_int(rng, 1, min(512 if kind == "decode" else 64, most // N))
        return _qk("train" if kind == "train" else "forward", B, N, H, Hk, D, dtype, R=R, norm=rng.choice(("rms", "rms", "l2")),
                   weight=rng.random() < 0.7, adjacent=rng.random() < 0.3, ragged=ragged and N > 1, strided=strided)
    kind = rng.choice(("step", "prefill", "train", "train"))
    D, M, H = rng.choice((32, 64, 64, 128, 128)), rng.choice((32, 48, 64, 64, 80, 128, 128, 256)), Hk * rng.choice((1, 1, 2, 4))
    if kind == "step":
        return _delta(kind, _log_int(rng, 1, MAX_STATE // 2 // (H * D * M)), 1, H, Hk, D, M, dtype, state=True)
    most = min((MAX_PROMPT if kind == "prefill" else MAX_DELTA) // 2 // (H * D * M), MAX_ROWS // 2 // (H * (D + M)))
    N = min(_log_int(rng, 1, 16384) | (rng.random() < 0.7), most)
    B = _log_int(rng, 1, min(64, most // N))
    return _delta(kind, B, N, H, Hk, D, M, dtype, ragged=ragged, state=rng.random() < 0.5, strided=strided)


# ---- inputs ---------------------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, N, H, Hk, D, dt = case["B"], case["N"], case["H"], case["Hk"], case["D"], _dtype(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    def uniform(lo, hi, *shape):
        return lo + (hi - lo) * torch.rand(shape, generator=g, device=DEV)

    def parts(*tensors):
        """The tensors [B, N, heads, width] in their type: parts of one projection's output rows, or each on its own."""
        if not case["strided"]:
            return [t.to(dt) for t in tensors]
        row, at, out = torch.cat([t.flatten(2) for t in tensors], -1).to(dt), 0, []
        for t in tensors:
            width = t.shape[2] * t.shape[3]
            out.append(row[..., at:at + width].unflatten(-1, t.shape[2:]))
            at += width
        return out

    x = {}
    if case["ragged"]:
        x["lengths"] = torch.randint(N // 4, N + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    if case["op"] == "qk":
        R = case["R"]
        # activations with a scale of their own in each head
        x["q"], x["k"] = parts(normal(B, N, H, D) * torch.exp(normal(H, 1)), normal(B, N, Hk, D) * torch.exp(normal(Hk, 1)))
        if case["weight"]:
            x["wq"], x["wk"] = 1 + 0.2 * normal(D), 1 + 0.2 * normal(D)
        if R:
            x["freq"] = 10000.0 ** (-torch.arange(0, R, 2, device=DEV, dtype=torch.float32) / R)
            if case["kind"] == "forward":        # tokens behind a cache of their own length; a training step counts from 0
                start = torch.randint(0, 1 << 17, (B, 1), generator=g, device=DEV, dtype=torch.int32)
                x["pos"] = start + torch.arange(N, device=DEV, dtype=torch.int32)
        if case["kind"] == "train":
            x["dyq"], x["dyk"] = normal(B, N, H, D).to(dt), normal(B, N, Hk, D).to(dt)
        return x
    M = case["M"]
    q, k = (t / torch.sqrt((t * t).sum(-1, keepdim=True) + EPS) for t in (normal(B, N, Hk, D), normal(B, N, Hk, D)))
    x["q"], x["k"], x["v"] = parts(q, k, normal(B, N, H, M))
    # decay rates of 1 to 16 times steps of 0.001 to 0.1; writes of all strengths
    x["g"] = -uniform(1.0, 16.0, H) * torch.exp(uniform(math.log(0.001), math.log(0.1), B, N, H))
    x["beta"] = torch.sigmoid(normal(B, N, H))
    if case["state"]:
        x["h0"] = 0.3 * normal(B, H, D, M)
    if case["kind"] == "train":
        x["do"] = normal(B, N, H, M).to(dt)
        if case["state"]:
            x["dh1"] = 0.3 * normal(B, H, D, M)
    if case["kind"] == "step":
        for n in ("q", "k", "v", "g", "beta"):
            x[n] = x[n][:, 0].contiguous()
    return x


def prepare(case, seed):
    """Inputs, the buffers that a user's loop keeps for the results, and the case."""
    x, o = _inputs(case, seed), {}

    def like(**named):
        for n, t in named.items():
            if t is not None:
                o[n] = torch.empty(t.shape, dtype=t.dtype, device=DEV)

    train = case["kind"] == "train"
    if case["op"] == "qk":
        like(yq=x["q"], yk=x["k"])
        if train:
            like(dq=x["q"], dk=x["k"], dwq=x.get("wq"), dwk=x.get("wk"))
    else:
        like(o=x["v"])
        if case["kind"] != "step" and case["state"]:
            like(h1=x["h0"])
        if train:
            like(dq=x["q"], dk=x["k"], dv=x["v"], dg=x["g"], dbeta=x["beta"], dh0=x.get("h0"))
    return {"case": case, "x": x, "out": o}


# ---- the calls -----------------------------------------------------------------------------------

def run(state):
    case, x, o = state["case"], state["x"], state["out"]
    if not own:
        if case["op"] == "qk":
            return _plain_qk(case, x)
        return _plain_delta_step(case, x) if case["kind"] == "step" else _plain_delta(case, x)
    import paper_2006_16236_amd as la
    train, lengths = case["kind"] == "train", x.get("lengths")
    if case["op"] == "qk":
        how = dict(wq=x.get("wq"), wk=x.get("wk"), freq=x.get("freq"), pos=x.get("pos"), lengths=lengths, norm=case["norm"],
                   adjacent=case["adjacent"], eps=EPS)
        la.la_qk_fwd(x["q"], o["yq"], k=x["k"], yk=o["yk"], **how)
        if train:
            la.la_qk_bwd(x["q"], x["dyq"], o["dq"], k=x["k"], dyk=x["dyk"], dk=o["dk"], dwq=o.get("dwq"), dwk=o.get("dwk"), **how)
        return o
    scale = case["D"] ** -0.5
    if case["kind"] == "step":
        la.la_delta_step(x["q"], x["k"], x["v"], x["g"], x["beta"], x["h0"], o["o"], scale=scale)
        return {"o": o["o"], "h1": x["h0"]}
    ws = la.la_delta_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], o["o"], h0=x.get("h0"), h1=o.get("h1"), lengths=lengths, scale=scale,
                         keep=train)
    if train:
        la.la_delta_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["do"], o["dq"], o["dk"], o["dv"], o["dg"], o["dbeta"], h0=x.get("h0"),
                        dh1=x.get("dh1"), dh0=o.get("dh0"), lengths=lengths, scale=scale, fwd_ws=ws)
    return o


# ---- plain forms, fp32 ---------------------------------------------------------------------------

def _real(case, x):
    """[B, N]: which tokens are part of their sequence."""
    at = torch.arange(case["N"], device=DEV)[None]
    return (at < (x["lengths"][:, None] if "lengths" in x else case["N"])).expand(case["B"], -1)


def _turn(n, cos, sin, R, adjacent):
    a, b = (n[..., :R:2], n[..., 1:R:2]) if adjacent else (n[..., :R // 2], n[..., R // 2:R])
    u, v = a * cos - b * sin, a * sin + b * cos
    return torch.cat((torch.stack((u, v), -1).flatten(-2) if adjacent else torch.cat((u, v), -1), n[..., R:]), -1)


def _plain_qk(case, x):
    """Angles in fp64 (a far position times a frequency has more digits than fp32), their cosines and sines rounded once."""
    dt, R, D, l2 = _dtype(case), case["R"], case["D"], case["norm"] == "l2"
    real, out = _real(case, x)[..., None, None], {}
    if R:
        pos = x["pos"] if "pos" in x else torch.arange(case["N"], device=DEV)[None].expand(case["B"], -1)
        angle = pos.double()[..., None, None] * x["freq"].double()
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    for name in ("q", "k"):
        t = x[name].float()
        squares = (t * t).sum(-1, keepdim=True)
        unit = t / torch.sqrt((squares if l2 else squares / D) + EPS)
        w = x.get("w" + name)
        n = unit if w is None else unit * w
        y = _turn(n, cos, sin, R, case["adjacent"]) if R else n
        out["y" + name] = torch.where(real, y, 0.0).to(dt)
        if case["kind"] == "train":
            dy = torch.where(real, x["dy" + name].float(), 0.0)
            dn = _turn(dy, cos, -sin, R, case["adjacent"]) if R else dy
            if w is not None:
                out["dw" + name] = (dn * unit).sum((0, 1, 2))
                dn = dn * w
            along = (dn * unit).sum(-1, keepdim=True)
            dx = (dn - unit * (along if l2 else along / D)) / torch.sqrt((squares if l2 else squares / D) + EPS)
            out["d" + name] = torch.where(real, dx, 0.0).to(dt)
    return out


def _inverse(a):
    """(1 + a)^-1 of strictly lower triangular a [.., C, C]: blocks of 1, 2, 4 .. are put together in pairs."""
    C = a.shape[-1]
    at = torch.arange(C, device=DEV)
    t = torch.eye(C, device=DEV).expand(a.shape)
    for w in (1, 2, 4, 8, 16, 32):
        block = at // w
        below = (block[:, None] == block[None] + 1) & (block[:, None] % 2 == 1)
        t = t - t @ (a * below) @ t
    return t


def _plain_delta(case, x):
    """Chunks of 64 tokens: what they write follows from a triangular system, and only the states go from chunk to chunk."""
    B, N, H, Hk, D, M = (case[n] for n in ("B", "N", "H", "Hk", "D", "M"))
    dt, scale, train, per = _dtype(case), D ** -0.5, case["kind"] == "train", H // Hk
    K = -(-N // CHUNK)
    real = _real(case, x)

    def chunks(t, heads):
        """[B, N, heads, ..] -> [B, H, K, 64, ..] in fp32, zeros at tokens that are none"""
        t = torch.where(real.reshape(B, N, *(1,) * (t.dim() - 2)), t.float(), 0.0)
        t = torch.cat((t, t.new_zeros(B, K * CHUNK - N, *t.shape[2:])), 1).unflatten(1, (K, CHUNK)).movedim(3, 1)
        return t.repeat_interleave(H // heads, 1)

    def tokens(t, heads):
        """back, the heads that share one added up"""
        t = t.unflatten(1, (heads, H // heads)).sum(2) if heads < H else t
        return t.movedim(1, 3).flatten(1, 2)[:, :N].contiguous()

    q, k, v, beta = chunks(x["q"], Hk), chunks(x["k"], Hk), chunks(x["v"], H), chunks(x["beta"], H)[..., None]
    # sums of many small logarithms, and differences of such sums, in fp64
    sums = chunks(x["g"], H).double().cumsum(-1)
    low = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=DEV).tril()
    decay = torch.where(low, sums[..., :, None] - sums[..., None, :], -math.inf).exp().float()
    since, until, whole = sums.exp().float()[..., None], (sums[..., -1:] - sums).exp().float()[..., None], sums[..., -1].exp().float()[..., None, None]
    kk = (k @ k.transpose(-1, -2)) * decay * low.tril(-1)
    qk = (q @ k.transpose(-1, -2)) * decay
    T = _inverse(beta * kk)
    S = x["h0"] if case["state"] else torch.zeros(B, H, D, M, device=DEV)
    ends, inner, o, rest = [], [], [], []
    for c in range(K):
        ends.append(S)
        r = v[:, :, c] - since[:, :, c] * (k[:, :, c] @ S)                  # what the state does not hold yet
        u = T[:, :, c] @ (beta[:, :, c] * r)
        o.append(scale * (since[:, :, c] * (q[:, :, c] @ S) + qk[:, :, c] @ u))
        S = whole[:, :, c] * S + k[:, :, c].transpose(-1, -2) @ (until[:, :, c] * u)
        if train:
            inner.append(u)
            rest.append(r)
        else:
            ends.pop()
    out = {"o": torch.where(real[..., None, None], tokens(torch.stack(o, 2), H), 0.0).to(dt)}
    if case["state"]:
        out["h1"] = S
    if not train:
        return out
    u, s0 = torch.stack(inner, 2), torch.stack(ends, 2)
    ut = torch.stack(rest, 2) - kk @ u                                      # u without beta
    do = scale * chunks(x["do"], H)
    dS = x["dh1"] if case["state"] else torch.zeros(B, H, D, M, device=DEV)
    write, later = [None] * K, [None] * K
    mixed = qk.transpose(-1, -2) @ do
    for c in range(K - 1, -1, -1):
        later[c] = dS
        write[c] = T[:, :, c].transpose(-1, -2) @ (mixed[:, :, c] + until[:, :, c] * (k[:, :, c] @ dS))
        dS = whole[:, :, c] * dS + q[:, :, c].transpose(-1, -2) @ (since[:, :, c] * do[:, :, c]) \
            - k[:, :, c].transpose(-1, -2) @ (since[:, :, c] * beta[:, :, c] * write[c])
    dy, s1 = torch.stack(write, 2), torch.stack(later, 2)
    dv = beta * dy
    P = (do @ u.transpose(-1, -2)) * decay
    Bk = -(dv @ u.transpose(-1, -2)) * decay * low.tril(-1)
    dq = since * (do @ s0.transpose(-1, -2)) + P @ k
    into = until * (u @ s1.transpose(-1, -2))
    dk = into - since * (dv @ s0.transpose(-1, -2)) + P.transpose(-1, -2) @ q + (Bk + Bk.transpose(-1, -2)) @ k
    # a token's decay acts on all later ones of its chunk and on the state behind it
    dsum = (q * dq - k * dk).double().sum(-1) - 2 * (dv * (v - ut)).double().sum(-1)
    dsum[..., -1] += (k * into).double().sum((-1, -2)) + (whole * s0 * s1).double().sum((-1, -2))
    dg = dsum.flip(-1).cumsum(-1).flip(-1).float()
    out.update(dq=tokens(dq, Hk).to(dt), dk=tokens(dk, Hk).to(dt), dv=tokens(dv, H).to(dt))
    out.update((n, torch.where(real[..., None], tokens(t, H), 0.0)) for n, t in (("dg", dg), ("dbeta", (dy * ut).sum(-1))))
    if case["state"]:
        out["dh0"] = dS
    return out


def _plain_delta_step(case, x):
    H, Hk, D = case["H"], case["Hk"], case["D"]
    q, k = (x[n].float().repeat_interleave(H // Hk, 1)[..., None] for n in ("q", "k"))
    S = x["h0"] * torch.exp(x["g"])[..., None, None]
    new = x["beta"][..., None] * (x["v"].float() - (S * k).sum(-2))
    S = S + k * new[..., None, :]
    x["h0"].copy_(S)
    return {"o": (D ** -0.5 * (S * q).sum(-2)).to(_dtype(case)), "h1": x["h0"]}


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    """Each input read once and each output written once; the arithmetic of the formulas above, an exp, a root or a
    division counted as one."""
    kind, B, N, H, Hk, D = (case[n] for n in ("kind", "B", "N", "H", "Hk", "D"))
    e = 2 if case["dtype"] == "bf16" else 4
    train = kind == "train"
    if case["op"] == "qk":
        P, R = B * N * (H + Hk) * D, case["R"]
        nbytes, flops = 2 * P * e + 2 * R, 5 * P + 3 * P * R // D
        nbytes += 4 * B * N * (R > 0 and not train) + 8 * D * case["weight"]
        if train:                                            # x, dy -> dx
            nbytes += 3 * P * e + 16 * D * case["weight"]
            flops += 10 * P + 3 * P * R // D
        return {"bytes": nbytes, "flops": flops}
    M, T = case["M"], B * N
    nbytes = T * (2 * Hk * D + 2 * H * M) * e + T * H * 8    # q, k, v, g, beta -> o
    flops = 7 * T * H * D * M                                # decay, S^T k, the update, S^T q
    if case["state"]:
        nbytes += 8 * B * H * D * M
    if train:                                                # q, k, v, do, g, beta -> dq, dk, dv, dg, dbeta
        nbytes += T * (4 * Hk * D + 3 * H * M) * e + T * H * 16
        flops += 17 * T * H * D * M
        if case["state"]:
            nbytes += 12 * B * H * D * M
    return {"bytes": nbytes, "flops": flops}


# ---- the same in fp64, from the definition -------------------------------------------------------

def _exact_qk(case, x):
    """Pairs as complex numbers."""
    D, R, ends = case["D"], case["R"], x["lengths"].tolist() if "lengths" in x else [case["N"]] * case["B"]
    out = {}
    if R:
        pos = x["pos"].double() if "pos" in x else torch.arange(case["N"], device=DEV).double().expand(case["B"], -1)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos[..., None] * x["freq"].double())[:, :, None]
    first, second = (slice(0, R, 2), slice(1, R, 2)) if case["adjacent"] else (slice(0, R // 2), slice(R // 2, R))

    def turned(t, by):
        t = t.clone()
        z = torch.complex(t[..., first], t[..., second]) * by
        t[..., first], t[..., second] = z.real, z.imag
        return t

    for name in ("q", "k"):
        t, w = x[name].double(), x["w" + name].double() if case["weight"] else torch.ones(D, dtype=torch.float64, device=DEV)
        r = (t.square().sum(-1, keepdim=True) / (1 if case["norm"] == "l2" else D) + EPS).rsqrt()
        y = t * r * w
        y = turned(y, turn) if R else y
        for b, n in enumerate(ends):
            y[b, n:] = 0.0
        out["y" + name] = y
        if case["kind"] == "train":
            dy = x["dy" + name].double().clone()
            for b, n in enumerate(ends):
                dy[b, n:] = 0.0
            dn = turned(dy, turn.conj()) if R else dy
            dx = dn * w * r - t * r ** 3 * (dn * w * t).sum(-1, keepdim=True) / (1 if case["norm"] == "l2" else D)
            for b, n in enumerate(ends):
                dx[b, n:] = 0.0
            out["d" + name] = dx
            if case["weight"]:
                out["dw" + name] = (dn * t * r).flatten(0, 2).sum(0)
    return out


def _exact_delta(case, x):
    """The recurrence and its adjoint, one token after the other; states kept at every 64th token and formed again from there."""
    B, N, H, Hk, D, M = (case[n] for n in ("B", "N", "H", "Hk", "D", "M"))
    step, train, per, scale = case["kind"] == "step", case["kind"] == "train", H // Hk, case["D"] ** -0.5
    if not step and N * (8 if train else 2) * (1 + B * H * D * M / 3e6) > 1e6:
        return None                                          # longer than about 20 seconds
    t = {n: x[n].double()[:, None] if step else x[n].double() for n in ("q", "k", "v", "g", "beta")}
    lengths = x["lengths"] if "lengths" in x else torch.full((B,), N, device=DEV)
    real = (torch.arange(N, device=DEV)[:, None] < lengths[None])[..., None]                   # [N, B, 1]
    # [N, B, H, ..], tokens that are none without decay and write
    q, k = (torch.where(real[..., None], t[n].transpose(0, 1), 0.0).repeat_interleave(per, 2) for n in ("q", "k"))
    v = torch.where(real[..., None], t["v"].transpose(0, 1), 0.0)
    a, beta = torch.where(real, t["g"].transpose(0, 1), 0.0).exp()[..., None, None], torch.where(real, t["beta"].transpose(0, 1), 0.0)[..., None]
    S = x["h0"].double().clone() if "h0" in x else torch.zeros(B, H, D, M, dtype=torch.float64, device=DEV)

    def forward(S, i):
        """S behind token i, and what the token finds missing"""
        S = S * a[i]
        miss = v[i] - torch.matmul(k[i][:, :, None], S)[:, :, 0]
        return S.addcmul_(k[i][..., None], (beta[i] * miss)[:, :, None]), miss

    kept, o = [], torch.empty(N, B, H, M, dtype=torch.float64, device=DEV)
    for i in range(N):
        if train and i % 64 == 0:
            kept.append(S.clone())
        S, _ = forward(S, i)
        o[i] = scale * torch.matmul(q[i][:, :, None], S)[:, :, 0]
    o = torch.where(real[..., None], o, 0.0).transpose(0, 1)
    out = {"o": o[:, 0] if step else o}
    if "h0" in x:
        out["h1"] = S
    if not train:
        return out
    do = scale * torch.where(real[..., None], x["do"].double().transpose(0, 1), 0.0)
    G = x["dh1"].double().clone() if "dh1" in x else torch.zeros_like(S)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dg, dbeta = torch.zeros(N, B, H, dtype=torch.float64, device=DEV), torch.zeros(N, B, H, dtype=torch.float64, device=DEV)
    for c in range(len(kept) - 1, -1, -1):
        states, first = [kept.pop()], 64 * c
        misses = []
        for i in range(first, min(first + 64, N)):
            S, miss = forward(states[-1], i)
            states.append(S)
            misses.append(miss)
        for i in range(min(first + 64, N) - 1, first - 1, -1):
            before, S, miss = states[i - first] * a[i], states[i - first + 1], misses[i - first]
            dq[i] = torch.matmul(S, do[i][..., None])[..., 0]
            G.addcmul_(q[i][..., None], do[i][:, :, None])                # gradient for S_i
            along = torch.matmul(k[i][:, :, None], G)[:, :, 0]            # for beta miss
            dbeta[i] = (along * miss).sum(-1)
            dv[i] = beta[i] * along                                       # for miss
            dk[i] = torch.matmul(G, (beta[i] * miss)[..., None])[..., 0] - torch.matmul(before, dv[i][..., None])[..., 0]
            G.addcmul_(k[i][..., None], dv[i][:, :, None], value=-1.0)    # for the decayed state
            dg[i] = torch.where(real[i], (G * before).sum((-1, -2)), 0.0)
            G *= a[i]
    out.update((n, d.unflatten(2, (Hk, per)).sum(3).transpose(0, 1)) for n, d in (("dq", dq), ("dk", dk)))
    out.update(dv=dv.transpose(0, 1), dg=dg.transpose(0, 1), dbeta=torch.where(real, dbeta, 0.0).transpose(0, 1))
    if "dh1" in x:
        out["dh0"] = G
    return out


def exact(case, seed):
    x = _inputs(case, seed)
    return _exact_qk(case, x) if case["op"] == "qk" else _exact_delta(case, x)
