"""Layer norm, short causal convolution and selective scan on the GPU against fp64, at sizes and masks where they
can go wrong; their states, gradients, streams and graphs."""
import numpy as np
import pytest
import torch

import layer_ref as ref
import paper_2006_16236_amd as la
from gpu_util import DEV

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return t.detach().to(torch.float32).cpu().numpy().astype(np.float64)


class Data:
    """Random arrays, exact in the type, on the host (fp32) and on the device; rows may be parts of wider ones."""

    def __init__(self, seed, dtype):
        self.rng, self.dtype = np.random.default_rng(seed), dtype

    def array(self, *shape, scale=1.0, f32=False):
        a = (self.rng.standard_normal(shape) * scale).astype(np.float32)
        return a if f32 or self.dtype == "f32" else ref.to_bf16(a)

    def dev(self, a, f32=False, wider=0):
        if a is None:
            return None
        t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
        t = t if f32 else t.to(TYPES[self.dtype])
        if wider:                                  # a part of rows `wider` elements longer, the rest NaN
            lead, width = t.shape[:2], t[0, 0].numel()
            big = torch.full((*lead, width + wider), float("nan"), dtype=t.dtype, device=DEV)
            big[..., 8:8 + width] = t.reshape(*lead, width)   # 8 elements: 16 or 32 bytes
            t = big[..., 8:8 + width].unflatten(-1, t.shape[2:])
        return t

    def empty(self, shape, f32=False):
        return torch.full(shape, float("nan"), dtype=torch.float32 if f32 else TYPES[self.dtype], device=DEV)


# ---- layer norm ------------------------------------------------------------------------------------------

NORMS = [(1, 1), (3, 1), (5, 7), (2, 64), (65, 63), (9, 255), (17, 257), (33, 512), (7, 771), (4, 1023), (3, 1024), (6, 1025),
         (5, 2048), (3, 4095), (4, 4097), (2, 8192), (2, 16383), (2, 16384), (700, 96), (4200, 33), (1030, 1100)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,E", NORMS)
@pytest.mark.parametrize("residual,affine", [(True, True), (False, True), (True, False)])
def test_norm(rows, E, dtype, residual, affine):
    d = Data(rows * 20011 + E, dtype)
    eps = 1e-5
    x = d.array(rows, E, scale=1.5) + (d.array(E) if dtype == "f32" else 0)
    r = d.array(rows, E) if residual else None
    gamma, beta = (1 + d.array(E, scale=0.2, f32=True), d.array(E, f32=True)) if affine else (None, None)
    dy, ds = d.array(rows, E), d.array(rows, E) if residual else None
    s = x.astype(np.float32) + r if residual else x                # fp32 sums of the type's values, rounded to it below
    if dtype == "bf16":
        s = ref.to_bf16(s)
    tx, tr, tdy, tds = (d.dev(a) for a in (x, r, dy, ds))
    tg, tb = d.dev(gamma, f32=True), d.dev(beta, f32=True)
    y, mean, rstd = d.empty((rows, E)), d.empty((rows,), True), d.empty((rows,), True)
    ts = d.empty((rows, E)) if residual else None
    la.la_norm_fwd(tx, tg, tb, y, mean, rstd, r=tr, s=ts, eps=eps)
    if residual:
        assert np.array_equal(host(ts), s)                         # one rounding of the sum, bit for bit
    dx = d.empty((rows, E))
    dg, db = (d.empty((E,), True), d.empty((E,), True)) if affine else (None, None)
    la.la_norm_bwd(ts if residual else tx, tg, mean, rstd, tdy, dx, dg, db, ds=tds)
    want = ref.norm(s, gamma, beta, eps, dy, ds)
    mag = ref.norm(s, gamma, beta, eps, dy, ds, mag=True)
    # a lane adds 16 elements, then 6 + 4 steps over lanes and waves, twice (mean, squares); a few more operations each
    k = 64
    ref.check("y", host(y), want["y"], mag["y"], dtype, k)
    ref.check("mean", host(mean), want["mean"], mag["mean"], "f32", k)
    ref.check("rstd", host(rstd), want["rstd"], mag["rstd"], "f32", k)
    ref.check("dx", host(dx), want["dx"], mag["dx"], dtype, 3 * k)
    if affine:
        # additionally the rows: those of a workgroup one after the other, 16 slots, then 256 workgroups in 16 slices
        k += rows // 256 + 48
        ref.check("dgamma", host(dg), want["dgamma"], mag["dgamma"], "f32", k)
        ref.check("dbeta", host(db), want["dbeta"], mag["dbeta"], "f32", k)


def test_norm_takes_leading_dimensions_and_leaves_out_what_is_not_asked_for():
    d = Data(5, "f32")
    x = d.array(3, 4, 5, 40)
    tx = d.dev(x)
    y = torch.empty_like(tx)
    la.la_norm_fwd(tx, None, None, y, eps=0.0)
    want = ref.norm(x.reshape(-1, 40), None, None, 0.0)["y"].reshape(x.shape)
    assert np.abs(host(y) - want).max() <= 1e-5
    mean, rstd = torch.empty(3, 4, 5, device=DEV), torch.empty(3, 4, 5, device=DEV)
    la.la_norm_fwd(tx, None, None, y, mean, rstd, eps=0.0)
    dx, db = torch.empty_like(tx), torch.empty(40, device=DEV)
    assert la.la_norm_bwd(tx, None, mean, rstd, tx, dx) is None    # no sums: no workspace
    la.la_norm_bwd(tx, None, mean, rstd, tx, dx, dbeta=db)         # one of the two
    assert np.abs(host(db) - x.reshape(-1, 40).sum(0)).max() <= 1e-4


def test_norm_of_rows_far_from_zero():
    """A mean a thousand times the spread: the squares are taken around the mean."""
    d = Data(6, "f32")
    x = (1000.0 + d.array(8, 640)).astype(np.float32)
    y, mean, rstd = (torch.empty(s, device=DEV) for s in ((8, 640), (8,), (8,)))
    la.la_norm_fwd(d.dev(x), None, None, y, mean, rstd, eps=1e-5)
    want = ref.norm(x, None, None, 1e-5)
    # the mean is off by at most (16 + 10 + 1) 2^-24 1000, which shifts all of a row's xhat alike
    assert np.abs(host(y) - want["y"]).max() <= 27 * 2.0 ** -24 * 1000 + 64 * 2.0 ** -24 * 5
    assert np.abs(host(rstd) / want["rstd"] - 1).max() <= 64 * 2.0 ** -24


# ---- convolution -------------------------------------------------------------------------------------------

CONVS = [  # B, N, E, W, wider, lengths, state, silu
    (1, 1, 1, 4, 0, None, False, True), (1, 1, 8, 2, 0, None, True, True), (2, 2, 9, 4, 0, None, True, True),
    (3, 3, 17, 3, 0, None, False, False), (2, 4, 64, 4, 0, [4, 2], True, True), (4, 7, 33, 4, 0, [0, 7, 1, 3], True, True),
    (3, 31, 65, 2, 0, [31, 0, 16], False, True), (2, 33, 100, 3, 16, None, True, True), (3, 64, 130, 4, 0, [64, 33, 2], True, False),
    (1, 257, 40, 4, 24, None, True, True), (2, 100, 1001, 3, 0, [100, 57], True, True), (5, 40, 512, 4, 512, [-3, 99, 40, 5, 32], True, True),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,E,W,wider,lengths,state,silu", CONVS)
def test_conv(B, N, E, W, wider, lengths, state, silu, dtype):
    d = Data(B * 7919 + N * 31 + E, dtype)
    x, w, bias = d.array(B, N, E), d.array(E, W, f32=True), d.array(E, f32=True)
    x0, dx1 = (d.array(B, W - 1, E), d.array(B, W - 1, E)) if state else (None, None)
    dy = d.array(B, N, E)
    tl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    xd, dyd = x.copy(), dy.copy()
    if lengths is not None:                                        # what lies behind a sequence does not matter
        for b, n in enumerate(lengths):
            xd[b, max(n, 0):], dyd[b, max(n, 0):] = np.nan, np.nan
    tx, tw, tb = d.dev(xd, wider=wider), d.dev(w, f32=True), d.dev(bias, f32=True)
    y = d.empty((B, N, E))
    x1 = d.empty((B, W - 1, E)) if state else None
    la.la_conv_fwd(tx, tw, tb, y, x0=d.dev(x0), x1=x1, lengths=tl, silu=silu)
    dx, dw, db = d.empty((B, N, E)), d.empty((E, W), True), d.empty((E,), True)
    dx0 = d.empty((B, W - 1, E)) if state else None
    la.la_conv_bwd(tx, tw, tb, d.dev(dyd), dx, dw, db, x0=d.dev(x0), dx1=d.dev(dx1), dx0=dx0, lengths=tl, silu=silu)
    want = ref.conv(x, w, bias, x0, lengths, silu, dy, dx1)
    mag = ref.conv(x, w, bias, x0, lengths, silu, dy, dx1, mag=True)
    k = 2 * W + 16                                                 # taps, bias, the sigmoid's exp, division and products
    ref.check("y", host(y), want["y"], mag["y"], dtype, k)
    ref.check("dx", host(dx), want["dx"], mag["dx"], dtype, 2 * k)
    k += 64 + B * N // 32                                          # a run of up to 32 tokens, then the runs
    ref.check("dw", host(dw), want["dw"], mag["dw"], "f32", k)
    ref.check("db", host(db), want["db"], mag["db"], "f32", k)
    if state:
        assert np.array_equal(host(x1), want["x1"])                # copies
        ref.check("dx0", host(dx0), want["dx0"], mag["dx0"], dtype, 2 * k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,E,W,silu", [(1, 1, 2, True), (3, 9, 3, True), (65, 100, 4, True), (2, 4096, 4, False)])
def test_conv_steps_are_the_convolution(B, E, W, silu, dtype):
    d = Data(E, dtype)
    N = 6
    x, w, bias = d.array(B, N, E), d.dev(d.array(E, W, f32=True), True), d.dev(d.array(E, f32=True), True)
    tx = d.dev(x)
    y, x1 = d.empty((B, N, E)), d.empty((B, W - 1, E))
    la.la_conv_fwd(tx, w, bias, y, x1=x1, silu=silu)
    state = torch.zeros(B, W - 1, E, dtype=tx.dtype, device=DEV)
    for t in range(N):
        out = d.empty((B, E))
        la.la_conv_step(tx[:, t].clone(memory_format=torch.contiguous_format), w, bias, state, out, silu=silu)
        assert torch.equal(out, y[:, t])                           # the same operations in the same order
    assert torch.equal(state, x1)


# ---- scan --------------------------------------------------------------------------------------------------

SCANS = [  # B, N, E, G, S, wider, lengths, state, gated, skip, softplus
    (1, 1, 1, 1, 8, 0, None, False, False, False, True),
    (1, 1, 3, 1, 16, 0, None, True, True, True, True),
    (2, 2, 64, 1, 16, 0, None, True, True, True, False),
    (1, 15, 65, 1, 32, 0, None, True, True, True, True),
    (2, 16, 63, 1, 16, 0, [16, 3], True, False, True, True),
    (3, 17, 130, 2, 8, 0, [0, 17, 16], True, True, False, True),
    (1, 33, 96, 4, 16, 32, None, False, True, True, True),
    (5, 40, 70, 1, 16, 8, [-1, 40, 99, 32, 33], True, True, True, True),
    (1, 200, 64, 1, 32, 0, None, True, True, True, True),          # one sequence: cut into pieces
    (2, 300, 72, 2, 16, 16, [300, 77], True, True, True, True),    # a sequence that ends inside the second piece
    (3, 129, 40, 1, 8, 0, [129, 0, 64], False, False, True, True),
    (40, 35, 250, 1, 16, 0, None, True, True, True, True),         # enough workgroups: not cut
]


def scan_data(B, N, E, G, S, lengths, state, gated, skip, softplus, dtype):
    d = Data(B * 7919 + N * 31 + E + S, dtype)
    a = {"x": d.array(B, N, E), "Bt": d.array(B, N, G, S), "Ct": d.array(B, N, G, S), "dy": d.array(B, N, E)}
    a["A"] = (-np.arange(1, S + 1) * np.exp(0.2 * d.array(E, S, f32=True))).astype(np.float32)
    if softplus:
        a["dt"], a["dt_bias"] = d.array(B, N, E, scale=0.5), (d.array(E, f32=True) - 3).astype(np.float32)
    else:
        a["dt"], a["dt_bias"] = np.abs(d.array(B, N, E, scale=0.1)), None
    a["z"] = d.array(B, N, E) if gated else None
    a["D"] = d.array(E, f32=True) if skip else None
    a["h0"], a["dh1"] = (d.array(B, E, S, f32=True), d.array(B, E, S, f32=True)) if state else (None, None)
    a["lengths"] = lengths
    return d, a


F32_NAMES = {"A", "D", "dt_bias", "h0", "dh1"}


def scan_on_device(d, a, wider, softplus, keep=True, stream=None, pad=True):
    """Forward and backward; the rows behind a sequence hold NaN."""
    B, N, E = a["x"].shape
    G, S = a["Bt"].shape[2:]
    tl = None if a["lengths"] is None else torch.tensor(a["lengths"], dtype=torch.int32, device=DEV)
    t = {}
    for n, v in a.items():
        if n == "lengths" or v is None:
            continue
        v = v.copy()
        if pad and a["lengths"] is not None and n in ("x", "dt", "z", "Bt", "Ct", "dy"):
            for b, end in enumerate(a["lengths"]):
                v[b, max(end, 0):] = np.nan
        t[n] = d.dev(v, f32=n in F32_NAMES, wider=wider if n in ("x", "dt", "z", "Bt", "Ct") else 0)
    o = {n: d.empty((B, N, E)) for n in ("y", "dx", "ddt")}
    o.update(dB=d.empty((B, N, G, S)), dC=d.empty((B, N, G, S)), dA=d.empty((E, S), True), dD=d.empty((E,), True),
             ddt_bias=d.empty((E,), True), h1=d.empty((B, E, S), True), dh0=d.empty((B, E, S), True))
    if "z" in t:
        o["dz"] = d.empty((B, N, E))
    args = (t["x"], t["dt"], t["A"], t["Bt"], t["Ct"])
    common = dict(D=t.get("D"), z=t.get("z"), dt_bias=t.get("dt_bias"), h0=t.get("h0"), lengths=tl, softplus=softplus)

    def call():
        ws = la.la_scan_fwd(*args, o["y"], h1=o["h1"], keep=keep, **common)
        la.la_scan_bwd(*args, t["dy"], o["dx"], o["ddt"], o["dA"], o["dB"], o["dC"], dD=o["dD"], dz=o.get("dz"),
                       ddt_bias=o["ddt_bias"], dh1=t.get("dh1"), dh0=o["dh0"], fwd_ws=ws if keep else None, **common)

    call()
    return o, call


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,E,G,S,wider,lengths,state,gated,skip,softplus", SCANS)
def test_scan(B, N, E, G, S, wider, lengths, state, gated, skip, softplus, dtype):
    d, a = scan_data(B, N, E, G, S, lengths, state, gated, skip, softplus, dtype)
    o, _ = scan_on_device(d, a, wider, softplus)
    want = ref.scan(**a, softplus=softplus)
    mag = ref.scan(**a, softplus=softplus, mag=True)
    raw = a["dt"] + (0 if a["dt_bias"] is None else a["dt_bias"])
    k = ref.roundings(N, S, a["A"], float(np.logaddexp(raw, 0).max() if softplus else raw.max()))
    for n in ("y", "dx", "ddt", "dz", "dB", "dC"):
        if n in o:
            extra = E if n in ("dB", "dC") else 0                  # sums over the channels
            ref.check(n, host(o[n]), want[n], mag[n], dtype, 2 * k + extra)
    for n in ("h1", "dA", "dD", "ddt_bias", "dh0"):
        ref.check(n, host(o[n]), want[n], mag[n], "f32", 2 * k + B * N)


# more workgroups than compute units, where a workgroup has fewer waves of more states: whole sequences, and pieces of them
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", [8, 16, 32])
@pytest.mark.parametrize("B,N,E,G,lengths", [(70, 35, 250, 1, None), (66, 18, 130, 2, [i % 19 for i in range(66)])])
def test_scan_of_many_sequences(B, N, E, G, lengths, S, dtype):
    test_scan(B, N, E, G, S, 0, lengths, True, True, True, True, dtype)


@pytest.mark.parametrize("S", [16, 32])
def test_scan_of_many_pieces(S):
    B, N, E = 17, 500, 250
    states, tiles = B * E * S * 4, (N + 15) // 16
    pieces = (la.la_scan_fwd_workspace(B, N, E, 1, S, 0, 1) - 512) // (states + B * E * 4)
    assert 4 * B * (pieces + 1) > 256 and pieces < tiles / 4       # four channel blocks a sequence
    test_scan(B, N, E, 1, S, 0, [500, 0, 1, 499, 64, 65] + [450 + i for i in range(11)], True, True, True, True, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", [SCANS[3], SCANS[9], SCANS[11]])
def test_scan_backward_with_and_without_the_forwards_states(case, dtype):
    B, N, E, G, S, wider, lengths, state, gated, skip, softplus = case
    d, a = scan_data(B, N, E, G, S, lengths, state, gated, skip, softplus, dtype)
    kept, call = scan_on_device(d, a, wider, softplus)
    first = {n: t.clone() for n, t in kept.items()}
    call()                                                         # and again: the same bits
    rebuilt, _ = scan_on_device(d, a, wider, softplus, keep=False)
    for n in kept:
        assert torch.equal(kept[n], first[n]) and torch.equal(kept[n], rebuilt[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,E,G,S,gated", [(1, 1, 1, 8, True), (3, 66, 2, 16, True), (65, 40, 1, 32, False), (2, 1000, 4, 16, True)])
def test_scan_steps(B, E, G, S, gated, dtype):
    N = 5
    d, a = scan_data(B, N, E, G, S, None, True, gated, True, True, dtype)
    t = {n: d.dev(v, f32=n in F32_NAMES) for n, v in a.items() if v is not None}
    h = t["h0"].clone()
    want, mag = ref.scan(**{**a, "dy": None}), ref.scan(**{**a, "dy": None}, mag=True)
    k = ref.roundings(N, S, a["A"], float(np.logaddexp(a["dt"] + a["dt_bias"], 0).max()))
    for i in range(N):
        at = {n: t[n][:, i].clone(memory_format=torch.contiguous_format) for n in ("x", "dt", "z", "Bt", "Ct") if n in t}
        y = d.empty((B, E))
        la.la_scan_step(at["x"], at["dt"], t["A"], at["Bt"], at["Ct"], h, y, D=t["D"], z=at.get("z"), dt_bias=t["dt_bias"])
        ref.check("y", host(y), want["y"][:, i], mag["y"][:, i], dtype, k)
    ref.check("h", host(h), want["h1"], mag["h1"], "f32", k)


def test_scan_gradients_against_differences():
    """The GPU's gradients against central differences of the fp64 forward, one direction per input."""
    B, N, E, G, S = 2, 37, 20, 2, 8
    d, a = scan_data(B, N, E, G, S, [37, 21], True, True, True, True, "f32")
    o, _ = scan_on_device(d, a, 0, True)
    rng = np.random.default_rng(3)

    def loss(v):
        out = ref.scan(**{**v, "dy": None, "dh1": None})
        return (out["y"] * a["dy"]).sum() + (out["h1"] * a["dh1"]).sum()

    for name, grad in (("x", "dx"), ("dt", "ddt"), ("z", "dz"), ("Bt", "dB"), ("Ct", "dC"), ("A", "dA"), ("D", "dD"),
                       ("dt_bias", "ddt_bias"), ("h0", "dh0")):
        way, step = rng.standard_normal(a[name].shape), 1e-4
        up, down = (loss({**a, name: a[name].astype(np.float64) + s * step * way}) for s in (1, -1))
        got, num = float((host(o[grad]) * way).sum()), (up - down) / (2 * step)
        # third-order remainder step^2 / 6 f''' and the fp32 gradient's error on the sum of magnitudes
        size = float((np.abs(host(o[grad])) * np.abs(way)).sum())
        assert abs(got - num) <= 2e-5 * size, (name, got, num, size)


def test_a_prompt_in_two_calls_is_the_prompt_in_one():
    """States and their gradients handed from call to call, convolution and scan, fp32."""
    B, N, E, S, W, cut = 2, 60, 48, 16, 4, 23
    d, a = scan_data(B, N, E, 1, S, None, True, True, True, True, "f32")
    o, _ = scan_on_device(d, a, 0, True)
    t = {n: d.dev(v, f32=True) for n, v in a.items() if v is not None}
    part = [{n: (v[:, s].contiguous() if n in ("x", "dt", "z", "Bt", "Ct", "dy") else v) for n, v in t.items()}
            for s in (slice(0, cut), slice(cut, N))]
    h, states, outs, kept = t["h0"], [], [], []
    for p in part:
        y, h1 = torch.empty_like(p["x"]), torch.empty_like(h)
        kept.append(la.la_scan_fwd(p["x"], p["dt"], p["A"], p["Bt"], p["Ct"], y, D=p["D"], z=p["z"], dt_bias=p["dt_bias"], h0=h, h1=h1, keep=True))
        states.append(h)
        outs.append(y)
        h = h1
    assert (torch.cat(outs, 1) - o["y"]).abs().max() <= 1e-5 * o["y"].abs().max()
    assert (h - o["h1"]).abs().max() <= 1e-5 * o["h1"].abs().max()
    g, dA = t["dh1"], 0
    for i in (1, 0):
        p = part[i]
        dx, ddt, dz, dB, dC = (torch.empty_like(p[n]) for n in ("x", "dt", "z", "Bt", "Ct"))
        pA, g0 = torch.empty_like(p["A"]), torch.empty_like(g)
        la.la_scan_bwd(p["x"], p["dt"], p["A"], p["Bt"], p["Ct"], p["dy"], dx, ddt, pA, dB, dC, D=p["D"], z=p["z"], dz=dz,
                       dt_bias=p["dt_bias"], h0=states[i], dh1=g, dh0=g0, fwd_ws=kept[i])
        g, dA = g0, dA + pA
        where = slice(0, cut) if i == 0 else slice(cut, N)
        for got, name in ((dx, "dx"), (ddt, "ddt"), (dz, "dz"), (dB, "dB"), (dC, "dC")):
            assert (got - o[name][:, where]).abs().max() <= 1e-5 * o[name].abs().max(), name
    assert (dA - o["dA"]).abs().max() <= 1e-5 * o["dA"].abs().max()
    assert (g - o["dh0"]).abs().max() <= 1e-5 * o["dh0"].abs().max()

    x, w = d.dev(d.array(B, N, E)), d.dev(d.array(E, W, f32=True), True)
    dy = d.dev(d.array(B, N, E))
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    la.la_conv_fwd(x, w, None, y)
    la.la_conv_bwd(x, w, None, dy, dx, dw)
    xa, xb = x[:, :cut].contiguous(), x[:, cut:].contiguous()
    ya, yb, mid = torch.empty_like(xa), torch.empty_like(xb), torch.empty(B, W - 1, E, device=DEV)
    la.la_conv_fwd(xa, w, None, ya, x1=mid)
    la.la_conv_fwd(xb, w, None, yb, x0=mid)
    assert torch.equal(torch.cat((ya, yb), 1), y)
    da, db_, dmid = torch.empty_like(xa), torch.empty_like(xb), torch.empty_like(mid)
    dwa, dwb = torch.empty_like(w), torch.empty_like(w)
    la.la_conv_bwd(xb, w, None, dy[:, cut:].contiguous(), db_, dwb, x0=mid, dx0=dmid)
    la.la_conv_bwd(xa, w, None, dy[:, :cut].contiguous(), da, dwa, dx1=dmid)
    assert (torch.cat((da, db_), 1) - dx).abs().max() <= 1e-6 * dx.abs().max()
    assert (dwa + dwb - dw).abs().max() <= 1e-5 * dw.abs().max()


# ---- streams, graphs ---------------------------------------------------------------------------------------

def test_calls_run_on_the_current_and_on_a_given_stream():
    d, a = scan_data(2, 150, 64, 1, 16, None, True, True, True, True, "bf16")
    want, _ = scan_on_device(d, a, 0, True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got, _ = scan_on_device(d, a, 0, True)
    side.synchronize()
    for n in want:
        assert torch.equal(got[n], want[n]), n
    x = d.dev(d.array(64, 96))
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    la.la_norm_fwd(x, None, None, y)
    torch.cuda.synchronize()
    la.la_norm_fwd(x, None, None, y2, stream=side)
    side.synchronize()
    assert torch.equal(y, y2)


def test_a_workspace_belongs_to_the_stream_that_uses_it():
    """Allocated by the call for a given stream: once it is dropped, the current stream must not be handed its memory."""
    d, a = scan_data(2, 150, 64, 1, 16, None, False, True, False, False, "f32")
    t = {n: d.dev(v, f32=n in F32_NAMES) for n, v in a.items() if v is not None}
    side, y, y2 = torch.cuda.Stream(), torch.empty_like(t["x"]), torch.empty_like(t["x"])
    la.la_scan_fwd(t["x"], t["dt"], t["A"], t["Bt"], t["Ct"], y2)
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        ws = la.la_scan_fwd(t["x"], t["dt"], t["A"], t["Bt"], t["Ct"], y, keep=True, stream=stream)
        at, size = ws.data_ptr(), ws.numel()
        del ws
        others = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(4)]
        assert at not in [o.data_ptr() for o in others]
        side.synchronize()
        assert torch.equal(y, y2)


def test_a_captured_layer_replays():
    """norm, convolution, scan forward and backward in one graph, replayed on new inputs between eager calls."""
    B, N, E, S, W = 2, 140, 72, 16, 4
    d, a = scan_data(B, N, E, 1, S, None, False, True, True, True, "bf16")
    t = {n: d.dev(v, f32=n in F32_NAMES) for n, v in a.items() if v is not None}
    w, bias, gamma = (d.dev(d.array(*s, f32=True), True) for s in ((E, W), (E,), (E,)))

    def layer(src):
        o = {n: torch.empty_like(src) for n in ("n", "c", "y", "dn", "dc", "dx", "ddt", "dz")}
        mean, rstd = torch.empty(B, N, device=DEV), torch.empty(B, N, device=DEV)
        o.update(dA=torch.empty_like(t["A"]), dB=torch.empty_like(t["Bt"]), dC=torch.empty_like(t["Ct"]), dg=torch.empty(E, device=DEV),
                 dw=torch.empty_like(w), db=torch.empty(E, device=DEV), h1=torch.empty(B, E, S, device=DEV))
        la.la_norm_fwd(src, gamma, None, o["n"], mean, rstd)
        la.la_conv_fwd(o["n"], w, bias, o["c"])
        common = dict(D=t["D"], z=t["z"], dt_bias=t["dt_bias"])
        ws = la.la_scan_fwd(o["c"], t["dt"], t["A"], t["Bt"], t["Ct"], o["y"], h1=o["h1"], keep=True, **common)
        la.la_scan_bwd(o["c"], t["dt"], t["A"], t["Bt"], t["Ct"], t["dy"], o["dc"], o["ddt"], o["dA"], o["dB"], o["dC"], dz=o["dz"],
                       fwd_ws=ws, **common)
        la.la_conv_bwd(o["n"], w, bias, o["dc"], o["dn"], o["dw"], o["db"])
        la.la_norm_bwd(src, gamma, mean, rstd, o["dn"], o["dx"], o["dg"])
        return o

    src = t["x"].clone()
    layer(src)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(src)
    for i in range(3):
        src.copy_(t["x"] * (1 + i))
        want = {n: v.clone() for n, v in layer(src).items()}
        torch.cuda.synchronize()
        for v in out.values():
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(out[n], want[n]), (i, n)
