"""The convolution at sizes whose threads take their longest runs of tokens: 32 and 16 steps backwards, 16 tokens forwards."""
import numpy as np
import pytest
import torch

import layer_ref as ref
import paper_2006_16236_amd as la

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def reference(x, w, bias, x0, lengths, silu, dy, dx1):
    """{name: (value, magnitude)} in fp64, all tokens at once; magnitudes as layer_ref.conv(mag=True) has them."""
    B, N, E = x.shape
    W = w.shape[1]
    x, w, bias, x0, dy, dx1 = (t.double() for t in (x, w, bias, x0, dy, dx1))
    end = torch.full((B,), N, device=x.device) if lengths is None else lengths.long().clamp(0, N)
    real = (torch.arange(N, device=x.device)[None] < end[:, None])[..., None]
    line = torch.cat((x0, torch.where(real, x, 0.0)), 1)
    rows = end[:, None] + torch.arange(W - 1, device=x.device)                # of the W - 1 last ones, in `line`
    rows = rows[..., None].expand(-1, -1, E)
    taps = [line[:, k:k + N] for k in range(W)]
    p = bias + sum(taps[k] * w[:, k] for k in range(W))
    pm = bias.abs() + sum((taps[k] * w[:, k]).abs() for k in range(W))
    q = torch.sigmoid(p)
    out = {"y": (p * q, pm * 1.1 + p.abs()) if silu else (p, pm), "x1": (line.gather(1, rows),) * 2}
    slope = q * (1 + p * (1 - q)) if silu else torch.ones_like(p)
    rough = 1.0 + p.abs() * q + 0.5 * pm if silu else torch.ones_like(p)
    dy = torch.where(real, dy, 0.0)
    d, dm = dy * slope, dy.abs() * rough
    into = []
    for v, wv, g in ((d, w, dx1), (dm, w.abs(), dx1.abs())):
        back = torch.zeros_like(line).scatter_add_(1, rows, g)
        for k in range(W):
            back[:, k:k + N] += v * wv[:, k]
        into.append(back)
    out["y"] = tuple(torch.where(real, t, 0.0) for t in out["y"])
    out["dx"] = tuple(torch.where(real, t[:, W - 1:], 0.0) for t in into)
    out["dx0"] = tuple(t[:, :W - 1] for t in into)
    out["dw"] = tuple(torch.stack([(v * (t.abs() if m else t)).sum((0, 1)) for t in taps], 1) for v, m in ((d, False), (dm, True)))
    out["db"] = d.sum((0, 1)), dm.sum((0, 1))
    return out


@pytest.mark.parametrize("lengths", [None, [9, 0, 2, 11]])
@pytest.mark.parametrize("W,silu", [(2, True), (3, False), (4, True)])
def test_the_reference_is_that_of_the_short_runs(W, silu, lengths):
    r = np.random.default_rng(W)
    B, N, E = 4, 9, 5
    a = [r.standard_normal(s).astype(np.float32) for s in ((B, N, E), (E, W), (E,), (B, W - 1, E))]
    dy, dx1 = (r.standard_normal(s).astype(np.float32) for s in ((B, N, E), (B, W - 1, E)))
    t = lambda v: torch.from_numpy(v)
    got = reference(*map(t, a), None if lengths is None else torch.tensor(lengths), silu, t(dy), t(dx1))
    for i, mag in enumerate((False, True)):
        for name, want in ref.conv(*a, lengths, silu, dy, dx1, mag=mag).items():
            if not (mag and name == "x1"):
                assert np.allclose(got[name][i].numpy(), want, rtol=1e-10, atol=1e-12), (name, mag)


RUNS = [  # B, N, E, W, silu, ragged, steps of a run backwards
    (9, 3781, 1030, 4, True, True, 32), (5, 7001, 1001, 2, False, False, 32), (7, 3001, 1697, 3, True, True, 32),
    (2, 1001, 1001, 3, True, True, 16), (3, 531, 1028, 4, True, False, 16), (64, 500, 40, 2, True, True, 16),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,E,W,silu,ragged,steps", RUNS)
def test_conv_of_long_runs(B, N, E, W, silu, ragged, steps, dtype):
    dev = "cuda:0"
    g = torch.Generator(device=dev).manual_seed(B * N + E)
    rand = lambda *s, t=TYPES[dtype]: torch.randn(*s, generator=g, device=dev).to(t)
    f32 = torch.float32
    x, dy, x0, dx1 = rand(B, N, E), rand(B, N, E), rand(B, W - 1, E), rand(B, W - 1, E)
    w, bias = rand(E, W, t=f32), rand(E, t=f32)
    lengths = None
    if ragged:
        lengths = torch.randint(0, N + 1, (B,), generator=g, device=dev, dtype=torch.int32)
        lengths[0] = N
    # the backward takes the runs that this test is about: a partial sum for each 256 / lanes of them
    pieces, lanes = -(-E // 4), 64
    while lanes // 2 >= pieces:
        lanes //= 2
    cuts = B * -(-N // (steps - W + 1))
    parts = -(-cuts // (256 // lanes))
    assert la.la_conv_bwd_workspace(B, N, E, W) == -(-parts * E * (W + 1) * 4 // 256) * 256

    y, x1, dx, dx0 = torch.empty_like(x), torch.empty_like(x0), torch.empty_like(x), torch.empty_like(x0)
    dw, db = torch.empty_like(w), torch.empty_like(bias)
    la.la_conv_fwd(x, w, bias, y, x0=x0, x1=x1, lengths=lengths, silu=silu)
    la.la_conv_bwd(x, w, bias, dy, dx, dw, db, x0=x0, dx1=dx1, dx0=dx0, lengths=lengths, silu=silu)
    want = reference(x, w, bias, x0, lengths, silu, dy, dx1)

    def check(name, got, k, kind):
        value, mag = want[name]
        room = k * U * mag * (1 + 2.0 ** -7) + ref.HALF_STEP[kind] * value.abs() + 1e-37
        bad = ((got.double() - value).abs() / room).max().item()
        assert bad <= 1.0, f"{name}: {bad:.3g} times the bound"          # (NaN is not)

    k = 2 * W + 16                                                       # taps, bias, the sigmoid's exp, division and products
    check("y", y, k, dtype)
    assert torch.equal(x1.double(), want["x1"][0])                       # copies
    check("dx", dx, 2 * k, dtype)
    check("dx0", dx0, 2 * k, dtype)
    # a run's tokens one after the other, the runs of a workgroup, the workgroups in 16 slices, the slices
    k += steps + 256 // lanes + -(-parts // 16) + 18
    check("dw", dw, k, "f32")
    check("db", db, k, "f32")
