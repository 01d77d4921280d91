"""The fp64 reference of the norm, convolution and scan against torch's autograd in fp64, closed forms and differences."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

import layer_ref as ref


def t64(a, grad=False):
    return None if a is None else torch.tensor(np.asarray(a, dtype=np.float64), requires_grad=grad)


def close(a, b):
    b = b.detach().numpy() if isinstance(b, torch.Tensor) else b
    return np.allclose(a, b, rtol=1e-10, atol=1e-12)


def test_norm_is_torchs():
    r = np.random.default_rng(0)
    s, g, b, dy, ds = r.standard_normal((7, 33)), r.standard_normal(33), r.standard_normal(33), r.standard_normal((7, 33)), r.standard_normal((7, 33))
    ts, tg, tb = t64(s, True), t64(g, True), t64(b, True)
    y = F.layer_norm(ts, (33,), tg, tb, 1e-5)
    ((y * t64(dy)).sum() + (ts * t64(ds)).sum()).backward()
    o = ref.norm(s, g, b, 1e-5, dy, ds)
    assert close(o["y"], y) and close(o["dx"], ts.grad) and close(o["dgamma"], tg.grad) and close(o["dbeta"], tb.grad)
    assert close(o["mean"], s.mean(1)) and close(o["rstd"], 1 / np.sqrt(s.var(1) + 1e-5))


@pytest.mark.parametrize("lengths", [None, [9, 0, 2]])
@pytest.mark.parametrize("W,silu", [(2, False), (3, True), (4, True)])
def test_conv_is_torchs(W, silu, lengths):
    r = np.random.default_rng(W)
    B, N, E = 3, 9, 5
    x, w, b, x0 = r.standard_normal((B, N, E)), r.standard_normal((E, W)), r.standard_normal(E), r.standard_normal((B, W - 1, E))
    dy, dx1 = r.standard_normal((B, N, E)), r.standard_normal((B, W - 1, E))
    tx, tw, tb, t0 = (t64(a, True) for a in (x, w, b, x0))
    line = torch.cat((t0, tx), 1)
    p = F.conv1d(line.transpose(1, 2), tw[:, None], tb, groups=E).transpose(1, 2)
    y = F.silu(p) if silu else p
    ends = [N] * B if lengths is None else lengths
    y = torch.cat([torch.cat((y[b_:b_ + 1, :n], torch.zeros(1, N - n, E, dtype=torch.float64)), 1) for b_, n in enumerate(ends)])
    x1 = torch.stack([line[b_, n:n + W - 1] for b_, n in enumerate(ends)])
    ((y * t64(dy)).sum() + (x1 * t64(dx1)).sum()).backward()
    o = ref.conv(x, w, b, x0, lengths, silu, dy, dx1)
    assert close(o["y"], y) and close(o["x1"], x1)
    assert close(o["dx"], tx.grad) and close(o["dw"], tw.grad) and close(o["db"], tb.grad) and close(o["dx0"], t0.grad)


@pytest.mark.parametrize("softplus,gated", [(True, True), (False, False)])
def test_scan_is_the_recurrence_under_autograd(softplus, gated):
    r = np.random.default_rng(5)
    B, N, E, G, S = 2, 7, 6, 2, 3
    a = {"x": r.standard_normal((B, N, E)), "dt": np.abs(r.standard_normal((B, N, E))), "A": -np.exp(r.standard_normal((E, S))),
         "Bt": r.standard_normal((B, N, G, S)), "Ct": r.standard_normal((B, N, G, S)), "D": r.standard_normal(E),
         "z": r.standard_normal((B, N, E)) if gated else None, "dt_bias": r.standard_normal(E) if softplus else None,
         "h0": r.standard_normal((B, E, S))}
    dy, dh1 = r.standard_normal((B, N, E)), r.standard_normal((B, E, S))
    t = {k: t64(v, True) for k, v in a.items()}
    h, ys, group = t["h0"], [], torch.arange(E) // (E // G)
    for i in range(N):
        d = t["dt"][:, i] + (t["dt_bias"] if softplus else 0)
        d = F.softplus(d) if softplus else d
        h = torch.exp(d[..., None] * t["A"]) * h + (d * t["x"][:, i])[..., None] * t["Bt"][:, i][:, group]
        v = (h * t["Ct"][:, i][:, group]).sum(-1) + t["D"] * t["x"][:, i]
        ys.append(v * F.silu(t["z"][:, i]) if gated else v)
    y = torch.stack(ys, 1)
    ((y * t64(dy)).sum() + (h * t64(dh1)).sum()).backward()
    o = ref.scan(**a, softplus=softplus, dy=dy, dh1=dh1)
    assert close(o["y"], y) and close(o["h1"], h)
    for name, grad in (("x", "dx"), ("dt", "ddt"), ("A", "dA"), ("Bt", "dB"), ("Ct", "dC"), ("D", "dD"), ("z", "dz"), ("dt_bias", "ddt_bias"),
                       ("h0", "dh0")):
        if t[name] is not None:
            assert close(o[grad], t[name].grad), name


def test_a_sequence_ends_at_its_length_and_a_state_stands_for_the_tokens_before_it():
    r = np.random.default_rng(8)
    B, N, E, S, cut = 2, 9, 4, 3, 4
    a = {n: r.standard_normal((B, N, E)) for n in ("x", "dt", "z", "dy")}
    a.update({n: r.standard_normal((B, N, 1, S)) for n in ("Bt", "Ct")}, A=-np.exp(r.standard_normal((E, S))))
    seq = ("x", "dt", "z", "dy", "Bt", "Ct")
    whole = ref.scan(**a)
    first = ref.scan(**{k: v[:, :cut] if k in seq else v for k, v in a.items()})
    second = ref.scan(**{k: v[:, cut:] if k in seq else v for k, v in a.items()}, h0=first["h1"])
    assert close(np.concatenate((first["y"], second["y"]), 1), whole["y"]) and close(second["h1"], whole["h1"])
    back = ref.scan(**{k: v[:, :cut] if k in seq else v for k, v in a.items()}, dh1=second["dh0"])
    assert close(np.concatenate((back["dx"], second["dx"]), 1), whole["dx"]) and close(back["dA"] + second["dA"], whole["dA"])
    cutoff = ref.scan(**a, lengths=[cut, 0])
    assert close(cutoff["y"][0, :cut], whole["y"][0, :cut]) and not cutoff["y"][0, cut:].any() and not cutoff["y"][1].any()
    assert close(cutoff["h1"][0], first["h1"][0]) and not cutoff["h1"][1].any() and not cutoff["dx"][1].any()


def test_magnitudes_bound_the_values():
    r = np.random.default_rng(9)
    B, N, E, S = 2, 6, 5, 4
    a = {n: r.standard_normal((B, N, E)) for n in ("x", "dt", "z", "dy")}
    a.update({n: r.standard_normal((B, N, 1, S)) for n in ("Bt", "Ct")}, A=-np.exp(r.standard_normal((E, S))), D=r.standard_normal(E),
             h0=r.standard_normal((B, E, S)), dh1=r.standard_normal((B, E, S)))
    pairs = [(ref.scan(**a), ref.scan(**a, mag=True))]
    w, b, dy = r.standard_normal((E, 4)), r.standard_normal(E), r.standard_normal((B, N, E))
    pairs.append((ref.conv(a["x"], w, b, None, None, True, dy), ref.conv(a["x"], w, b, None, None, True, dy, mag=True)))
    s, g = r.standard_normal((5, 11)), r.standard_normal(11)
    pairs.append((ref.norm(s, g, g, 1e-5, s, s), ref.norm(s, g, g, 1e-5, s, s, mag=True)))
    for values, sizes in pairs:
        for n in values:
            if n != "x1":
                assert (np.abs(values[n]) <= sizes[n] * (1 + 1e-12) + 1e-300).all(), n


def test_bf16_rounding_is_torchs():
    x = np.random.default_rng(1).standard_normal(4096).astype(np.float32) * 3
    assert np.array_equal(ref.to_bf16(x), torch.from_numpy(x).bfloat16().float().numpy())
