"""The norm, convolution and scan as a model uses them: through autograd in a residual layer, prompt and then token by token,
and at the edges of what a call may be (large tensors, extreme values, unfinished sequences, side streams)."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

import layer_ref as ref
import paper_2006_16236_amd as la
from gpu_util import DEV, TOL_F32
from paper_2006_16236_amd import autograd

pytestmark = pytest.mark.gpu


# ---- a residual layer ---------------------------------------------------------------------------------------

M, E, S, R, W = 40, 64, 16, 8, 4                                     # model, inner width, states, rank of dt, taps


def weights(seed, device, dtype):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, scale=1.0: (torch.randn(s, generator=g, dtype=torch.float64) * scale).to(device, dtype)
    p = {"gamma": 1 + n(M, scale=0.1), "beta": n(M, scale=0.1), "win": n(M, 2 * E, scale=M ** -0.5), "w": n(E, W, scale=0.5), "cb": n(E, scale=0.1),
         "wx": n(E, R + 2 * S, scale=E ** -0.5), "wdt": n(R, E, scale=R ** -0.5), "tb": n(E) - 3, "A": -torch.exp(n(E, S, scale=0.3)) * torch.arange(1, S + 1).to(device, dtype),
         "D": n(E), "wout": n(E, M, scale=E ** -0.5)}
    return {k: v.requires_grad_(True) for k, v in p.items()}


def layer(p, x, r, states=None):
    """norm of the residual sum, projection, convolution, scan, projection: (output, residual sum, states)"""
    n, s = la.layer_norm(x, p["gamma"], p["beta"], residual=r)
    xi, z = (n @ p["win"]).split(E, -1)                              # halves of one projection, never copied
    xi, conv = la.causal_conv(xi, p["w"], p["cb"], state=None if states is None else states[0])
    proj = xi @ p["wx"]
    dt, (Bt, Ct) = proj[..., :R] @ p["wdt"], (proj[..., R + i * S:R + (i + 1) * S].unflatten(-1, (1, S)) for i in (0, 1))
    y, h = la.selective_scan(xi, dt, p["A"], Bt, Ct, D=p["D"], z=z, dt_bias=p["tb"], state=None if states is None else states[1])
    return y @ p["wout"], s, (conv, h)


def layer64(p, x, r):
    s = x + r
    n = F.layer_norm(s, (M,), p["gamma"], p["beta"], 1e-5)
    xi, z = (n @ p["win"]).split(E, -1)
    xi = F.silu(F.conv1d(F.pad(xi.transpose(1, 2), (W - 1, 0)), p["w"][:, None], p["cb"], groups=E).transpose(1, 2))
    proj = xi @ p["wx"]
    d = F.softplus(proj[..., :R] @ p["wdt"] + p["tb"])
    h, out = torch.zeros(x.shape[0], E, S, dtype=torch.float64), []
    for t in range(x.shape[1]):
        h = torch.exp(d[:, t, :, None] * p["A"]) * h + (d[:, t] * xi[:, t])[..., None] * proj[:, t, None, R:R + S]
        out.append((h * proj[:, t, None, R + S:]).sum(-1) + p["D"] * xi[:, t])
    return (torch.stack(out, 1) * F.silu(z)) @ p["wout"], s, h


def test_a_residual_layer_and_its_gradients():
    B, N = 3, 45
    g = torch.Generator().manual_seed(1)
    x64, r64, go, gs, gh = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((B, N, M), (B, N, M), (B, N, M), (B, N, M), (B, E, S)))
    p64, p = weights(2, "cpu", torch.float64), weights(2, DEV, torch.float32)
    x, r = x64.float().to(DEV).requires_grad_(True), r64.float().to(DEV).requires_grad_(True)
    x64, r64 = x64.requires_grad_(True), r64.requires_grad_(True)
    o64, s64, h64 = layer64(p64, x64, r64)
    ((o64 * go).sum() + (s64 * gs).sum() + (h64 * gh).sum()).backward()
    o, s, (conv, h) = layer(p, x, r)
    dev = lambda t: t.float().to(DEV)
    ((o * dev(go)).sum() + (s * dev(gs)).sum() + (h * dev(gh)).sum()).backward()
    pairs = [(o, o64), (s, s64), (h, h64), (x.grad, x64.grad), (r.grad, r64.grad)] + [(p[k].grad, p64[k].grad) for k in p]
    for i, (got, want) in enumerate(pairs):
        err = (got.detach().double().cpu() - want.detach()).abs().max() / want.detach().abs().max()
        assert err <= TOL_F32, (i, float(err))                       # the library's fp32 gate up to 4096 tokens


def test_a_prompt_then_token_by_token_is_the_whole_sequence():
    B, N, first = 4, 23, 17
    g = torch.Generator().manual_seed(3)
    x, r = (torch.randn(B, N, M, generator=g).to(DEV) for _ in range(2))
    p = {k: v.detach() for k, v in weights(4, DEV, torch.float32).items()}
    want, _, (conv1, h1) = layer(p, x, r)
    got, _, (conv, h) = layer(p, x[:, :first].contiguous(), r[:, :first].contiguous())
    assert (got - want[:, :first]).abs().max() <= TOL_F32 * want.abs().max()
    for t in range(first, N):
        n, s = torch.empty(B, M, device=DEV), torch.empty(B, M, device=DEV)
        la.la_norm_fwd(x[:, t].contiguous(), p["gamma"], p["beta"], n, r=r[:, t].contiguous(), s=s)
        xi, z = ((n @ p["win"])[:, i * E:(i + 1) * E].contiguous() for i in (0, 1))
        c, y = torch.empty_like(xi), torch.empty_like(xi)
        la.la_conv_step(xi, p["w"], p["cb"], conv, c)
        proj = c @ p["wx"]
        Bt, Ct = (proj[:, R + i * S:R + (i + 1) * S].reshape(B, 1, S).contiguous() for i in (0, 1))
        la.la_scan_step(c, proj[:, :R] @ p["wdt"], p["A"], Bt, Ct, h, y, D=p["D"], z=z, dt_bias=p["tb"])
        assert (y @ p["wout"] - want[:, t]).abs().max() <= TOL_F32 * want.abs().max(), t
    assert (h - h1).abs().max() <= TOL_F32 * h1.abs().max() and (conv - conv1).abs().max() <= TOL_F32 * conv1.abs().max()


def test_prompts_of_different_lengths_leave_the_states_of_each():
    B, N = 4, 50
    lengths = torch.tensor([50, 1, 0, 33], dtype=torch.int32, device=DEV)
    x = torch.randn(B, N, E, device=DEV)
    w = torch.randn(E, W, device=DEV)
    dt, z = torch.randn(B, N, E, device=DEV), torch.randn(B, N, E, device=DEV)
    A, Bt, Ct = -torch.rand(E, S, device=DEV), torch.randn(B, N, 1, S, device=DEV), torch.randn(B, N, 1, S, device=DEV)
    c0, h0 = torch.randn(B, W - 1, E, device=DEV), torch.randn(B, E, S, device=DEV)
    c, conv = la.causal_conv(x, w, state=c0, lengths=lengths)
    y, h = la.selective_scan(c, dt, A, Bt, Ct, z=z, state=h0, lengths=lengths)
    for b, n in enumerate(lengths.tolist()):
        assert not c[b, n:].any() and not y[b, n:].any()
        if n == 0:
            assert torch.equal(conv[b], c0[b]) and torch.equal(h[b], h0[b])
            continue
        one = lambda t: t[b:b + 1, :n].clone()
        cb, convb = la.causal_conv(one(x), w, state=c0[b:b + 1].clone())
        yb, hb = la.selective_scan(one(c), one(dt), A, one(Bt), one(Ct), z=one(z), state=h0[b:b + 1].clone())
        assert torch.equal(cb[0], c[b, :n]) and torch.equal(convb[0], conv[b])
        assert (yb[0] - y[b, :n]).abs().max() <= 1e-5 * y.abs().max() and (hb[0] - h[b]).abs().max() <= 1e-5 * h.abs().max()


# ---- autograd's corners -------------------------------------------------------------------------------------

def test_gradients_when_only_part_of_the_outputs_is_used():
    B, N = 2, 9
    leaf = lambda *s: torch.randn(*s, device=DEV).requires_grad_(True)
    x, r, g = leaf(B, N, E), leaf(B, N, E), leaf(E)
    _, s = la.layer_norm(x, g, None, residual=r)
    s.sum().backward()
    assert torch.equal(x.grad, torch.ones_like(x)) and torch.equal(r.grad, x.grad) and not g.grad.any()
    w, c0 = leaf(E, W), leaf(B, W - 1, E)
    x.grad = None
    _, state = la.causal_conv(x, w, state=c0)
    state.sum().backward()
    assert not x.grad[:, :N - W + 1].any() and torch.equal(x.grad[:, N - W + 1:], torch.ones(B, W - 1, E, device=DEV)) and not w.grad.any()
    A, Bt, Ct, dt, h0 = leaf(E, S), leaf(B, N, 1, S), leaf(B, N, 1, S), leaf(B, N, E), leaf(B, E, S)
    _, h = la.selective_scan(x, dt, A, Bt, Ct, state=h0)
    h.sum().backward()
    assert h0.grad.abs().sum() > 0 and not Ct.grad.any()
    y, _ = la.selective_scan(x.detach(), dt.detach(), A.detach(), Bt.detach(), Ct.detach(), D=g)
    g.grad = None
    y.sum().backward()                                               # only D wants a gradient
    assert (g.grad - x.detach().sum((0, 1))).abs().max() <= 1e-4 * x.detach().abs().sum((0, 1)).max()
    with torch.no_grad():
        y2, _ = la.selective_scan(x, dt, A, Bt, Ct, D=g)
    assert torch.equal(y, y2)


def test_rows_that_need_no_copy_are_not_copied():
    both = torch.randn(2, 5, 2 * E, device=DEV)
    assert autograd._rows(both[..., E:]).data_ptr() == both[..., E:].data_ptr()
    assert autograd._rows(both[:, 1:4]).is_contiguous()              # sequences further apart than their tokens
    assert autograd._rows(both[..., 1:E]).data_ptr() % 16 == 0       # starts off 16 bytes
    assert autograd._rows(both.transpose(1, 2)).is_contiguous()
    w, x = torch.randn(E - 1, W, device=DEV), both[..., 1:E]
    y, _ = la.causal_conv(x, w)
    y2, _ = la.causal_conv(x.contiguous(), w)
    assert torch.equal(y, y2)


def test_autograd_on_a_side_stream_and_twice_through_one_leaf():
    B, N = 2, 40
    x = torch.randn(B, N, E, device=DEV, requires_grad=True)
    w = torch.randn(E, W, device=DEV, requires_grad=True)

    def run():
        y, _ = la.causal_conv(x, w)
        y, _ = la.causal_conv(y, w)                                  # the same weight twice
        return torch.autograd.grad(la.layer_norm(y).square().sum(), (x, w))

    want = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_second_derivatives_are_refused():
    """The gradient kernels have no gradient of their own: asking for one must not leave a term out in silence."""
    x = torch.randn(2, 20, E, device=DEV, requires_grad=True)
    w = torch.randn(E, W, device=DEV, requires_grad=True)
    A, Bt = -torch.rand(E, S, device=DEV), torch.randn(2, 20, 1, S, device=DEV)
    for y in (la.layer_norm(x), la.causal_conv(x, w)[0], la.selective_scan(x, x, A, Bt, Bt)[0]):
        g, = torch.autograd.grad((y * x).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.sum().backward()


# ---- edges --------------------------------------------------------------------------------------------------

def test_what_follows_a_token_does_not_reach_it():
    B, N, t = 2, 70, 37
    a = {n: torch.randn(B, N, E, device=DEV) for n in ("x", "dt", "z")}
    a.update({n: torch.randn(B, N, 1, S, device=DEV) for n in ("Bt", "Ct")})
    A, w = -torch.rand(E, S, device=DEV), torch.randn(E, W, device=DEV)
    y, c = (torch.empty(B, N, E, device=DEV) for _ in range(2))
    la.la_scan_fwd(a["x"], a["dt"], A, a["Bt"], a["Ct"], y, z=a["z"])
    la.la_conv_fwd(a["x"], w, None, c)
    for bad in (float("nan"), float("inf"), 1e30):
        b = {n: v.clone() for n, v in a.items()}
        for v in b.values():
            v[:, t:] = bad
        y2, c2 = torch.empty_like(y), torch.empty_like(c)
        la.la_scan_fwd(b["x"], b["dt"], A, b["Bt"], b["Ct"], y2, z=b["z"])
        la.la_conv_fwd(b["x"], w, None, c2)
        assert torch.equal(y2[:, :t], y[:, :t]) and torch.equal(c2[:, :t], c[:, :t])


def test_extreme_values():
    """Steps that underflow and steps of 100, gates that saturate, decays of 0, exp(-1600) and growth: against fp64."""
    B, N, e, s = 1, 12, 8, 8
    r = np.random.default_rng(4)
    x = r.standard_normal((B, N, e)).astype(np.float32)
    dt = np.tile(np.array([-100, -30, -5, 0, 3, 20, 60, 100], dtype=np.float32), (B, N, 1))
    z = np.tile(np.array([-200, -20, -1, 0, 1, 20, 88, 200], dtype=np.float32), (B, N, 1))
    A = np.tile(np.array([0, -0.001, -0.1, -1, -4, -16, 0.001, -0.5], dtype=np.float32), (e, 1))
    Bt, Ct, dy = (r.standard_normal(sh).astype(np.float32) for sh in ((B, N, 1, s), (B, N, 1, s), (B, N, e)))
    dev = lambda v: torch.from_numpy(v).to(DEV)
    t = {n: dev(v) for n, v in (("x", x), ("dt", dt), ("z", z), ("A", A), ("Bt", Bt), ("Ct", Ct), ("dy", dy))}
    o = {n: torch.empty_like(t[m]) for n, m in (("y", "x"), ("dx", "x"), ("ddt", "x"), ("dz", "x"), ("dA", "A"), ("dB", "Bt"), ("dC", "Ct"))}
    la.la_scan_fwd(t["x"], t["dt"], t["A"], t["Bt"], t["Ct"], o["y"], z=t["z"])
    la.la_scan_bwd(t["x"], t["dt"], t["A"], t["Bt"], t["Ct"], t["dy"], o["dx"], o["ddt"], o["dA"], o["dB"], o["dC"], z=t["z"], dz=o["dz"])
    want, mag = (ref.scan(x, dt, A, Bt, Ct, z=z, dy=dy, mag=m) for m in (False, True))
    # an exponent of d A = 1600 is off by 3 2^-24 of itself, but its power is 0 then; what counts is |d A| exp(d A) <= 1 / e and,
    # with growth, 0.1 a token.  The sigmoids of the gate and of softplus add the relative error of exp(-v), |v| 2^-24, up to
    # where they vanish: 100
    k = ref.roundings(N, s, np.ones(1), 1.0) + 2 * 104
    for n in o:
        # values that underflow in fp32 (below 2^-126, flushed) are nothing to be compared
        ref.check(n, o[n].double().cpu().numpy() * (np.abs(want[n]) > 1e-30), want[n] * (np.abs(want[n]) > 1e-30), mag[n] + 1e-30, "f32", 2 * k)


def test_more_rows_than_a_grid_has_workgroups():
    for rows, width in ((4 * (1 << 20) + 5, 8), (2051, 8200)):
        x = torch.randn(rows, width, device=DEV).bfloat16()
        y, m, r = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        la.la_norm_fwd(x, None, None, y, m, r)
        tail = x[-7:].clone()
        want = torch.empty_like(tail)
        la.la_norm_fwd(tail, None, None, want)
        assert torch.equal(y[-7:], want)
        dx, db = torch.empty_like(x), torch.empty(width, device=DEV)
        la.la_norm_bwd(x, None, m, r, x, dx, dbeta=db)
        dw = torch.empty_like(tail)
        la.la_norm_bwd(tail, None, m[-7:].clone(), r[-7:].clone(), tail, dw)
        assert torch.equal(dx[-7:], dw)
        exact = x.double().sum(0)
        assert (db.double() - exact).abs().max() <= 2.0 ** -24 * (rows / 4096 + 100) * x.double().abs().sum(0).max()


def test_tensors_of_more_than_2_to_the_31_elements():
    """Rows far behind 2^32 bytes: the end of one long sequence against the same tokens on their own, from the state before."""
    N, width, tail = (1 << 19) + 96, 4096, 96
    x = torch.empty(1, N, width, dtype=torch.bfloat16, device=DEV).normal_()
    assert x.numel() > 1 << 31
    cut = N - tail
    w = torch.randn(width, W, device=DEV)
    y, end = torch.empty_like(x), x[:, cut:].clone()
    la.la_conv_fwd(x, w, None, y)
    want = torch.empty_like(end)
    la.la_conv_fwd(end, w, None, want, x0=x[:, cut - W + 1:cut].clone())
    assert torch.equal(y[:, cut:], want)
    dx = torch.empty_like(x)
    la.la_conv_bwd(x, w, None, y, dx)
    dwant = torch.empty_like(end)
    la.la_conv_bwd(end, w, None, want, dwant, x0=x[:, cut - W + 1:cut].clone())
    assert torch.equal(dx[:, cut:], dwant)
    la.la_norm_fwd(x, None, None, y)
    la.la_norm_fwd(end, None, None, want)
    assert torch.equal(y[:, cut:], want)
    s = 8
    dt = torch.full((1, N, width), -3.0, dtype=torch.bfloat16, device=DEV)
    A, Bt, Ct = -torch.rand(width, s, device=DEV) - 0.1, torch.randn(1, N, 1, s, device=DEV).bfloat16(), torch.randn(1, N, 1, s, device=DEV).bfloat16()
    ws = la.la_scan_fwd(x, dt, A, Bt, Ct, y, keep=True)
    h = torch.empty(1, width, s, device=DEV)
    head = slice(cut - 4096, cut)                                    # decays of at least 0.1 x softplus(-3) a token: nothing older is left
    la.la_scan_fwd(x[:, head].clone(), dt[:, head].clone(), A, Bt[:, head].clone(), Ct[:, head].clone(), torch.empty(1, 4096, width, dtype=x.dtype, device=DEV), h1=h)
    e = [t[:, cut:].clone() for t in (dt, Bt, Ct)]
    ws2 = la.la_scan_fwd(end, e[0], A, e[1], e[2], want, h0=h, keep=True)
    assert (y[:, cut:].float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()
    ddt, dB, dC, dA = torch.empty_like(x), torch.empty_like(Bt), torch.empty_like(Ct), torch.empty_like(A)
    la.la_scan_bwd(x, dt, A, Bt, Ct, x, dx, ddt, dA, dB, dC, fwd_ws=ws)
    o = [torch.empty_like(t) for t in (end, end, A, e[1], e[2])]
    la.la_scan_bwd(end, e[0], A, e[1], e[2], end, o[0], o[1], o[2], o[3], o[4], h0=h, fwd_ws=ws2)
    for got, one in ((dx, o[0]), (ddt, o[1]), (dB, o[3]), (dC, o[4])):
        assert (got[:, cut:].float() - one.float()).abs().max() <= 2.0 ** -7 * one.float().abs().max()
