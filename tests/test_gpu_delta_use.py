"""The head norm and the gated delta rule as a model uses them: one after the other through autograd in a layer, prompt and then
token by token, and at the edges of what a call may be (pieces, far rows, streams, what a step changes)."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

import delta_ref as ref
import paper_2006_16236_amd as la
from gpu_util import DEV, TOL_F32
from test_gpu_delta import Case
from test_gpu_layer import host

pytestmark = pytest.mark.gpu


# ---- a layer: projection, norm and rotation, delta rule, norm, projection ----------------------------------------

E, H, HK, D, M, R = 40, 4, 2, 32, 16, 16
FREQ = 100.0 ** (-torch.arange(R // 2, dtype=torch.float64) / (R // 2))


def weights(seed, device, dtype):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, scale=1.0: (torch.randn(s, generator=g, dtype=torch.float64) * scale).to(device, dtype)
    p = {"win": n(E, 2 * HK * D + H * M, scale=E ** -0.5), "wq": 1 + n(D, scale=0.2), "wk": 1 + n(D, scale=0.2), "wg": n(E, H, scale=E ** -0.5), "wb": n(E, H, scale=E ** -0.5),
         "rate": torch.exp(n(H, scale=0.5)), "gamma": 1 + n(M, scale=0.1), "wout": n(H * M, E, scale=(H * M) ** -0.5)}
    return {k: v.requires_grad_(True) for k, v in p.items()}


def parts(p, x):
    proj = x @ p["win"]
    q, k, v = proj.split((HK * D, HK * D, H * M), -1)               # parts of one projection, never copied
    g, beta = -p["rate"] * F.softplus(x @ p["wg"] - 2), torch.sigmoid(x @ p["wb"])
    return q.unflatten(-1, (HK, D)), k.unflatten(-1, (HK, D)), v.unflatten(-1, (H, M)), g, beta


def layer(p, x, pos, state=None):
    q, k, v, g, beta = parts(p, x)
    q, k = la.qk_norm(q, k, p["wq"], p["wk"], FREQ.float().to(x.device), pos, norm="rms")
    k = la.qk_norm(k, norm="l2")
    o, state = la.gated_delta(q, k, v, g, beta, state=state, scale=D ** -0.5)
    return la.layer_norm(o, p["gamma"]).flatten(2) @ p["wout"], state


def layer64(p, x, pos):
    q, k, v, g, beta = parts(p, x)
    angle = pos.double()[..., None, None] * FREQ

    def rms(t, w):
        t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w
        a, b = t[..., :R // 2], t[..., R // 2:R]
        return torch.cat((a * torch.cos(angle) - b * torch.sin(angle), b * torch.cos(angle) + a * torch.sin(angle), t[..., R:]), -1)

    q, k = rms(q, p["wq"]), rms(k, p["wk"])
    k = k * torch.rsqrt((k * k).sum(-1, keepdim=True) + 1e-6)
    q, k = q.repeat_interleave(H // HK, 2), k.repeat_interleave(H // HK, 2)
    S, out = torch.zeros(x.shape[0], H, D, M, dtype=torch.float64), []
    for t in range(x.shape[1]):
        S = S * torch.exp(g[:, t])[..., None, None]
        new = beta[:, t, :, None] * (v[:, t] - (S * k[:, t, ..., None]).sum(2))
        S = S + k[:, t, ..., None] * new[:, :, None]
        out.append(D ** -0.5 * (S * q[:, t, ..., None]).sum(2))
    mixed = torch.stack(out, 1)
    o = F.layer_norm(mixed, (M,), p["gamma"], None, 1e-5)
    return o.flatten(2) @ p["wout"], S, mixed


@pytest.mark.parametrize("N", [1, 37, 150])
def test_a_layer_and_its_gradients(N):
    B = 3
    g = torch.Generator().manual_seed(N)
    x64, go, gh = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((B, N, E), (B, N, E), (B, H, D, M)))
    pos = torch.randint(0, 5000, (B, N), generator=g, dtype=torch.int32)
    p64, p = weights(2, "cpu", torch.float64), weights(2, DEV, torch.float32)
    x, x64 = x64.float().to(DEV).requires_grad_(True), x64.float().double().requires_grad_(True)
    o64, h64, mixed = layer64(p64, x64, pos)
    mixed.retain_grad()
    ((o64 * go).sum() + (h64 * gh).sum()).backward()
    o, h = layer(p, x, pos.to(DEV))
    ((o * go.float().to(DEV)).sum() + (h * gh.float().to(DEV)).sum()).backward()
    for name, got, want in [("o", o, o64), ("h", h, h64), ("x", x.grad, x64.grad)] + [(k, p[k].grad, p64[k].grad) for k in p]:
        if N == 1 and name in ("wg", "rate"):
            # A zero state has nothing to lose: the exact gradient of g is 0.  It is formed as q . dq - k . dk (- dv . (v - u), where u = v
            # to the bit), here two sums of the same value T = o . do, and <dh1, h1> enters both k . dk and the chunk's end.  Each goes through
            # at most D + 2 * 64 + 32 = 192 roundings of 2^-24 of its terms' magnitudes, four sums: 768 2^-24 (T + |dh1| |h1|), and
            # |dg / d(x wg)| <= rate, |dg / d rate| <= softplus < 8, |x| < 8.
            T = (mixed.detach().abs() * mixed.grad.abs()).sum() + (gh.abs() * h64.detach().abs()).sum()
            assert got.abs().max() <= 768 * 2.0 ** -24 * T * 8 * max(1.0, float(p64["rate"].detach().max())), name
            continue
        err = (got.detach().double().cpu() - want.detach()).abs().max() / want.detach().abs().max()
        assert err <= TOL_F32, (name, float(err))                    # the library's fp32 gate up to 4096 tokens


def test_a_prompt_then_token_by_token_is_the_whole_sequence():
    B, N, first = 4, 75, 69
    x = torch.randn(B, N, E, generator=torch.Generator().manual_seed(3)).to(DEV)
    pos = (torch.arange(N, dtype=torch.int32) + torch.tensor([[0], [7], [100], [99999]], dtype=torch.int32)).to(DEV)
    p = {k: v.detach() for k, v in weights(4, DEV, torch.float32).items()}
    want, h1 = layer(p, x, pos)
    got, h = layer(p, x[:, :first].contiguous(), pos[:, :first].contiguous())
    assert (got - want[:, :first]).abs().max() <= TOL_F32 * want.abs().max()
    for t in range(first, N):
        q, k, v, g, beta = parts(p, x[:, t:t + 1])
        at = pos[:, t:t + 1].contiguous()
        q, k = la.qk_norm(q, k, p["wq"], p["wk"], FREQ.float().to(DEV), at)
        k = la.qk_norm(k, norm="l2")
        o = torch.empty(B, H, M, device=DEV)
        la.la_delta_step(q[:, 0], k[:, 0], v[:, 0].contiguous(), g[:, 0].contiguous(), beta[:, 0].contiguous(), h, o)
        got = la.layer_norm(o[:, None], p["gamma"]).flatten(2) @ p["wout"]
        assert (got[:, 0] - want[:, t]).abs().max() <= TOL_F32 * want.abs().max(), t
    assert (h - h1).abs().max() <= TOL_F32 * h1.abs().max()


def test_the_attention_on_normed_and_turned_heads():
    """qk_norm in front of the attention of the same layout."""
    B, N, H_, D_ = 2, 50, 2, 64
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(B, N, H_, D_, generator=g).to(DEV).requires_grad_(True) for _ in range(3))
    freq = (100.0 ** (-torch.arange(32) / 32)).to(DEV)
    a, b = la.qk_norm(q, k, freq=freq)
    la.causal_linear_attention(a, b, v, layout="bnhd").sum().backward()
    q2, k2 = (t.detach().clone().requires_grad_(True) for t in (q, k))
    angle = torch.arange(N, device=DEV)[:, None, None] * freq

    def plain(t):
        t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6)
        x, y = t.split(32, -1)
        return torch.cat((x * angle.cos() - y * angle.sin(), x * angle.sin() + y * angle.cos()), -1)

    c, d = plain(q2), plain(k2)
    assert (a - c).abs().max() <= 1e-5 and (b - d).abs().max() <= 1e-5
    la.causal_linear_attention(c, d, v.detach(), layout="bnhd").sum().backward()
    for x, y in ((q.grad, q2.grad), (k.grad, k2.grad)):
        assert (x - y).abs().max() <= TOL_F32 * y.abs().max()


# ---- front ends -----------------------------------------------------------------------------------------------

def test_front_ends_take_any_strides_and_only_what_is_asked_for():
    c = Case(3, "f32", 2, 70, 4, 2, 32, 48)
    x, _ = c.inputs()
    h0 = c.d.dev(c.h0, True)
    want = la.gated_delta(*x, state=h0)
    odd = torch.zeros(2, 70, 2 * 32 + 3, device=DEV)
    odd[..., :64] = x[0].flatten(2)
    q = odd[..., :64].unflatten(-1, (2, 32))                          # tokens 67 elements apart: copied
    k = x[1].permute(2, 3, 0, 1).contiguous().permute(2, 3, 0, 1)
    got = la.gated_delta(q, k, x[2], x[3].transpose(0, 1).contiguous().transpose(0, 1), x[4], state=h0)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q = x[0].clone().requires_grad_(True)                             # one gradient, from the state alone
    la.gated_delta(q, *x[1:])[1].sum().backward()
    assert not q.grad.any()
    beta = x[4].clone().requires_grad_(True)
    la.gated_delta(*x[:3], None, beta)[1].sum().backward()
    assert beta.grad.abs().max() > 0
    w = torch.ones(32, device=DEV, requires_grad=True)
    la.qk_norm(x[0], wq=w).sum().backward()
    assert w.grad is not None


def test_a_second_derivative_is_refused_and_a_stepped_state_too():
    c = Case(4, "f32", 1, 5, 1, 1, 32, 16)
    x, _ = c.inputs()
    v = x[2].requires_grad_(True)
    h = c.d.dev(c.h0, True)
    o, _ = la.gated_delta(x[0], x[1], v, x[3], x[4], state=h)
    g, = torch.autograd.grad(o.sum(), v, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
    o, _ = la.gated_delta(x[0], x[1], v, x[3], x[4], state=h)
    la.la_delta_step(*(t[:, 0].detach().contiguous() for t in x), h, torch.empty(1, 1, 16, device=DEV))
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        o.sum().backward()


# ---- edges ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D_,M_", [(32, 80), (64, 64), (128, 48)])
def test_pieces_of_sequences_of_different_lengths(D_, M_, dtype):
    """Few heads, long sequences: pieces, of which some sequences have all, one, two, or none."""
    Case(D_, dtype, 5, 1100, 1, 1, D_, M_, [1100, 700, 150, 0, 64]).check()


@pytest.mark.parametrize("D_,M_,dtype", [(64, 64, "f32"), (32, 32, "bf16")])
def test_more_pieces_than_compute_units(D_, M_, dtype):
    """24 heads of 32 chunks: eight pieces each, whose transitions are 312 workgroups."""
    n = 1024 if dtype == "f32" else 2048
    Case(D_ + 1, dtype, 3, n - 1, 8, 4, D_, M_, [n - 1, 7, n // 2]).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_sequence_of_a_batch_alone_is_the_same_within_the_bounds(dtype):
    """Alone it goes in pieces, beside 63 others it does not."""
    c = Case(6, dtype, 1, 640, 4, 4, 64, 64)
    want = c.want()
    alone = c.run()
    for n in ("q", "k", "v", "do", "g", "beta", "h0", "dh1"):
        setattr(c, n, np.repeat(getattr(c, n), 64, 0))
    c.dims = (64, *c.dims[1:])
    many = c.run()
    for n in alone:
        ref.check(n, host(alone[n]), want, dtype)
        ref.check(n, host(many[n][17:18]), want, dtype)
        assert torch.equal(many[n][0], many[n][63]), n


def test_rows_far_apart():
    """Tokens 2^23 elements apart: 5 GB of rows, of which the values are a part."""
    c = Case(7, "bf16", 1, 300, 1, 1, 32, 16)
    x, more = c.inputs()
    big = torch.empty(1, 300, 1 << 23, dtype=torch.bfloat16, device=DEV)
    v = big[..., -16:].unflatten(-1, (1, 16))
    v.copy_(x[2])
    out, _, _ = c.outputs()
    la.la_delta_fwd(x[0], x[1], v, x[3], x[4], **out, **more)
    want = c.want(back=False)
    for n, t in out.items():
        ref.check(n, host(t), want, "bf16")
    wide = torch.empty(1, 300, (1 << 23) + 8, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(la.LaError):
        la.la_delta_fwd(x[0], x[1], wide[..., :16].unflatten(-1, (1, 16)), x[3], x[4], **out, **more)


def test_two_calls_at_once_on_two_streams():
    c, d = Case(8, "bf16", 2, 400, 2, 1, 64, 64), Case(9, "bf16", 2, 400, 2, 1, 64, 64)
    a, b = c.run(), d.run()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for case, stream in ((c, s), (d, t)):
        with torch.cuda.stream(stream):
            x, more = case.inputs()
            out, grads, dh0 = case.outputs()
            do, dh1 = case.d.dev(case.do), case.d.dev(case.dh1, True)
            ws = la.la_delta_fwd(*x, **out, **more, keep=True)
            la.la_delta_bwd(*x, do, **grads, **more, dh1=dh1, dh0=dh0, fwd_ws=ws)
            got.append({**out, **grads, "dh0": dh0})
    torch.cuda.synchronize()
    for want, have in zip((a, b), got):
        for n in want:
            assert torch.equal(want[n], have[n]), n

