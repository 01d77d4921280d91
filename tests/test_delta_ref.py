"""The fp64 reference of the gated delta rule and of the head norm: against autograd, against differences, and its bounds
against a reference that rounds what must not be rounded."""
import numpy as np
import pytest
import torch

import delta_ref as ref


def inputs(seed, B, N, H, Hk, D, M):
    rng = np.random.default_rng(seed)
    q, k = (x / np.sqrt((x * x).sum(-1, keepdims=True)) for x in rng.standard_normal((2, B, N, Hk, D)))
    v, do = rng.standard_normal((2, B, N, H, M))
    g = -np.exp(rng.uniform(-6, 0.5, (B, N, H)))
    beta = rng.uniform(0.0, 1.0, (B, N, H))
    h0, dh1 = 0.3 * rng.standard_normal((2, B, H, D, M))
    return dict(q=q, k=k, v=v, g=g, beta=beta, h0=h0), dict(do=do, dh1=dh1)


def test_delta_gradients_are_those_of_autograd():
    x, up = inputs(1, 2, 13, 4, 2, 5, 3)
    lengths, scale = np.array([13, 6]), 0.7
    want = ref.delta(**x, lengths=lengths, scale=scale, **up)
    t = {n: torch.tensor(a, requires_grad=True) for n, a in x.items()}
    loss = 0.0
    for b in range(2):
        for h in range(4):
            S = t["h0"][b, h]
            for i in range(lengths[b]):
                q, k = t["q"][b, i, h // 2], t["k"][b, i, h // 2]
                S = torch.exp(t["g"][b, i, h]) * S
                S = S + t["beta"][b, i, h] * torch.outer(k, t["v"][b, i, h] - S.T @ k)
                o = scale * S.T @ q
                assert np.abs(o.detach().numpy() - want["o"][b, i, h]).max() < 1e-13
                loss = loss + (o * torch.tensor(up["do"][b, i, h])).sum()
            assert np.abs(S.detach().numpy() - want["h1"][b, h]).max() < 1e-13
            loss = loss + (S * torch.tensor(up["dh1"][b, h])).sum()
    loss.backward()
    for n, a in t.items():
        got = want["dh0" if n == "h0" else "d" + n]
        assert np.abs(a.grad.numpy() - got).max() < 1e-12, n


def test_delta_gradients_are_differences():
    x, up = inputs(2, 1, 7, 2, 1, 4, 3)
    want = ref.delta(**x, scale=1.3, **up)

    def loss(**changed):
        r = ref.delta(**{**x, **changed}, scale=1.3)
        return (r["o"] * up["do"]).sum() + (r["h1"] * up["dh1"]).sum()

    rng = np.random.default_rng(3)
    for n in x:
        way = rng.standard_normal(x[n].shape)
        step = 1e-5
        got = (loss(**{n: x[n] + step * way}) - loss(**{n: x[n] - step * way})) / (2 * step)
        assert abs(got - (want["dh0" if n == "h0" else "d" + n] * way).sum()) < 1e-7, n


def test_a_state_handed_on_is_the_uncut_sequence():
    x, up = inputs(3, 2, 20, 2, 2, 4, 5)
    whole = ref.delta(**x, **up)
    a = {n: t[:, :9] for n, t in x.items() if n != "h0"}
    b = {n: t[:, 9:] for n, t in x.items() if n != "h0"}
    first = ref.delta(**a, h0=x["h0"])
    second = ref.delta(**b, h0=first["h1"], do=up["do"][:, 9:], dh1=up["dh1"])
    back = ref.delta(**a, h0=x["h0"], do=up["do"][:, :9], dh1=second["dh0"])
    assert np.allclose(np.concatenate((first["o"], second["o"]), 1), whole["o"], atol=1e-13)
    for n in ("dq", "dk", "dv", "dg", "dbeta"):
        assert np.allclose(np.concatenate((back[n], second[n]), 1), whole[n], atol=1e-12), n
    assert np.allclose(back["dh0"], whole["dh0"], atol=1e-12)


@pytest.mark.parametrize("N", [20, 100, 300])
def test_the_bounds_refuse_states_in_bf16(N):
    """A state rounded to bf16 once in 64 tokens (or at the end) is outside the bounds of o and h1; one in fp32 inside."""
    from layer_ref import to_bf16
    x, _ = inputs(4, 1, N, 2, 1, 32, 16)
    x["h0"] = to_bf16(x["h0"]).astype(np.float64)          # the first state is one in bf16
    want = ref.delta(**x)
    for rounded in (False, True):
        cut = to_bf16 if rounded else (lambda s: s.astype(np.float32))
        S, o = cut(x["h0"]), []
        for at in range(0, N, 64):
            r = ref.delta(**{n: t[:, at:at + 64] for n, t in x.items() if n != "h0"}, h0=S)
            S = cut(r["h1"])
            o.append(r["o"])
        for name, got in (("o", np.concatenate(o, 1)), ("h1", S)):
            if rounded and (name == "h1" or N > 64):
                with pytest.raises(AssertionError, match="times the bound"):
                    ref.check(name, got, want, "f32")
            else:
                ref.check(name, got if rounded else got.astype(np.float32), want, "f32")


@pytest.mark.parametrize("kind", ["rms", "l2", None])
@pytest.mark.parametrize("adjacent", [False, True])
def test_qk_gradients_are_those_of_autograd(kind, adjacent):
    rng = np.random.default_rng(5)
    x, dy, w = rng.standard_normal((2, 5, 3, 24)), rng.standard_normal((2, 5, 3, 24)), 1 + 0.2 * rng.standard_normal(24)
    freq, pos, lengths = 10000.0 ** (-np.arange(8) / 8), rng.integers(-50, 100000, (2, 5)), np.array([5, 2])
    want = ref.qk(x, w, freq, pos, lengths, kind, adjacent, 1e-6, dy)
    tx, tw = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    squares = (tx * tx).sum(-1, keepdim=True)
    n = tx * tw * (1.0 if kind is None else torch.rsqrt((squares / 24 if kind == "rms" else squares) + 1e-6))
    z = torch.polar(torch.ones(2, 5, 1, 8, dtype=torch.float64), torch.tensor(pos[..., None, None] * freq))
    a, b = (n[..., 0:16:2], n[..., 1:16:2]) if adjacent else (n[..., :8], n[..., 8:16])
    turned = torch.complex(a, b) * z
    y = torch.cat((torch.stack((turned.real, turned.imag), -1).flatten(-2) if adjacent else torch.cat((turned.real, turned.imag), -1), n[..., 16:]), -1)
    y = torch.where(torch.tensor(np.arange(5)[None] < lengths[:, None])[..., None, None], y, 0.0)
    assert np.abs(y.detach().numpy() - want["y"]).max() < 1e-10
    y.backward(torch.tensor(dy))
    assert np.abs(tx.grad.numpy() - want["dx"]).max() < 1e-10 and np.abs(tw.grad.numpy() - want["dw"]).max() < 1e-9
    # differences
    way, step = rng.standard_normal(x.shape), 1e-6
    loss = lambda t: (ref.qk(t, w, freq, pos, lengths, kind, adjacent, 1e-6)["y"] * dy).sum()  # noqa: E731
    assert abs((loss(x + step * way) - loss(x - step * way)) / (2 * step) - (want["dx"] * way).sum()) < 1e-6
