"""The head norm's front end and the two front ends together in bf16, and the head norm where few heads meet many tokens."""
import numpy as np
import pytest
import torch

import delta_ref as ref
import paper_2006_16236_amd as la
import test_gpu_qk as qk
from gpu_util import DEV
from layer_ref import check
from test_gpu_layer import Data, host

pytestmark = pytest.mark.gpu


def test_a_weight_for_keys_that_are_not_there_has_no_gradient():
    d = Data(1, "f32")
    q, wq, wk = (d.dev(d.array(*s), True).requires_grad_(True) for s in ((2, 5, 3, 32), (32,), (32,)))
    y = la.qk_norm(q, wq=wq, wk=wk)
    y.sum().backward()
    assert wk.grad is None
    want = torch.autograd.grad(la.qk_norm(q, wq=wq).sum(), (q, wq))
    assert torch.equal(q.grad, want[0]) and torch.equal(wq.grad, want[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", [  # few heads: most of a wave's places for heads stay empty
    (1, 16400, 1, 1, 32, 32, "rms", True, False, None, 8, True), (2, 8197, 1, 0, 64, 64, "l2", True, True, [8197, 5000], 0, False),
    (1, 12001, 4, 1, 64, 32, "rms", True, False, None, 16, False), (3, 4099, 3, 1, 48, 16, "l2", False, False, [4099, 0, 1], 0, True),
    (1, 9001, 1, 1, 8, 8, "rms", True, False, None, 0, True)], ids=lambda c: "x".join(str(i) for i in c[:6]))
def test_few_heads_of_many_tokens(case, dtype):
    qk.test_qk(case, dtype)


@pytest.mark.parametrize("N,lengths", [(1, None), (64, [64, 20]), (150, [131, 150]), (700, None)])
def test_both_front_ends_and_their_gradients_in_bf16(N, lengths):
    """Parts of one projection through qk_norm and gated_delta: each one's outputs and gradients against fp64, from the other's bf16 results."""
    B, H, Hk, D, M, R = 2, 4, 2, 32, 48, 16
    d = Data(N, "bf16")
    wide = d.dev(d.array(B, N, 2 * Hk * D + H * M, scale=1.5)).requires_grad_(True)
    q, k, v = wide.split((Hk * D, Hk * D, H * M), -1)
    q, k, v = q.unflatten(-1, (Hk, D)), k.unflatten(-1, (Hk, D)), v.unflatten(-1, (H, M))
    wq, wk = (d.dev(1 + d.array(D, scale=0.2, f32=True), True).requires_grad_(True) for _ in range(2))
    g, beta = (d.dev(t.astype(np.float32), True).requires_grad_(True) for t in (-np.exp(d.rng.uniform(-7, 1, (B, N, H))), d.rng.uniform(0, 1, (B, N, H))))
    h0 = d.dev(d.array(B, H, D, M, scale=0.3, f32=True), True).requires_grad_(True)
    freq = (100.0 ** (-np.arange(R // 2) / (R // 2))).astype(np.float32)
    pos = d.rng.integers(0, 5000, (B, N)).astype(np.int32)
    ends = None if lengths is None else np.asarray(lengths, dtype=np.int32)
    dev = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
    u, w = la.qk_norm(q, k, wq, wk, dev(freq), dev(pos), dev(ends), norm="l2")
    u.retain_grad(), w.retain_grad(), v.retain_grad()
    o, h1 = la.gated_delta(u, w, v, g, beta, state=h0, lengths=dev(ends))
    do, dh1 = d.array(B, N, H, M), d.array(B, H, D, M, f32=True)
    ((o * d.dev(do)).sum(dtype=torch.float32) + (h1 * d.dev(dh1, True)).sum()).backward()
    want = ref.delta(host(u), host(w), host(v), host(g), host(beta), host(h0), ends, D ** -0.5, do, dh1)
    for name, got in (("o", o), ("h1", h1), ("dq", u.grad), ("dk", w.grad), ("dv", v.grad), ("dg", g.grad), ("dbeta", beta.grad), ("dh0", h0.grad)):
        ref.check(name, host(got), want, "bf16")
    dq, dk, dv = host(wide.grad).reshape(B * N, -1)[:, :Hk * D], host(wide.grad).reshape(B * N, -1)[:, Hk * D:2 * Hk * D], host(wide.grad)[..., 2 * Hk * D:]
    assert np.array_equal(dv.reshape(B, N, H, M), host(v.grad))
    for x, y, weight, dx, dw in ((q, u, wq, dq, wq.grad), (k, w, wk, dk, wk.grad)):
        args = (host(x), host(weight), freq, pos, ends, "l2", False, 1e-6, host(y.grad))
        exact, mag = ref.qk(*args), ref.qk(*args, mag=True)
        check("y", host(y), exact["y"], mag["y"], "bf16", 20)            # the counts of the head norm's own test
        check("dx", dx.reshape(B, N, Hk, D), exact["dx"], mag["dx"], "bf16", 54)
        check("dw", host(dw), exact["dw"], mag["dw"], "f32", 2 * 20 + 64 + 80 + 2 * (Hk * D / 512 + 1))
