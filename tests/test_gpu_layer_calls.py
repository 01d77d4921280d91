"""Calls of the norm, convolution and scan as a program around them makes them: parts of its tensors, states it goes on using."""
import pytest
import torch

import paper_2006_16236_amd as la
from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("part", [lambda n: n[1:], lambda n: n[::2], lambda n: n[:1].expand(3)])
def test_lengths_are_a_part_of_a_batchs_lengths(part):
    """Like every other tensor of these functions: a slice (off 16 bytes), a strided one and a broadcast one."""
    B, N, E, S, W = 3, 21, 40, 8, 3
    lengths = part(torch.tensor([7, 21, 0, 12, 3, 1], dtype=torch.int32, device=DEV))[:B]
    dense = lengths.clone(memory_format=torch.contiguous_format)
    leaf = lambda *s: torch.randn(*s, device=DEV).requires_grad_(True)
    x, w, dt, A, Bt = leaf(B, N, E), leaf(E, W), leaf(B, N, E), -torch.rand(E, S, device=DEV), leaf(B, N, 1, S)

    def run(n):
        c, _ = la.causal_conv(x, w, lengths=n)
        y, h = la.selective_scan(c, dt, A, Bt, Bt, lengths=n)
        return y, h, *torch.autograd.grad(y.square().sum() + h.sum(), (x, w, dt, Bt))

    for got, want in zip(run(lengths), run(dense)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("given_stream", [False, True])
def test_a_state_stepped_on_before_its_backward_is_noticed(given_stream):
    """The gradients would be those of another state: an error, as with torch's own operations in place.  Both ways of a call."""
    B, N, E, S, W = 2, 9, 40, 8, 4
    kw = {"stream": torch.cuda.current_stream()} if given_stream else {}
    rand = lambda *s: torch.randn(*s, device=DEV)
    x, w, A, Bt = rand(B, N, E), rand(E, W).requires_grad_(True), -torch.rand(E, S, device=DEV), rand(B, N, 1, S)
    one, bc, out = rand(B, E), rand(B, 1, S), torch.empty(B, E, device=DEV)
    c0, h0 = rand(B, W - 1, E), rand(B, E, S)
    y, c1 = la.causal_conv(x, w, state=c0)
    y, h1 = la.selective_scan(y, x, A, Bt, Bt, state=h0)
    la.la_conv_step(one, w.detach(), None, c1.detach(), out, **kw)                # the states handed on may be stepped on
    la.la_scan_step(one, one, A, bc, bc, h1.detach(), out, **kw)
    want = torch.autograd.grad(y.sum(), w, retain_graph=True)
    for step in (lambda: la.la_conv_step(one, w.detach(), None, c0, out, **kw), lambda: la.la_scan_step(one, one, A, bc, bc, h0, out, **kw)):
        c0, h0 = rand(B, W - 1, E), rand(B, E, S)
        y = la.selective_scan(la.causal_conv(x, w, state=c0)[0], x, A, Bt, Bt, state=h0)[0]
        step()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    assert torch.isfinite(want[0]).all() and w.grad is None


@pytest.mark.parametrize("given_stream", [False, True])
def test_every_written_tensor_counts_as_changed_once(given_stream):
    B, N, E, S, W = 2, 9, 40, 8, 4
    kw = {"stream": torch.cuda.current_stream()} if given_stream else {}
    new = lambda *s: torch.zeros(*s, device=DEV)
    x, g, st, w, c, A, Bt, h = new(B, N, E), new(E), new(B, N), new(E, W), new(B, W - 1, E), new(E, S), new(B, N, 1, S), new(B, E, S)
    inputs = (x, g, st, w, c, A, Bt, h)
    before = [t._version for t in inputs]

    def check(call, *outs):
        seen = [t._version for t in outs]
        call()
        assert [t._version - v for t, v in zip(outs, seen)] == [1] * len(outs)

    o = [new(B, N, E) for _ in range(4)]
    a, b, m, r = new(E), new(E), new(B, N), new(B, N)
    check(lambda: la.la_norm_fwd(x, g, g, o[0], m, r, r=x, s=o[1], **kw), o[0], m, r, o[1])
    check(lambda: la.la_norm_fwd(x, g, g, o[0], **kw), o[0])
    check(lambda: la.la_norm_bwd(x, g, st, st, x, o[0], a, b, **kw), o[0], a, b)
    check(lambda: la.la_norm_bwd(x, g, st, st, x, o[0], **kw), o[0])              # not taken by the native path
    c1, dw = new(B, W - 1, E), new(E, W)
    check(lambda: la.la_conv_fwd(x, w, g, o[0], x0=c, x1=c1, **kw), o[0], c1)
    check(lambda: la.la_conv_bwd(x, w, g, x, o[0], dw, a, x0=c, dx0=c1, **kw), o[0], dw, a, c1)
    one, bc, y = new(B, E), new(B, 1, S), new(B, E)
    check(lambda: la.la_conv_step(one, w, g, c1, y, **kw), c1, y)
    h1, dA, dB, dC = new(B, E, S), new(E, S), new(B, N, 1, S), new(B, N, 1, S)
    check(lambda: la.la_scan_fwd(x, x, A, Bt, Bt, o[0], z=x, h0=h, h1=h1, keep=True, **kw), o[0], h1)
    ws = la.la_scan_fwd(x, x, A, Bt, Bt, o[0], z=x, keep=True)
    check(lambda: la.la_scan_bwd(x, x, A, Bt, Bt, x, o[0], o[1], dA, dB, dC, D=g, z=x, dt_bias=g, dD=a, dz=o[2], ddt_bias=b, h0=h, dh0=h1, fwd_ws=ws, **kw),
          o[0], o[1], dA, dB, dC, a, o[2], b, h1)
    check(lambda: la.la_scan_step(one, one, A, bc, bc, h1, y, z=one, **kw), h1, y)
    assert [t._version for t in inputs] == before
    with torch.inference_mode():                                                   # tensors that count nothing
        n = torch.zeros(4, E, device=DEV)
        out = torch.empty_like(n)
        la.la_norm_fwd(n, None, None, out, **kw)
        la.la_conv_step(n[:B].clone(), w, g, torch.zeros(B, W - 1, E, device=DEV), out[:B], **kw)
