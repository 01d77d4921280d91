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
