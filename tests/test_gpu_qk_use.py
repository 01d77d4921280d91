"""The head norm's front end."""
import pytest
import torch

import paper_2006_16236_amd as la
from gpu_util import DEV
from test_gpu_layer import Data

pytestmark = pytest.mark.gpu


def test_a_weight_for_keys_that_are_not_there_has_no_gradient():
    d = Data(1, "f32")
    q, wq, wk = (d.dev(d.array(*s), True).requires_grad_(True) for s in ((2, 5, 3, 32), (32,), (32,)))
    y = la.qk_norm(q, wq=wq, wk=wk)
    y.sum().backward()
    assert wk.grad is None
    want = torch.autograd.grad(la.qk_norm(q, wq=wq).sum(), (q, wq))
    assert torch.equal(q.grad, want[0]) and torch.equal(wq.grad, want[1])
