"""Calls whose sums over rows have more columns than one launch has lanes: sizes that the entry points take."""
import pytest
import torch

import paper_2006_16236_amd as la
from gpu_util import DEV

pytestmark = pytest.mark.gpu


def rand(*shape):
    return torch.randn(*shape, device=DEV)


def test_weight_gradients_of_very_many_channels_convolution():
    """E (W + 1) columns in workgroups of 1024 lanes for 64 of them: beyond 2^32 lanes.  One token: a tap's gradient is one
    product, and the bias's is dy itself, to the bit."""
    E, W = 60_000_000, 4
    assert (E * (W + 1) + 63) // 64 * 1024 > 1 << 32
    x, x0, dy, w = rand(1, 1, E), rand(1, W - 1, E), rand(1, 1, E), rand(E, W)
    dx, dw, db = torch.empty_like(x), torch.full_like(w, float("nan")), torch.full((E,), float("nan"), device=DEV)
    la.la_conv_bwd(x, w, None, dy, dx, dw, db, x0=x0, silu=False)
    assert torch.equal(dx[0, 0], dy[0, 0] * w[:, W - 1])
    assert torch.equal(db, dy[0, 0])
    line = torch.cat((x0, x), 1)[0]
    for k in range(W):
        assert torch.equal(dw[:, k], dy[0, 0] * line[k]), k


def test_weight_gradients_of_very_many_channels_scan():
    """E (S + 2) columns likewise.  One token and no gate: dA = d g exp(d A) h0 with g = C dy, dD = dy x, and the
    bias's gradient is that of dt, to the bit."""
    E, S = 8_000_000, 32
    assert (E * (S + 2) + 63) // 64 * 1024 > 1 << 32
    x, dt, dy, h0 = rand(1, 1, E), torch.rand(1, 1, E, device=DEV), rand(1, 1, E), rand(1, E, S)
    A, Bt, Ct = -torch.rand(E, S, device=DEV), rand(1, 1, 1, S), rand(1, 1, 1, S)
    nan = lambda *shape: torch.full(shape, float("nan"), device=DEV)
    y, dx, ddt, dA, dD, db, dB, dC = nan(1, 1, E), nan(1, 1, E), nan(1, 1, E), nan(E, S), nan(E), nan(E), nan(1, 1, 1, S), nan(1, 1, 1, S)
    ws = la.la_scan_fwd(x, dt, A, Bt, Ct, y, h0=h0, softplus=False, keep=True)
    la.la_scan_bwd(x, dt, A, Bt, Ct, dy, dx, ddt, dA, dB, dC, dD=dD, ddt_bias=db, h0=h0, softplus=False, fwd_ws=ws)
    assert torch.equal(dD, dy[0, 0] * x[0, 0])
    assert torch.isfinite(ddt).all() and torch.equal(db, ddt[0, 0])
    d = dt[0, 0].double()[:, None]
    want = d * (dy[0, 0].double()[:, None] * Ct[0, 0].double()) * torch.exp(d * A.double()) * h0[0].double()
    # four products, and an exponential of at most 1 (|d A| <= 1): A log2(e), its product with d and the power, 1 + 1 + 1 + 2 more
    assert ((dA.double() - want).abs() <= 16 * 2.0 ** -24 * want.abs() + 1e-37).all()
