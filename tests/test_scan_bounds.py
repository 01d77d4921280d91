"""The element-wise bounds of scan_bounds.py, on the CPU: their values are those of the fp64 reference, fp32 arithmetic keeps
to them, and states or gradients held in bf16 do not, at any size that the GPU tests hold to them."""
import numpy as np
import pytest
import torch

import layer_ref as ref
import scan_bounds
from test_gpu_layer import scan_data
from test_gpu_scan_pieces import BOUNDED, bounded_data, case_id, pieces_of

SMALL = [(2, 9, 6, 2, 8, [9, 4], True, True, True, True), (1, 20, 5, 1, 8, None, False, False, False, False), (2, 7, 70, 1, 16, [0, 7], True, True, True, True)]


@pytest.mark.parametrize("case", SMALL)
def test_values_are_those_of_the_reference(case):
    *_, softplus = case
    _, a = scan_data(*case, "f32")
    want = ref.scan(**a, softplus=softplus)
    for name, (value, bound) in scan_bounds.scan(**a, softplus=softplus).items():
        assert np.allclose(value, want[name], rtol=1e-10, atol=1e-12), name
        assert (bound >= 0).all() and bound.shape == value.shape, name


def f32_scan(a, piece):
    """The forward in fp32, token by token, or from the states of pieces of `piece` tokens."""
    t = {n: torch.from_numpy(v) for n, v in a.items() if n != "lengths" and v is not None}
    B, N, E = t["x"].shape
    G, S = t["Bt"].shape[2:]
    raw = t["dt"] + t["dt_bias"]
    d = raw.clamp(min=0) + torch.log1p(torch.exp(-raw.abs()))
    w, A = d * t["x"], t["A"] * np.float32(1.44269504)
    chan = lambda v, i: v[:, i].repeat_interleave(E // G, 1)

    def run(h, lo, hi, y=None):
        for i in range(lo, hi):
            h = torch.exp2(d[:, i, :, None] * A) * h + w[:, i, :, None] * chan(t["Bt"], i)
            if y is not None:
                y[:, i] = ((h * chan(t["Ct"], i)).sum(-1) + t["D"] * t["x"][:, i]) * (t["z"][:, i] * torch.sigmoid(t["z"][:, i]))
        return h

    y, h = torch.empty_like(t["x"]), t["h0"]
    for lo in range(0, N, piece):
        hi = min(lo + piece, N)
        run(h, lo, hi, y)
        h = torch.exp2(d[:, lo:hi].sum(1)[..., None] * A) * h + run(torch.zeros_like(h), lo, hi) if piece < N else run(h, lo, hi)
    return y.numpy(), h.numpy()


@pytest.mark.parametrize("piece", [1 << 20, 64])
def test_fp32_keeps_to_the_bounds(piece):
    _, a = scan_data(2, 300, 20, 1, 16, None, True, True, True, True, "f32")
    a["A"] /= 16                                                                   # states that outlive a piece
    pieces = 1 if piece > 300 else -(-300 // piece)
    got = f32_scan(a, piece)
    bound = scan_bounds.scan(**{**a, "dy": None, "dh1": None}, pieces=(pieces, pieces))
    for name, v in zip(("y", "h1"), got):
        ref.check(name, v, *bound[name], "f32", 1)


@pytest.mark.parametrize("case", BOUNDED, ids=case_id)
def test_states_in_bf16_exceed_the_bounds(case):
    """Rounded only behind every 16th token (of a sequence of no more, behind each); gradients of states likewise, backwards.
    Outputs rounded to bf16 themselves hide it: there the final state and its gradient show it."""
    a, pieces, every = bounded_data(case), pieces_of(*case[:5]), 16 if case[1] > 16 else 1
    softplus, dtype = case[6:8]
    right = scan_bounds.scan(**a, softplus=softplus, pieces=pieces)
    bf16 = lambda v: v.to(torch.bfloat16).double()
    for change, outputs, final in ((dict(touch=lambda h, t: bf16(h) if (t + 1) % every == 0 else h), ("y",), "h1"),
                                   (dict(touch_grad=lambda g, t: bf16(g) if t % every == 0 else g), ("dx",), "dh0")):
        got = scan_bounds.scan(**a, softplus=softplus, pieces=pieces, **change)
        for name in (*(outputs if dtype == "f32" and case[1] > 1 else ()), final):
            with pytest.raises(AssertionError, match=f"{name}: .* times the bound"):
                ref.check(name, got[name][0], *right[name], "f32", 1)
