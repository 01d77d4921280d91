"""The scan of sequences that are cut into pieces, whose states are formed side by side and then carried from piece to piece."""
import numpy as np
import pytest
import torch

import layer_ref as ref
import paper_2006_16236_amd as la
from gpu_util import DEV

pytestmark = pytest.mark.gpu


def pieces_of(B, N, E, G, S):
    """Pieces of the forward and of the backward, as their workspaces show them: a state and a sum of steps for each piece
    (rounded up to 256 bytes each); backward also the kept states, channel blocks' dB and dC, and sums for each piece."""
    up = lambda n: -(-n // 256) * 256
    room = lambda p: 0 if p < 2 else up(B * E * S * 4 * p) + up(B * p * E * 4)
    tiles, blocks = -(-N // 16), G * -(-(E // G) // 64)
    fwd, bwd = la.la_scan_fwd_workspace(B, N, E, G, S, 0, 1), la.la_scan_bwd_workspace(B, N, E, G, S, 0, 3)
    found = [p for p in range(1, tiles + 1) if room(p) == fwd]
    back = [p for p in range(1, tiles + 1) if room(p) + up(blocks * B * N * 2 * S * 4) + up(B * p * E * (S + 2) * 4) == bwd]
    assert len(found) == len(back) == 1
    return found[0], back[0]


def test_decays_of_a_piece_beyond_the_range_of_fp32():
    """exp(A sum d) over a piece: infinite before a state (backwards: a gradient) that is still zero, zero behind a state
    that is large enough to survive it.  Steps given as they are, so A is what a state grows or falls by at each token."""
    B, N, E, S, some = 1, 512, 64, 8, 20
    assert min(pieces_of(B, N, E, 1, S)) > 2
    r = np.random.default_rng(11)
    a = {n: r.standard_normal((B, N, E)).astype(np.float32) for n in ("x", "dy")}
    a.update({n: r.standard_normal((B, N, 1, S)).astype(np.float32) for n in ("Bt", "Ct")}, dt=np.ones((B, N, E), np.float32))
    a["A"] = np.tile(np.array([2, -2, -1.5, 0.01, 1.5, -0.01, 0, -1], np.float32), (E, 1))
    a["x"][:, :N - some] = 0                                       # growth by exp(2 * 20) of what enters near the end,
    a["dy"][:, some:] = 0                                          # and of the gradient that enters near the start
    a["dy"] *= 0.1
    a["h0"] = np.zeros((B, E, S), np.float32)
    a["h0"][:, :, 2] = 1e34                                        # exp(-1.5 * 64) 1e34 is 2e-8
    t = {n: torch.from_numpy(v).to(DEV) for n, v in a.items()}
    o = {n: torch.empty_like(t[m]) for n, m in (("y", "x"), ("dx", "x"), ("ddt", "x"), ("dA", "A"), ("dB", "Bt"), ("dC", "Ct"), ("h1", "h0"), ("dh0", "h0"))}
    args = (t["x"], t["dt"], t["A"], t["Bt"], t["Ct"])
    ws = la.la_scan_fwd(*args, o["y"], h0=t["h0"], h1=o["h1"], softplus=False, keep=True)
    la.la_scan_bwd(*args, t["dy"], o["dx"], o["ddt"], o["dA"], o["dB"], o["dC"], h0=t["h0"], dh0=o["dh0"], softplus=False, fwd_ws=ws)
    want, mag = (ref.scan(**a, softplus=False, mag=m) for m in (False, True))
    # |A| <= 2 and steps of 1: the exponent of a piece is off by its sum's roundings too, at most one for each of its tokens
    k = ref.roundings(N, S, a["A"], 1.0) + 2 * N
    for n in o:
        ref.check(n, o[n].double().cpu().numpy(), want[n], mag[n] + 1e-30, "f32", 2 * k + E)


# Against bounds that follow the recurrence (scan_bounds.py).  B, N, E, G, S, lengths, softplus, dtype, slow: how much slower than
# 1 to S the states fall.  The pieces' states are carried from piece to piece 16 at a time: exactly one batch, one piece more,
# two, and three with one that is not full; lengths that end in different batches; both widths of a workgroup forwards.
BOUNDED = [
    (1, 1, 3, 1, 8, None, True, "f32", 1), (2, 16, 63, 1, 16, [16, 3], True, "f32", 1), (3, 17, 130, 2, 8, [0, 17, 16], True, "bf16", 1),
    (1, 33, 96, 4, 16, None, False, "f32", 1), (1, 200, 64, 1, 32, None, True, "f32", 4), (2, 300, 72, 2, 16, [300, 77], True, "bf16", 4),
    (70, 35, 250, 1, 16, None, True, "f32", 1), (66, 18, 130, 2, 32, [i % 19 for i in range(66)], True, "f32", 1),
    (66, 18, 130, 2, 16, [i % 19 for i in range(66)], True, "bf16", 1), (70, 35, 250, 1, 32, None, True, "bf16", 1),
    (17, 500, 250, 1, 16, [500, 0, 1, 499, 64, 65] + [450 + i for i in range(11)], True, "bf16", 4),
    (17, 500, 250, 1, 32, [500, 0, 1, 499, 64, 65] + [450 + i for i in range(11)], True, "f32", 4),
    (1, 1024, 40, 1, 8, None, True, "f32", 16), (1, 1300, 64, 1, 16, [1281], True, "f32", 16), (2, 2500, 24, 2, 8, [2500, 1100], True, "f32", 16),
    (1, 3001, 40, 1, 8, None, False, "f32", 16), (1, 3001, 20, 1, 32, None, True, "f32", 16), (3, 3001, 20, 1, 16, [3001, 1, 1800], True, "bf16", 16),
]


def case_id(case):
    return "-".join(map(str, case[:5])) + f"-{case[7]}"


def bounded_data(case):
    from test_gpu_layer import scan_data
    B, N, E, G, S, lengths, softplus, dtype, slow = case
    _, a = scan_data(B, N, E, G, S, lengths, True, True, True, softplus, dtype)
    a["A"] = (a["A"] / slow).astype(np.float32)
    return a


def test_the_bounded_scans_have_one_batch_of_pieces_and_more():
    pieces = {(c[1], c[4]): pieces_of(*c[:5]) for c in BOUNDED if c[1] > 1000}
    assert pieces[1024, 8] == (16, 16) and pieces[1300, 16] == (17, 17) and pieces[2500, 8] == (32, 32)
    assert all(min(pieces[3001, S]) > 32 and all(p % 16 for p in pieces[3001, S]) for S in (8, 16, 32))


@pytest.mark.parametrize("case", BOUNDED, ids=case_id)
def test_scan_within_the_bounds_of_its_recurrence(case):
    import scan_bounds
    from test_gpu_layer import Data, scan_on_device
    softplus, dtype = case[6:8]
    a = bounded_data(case)
    o, _ = scan_on_device(Data(0, dtype), a, 0, softplus)
    for name, (want, bound) in scan_bounds.scan(**a, softplus=softplus, pieces=pieces_of(*case[:5])).items():
        kind = dtype if name in ("y", "dx", "ddt", "dz", "dB", "dC") else "f32"
        ref.check(name, o[name].double().cpu().numpy(), want, bound, kind, 1)
