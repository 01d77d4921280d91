"""What the forward of the gated delta rule does with values at the ends of the range: outputs that cancel, and values that are no
finite numbers, in each of its ways through a sequence."""
import numpy as np
import pytest
import torch

import paper_2006_16236_amd as la
from gpu_util import DEV
from test_gpu_delta import Case
from test_gpu_layer import TYPES, host

pytestmark = pytest.mark.gpu

WAYS = [  # B, N, H, Hk, D, M, keep
    (3, 9, 2, 1, 64, 32, False), (2, 33, 2, 2, 32, 256, False), (2, 64, 1, 1, 128, 144, False), (1, 60, 2, 1, 64, 80, True), (2, 150, 2, 1, 128, 64, True),
    (300, 70, 1, 1, 32, 16, False), (1, 1100, 2, 1, 64, 48, False), (1, 1100, 1, 1, 128, 64, True), (1, 1100, 1, 1, 32, 32, True)]


def pieces(dims, dtype, keep):
    """Whether the call cuts its sequences: the workspace then holds more than its matrices, gates and what is kept."""
    B, N, H, Hk, D, M = dims
    C, tri = (32, 32 * 32) if dtype == "f32" else (64, 96 * 32)
    units, up = B * H * -(-N // C), lambda n: -(-n // 256) * 256
    whole = up(units * 2 * tri * 4) + up(units * 4 * C * 4) + (up(units * C * M * 4) + up(units * D * M * 4) if keep else 0)
    return la.la_delta_fwd_workspace(B, N, H, Hk, D, M, 0 if dtype == "f32" else 1, 1 if keep else 0) > whole


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("way", WAYS, ids=lambda w: "x".join(map(str, w)))
def test_outputs_that_cancel(way, dtype):
    """Keys that are unit vectors, queries alike, strengths of one: a token's output is its value, whatever the state held: o = S + (v - S), S up to 2^17
    and v about 1.  The products with zeros and ones are exact; a token rounds where it is compared with the state (one), where earlier tokens of the
    chunk with the same key are taken off (three part products, a difference), where a written value is added to S (three part products for each
    of at most two such tokens) and once where the next chunk starts: at most 16 roundings of 2^-23 (a matrix instruction's sum need not round to the
    nearest) of 2^17, and the result's own."""
    B, N, H, Hk, D, M, keep = way
    assert pieces(way[:6], dtype, keep) == (N == 1100)
    rng = np.random.default_rng(D + N)
    k = np.zeros((B, N, Hk, D), dtype=np.float32)
    k[:, np.arange(N), :, np.arange(N) % D] = 1.0
    k = torch.from_numpy(k).to(DEV, TYPES[dtype])
    v = torch.from_numpy(rng.uniform(-2, 2, (B, N, H, M)).astype(np.float32)).to(DEV, TYPES[dtype])
    h0 = torch.from_numpy((rng.uniform(2.0 ** 16, 2.0 ** 17, (B, H, D, M)) * rng.choice((-1.0, 1.0), (B, H, D, M))).astype(np.float32)).to(DEV)
    o, h1 = torch.full_like(v, float("nan")), torch.full_like(h0, float("nan"))
    la.la_delta_fwd(k, k, v, None, torch.ones(B, N, H, device=DEV), o, h0=h0, h1=h1, scale=1.0, keep=keep)
    room = 16 * 2.0 ** -23 * 2.0 ** 17
    half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    off = np.abs(host(o) - host(v))
    assert (off <= room + half * (2 + room)).all(), off.max()
    want = host(h0)
    for t in range(N):
        want[:, :, t % D] = host(v[:, t])
    assert np.abs(host(h1) - want).max() <= room
