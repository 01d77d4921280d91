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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("way", WAYS, ids=lambda w: "x".join(map(str, w)))
def test_what_is_no_finite_number_shows(way, dtype):
    """In v of one column, in beta of one head, in a key, in a state handed in: outputs from its token on and the state behind have no finite
    value where it reaches, as token by token; all others are as without it."""
    B, N, H, Hk, D, M, keep = way
    c = Case(21, dtype, *way[:6])
    assert pieces(way[:6], dtype, keep) == (N == 1100)
    per, b, col = H // Hk, B - 1, M - 3
    clean = c.run(back=False)
    if keep:
        x, more = c.inputs()
        out, _, _ = c.outputs()
        la.la_delta_fwd(*x, **out, **more, keep=True)
        assert all(torch.equal(out[n], clean[n]) for n in out)
    for bad in (float("nan"), float("inf"), -float("inf")):
        for at in sorted({0, 1, N // 2, N - 1}):
            for what in ("v", "beta", "k", "h0"):
                x, more = c.inputs()
                hit = torch.zeros(B, N, H, M, dtype=torch.bool, device=DEV)
                last = torch.zeros(B, H, D, M, dtype=torch.bool, device=DEV)
                if what == "v":
                    x[2][b, at, H - 1, col] = bad
                    hit[b, at:, H - 1, col] = last[b, H - 1, :, col] = True
                elif what == "beta":
                    x[4][b, at, H - 1] = bad
                    hit[b, at:, H - 1] = last[b, H - 1] = True
                elif what == "k":
                    x[1][b, at, Hk - 1, D // 2] = bad
                    hit[b, at:, H - per:] = last[b, H - per:] = True
                else:
                    more["h0"] = more["h0"].clone()
                    more["h0"][b, H - 1, D - 1, col] = bad
                    hit[b, :, H - 1, col] = last[b, H - 1, :, col] = True
                out, _, _ = c.outputs()
                la.la_delta_fwd(*x, **out, **more, keep=keep)
                where = (what, bad, at)
                assert not out["o"][hit].isfinite().any() and not out["h1"][last].isfinite().any(), where
                assert torch.equal(out["o"][~hit], clean["o"][~hit]) and torch.equal(out["h1"][~last], clean["h1"][~last]), where


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_token_by_itself_shows_it_too(dtype):
    c = Case(22, dtype, 2, 1, 2, 1, 64, 48)
    for bad in (float("nan"), float("inf")):
        for what in range(1, 5):
            x, _ = c.inputs()
            x[what].view(-1)[-1] = bad if what != 3 else float("nan")
            h, o = c.d.dev(c.h0, True), c.d.empty((2, 2, 48))
            la.la_delta_step(*(t[:, 0].contiguous() for t in x), h, o)
            hit = slice(47, 48) if what == 2 else slice(0, 48)
            assert not o[1, 1, hit].isfinite().any() and not h[1, 1, :, hit].isfinite().any(), (bad, what)
