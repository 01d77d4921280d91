"""Sequences that the gated delta rule cuts into pieces, as calls make them: without states, without a decay, parts of wider rows, the
backward that forms the forward again, values behind a sequence and behind a token.  Each asserts that its sizes are cut."""
import numpy as np
import pytest
import torch

import paper_2006_16236_amd as la
from gpu_util import DEV
from test_gpu_delta import Case
from test_gpu_delta_values import pieces
from test_gpu_layer import host

pytestmark = pytest.mark.gpu

SIZES = [  # B, N, H, Hk, D, M, lengths
    (1, 1100, 1, 1, 64, 48, None), (1, 1101, 2, 1, 128, 64, None), (1, 1100, 2, 2, 32, 32, None), (2, 1300, 2, 1, 64, 80, [1300, 517]),
    (3, 1200, 1, 1, 128, 16, [0, 1200, 90]), (4, 900, 2, 1, 32, 144, [900, 1, 300, 899])]
ids = dict(ids=lambda c: "x".join(map(str, c[:6])))


def case(seed, dtype, size, **more):
    c = Case(seed, dtype, *size, **more)
    assert pieces(size[:6], dtype, False) and pieces(size[:6], dtype, True)
    return c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("state,decay,wider", [(False, True, 0), (True, False, 16), (False, False, 8)])
@pytest.mark.parametrize("size", SIZES, **ids)
def test_without_states_or_a_decay(size, state, decay, wider, dtype):
    case(31, dtype, size, state=state, decay=decay, wider=wider).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("size", SIZES, **ids)
def test_a_backward_without_the_forwards_workspace_is_the_same(size, state, dtype):
    c = case(32, dtype, size, state=state, decay=state)
    a, b = c.run(), c.run(given=False)
    for n in a:
        assert a[n] is None and b[n] is None or torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 1e30])
def test_outputs_before_a_token_do_not_depend_on_it(dtype, bad):
    c = case(33, dtype, (1, 1100, 2, 1, 64, 48))
    clean = c.run(back=False)["o"]
    for at in (3, 64, 500, 777, 1099):
        for what in ("q", "k", "v", "g", "beta"):
            x, more = c.inputs()
            x["qkvgb".index(what[0])][0, at:] = bad
            out, _, _ = c.outputs()
            la.la_delta_fwd(*x, **out, **more)
            assert torch.equal(out["o"][:, :at], clean[:, :at]), (what, at)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [s for s in SIZES if s[6]], **ids)
def test_rows_behind_a_sequence_may_hold_anything(size, dtype):
    c = case(34, dtype, size)
    a = c.run()
    for t in (c.q, c.k, c.v, c.do, c.g, c.beta):
        for b, n in enumerate(c.lengths):
            t[b, n:] = np.nan
    b, again = c.run(), c.run(given=False)
    for n in a:
        assert torch.equal(a[n], b[n]) and torch.equal(a[n], again[n]), n
    for n in ("o", "dq", "dk", "dv", "dg", "dbeta"):
        for i, end in enumerate(c.lengths):
            assert not host(b[n])[i, end:].any(), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_training_step_in_a_graph(dtype):
    """Replays with other lengths in the same place: other pieces take part."""
    size = SIZES[3]
    c = case(35, dtype, size)
    x, more = c.inputs()
    do, dh1 = c.d.dev(c.do), c.d.dev(c.dh1, True)
    out, grads, dh0 = c.outputs()
    B, N, H, Hk, D, M = c.dims
    code = 0 if dtype == "f32" else 1
    ws = torch.empty(la.la_delta_fwd_workspace(B, N, H, Hk, D, M, code, 1), dtype=torch.uint8, device=DEV)
    wb = torch.empty(la.la_delta_bwd_workspace(B, N, H, Hk, D, M, code, 1), dtype=torch.uint8, device=DEV)

    def step():
        la.la_delta_fwd(*x, **out, **more, keep=True, ws=ws)
        la.la_delta_bwd(*x, do, **grads, **more, dh1=dh1, dh0=dh0, fwd_ws=ws, ws=wb)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lengths in ([1300, 517], [70, 1300], [0, 1290], [1300, 517]):
        more["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
        c.lengths = np.asarray(lengths, dtype=np.int32)
        want = c.run()
        for t in (*out.values(), *grads.values(), dh0):
            t.fill_(float("nan"))
        ws.fill_(255), wb.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for n, t in {**out, **grads, "dh0": dh0}.items():
            assert torch.equal(t, want[n]), (lengths, n)
