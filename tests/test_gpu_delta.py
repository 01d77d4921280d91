"""Gated delta rule on the GPU against fp64, at sizes and masks where it can go wrong; its states, gradients, streams, graphs."""
import numpy as np
import pytest
import torch

import delta_ref as ref
import paper_2006_16236_amd as la
from gpu_util import DEV
from layer_ref import to_bf16
from test_gpu_layer import Data, host

pytestmark = pytest.mark.gpu


class Case:
    """Inputs of a call: keys of unit length, decays from nearly none to nearly all, strengths from 0 to 1."""

    def __init__(self, seed, dtype, B, N, H, Hk, D, M, lengths=None, state=True, wider=0, decay=True):
        d = self.d = Data(seed, dtype)
        self.dtype, self.dims, self.scale = dtype, (B, N, H, Hk, D, M), D ** -0.5

        def units(*shape):
            t = d.rng.standard_normal(shape)
            t = (t / np.sqrt((t * t).sum(-1, keepdims=True) + 1e-6)).astype(np.float32)
            return t if dtype == "f32" else to_bf16(t)

        self.q, self.k, self.v, self.do = units(B, N, Hk, D), units(B, N, Hk, D), d.array(B, N, H, M), d.array(B, N, H, M)
        self.g = -np.exp(d.rng.uniform(-7, 1, (B, N, H))).astype(np.float32) if decay else None
        self.beta = d.rng.uniform(0, 1, (B, N, H)).astype(np.float32)
        self.h0, self.dh1 = (d.array(B, H, D, M, scale=0.3, f32=True) if state else None for _ in range(2))
        self.lengths = None if lengths is None else np.asarray(lengths, dtype=np.int32)
        self.wider = wider

    def want(self, back=True):
        return ref.delta(self.q, self.k, self.v, self.g, self.beta, self.h0, self.lengths, self.scale, *((self.do, self.dh1) if back else ()))

    def inputs(self):
        d, w = self.d, self.wider
        x = [d.dev(self.q, wider=w), d.dev(self.k, wider=w and w + 24), d.dev(self.v, wider=w and w + 56), d.dev(self.g, True), d.dev(self.beta, True)]
        more = dict(h0=d.dev(self.h0, True), lengths=None if self.lengths is None else torch.from_numpy(self.lengths).to(DEV), scale=self.scale)
        return x, more

    def outputs(self):
        B, N, H, Hk, D, M = self.dims
        d, state = self.d, self.h0 is not None
        return dict(o=d.empty((B, N, H, M)), h1=d.empty((B, H, D, M), True) if state else None), \
            dict(dq=d.empty((B, N, Hk, D)), dk=d.empty((B, N, Hk, D)), dv=d.empty((B, N, H, M)),
                 dg=None if self.g is None else d.empty((B, N, H), True), dbeta=d.empty((B, N, H), True)), d.empty((B, H, D, M), True) if state else None

    def run(self, back=True, given=True, **how):
        x, more = self.inputs()
        out, grads, dh0 = self.outputs()
        ws = la.la_delta_fwd(*x, **out, **more, keep=back and given, **how)
        if back:
            la.la_delta_bwd(*x, self.d.dev(self.do), **grads, **more, dh1=self.d.dev(self.dh1, True), dh0=dh0, fwd_ws=ws if given else None, **how)
            out.update(grads, dh0=dh0)
        torch.cuda.synchronize()
        return out

    def check(self, back=True, **how):
        got, want = self.run(back, **how), self.want(back)
        return {n: ref.check(n, host(t), want, self.dtype) for n, t in got.items() if t is not None}


CASES = [  # B, N, H, Hk, D, M, lengths, state, wider, decay
    (1, 1, 1, 1, 32, 16, None, False, 0, True), (1, 1, 2, 1, 64, 48, None, True, 0, True), (3, 2, 2, 2, 128, 32, [2, 0, 1], True, 0, True),
    (2, 17, 2, 1, 32, 32, [17, 16], True, 16, True), (1, 31, 3, 3, 64, 64, None, True, 0, False), (1, 32, 1, 1, 128, 128, None, True, 0, True),
    (2, 33, 4, 2, 64, 80, [1, 33], True, 0, True), (1, 63, 2, 2, 32, 112, None, False, 8, True), (2, 64, 2, 1, 128, 64, [63, 64], True, 0, True),
    (2, 65, 2, 2, 64, 64, [65, 64], True, 16, False), (1, 96, 3, 1, 128, 144, None, True, 0, True), (4, 97, 2, 2, 32, 64, [0, 97, 32, 96], True, 24, True),
    (2, 127, 6, 2, 64, 32, [127, 5], False, 0, True), (1, 128, 1, 1, 64, 256, None, True, 0, True), (2, 129, 2, 1, 128, 128, [129, 128], True, 16, True),
    (1, 193, 9, 3, 32, 16, None, True, 0, False), (3, 300, 2, 2, 64, 64, [300, 193, 64], True, 0, True), (1, 515, 2, 1, 128, 80, None, True, 0, True),
    (1, 20, 1, 1, 32, 512, None, True, 0, True), (12, 40, 1, 1, 64, 16, None, True, 0, True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(i) for i in c[:6]))
def test_delta(case, dtype):
    B, N, H, Hk, D, M, lengths, state, wider, decay = case
    Case(sum(case[:6]) * 31 + N, dtype, B, N, H, Hk, D, M, lengths, state, wider, decay).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_long_sequence(dtype):
    Case(7, dtype, 1, 2113, 2, 1, 64, 32).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_backward_without_the_forwards_workspace_is_the_same(dtype):
    c = Case(8, dtype, 2, 100, 4, 2, 64, 80, [100, 41])
    a, b = c.run(), c.run(given=False)
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_outputs_do_not_depend_on_what_is_kept(dtype):
    c = Case(9, dtype, 2, 150, 2, 2, 128, 48, [150, 149])
    a, b = c.run(back=False), c.run()
    assert torch.equal(a["o"], b["o"]) and torch.equal(a["h1"], b["h1"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,M", [(32, 16), (64, 80), (128, 128), (128, 512)])
def test_step(D, M, dtype):
    B, H, Hk = 5, 4, 2
    c = Case(D + M, dtype, B, 6, H, Hk, D, M, decay=D != 64)
    x, _ = c.inputs()
    h = c.d.dev(c.h0, True)
    outs = []
    for t in range(6):
        o = c.d.empty((B, H, M))
        la.la_delta_step(*(None if y is None else y[:, t].contiguous() for y in x), h, o, scale=c.scale)
        outs.append(o)
    want = c.want(back=False)
    ref.check("o", host(torch.stack(outs, 1)), want, dtype)
    ref.check("h1", host(h), want, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_prompt_then_pieces_then_tokens(dtype):
    """A prompt in parallel, a piece of a few tokens, single tokens: the uncut sequence."""
    c = Case(10, dtype, 2, 90, 4, 2, 64, 48)
    x, more = c.inputs()
    h, outs = c.d.dev(c.h0, True), []
    for a, b in ((0, 70), (70, 83)):
        o, h1 = c.d.empty((2, b - a, 4, 48)), torch.empty_like(h)
        la.la_delta_fwd(*(y[:, a:b].contiguous() for y in x), o, h0=h, h1=h1)
        h = h1
        outs.append(o)
    for t in range(83, 90):
        o = c.d.empty((2, 4, 48))
        la.la_delta_step(*(y[:, t].contiguous() for y in x), h, o)
        outs.append(o[:, None])
    want = c.want(back=False)
    # three calls: their errors add up
    for n, e in (("o", torch.cat(outs, 1)), ("h1", h)):
        ref.check(n, host(e), {n: want[n], "e_" + n: 2 * want["e_" + n]}, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_to_nothing_and_strengths_of_zero_and_one(dtype):
    """g = -inf and -1e30 forget everything before, beta = 0 writes nothing, beta = 1 writes all; two keys alike in a row."""
    c = Case(11, dtype, 1, 140, 2, 1, 64, 32)
    c.g[0, 5] = c.g[0, 64] = c.g[0, 100, 1] = -np.inf
    c.g[0, 31, 0] = -1e30
    c.g[0, 70:80] = 0.0
    c.beta[0, 10:20] = 0.0
    c.beta[0, 40:60] = 1.0
    c.k[0, 45:50] = c.k[0, 45]
    got, want = c.run(), None
    c.g = np.maximum(c.g, -1000.0)
    want = c.want()
    for n, t in got.items():
        ref.check(n, host(t), want, dtype)
    assert not host(got["dv"])[0, 10:20].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 1e30])
def test_outputs_before_a_token_do_not_depend_on_it(dtype, bad):
    c = Case(12, dtype, 1, 130, 2, 1, 64, 48)
    clean = c.run(back=False)["o"]
    for at in (3, 40, 77, 129):
        for what in ("q", "k", "v", "g", "beta"):
            x, more = c.inputs()
            x["qkvgb".index(what[0])][0, at:] = bad
            out, _, _ = c.outputs()
            la.la_delta_fwd(*x, **out, **more)
            assert torch.equal(out["o"][:, :at], clean[:, :at]), (what, at)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [(3, 1, 2, 1, 32, 16), (3, 29, 4, 2, 64, 80), (2, 32, 2, 2, 128, 128), (5, 64, 3, 1, 64, 64), (3, 65, 2, 1, 64, 48), (2, 31, 2, 1, 128, 144), (3, 32, 2, 1, 32, 256)])
def test_with_and_without_what_the_backward_needs(sizes, dtype):
    """Sequences of one chunk go another way without it: the same outputs."""
    B, N = sizes[:2]
    for lengths in (None, [N, N // 2, 0, 1, N - 1][:B]):
        c = Case(19, dtype, *sizes, lengths)
        a, b = c.run(back=True), c.run(back=False)
        for n in ("o", "h1"):
            assert torch.equal(a[n], b[n]), n
            ref.check(n, host(b[n]), c.want(), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_decay_that_is_no_number_shows(dtype):
    c = Case(18, dtype, 1, 130, 2, 1, 64, 48)
    x, more = c.inputs()
    x[3][0, 40, 0] = float("nan")
    out, _, _ = c.outputs()
    la.la_delta_fwd(*x, **out, **more)
    assert out["o"][0, 40:, 0].isnan().all() and out["h1"][0, 0].isnan().all()
    assert not out["o"][0, :40].isnan().any() and not out["o"][0, :, 1].isnan().any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_behind_a_sequence_may_hold_anything(dtype):
    c = Case(13, dtype, 3, 100, 2, 1, 64, 48, [100, 33, 0])
    a = c.run()
    for t in (c.q, c.k, c.v, c.do, c.g, c.beta):
        for b, n in enumerate(c.lengths):
            t[b, n:] = np.nan
    b = c.run()
    for n in a:
        assert torch.equal(a[n], b[n]), n
    for n in ("o", "dq", "dk", "dv", "dg", "dbeta"):
        for i, end in enumerate(c.lengths):
            assert not host(b[n])[i, end:].any(), n
    assert torch.equal(b["h1"][2], c.d.dev(c.h0, True)[2]) and torch.equal(b["dh0"][2], c.d.dev(c.dh1, True)[2])


def test_lengths_outside_the_sequence_are_taken_as_the_nearest():
    c = Case(14, "bf16", 3, 70, 2, 2, 32, 32, [-5, 70, 1 << 30])
    a = c.run()
    c.lengths = np.array([0, 70, 70], dtype=np.int32)
    b = c.run()
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_runs_repeat_bit_for_bit_and_on_another_stream():
    c = Case(15, "bf16", 4, 333, 4, 2, 64, 64, [333, 1, 64, 200])
    a = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = c.run(stream=s)
    torch.cuda.synchronize()
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_training_step_in_a_graph(dtype):
    c = Case(16, dtype, 2, 150, 4, 2, 64, 64, [150, 97])
    eager = c.run()
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
    for turn in range(4):
        for t in (*out.values(), *grads.values(), dh0):
            t.fill_(float("nan"))
        ws.fill_(255), wb.fill_(255)
        if turn == 2:                                                # other inputs in the same places
            x[2].mul_(2), do.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        if turn < 2:
            for n, t in {**out, **grads, "dh0": dh0}.items():
                assert torch.equal(t, eager[n]), n
        else:
            again = {n: t.clone() for n, t in {**out, **grads, "dh0": dh0}.items()}
            step()
            torch.cuda.synchronize()
            for n, t in {**out, **grads, "dh0": dh0}.items():
                assert torch.equal(t, again[n]), n


def test_the_native_path_and_the_checked_one_are_the_same(monkeypatch):
    from paper_2006_16236_amd import layer
    c = Case(17, "bf16", 2, 70, 4, 2, 64, 48, [70, 3])
    a = c.run()
    monkeypatch.setattr(layer, "_call", type("none", (), {n: staticmethod(lambda *x: None) for n in ("delta_fwd", "delta_step", "qk_fwd")}))
    b = c.run()
    for n in a:
        assert torch.equal(a[n], b[n]), n
