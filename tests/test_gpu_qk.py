"""Norm of queries and keys for each head with the rotation, on the GPU against fp64."""
import numpy as np
import pytest
import torch

import delta_ref as ref
import paper_2006_16236_amd as la
from gpu_util import DEV
from layer_ref import check
from test_gpu_layer import Data, host

pytestmark = pytest.mark.gpu
EPS = 1e-6

CASES = [  # B, N, H, Hk, D, R, norm, weight, adjacent, lengths, wider, positions
    (1, 1, 1, 0, 8, 8, "rms", True, False, None, 0, False), (1, 1, 1, 1, 8, 0, "l2", False, False, None, 0, False),
    (2, 3, 3, 2, 16, 8, "rms", True, True, [3, 0], 0, True), (1, 5, 2, 1, 24, 16, "l2", True, False, None, 8, True),
    (3, 7, 5, 1, 32, 32, "rms", False, False, [1, 7, 6], 0, True), (2, 9, 6, 2, 96, 48, "rms", True, False, None, 16, True),
    (1, 65, 8, 8, 64, 64, None, True, True, None, 0, True), (2, 33, 8, 2, 80, 80, "rms", True, False, [33, 20], 8, False),
    (2, 31, 16, 16, 128, 128, "rms", True, False, None, 8, True), (1, 12, 7, 1, 136, 136, "l2", True, True, None, 0, True),
    (1, 12, 3, 3, 256, 64, "rms", True, False, None, 0, True), (2, 5, 2, 1, 264, 264, "rms", True, False, [5, 2], 0, True),
    (1, 4, 2, 2, 512, 512, "l2", True, False, None, 24, True), (64, 1, 8, 8, 64, 64, "rms", True, False, None, 0, True),
    (1, 3000, 4, 1, 64, 64, "rms", True, False, None, 0, False), (1, 1, 130, 70, 40, 40, "rms", True, True, None, 0, True)]


class Case:
    def __init__(self, dtype, B, N, H, Hk, D, R, kind, weight, adjacent, lengths, wider, positions):
        d = self.d = Data(B * 7919 + N * 31 + D, dtype)
        self.dtype, self.kind, self.adjacent, self.Hk = dtype, kind, adjacent, Hk
        self.q, self.dyq = d.array(B, N, H, D, scale=1.5), d.array(B, N, H, D)
        self.k, self.dyk = (d.array(B, N, Hk, D) if Hk else None for _ in range(2))
        self.wq, self.wk = ((1 + d.array(D, scale=0.2, f32=True)) if weight else None for _ in range(2))
        self.freq = (10000.0 ** (-np.arange(R // 2) / (R // 2))).astype(np.float32) if R else None
        self.pos = d.rng.integers(-1000, 1 << 20, (B, N)).astype(np.int32) if positions else None
        self.lengths = None if lengths is None else np.asarray(lengths, dtype=np.int32)
        self.wider = wider

    def run(self, **how):
        d, dev = self.d, lambda a: None if a is None else torch.from_numpy(a).to(DEV)
        q, k = d.dev(self.q, wider=self.wider), d.dev(self.k, wider=self.wider and self.wider + 16)
        more = dict(wq=dev(self.wq), wk=dev(self.wk) if self.Hk else None, freq=dev(self.freq), pos=dev(self.pos), lengths=dev(self.lengths), norm=self.kind,
                    adjacent=self.adjacent, eps=EPS)
        of = lambda a: None if a is None else d.empty(a.shape)  # noqa: E731
        out = dict(yq=of(self.q), yk=of(self.k))
        la.la_qk_fwd(q, out["yq"], k=k, yk=out["yk"], **more, **how)
        D = self.q.shape[3]
        grads = dict(dq=of(self.q), dk=of(self.k), dwq=d.empty((D,), True), dwk=d.empty((D,), True) if self.Hk else None)
        la.la_qk_bwd(q, d.dev(self.dyq), grads["dq"], k=k, dyk=d.dev(self.dyk), dk=grads["dk"], dwq=grads["dwq"], dwk=grads["dwk"], **more, **how)
        torch.cuda.synchronize()
        return {n: t for n, t in {**out, **grads}.items() if t is not None}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(i) for i in c[:6]))
def test_qk(case, dtype):
    c = Case(dtype, *case)
    got = c.run()
    D = c.q.shape[3]
    tokens = c.q.shape[0] * c.q.shape[1]
    for name, x, w, dy in (("q", c.q, c.wq, c.dyq), ("k", c.k, c.wk, c.dyk)):
        if x is None:
            continue
        args = (x, w, c.freq, c.pos, c.lengths, c.kind, c.adjacent, EPS, dy)
        want, mag = ref.qk(*args), ref.qk(*args, mag=True)
        # a sum of squares: 8 elements a lane and 6 steps over lanes, halved by the root; its inverse, the weight, two of the
        # rotation, and cosine and sine, off by 2 2^-24 of 1 and by the angle's: what is left of a turn is rounded once (2 pi 2^-25)
        k = 7 + 3 + 2 + 8
        check("y" + name, host(got["y" + name]), want["y"], mag["y"], dtype, k)
        # the same for dy turned back and for the sum along the head (14 more)
        check("d" + name, host(got["d" + name]), want["dx"], mag["dx"], dtype, 2 * k + 14)
        # a wave's tokens and heads one after the other, 64 lanes' slots, 1024 workgroups in 16 slices
        heads = x.shape[2] * D / 512
        check("dw" + name, host(got["dw" + name]), want["dw"], mag["dw"], "f32", 2 * k + 64 + 80 + (tokens / 1024 + 1) * (heads + 1))


@pytest.mark.parametrize("kind", ["rms", "l2"])
def test_gradients_without_eps(kind, monkeypatch):
    """eps = 0: what is left over of a wave's places for heads, three of sixteen here, has no length to divide by."""
    monkeypatch.setattr(f"{__name__}.EPS", 0.0)
    c = Case("f32", 2, 5, 2, 1, 24, 16, kind, True, False, None, 0, True)
    got = c.run()
    for name, x, w, dy in (("q", c.q, c.wq, c.dyq), ("k", c.k, c.wk, c.dyk)):
        args = (x, w, c.freq, c.pos, None, kind, False, 0.0, dy)
        want, mag = ref.qk(*args), ref.qk(*args, mag=True)
        check("d" + name, host(got["d" + name]), want["dx"], mag["dx"], "f32", 2 * 20 + 14)       # as above
        check("dw" + name, host(got["dw" + name]), want["dw"], mag["dw"], "f32", 2 * 20 + 64 + 80 + 2)


def test_a_single_tensor_without_anything():
    d = Data(3, "f32")
    x = d.array(2, 5, 3, 24)
    y, dx = d.empty(x.shape), d.empty(x.shape)
    la.la_qk_fwd(d.dev(x), y, norm=None)
    assert torch.equal(y, d.dev(x))
    assert la.la_qk_bwd(d.dev(x), d.dev(x), dx, norm=None) is None
    assert torch.equal(dx, d.dev(x))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_behind_a_sequence_may_hold_anything(dtype):
    case = list(CASES[7])
    c = Case(dtype, *case)
    a = c.run()
    for t in (c.q, c.k, c.dyq, c.dyk):
        for b, n in enumerate(c.lengths):
            t[b, n:] = np.nan
    b = c.run()
    for n in a:
        assert torch.equal(a[n], b[n]), n
    assert not host(b["yq"])[1, 20:].any() and not host(b["dk"])[1, 20:].any()


def test_far_positions_keep_their_angles():
    """Positions up to 2^31 - 1: the product with a frequency of 1 has 31 bits before its fraction."""
    d = Data(4, "f32")
    pos = np.array([[2 ** 31 - 1, 2 ** 31 - 2, -2 ** 31, 123456789]], dtype=np.int32)
    x = np.zeros((1, 4, 1, 8), dtype=np.float32)
    x[..., :4] = 1.0
    freq = np.array([1.0, 0.7, 0.1, 1e-4], dtype=np.float32)
    y = d.empty(x.shape)
    la.la_qk_fwd(d.dev(x), y, freq=torch.from_numpy(freq).to(DEV), pos=torch.from_numpy(pos).to(DEV), norm=None)
    angle = pos[0].astype(np.longdouble)[:, None] * freq.astype(np.longdouble)
    want = np.concatenate((np.cos(angle), np.sin(angle)), -1).astype(np.float64)
    # the turns are rounded to 53 bits twice (pos * (freq / 2 pi)): 2 2^-53 2^31 / (2 pi) turns, 2 pi of that as an angle
    assert np.abs(host(y)[0, :, 0] - want).max() <= 8 * 2.0 ** -24 + 2 * 2.0 ** -53 * 2.0 ** 31


def test_graph_stream_and_native_path(monkeypatch):
    from paper_2006_16236_amd import layer
    c = Case("bf16", *CASES[8])
    a = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = c.run(stream=s)
    for n in a:
        assert torch.equal(a[n], b[n]), n
    d = c.d
    q, k, freq = d.dev(c.q), d.dev(c.k), torch.from_numpy(c.freq).to(DEV)
    wq, wk, pos = (torch.from_numpy(t).to(DEV) for t in (c.wq, c.wk, c.pos))
    yq, yk = d.empty(c.q.shape), d.empty(c.k.shape)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        la.la_qk_fwd(q, yq, k=k, yk=yk, wq=wq, wk=wk, freq=freq, pos=pos)
    for _ in range(3):
        yq.fill_(float("nan")), yk.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(yq, a["yq"]) and torch.equal(yk, a["yk"])
    monkeypatch.setattr(layer, "_call", type("none", (), {"qk_fwd": staticmethod(lambda *x: None)}))
    b = c.run()
    for n in a:
        assert torch.equal(a[n], b[n]), n
