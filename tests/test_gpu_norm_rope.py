"""Norm and rotation of q and k on the GPU against the float64 oracle.

Tolerances, before any run: fp32 2e-5 (a dozen fp32 operations per value, 2^-24 each, and the sum of d squares; cos and
sin are off by 2^-23 at most), bf16 one rounding of the result, 2^-9 of the value and half the spacing at the RMS, so 2^-8;
the weights' gradients are fp32 sums of n rows, n 2^-24 of their terms at worst and sqrt(n) 2^-24 at random: 5e-5."""
import math

import numpy as np
import pytest
import torch

from oracle import decay_oracle as orc
from paper_2406_07368_b200 import binding, rope
from tests._util import rel_err

pytestmark = pytest.mark.gpu

TOL = {"f32": 2e-5, "bf16": 2.0 ** -8}
EPS = 1e-6


def host(t):
    return t.detach().double().cpu().numpy()


class Case:
    def __init__(self, io, d, B, H, T, rot, interleaved=False, far=0, seed=0, layout="fused", weights=True, scaling=None):
        r = np.random.default_rng(seed)
        x = torch.from_numpy(r.normal(size=(B, T, 4, H, d)).astype(np.float32) * 1.5).to(binding.TORCH_DTYPE[io]).cuda()
        if layout == "fused":
            self.q, self.k, self.gq, self.gk = (x[:, :, i].transpose(1, 2) for i in range(4))
        else:
            self.q, self.k, self.gq, self.gk = (x[:, :, i].transpose(1, 2).contiguous() for i in range(4))
        self.wq, self.wk = ((torch.from_numpy(1 + 0.3 * r.normal(size=d)).float().cuda() for _ in range(2)) if weights else (None, None))
        self.freq, self.mscale = (None, 1.0) if not rot else rope.inv_freq(rot, device="cuda", **(scaling or {}))
        self.pos = torch.from_numpy(r.integers(0, far + 1, size=B)).cuda() if far else None
        self.io, self.d, self.B, self.H, self.T, self.interleaved = io, d, B, H, T, interleaved
        self.ctx = binding.Context(H, d, 1, io=io)

    def kw(self):
        return dict(interleaved=self.interleaved, mscale=self.mscale, pos=self.pos)

    def check(self, norm=True, **out):
        f, p = (None if x is None else host(x) for x in (self.freq, self.pos))
        opts = dict(interleaved=self.interleaved, mscale=self.mscale, norm=norm, pos=p)
        want = [orc.norm_rope(host(x), None if w is None else host(w), EPS, f, **opts) for x, w in ((self.q, self.wq), (self.k, self.wk))]
        back = [orc.norm_rope_backward(host(x), host(g), None if w is None else host(w), EPS, f, **opts)
                for x, g, w in ((self.q, self.gq, self.wq), (self.k, self.gk, self.wk))]
        grads = self.ctx.la_norm_rope_backward(self.q, self.k, self.gq, self.gk, self.wq, self.wk, EPS, self.freq, norm=norm, **self.kw())
        got = self.ctx.la_norm_rope(self.q, self.k, self.wq, self.wk, EPS, self.freq, norm=norm, **self.kw(), **out)
        for x, y in zip(got, want):
            assert rel_err(host(x), y) < TOL[self.io]
        for i in range(2):
            assert rel_err(host(grads[i]), back[i][0]) < TOL[self.io]
            if norm:
                assert rel_err(host(grads[2 + i]), back[i][1]) < 5e-5
            else:
                assert grads[2 + i] is None
        return got, grads


TYPES = [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)]


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 128])
def test_rotated_parts_and_layouts(io, d, interleaved, rot):
    if rot > d:
        rot = 32
    Case(io, d, 2, 3, 37, rot, interleaved, far=5000, layout="fused" if rot % 32 else "dense").check()


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("B,H,T", [(1, 1, 1), (1, 32, 1), (64, 7, 1), (3, 5, 129), (2, 32, 600)])
def test_shapes(io, d, B, H, T):
    Case(io, d, B, H, T, d, seed=1, far=100).check()


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("norm,weights", [(True, False), (False, False), (False, True)])
def test_without_weights_or_norm(io, d, norm, weights):
    Case(io, d, 2, 4, 20, 32, True, seed=2, weights=weights).check(norm=norm)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("scaling", [dict(), dict(scaling="linear", factor=8.0), dict(scaling="base", factor=8.0),
                                     dict(scaling="parts", factor=8.0, trained_len=4096)])
def test_far_positions_and_scaled_tables(interleaved, scaling):
    """fp32 results at positions up to 2^40: the angle is formed in 64 bits (2^40 x 2^-53 = 1e-4 of a radian there; half of
    that position's error in the oracle too), at 10^6 in fp32's own precision."""
    Case("f32", 128, 4, 2, 9, 128, interleaved, far=10 ** 6, seed=3, scaling=scaling).check()
    c = Case("f32", 128, 1, 2, 9, 128, interleaved, seed=4, scaling=scaling)
    c.pos = torch.tensor([2 ** 40], device="cuda")
    want = orc.norm_rope(host(c.q), host(c.wq), EPS, host(c.freq), interleaved, c.mscale, True, [2 ** 40])
    got = c.ctx.la_norm_rope(c.q, c.k, c.wq, c.wk, EPS, c.freq, **c.kw())[0]
    assert rel_err(host(got), want) < 1e-3


@pytest.mark.parametrize("io,d", TYPES)
def test_in_place_and_given_buffers(io, d):
    c = Case(io, d, 2, 5, 33, 32, seed=5)
    want, grads = c.check()
    q, k = c.q.clone(), c.k.clone()
    got = c.ctx.la_norm_rope(q, k, c.wq, c.wk, EPS, c.freq, q_out=q, k_out=k, **c.kw())
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
    gq, gk, dwq, dwk = c.gq.clone(), c.gk.clone(), torch.full((d,), 9.0, device="cuda"), torch.full((d,), 9.0, device="cuda")
    c.ctx.la_norm_rope_backward(c.q, c.k, gq, gk, c.wq, c.wk, EPS, c.freq, dq=gq, dk=gk, dwq=dwq, dwk=dwk, **c.kw())
    assert all(torch.equal(x, y) for x, y in zip((gq, gk, dwq, dwk), grads))
    got = c.ctx.la_norm_rope_backward(c.q, c.k, c.gq, c.gk, c.wq, c.wk, EPS, c.freq, weights=False, **c.kw())
    assert torch.equal(got[0], grads[0]) and got[2] is None


@pytest.mark.parametrize("io,d", TYPES)
def test_rows_of_zeros_and_of_extremes(io, d):
    c = Case(io, d, 1, 2, 4, 32, seed=6)
    c.q[:, :, 0] = 0
    c.q[:, :, 1] = 1e-30
    c.q[:, :, 2] = 1e18
    q, _ = c.ctx.la_norm_rope(c.q, c.k, c.wq, c.wk, EPS, c.freq, **c.kw())
    want = orc.norm_rope(host(c.q), host(c.wq), EPS, host(c.freq))
    assert not q[:, :, 0].any() and rel_err(host(q)[:, :, 2:], want[:, :, 2:]) < TOL[io]
    c.q[:, 0, 3, 1] = float("nan")
    q, k = c.ctx.la_norm_rope(c.q, c.k, c.wq, c.wk, EPS, c.freq, **c.kw())
    assert q[0, 0, 3].isnan().all() and q.isnan().sum() == d and k.isfinite().all()


def test_guards_and_repeated_bits():
    from tests.test_gpu_guards import Arena
    for io, d in TYPES:
        c = Case(io, d, 2, 3, 41, 32, seed=7)
        ar = Arena(16 << 20)
        bufs = [ar.take((2, 3, 41, d), c.q.dtype, 3.0) for _ in range(4)]
        dw = [ar.take((d,), torch.float32, 3.0) for _ in range(2)]
        seen = None
        for _ in range(2):
            c.ctx.la_norm_rope(c.q, c.k, c.wq, c.wk, EPS, c.freq, q_out=bufs[0], k_out=bufs[1], **c.kw())
            c.ctx.la_norm_rope_backward(c.q, c.k, c.gq, c.gk, c.wq, c.wk, EPS, c.freq, dq=bufs[2], dk=bufs[3], dwq=dw[0], dwk=dw[1], **c.kw())
            now = [x.clone() for x in bufs + dw]
            assert seen is None or all(torch.equal(x, y) for x, y in zip(now, seen))
            seen = now
        ar.check()


def test_refusals():
    c = Case("bf16", 64, 2, 4, 12, 32, seed=8)
    call = lambda **kw: c.ctx.la_norm_rope(kw.pop("q", c.q), kw.pop("k", c.k), kw.pop("wq", c.wq), c.wk, kw.pop("eps", EPS),  # noqa: E731
                                           kw.pop("freq", c.freq), **kw)
    call()
    for kw, what in ((dict(q=c.q.float()), "dtype"), (dict(k=c.k[:1]), "shape"), (dict(wq=c.wq[:3]), "shape"),
                     (dict(freq=c.freq.float()), "dtype"), (dict(pos=torch.zeros(2, device="cuda")), "dtype"),
                     (dict(freq=c.freq.cpu()), "CUDA"), (dict(q_out=c.q[:1]), "shape")):
        with pytest.raises(ValueError, match=what):
            call(**kw)
    for kw in (dict(freq=c.freq[:3].contiguous()), dict(freq=c.freq.repeat(3)), dict(eps=-1.0), dict(eps=float("nan")),
               dict(mscale=float("inf")), dict(k=None), dict(q_out=c.k, k_out=c.q), dict(q_out=c.q, k_out=c.q)):
        with pytest.raises(binding.LaError) as e:
            call(**kw)
        assert e.value.code == binding.LA_ERR_INVALID_ARG
    with pytest.raises(binding.LaError):
        c.ctx.la_norm_rope_backward(c.q, c.k, c.gq, c.gk, c.wq, c.wk, EPS, c.freq, dq=c.gk)
    with pytest.raises(ValueError, match="shape"):
        c.ctx.la_norm_rope_backward(c.q, c.k, c.gq, c.gk, c.wq, c.wk, EPS, c.freq, dwq=torch.zeros(3, device="cuda"))


def test_weights_gradients_on_several_streams_and_in_graphs():
    """The partial sums of each call are its own."""
    c = Case("bf16", 128, 2, 8, 300, 128, seed=9)
    call = lambda: c.ctx.la_norm_rope_backward(c.q, c.k, c.gq, c.gk, c.wq, c.wk, EPS, c.freq, **c.kw())  # noqa: E731
    want = call()
    streams = [torch.cuda.Stream() for _ in range(3)]
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, call()))
    torch.cuda.synchronize()
    got = []
    for i in range(12):
        with torch.cuda.stream(streams[i % 3]):
            got.append(call())
            if i % 3 < 2:
                graphs[i % 3][0].replay()
    c.ctx.la_norm_rope_backward(c.q, c.k, c.gq, c.gk, c.wq, c.wk, EPS, c.freq, stream=streams[0], **c.kw())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for g in [*got, *(o for _, o in graphs)] for x, y in zip(g, want))


def test_gradient_of_a_layer_by_differences():
    """fp32: the directional derivative of sum(gq qo) + sum(gk ko) in q, k, wq, wk against a central difference of the
    kernel's own outputs summed in 64 bits: step 1e-2, so a truncation of 1e-4 and 2^-24 sqrt(n) / 1e-2 of rounding."""
    c = Case("f32", 64, 2, 3, 11, 32, seed=10)
    grads = c.ctx.la_norm_rope_backward(c.q, c.k, c.gq, c.gk, c.wq, c.wk, EPS, c.freq, **c.kw())

    def value(q, k, wq, wk):
        a, b = c.ctx.la_norm_rope(q, k, wq, wk, EPS, c.freq, **c.kw())
        return (host(a) * host(c.gq)).sum() + (host(b) * host(c.gk)).sum()

    args = [c.q, c.k, c.wq, c.wk]
    for i, g in enumerate(grads):
        step = torch.from_numpy(np.random.default_rng(i).normal(size=tuple(g.shape))).float().cuda() * 1e-2
        up, down = (value(*[x + s * step if j == i else x for j, x in enumerate(args)]) for s in (1.0, -1.0))
        size = math.sqrt(float((host(g) ** 2).sum())) * 1e-2
        assert abs((up - down) / 2 - (host(g) * host(step)).sum()) < 2e-3 * size, i
