"""The layer with a decay on the GPU against the float64 oracle: prefill, gradients, single tokens.

Tolerances, before any run: outputs and gradients of the io type as everywhere in these tests (_util.TOL): fp32 1e-4 (sums
of up to 2000 fp32 terms: 2^-24 sqrt(2000) = 3e-6 of the RMS of the sum); bf16 2e-2 (the result's own rounding 2^-8 of the
value at most, and two sums whose terms carry up to 2^-8 at random, which leave about 2^-8 / sqrt(3) of the sum's RMS each,
at five standard deviations 2 x 1.1e-2 / sqrt(2)).  States, which are fp32 whatever the io type, 3e-5: where a product takes
its factor as two bf16 numbers each term is off by 2^-17 = 7.6e-6 at most, at random.
The metric is taken per octave of the position: without a decay the outputs grow with it.  In the first rows one term may
be all there is, s x with s = scale q . k, a dot product that cancels: rounded relative to its terms, it is off by 2^-24
(fp32) or 2^-9 (bf16) of its standard deviation, which is 1 for these inputs, however small s itself comes out.  An error
is therefore measured against 1 at least, the size of one term, which a row with any number of terms has in the mean.
"""
import numpy as np
import pytest
import torch

from oracle import decay_oracle as orc
from paper_2406_07368_b200 import binding
from tests._util import TOL, position_octaves, rel_err

pytestmark = pytest.mark.gpu

STATE_TOL = 3e-5
DECAYS = [-0.004, -0.05, -0.7, -1e-4, -6.0, 0.0, -np.inf, -40.0]


def rounded(x, io):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(binding.TORCH_DTYPE[io]).cuda()


def rel_err_octaves(x, y):
    worst = 0.0
    for lo, hi in position_octaves(y.shape[2]):
        a, b = x[:, :, lo:hi], y[:, :, lo:hi]
        floor = max(1.0, np.sqrt(np.mean(b * b)))
        worst = max(worst, float(np.max(np.abs(a - b) / np.maximum(np.abs(b), floor))))
    return worst


def host(t):
    return t.detach().double().cpu().numpy()


class Case:
    """Inputs on both sides.  layout: "bhtd" dense, "bthd" as a projection leaves it, "fused" slices of one buffer."""

    def __init__(self, io, d, B, H, T, seed=0, layout="bthd", cont=False, lens=None, decays=None):
        r = np.random.default_rng(seed)
        self.io, self.B, self.H, self.T, self.d, self.scale = io, B, H, T, d, d ** -0.5
        x = rounded(r.normal(size=(B, T, 4, H, d)), io)
        if layout == "fused":
            self.q, self.k, self.v, self.do = (x[:, :, i].transpose(1, 2) for i in range(4))
        elif layout == "bthd":
            self.q, self.k, self.v, self.do = (x[:, :, i].contiguous().transpose(1, 2) for i in range(4))
        else:
            self.q, self.k, self.v, self.do = (x[:, :, i].transpose(1, 2).contiguous() for i in range(4))
        g = np.array((decays or DECAYS) * (H // len(decays or DECAYS) + 1), dtype=np.float32)[:H]
        self.g = torch.from_numpy(g).cuda()
        self.S_in = torch.from_numpy(r.normal(size=(B, H, d, d)).astype(np.float32) * 2).cuda() if cont else None
        self.dS_out = torch.from_numpy(r.normal(size=(B, H, d, d)).astype(np.float32) * 0.3).cuda() if cont else None
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.ctx = binding.Context(H, d, 1, io=io)

    def oracle_args(self):
        return [host(x) for x in (self.q, self.k, self.v)]

    def state(self):
        return None if self.S_in is None else host(self.S_in)

    def check_prefill(self):
        S = torch.full((self.B, self.H, self.d, self.d), 7.0, device="cuda")
        o = self.ctx.la_decay_prefill(self.q, self.k, self.v, self.g, self.scale, S_in=self.S_in, S_out=S, lens=self.lens)
        assert self.ctx.la_last_device_status() == binding.LA_OK
        want, wS = orc.decay_prefill(*self.oracle_args(), host(self.g), self.scale, self.state(),
                                     None if self.lens is None else self.lens.tolist())
        for h in range(self.H):                                 # (heads differ in scale)
            assert rel_err_octaves(host(o)[:, h:h + 1], want[:, h:h + 1]) < TOL[self.io], h
            assert rel_err(host(S)[:, h], wS[:, h]) < STATE_TOL, h
        return o, S

    def check_backward(self):
        dS = torch.full((self.B, self.H, self.d, self.d), 7.0, device="cuda") if self.S_in is not None else None
        got = self.ctx.la_decay_backward(self.q, self.k, self.v, self.do, self.g, self.scale, S_in=self.S_in,
                                         dS_out=self.dS_out, dS_in=dS, lens=self.lens)
        assert self.ctx.la_last_device_status() == binding.LA_OK
        want = orc.decay_backward(*self.oracle_args(), host(self.do), host(self.g), self.scale, self.state(),
                                  None if self.dS_out is None else host(self.dS_out),
                                  None if self.lens is None else self.lens.tolist())
        lens = [self.T] * self.B if self.lens is None else self.lens.tolist()
        for i, (x, y) in enumerate(zip(got, want)):
            x = host(x)
            for b in range(self.B):
                assert not x[b, :, lens[b]:].any()
                for h in range(self.H):
                    if lens[b]:
                        a, c = x[b, h, None, None, :lens[b]], y[b, h, None, None, :lens[b]]
                        if i:                                   # dk, dv depend on what comes later: octaves from the end
                            a, c = a[:, :, ::-1], c[:, :, ::-1]
                        assert rel_err_octaves(a, c) < TOL[self.io], (i, b, h)
        if dS is not None:
            for h in range(self.H):
                assert rel_err(host(dS)[:, h], want[3][:, h]) < STATE_TOL, h
        return got, dS


TYPES = [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)]


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("T", [1, 2, 15, 17, 63, 127, 128, 129, 300])
def test_prefill_lengths(io, d, T):
    Case(io, d, 1, 8, T, seed=T, cont=T % 2 == 1).check_prefill()


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("layout", ["bhtd", "bthd", "fused"])
@pytest.mark.parametrize("cont", [False, True])
def test_prefill_layouts(io, d, layout, cont):
    Case(io, d, 2, 5, 200, seed=3, layout=layout, cont=cont).check_prefill()


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("B,H,T", [(1, 1, 2000), (1, 8, 1500), (40, 4, 140), (200, 1, 257)])
def test_prefill_shapes(io, d, B, H, T):
    Case(io, d, B, H, T, seed=4, cont=True, decays=[-0.01, 0.0, -0.3, -2.0]).check_prefill()


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("T,lens", [(150, [150, 0, 1, 77, 128]), (700, [129, 640, 256, 699, 3]), (9, [0, 0, 9, 1, 8])])
@pytest.mark.parametrize("cont", [False, True])
def test_padded_batches(io, d, T, lens, cont):
    """What lies behind a sequence's length reaches nothing, whatever it is."""
    c = Case(io, d, 5, 3, T, seed=5, cont=cont, lens=lens)
    o, S = c.check_prefill()
    got, dS = c.check_backward()
    for b, L in enumerate(lens):
        for x in (c.q, c.k, c.v, c.do):
            x[b, :, L:] = float("nan")
    S2 = torch.empty_like(S)
    o2 = c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_in=c.S_in, S_out=S2, lens=c.lens)
    assert torch.equal(o, o2) and torch.equal(S, S2)
    dS2 = None if dS is None else torch.empty_like(dS)
    got2 = c.ctx.la_decay_backward(c.q, c.k, c.v, c.do, c.g, c.scale, S_in=c.S_in, dS_out=c.dS_out, dS_in=dS2, lens=c.lens)
    assert all(torch.equal(x, y) for x, y in zip(got, got2)) and (dS is None or torch.equal(dS, dS2))


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("lens", [None, [130, 1], [700, 0], [2000, 129]])
def test_state_in_place_over_segments(io, d, lens):
    """S_out = S_in where a chain is cut into segments, the last ones of them empty: as with a buffer of its own."""
    c = Case(io, d, 2, 3, 2000, seed=18, cont=True, lens=lens)
    want = torch.empty_like(c.S_in)
    o = c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_in=c.S_in, S_out=want, lens=c.lens)
    for _ in range(20):
        S = c.S_in.clone()
        got = c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_in=S, S_out=S, lens=c.lens)
        assert torch.equal(got, o) and torch.equal(S, want)


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("T", [1, 2, 16, 65, 128, 129, 260])
@pytest.mark.parametrize("cont", [False, True])
def test_backward_lengths(io, d, T, cont):
    Case(io, d, 2, 4, T, seed=T, cont=cont, decays=[-0.01, 0.0, -0.7, -np.inf]).check_backward()


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("B,H,T,layout", [(1, 2, 1100, "bthd"), (30, 2, 140, "bhtd"), (2, 8, 200, "fused")])
def test_backward_shapes(io, d, B, H, T, layout):
    Case(io, d, B, H, T, seed=6, layout=layout, cont=True).check_backward()


@pytest.mark.parametrize("io,d", TYPES)
def test_gradient_against_differences(io, d):
    """The gradient in a direction against the difference of the layer's own outputs (their sums in 64 bits): both sides of
    the difference carry the roundings of the outputs, TOL of the outputs' size at random over B H T d values."""
    c = Case(io, d, 2, 2, 70, seed=9, cont=True, decays=[-0.05, -0.4])
    got, _ = c.check_backward()
    # the layer is linear in each of q, k, v by itself: a step as large as the input itself is exact
    for i, name in enumerate(("q", "k", "v")):
        step = rounded(np.random.default_rng(i).normal(size=(c.B, c.H, c.T, c.d)), io)
        args = dict(q=c.q, k=c.k, v=c.v)
        vals = []
        for x in (args[name] + step, args[name]):
            S = torch.empty_like(c.S_in)
            o = c.ctx.la_decay_prefill(*({**args, name: x}[n] for n in ("q", "k", "v")), c.g, c.scale, S_in=c.S_in, S_out=S)
            vals.append((host(o) * host(c.do)).sum() + (host(S) * host(c.dS_out)).sum())
        real_step = host((args[name] + step)) - host(args[name])
        want, n = (host(got[i]) * real_step).sum(), c.B * c.H * c.T * c.d
        size = np.sqrt((host(got[i]) ** 2).mean()) * np.sqrt(n)
        assert abs(vals[0] - vals[1] - want) < 5 * TOL[io] * size, name


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("B,H", [(1, 1), (3, 8), (70, 5), (100, 32)])
def test_steps_follow_a_prefill(io, d, B, H):
    """Tokens one by one from the state of a prefill, and the same tokens as one more prefill, against the oracle."""
    T, N = 20, 3
    c = Case(io, d, B, H, T + N, seed=10)
    S = torch.empty(B, H, d, d, device="cuda")
    pos = torch.arange(B, device="cuda")
    args = [x[:, :, :T] for x in (c.q, c.k, c.v)]
    c.ctx.la_decay_prefill(*args, c.g, c.scale, S_out=S, pos=pos)
    assert torch.equal(pos, torch.arange(B, device="cuda") + T)
    want, wS = orc.decay_prefill(*c.oracle_args(), host(c.g), c.scale)
    S2 = S.clone()
    o2 = c.ctx.la_decay_prefill(*(x[:, :, T:] for x in (c.q, c.k, c.v)), c.g, c.scale, S_in=S2, S_out=S2, pos=pos)
    for t in range(N):
        o = c.ctx.la_decay_step(*(x[:, :, T + t] for x in (c.q, c.k, c.v)), c.g, c.scale, S, pos=pos)
        for h in range(min(H, 8)):
            assert rel_err(host(o)[:, h], want[:, h, T + t]) < TOL[io], (t, h)
    assert torch.equal(pos, torch.arange(B, device="cuda") + T + 2 * N)
    for h in range(min(H, 8)):
        assert rel_err_octaves(host(o2)[:, h:h + 1], want[:, h:h + 1, T:]) < TOL[io]
        assert rel_err(host(S)[:, h], wS[:, h]) < STATE_TOL and rel_err(host(S2)[:, h], wS[:, h]) < STATE_TOL


@pytest.mark.parametrize("io,d", TYPES)
def test_slow_decay_over_many_steps(io, d):
    """lam = 1 - 1e-5 for 3000 tokens one by one: the factor's own rounding must not add up (3000 x 2^-25 = 9e-5)."""
    c = Case(io, d, 1, 2, 3000, seed=11, decays=[-1e-5])
    S = torch.zeros(1, 2, d, d, device="cuda")
    for t in range(c.T):
        c.ctx.la_decay_step(c.q[:, :, t], c.k[:, :, t], c.v[:, :, t], c.g, c.scale, S)
    _, wS = orc.decay_prefill(*c.oracle_args(), host(c.g), c.scale)
    assert rel_err(host(S), wS) < STATE_TOL
    S = torch.zeros(1, 2, d, d, device="cuda")
    c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_out=S)
    assert rel_err(host(S), wS) < STATE_TOL


@pytest.mark.parametrize("io,d", TYPES)
def test_shared_heads_and_outputs_in_place_of_others(io, d):
    """k and v of one head for all (stride 0), outputs into slices of one buffer; what lies between them survives."""
    c = Case(io, d, 2, 4, 150, seed=12)
    k, v = (x[:, :1].expand(-1, 4, -1, -1) for x in (c.k, c.v))
    want = orc.decay_prefill(host(c.q), host(k), host(v), host(c.g), c.scale)[0]
    buf = torch.full((2, 150, 3, 4, d), 5.0, dtype=c.q.dtype, device="cuda")
    out = buf[:, :, 1].transpose(1, 2)
    got = c.ctx.la_decay_prefill(c.q, k, v, c.g, c.scale, out=out)
    assert got is out and rel_err_octaves(host(out), want) < TOL[io]
    assert (buf[:, :, 0] == 5).all() and (buf[:, :, 2] == 5).all()
    buf.fill_(5.0)
    grads = [buf[:, :, i].transpose(1, 2) for i in range(3)]
    c.ctx.la_decay_backward(c.q, k, v, c.do, c.g, c.scale, dq=grads[0], dk=grads[1], dv=grads[2])
    for x, y in zip(grads, orc.decay_backward(host(c.q), host(k), host(v), host(c.do), host(c.g), c.scale)):
        assert rel_err(host(x), y) < TOL[io]


def test_outputs_have_the_order_of_q():
    c = Case("bf16", 64, 2, 4, 40, layout="bthd")
    o = c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale)
    assert o.transpose(1, 2).is_contiguous()
    o = c.ctx.la_decay_prefill(c.q.contiguous(), c.k, c.v, c.g, c.scale)
    assert o.is_contiguous()


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("T", [5, 400])
def test_heads_and_lengths_the_device_refuses(io, d, T):
    c = Case(io, d, 3, 3, T, seed=13, cont=True, decays=[-0.1, -0.2, -0.3])
    o, S, pos = torch.full_like(c.q, 5.0), torch.full_like(c.S_in, 5.0), torch.zeros(3, dtype=torch.int64, device="cuda")
    want, wS = c.check_prefill()
    for bad in (0.5, float("nan"), float("inf")):
        c.g[1] = bad
        c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_in=c.S_in, S_out=S, out=o)
        assert c.ctx.la_last_device_status() == binding.LA_ERR_INVALID_ARG
        c.ctx.la_clear_device_status()
        assert (o[:, 1] == 5).all() and (S[:, 1] == 5).all()
        assert torch.equal(o[:, ::2], want[:, ::2]) and torch.equal(S[:, ::2], wS[:, ::2])
        before = S.clone()
        step = torch.full_like(o[:, :, 0], 5.0)
        c.ctx.la_decay_step(c.q[:, :, 0], c.k[:, :, 0], c.v[:, :, 0], c.g, c.scale, S, out=step)
        assert c.ctx.la_last_device_status() == binding.LA_ERR_INVALID_ARG
        c.ctx.la_clear_device_status()
        assert (step[:, 1] == 5).all() and torch.equal(S[:, 1], before[:, 1])
        o.fill_(5.0)
        S.fill_(5.0)
    c.g[1] = -0.2
    for bad in (-1, T + 1, -2**31, 2**31 - 1):
        lens = torch.tensor([T, bad, T], dtype=torch.int32, device="cuda")
        pos.zero_()
        c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_in=c.S_in, S_out=S, out=o, lens=lens, pos=pos)
        assert c.ctx.la_last_device_status() == binding.LA_ERR_INVALID_ARG
        c.ctx.la_clear_device_status()
        assert (o[1] == 5).all() and (S[1] == 5).all() and pos.tolist() == [T, 0, T]
        assert torch.equal(o[::2], want[::2])


def test_refusals():
    c = Case("bf16", 64, 2, 4, 24, cont=True)
    p = lambda **kw: c.ctx.la_decay_prefill(*(kw.pop(n, getattr(c, n)) for n in ("q", "k", "v")), kw.pop("g", c.g),  # noqa: E731
                                            kw.pop("scale", c.scale), **kw)
    p()
    for kw, what in ((dict(k=c.k.float()), "dtype"), (dict(k=c.k[:1]), "shape"), (dict(v=c.v.cpu()), "CUDA"),
                     (dict(q=c.q.transpose(2, 3).contiguous().transpose(2, 3)), "dense rows"), (dict(g=c.g[:3]), "shape"),
                     (dict(g=c.g.double()), "dtype"), (dict(S_in=c.S_in[:, :, :, ::2]), "contiguous"),
                     (dict(S_out=c.S_in.bfloat16()), "dtype"), (dict(lens=torch.ones(2, device="cuda")), "dtype"),
                     (dict(pos=torch.ones(3, dtype=torch.int64, device="cuda")), "shape"), (dict(out=c.q[:1]), "shape")):
        with pytest.raises(ValueError, match=what):
            p(**kw)
    wide = torch.zeros(2, 4, 24, 68, dtype=torch.bfloat16, device="cuda")
    odd = torch.zeros(2 * 4 * 24 * 64 + 8, dtype=torch.bfloat16, device="cuda")[1:1 + 2 * 4 * 24 * 64].view(2, 4, 24, 64)
    same = c.q[:, :, :1].expand(-1, -1, 24, -1)
    for kw in (dict(q=wide[..., :64]), dict(k=odd), dict(v=same), dict(out=c.q), dict(out=c.v), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(k=None), dict(out=torch.zeros_like(c.q[:, :1]).expand(-1, 4, -1, -1)),
               dict(g=None)):
        with pytest.raises(binding.LaError) as e:
            p(**kw)
        assert e.value.code == binding.LA_ERR_INVALID_ARG
    g = torch.zeros_like(c.S_in)
    for kw in (dict(dq=c.q), dict(dk=c.do), dict(dS_in=c.S_in), dict(dS_out=g, dS_in=g)):
        with pytest.raises(binding.LaError) as e:
            c.ctx.la_decay_backward(c.q, c.k, c.v, c.do, c.g, c.scale, S_in=c.S_in, **kw)
        assert e.value.code == binding.LA_ERR_INVALID_ARG
    one = [x[:, :, 0] for x in (c.q, c.k, c.v)]
    for kw, err in ((dict(S=c.S_in[:1]), ValueError), (dict(S=None), binding.LaError), (dict(S=c.S_in, out=one[0]), binding.LaError)):
        with pytest.raises(err):
            c.ctx.la_decay_step(*one, c.g, c.scale, **kw)
    with pytest.raises(TypeError):
        c.ctx.la_decay_step("q", *one[1:], c.g, c.scale, c.S_in)
    c.ctx.close()
    with pytest.raises(binding.LaError):
        p()


def test_graph_replays_and_streams():
    """Captured and replayed on new inputs; on a given stream that is not the current one."""
    c = Case("bf16", 128, 2, 4, 300, seed=14, cont=True, decays=[-0.1])
    S, dS = torch.empty_like(c.S_in), torch.empty_like(c.S_in)
    call = lambda: (c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_in=c.S_in, S_out=S),  # noqa: E731
                    *c.ctx.la_decay_backward(c.q, c.k, c.v, c.do, c.g, c.scale, S_in=c.S_in, dS_out=c.dS_out, dS_in=dS))
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for seed in (1, 2):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for x in (c.q, c.k, c.v, c.do):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        graph.replay()
        snap = [x.clone() for x in (*got, S, dS)]
        want = call()
        assert all(torch.equal(x, y) for x, y in zip(snap, (*want, S, dS)))
    s, out = torch.cuda.Stream(), torch.full_like(c.q, 7.0)
    want = c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(100_000_000)
    c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, out=out, stream=s)
    before = out.clone()
    torch.cuda.current_stream().synchronize()
    assert (before == 7.0).all()
    s.synchronize()
    assert torch.equal(out, want)


def test_calls_on_two_streams_at_once():
    c = Case("bf16", 128, 2, 8, 700, seed=15, decays=[-0.1])
    want = c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale)
    grads = c.ctx.la_decay_backward(c.q, c.k, c.v, c.do, c.g, c.scale)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                got.append((c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale),
                            *c.ctx.la_decay_backward(c.q, c.k, c.v, c.do, c.g, c.scale)))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for g in got for x, y in zip(g, (want, *grads)))


@pytest.mark.parametrize("io,d", TYPES)
@pytest.mark.parametrize("T", [1, 100, 130, 517])
def test_guards_and_repeated_bits(io, d, T):
    """Outputs between guard words that survive; the same call twice gives the same bits."""
    from tests.test_gpu_guards import Arena
    c = Case(io, d, 2, 3, T, seed=16, cont=True)
    ar = Arena(64 << 20)
    bufs = [ar.take((2, 3, T, d), c.q.dtype, 3.0) for _ in range(4)]
    states = [ar.take((2, 3, d, d), torch.float32, 3.0) for _ in range(3)]
    pos = ar.take((2,), torch.int64, 0)
    states[2].copy_(c.S_in)
    one = ar.take((2, 3, d), c.q.dtype, 3.0)
    seen = None
    for _ in range(2):
        states[2].copy_(c.S_in)
        c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_in=c.S_in, S_out=states[0], out=bufs[0], pos=pos)
        c.ctx.la_decay_backward(c.q, c.k, c.v, c.do, c.g, c.scale, S_in=c.S_in, dS_out=c.dS_out, dS_in=states[1],
                                dq=bufs[1], dk=bufs[2], dv=bufs[3])
        c.ctx.la_decay_step(c.q[:, :, 0], c.k[:, :, 0], c.v[:, :, 0], c.g, c.scale, states[2], out=one)
        now = [x.clone() for x in (*bufs, *states, one)]
        assert seen is None or all(torch.equal(x, y) for x, y in zip(now, seen))
        seen = now
    ar.check()
    assert c.ctx.la_last_device_status() == binding.LA_OK


@pytest.mark.parametrize("io,d", TYPES)
def test_nan_shows_from_its_token_on(io, d):
    """A NaN in q, k or v reaches the outputs that depend on it; earlier tokens of other tiles, other heads: untouched."""
    c = Case(io, d, 2, 2, 300, seed=17, decays=[-0.1, -0.2])
    clean = c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale)
    for name, t in (("q", 40), ("k", 140), ("v", 140)):
        x = getattr(c, name)
        keep = x[1, 0, t, 5].clone()
        x[1, 0, t, 5] = float("nan")
        S = torch.empty(2, 2, d, d, device="cuda")
        o = c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_out=S)
        x[1, 0, t, 5] = keep
        assert torch.equal(o[0], clean[0]) and torch.equal(o[1, 1], clean[1, 1]) and torch.equal(o[1, 0, :128], clean[1, 0, :128]) or name == "q"
        if name == "q":
            assert o[1, 0, 40].isnan().all() and o.isnan().sum() == d and S.isfinite().all()
        elif name == "k":
            assert o[1, 0, 140:].isnan().all() and o[1, 0, :140].isfinite().all() and S[1, 0, 5].isnan().all()
        else:
            assert o[1, 0, 140:, 5].isnan().all() and o[1, 0, :, :5].isfinite().all() and S[1, 0, :, 5].isnan().all()


def norms_off(x, y, lens):
    """Largest error over sequences, heads and runs of 64 tokens, 2-norm over 2-norm (of entries of 1 at least)."""
    worst = 0.0
    for b, L in enumerate(lens):
        assert not x[b, :, L:].any()
        for t in range(0, L, 64):
            e, w = x[b, :, t:min(t + 64, L)] - y[b, :, t:min(t + 64, L)], y[b, :, t:min(t + 64, L)]
            size = np.maximum(np.sqrt((w * w).sum(axis=(1, 2))), np.sqrt(w[0].size))
            worst = max(worst, float(np.max(np.sqrt((e * e).sum(axis=(1, 2))) / size)))
    return worst


@pytest.mark.parametrize("io,d", [("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("B,H,T", [(2, 8, 1030), (3, 7, 1500), (9, 4, 700), (15, 4, 2000), (74, 1, 1800), (25, 3, 1900)])
def test_as_many_segments_as_run_at_once(io, d, B, H, T):
    """Chains from a few to half the GPU and more: cut into 8, 4, 2 and no segments, some of them ragged or empty.

    Measured by 2-norms of runs of tokens.  Single entries say less with this many of them: a row's scores p_j carry up to
    2^-8 |p_j| each, and where one of them is 4.5 standard deviations, as among 10^4 rows one is, the entry in which its
    v_j has 2 and the other terms take the sum back to the mean size, r, is off by up to 4.5 x 2 x 2^-8 / r = 0.035 / r;
    with a decay of exp(-0.3) r is 1.5: 0.023 (0.0205 was seen, token by token without rounded scores 0.004).  A 2-norm has
    the mean of the v_j: the result's rounding leaves 2^-8 of it at most, and scores, state and (gradients) K rounded once
    each 2^-8 of their own part at most, independent of one another: 2^-8 (1 + sqrt(2)) and 2^-8 (1 + sqrt(3))."""
    lens = [(T, T // 3, T - 1, 129, 0)[b % 5] for b in range(B)]
    c = Case(io, d, B, H, T, seed=20, cont=True, lens=lens, decays=[-0.01, 0.0, -0.3, -2.0])
    S = [torch.full_like(c.S_in, 7.0) for _ in range(2)]
    o = [c.ctx.la_decay_prefill(c.q, c.k, c.v, c.g, c.scale, S_in=c.S_in, S_out=x, lens=c.lens) for x in S]
    assert c.ctx.la_last_device_status() == binding.LA_OK
    assert torch.equal(*o) and torch.equal(*S)
    want, wS = orc.decay_prefill(*c.oracle_args(), host(c.g), c.scale, c.state(), lens)
    assert norms_off(host(o[0]), want, lens) < 2 ** -8 * (1 + 2 ** 0.5)
    for h in range(H):
        assert rel_err(host(S[0])[:, h], wS[:, h]) < STATE_TOL, h
    if B * H <= 25:
        dS = torch.full_like(c.S_in, 7.0)
        got = c.ctx.la_decay_backward(c.q, c.k, c.v, c.do, c.g, c.scale, S_in=c.S_in, dS_out=c.dS_out, dS_in=dS, lens=c.lens)
        want = orc.decay_backward(*c.oracle_args(), host(c.do), host(c.g), c.scale, c.state(), host(c.dS_out), lens)
        for x, y in zip(got, want):
            assert norms_off(host(x), y, lens) < 2 ** -8 * (1 + 3 ** 0.5)
        for h in range(H):
            assert rel_err(host(dS)[:, h], want[3][:, h]) < STATE_TOL, h
