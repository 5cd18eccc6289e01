"""The operators of the layer with a decay together, as a model calls them: norm and rotation, prefill of a padded batch,
single tokens after it; and a training step's gradients back to the projections.

Tolerances: fp32 the pieces' own.  bf16 twice theirs: between the pieces q and k are rounded once more.  Each is off by up to
2^-9 of its values at random (standard deviation 2^-9 / sqrt(3)), so s = scale q . k, of standard deviation 1 here, by
sqrt(2) 2^-9 / sqrt(3) = 1.6e-3, four standard deviations 6.4e-3; in the first rows an output is s v with |v| up to 4, off by
2.6e-2 where the metric's floor is 1, beside what the layer alone is off by, against 2 x 2e-2."""
import numpy as np
import pytest
import torch

from oracle import decay_oracle as orc
from paper_2406_07368_b200 import binding, rope
from tests._util import TOL, rel_err
from tests.test_gpu_decay import STATE_TOL, host, rel_err_octaves

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _weights(d, seed):
    r = np.random.default_rng(seed)
    return [torch.from_numpy(1 + 0.2 * r.normal(size=d)).float().cuda() for _ in range(2)]


@pytest.mark.parametrize("io,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
def test_serving_a_padded_batch_and_then_tokens(io, d):
    B, H, T, N = 3, 4, 150, 3
    lens = [150, 61, 0]
    r = np.random.default_rng(1)
    ctx = binding.Context(H, d, 1, io=io)
    x = torch.from_numpy(r.normal(size=(B, T + N, 3, H, d)).astype(np.float32)).to(ctx.dtype).cuda()
    wq, wk = _weights(d, 2)
    freq, mscale = rope.inv_freq(32, scaling="linear", factor=4.0, device="cuda")
    g = torch.tensor([-0.01, -0.1, -0.5, -2.0], device="cuda")
    st = ctx.new_state(B)
    st.pos.copy_(torch.tensor([0, 1000, 7]))
    pos = st.pos.clone()
    dlens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kw = dict(mscale=mscale)

    def qkv(a, b):
        return [x[:, a:b, i].transpose(1, 2) for i in range(3)]

    q, k, v = qkv(0, T)
    qn, kn = ctx.la_norm_rope(q, k, wq, wk, EPS, freq, pos=st.pos, **kw)
    o = ctx.la_decay_prefill(qn, kn, v, g, d ** -0.5, S_in=st.S, S_out=st.S, lens=dlens, pos=st.pos)
    assert st.pos.tolist() == [150, 1061, 7]
    steps = []
    for n in range(N):
        q, k, v = qkv(T + n, T + n + 1)
        qn, kn = ctx.la_norm_rope(q, k, wq, wk, EPS, freq, pos=st.pos, **kw)
        steps.append(ctx.la_decay_step(qn[:, :, 0], kn[:, :, 0], v[:, :, 0], g, d ** -0.5, st.S, pos=st.pos))
    assert st.pos.tolist() == [153, 1064, 10] and ctx.la_last_device_status() == binding.LA_OK
    for b in range(B):                                         # each sequence without its padding, from the definition
        tok = list(range(lens[b])) + list(range(T, T + N))
        q, k, v = (host(x[b:b + 1, tok, i]).transpose(0, 2, 1, 3) for i in range(3))
        f = dict(pos=[int(pos[b])], mscale=mscale)
        q, k = (orc.norm_rope(y, host(w), EPS, host(freq), **f) for y, w in ((q, wq), (k, wk)))
        want, S = orc.decay_prefill(q, k, v, host(g), d ** -0.5)
        got = np.concatenate([host(o[b:b + 1, :, :lens[b]])] + [host(s[b:b + 1, :, None]) for s in steps], axis=2)
        for h in range(H):
            assert rel_err_octaves(got[:, h:h + 1], want[:, h:h + 1]) < (2 if io == "bf16" else 1) * TOL[io], (b, h)
            # (bf16: k enters the state rounded, 2^-9 of each term at random; fp32 as the state alone)
            assert rel_err(host(st.S)[b, h], S[0, h]) < (TOL[io] if io == "bf16" else STATE_TOL), (b, h)
        assert not host(o)[b, :, lens[b]:].any()


@pytest.mark.parametrize("io,d", [("f32", 64), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_a_training_step_against_autograd(io, d, interleaved):
    """Gradients of sum(go o) in the projections and the norms' weights, against autograd through the layer in 64 bits."""
    B, H, T = 2, 3, 140
    r = np.random.default_rng(3)
    ctx = binding.Context(H, d, 1, io=io)
    x = torch.from_numpy(r.normal(size=(B, T, 3, H, d)).astype(np.float32)).to(ctx.dtype).cuda()
    go = torch.from_numpy(r.normal(size=(B, T, H, d)).astype(np.float32)).to(ctx.dtype).cuda().transpose(1, 2)
    wq, wk = _weights(d, 4)
    freq, _ = rope.inv_freq(d, device="cuda")
    g = torch.tensor([-0.02, -0.2, -1.0], device="cuda")
    q, k, v = (x[:, :, i].transpose(1, 2) for i in range(3))
    qn, kn = ctx.la_norm_rope(q, k, wq, wk, EPS, freq, interleaved=interleaved)
    ctx.la_decay_prefill(qn, kn, v, g, d ** -0.5)
    dqn, dkn, dv = ctx.la_decay_backward(qn, kn, v, go, g, d ** -0.5)
    dq, dk, dwq, dwk = ctx.la_norm_rope_backward(q, k, dqn, dkn, wq, wk, EPS, freq, interleaved=interleaved)

    leaf = [y.detach().double().requires_grad_() for y in (q, k, v, wq, wk)]
    ang = torch.arange(T, device="cuda").double()[:, None] * freq
    a = torch.arange(d // 2, device="cuda") * (2 if interleaved else 1)
    b = a + (1 if interleaved else d // 2)

    def turned(y, w):
        y = y / (y.square().mean(-1, keepdim=True) + EPS).sqrt() * w
        out = torch.empty_like(y)
        out[..., a] = y[..., a] * ang.cos() - y[..., b] * ang.sin()
        out[..., b] = y[..., b] * ang.cos() + y[..., a] * ang.sin()
        return out

    t = torch.arange(T, device="cuda").double()
    far = t[:, None] - t[None, :]
    m = torch.where(far >= 0, torch.exp(g.double()[:, None, None] * far.clamp(min=0)), torch.zeros_like(far))
    o = ((turned(leaf[0], leaf[3]) @ turned(leaf[1], leaf[4]).transpose(-1, -2)) * m * d ** -0.5) @ leaf[2]
    (o * go.double()).sum().backward()
    for name, got, y in zip(("dq", "dk", "dv", "dwq", "dwk"), (dq, dk, dv, dwq, dwk), leaf):
        got, want = host(got), y.grad.cpu().numpy()
        if got.ndim == 1:
            # a sum over B H T rows of products of the roundings above: their random part, TOL at sqrt(rows) terms
            assert rel_err(got, want) < TOL[io], name
        else:
            for h in range(H):
                assert rel_err(got[:, h], want[:, h]) < 2 * TOL[io], (name, h)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_value_that_is_not_finite_keeps_to_its_block_of_32(d, bad):
    """On the tensor cores: earlier blocks of 32 tokens, other channels, other heads are as without it."""
    B, H, T = 1, 2, 300
    ctx = binding.Context(H, d, 1)
    q, k, v = (torch.randn(B, H, T, d, device="cuda", generator=torch.Generator("cuda").manual_seed(i)).bfloat16() for i in range(3))
    g = torch.tensor([-0.1, -0.3], device="cuda")
    clean = ctx.la_decay_prefill(q, k, v, g, d ** -0.5)
    for t in (0, 31, 32, 100, 170, 255, 299):
        v2 = v.clone()
        v2[0, 1, t, 7] = bad
        o = ctx.la_decay_prefill(q, k, v2, g, d ** -0.5)
        first = t // 32 * 32
        assert torch.equal(o[:, 0], clean[:, 0]) and torch.equal(o[0, 1, :first], clean[0, 1, :first]), t
        assert not o[0, 1, t, 7].isfinite()
        assert torch.equal(o[0, 1, :, :7], clean[0, 1, :, :7]) and torch.equal(o[0, 1, :, 8:], clean[0, 1, :, 8:])
