"""Pins of the float64 oracle of the layer with a decay: hand-worked values, other forms, differences."""
import math

import numpy as np
import pytest
import torch

from oracle import decay_oracle as orc
from paper_2406_07368_b200 import rope


def _case(seed, B=2, H=3, T=9, d=4):
    r = np.random.default_rng(seed)
    q, k, v, do = (r.normal(size=(B, H, T, d)) for _ in range(4))
    return q, k, v, do, -r.uniform(0.01, 1.5, H), r.normal(size=(B, H, d, d)), r.normal(size=(B, H, d, d))


def test_hand_worked_example():
    # d = 1, lam = 1/2, scale 2: S = 3, 3/2 + 4 = 11/2, 11/4 + 5 = 31/4; o = 2 q S
    g = [math.log(0.5)]
    q, k, v = (np.array(x, dtype=float).reshape(1, 1, 3, 1) for x in ([1, 1, 2], [1, 2, 1], [3, 2, 5]))
    o, S = orc.decay_prefill(q, k, v, g, 2.0)
    assert np.allclose(o.ravel(), [6, 11, 31]) and np.allclose(S, 31 / 4)
    o, S = orc.decay_prefill(q, k, v, g, 2.0, S_in=np.full((1, 1, 1, 1), 8.0))
    assert np.allclose(o.ravel(), [6 + 8, 11 + 4, 31 + 4]) and np.allclose(S, 31 / 4 + 1)
    # loss = sum o, behind the last token nothing: D = 2 q_2 = 4, 2 + 2 q_1 = 4, 2 + 2 q_0 = 4
    dq, dk, dv, dS = orc.decay_backward(q, k, v, np.ones_like(q), g, 2.0)
    assert np.allclose(dq.ravel(), [6, 11, 31 / 2]) and np.allclose(dk.ravel(), [12, 8, 20])
    assert np.allclose(dv.ravel(), [4, 8, 4]) and np.allclose(dS, 2)


@pytest.mark.parametrize("cont", [False, True])
def test_forms_agree(cont):
    q, k, v, _, g, S0, _ = _case(1)
    S0 = S0 if cont else None
    a, b = orc.decay_prefill(q, k, v, g, 0.7, S0), orc.decay_recurrent(q, k, v, g, 0.7, S0)
    assert np.allclose(a[0], b[0]) and np.allclose(a[1], b[1])


def test_special_decays():
    q, k, v, _, _, S0, _ = _case(2, H=2)
    o, S = orc.decay_prefill(q, k, v, [0.0, -np.inf], 1.0, S0)
    c = np.cumsum(k[:, 0, :, :, None] * v[:, 0, :, None, :], axis=1) + S0[:, 0, None]
    assert np.allclose(o[:, 0], np.einsum("bta,btac->btc", q[:, 0], c)) and np.allclose(S[:, 0], c[:, -1])
    assert np.allclose(o[:, 1], (q[:, 1] * k[:, 1]).sum(-1, keepdims=True) * v[:, 1])
    assert np.allclose(S[:, 1], k[:, 1, -1, :, None] * v[:, 1, -1, None, :])


def test_lengths_cut_the_sequences():
    q, k, v, do, g, S0, D = _case(3)
    lens = [5, 0]
    o, S = orc.decay_prefill(q, k, v, g, 0.5, S0, lens)
    o5, S5 = orc.decay_prefill(q[:1, :, :5], k[:1, :, :5], v[:1, :, :5], g, 0.5, S0[:1])
    assert np.allclose(o[:1, :, :5], o5) and not o[0, :, 5:].any() and not o[1].any()
    assert np.allclose(S[:1], S5) and np.array_equal(S[1], S0[1])
    dq, dk, dv, dS = orc.decay_backward(q, k, v, do, g, 0.5, S0, D, lens)
    assert not dq[1].any() and not dk[0, :, 5:].any() and not dv[1].any() and np.array_equal(dS[1], D[1])


def test_gradients_against_autograd_and_differences():
    q, k, v, do, g, S0, D = _case(4)
    x = [torch.tensor(t, requires_grad=True) for t in (q, k, v, S0)]
    lam = torch.exp(torch.tensor(g))[None, :, None, None]
    S, loss = x[3], 0.0
    for t in range(q.shape[2]):
        S = lam * S + x[1][:, :, t, :, None] * x[2][:, :, t, None, :]
        loss = loss + (0.6 * torch.einsum("bha,bhac->bhc", x[0][:, :, t], S) * torch.tensor(do[:, :, t])).sum()
    (loss + (S * torch.tensor(D)).sum()).backward()
    got = orc.decay_backward(q, k, v, do, g, 0.6, S0, D)
    for a, b in zip(got, x):
        assert np.allclose(a, b.grad.numpy())

    def value(*t):
        o, S = orc.decay_prefill(*t[:3], g, 0.6, t[3])
        return (o * do).sum() + (S * D).sum()

    r, args = np.random.default_rng(5), [q, k, v, S0]
    for i, grad in enumerate(got):
        step = r.normal(size=grad.shape) * 1e-5
        up, down = (value(*[t + s * step if j == i else t for j, t in enumerate(args)]) for s in (1, -1))
        assert math.isclose((up - down) / 2, (grad * step).sum(), rel_tol=1e-6, abs_tol=1e-10)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_by_hand_and_by_invariants(interleaved):
    x = np.array([1.0, 2.0, 3.0, 4.0, 5.0]).reshape(1, 1, 1, 5)
    y = orc.norm_rope(x, None, 0.0, [math.pi / 2, math.pi], interleaved, 1.0, norm=False, pos=[1])
    want = [-2, 1, -3, -4, 5] if interleaved else [-3, -2, 1, -4, 5]
    assert np.allclose(y.ravel(), want)
    # q . k after the rotation depends on the distance of their positions only
    r = np.random.default_rng(6)
    q, k = r.normal(size=(2, 1, 1, 1, 8))
    f = rope.inv_freq(8)[0].numpy()
    dots = [(orc.norm_rope(q, None, 0, f, interleaved, norm=False, pos=[p + 3]) *
             orc.norm_rope(k, None, 0, f, interleaved, norm=False, pos=[p])).sum() for p in (0, 5, 1000)]
    assert np.allclose(dots, dots[0])


@pytest.mark.parametrize("interleaved,norm,rot", [(False, True, 8), (True, True, 4), (True, False, 8), (False, True, 0)])
def test_norm_rope_gradients_against_differences(interleaved, norm, rot):
    r = np.random.default_rng(7)
    x, gy, w = r.normal(size=(2, 2, 3, 8)), r.normal(size=(2, 2, 3, 8)), r.normal(size=8)
    f = rope.inv_freq(rot)[0].numpy() if rot else None
    kw = dict(interleaved=interleaved, mscale=1.3, norm=norm, pos=[4, 100])
    dx, dw = orc.norm_rope_backward(x, gy, w, 1e-3, f, **kw)
    value = lambda x, w: (orc.norm_rope(x, w, 1e-3, f, **kw) * gy).sum()  # noqa: E731
    step = r.normal(size=x.shape) * 1e-5
    assert math.isclose((value(x + step, w) - value(x - step, w)) / 2, (dx * step).sum(), rel_tol=1e-6, abs_tol=1e-10)
    if norm:
        step = r.normal(size=8) * 1e-5
        assert math.isclose((value(x, w + step) - value(x, w - step)) / 2, (dw * step).sum(), rel_tol=1e-6, abs_tol=1e-10)
    else:
        assert dw is None


def test_unit_rms_and_weights():
    x = np.random.default_rng(8).normal(size=(1, 1, 2, 8)) * 5
    y = orc.norm_rope(x, None, 0.0, None)
    assert np.allclose((y * y).mean(-1), 1) and np.allclose(orc.norm_rope(x, 2 * np.ones(8), 0.0, None), 2 * y)


def test_frequency_tables():
    f, m = rope.inv_freq(8, 10000.0)
    assert m == 1.0 and f.dtype == torch.float64 and np.allclose(f.numpy(), [1, 0.1, 0.01, 0.001])
    assert np.allclose(rope.inv_freq(8, 10000.0, "linear", 4.0)[0].numpy(), f.numpy() / 4)
    g = rope.inv_freq(8, 10000.0, "base", 4.0)[0].numpy()
    assert math.isclose(g[0], 1.0) and math.isclose(g[-1], 0.001 / 4)
    p, m = rope.inv_freq(8, 10000.0, "parts", 4.0, trained_len=2048, fast=32, slow=1)
    turns = 2048 * f.numpy() / (2 * math.pi)                    # 326, 32.6, 3.26, 0.33
    keep = [1, 1, (turns[2] - 1) / 31, 0]
    assert np.allclose(p.numpy(), [a * x + (1 - a) * x / 4 for a, x in zip(keep, f.numpy())])
    assert math.isclose(m, 1 + 0.1 * math.log(4))
    for bad in (dict(rot=7), dict(rot=8, factor=0.5), dict(rot=8, scaling="other"), dict(rot=8, scaling="parts"),
                dict(rot=2, scaling="base"), dict(rot=8, base=0.0)):
        with pytest.raises(ValueError):
            rope.inv_freq(**bad)
