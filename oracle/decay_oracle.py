"""Float64 oracle of the layer with a decay, its gradients, and the norm and rotation of q and k (numpy, no blocking).

Test infrastructure only.  Shapes as in include/la.h: q, k, v, do [B, H, T, d]; log_decay [H]; states [B, H, d, d] with the
value's index last; lens [B].
"""
from __future__ import annotations

import numpy as np


def _powers(g, n):
    """lam^n for integer arrays n >= 0, lam = exp(g); lam^0 = 1 also where lam is 0; 0 where n < 0."""
    n = np.asarray(n, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        p = np.exp(g * np.maximum(n, 0.0))
    return np.where(n > 0, p, np.where(n == 0, 1.0, 0.0))


def decay_prefill(q, k, v, log_decay, scale, S_in=None, lens=None):
    """(o, S_out): every pair of tokens, and the state as a weighted sum."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    B, H, T, d = q.shape
    o = np.zeros_like(q)
    S = np.zeros((B, H, d, d)) if S_in is None else np.asarray(S_in, dtype=np.float64).copy()
    for b in range(B):
        L = T if lens is None else int(lens[b])
        if L == 0:
            continue
        t = np.arange(L)
        for h in range(H):
            g = float(log_decay[h])
            x, y, z = q[b, h, :L], k[b, h, :L], v[b, h, :L]
            o[b, h, :L] = ((x @ y.T) * _powers(g, t[:, None] - t[None, :])) @ z + _powers(g, t + 1)[:, None] * (x @ S[b, h])
            S[b, h] = _powers(g, L) * S[b, h] + (y * _powers(g, L - 1 - t)[:, None]).T @ z
    return o * scale, S


def decay_recurrent(q, k, v, log_decay, scale, S_in=None):
    """The same token by token: S = lam S + k v^T, o = scale q^T S."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    B, H, T, d = q.shape
    S = np.zeros((B, H, d, d)) if S_in is None else np.asarray(S_in, dtype=np.float64).copy()
    lam = np.exp(np.asarray(log_decay, dtype=np.float64))[None, :, None, None]
    o = np.zeros_like(q)
    for t in range(T):
        S = lam * S + k[:, :, t, :, None] * v[:, :, t, None, :]
        o[:, :, t] = scale * np.einsum("bha,bhac->bhc", q[:, :, t], S)
    return o, S


def decay_backward(q, k, v, do, log_decay, scale, S_in=None, dS_out=None, lens=None):
    """(dq, dk, dv, dS_in) by the recurrence of the states forwards and of their gradients backwards."""
    q, k, v, do = (np.asarray(x, dtype=np.float64) for x in (q, k, v, do))
    B, H, T, d = q.shape
    dq, dk, dv = np.zeros_like(q), np.zeros_like(q), np.zeros_like(q)
    dS = np.zeros((B, H, d, d)) if dS_out is None else np.asarray(dS_out, dtype=np.float64).copy()
    for b in range(B):
        L = T if lens is None else int(lens[b])
        for h in range(H):
            lam = np.exp(float(log_decay[h]))
            S = np.zeros((d, d)) if S_in is None else np.asarray(S_in[b, h], dtype=np.float64).copy()
            for t in range(L):
                S = lam * S + np.outer(k[b, h, t], v[b, h, t])
                dq[b, h, t] = scale * (S @ do[b, h, t])
            D = dS[b, h]
            for t in reversed(range(L)):
                D = D + scale * np.outer(q[b, h, t], do[b, h, t])
                dk[b, h, t] = D @ v[b, h, t]
                dv[b, h, t] = D.T @ k[b, h, t]
                D = lam * D
            dS[b, h] = D
    return dq, dk, dv, dS


def _turns(pos, T, inv_freq):
    """exp(i p f) [B, 1, T, rot / 2]."""
    p = np.asarray(pos, dtype=np.float64)[:, None] + np.arange(T)
    return np.exp(1j * p[:, None, :, None] * np.asarray(inv_freq, dtype=np.float64))


def _rotate(y, turn, interleaved, mscale):
    y = y.copy()
    n = turn.shape[-1]
    a = np.arange(n) * (2 if interleaved else 1)
    b = a + (1 if interleaved else n)
    x = (y[..., a] + 1j * y[..., b]) * turn * mscale
    y[..., a], y[..., b] = x.real, x.imag
    return y


def norm_rope(x, w, eps, inv_freq, interleaved=False, mscale=1.0, norm=True, pos=None):
    """One of q, k [B, H, T, d], normalised by row, weighted, rotated."""
    x = np.asarray(x, dtype=np.float64)
    B, _, T, d = x.shape
    y = x
    if norm:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if w is None else np.asarray(w, dtype=np.float64))
    if inv_freq is None or len(inv_freq) == 0:
        return y
    return _rotate(y, _turns(np.zeros(B) if pos is None else pos, T, inv_freq), interleaved, mscale)


def norm_rope_backward(x, gy, w, eps, inv_freq, interleaved=False, mscale=1.0, norm=True, pos=None):
    """(dx, dw) from gy, the gradient of norm_rope's result."""
    x, u = np.asarray(x, dtype=np.float64), np.asarray(gy, dtype=np.float64)
    B, _, T, d = x.shape
    if inv_freq is not None and len(inv_freq):
        u = _rotate(u, _turns(np.zeros(B) if pos is None else pos, T, inv_freq).conj(), interleaved, mscale)
    if not norm:
        return u, None
    w = np.ones(d) if w is None else np.asarray(w, dtype=np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh = x * r
    return r * (u * w - xh * (u * w * xh).mean(-1, keepdims=True)), (u * xh).sum((0, 1, 2))
