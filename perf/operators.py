"""Timed cases of the layer with a decay: the operators a model calls for it, in their plain form (elementary torch
operations in 32 bits) and through the public binding (`paper_2406_07368_b200.binding.Context`).

  prefill   `la_decay_prefill`: S_i = lam S_(i-1) + k_i v_i^T, o_i = scale q_i^T S_i over a prompt, lam = exp(log_decay[h])
  backward  `la_decay_backward`: the gradients of q, k, v and, where the sequence continues a state, of that state
  step      `la_decay_step`: one token for every sequence of the batch; the state is advanced in place
  rotate    `la_norm_rope`: each head's q and k divided by their RMS, weighted, rotated by their position
  unrotate  `la_norm_rope_backward`: the gradients of q, k and of the two weights

A case says the operator (kind), B (sequences), H (heads), T (tokens), d (head dimension), io ("bf16" or "f32").
prefill and backward add cont (the sequences continue a state) and ragged (the batch is padded: each sequence has a length
of its own); rotate and unrotate add rot (values of a head that are rotated), pairs ("half" or "interleaved") and far
(positions up to a million, frequencies scaled for a long context).
"""
from __future__ import annotations

import math

import torch

own = False

_IO = {"bf16": torch.bfloat16, "f32": torch.float32}
_CHUNK = 128           # tokens per chunk of the plain form
_EPS = 1e-6
_contexts = {}


def _decay(name, kind, B, T, H=32, d=128, io="bf16", cont=False, ragged=False):
    return {"name": name, "kind": kind, "B": B, "H": H, "T": T, "d": d, "io": io, "cont": cont, "ragged": ragged}


def _rotate(name, kind, B, T, H=32, d=128, io="bf16", rot=128, pairs="half", far=False):
    return {"name": name, "kind": kind, "B": B, "H": H, "T": T, "d": d, "io": io, "rot": rot, "pairs": pairs, "far": far}


def listed():
    return [
        # A single user's token: the inner step of interactive generation.
        _decay("step_one", "step", B=1, T=1),
        # The step of a serving batch (the batched_decode shapes).
        _decay("step_batch", "step", B=64, T=1),
        # One user's prompt, ragged, that continues an earlier part of the conversation (a prompt_gen shape).
        _decay("prompt_one", "prefill", B=1, T=1700, cont=True),
        # A batch of prompts (the llama7b_prefill shapes).
        _decay("prefill_batch", "prefill", B=4, T=2048),
        # A long document (the long_prefill shapes).
        _decay("prefill_long", "prefill", B=1, T=32768),
        # Prompts of different lengths, padded to the longest, of a model with heads of 64.
        _decay("prefill_padded", "prefill", B=7, T=777, H=12, d=64, ragged=True),
        # A small model in full precision (the prefill_fp32 shapes).
        _decay("prefill_fp32", "prefill", B=4, T=1000, H=12, d=64, io="f32"),
        # A training step's backward pass over a batch of sequences.
        _decay("train_batch", "backward", B=4, T=2048),
        # Full precision, the sequences continue a state (training by segments), padded.
        _decay("train_fp32", "backward", B=3, T=500, H=12, d=64, io="f32", cont=True, ragged=True),
        # The q and k of a serving batch's tokens: positions far out, frequencies scaled.
        _rotate("rotate_tokens", "rotate", B=64, T=1, far=True),
        # The q and k of a batch of prompts, half of each head rotated.
        _rotate("rotate_batch", "rotate", B=4, T=2048, rot=64),
        # ... and the gradients on the way back, interleaved pairs.
        _rotate("unrotate_batch", "unrotate", B=4, T=2048, pairs="interleaved"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _nameless(case):
    return {key: x for key, x in case.items() if key != "name"}


def draw(rng):
    kind = rng.choice(["prefill", "prefill", "backward", "backward", "step", "rotate", "unrotate"])
    d, io = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "f32"])
    H = _log_uniform(rng, 1, 32)
    row = H * d * (2 if io == "bf16" else 4)
    if kind == "step":
        B = _log_uniform(rng, 1, min(128, max(1, (32 << 20) // (H * d * d))))
        return _nameless(_decay("", kind, B, 1, H, d, io))
    T = _log_uniform(rng, 1, 16384)
    B = _log_uniform(rng, 1, min(64, max(1, (64 << 20) // (T * row))))
    if kind in ("rotate", "unrotate"):
        c = _rotate("", kind, B, T, H, d, io, rng.choice([d, d // 2, d // 4]), rng.choice(["half", "interleaved"]),
                    rng.random() < 0.5)
    else:
        c = _decay("", kind, B, T, H, d, io, rng.random() < 0.5, B > 1 and rng.random() < 0.4)
    return _nameless(c)


def _inv_freq(c):
    """Frequencies of the rotated pairs, 64 bits: base 10000, or for a long context the base raised eightfold and more
    (so that the slowest pair turns eight times more slowly)."""
    rot = c["rot"]
    base = 10000.0 * (8.0 ** (rot / (rot - 2)) if c["far"] and rot > 2 else 1.0)
    return base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    io, (B, H, T, d) = _IO[c["io"]], (c["B"], c["H"], c["T"], c["d"])

    def normal(*shape, scale=1.0, dtype=io):
        return (torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)

    def heads():
        """[B, H, T, d] as a projection leaves it: the heads of a token side by side."""
        return normal(B, T, H, d).transpose(1, 2)

    s = {"case": c}
    if c["kind"] in ("rotate", "unrotate"):
        # q and k of one projection's output [B, T, (q, k, v), H, d], not normalised yet
        qkv = normal(B, T, 3, H, d, scale=1.7)
        s["q"], s["k"] = qkv[:, :, 0].transpose(1, 2), qkv[:, :, 1].transpose(1, 2)
        s["wq"], s["wk"] = (1.0 + normal(d, scale=0.2, dtype=torch.float32) for _ in range(2))
        s["inv_freq"] = _inv_freq(c)
        s["pos"] = torch.randint(0, 1000000 if c["far"] else 2048, (B,), generator=gen, device="cuda")
        if c["kind"] == "unrotate":
            s["dq"], s["dk"] = heads(), heads()
        return s
    s["scale"] = d ** -0.5
    # the heads' memories: from a token or two to a few hundred, drawn around a geometric series
    jitter = torch.rand(H, generator=gen, device="cuda") * 0.5 + 0.75
    s["log_decay"] = -(2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda", dtype=torch.float32) / H)) * jitter
    if c["kind"] == "step":
        s["q"], s["k"], s["v"] = (normal(B, H, d) for _ in range(3))
        s["S"] = normal(B, H, d, d, scale=4.0, dtype=torch.float32)
        s["pos"] = torch.randint(1, 4096, (B,), generator=gen, device="cuda")
        return s
    s["q"], s["k"], s["v"] = heads(), heads(), heads()
    s["lens"] = torch.randint((T + 1) // 2, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if c["ragged"] else None
    s["S_in"] = normal(B, H, d, d, scale=4.0, dtype=torch.float32) if c["cont"] else None
    if c["kind"] == "backward":
        s["do"] = heads()
        s["dS_out"] = normal(B, H, d, d, scale=0.3, dtype=torch.float32) if c["cont"] else None
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _powers(g, n):
    """lam^n for integers n >= 0 (0 where n < 0), [H, *n.shape]."""
    p = torch.exp(g.view(-1, *[1] * n.dim()) * n.clamp(min=0))
    return torch.where(n >= 0, p, torch.zeros_like(p))


def _scan(q, k, v, g, S0, first):
    """o_i = q_i^T (sum_(j<=i) lam^(i-j) k_j v_j^T + lam^(i+first) S0) in chunks; fp32 [B, H, T, d]."""
    B, H, T, d = q.shape
    n = -(-T // _CHUNK)
    q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, n * _CHUNK - T)).view(B, H, n, _CHUNK, d) for x in (q, k, v))
    i, c = torch.arange(_CHUNK, device=q.device), torch.arange(n, device=q.device)
    inside = (q @ k.transpose(-1, -2)) * _powers(g, i[:, None] - i[None, :])[None, :, None]
    sums = (k * _powers(g, _CHUNK - 1 - i)[None, :, None, :, None]).transpose(-1, -2) @ v
    carry = _powers(g, (c[:, None] - c[None, :] - 1) * _CHUNK)               # [H, chunk, earlier chunk]
    before = (carry @ sums.reshape(B, H, n, d * d)).view(B, H, n, d, d)
    o = inside @ v + (q * _powers(g, i + 1)[None, :, None, :, None]) @ before
    o = o.view(B, H, n * _CHUNK, d)[:, :, :T]
    if S0 is not None:
        t = torch.arange(T, device=q.device)
        o = o + (q.view(B, H, n * _CHUNK, d)[:, :, :T] * _powers(g, t + first)[None, :, :, None]) @ S0
    return o


def _alive(s, T):
    """[B, T] of whether a token belongs to its sequence, and each sequence's length."""
    t = torch.arange(T, device="cuda")
    lens = s["lens"] if s["lens"] is not None else torch.full((s["q"].shape[0],), T, device="cuda", dtype=torch.int32)
    return t[None, :] < lens[:, None], lens.long()


def _plain_prefill(s):
    q, k, v = (s[n].float() for n in ("q", "k", "v"))
    g, T = s["log_decay"], q.shape[2]
    live, lens = _alive(s, T)
    q, k, v = (torch.where(live[:, None, :, None], x, torch.zeros_like(x)) for x in (q, k, v))
    o = _scan(q, k, v, g, s["S_in"], 1) * s["scale"]
    left = (lens[:, None] - 1 - torch.arange(T, device="cuda")).clamp(min=0)  # (a dead token's k is 0)
    S = (k * torch.exp(g[None, :, None] * left[:, None])[..., None]).transpose(-1, -2) @ v
    if s["S_in"] is not None:
        S = S + torch.exp(g[None, :] * lens[:, None])[..., None, None] * s["S_in"]
    return {"o": o.to(s["q"].dtype), "S_out": S}


def _plain_backward(s):
    q, k, v, do = (s[n].float() for n in ("q", "k", "v", "do"))
    g, T = s["log_decay"], q.shape[2]
    live, lens = _alive(s, T)
    q, k, v, do = (torch.where(live[:, None, :, None], x, torch.zeros_like(x)) for x in (q, k, v, do))
    # time backwards, each sequence from its own last token
    back = torch.where(live, lens[:, None] - 1 - torch.arange(T, device="cuda"), torch.arange(T, device="cuda"))
    at = back[:, None, :, None].expand(q.shape)
    rq, rk, rv, rdo = (x.gather(2, at) for x in (q, k, v, do))
    S0, D = s["S_in"], s["dS_out"]
    dq = _scan(do, v, k, g, None if S0 is None else S0.transpose(-1, -2), 1) * s["scale"]
    one = s["scale"]
    dk = _scan(rv, rdo, rq, g, None if D is None else D.transpose(-1, -2) / one, 0) * one
    dv = _scan(rk, rq, rdo, g, None if D is None else D / one, 0) * one
    out = {"dq": dq, "dk": dk.gather(2, at), "dv": dv.gather(2, at)}
    out = {n: torch.where(live[:, None, :, None], x, torch.zeros_like(x)).to(s["q"].dtype) for n, x in out.items()}
    if S0 is not None:
        t = torch.arange(1, T + 1, device="cuda")
        out["dS_in"] = ((q * _powers(g, t)[None, :, :, None]).transpose(-1, -2) @ do) * s["scale"] + torch.exp(
            g[None, :] * lens[:, None])[..., None, None] * D
    return out


def _plain_step(s):
    q, k, v, S = s["q"].float(), s["k"].float(), s["v"].float(), s["S"]
    S.mul_(torch.exp(s["log_decay"])[None, :, None, None])
    S.add_(k[..., :, None] * v[..., None, :])
    o = (q[..., :, None] * S).sum(-2) * s["scale"]
    s["pos"] += 1
    return {"o": o.to(s["q"].dtype), "S": S, "pos": s["pos"]}


def _angles(s, T):
    """cos and sin [B, 1, T, rot / 2]; the angles in 64 bits."""
    p = (s["pos"][:, None] + torch.arange(T, device="cuda")).double()
    a = torch.remainder(p[:, None, :, None] * s["inv_freq"], 2.0 * math.pi)
    return torch.cos(a).float(), torch.sin(a).float()


def _pairs(c, x):
    rot = c["rot"]
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if c["pairs"] == "interleaved" else (x[..., : rot // 2], x[..., rot // 2 : rot])


def _join(c, a, b, x):
    turned = torch.stack((a, b), -1).flatten(-2) if c["pairs"] == "interleaved" else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., c["rot"]:]), -1)


def _plain_rotate(s):
    c = s["case"]
    cos, sin = _angles(s, c["T"])

    def one(x, w):
        x = x.float()
        y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * w
        a, b = _pairs(c, y)
        return _join(c, a * cos - b * sin, b * cos + a * sin, y).to(_IO[c["io"]])

    return {"q": one(s["q"], s["wq"]), "k": one(s["k"], s["wk"])}


def _plain_unrotate(s):
    c = s["case"]
    cos, sin = _angles(s, c["T"])

    def one(x, dy, w):
        x, dy = x.float(), dy.float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS)
        xh = x * r
        a, b = _pairs(c, dy)
        u = _join(c, a * cos + b * sin, b * cos - a * sin, dy)
        wu = u * w
        dx = r * (wu - xh * (wu * xh).mean(-1, keepdim=True))
        return dx.to(_IO[c["io"]]), (u * xh).sum((0, 1, 2))

    dq, dwq = one(s["q"], s["dq"], s["wq"])
    dk, dwk = one(s["k"], s["dk"], s["wk"])
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


_PLAIN = {"prefill": _plain_prefill, "backward": _plain_backward, "step": _plain_step, "rotate": _plain_rotate,
          "unrotate": _plain_unrotate}


# ---- the framework's calls ------------------------------------------------------------------------------------------
def _context(c):
    """A program keeps one context for its layers."""
    from paper_2406_07368_b200 import binding

    key = (c["H"], c["d"], c["io"])
    if key not in _contexts:
        _contexts[key] = binding.Context(c["H"], c["d"], 1, io=c["io"])
    return _contexts[key]


def _own_prefill(s):
    c = s["case"]
    S = torch.empty(c["B"], c["H"], c["d"], c["d"], dtype=torch.float32, device="cuda")
    o = _context(c).la_decay_prefill(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], S_in=s["S_in"], S_out=S,
                                     lens=s["lens"])
    return {"o": o, "S_out": S}


def _own_backward(s):
    dS = torch.empty_like(s["S_in"]) if s["S_in"] is not None else None
    dq, dk, dv = _context(s["case"]).la_decay_backward(s["q"], s["k"], s["v"], s["do"], s["log_decay"], s["scale"],
                                                       S_in=s["S_in"], dS_out=s["dS_out"], dS_in=dS, lens=s["lens"])
    return {"dq": dq, "dk": dk, "dv": dv, **({"dS_in": dS} if dS is not None else {})}


def _own_step(s):
    o = _context(s["case"]).la_decay_step(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["S"], pos=s["pos"])
    return {"o": o, "S": s["S"], "pos": s["pos"]}


def _own_rotate(s):
    c = s["case"]
    q, k = _context(c).la_norm_rope(s["q"], s["k"], s["wq"], s["wk"], _EPS, s["inv_freq"],
                                    interleaved=c["pairs"] == "interleaved", pos=s["pos"])
    return {"q": q, "k": k}


def _own_unrotate(s):
    c = s["case"]
    dq, dk, dwq, dwk = _context(c).la_norm_rope_backward(s["q"], s["k"], s["dq"], s["dk"], s["wq"], s["wk"], _EPS,
                                                         s["inv_freq"], interleaved=c["pairs"] == "interleaved",
                                                         pos=s["pos"])
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


_OWN = {"prefill": _own_prefill, "backward": _own_backward, "step": _own_step, "rotate": _own_rotate,
        "unrotate": _own_unrotate}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


def work(case):
    B, H, T, d = case["B"], case["H"], case["T"], case["d"]
    e = 2 if case["io"] == "bf16" else 4
    rows, state = B * H * T, 4 * B * H * d * d
    if case.get("ragged"):
        rows = rows * 3 // 4                                # lengths are between half of T and T
    if case["kind"] == "step":
        return {"bytes": 2 * state + 4 * e * d * B * H, "flops": 5.0 * d * d * B * H}
    if case["kind"] == "rotate":
        return {"bytes": 4 * e * d * rows, "flops": 16.0 * d * rows}
    if case["kind"] == "unrotate":
        return {"bytes": 6 * e * d * rows, "flops": 32.0 * d * rows}
    short = min(T, 64)                                      # tokens that meet each other directly, the others by the state
    flops = rows * (2.0 * short * d + (4.0 * d * d if T > 64 or case["cont"] else 2.0 * d * d))
    if case["kind"] == "prefill":
        return {"bytes": 4 * e * d * rows + state * (2 if case["cont"] else 1), "flops": flops}
    return {"bytes": 7 * e * d * rows + (3 * state if case["cont"] else 0), "flops": 2.5 * flops}


# ---- 64 bits, from the definition -----------------------------------------------------------------------------------
def _exact_layer(s):
    """Outputs, the last state and, where there is a do, the gradients, of a sequence at a time: every pair of tokens."""
    c = s["case"]
    B, H, T, d = (c[n] for n in ("B", "H", "T", "d"))
    z = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")  # noqa: E731
    back = c["kind"] == "backward"
    got = {n: z(B, H, T, d) for n in (("dq", "dk", "dv") if back else ("o",))}
    got["dS_in" if back else "S_out"] = z(B, H, d, d)
    lens = [T] * B if s["lens"] is None else s["lens"].tolist()
    for b in range(B):
        L = lens[b]
        t = torch.arange(L, device="cuda", dtype=torch.float64)
        for h in range(H):
            g, scale = s["log_decay"][h].double(), s["scale"]
            q, k, v = (s[n][b, h, :L].double() for n in ("q", "k", "v"))
            do = s["do"][b, h, :L].double() if back else None
            S0 = s["S_in"][b, h].double() if s["S_in"] is not None else z(d, d)
            fade, left = torch.exp(g * (t + 1))[:, None], torch.exp(g * (L - 1 - t))[:, None]
            for lo in range(0, L, 2048):
                hi = min(L, lo + 2048)
                m = torch.exp((g * (t[lo:hi, None] - t[None, :hi])).clamp(max=0)) * (t[lo:hi, None] >= t[None, :hi]) * scale
                a = (q[lo:hi] @ k[:hi].T) * m
                if back:
                    e = (do[lo:hi] @ v[:hi].T) * m
                    got["dq"][b, h, lo:hi] = e @ k[:hi]
                    got["dk"][b, h, :hi] += e.T @ q[lo:hi]
                    got["dv"][b, h, :hi] += a.T @ do[lo:hi]
                else:
                    got["o"][b, h, lo:hi] = a @ v[:hi]
            if back:
                D = s["dS_out"][b, h].double() if s["dS_out"] is not None else z(d, d)
                got["dq"][b, h, :L] += scale * fade * (do @ S0.T)
                got["dk"][b, h, :L] += left * (v @ D.T)
                got["dv"][b, h, :L] += left * (k @ D)
                got["dS_in"][b, h] = torch.exp(g * L) * D + scale * (q * fade).T @ do
            else:
                got["o"][b, h, :L] += scale * fade * (q @ S0)
                got["S_out"][b, h] = torch.exp(g * L) * S0 + (k * left).T @ v
    if back and s["S_in"] is None:
        del got["dS_in"]
    return got


def _exact_rows(s):
    c = s["case"]
    p = (s["pos"][:, None] + torch.arange(c["T"], device="cuda")).double()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), p[:, None, :, None] * s["inv_freq"])
    n, rot = c["rot"] // 2, c["rot"]
    first = torch.arange(n, device="cuda") * (2 if c["pairs"] == "interleaved" else 1)
    second = first + (1 if c["pairs"] == "interleaved" else n)

    def rotated(y, turn):
        y = y.clone()
        x = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = x.real, x.imag
        return y

    got = {}
    for n_ in ("q", "k"):
        x, w = s[n_].double(), s["w" + n_].double()
        rms = (x.pow(2).sum(-1, keepdim=True) / c["d"] + _EPS).sqrt()
        if c["kind"] == "rotate":
            got[n_] = rotated(x / rms * w, turn)
        else:
            u = rotated(s["d" + n_].double(), turn.conj())
            got["dw" + n_] = (u * x / rms).flatten(0, 2).sum(0)
            along = (u * w * x).sum(-1, keepdim=True) / (c["d"] * rms.pow(3))
            got["d" + n_] = u * w / rms - x * along
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("rotate", "unrotate"):
        return _exact_rows(s)
    if case["kind"] in ("prefill", "backward"):
        return _exact_layer(s)
    S = torch.exp(s["log_decay"].double())[:, None, None] * s["S"].double()
    S = S + torch.einsum("bhi,bhj->bhij", s["k"].double(), s["v"].double())
    return {"o": torch.einsum("bhi,bhij->bhj", s["q"].double(), S) * s["scale"], "S": S, "pos": None}
