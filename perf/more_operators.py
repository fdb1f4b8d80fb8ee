"""What a training step needs around the differential attention, as cases that can be timed and compared.

A case is a dict of plain values; `kind` says which entry points it goes through:

  attn    a training pass of the attention: `hgf.diff_attention_forward_train` and `hgf.diff_attention_backward`
  rotate  one `hgf.qk_norm_rotate`: the heads of Q and K normalised and rotated by their positions
  unrotate  one `hgf.qk_norm_rotate_backward`: the gradients of that
  clip    one `hgf.GradList.clip`: the norm over all gradients of some blocks, and the gradients scaled by it

The plain forms are elementary torch operations in fp32 on the same arrays (angles and the norm over all gradients in fp64).  Head
counts and widths are those of the attention elsewhere in this repository; gradients have the shapes of the blocks of `inputs.CONFIGS`.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6


def _attn(name, B, L, h, dh, out_scale=1.0):
    return {"name": name, "kind": "attn", "B": B, "L": L, "h": h, "dh": dh, "out_scale": out_scale}


def _rot(name, kind, n, h, kv, dh, *, rot=None, pairs=False, far=8192):
    """n tokens; Q has two streams of h heads, K two streams of kv heads; positions below `far`; `rot` of the dh dims are rotated."""
    return {"name": name, "kind": kind, "n": n, "h": h, "kv": kv, "dh": dh, "rot": dh if rot is None else rot, "pairs": pairs, "far": far}


def listed():
    return [
        # One short text: three launches whose time is latency.
        _attn("attn_b1_l61", 1, 61, 16, 64),
        # A few texts of a fine-tuning batch, padded to an odd length.
        _attn("attn_b3_l517", 3, 517, 16, 64, 0.5),
        # The ordinary training batch.
        _attn("attn_b4_l4096", 4, 4096, 16, 64),
        # Wide heads, a ragged length.
        _attn("attn_b2_l1500_d128", 2, 1500, 16, 128),
        # One long document.
        _attn("attn_b1_l16383_d128", 1, 16383, 8, 128),
        # A decode step's tokens, one for each sequence, far into their texts.
        _rot("rotate_n48", "rotate", 48, 16, 16, 64, far=131072),
        # The ordinary training batch, 4 x 4096 tokens.
        _rot("rotate_n16384", "rotate", 16384, 16, 16, 64, far=4096),
        # A prompt of an odd length: wide heads, four query heads on each of K's, neighbours paired, half of the dims rotated.
        _rot("rotate_n2999_d128_g4", "rotate", 2999, 16, 4, 128, rot=64, pairs=True),
        # The gradients of the ordinary training batch.
        _rot("unrotate_n16384", "unrotate", 16384, 16, 16, 64, far=4096),
        # Those of a short text with wide heads.
        _rot("unrotate_n700_d128", "unrotate", 700, 8, 8, 128, pairs=True, far=1024),
        # Gradients of the low-rank corrections and the gates alone (the ternary backbone frozen), in bf16: many small tensors.
        {"name": "clip_corrections", "kind": "clip", "d": 2048, "ffn": 5632, "r": 32, "blocks": 6, "bf16": True, "backbone": False},
        # All gradients of two blocks of the 1.2B class, as the layers' backward pass leaves them.
        {"name": "clip_blocks", "kind": "clip", "d": 2048, "ffn": 5632, "r": 32, "blocks": 2, "bf16": False, "backbone": True},
    ]


# ---- drawn cases ------------------------------------------------------------------------------------------
_MAX_ATTN = 8 * 16383 * 16383 * 128     # heads x pairs x width of the listed long document
_MAX_ROWS = 16384 * 4 * 16 * 64         # tokens x heads x width of the listed batch
_MAX_CLIP = 2 * (4 * 2048 * 2048 + 3 * 2048 * 5632 + 40 * 2048 * 32)


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "rotate", "unrotate", "clip"])
    while True:
        if kind == "attn":
            h, dh = rng.choice([(16, 64), (16, 64), (8, 128), (16, 128), (5, 64), (3, 128)])
            c = {"kind": kind, "B": rng.choice([1, 1, 2, 3, 4, 7]), "L": _log_int(rng, 2, 16383), "h": h, "dh": dh, "out_scale": rng.choice([1.0, 1.0, 0.5])}
            if c["B"] * h * c["L"] ** 2 * dh <= _MAX_ATTN and c["B"] * h * c["L"] * dh <= 4 * 16 * 4096 * 64:
                return c
        elif kind != "clip":
            h, dh = rng.choice([(16, 64), (16, 64), (8, 128), (16, 128), (5, 64), (3, 128)])
            c = {"kind": kind, "n": _log_int(rng, 1, 32768), "h": h, "kv": h // rng.choice([1, 1, 1, 2, 4]) or 1, "dh": dh,
                 "rot": rng.choice([dh, dh, dh // 2, dh // 4]), "pairs": rng.random() < 0.4, "far": _log_int(rng, 64, 1000000)}
            if c["n"] * 2 * (h + c["kv"]) * dh <= _MAX_ROWS:
                return c
        else:
            c = {"kind": kind, "d": 64 * _log_int(rng, 4, 64), "ffn": 64 * _log_int(rng, 8, 172), "r": rng.choice([16, 32, 48, 64]), "blocks": _log_int(rng, 1, 16),
                 "bf16": rng.random() < 0.4, "backbone": rng.random() < 0.6}
            if sum(map(math.prod, _gradients(c))) <= _MAX_CLIP:
                return c


def _gradients(c):
    """Shapes of the gradients of a clip case: the seven projections of each block, the norms of its heads and its lambda."""
    d, f, r = c["d"], c["ffn"], c["r"]
    shapes = []
    for _ in range(c["blocks"]):
        for k, n in [(d, d)] * 4 + [(d, f)] * 2 + [(f, d)]:
            shapes += ([(n, k)] if c["backbone"] else []) + [(r, k), (n, r), (n,)]
        shapes += [(64,), (64,), (1,)]
    return shapes


def _room(g):
    return -(-g.numel() // 64) * 64


def _pieces(flat, grads):
    at, out = 0, []
    for g in grads:
        out.append(flat[at:at + g.numel()].view(g.shape))
        at += _room(g)
    return out


def work(case):
    c = case
    if c["kind"] == "attn":
        width, pairs = c["h"] * c["dh"], c["L"] * (c["L"] + 1) // 2
        # q, k, v and the output's gradient in, the output and three gradients out, bf16.  Products: four forward, and backward the two
        # of the scores again (nothing of their size is kept), one for the probabilities' gradient, one for V's, two for Q's, two for K's.
        return {"bytes": 24 * c["B"] * c["L"] * width, "flops": 2.0 * 12 * c["B"] * pairs * width}
    if c["kind"] == "clip":
        n = sum(map(math.prod, _gradients(c)))
        return {"bytes": 2 * n * (2 if c["bf16"] else 4), "flops": 3.0 * n}
    n = c["n"] * 2 * (c["h"] + c["kv"]) * c["dh"]
    return {"bytes": (4 if c["kind"] == "rotate" else 6) * n + 4 * c["n"], "flops": (8.0 if c["kind"] == "rotate" else 16.0) * n}


# ---- inputs -----------------------------------------------------------------------------------------------
class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed) * 1000003 + 41)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device=DEV)


def prepare(case, seed):
    c, rand = case, _Rand(seed)
    s = {"case": c}
    if c["kind"] == "attn":
        n, w, dh = c["B"] * c["L"], c["h"] * c["dh"], c["dh"]
        # Heads whose rows are nearly even and heads that look at few tokens; small gradients, as a mean over tokens gives.
        sharp = (0.5 + 2.5 * rand.uniform(2 * c["h"], 1)).expand(-1, dh).reshape(-1)
        s["q"] = (rand.normal(n, 2 * w) * sharp).to(torch.bfloat16)
        s["k"], s["v"] = rand.normal(n, 2 * w).to(torch.bfloat16), rand.normal(n, w).to(torch.bfloat16)
        s["dout"] = (rand.normal(n, w) * 0.01).to(torch.bfloat16)
        s["lam"] = 0.8 - 0.6 * math.exp(-0.3 * dh) - 0.1 * random.Random(int(seed)).random()
        return s
    if c["kind"] == "clip":
        dt = torch.bfloat16 if c["bf16"] else torch.float32
        s["grads"] = [(rand.normal(*shape) * 0.01).to(dt) for shape in _gradients(c)]
        # what the optimiser reads: one buffer, in which each gradient begins at a multiple of 64; the gradients stay as they are
        s["flat"] = torch.zeros(sum(map(_room, s["grads"])), dtype=dt, device=DEV)
        s["out"] = _pieces(s["flat"], s["grads"])
        s["norm"] = torch.empty(1, device=DEV)
        s["max_norm"] = 1.0
        return s
    # Sequences of the batch begin at 0 or, cut into pieces, anywhere below `far`.
    n, r = c["n"], random.Random(int(seed) * 7 + c["n"])
    pos = []
    while len(pos) < n:
        at = r.randrange(c["far"])
        pos += range(at, min(at + r.randint(1, c["far"]), c["far"]))
    s["pos"] = torch.tensor(pos[:n], dtype=torch.int32, device=DEV)
    widths = {"q": 2 * c["h"] * c["dh"], "k": 2 * c["kv"] * c["dh"]}
    for name, w in widths.items():
        s[name] = (rand.normal(n, w) * (0.3 + 3.0 * rand.uniform(1, w))).to(torch.bfloat16)
        s["w" + name] = 1.0 + 0.2 * rand.normal(c["dh"])
        s["d" + name] = (rand.normal(n, w) * 0.01).to(torch.bfloat16)
        s[name + "_out"] = torch.empty_like(s[name])
    return s


# ---- plain forms ------------------------------------------------------------------------------------------
def _plain_attn(s):
    c = s["case"]
    B, L, h, dh, scale, lam = c["B"], c["L"], c["h"], c["dh"], c["out_scale"], s["lam"]
    split = lambda x, n: x.view(B, L, n, h, dh).permute(2, 0, 3, 1, 4).reshape(n, B * h, L, dh)  # noqa: E731
    Q, K, V, G = split(s["q"], 2), split(s["k"], 2), split(s["v"], 1)[0], split(s["dout"], 1)[0]
    hidden = torch.ones(L, L, dtype=torch.bool, device=DEV).triu(1)
    parts, dlam = [], torch.zeros((), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 28) // (L * L))
    for at in range(0, B * h, step):
        q, k, v, g = Q[:, at:at + step].float(), K[:, at:at + step].float(), V[at:at + step].float(), G[at:at + step].float() * scale
        x = (q @ k.transpose(-1, -2) / math.sqrt(dh)).masked_fill_(hidden, -math.inf)
        p = torch.exp(x - x.amax(-1, keepdim=True))
        p /= p.sum(-1, keepdim=True)
        a = p[0] - lam * p[1]
        out, dv = scale * (a @ v), a.transpose(-1, -2) @ g
        dp = g @ v.transpose(-1, -2)
        d = (p * dp).sum(-1, keepdim=True)
        dlam -= d[1].sum(dtype=torch.float64)
        ds = p * (dp - d) / math.sqrt(dh)
        ds[1] *= -lam
        parts.append((out, ds @ k, ds.transpose(-1, -2) @ q, dv))
    join = lambda i, n: torch.cat([p[i].view(n, -1, L, dh) for p in parts], 1).view(n, B, h, L, dh).permute(1, 3, 0, 2, 4).reshape(B * L, n * h * dh).to(torch.bfloat16)  # noqa: E731
    return {"out": join(0, 1), "dq": join(1, 2), "dk": join(2, 2), "dv": join(3, 1), "dlambda": dlam.float().view(1)}


def _turn(c, pos):
    """Cosine and sine of each token's angles, fp32 [n][1][rot / 2]."""
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV)
    angle = pos.double()[:, None] * 10000.0 ** (-2.0 * i / c["rot"])
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _rotated(x, c, cos, sin):
    half = c["rot"] // 2
    y = x.clone()
    a, b = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["pairs"] else (slice(0, half), slice(half, c["rot"]))
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., a] * sin + x[..., b] * cos
    return y


def _plain_rotate(s):
    c, out = s["case"], {}
    cos, sin = _turn(c, s["pos"])
    for name in ("q", "k"):
        x = s[name].float().view(c["n"], -1, c["dh"])
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["w" + name]
        out[name] = _rotated(x, c, cos, sin).view(c["n"], -1).to(torch.bfloat16)
    return out


def _plain_unrotate(s):
    c, out = s["case"], {}
    cos, sin = _turn(c, s["pos"])
    for name in ("q", "k"):
        x, g = s[name].float().view(c["n"], -1, c["dh"]), s["d" + name].float().view(c["n"], -1, c["dh"])
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        u, g = x * r, _rotated(g, c, cos, -sin)
        out["dw" + name] = (g * u).sum((0, 1), dtype=torch.float64).float()
        g = g * s["w" + name]
        out["d" + name] = (r * (g - u * (g * u).mean(-1, keepdim=True))).view(c["n"], -1).to(torch.bfloat16)
    return out


def _plain_clip(s):
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    factor = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0).float()
    for y, g in zip(s["out"], s["grads"]):
        y.copy_(g.float() * factor)
    s["norm"].copy_(norm)
    return {"norm": s["norm"], "grads": s["flat"]}


# ---- one pass ---------------------------------------------------------------------------------------------
def _own(s):
    """A pass by the framework's calls; outputs, what the backward pass needs and its workspace are made once, as a training loop does."""
    from paper_2602_05269_b200 import hgf
    c = s["case"]
    if c["kind"] == "attn":
        size = (c["B"], c["L"], c["h"], c["dh"], s["lam"], c["out_scale"])
        out, streams, lse = hgf.diff_attention_forward_train(s["q"], s["k"], s["v"], *size, out=s.get("out"), streams=s.get("streams"), lse=s.get("lse"),
                                                             flags=hgf.FLAG_OUT_BF16)
        g = hgf.diff_attention_backward(s["q"], s["k"], s["v"], s["dout"], streams, lse, *size, out=s.get("g"))
        s.update(out=out, streams=streams, lse=lse, g=g)
        return {"out": out, **{n: g[n] for n in ("dq", "dk", "dv", "dlambda")}}
    if c["kind"] == "clip":
        if "list" not in s:
            s["list"] = hgf.GradList(s["grads"], s["out"])
        s["list"].clip(s["max_norm"], norm=s["norm"])
        return {"norm": s["norm"], "grads": s["flat"]}
    how = {"eps": EPS, "base": 10000.0, "rotary_dim": c["rot"], "flags": hgf.FLAG_ROTATE_PAIRS if c["pairs"] else 0}
    if c["kind"] == "rotate":
        q, k = hgf.qk_norm_rotate(s["q"], s["k"], s["pos"], c["dh"], s["wq"], s["wk"], q_out=s["q_out"], k_out=s["k_out"], **how)
        return {"q": q, "k": k}
    s["g"] = g = hgf.qk_norm_rotate_backward(s["q"], s["k"], s["pos"], c["dh"], s["dq"], s["dk"], s["wq"], s["wk"], out=s.get("g"), **how)
    return {n: g[n] for n in ("dwq", "dq", "dwk", "dk")}


def run(state):
    if own:
        return _own(state)
    return {"attn": _plain_attn, "rotate": _plain_rotate, "unrotate": _plain_unrotate, "clip": _plain_clip}[state["case"]["kind"]](state)


# ---- the same in 64 bits ----------------------------------------------------------------------------------
def _exact_attn(c, s):
    """A head at a time, gradients by differentiation of the definition."""
    B, L, h, dh = c["B"], c["L"], c["h"], c["dh"]
    q, k, v, g = (s[n].view(B, L, -1, h, dh) for n in ("q", "k", "v", "dout"))
    lam = torch.tensor(s["lam"], dtype=torch.float64, device=DEV, requires_grad=True)
    res = {n: torch.empty(x.shape, dtype=torch.float64, device=DEV) for n, x in (("out", v), ("dq", q), ("dk", k), ("dv", v))}
    dlam, later = 0.0, torch.full((L, L), -math.inf, dtype=torch.float64, device=DEV).triu(1)
    for b in range(B):
        for a in range(h):
            Q, K, V = (x[b, :, :, a].double().requires_grad_() for x in (q, k, v))
            with torch.enable_grad():
                one, two = (torch.softmax(torch.einsum("id,jd->ij", Q[:, t], K[:, t]) * dh ** -0.5 + later, 1) for t in (0, 1))
                y = (one @ V[:, 0] - lam * (two @ V[:, 0])) * c["out_scale"]
                dQ, dK, dV, dl = torch.autograd.grad(y, (Q, K, V, lam), g[b, :, 0, a].double())
            for n, x in (("out", y.detach()[:, None]), ("dq", dQ), ("dk", dK), ("dv", dV)):
                res[n][b, :, :, a] = x
            dlam = dlam + dl
    return {**{n: x.reshape(B * L, -1) for n, x in res.items()}, "dlambda": dlam.detach().view(1)}


def _exact_rotate(c, x, w, pos):
    """x [n][heads][dh]: the norm, and each pair of dims as a complex number that is multiplied by e^(i angle)."""
    y = x / (x.pow(2).sum(-1, keepdim=True) / c["dh"] + EPS).sqrt() * w
    turned, rest = y[..., :c["rot"]], y[..., c["rot"]:]
    turned = turned.unflatten(-1, (-1, 2)) if c["pairs"] else turned.unflatten(-1, (2, -1)).transpose(-1, -2)
    theta = torch.exp(torch.arange(c["rot"] // 2, device=DEV, dtype=torch.float64) * (-2.0 / c["rot"] * math.log(10000.0)))
    z = torch.view_as_complex(turned.contiguous()) * torch.polar(torch.ones_like(theta), pos.double()[:, None, None] * theta)
    z = torch.view_as_real(z)
    return torch.cat([z.flatten(-2) if c["pairs"] else z.transpose(-1, -2).flatten(-2), rest], -1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "attn":
        return _exact_attn(c, s)
    if c["kind"] == "clip":
        total = sum(float((g.double() ** 2).sum()) for g in s["grads"]) ** 0.5
        factor = min(1.0, s["max_norm"] / (total + 1e-6))
        flat = torch.cat([torch.nn.functional.pad(g.double().flatten() * factor, (0, _room(g) - g.numel())) for g in s["grads"]])
        return {"norm": torch.tensor([total], dtype=torch.float64, device=DEV), "grads": flat}
    out = {}
    for name in ("q", "k"):
        x, w = s[name].double().view(c["n"], -1, c["dh"]), s["w" + name].double()
        if c["kind"] == "rotate":
            out[name] = _exact_rotate(c, x, w, s["pos"]).reshape(c["n"], -1)
            continue
        with torch.enable_grad():
            x.requires_grad_()
            w.requires_grad_()
            dx, dw = torch.autograd.grad(_exact_rotate(c, x, w, s["pos"]), (x, w), s["d" + name].double().view(c["n"], -1, c["dh"]))
        out["dw" + name], out["d" + name] = dw, dx.reshape(c["n"], -1)
    return out
