"""The differential attention and its gradients in 64 bits, from the definition, with bounds of what roundings to bf16 can move.

For a (batch element, head), c = 1 / sqrt(d), P_s the causal softmax of c Q_s K_s^T, G the output's gradient, A = G V^T, D_s = rowsum(P_s (.) A):
    O = scale (P_1 - lambda P_2) V,  dV = scale (P_1 - lambda P_2)^T G,  T_s = P_s (.) (A - D_s),  dQ_s = c w_s T_s K_s,  dK_s = c w_s T_s^T Q_s,
    w = (scale, -lambda scale),  dlambda = -scale sum(P_2 (.) A)
"""
import math

import torch

HALF = 2.0 ** -8   # half a step of bf16, relative to the value, at most
SLACK = 2.0 ** -18  # exponentials, lse and fp32 sums, relative to the sum of magnitudes: exponents up to 2^5 are off by 2^5 2^-24 a few times over


def reference(q, k, v, g, B, L, h, dh, lam, scale):
    """q, k [B*L][2*h*dh], v, g [B*L][h*dh] -> {name: (value, bound of its error)} in 64 bits, laid out as the call's outputs."""
    two = lambda x: x.double().view(B, L, 2, h, dh).permute(2, 0, 3, 1, 4)  # noqa: E731  [2][B][h][L][dh]
    one = lambda x: x.double().view(B, L, h, dh).permute(0, 2, 1, 3)  # noqa: E731
    Q, K, V, G = two(q), two(k), one(v), one(g)
    c, w = 1.0 / math.sqrt(dh), (scale, -lam * scale)
    hidden = torch.ones(L, L, dtype=torch.bool, device=q.device).triu(1)
    P = torch.softmax((c * Q @ K.transpose(-1, -2)).masked_fill(hidden, -math.inf), -1)
    A = G @ V.transpose(-1, -2)
    O = P @ V
    D = (P * A).sum(-1, keepdim=True)
    T = P * (A - D)
    mix = P[0] - lam * P[1]
    T_ = lambda x: x.transpose(-1, -2)  # noqa: E731
    out, dv = scale * mix @ V, scale * T_(mix) @ G
    dq = torch.stack([c * w[s] * T[s] @ K[s] for s in (0, 1)])
    dk = torch.stack([c * w[s] * T_(T[s]) @ Q[s] for s in (0, 1)])
    # D comes from O in fp32, which comes from P in two bf16 parts: half a step of the half step that the first is off by
    off = (HALF * HALF + SLACK) * (G.abs() * (P @ V.abs())).sum(-1, keepdim=True)
    # every T is rounded to bf16 (up to 64 tokens: taken in two bf16 parts, half a step of half a step); the probability has SLACK, D has `off`; what
    # A - D is made of counts where they cancel
    near = HALF if L > 64 else HALF * HALF
    each = near * T.abs() + P * (off + SLACK * (A.abs() + D.abs()))
    e_dq = torch.stack([c * abs(w[s]) * each[s] @ K[s].abs() for s in (0, 1)])
    e_dk = torch.stack([c * abs(w[s]) * T_(each[s]) @ Q[s].abs() for s in (0, 1)])
    size = P[0] + abs(lam) * P[1]
    # heads of 64: P_1 - lambda P_2 is rounded once; of 128, where a stream follows the other: P_1 and lambda P_2 each, half a step of |P_1| and
    # one of |lambda P_2|, and those do not cancel as the values do
    e_dv = abs(scale) * T_(near * (mix.abs() if dh < 128 else size) + SLACK * size) @ G.abs()
    e_out = abs(scale) * (HALF * HALF + SLACK) * size @ V.abs()
    back2 = lambda x: x.permute(1, 3, 0, 2, 4).reshape(B * L, -1)  # noqa: E731
    back1 = lambda x: x.permute(0, 2, 1, 3).reshape(B * L, -1)  # noqa: E731
    final = lambda x, e: (x, e + HALF * (x.abs() + e))  # noqa: E731  (the output is bf16)
    terms = P[1] * A
    return {"out": final(back1(out), back1(e_out)), "dq": final(back2(dq), back2(e_dq)), "dk": final(back2(dk), back2(e_dk)), "dv": final(back1(dv), back1(e_dv)),
            "dlambda": (-scale * terms.sum().view(1), abs(scale) * SLACK * (terms.abs().sum() + (P[1] * D[1].abs()).sum()).view(1)),
            "streams": (back2(O), back2((HALF * HALF + SLACK) * P @ V.abs())),
            "lse": (torch.logsumexp((c * Q @ K.transpose(-1, -2)).masked_fill(hidden, -math.inf), -1).permute(1, 2, 0, 3) / math.log(2.0), None)}


def inputs(B, L, h, dh, seed, device, spread=1.0):
    r = torch.Generator().manual_seed(seed)
    n = lambda w, s=1.0: (torch.randn(B * L, w, generator=r) * s).to(torch.bfloat16).to(device)  # noqa: E731
    return n(2 * h * dh, spread), n(2 * h * dh), n(h * dh), n(h * dh, 0.03)
