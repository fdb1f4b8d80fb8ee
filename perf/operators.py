"""Differential attention over an 8-bit paged K/V cache and the operators that keep the cache, as cases that can be timed and compared.

A case is a dict of plain values; `kind` says which entry points it goes through:

  attn    one `hgf.diff_attention_cached`: the new tokens of `S` sequences attend to the tokens that the cache holds
  append  one `hgf.cache_append` of new tokens, and one `hgf.cache_read` of the blocks that it touched
  read    one `hgf.cache_read`: ranges of tokens of `S` sequences as values
  pages   a step of a beam search: `hgf.cache_free` of the beams that lost, `hgf.cache_fork` of those that won, `hgf.cache_reserve` of the next pages

The plain forms are elementary torch operations in fp32 on the same arrays.  Head counts and widths are those of the differential
attention elsewhere in this repository (16 heads of 64, 8 heads of 128) and shared heads of the same widths.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = 64  # tokens of a page


def _attn(name, S, L, H, dh, *, ragged=True, group=1, m=1, bf16=True):
    return {"name": name, "kind": "attn", "S": S, "L": L, "H": H, "dh": dh, "group": group, "m": m, "ragged": ragged, "bf16": bf16}


def listed():
    return [
        # One conversation, a few sentences in: the call's latency.
        _attn("attn_s1_l200", 1, 200, 16, 64),
        # An ordinary decode batch of mixed lengths; the output stays in fp32.
        _attn("attn_s32_l2048_f32", 32, 2048, 16, 64, bf16=False),
        # One very long document: a single token's attention split over the whole chip.
        _attn("attn_s1_l131071", 1, 131071, 16, 64, ragged=False),
        # A full serving batch of wide heads: the cache's stream from memory.
        _attn("attn_s64_l4096_d128", 64, 4096, 16, 128, ragged=False),
        # Draft tokens being verified, four query heads on each K/V head.
        _attn("attn_s16_l2900_m5_g4", 16, 2900, 8, 128, group=4, m=5),
        # A piece of a long prompt over what is cached of it.
        _attn("attn_s2_l6000_m256", 2, 6000, 16, 64, m=256, bf16=False),
        # A decode step's tokens: one row for each sequence, now and then a block that is complete.
        {"name": "append_s64_m1", "kind": "append", "S": 64, "L": 1500, "H": 16, "dh": 64, "m": 1, "bf16": True},
        # Prompts that are admitted together.
        {"name": "append_s6_m1400", "kind": "append", "S": 6, "L": 256, "H": 16, "dh": 64, "m": 1400, "bf16": False},
        # The newest tokens of a few sequences.
        {"name": "read_s8_l100", "kind": "read", "S": 8, "L": 100, "H": 16, "dh": 64, "bf16": True},
        # Whole sequences, to be handed on.
        {"name": "read_s4_l8192_d128", "kind": "read", "S": 4, "L": 8192, "H": 8, "dh": 128, "bf16": False},
        # A beam search with four beams.
        {"name": "pages_s1_b4", "kind": "pages", "S": 1, "beams": 4, "L": 300, "H": 16, "dh": 64},
        # Many beam searches that step together.
        {"name": "pages_s48_b4", "kind": "pages", "S": 48, "beams": 4, "L": 4000, "H": 16, "dh": 64},
    ]


# ---- drawn cases ------------------------------------------------------------------------------------------
_MAX_CACHE = 64 * 4096 * 16 * 128      # tokens x heads x width of the largest listed attention
_MAX_PAIRS = 2 * 6000 * 256 * 16 * 64  # query rows x tokens x heads x width of the listed prompt piece


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "read", "pages"])
    H, dh = rng.choice([(16, 64), (16, 64), (8, 128), (16, 128), (5, 64), (4, 128)])
    while True:
        if kind == "attn":
            m = rng.choice([1, 1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 256)])
            c = {"kind": kind, "S": _log_int(rng, 1, 128), "L": _log_int(rng, 1, 131071), "H": H, "dh": dh, "group": rng.choice([1, 1, 1, 2, 4, 8]),
                 "m": m, "ragged": rng.random() < 0.7, "bf16": rng.random() < 0.6}
            pairs = c["S"] * c["L"] * m * H * c["group"] * dh
            if c["S"] * c["L"] * H * dh <= _MAX_CACHE and (m == 1 or pairs <= _MAX_PAIRS):
                return c
        elif kind == "append":
            c = {"kind": kind, "S": _log_int(rng, 1, 128), "L": _log_int(rng, 64, 4096), "H": H, "dh": dh, "m": rng.choice([1, 1, _log_int(rng, 2, 2000)]),
                 "bf16": rng.random() < 0.5}
            if c["S"] * (c["L"] + c["m"]) * H * dh <= _MAX_CACHE // 8 and c["S"] * c["m"] <= 8400:
                return c
        elif kind == "read":
            c = {"kind": kind, "S": _log_int(rng, 1, 64), "L": _log_int(rng, 1, 20000), "H": H, "dh": dh, "bf16": rng.random() < 0.5}
            if c["S"] * c["L"] * H * dh <= 4 * 8192 * 8 * 128:
                return c
        else:
            return {"kind": kind, "S": _log_int(rng, 1, 48), "beams": rng.randint(2, 5), "L": _log_int(rng, 1, 4000), "H": H, "dh": dh}


def _lengths(c):
    """Tokens that each sequence of the case holds; the first is as long as the case says."""
    r = random.Random("%(S)d %(L)d %(H)d %(dh)d" % c)
    S, L, kind = c["S"], c["L"], c["kind"]
    if kind == "attn":
        low = min(c["m"], L)
        return [L] + [r.randint(max(low, L // 3), L) if c["ragged"] else L for _ in range(S - 1)]
    if kind == "append" and c["m"] == 1:  # (every second sequence of the first eight completes a block)
        return [L // BLOCK * BLOCK + 63 if i in (0, 2, 4, 6) else r.randint(0, L) for i in range(S)]
    if kind == "append":
        return [r.choice([0, 0, r.randint(0, L // BLOCK) * BLOCK]) for _ in range(S)]
    if kind == "read":
        return [L] + [r.randint(max(1, L // 3), L) for _ in range(S - 1)]
    return [r.randint(max(1, L // 2), L) for _ in range(S * c["beams"])]


def _new_rows(c):
    """Rows that each sequence brings (attn: query tokens, append: tokens)."""
    r = random.Random("rows %(S)d %(L)d %(m)d" % c)
    return [c["m"]] + [c["m"] if c["m"] == 1 else r.randint(max(1, c["m"] // 3), c["m"]) for _ in range(c["S"] - 1)]


def work(case):
    c, lens = case, _lengths(case)
    H, dh = c["H"], c["dh"]
    full = lambda n: n // BLOCK  # noqa: E731
    held = lambda n: full(n) * (BLOCK * 3 * H * dh + 12 * H) + n % BLOCK * 6 * H * dh  # noqa: E731  bytes of a sequence's cache
    if c["kind"] == "attn":
        rows, heads = _new_rows(c), H * c["group"]
        pairs = sum(max(0, n - m + j + 1) for n, m in zip(lens, rows) for j in range(m))
        return {"bytes": sum(map(held, lens)) + sum(rows) * heads * dh * (4 + (2 if c["bf16"] else 4)), "flops": 8.0 * dh * heads * pairs}
    if c["kind"] == "append":
        rows = _new_rows(c)
        done = [full(n + m) - full(n) for n, m in zip(lens, rows)]
        back = sum(n + m - full(n) * BLOCK for n, m in zip(lens, rows))
        write = sum(d * (BLOCK * 3 * H * dh + 12 * H) for d in done) + sum(((n + m) % BLOCK if d else m) * 6 * H * dh for n, m, d in zip(lens, rows, done))
        return {"bytes": sum(rows) * 6 * H * dh + 2 * write + back * 3 * H * dh * (2 if c["bf16"] else 4), "flops": 0}
    if c["kind"] == "read":
        return {"bytes": sum(map(held, lens)) + sum(lens) * 3 * H * dh * (2 if c["bf16"] else 4), "flops": 0}
    forks = c["S"] * (c["beams"] - 1)
    n = sum(lens) / len(lens)
    return {"bytes": forks * (n % BLOCK * 12 * H * dh + 24 * full(n)) + 8 * len(lens) * full(c["L"] + BLOCK), "flops": 0}


# ---- inputs -----------------------------------------------------------------------------------------------
class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed) * 1000003 + 29)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV)

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device=DEV).int()


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _cache(c, rand, lens, room, spare=0):
    """A cache whose slots hold `lens` tokens of N(0, 1) values, each with pages for `room` tokens, in pages of no order."""
    H, dh, n = c["H"], c["dh"], len(lens)
    held = [max(a // BLOCK, r // BLOCK) for a, r in zip(lens, room)]
    n_pages, max_pages = sum(held) + spare, max(max(held), max(r // BLOCK for r in room), 1) + 1
    n_pages = max(n_pages, 1)
    codes = torch.empty((n_pages, H, 3 * BLOCK * dh), dtype=torch.int8, device=DEV)
    scales = torch.zeros((n_pages, H, 4), device=DEV)
    step = max(1, (1 << 28) // (H * 3 * BLOCK * dh))
    for at in range(0, n_pages, step):  # (any order of iid values is one: they are drawn in the order that the page has)
        x = rand.normal(min(step, n_pages - at), H, 3, BLOCK * dh)
        top = x.abs().amax(-1)
        codes[at:at + step] = torch.round(127.0 * x / top[..., None]).to(torch.int8).flatten(2)
        scales[at:at + step, :, :3] = top / 127.0
    order = rand.perm(n_pages)[: sum(held)].cpu()
    table = torch.zeros((n, max_pages), dtype=torch.int32)
    at = 0
    for i, h in enumerate(held):
        table[i, :h] = order[at:at + h]
        at += h
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[order.long()] = 1
    return {"H": H, "dh": dh, "codes": codes, "scales": scales, "open": rand.normal(n, H, 3, BLOCK, dh).to(torch.bfloat16), "table": table.to(DEV), "held": _ints(held),
            "length": _ints(lens), "refs": refs.to(DEV), "arrivals": torch.zeros(n, dtype=torch.int32, device=DEV)}


def _starts(rows):
    at = [0]
    for m in rows:
        at.append(at[-1] + m)
    return at


def prepare(case, seed):
    c, rand, lens = case, _Rand(seed), _lengths(case)
    H, dh = c["H"], c["dh"]
    s = {"case": c}
    if c["kind"] == "pages":
        s["cache"] = _cache(c, rand, lens, [n + BLOCK for n in lens], spare=len(lens) * (c["L"] // BLOCK + 2))
        r, win, lose, frm = random.Random(int(seed)), [], [], []
        for i in range(c["S"]):
            w = r.randrange(c["beams"])
            out = [i * c["beams"] + b for b in range(c["beams"]) if b != w]
            win.append(i * c["beams"] + w)
            lose += out
            frm += [i * c["beams"] + w] * len(out)
        every = win + lose
        s.update(lose=_ints(lose), win=_ints(frm), every=_ints(every),
                 ahead=_ints([lens[w] + BLOCK for w in win] + [lens[w] + BLOCK for w in frm]), granted=torch.zeros(len(every), dtype=torch.int32, device=DEV))
        return s
    rows = _new_rows(c) if c["kind"] in ("attn", "append") else lens
    s["cache"] = _cache(c, rand, lens, [n + m for n, m in zip(lens, rows)] if c["kind"] == "append" else lens)
    s["slots"] = rand.perm(len(lens))  # the batch's order is not the slots'
    of = s["slots"].tolist()
    rows, lens = ([rows[j] for j in of] if c["kind"] != "read" else [lens[j] for j in of]), [lens[j] for j in of]
    at = _starts(rows)
    s["starts"] = _ints(at)
    dt = torch.bfloat16 if c["bf16"] else torch.float32
    if c["kind"] == "attn":
        heads = H * c["group"]
        s["q"] = rand.normal(at[-1], 2 * heads * dh).to(torch.bfloat16)
        s["lam"] = 0.8 - 0.6 * math.exp(-0.3 * dh)
        s["out"] = torch.empty((at[-1], heads * dh), dtype=dt, device=DEV)
        s["longest"], s["most"] = max(lens), max(rows)
        return s
    first = [0] * len(lens)
    if c["kind"] == "append":
        # K with a few channels that are larger than the others, as projections of such activations have
        wide = 1.0 + 7.0 * (torch.rand(2 * H * dh, generator=rand.g, device=DEV) < 0.02)
        s["k"] = (rand.normal(at[-1], 2 * H * dh) * wide).to(torch.bfloat16)
        s["v"] = rand.normal(at[-1], H * dh).to(torch.bfloat16)
        s["before"] = _ints(lens)
        s["done"] = torch.zeros(len(lens), dtype=torch.int32, device=DEV)
        first = [n // BLOCK * BLOCK for n in lens]
        # which blocks become complete (sequence of the batch, block) and which rows stay open (sequence, token)
        s["blocks"] = _ints([[i, b] for i, (n, m) in enumerate(zip(lens, rows)) for b in range(n // BLOCK, (n + m) // BLOCK)] or [[0, 0]][:0]).view(-1, 2)
        s["tails"] = _ints([[i, p] for i, (n, m) in enumerate(zip(lens, rows)) for p in range(max(n, (n + m) // BLOCK * BLOCK), n + m)]).view(-1, 2)
        at = _starts([n + m - f for n, m, f in zip(lens, rows, first)])
    # what is read back: (sequence, token) of each row
    s["first"], s["read_starts"] = _ints(first), _ints(at)
    s["read_of"] = torch.cat([torch.stack([torch.full((b - a,), i), f + torch.arange(b - a)], 1) for i, (f, a, b) in enumerate(zip(first, at, at[1:]))]).to(DEV)
    s["k_out"] = torch.empty((at[-1], 2 * H * dh), dtype=dt, device=DEV)
    s["v_out"] = torch.empty((at[-1], H * dh), dtype=dt, device=DEV)
    return s


# ---- plain forms ------------------------------------------------------------------------------------------
# A page holds, for each head, the codes of K1, K2 [64 tokens][dh] and of V transposed [dh][64 tokens], each as tiles of 16 rows by 32
# columns: with row 16 i + 8 a + g and column 32 j + 16 h + 4 t + b, byte ((i, j), g, t, h, a, b).  Eight values of an open row r are
# stored at place (their index) ^ (r & 7).
def _page_values(codes, scales, dh):
    """codes [..., H, 3 * 64 * dh], scales [..., H, 4] -> K1, K2, V [..., H, 64, dh] in fp32."""
    lead = codes.shape[:-1]
    n = len(lead)
    d = list(range(n))
    k = codes[..., : 2 * BLOCK * dh].reshape(*lead, 2, 4, dh // 32, 8, 4, 2, 2, 4).permute(*d, n, n + 1, n + 6, n + 3, n + 2, n + 5, n + 4, n + 7)
    k = k.reshape(*lead, 2, BLOCK, dh).float() * scales[..., :2, None, None]
    v = codes[..., 2 * BLOCK * dh:].reshape(*lead, dh // 16, 2, 8, 4, 2, 2, 4).permute(*d, n + 1, n + 4, n + 3, n + 6, n, n + 5, n + 2)
    return k[..., 0, :, :], k[..., 1, :, :], v.reshape(*lead, BLOCK, dh).float() * scales[..., 2, None, None]


def _page_codes(c, dh):
    """codes of K1, K2, V [n, H, 3, 64, dh] -> [n, H, 3 * 64 * dh] as a page holds them."""
    n, H = c.shape[:2]
    k = c[:, :, :2].reshape(n, H, 2, 4, 2, 8, dh // 32, 2, 4, 4).permute(0, 1, 2, 3, 6, 5, 8, 7, 4, 9).reshape(n, H, -1)
    v = c[:, :, 2].transpose(-1, -2).reshape(n, H, dh // 16, 2, 8, 2, 2, 4, 4).permute(0, 1, 2, 5, 4, 7, 6, 3, 8).reshape(n, H, -1)
    return torch.cat([k, v], -1)


def _swizzled(x, dh):
    """[..., 64, dh] with the eights of each row in the order of the open rows, or back."""
    r = torch.arange(BLOCK, device=DEV)[:, None]
    at = torch.arange(dh // 8, device=DEV)[None] ^ (r & 7)
    return x.reshape(*x.shape[:-1], dh // 8, 8)[..., r, at, :].reshape(x.shape)


def _plain_attn(s):
    c, k = s["case"], s["cache"]
    H, dh, G, M = c["H"], c["dh"], c["group"], s["most"]
    slots, starts = s["slots"].long(), s["starts"].long()
    S, P, n = slots.numel(), -(-s["longest"] // BLOCK), s["q"].shape[0]
    length = k["length"][slots].long()
    full = length // BLOCK
    pages = k["table"][slots, :P].long().clamp(0, k["codes"].shape[0] - 1)
    pages = torch.where(torch.arange(pages.shape[1], device=DEV)[None] < full[:, None], pages, 0)
    K1, K2, V = (x.transpose(1, 2).reshape(S, H, -1, dh) for x in _page_values(k["codes"][pages], k["scales"][pages], dh))
    o = _swizzled(k["open"][slots], dh).float()
    K1, K2, V = torch.cat([K1, o[:, :, 0]], 2), torch.cat([K2, o[:, :, 1]], 2), torch.cat([V, o[:, :, 2]], 2)
    j = torch.arange(pages.shape[1] * BLOCK, device=DEV)[None]
    pos = torch.cat([j.expand(S, -1), full[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)], 1)
    held = torch.cat([j < full[:, None] * BLOCK, pos[:, -BLOCK:] < length[:, None]], 1)
    # the rows of each sequence side by side: [S, M]
    row = starts[:-1, None] + torch.arange(M, device=DEV)
    there = row < starts[1:, None]
    q = s["q"].float()[torch.where(there, row, 0)].view(S, M, 2, H, G, dh).permute(2, 0, 3, 1, 4, 5).reshape(2, S, H, M * G, dh)
    qpos = length[:, None] - (starts[1:] - starts[:-1])[:, None] + torch.arange(M, device=DEV)
    sees = (held[:, None] & (pos[:, None] <= qpos[..., None])).repeat_interleave(G, 1)[:, None]
    V = torch.where(held[:, None, :, None], V, 0.0)

    def stream(q, K):
        x = torch.where(sees, q @ K.transpose(-1, -2) / math.sqrt(dh), -math.inf)
        top = x.amax(-1, keepdim=True)
        p = torch.exp(x - torch.where(top.isinf(), 0.0, top))
        total = p.sum(-1, keepdim=True)
        return torch.where(total > 0, p @ V / total, 0.0)

    y = (stream(q[0], K1) - s["lam"] * stream(q[1], K2)).view(S, H, M, G, dh).permute(0, 2, 1, 3, 4).reshape(S * M, H * G * dh)
    # back to the batch's rows
    seq = torch.searchsorted(starts[1:], torch.arange(n, device=DEV), right=True)
    return y[seq * M + torch.arange(n, device=DEV) - starts[seq]].to(s["out"].dtype)


def _plain_read(s):
    k, dh, H = s["cache"], s["case"]["dh"], s["case"]["H"]
    slot, pos = s["slots"].long()[s["read_of"][:, 0]], s["read_of"][:, 1]
    full = (k["length"][slot] // BLOCK).long()
    block, at = pos // BLOCK, pos % BLOCK
    page = torch.where(block < full, k["table"][slot, block.clamp(max=k["table"].shape[1] - 1)].long(), 0)
    kinds = torch.arange(2, device=DEV)
    # bytes of (token, dim) in a page
    d = torch.arange(dh, device=DEV)
    tile = lambda r, col, cols: ((r // 16 * (cols // 32) + col // 32) * 32 + r % 8 * 4 + col % 16 // 4) * 16 + col % 32 // 16 * 8 + r % 16 // 8 * 4 + col % 4  # noqa: E731
    kb = kinds[:, None] * BLOCK * dh + tile(at[:, None, None], d, dh)
    vb = 2 * BLOCK * dh + tile(d, at[:, None], BLOCK)
    h = torch.arange(H, device=DEV)
    kc = k["codes"][page[:, None, None, None], h[:, None], kb[:, :, None]].float() * k["scales"][page][:, :, :2].transpose(1, 2)[..., None]
    vc = k["codes"][page[:, None, None], h[:, None], vb[:, None]].float() * k["scales"][page][:, :, 2, None]
    o = k["open"][slot, :, :, at].float().view(-1, H, 3, dh // 8, 8)
    o = o.gather(3, (torch.arange(dh // 8, device=DEV) ^ (at[:, None] & 7))[:, None, None, :, None].expand_as(o)).reshape(-1, H, 3, dh)
    closed = (block < full)[:, None, None]
    dt = s["k_out"].dtype
    return {"k": torch.where(closed[..., None], kc, o[:, :, :2].transpose(1, 2)).reshape(len(pos), -1).to(dt), "v": torch.where(closed, vc, o[:, :, 2]).reshape(len(pos), -1).to(dt)}


def _plain_append(s):
    k, c = s["cache"], s["case"]
    H, dh, n = c["H"], c["dh"], s["k"].shape[0]
    slots, starts, before = s["slots"].long(), s["starts"].long(), s["before"].long()
    S = slots.numel()
    new = torch.cat([s["k"].view(n, 2, H, dh), s["v"].view(n, 1, H, dh)], 1)
    old = _swizzled(k["open"][slots], dh).permute(0, 3, 2, 1, 4).reshape(S * BLOCK, 3, H, dh)
    rows = torch.cat([new, old])
    seq, block = s["blocks"].long().unbind(1)
    pos = block[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)
    x = rows[torch.where(pos >= before[seq][:, None], starts[seq][:, None] + pos - before[seq][:, None], n + seq[:, None] * BLOCK + pos % BLOCK)].float()
    x = x.permute(0, 3, 2, 1, 4)  # block, head, tensor, token, dim
    top = x.abs().amax((3, 4))
    codes = torch.where(top[..., None, None] > 0, torch.round(127.0 * x / top[..., None, None]), 0.0).to(torch.int8)
    page = k["table"][slots[seq], block].long()
    k["codes"][page] = _page_codes(codes, dh)
    k["scales"][page, :, :3] = top / 127.0
    seq, pos = s["tails"].long().unbind(1)
    at = torch.arange(dh // 8, device=DEV) ^ (pos[:, None] & 7)
    put = new[starts[seq] + pos - before[seq]].transpose(1, 2).reshape(-1, H, 3, dh // 8, 8)
    k["open"][slots[seq], :, :, pos % BLOCK] = put.gather(3, at[:, None, None, :, None].expand_as(put)).reshape(-1, H, 3, dh)
    k["length"][slots] = (before + starts[1:] - starts[:-1]).int()
    s["done"].fill_(1)


def _plain_pages(s):
    k, n_pages, width = s["cache"], s["cache"]["refs"].numel(), s["cache"]["table"].shape[1]
    col = torch.arange(width, device=DEV)
    refs = torch.cat([k["refs"], k["refs"].new_zeros(1)])  # (the last takes what concerns no page)
    lose, win, every = s["lose"].long(), s["win"].long(), s["every"].long()
    # free
    has = col < k["held"][lose][:, None]
    refs.index_add_(0, torch.where(has, k["table"][lose], n_pages).flatten().long(), k["refs"].new_full((has.numel(),), -1))
    k["held"][lose] = 0
    k["length"][lose] = 0
    # fork
    full = k["length"][win] // BLOCK
    has = col < full[:, None]
    refs.index_add_(0, torch.where(has, k["table"][win], n_pages).flatten().long(), k["refs"].new_ones(has.numel()))
    k["table"][lose] = torch.where(has, k["table"][win], k["table"][lose])
    rows = torch.arange(BLOCK, device=DEV) < (k["length"][win] % BLOCK)[:, None]
    k["open"][lose] = torch.where(rows[:, None, None, :, None], k["open"][win], k["open"][lose])
    k["held"][lose], k["length"][lose] = full, k["length"][win]
    # reserve: the lowest free pages, in the order of the list, until one request cannot be met (later ones get none, but may need none)
    refs[n_pages] = 1
    free = torch.sort((refs != 0).int(), stable=True)[1]
    need = (s["ahead"] // BLOCK - k["held"][every]).clamp(min=0) * (s["ahead"] // BLOCK <= width)
    upto = need.cumsum(0)
    met = ((need == 0) | (upto <= (refs[:n_pages] == 0).sum())) & (s["ahead"] // BLOCK <= width)
    at = col - k["held"][every][:, None]
    gets = (at >= 0) & (at < need[:, None]) & met[:, None]
    page = torch.where(gets, free[((upto - need)[:, None] + at).clamp(0, n_pages)].int(), n_pages)
    refs[page.flatten().long()] = 1
    k["table"][every] = torch.where(gets, page, k["table"][every])
    k["held"][every] += need * met
    k["refs"].copy_(refs[:n_pages])
    s["granted"].copy_(met.int())


# ---- one pass ---------------------------------------------------------------------------------------------
def _handle(s):
    """The framework's cache object on the state's arrays (made once, as a program keeps it)."""
    from paper_2602_05269_b200 import hgf
    if "handle" not in s:
        k = s["cache"]
        s["handle"] = hgf.KVCache.of(k["H"], k["dh"], **{n: v for n, v in k.items() if n not in ("H", "dh")})
        if "q" in s:
            s["workspace"] = torch.empty(hgf.cached_workspace_bytes(s["handle"], s["slots"].numel(), s["q"].shape[0], s["case"]["H"] * s["case"]["group"]),
                                         dtype=torch.uint8, device=DEV)
    return hgf, s["handle"]


def run(state):
    s, kind = state, state["case"]["kind"]
    if kind == "attn":
        if not own:
            return _plain_attn(s)
        hgf, cache = _handle(s)
        return hgf.diff_attention_cached(cache, s["q"], s["slots"], s["starts"], s["lam"], out=s["out"], workspace=s["workspace"],
                                         flags=hgf.FLAG_OUT_BF16 if s["case"]["bf16"] else 0)
    if kind == "read" or kind == "append":
        k = s["cache"]
        if kind == "append":  # (the sequences are as they were before these tokens, as after tokens that were taken back)
            k["length"][s["slots"].long()] = s["before"]
        if own:
            hgf, cache = _handle(s)
            if kind == "append":
                hgf.cache_append(cache, s["k"], s["v"], s["slots"], s["starts"], done=s["done"])
            hgf.cache_read(cache, s["slots"], s["first"], s["read_starts"], k=s["k_out"], v=s["v_out"])
            out = {"k": s["k_out"], "v": s["v_out"]}
        else:
            if kind == "append":
                _plain_append(s)
            out = _plain_read(s)
        return {**out, "length": k["length"], "scales": k["scales"], "open": k["open"], "done": s["done"]} if kind == "append" else out
    k = s["cache"]
    if own:
        hgf, cache = _handle(s)
        hgf.cache_free(cache, s["lose"])
        hgf.cache_fork(cache, s["win"], s["lose"])
        hgf.cache_reserve(cache, s["every"], s["ahead"], granted=s["granted"])
    else:
        _plain_pages(s)
    return {n: k[n] for n in ("table", "held", "length", "refs", "open")} | {"granted": s["granted"]}


# ---- the same in 64 bits ----------------------------------------------------------------------------------
def _sequence(k, slot, length, dh):
    """K1, K2, V [H, length, dh] of a slot in 64 bits, found byte by byte."""
    H = k["codes"].shape[1]
    tok, d = torch.arange(length, device=DEV)[:, None], torch.arange(dh, device=DEV)[None]
    j, out = tok % BLOCK, []
    page = k["table"][slot].long()[(tok // BLOCK).clamp(max=k["table"].shape[1] - 1)]
    closed = (tok < length // BLOCK * BLOCK)[None]
    page = torch.where(closed[0], page, 0)
    for n in range(3):
        r, col, cols = (j, d, dh) if n < 2 else (d, j, BLOCK)
        byte = n * BLOCK * dh + (r // 16 * (cols // 32) + col // 32) * 512 + (r % 8) * 64 + (col // 4 % 4) * 16 + (col // 16 % 2) * 8 + (r // 8 % 2) * 4 + col % 4
        flat = k["codes"].view(-1)
        at = (page * H)[None] + torch.arange(H, device=DEV)[:, None, None]
        x = flat[at * (3 * BLOCK * dh) + byte].double() * k["scales"].view(-1)[at * 4 + n].double()
        o = k["open"][slot, :, n].double()
        o = o[:, j, (d // 8 ^ (j & 7)) * 8 + d % 8]
        out.append(torch.where(closed, x, o))
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    k, H, dh = s["cache"], c["H"], c["dh"]
    if c["kind"] == "pages":
        return None  # nothing is computed: whole numbers and copies
    slots, starts = s["slots"].tolist(), s["starts"].tolist()
    length = k["length"].tolist()
    if c["kind"] == "attn":
        G, ys = c["group"], []
        for i, slot in enumerate(slots):
            m, n = starts[i + 1] - starts[i], length[slot]
            K1, K2, V = _sequence(k, slot, n, dh)
            q = s["q"][starts[i]:starts[i + 1]].double().view(m, 2, H, G, dh)
            sees = torch.arange(n, device=DEV)[None] <= (n - m + torch.arange(m, device=DEV))[:, None]
            a = [torch.softmax(torch.einsum("mhgd,hnd->hgmn", q[:, j], K).div(math.sqrt(dh)).masked_fill(~sees, -math.inf), -1) for j, K in enumerate((K1, K2))]
            y = torch.einsum("hgmn,hnd->mhgd", a[0], V) - s["lam"] * torch.einsum("hgmn,hnd->mhgd", a[1], V)
            ys.append(y.nan_to_num(0.0).reshape(m, -1))  # (a row that sees nothing is zero)
        return torch.cat(ys)
    ks, vs, scales = [], [], k["scales"].double().clone() if c["kind"] == "append" else None
    first = s["first"].tolist()
    for i, slot in enumerate(slots):
        x = torch.stack(_sequence(k, slot, length[slot], dh), 1)  # H, 3, tokens, dh
        if c["kind"] == "append":
            n0, a, b = length[slot], starts[i], starts[i + 1]
            new = torch.cat([s["k"][a:b].view(b - a, 2, H, dh), s["v"][a:b].view(b - a, 1, H, dh)], 1).double().permute(2, 1, 0, 3)
            x = torch.cat([x, new], 2)
            for blk in range(n0 // BLOCK, (n0 + b - a) // BLOCK):
                part = x[:, :, blk * BLOCK:(blk + 1) * BLOCK]
                top = part.abs().amax((2, 3), keepdim=True)
                part.copy_(torch.round(127.0 * part / top) * top / 127.0)
                scales[int(k["table"][slot, blk]), :, :3] = top[..., 0, 0] / 127.0
        x = x[:, :, first[i]:]
        ks.append(x[:, :2].permute(2, 1, 0, 3).reshape(x.shape[2], -1))
        vs.append(x[:, 2].transpose(0, 1).reshape(x.shape[2], -1))
    return {"k": torch.cat(ks), "v": torch.cat(vs), **({"length": None, "scales": scales, "open": None, "done": None} if scales is not None else {})}
