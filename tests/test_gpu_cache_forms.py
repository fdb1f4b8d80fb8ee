"""Cached attention (hgf_diff_attention_cached) gives the same answer in each of its forms: single tokens, tiles of eight, of sixteen and of 128 rows.

Which form a call takes goes by its rows times the heads that share a K/V head, per entry of its list; entries -1 without rows set that average here."""
import numpy as np
import pytest
import torch

from cache_reference import BLOCK, attention, rows
from paper_2602_05269_b200.inputs import bf16_bits_to_f32, f32_to_bf16_bits
from test_gpu_cache import Pair, bf16, hgf, ints  # noqa: F401  (hgf is the fixture)

pytestmark = pytest.mark.gpu

AVERAGES = [1, 8, 16, 32, 300]


def call(p, q, slot, n, average, out_bf16, group=1, lam=0.5):
    """The last n tokens of `slot`, in the form for `average` rows times heads an entry: [rows of q][heads][dh] in binary32, and the output as it came."""
    idle = -(-n * group // average) - 1
    flags = p.hgf.FLAG_OUT_BF16 if out_bf16 else 0
    out = p.hgf.diff_attention_cached(p.cache, bf16(q), ints([slot] + [-1] * idle), ints([0] + [n] * (idle + 1)), lam, flags=flags)
    return out.float().cpu().numpy().reshape(len(q), -1, p.dh), out


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("average", AVERAGES)
def test_bf16_output_is_the_rounding_of_binary32(hgf, dh, group, average):  # noqa: F811
    """The type of the output says how the output is rounded, and nothing of how it is computed."""
    p = Pair(hgf, 2, dh, n_pages=120, n_slots=3, max_pages=60)
    p.fill([700, 60, 3333])
    n = {1: 60, 8: 5, 16: 9, 32: 40, 300: 130}[average]
    for slot, spread in ((0, 1.0), (1, 3.0), (2, 1.0), (2, 0.1)):
        q = rows(p.rng, n, 4 * group * dh, spread)
        one, two = (call(p, q, slot, n, average, b, group=group, lam=0.7)[1] for b in (False, True))
        assert torch.equal(one.bfloat16(), two)
    hgf.check_status()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("average", AVERAGES)
@pytest.mark.parametrize("out_bf16", [False, True])
def test_a_page_that_is_none_is_left_out(hgf, dh, average, out_bf16):  # noqa: F811
    """Rows attend to the tokens of the pages that are there; with none of these and no open token a row is zero."""
    H, n = 2, 100 if average == 300 else 5
    p = Pair(hgf, H, dh, n_pages=20, n_slots=4)
    p.fill([200, 64, 300, 70])
    for slot, block in ((0, 1), (1, 0), (2, 3), (2, 0), (3, 0)):
        length, good = len(p.ref.tokens[slot]), p.cache.table[slot, block].item()
        q = rows(p.rng, n, 2 * H * dh)
        qf = bf16_bits_to_f32(q).astype(np.float64).reshape(n, 2, H, dh)
        kept = np.delete(np.arange(length), np.s_[block * BLOCK:(block + 1) * BLOCK])
        for page in (-1, 20):
            p.cache.table[slot, block] = page
            got, _ = call(p, q, slot, n, average, out_bf16, lam=0.7)
            with pytest.raises(hgf.HgfError) as e:
                hgf.check_status()
            assert e.value.status == 8
            for j in range(n):
                seen = kept[kept < length - n + j + 1]
                if not len(seen):
                    assert (got[j] == 0.0).all()
                    continue
                want, tol = attention(p.ref.values(slot)[:, :, seen], qf[j:j + 1], 1, H, 0.7, 1.0)
                tol = tol[0][:, None] + (2.0 ** -8 * np.abs(want[0]) if out_bf16 else 0)   # (half a step of bf16)
                assert (np.abs(got[j] - want[0]) <= tol).all()
        p.cache.table[slot, block] = good


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("group", [1, 3])
@pytest.mark.parametrize("average", AVERAGES)
@pytest.mark.parametrize("value", [0x7f80, 0xff80, 0x7fc0])
def test_a_query_that_is_not_finite_is_seen_in_its_row_and_head(hgf, dh, group, average, value):  # noqa: F811
    """One such element, where every key that the row sees has the sign that makes the score minus infinity (or NaN): no row may pass for one without weight."""
    H, dim = 2, 11
    p = Pair(hgf, H, dh, n_pages=20, n_slots=3)

    def change(k, v):  # K of stream 1 in head 0, of stream 2 in head 1: never 0 in that dim, nor rounded to it
        sign = np.float32(-1.0 if value == 0x7f80 else 1.0)
        for stream, head in ((0, 0), (1, 1)):
            k.reshape(-1, 2, H, dh)[:, stream, head, dim] = f32_to_bf16_bits(sign * (1.0 + np.arange(len(k)) % 3).astype(np.float32))[:]

    p.reserve([0, 1, 2], [200] * 3)
    p.append([0, 1, 2], [30, 134, 200], change=change)
    for slot, n in ((0, 100), (1, 100), (2, 100), (2, 1), (0, 30)):
        length, heads = len(p.ref.tokens[slot]), H * group
        for at in {0, max(0, n - length), n // 2, n - 1}:   # (the second: the first row that sees a token)
            q = rows(p.rng, n, 2 * heads * dh)
            qq = q.reshape(n, 2, heads, dh)
            qq[at, 0, group - 1, dim] = value        # a head of the group on K/V head 0
            qq[at, 1, group, dim] = value            # and one on K/V head 1
            for out_bf16 in (False, True):
                got, _ = call(p, q, slot, n, average, out_bf16, group=group)
                odd = ~np.isfinite(got)
                want = np.zeros((n, heads), bool)
                want[at, [group - 1, group]] = length - n + at + 1 > 0
                assert (odd.all(2) == want).all() and (odd.any(2) == want).all()
    hgf.check_status()


# ---- long walks of one worker -----------------------------------------------------------------------------------------
# Tiles of 128 rows keep a running maximum and begin their sums anew every eight pages.  80 entries that name one sequence of 21 blocks, two heads each, are
# more than 21 blocks for each of 148 to 160 workers: most walk through a whole item.
ENTRIES, M, LENGTH, HEADS = 80, 100, 1300, 2


def walk(p, q, out_bf16, lam=0.7):
    starts = ints(range(0, ENTRIES * M + 1, M))
    out = p.hgf.diff_attention_cached(p.cache, bf16(q), ints([0] * ENTRIES), starts, lam, flags=p.hgf.FLAG_OUT_BF16 if out_bf16 else 0)
    p.hgf.check_status()
    return out.view(ENTRIES, M, HEADS, p.dh)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("way", ["up", "down", "jump"])
def test_the_largest_score_moves_along_a_walk(hgf, dh, way):  # noqa: F811
    """Keys that grow or shrink along the sequence, or are large from block 12 on, against 64 bits."""
    p = Pair(hgf, HEADS, dh, n_pages=90, n_slots=1, max_pages=21)
    size = {"up": np.geomspace(0.2, 20.0, LENGTH), "down": np.geomspace(20.0, 0.2, LENGTH), "jump": np.where(np.arange(LENGTH) < 12 * BLOCK, 0.5, 30.0)}[way]

    def change(k, v):
        k[:] = f32_to_bf16_bits(bf16_bits_to_f32(k) * size.astype(np.float32)[:, None])

    p.reserve([0], [LENGTH])
    p.append([0], [LENGTH], change=change)
    bits = rows(p.rng, ENTRIES * M, 2 * HEADS * dh)
    q = torch.from_numpy(bf16_bits_to_f32(bits)).cuda().double().view(ENTRIES, M, 2, HEADS, dh)
    kv, lam, root = torch.from_numpy(p.ref.values(0)).cuda(), 0.7, dh ** -0.5
    sees = torch.arange(LENGTH, device="cuda")[None] <= LENGTH - M + torch.arange(M, device="cuda")[:, None]
    big, want, tol = kv[2].abs().amax((1, 2)), 0.0, 0.0
    for st, w in ((0, 1.0), (1, -lam)):
        s = torch.einsum("emhd,hnd->emhn", q[:, :, st], kv[st]) * root
        s = s.masked_fill(~sees[:, None], -torch.inf)
        e = torch.exp(s - s.amax(-1, keepdim=True))
        want = want + w * torch.einsum("emhn,hnd->emhd", e / e.sum(-1, keepdim=True), kv[2])
        # cache_reference.attention's tolerance, its largest over all tokens, and 96 terms of a sum that are cut off, 2^-23 each, where it counts one rounding a page
        ds = 2.0 ** -22 * q[:, :, st].abs().amax(-1) * kv[st].abs().sum(-1).amax(-1) * root
        ds = ds + 4 * 2.0 ** -24 * torch.einsum("emhd,hnd->emhn", q[:, :, st].abs(), kv[st].abs()).amax(-1) * root
        tol = tol + abs(w) * big * (2 * (ds + 2.0 ** -21) + 2 * LENGTH * 2.0 ** -24 / e.sum(-1) + (LENGTH / BLOCK + 20 + 96) * 2.0 ** -23)
    for out_bf16 in (False, True):
        off = (walk(p, bits, out_bf16).double() - want).abs()
        assert (off <= tol[..., None] + (2.0 ** -8 * want.abs() if out_bf16 else 0)).all()   # (half a step of bf16)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("out_bf16", [False, True])
@pytest.mark.parametrize("block", [0, 7, 8, 12, 19])
@pytest.mark.parametrize("large", [13, 17, 18])
def test_a_value_that_is_not_finite_is_not_forgotten(hgf, dh, out_bf16, block, large):  # noqa: F811
    """A block with a NaN in front of scores that leave it no weight: 0 times NaN, in every row that sees it."""
    p = Pair(hgf, HEADS, dh, n_pages=90, n_slots=1, max_pages=21)

    def change(k, v):
        k[large * BLOCK:] = f32_to_bf16_bits(bf16_bits_to_f32(k[large * BLOCK:]) * np.float32(1000.0))
        v.reshape(-1, HEADS, dh)[block * BLOCK + 5, 0, 3] = 0x7fc0

    p.reserve([0], [LENGTH])
    p.append([0], [LENGTH], change=change)
    out = walk(p, rows(p.rng, ENTRIES * M, 2 * HEADS * dh), out_bf16)
    sees = LENGTH - M + 1 + torch.arange(M, device="cuda") > block * BLOCK
    assert torch.isnan(out[:, sees, 0]).all() and torch.isfinite(out[:, ~sees, 0]).all() and torch.isfinite(out[:, :, 1]).all()


@pytest.mark.parametrize("native", [True, False])
def test_an_output_or_workspace_elsewhere_is_refused(hgf, monkeypatch, native):  # noqa: F811
    if not native:
        monkeypatch.setattr(hgf, "_native_cache", None)
    p = Pair(hgf, 2, 64, n_slots=1)
    p.fill([70])
    q, slots, starts = torch.zeros((1, 256), dtype=torch.bfloat16, device="cuda"), ints([0]), ints([0, 1])
    out, ws = torch.zeros((1, 128), device="cuda"), torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    before = hgf.launch_count()
    for args in ({"out": out.cpu(), "workspace": ws}, {"out": out.cpu()}, {"out": out, "workspace": ws.cpu()}, {"workspace": ws.cpu()}, {"out": out, "workspace": ws.float()},
                 {"out": out, "workspace": ws[::2]}):
        with pytest.raises(AssertionError):
            hgf.diff_attention_cached(p.cache, q, slots, starts, 0.5, **args)
    with pytest.raises(AssertionError):
        hgf.diff_attention_cached(p.cache, q.view(1, 256, 1).expand(1, 256, 2).contiguous(), slots, starts, 0.5, out=out, workspace=ws)
    assert hgf.launch_count() == before
    assert torch.equal(hgf.diff_attention_cached(p.cache, q, slots, starts, 0.5, out=out, workspace=ws), hgf.diff_attention_cached(p.cache, q, slots, starts, 0.5))


@pytest.mark.parametrize("tokens", [1, 5, 100])
def test_a_block_between_its_layers(hgf, tokens):  # noqa: F811
    """LayerNorm and projections, append, attention, output layer, read-back: back to back, where each launch may begin under the one before, and in a graph,
    with the bits that the same calls give when the device is waited for after each."""
    H, dh, S, steps = 2, 64, 3, 30
    d, n = H * dh, tokens * S
    g = torch.Generator().manual_seed(17)
    weights = {name: (*hgf.pack_ternary(torch.randn(rows_, d, generator=g).cuda()), d, rows_) for name, rows_ in (("q", 2 * d), ("k", 2 * d), ("v", d), ("o", d))}
    slots, starts, first = ints([2, 0, 1]), ints(range(0, n + 1, tokens)), ints([0] * S)
    norm = {"ln_weight": torch.ones(d, device="cuda"), "ln_bias": torch.zeros(d, device="cuda")}
    x0 = torch.randn(n, d, generator=g).cuda().bfloat16()

    def run(wait, graph=False):
        cache = hgf.KVCache(H, dh, S * (steps * tokens // 64 + 2), S, steps * tokens // 64 + 2)
        hgf.cache_reserve(cache, slots, ints([steps * tokens] * S))
        x, q, k, v = x0.clone(), *(torch.empty(n, w * d, dtype=torch.bfloat16, device="cuda") for w in (2, 2, 1))
        out, done = torch.empty(n, d, dtype=torch.bfloat16, device="cuda"), torch.empty(S, dtype=torch.int32, device="cuda")
        kr, vr = torch.zeros(n, 2 * d, device="cuda"), torch.zeros(n, d, device="cuda")
        ws = torch.empty(hgf.cached_workspace_bytes(cache, S, n, H), dtype=torch.uint8, device="cuda")
        lws = [torch.empty(hgf.workspace_bytes(n, d, w * d, 0), dtype=torch.uint8, device="cuda") for w in (2, 2, 1, 1)]

        def layer(name, src, dst, i):
            packed, gamma, d_in, d_out = weights[name]
            hgf.linear_forward(src, packed, gamma, d_in, d_out, y=dst, workspace=lws[i], flags=hgf.FLAG_OUT_BF16, **({} if name == "o" else norm))
            wait()

        def step():
            for i, (name, dst) in enumerate((("q", q), ("k", k), ("v", v))):
                layer(name, x, dst, i)
            hgf.cache_append(cache, k, v, slots, starts, done=done)
            wait()
            hgf.diff_attention_cached(cache, q, slots, starts, 0.3, out=out, workspace=ws, flags=hgf.FLAG_OUT_BF16)
            wait()
            layer("o", out, x, 3)
            hgf.cache_read(cache, slots, first, starts, k=kr, v=vr)
            wait()

        outs = []
        if graph:
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                step()
        for _ in range(steps):
            captured.replay() if graph else step()
            outs += [x.clone(), out.clone(), kr.clone(), done.clone()]
        hgf.check_status()
        return outs + [cache.length.clone(), cache.codes[cache.table[:, :steps * tokens // 64].flatten().long()], cache.open[:, :, :, :steps * tokens % 64].clone()]

    want = run(torch.cuda.synchronize)
    assert all(torch.isfinite(t.float()).all() for t in want) and want[-3].tolist() == [steps * tokens] * S
    for kind in (False, True, False):
        for a, b in zip(run(lambda: None, kind), want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("average", AVERAGES)
def test_a_workspace_may_hold_anything_and_calls_overlap(hgf, dh, average):  # noqa: F811
    """The same bits with a workspace of ones and of NaN, of exactly the bytes that are asked for, and from calls on two streams with a workspace each."""
    p = Pair(hgf, 2, dh, n_pages=120, n_slots=2, max_pages=60)
    p.fill([3333, 1300])
    S, m = (60, 1) if average == 1 else (60, {8: 5, 16: 13, 32: 40, 300: 110}[average])
    slots, starts = ints([i % 2 for i in range(S)]), ints(range(0, S * m + 1, m))
    q = [bf16(rows(p.rng, S * m, 4 * dh)) for _ in range(2)]
    n = hgf.cached_workspace_bytes(p.cache, S, S * m, 2)
    ws = [torch.full((n,), fill, dtype=torch.uint8, device="cuda") for fill in (0xff, 1)]
    call = lambda i, w, **kw: hgf.diff_attention_cached(p.cache, q[i], slots, starts, 0.7, workspace=w, **kw)  # noqa: E731
    want = [call(i, torch.zeros(n, dtype=torch.uint8, device="cuda")) for i in range(2)]
    for i in range(2):
        for w in ws:
            w.fill_(0xff if w is ws[0] else 1)
            assert torch.equal(call(i, w), want[i])
    with pytest.raises(hgf.HgfError):
        call(0, ws[0][:-256])
    outs = [[torch.empty_like(want[i]) for _ in range(8)] for i in range(2)]
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for j in range(8):
        for i in range(2):
            call(i, ws[i], out=outs[i][j], stream=side[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in outs[i])
    hgf.check_status()
