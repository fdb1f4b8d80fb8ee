"""The 8-bit paged K/V cache (hgf_cache_*) and the attention over it (hgf_diff_attention_cached) against tests/cache_reference.py.

What the cache holds is exact on both sides: codes, scales, open rows, tables, counts and the values that are read back are compared for equality
(a bf16 read is the rounding of the binary32 product).  The attention's tolerance is derived there, row by row; a bf16 output adds half a step,
2^-8 of the value."""
import numpy as np
import pytest
import torch

import oracle
from cache_reference import BLOCK, Reference, attention, page_bytes, rows
from paper_2602_05269_b200.inputs import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hgf():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    from paper_2602_05269_b200 import hgf as binding
    binding.lib()
    torch.cuda.set_device(0)
    return binding


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits)).view(torch.bfloat16).cuda()


def bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


class Pair:
    """The library's cache and the reference, given the same calls."""

    def __init__(self, hgf, H, dh, n_pages=40, n_slots=8, max_pages=20, seed=0):
        self.hgf, self.H, self.dh, self.rng = hgf, H, dh, np.random.default_rng([83, seed])
        self.cache = hgf.KVCache(H, dh, n_pages, n_slots, max_pages)
        # what no call has written may be anything
        self.cache.codes.fill_(77)
        self.cache.scales.fill_(float("nan"))
        self.cache.open.fill_(float("nan"))
        self.cache.table.fill_(-5)
        self.ref = Reference(H, dh, n_pages, n_slots, max_pages)

    def reserve(self, slots, tokens):
        got = self.hgf.cache_reserve(self.cache, ints(slots), ints(tokens)).tolist()
        assert got == self.ref.reserve(slots, tokens)

    def append(self, slots, counts, spread=1.0, change=None):
        starts = np.concatenate([[0], np.cumsum(counts)]).tolist()
        n = max(1, starts[-1])
        k, v = rows(self.rng, n, 2 * self.H * self.dh, spread), rows(self.rng, n, self.H * self.dh, spread)
        if change:
            change(k, v)
        got = self.hgf.cache_append(self.cache, bf16(k), bf16(v), ints(slots), ints(starts)).tolist()
        assert got == self.ref.append(slots, starts, k, v)

    def fill(self, lengths, **kw):
        """Slot i gets lengths[i] tokens."""
        self.reserve(range(len(lengths)), lengths)
        self.append(range(len(lengths)), lengths, **kw)

    def check(self):
        c, r = self.cache, self.ref
        assert c.length.tolist() == [len(t) for t in r.tokens] and c.held.tolist() == [len(p) for p in r.pages]
        assert c.refs.tolist() == r.refs and not c.arrivals.any()
        table, codes, scales = c.table.cpu().numpy(), c.codes.cpu().numpy(), c.scales.cpu().numpy()
        stored = bits(c.open)
        for s, tokens in enumerate(r.tokens):
            assert table[s, :len(r.pages[s])].tolist() == r.pages[s]
            for b in range(len(tokens) // BLOCK):
                want, sc = r.content[r.pages[s][b]]
                for h in range(self.H):
                    assert np.array_equal(codes[r.pages[s][b], h], page_bytes(want[0, h], want[1, h], want[2, h]))
                assert np.array_equal(scales[r.pages[s][b], :, :3].T, sc, equal_nan=True)
            for j in range(len(tokens) % BLOCK):
                e = np.arange(self.dh // 8) ^ (j % 8)
                got = stored[s, :, :, j].reshape(self.H, 3, -1, 8)[:, :, e].reshape(self.H, 3, -1)
                assert np.array_equal(got.transpose(1, 0, 2), tokens[len(tokens) // BLOCK * BLOCK + j])

    def attend(self, slots, counts, group=1, lam=0.7, out_scale=1.0, out_bf16=False, spread=1.0, q=None, pad=2):
        """Attention of the last counts[i] tokens of each listed sequence; rows of slots that are skipped have to stay as they were.  `pad` sequences
        without rows at the end: with as many as there are rows behind the last sequence, single tokens take the form for single tokens."""
        slots, counts = list(slots) + [-1] * pad, list(counts) + [0] * pad
        heads, starts = self.H * group, np.concatenate([[0], np.cumsum(counts)]).tolist()
        n = starts[-1] + 2  # (two rows behind the last sequence)
        q = rows(self.rng, n, 2 * heads * self.dh, spread) if q is None else q
        out = torch.full((n, heads * self.dh), 123.0, dtype=torch.bfloat16 if out_bf16 else torch.float32, device="cuda")
        got = self.hgf.diff_attention_cached(self.cache, bf16(q), ints(slots), ints(starts), lam, out_scale, out=out,
                                             flags=self.hgf.FLAG_OUT_BF16 if out_bf16 else 0).float().cpu().numpy().astype(np.float64)
        self.hgf.check_status()
        assert (got[starts[-1]:] == 123.0).all()
        got = got.reshape(n, heads, self.dh)
        qf = bf16_bits_to_f32(q).astype(np.float64).reshape(n, 2, heads, self.dh)
        for i, s in enumerate(slots):
            a, b = starts[i], starts[i + 1]
            if s < 0:
                assert (got[a:b] == 123.0).all()
                continue
            want, tol = attention(self.ref.values(s), qf[a:b], b - a, heads, lam, out_scale, coarse=out_bf16 and n * group > len(slots))
            tol = tol[:, :, None] + (2.0 ** -8 * np.abs(want) if out_bf16 else 0)
            off = np.abs(got[a:b] - want)
            assert (off <= tol).all(), f"slot {s}, {b - a} rows of {len(self.ref.tokens[s])} tokens: {np.nanmax(off / np.maximum(tol, 1e-30)):.3g} times the tolerance, {np.isnan(off).sum()} NaN"
        return got


# ---- append, read -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,dh", [(1, 64), (3, 64), (2, 128)])
def test_append_in_pieces(hgf, H, dh):
    p = Pair(hgf, H, dh)
    p.fill([1, 63, 64, 65, 0, 200, 127, 128])
    p.check()
    p.reserve(range(8), [250] * 8)
    for counts in ([1] * 8, [62, 1, 64, 3, 5, 0, 1, 70], [0, 0, 0, 0, 0, 0, 0, 1], [30, 2, 1, 1, 100, 0, 0, 0]):
        p.append([3, 1, 7, 0, 2, 5, 4, 6], counts)
        p.check()
    hgf.check_status()


def test_codes_do_not_depend_on_how_tokens_arrive(hgf):
    H, dh, n = 2, 64, 150
    rng = np.random.default_rng(5)
    k, v = rows(rng, n, 2 * H * dh), rows(rng, n, H * dh)
    cache = hgf.KVCache(H, dh, 8, 2, 4)
    hgf.cache_reserve(cache, ints([0, 1]), ints([n, n]))
    hgf.cache_append(cache, bf16(k), bf16(v), ints([0]), ints([0, n]))
    for j in range(n):
        hgf.cache_append(cache, bf16(k[j:j + 1]), bf16(v[j:j + 1]), ints([1]), ints([0, 1]))
    a, b = cache.table[0, :2].long(), cache.table[1, :2].long()
    assert torch.equal(cache.codes[a], cache.codes[b]) and torch.equal(cache.scales[a][..., :3], cache.scales[b][..., :3])
    assert cache.length.tolist() == [n, n] and torch.equal(cache.open[0, :, :, :n % 64], cache.open[1, :, :, :n % 64])


def test_codes_at_the_edges_of_the_quantiser(hgf):
    """Exact ties of the quotient, a block of zeros, magnitudes at both ends of bf16, blocks with infinities and NaN."""
    p = Pair(hgf, 5, 64, n_slots=2)

    def change(k, v):
        kk, vv = k.reshape(-1, 2, 5, 64), v.reshape(-1, 5, 64)
        kk[:64, 0, 0] = f32_to_bf16_bits(np.random.default_rng(1).choice(np.float32([1.0, 0.5, -0.5, 0.25, 1 / 128, -1.0]), (64, 64)))  # x = max / 2: 63.5
        kk[:64, 1, 0] = 0
        vv[:64, 0] = f32_to_bf16_bits(np.float32(2.0 ** -130) * np.random.default_rng(2).integers(-8, 9, (64, 64)).astype(np.float32))  # subnormal
        kk[:64, 0, 1] = f32_to_bf16_bits(np.float32(3e38) * np.random.default_rng(3).uniform(-1, 1, (64, 64)).astype(np.float32))
        kk[7, 1, 1, 3] = 0x7f80
        vv[9, 1, 5] = 0x7fc0
        kk[3, 0, 2, 1] = 0xff80
        vv[:64, 2] = f32_to_bf16_bits(np.float32(1e-31) * np.random.default_rng(4).standard_normal((64, 64)).astype(np.float32))

    p.fill([64, 130], change=change)
    p.check()


@pytest.mark.parametrize("exponent", [-133, -100, -60, 0, 119])
def test_codes_for_every_pair_of_mantissas(hgf, exponent):
    """128 heads whose largest value has each of the mantissas of bf16, and values with each mantissa, sign and eight exponents under it."""
    H, dh = 128, 64
    values = np.stack([np.ldexp(128.0 + (np.arange(64 * 64) // 16) % 128, -(np.arange(64 * 64) % 8)) * np.where(np.arange(64 * 64) // 8 % 2, 1, -1)] * H).reshape(H, 64, 64)
    top = 128.0 + np.arange(H)
    values[np.abs(values) > top[:, None, None]] *= 0.5
    values[:, 5, 7] = top
    bits_ = f32_to_bf16_bits(np.ldexp(values, exponent).astype(np.float32)).transpose(1, 0, 2)      # token, head, dim (below 2^-126 some round: they are bf16 all the same)
    p = Pair(hgf, H, dh, n_pages=1, n_slots=1, max_pages=1)
    p.reserve([0], [64])

    def change(k, v):
        k.reshape(64, 2, H, dh)[:] = bits_[:, None]
        v.reshape(64, H, dh)[:] = bits_

    p.append([0], [64], change=change)
    p.check()


def test_rows_that_begin_later(hgf):
    """The first sequence's rows need not be the call's first."""
    p = Pair(hgf, 2, 64)
    p.reserve([0, 1], [200, 200])
    k, v = rows(p.rng, 400, 256), rows(p.rng, 400, 128)
    for starts in ([130, 200, 390], [64, 64, 70], [399, 400, 400]):
        got = hgf.cache_append(p.cache, bf16(k), bf16(v), ints([0, 1]), ints(starts)).tolist()
        assert got == p.ref.append([0, 1], starts, k, v) == [1, 1]
        p.check()
    kk, vv = torch.full((400, 256), 7.0, device="cuda"), torch.full((400, 128), 7.0, device="cuda")
    hgf.cache_read(p.cache, ints([1]), ints([0]), ints([300, 400]), k=kk, v=vv)
    want = torch.from_numpy(p.ref.values(1)).float()[:, :, :100]
    assert torch.equal(vv[300:].cpu().view(100, 2, 64), want[2].permute(1, 0, 2)) and (vv[:300] == 7.0).all() and (kk[:300] == 7.0).all()
    hgf.check_status()


def test_append_to_more_sequences_than_run_at_once(hgf):
    """Blocks of threads that a sequence turns out not to need may run long after those that it needs: they must not take its new length for the old one."""
    n, m = 1024, 70
    cache = hgf.KVCache(1, 64, 3 * n, n, 4)
    hgf.cache_reserve(cache, ints(range(n)), ints([200] * n))
    k, v = torch.randn(n * m, 128, device="cuda").bfloat16(), torch.randn(n * m, 64, device="cuda").bfloat16()
    starts = ints(range(0, n * m + 1, m))
    for step in range(2):                    # 70, 140 tokens: of each step's two possible blocks one is complete
        assert hgf.cache_append(cache, k, v, ints(range(n)), starts).all()
        assert (cache.length == m * (step + 1)).all() and not cache.arrivals.any()
    got_k, got_v = hgf.cache_read(cache, ints(range(n)), ints([128] * n), ints(range(0, 12 * n + 1, 12)), 12 * n)
    assert torch.equal(got_v.view(n, 12, 64), v.view(n, m, 64)[:, 58:].float()) and torch.equal(got_k.view(n, 12, 128), k.view(n, m, 128)[:, 58:].float())
    got_k, _ = hgf.cache_read(cache, ints(range(n)), ints([0] * n), ints(range(0, 128 * n + 1, 128)), 128 * n)
    want = torch.cat([k.view(n, m, 128), k.view(n, m, 128)[:, :58]], 1).float()
    # half a step, 1 / 127 of each block's and stream's largest; the value's two roundings beside it
    top = want.view(n, 2, 64, 2, 64).abs().amax((2, 4), keepdim=True)
    assert ((got_k.view(n, 128, 128) - want).view(n, 2, 64, 2, 64).abs() <= top * (0.5 / 127 + 2.0 ** -22)).all()
    out = hgf.diff_attention_cached(cache, torch.zeros(n, 128, device="cuda").bfloat16(), ints(range(n)), ints(range(n + 1)), 0.25)
    got_k, got_v = hgf.cache_read(cache, ints(range(n)), ints([0] * n), ints(range(0, 140 * n + 1, 140)), 140 * n)
    mean = 0.75 * got_v.view(n, 140, 64).double().mean(1)
    assert (out - mean).abs().max() <= 1.25 * got_v.abs().max() * (2 * 140 * 2.0 ** -24 / 140 + 30 * 2.0 ** -23)   # (all probabilities are equal)
    hgf.check_status()


def test_append_without_room_leaves_the_sequence(hgf):
    p = Pair(hgf, 2, 64, n_pages=4, n_slots=6, max_pages=3)
    p.reserve([0, 1], [64, 64])
    p.append([0, 1, 2], [130, 127, 63])      # slot 0 asks for two pages and has one
    p.check()
    p.append([0, 2, 2, 1, -1], [10, 1, 5, 1, 3])  # slot 2 has none, and is named twice; slot 1's block needs another
    p.check()
    p.reserve([3], [64])
    p.append([3], [64])
    assert hgf.cache_fork(p.cache, ints([3]), ints([4])).tolist() == p.ref.fork([3], [4])
    p.cache.length[4] = 60                   # tokens taken back into a page that is shared: it must not be written
    assert hgf.cache_append(p.cache, *(torch.zeros((4, w), dtype=torch.bfloat16, device="cuda") for w in (256, 128)), ints([4]), ints([0, 4])).tolist() == [0]
    p.cache.length[4] = 64
    p.check()
    hgf.check_status()


@pytest.mark.parametrize("H,dh", [(3, 64), (2, 128)])
@pytest.mark.parametrize("out_bf16", [False, True])
def test_read(hgf, H, dh, out_bf16):
    p = Pair(hgf, H, dh)
    lengths = [1, 63, 64, 65, 0, 200, 127, 300]
    p.fill(lengths)
    slots, first = [5, 7, 0, 3, -1, 2, 6, 4, 5], [0, 70, 0, 10, 0, 60, 64, 0, 199]
    counts = [200, 100, 1, 60, 5, 10, 0, 3, 4]   # (some reach behind the sequence's end)
    starts = np.concatenate([[0], np.cumsum(counts)]).tolist()
    dt = torch.bfloat16 if out_bf16 else torch.float32
    k, v = (torch.full((starts[-1] + 1, w), 7.0, dtype=dt, device="cuda") for w in (2 * H * dh, H * dh))
    hgf.cache_read(p.cache, ints(slots), ints(first), ints(starts), k=k, v=v)
    hgf.check_status()
    want = torch.full((starts[-1] + 1, 3, H, dh), 7.0, dtype=dt)
    for i, s in enumerate(slots):
        if s >= 0:
            x = torch.from_numpy(p.ref.values(s)).float()[:, :, first[i]:first[i] + counts[i]].permute(2, 0, 1, 3)  # (one rounding to binary32, as the product's)
            want[starts[i]:starts[i] + len(x)] = x.to(dt)
    assert torch.equal(k.cpu(), want[:, :2].reshape(len(want), -1)) and torch.equal(v.cpu(), want[:, 2].reshape(len(want), -1))


# ---- pages ------------------------------------------------------------------------------------------------
def test_reserve_fork_free(hgf):
    p = Pair(hgf, 2, 64, n_pages=30, n_slots=12, max_pages=9)
    p.fill([300, 64, 10, 127])
    p.reserve([0, 1, 0, 2, 3, -1, 5], [400, 200, 900, 20, 64 * 10, 70, 64])   # twice named, padding, more than max_pages
    src, dst = [0, 0, 2, 3, 1, 4, 0, 3], [4, 5, 6, 7, 8, 9, 4, 1]           # 5 holds a page, 4 is a source as well and named twice, 1 is a source
    assert hgf.cache_fork(p.cache, ints(src), ints(dst)).tolist() == p.ref.fork(src, dst)
    p.check()
    hgf.cache_free(p.cache, ints([4, 6, 7, 8]))
    p.ref.free([4, 6, 7, 8])
    p.check()
    src, dst = [0, 0, 2, 3, 1], [4, 9, 6, 7, 8]
    assert hgf.cache_fork(p.cache, ints(src), ints(dst)).tolist() == p.ref.fork(src, dst) == [1] * 5
    p.check()
    p.reserve([4, 9, 6, 7, 8, 10, 11], [320, 384, 64, 128, 200, 64 * 9, 64])
    p.reserve([0, 4, 10, 9, 11], [64 * 9, 300, 64 * 9, 64 * 9, 60])   # the pool ends on the way; slot 4 and 11 need none
    p.check()
    p.append([4, 0, 9, 6], [1, 20, 84, 54])
    p.check()
    for slots in ([0, 0, -1, 2], [4, 9]):
        hgf.cache_free(p.cache, ints(slots))
        p.ref.free(slots)
        p.check()
    p.reserve([0, 2, 10], [64 * 9, 64, 64])
    p.check()
    hgf.check_status()


def test_reserve_across_many_steps(hgf):
    """More pages than one step of the walk looks at, the free ones far apart; requests that end inside a step."""
    n = 50000
    cache = hgf.KVCache(1, 64, n, 4, 30000)
    free = torch.zeros(n, dtype=torch.bool)
    free[torch.randperm(n, generator=torch.Generator().manual_seed(3))[:20000]] = True
    cache.refs.copy_((~free).int())
    want = free.nonzero().flatten()
    got = hgf.cache_reserve(cache, ints([2, 0, 3, 1]), ints([64 * 7001 + 5, 64 * 12000, 64 * 1000, 64 * 999])).tolist()
    assert got == [1, 1, 0, 0] and cache.held.tolist() == [12000, 0, 7001, 0]  # 999 are left, but the first request to miss ends the dealing
    assert torch.equal(cache.table[2, :7001].cpu().long(), want[:7001]) and torch.equal(cache.table[0, :12000].cpu().long(), want[7001:19001])
    assert int((cache.refs == 0).sum()) == 999
    hgf.check_status()


# ---- attention --------------------------------------------------------------------------------------------
LENGTHS = [1, 2, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 700, 1279]


@pytest.mark.parametrize("H,dh", [(1, 64), (3, 64), (2, 128)])
@pytest.mark.parametrize("out_bf16", [False, True])
def test_single_tokens(hgf, H, dh, out_bf16):
    p = Pair(hgf, H, dh, n_pages=90, n_slots=16)
    p.fill(LENGTHS)
    for pad in (2, 0):
        p.attend(range(16), [1] * 16, out_bf16=out_bf16, pad=pad)
    for s in (0, 3, 14):
        p.attend([s], [1], lam=-0.3, out_scale=0.5, out_bf16=out_bf16)


@pytest.mark.parametrize("H,dh,group", [(2, 64, 1), (1, 64, 3), (2, 128, 4), (1, 128, 8), (2, 64, 11)])
@pytest.mark.parametrize("out_bf16", [False, True])
def test_several_tokens_and_shared_heads(hgf, H, dh, group, out_bf16):
    p = Pair(hgf, H, dh, n_pages=90, n_slots=16)
    p.fill(LENGTHS)
    p.attend(range(16), [1, 2, 3, 9, 1, 5, 4, 2, 33, 1, 0, 70, 1, 8, 17, 6], group=group, out_bf16=out_bf16)
    if group > 1:
        p.attend([14, 6], [1, 1], group=group, out_bf16=out_bf16)


@pytest.mark.parametrize("dh", [64, 128])
def test_rows_that_see_nothing_and_padding(hgf, dh):
    p = Pair(hgf, 2, dh, n_pages=90, n_slots=16)
    p.fill([0, 3, 64, 0, 130])
    p.attend([0, 1, -1, 2, 3, 4, -1], [1, 1, 1, 1, 1, 1, 1])
    p.attend([0, 1, -1, 2, 3, 4, -1], [3, 5, 2, 70, 1, 131, 4])     # more rows than tokens: the first see nothing
    p.attend([3], [1])
    p.attend([-1, 4], [0, 1])


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("group", [1, 3])
def test_many_rows(hgf, dh, group):
    """Tiles of 128 rows: rows that see nothing, tiles that end inside, open tokens alone, skipped sequences; items that many workers share and workers with many."""
    p = Pair(hgf, 2, dh, n_pages=200, n_slots=8)
    p.fill([0, 3, 64, 130, 1000, 63, 5000, 321])
    for out_bf16 in (True, False):
        p.attend([4], [300 // group], group=group, out_bf16=out_bf16, pad=0)
        p.attend([6], [128], group=group, out_bf16=out_bf16, pad=0)
        p.attend([5, 0, -1, 3, 1, 4, 2], [90, 100, 70, 250, 5, 129, 64], group=group, out_bf16=out_bf16, pad=0)
        p.attend([7, 6], [321, 1], group=group, out_bf16=out_bf16, pad=0, spread=4.0)
        p.attend([2], [200], group=group, out_bf16=out_bf16, pad=0)
    p.attend([0], [150], group=group, out_bf16=True, pad=0)


def test_many_rows_of_many_sequences(hgf):
    p = Pair(hgf, 5, 64, n_pages=400, n_slots=90)
    p.fill([65 + 2 * i for i in range(90)])
    p.attend(list(range(90)), [85] * 90, out_bf16=True, pad=0)
    p.attend(list(range(90)), [84] * 90, pad=0)


def test_many_rows_in_a_small_pool(hgf):
    p = Pair(hgf, 2, 64, n_pages=2, n_slots=3)
    p.fill([63, 2, 100])
    for out_bf16 in (True, False):
        p.attend([0, 1, 2], [90, 120, 81], out_bf16=out_bf16, pad=0)


def test_many_rows_with_blocks_of_zeros(hgf):
    p = Pair(hgf, 2, 64, n_pages=20, n_slots=1)

    def change(k, v):
        k.reshape(-1, 2, 2, 64)[:64, 0] = 0
        k.reshape(-1, 2, 2, 64)[128:200] = 0
        v[64:128] = 0

    p.reserve([0], [200])
    p.append([0], [200], change=change)
    p.attend([0], [150], out_bf16=True, pad=0)
    p.attend([0], [150], out_bf16=True, pad=0, spread=5.0)


@pytest.mark.parametrize("m", [1, 3, 40, 100])
@pytest.mark.parametrize("out_bf16", [False, True])
def test_scores_far_below_zero(hgf, m, out_bf16):
    """Equal scores of about -2^102 * 64 / 8: every token that a row sees has the same weight."""
    p = Pair(hgf, 2, 64, n_pages=20, n_slots=1)

    def change(k, v):
        k[:] = f32_to_bf16_bits(np.full(1, -2.0 ** 50, np.float32))[0]

    p.reserve([0], [192])
    p.append([0], [192], change=change)
    q = np.full((m, 256), f32_to_bf16_bits(np.full(1, 2.0 ** 52, np.float32))[0], np.uint16)
    out = hgf.diff_attention_cached(p.cache, bf16(q), ints([0]), ints([0, m]), 0.25, flags=hgf.FLAG_OUT_BF16 if out_bf16 else 0).float().cpu().numpy().reshape(m, 2, 64)
    v = p.ref.values(0)[2]
    for j in range(m):
        want = 0.75 * v[:, :192 - m + j + 1].mean(1)
        # (sums of up to 192 terms in binary32, a probability to 2^-16 at least, half a step of bf16)
        tol = np.abs(v).max() * (2 * 192 * 2.0 ** -24 + (2 * 2.0 ** -16 if out_bf16 else 2.0 ** -22)) + (2.0 ** -8 * np.abs(want) if out_bf16 else 0)
        assert (np.abs(out[j] - want) <= tol).all()


def test_many_rows_skip_a_page_that_is_none(hgf):
    p = Pair(hgf, 2, 64, n_pages=20, n_slots=2)
    p.fill([200, 200])
    q, slots, starts = rows(p.rng, 240, 256), ints([0, 1]), ints([0, 120, 240])
    want = hgf.diff_attention_cached(p.cache, bf16(q), slots, starts, 0.5, flags=hgf.FLAG_OUT_BF16)
    good = p.cache.table[1, 1].item()
    for page in (-1, 20):
        p.cache.table[1, 1] = page
        out = hgf.diff_attention_cached(p.cache, bf16(q), slots, starts, 0.5, flags=hgf.FLAG_OUT_BF16)
        with pytest.raises(hgf.HgfError) as e:
            hgf.check_status()
        assert e.value.status == 8 and torch.equal(out[:120], want[:120])
    p.cache.table[1, 1] = good
    assert torch.equal(hgf.diff_attention_cached(p.cache, bf16(q), slots, starts, 0.5, flags=hgf.FLAG_OUT_BF16), want)
    hgf.check_status()


def test_one_row_form_takes_any_counts(hgf):
    """No more rows than sequences on the whole picks the form for single tokens; a sequence may have several all the same."""
    p = Pair(hgf, 3, 64, n_pages=90, n_slots=16)
    p.fill(LENGTHS)
    slots, counts, n = range(16), [1, 2, 0, 0, 1, 0, 3, 1, 0, 2, 0, 1, 1, 0, 4, 0], 16
    q, starts = rows(p.rng, n, 6 * 64), np.concatenate([[0], np.cumsum(counts)]).tolist()
    assert starts[-1] == n
    got = hgf.diff_attention_cached(p.cache, bf16(q), ints(slots), ints(starts), 0.7).cpu().numpy().reshape(n, 3, 64)
    qf = bf16_bits_to_f32(q).astype(np.float64).reshape(n, 2, 3, 64)
    for i in slots:
        a, b = starts[i], starts[i + 1]
        want, tol = attention(p.ref.values(i), qf[a:b], b - a, 3, 0.7, 1.0)
        assert (np.abs(got[a:b] - want) <= tol[:, :, None]).all()


def test_one_row_form_leaves_padding(hgf):
    p = Pair(hgf, 2, 64, n_slots=4)
    p.fill([0, 70, 64, 33])
    q = rows(p.rng, 6, 256)
    out = torch.full((6, 128), 5.0, device="cuda")
    hgf.diff_attention_cached(p.cache, bf16(q), ints([3, -1, 0, 1, 2, -1]), ints(range(7)), 0.7, out=out)
    got, qf = out.cpu().numpy().reshape(6, 2, 64), bf16_bits_to_f32(q).astype(np.float64).reshape(6, 2, 2, 64)
    assert (got[[1, 5]] == 5.0).all() and (got[2] == 0.0).all()
    for i, s in ((0, 3), (3, 1), (4, 2)):
        want, tol = attention(p.ref.values(s), qf[i:i + 1], 1, 2, 0.7, 1.0)
        assert (np.abs(got[i] - want[0]) <= tol[0][:, None]).all()
    hgf.check_status()


@pytest.mark.parametrize("dh,m", [(64, 1), (128, 1), (64, 3), (128, 3)])
def test_items_shared_by_many_workers(hgf, dh, m):
    """One long sequence and little else: every head is in parts."""
    p = Pair(hgf, 2, dh, n_pages=130, n_slots=3, max_pages=128)
    p.fill([8000, 5, 66])
    p.attend([1, 0, 2], [1, m, 1])
    p.attend([0], [m], out_bf16=True)


def test_more_items_than_workers(hgf):
    p = Pair(hgf, 7, 64, n_pages=400, n_slots=260, max_pages=4)
    lengths = [(37 * i) % 200 for i in range(260)]
    p.reserve(range(260), [200] * 130 + [60] * 130)
    p.append(range(260), [n if i < 130 else n % 60 for i, n in enumerate(lengths)])
    p.attend(range(260), [1] * 260)
    p.attend(list(range(100)) + [-1] * 20, [1 + i % 3 for i in range(120)])


@pytest.mark.parametrize("m", [1, 4])
def test_scores_of_all_sizes(hgf, m):
    """Peaked rows, flat ones, and keys that grow along the sequence, so that the running maximum moves page by page."""
    p = Pair(hgf, 2, 64, n_pages=90, n_slots=4)

    def grow(k, v):
        kk = bf16_bits_to_f32(k) * np.linspace(0.2, 5.0, len(k), dtype=np.float32)[:, None]
        k[:] = f32_to_bf16_bits(kk)

    p.reserve([0, 1, 2], [700, 700, 700])
    p.append([0], [700], change=grow)
    p.append([1], [700], spread=6.0)
    p.append([2], [700], spread=1e-3)
    slots, counts = [0, 1, 2], [m] * 3
    p.attend(slots, counts)
    p.attend(slots, counts, spread=8.0)
    p.attend(slots, counts, spread=1e-30)
    p.attend(slots, counts, q=np.zeros((3 * m + 2, 256), np.uint16))


@pytest.mark.parametrize("m", [1, 40])
def test_blocks_of_zeros(hgf, m):
    """Keys that are all zero (a scale of zero), behind and in front of others, in rows that see part of them."""
    p = Pair(hgf, 2, 64, n_pages=20, n_slots=2)

    def change(k, v):
        k.reshape(-1, 2, 2, 64)[:64, 0] = 0
        k.reshape(-1, 2, 2, 64)[128:200] = 0
        v[64:128] = 0

    p.reserve([0, 1], [200, 256])
    p.append([0], [200], change=change)
    p.append([1], [256], change=change)
    p.attend([0, 1], [m, m])
    p.attend([0, 1], [m, m], spread=5.0)


@pytest.mark.parametrize("m", [1, 3])
def test_values_that_are_not_finite(hgf, m):
    """A page or an open row with a NaN reaches the rows and heads that see it, and no others; so does a query's."""
    p = Pair(hgf, 2, 64, n_pages=20, n_slots=4)

    def change(k, v):
        bits_ = k.reshape(-1, 2, 2, 64)
        bits_[70, 0, 0, 5] = 0x7fc0           # slot 0, block 1, head 0: K1
        v.reshape(-1, 2, 64)[200 + 127, 1, 7] = 0x7f80   # slot 1, last token of block 1, head 1: V
        v.reshape(-1, 2, 64)[400 + 129, 0, 7] = 0x7fc0   # slot 2, open row 129 of 130, head 0: V

    p.reserve([0, 1, 2, 3], [200] * 4)
    p.append([0, 1, 2, 3], [200, 200, 130, 100], change=change)
    q = rows(p.rng, 4 * m, 256)
    q[3 * m, 64:128] = 0x7f80                 # slot 3's first row, stream 1, head 1
    out = p.hgf.diff_attention_cached(p.cache, bf16(q), ints(range(4)), ints(range(0, 4 * m + 1, m)), 0.5).cpu().numpy().reshape(4, m, 2, 64)
    nan = np.isnan(out)
    assert nan[0, :, 0].all() and not nan[0, :, 1].any()
    assert not np.isfinite(out[1, :, 1]).any() and np.isfinite(out[1, :, 0]).all()
    assert nan[2, m - 1, 0, 7] and np.isfinite(out[2, :, 1]).all()
    assert nan[3, 0, 1].all() and np.isfinite(out[3, :, 0]).all() and np.isfinite(out[3, 1:]).all()
    # the blocks before it, when the sequence ends there
    p.cache.length[0] = 64
    p.ref.tokens[0] = p.ref.tokens[0][:64]
    p.attend([0], [m])


def test_rows_before_a_block_that_is_not_finite(hgf):
    """Rows of one call on both sides of a block whose V scale is NaN, and of 32 open tokens with an infinite value."""
    p = Pair(hgf, 1, 64, n_pages=20, n_slots=2)

    def change(k, v):
        v[130, 3] = 0x7fc0
        v[200 + 40, 9] = 0x7f80

    p.reserve([0], [200])
    p.append([0, 1], [200, 50], change=change)
    q = rows(p.rng, 120, 128)
    out = p.hgf.diff_attention_cached(p.cache, bf16(q), ints([0, 1]), ints([0, 100, 120]), 0.5).cpu().numpy()
    assert np.isfinite(out[:28]).all() and np.isnan(out[28:100]).all()   # rows are tokens 100 .. 199; block 2 begins at 128
    assert np.isfinite(out[100:102]).all() and not np.isfinite(out[110:120, 9]).any() and np.isfinite(np.delete(out[110:120], 9, 1)).all()   # tokens 30 .. 49


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("group", [1, 3])
@pytest.mark.parametrize("a_sequence", [1, 8, 16, 32, 300])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(hgf, dh, group, a_sequence):
    """Rows on both sides of a page whose K scale is NaN, of an open value and of an open key that are not finite; queries that are not, of rows without tokens.

    `a_sequence`: rows times heads of a group that a sequence has on average, with sequences that have none."""
    L, m = 148, 100
    p = Pair(hgf, 2, dh, n_pages=20, n_slots=2)

    def change(k, v):
        k.reshape(-1, 2, 2, dh)[70, 0, 0, 5] = 0x7fc0     # block 1 of head 0, K1
        v.reshape(-1, 2, dh)[135, 1, 7] = 0xff80          # head 1, open: V, and K2 below
        k.reshape(-1, 2, 2, dh)[140, 1, 1, 9] = 0x7f80

    p.reserve([0, 1], [L, 70])
    p.append([0], [L], change=change)
    p.append([1], [70])
    idle = -(-m * group // a_sequence) - 1
    for n, slot in ((m, 0), (72, 1)):
        q = rows(p.rng, m, 2 * 2 * group * dh)
        if slot == 1:
            q[:2] = 0x7fc0
        for flat in (False, True):
            out = torch.full((m, 2 * group * dh), 5.0, dtype=torch.bfloat16 if flat else torch.float32, device="cuda")
            hgf.diff_attention_cached(p.cache, bf16(q), ints([slot] + [-1] * idle), ints([0] + [n] * (idle + 1)), 0.5, out=out,
                                      flags=hgf.FLAG_OUT_BF16 if flat else 0)
            out = out.float().cpu().numpy().reshape(m, 2, group, dh)
            assert (out[n:] == 5.0).all()
            if slot == 1:
                assert (out[:2] == 0.0).all() and np.isfinite(out[:n]).all()
                continue
            sees, bad = L - m + 1 + np.arange(m), ~np.isfinite(out)
            assert (bad[:, 0].all((1, 2)) == (sees > 64)).all() and not bad[sees <= 64, 0].any()
            assert not bad[sees <= 135, 1].any()
            some = (sees > 135) & (sees <= 140)
            assert bad[some, 1, :, 7].all() and not np.delete(bad[some, 1], 7, 2).any()
            # the open key's score is infinity with the sign of the query there: no weight, or a NaN
            nan = (bf16_bits_to_f32(q).reshape(m, 2, 2, group, dh)[:, 1, 1, :, 9] >= 0)[sees > 140]
            assert bad[sees > 140, 1, :, 7].all() and (np.delete(bad[sees > 140, 1], 7, 2) == nan[:, :, None]).all()


def test_agrees_with_the_definition_while_nothing_is_quantised(hgf):
    """Up to 63 tokens the cache holds bf16, so the attention is that of whole sequences."""
    H, dh, n = 3, 64, 63
    rng = np.random.default_rng(11)
    q, k, v = rows(rng, n, 2 * H * dh), rows(rng, n, 2 * H * dh), rows(rng, n, H * dh)
    cache = hgf.KVCache(H, dh, 1, 1, 1)
    hgf.cache_append(cache, bf16(k), bf16(v), ints([0]), ints([0, n]))
    out = hgf.diff_attention_cached(cache, bf16(q), ints([0]), ints([0, n]), 0.8).cpu().numpy()
    want = oracle.diff_attention(q, k, v, 1, n, H, dh, 0.8)
    _, tol = attention(bf16_bits_to_f32(np.concatenate([k.reshape(n, 2, H, dh), v.reshape(n, 1, H, dh)], 1)).astype(np.float64).transpose(1, 2, 0, 3),
                       bf16_bits_to_f32(q).astype(np.float64).reshape(n, 2, H, dh), n, H, 0.8, 1.0)
    assert (np.abs(out - want).reshape(n, H, dh) <= tol[:, :, None] + 2.0 ** -23 * np.abs(want).max()).all()   # (the oracle's output is binary32 at least)


def test_pages_beyond_32_bit_offsets(hgf):
    """A pool of more than 2^32 bytes and a table that names its last pages."""
    H, dh, n_pages = 16, 64, 22500
    cache = hgf.KVCache(H, dh, n_pages, 2, 8)
    cache.refs[:n_pages - 6] = 1
    hgf.cache_reserve(cache, ints([1, 0]), ints([150, 200]))
    assert cache.table[1, :2].tolist() == [n_pages - 6, n_pages - 5] and cache.table[0, :3].tolist() == list(range(n_pages - 4, n_pages - 1))
    p = Pair.__new__(Pair)
    p.hgf, p.H, p.dh, p.cache, p.rng = hgf, H, dh, cache, np.random.default_rng(13)
    p.ref = Reference(H, dh, n_pages, 2, 8)
    p.ref.pages, p.ref.refs = [cache.table[s, :n].tolist() for s, n in ((0, 3), (1, 2))], cache.refs.tolist()
    p.append([0, 1], [200, 150])
    p.attend([0, 1], [1, 1])
    p.attend([1, 0], [4, 1])
    k, v = hgf.cache_read(cache, ints([0]), ints([0]), ints([0, 200]), 200)
    want = torch.from_numpy(p.ref.values(0)).float()
    assert torch.equal(k.cpu().view(200, 2, H, dh), want[:2].permute(2, 0, 1, 3)) and torch.equal(v.cpu().view(200, H, dh), want[2].permute(1, 0, 2))


# ---- indices that are out of range, streams, graphs -------------------------------------------------------
def test_indices_out_of_range_are_skipped_and_reported(hgf):
    p = Pair(hgf, 2, 64, n_slots=4)
    p.fill([70, 70, 70, 70])
    q, big = torch.zeros((4, 256), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 128), dtype=torch.bfloat16, device="cuda")

    def reported():
        with pytest.raises(hgf.HgfError) as e:
            hgf.check_status()
        assert e.value.status == 8
        hgf.check_status()                     # once

    def attend(slots, starts):
        out = torch.full((4, 128), 5.0, device="cuda")
        hgf.diff_attention_cached(p.cache, q, ints(slots), ints(starts), 0.5, out=out)
        return out

    out = attend([0, 4, -2, 1], [0, 1, 2, 3, 4])
    reported()
    assert (out[1:3] == 5.0).all() and (out[0] != 5.0).any() and (out[3] != 5.0).any()
    for starts in ([0, 1, 1, 2, 5], [0, 2, 1, 2, 3], [-1, 0, 1, 2, 3]):
        attend([0, 1, 2, 3], starts)
        reported()
        assert hgf.cache_append(p.cache, q, big, ints([0, 1, 2, 3]), ints(starts)).tolist() == [0] * 4
        reported()
        hgf.cache_read(p.cache, ints([0, 1, 2, 3]), ints([0] * 4), ints(starts), 4)
        reported()
    assert hgf.cache_append(p.cache, q, big, ints([9, -7]), ints([0, 1, 2])).tolist() == [0, 0]
    reported()
    assert hgf.cache_fork(p.cache, ints([0, 77]), ints([-3, 2])).tolist() == [0, 0]
    reported()
    hgf.cache_free(p.cache, ints([4]))
    reported()
    assert hgf.cache_reserve(p.cache, ints([4, 0]), ints([64, -1])).tolist() == [0, 0]
    reported()
    hgf.cache_read(p.cache, ints([0, 5]), ints([-1, 0]), ints([0, 1, 2]), 2)
    reported()
    p.check()
    good = p.cache.table[2, 0].item()
    p.cache.table[2, 0] = p.cache.n_pages
    attend([2, 1], [0, 2, 4])
    reported()
    hgf.cache_read(p.cache, ints([2]), ints([0]), ints([0, 4]), 4)
    reported()
    p.cache.table[2, 0] = good
    p.cache.length[3] = 64 * 3
    attend([3], [0, 1])
    reported()
    p.cache.length[3] = 70
    p.check()
    p.attend(range(4), [1] * 4)


@pytest.mark.parametrize("native", [True, False])
def test_arguments_that_do_not_fit_are_refused(hgf, monkeypatch, native):
    """The same answers with the native marshalling and without it."""
    if not native:
        monkeypatch.setattr(hgf, "_native_cache", None)
    p = Pair(hgf, 2, 64, n_slots=4)
    p.fill([70, 70])
    c, one, two = p.cache, ints([0]), ints([0, 1])
    k, v = (torch.zeros((1, w), dtype=torch.bfloat16, device="cuda") for w in (256, 128))
    out, ws, done = torch.zeros((1, 128), device="cuda"), torch.zeros(1 << 22, dtype=torch.uint8, device="cuda"), ints([0])
    before = hgf.launch_count()
    bad = [lambda: hgf.cache_reserve(c, one, two, granted=done), lambda: hgf.cache_reserve(c, one.long(), one, granted=done), lambda: hgf.cache_reserve(c, one.cpu(), one, granted=done),
           lambda: hgf.cache_append(c, k.float(), v, one, two, done=done), lambda: hgf.cache_append(c, v, v, one, two, done=done), lambda: hgf.cache_append(c, k, v, one, one, done=done),
           lambda: hgf.cache_append(c, k.expand(2, -1), v.expand(2, -1), one, two, done=done), lambda: hgf.cache_append(c, k, v.cpu(), one, two, done=done),
           lambda: hgf.cache_fork(c, one, two, done=done), lambda: hgf.cache_free(c, one.long()), lambda: hgf.cache_free(c, ints(range(4))[::2]),
           lambda: hgf.cache_read(c, one, one, two, k=k.float(), v=v), lambda: hgf.cache_read(c, one, one, two, k=v, v=v), lambda: hgf.cache_read(c, one, two, two, k=k, v=v),
           lambda: hgf.diff_attention_cached(c, k[:, :200].contiguous(), one, two, 0.5, out=out, workspace=ws), lambda: hgf.diff_attention_cached(c, k, one, two, 0.5, out=out[:, :64], workspace=ws),
           lambda: hgf.diff_attention_cached(c, k, one, two, 0.5, out=out, workspace=ws, flags=hgf.FLAG_OUT_BF16), lambda: hgf.diff_attention_cached(c, k, one, one, 0.5, out=out, workspace=ws)]
    for call in bad:
        with pytest.raises(AssertionError):
            call()
    for call, status in ((lambda: hgf.diff_attention_cached(c, k, one, two, 0.5, out=out, workspace=ws[:512]), 4), (lambda: hgf.diff_attention_cached(c, k, one, two, 0.5, out=out, workspace=ws[16:]), 3),
                         (lambda: hgf.diff_attention_cached(c, torch.zeros((1, 3 * 128), dtype=torch.bfloat16, device="cuda"), one, two, 0.5), 2),
                         (lambda: hgf.cache_free(c, ints(range(1025))), 2), (lambda: hgf.cache_append(c, k[:0], v[:0], one, two, done=done), 1)):
        with pytest.raises(hgf.HgfError) as e:
            call()
        assert e.value.status == status
    assert hgf.launch_count() == before
    assert torch.equal(hgf.diff_attention_cached(c, k, one, two, 0.5, out=out, workspace=ws), hgf.diff_attention_cached(c, k, one, two, 0.5))
    p.check()


def test_tokens_taken_back(hgf):
    """Lowering a length within the open block, then going on: as if the tokens had never come."""
    p = Pair(hgf, 2, 64)
    p.fill([100])
    p.cache.length[0] = 90
    p.ref.tokens[0] = p.ref.tokens[0][:90]
    p.reserve([0], [200])
    p.append([0], [50])
    p.check()
    p.attend([0], [4])


@pytest.mark.parametrize("group", [1, 4])
def test_captured_decode_loop(hgf, group):
    """Append and attention of a step captured once and replayed over block ends, among eager calls on another workspace."""
    H, dh, S, steps = 2, 64, 3, 70
    p = Pair(hgf, H, dh, n_slots=4)
    p.fill([60, 127, 5])
    p.reserve(range(S), [60 + steps, 127 + steps, 5 + steps])
    slots, starts = ints([2, 0, 1, -1]), ints([0, 1, 2, 3, 4])
    k, v = (torch.zeros((4, w * dh), dtype=torch.bfloat16, device="cuda") for w in (2 * H, H))
    q = torch.zeros((4, 2 * H * group * dh), dtype=torch.bfloat16, device="cuda")
    out, done = torch.zeros((4, H * group * dh), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    ws = torch.empty(hgf.cached_workspace_bytes(p.cache, 4, 4, H * group), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hgf.cache_append(p.cache, k, v, slots, starts, done=done)
        hgf.diff_attention_cached(p.cache, q, slots, starts, 0.6, out=out, workspace=ws)
    for step in range(steps):
        kb, vb, qb = rows(p.rng, 4, 2 * H * dh), rows(p.rng, 4, H * dh), rows(p.rng, 4, 2 * H * group * dh)
        k.copy_(bf16(kb)), v.copy_(bf16(vb)), q.copy_(bf16(qb))
        graph.replay()
        assert done.tolist() == p.ref.append([2, 0, 1, -1], [0, 1, 2, 3, 4], kb, vb) == [1, 1, 1, 0]
        if step % 9 == 0 or step in (3, 4, 58, 59, 69):
            got = out.cpu().numpy().reshape(4, H * group, dh)
            qf = bf16_bits_to_f32(qb).astype(np.float64).reshape(4, 2, H * group, dh)
            for i, s in enumerate([2, 0, 1]):
                want, tol = attention(p.ref.values(s), qf[i:i + 1], 1, H * group, 0.6, 1.0)
                assert (np.abs(got[i] - want[0]) <= tol[0][:, None]).all()
            p.attend([0, 1, 2], [1, 2, 1], group=group)
    p.check()
    hgf.check_status()


@pytest.mark.parametrize("dh, group, out_bf16", [(64, 1, False), (64, 3, True), (128, 1, True)])
def test_captured_pieces_of_a_prompt(hgf, dh, group, out_bf16):
    """Pieces of two prompts, appended and attended to in one captured graph, replayed without a stop between them: the tiles of 128 rows."""
    H, piece, pieces = 2, 97, 6
    p = Pair(hgf, H, dh, n_pages=40, n_slots=2)
    p.fill([0, 77])
    p.reserve([0, 1], [piece * pieces, 77 + piece * pieces])
    slots, starts, n = ints([1, 0]), ints([0, piece, 2 * piece]), 2 * piece
    k, v, q = (torch.zeros((n, w * dh), dtype=torch.bfloat16, device="cuda") for w in (2 * H, H, 2 * H * group))
    out = torch.zeros((n, H * group * dh), dtype=torch.bfloat16 if out_bf16 else torch.float32, device="cuda")
    ws = torch.empty(hgf.cached_workspace_bytes(p.cache, 2, n, H * group), dtype=torch.uint8, device="cuda")
    done, flags = torch.zeros(2, dtype=torch.int32, device="cuda"), hgf.FLAG_OUT_BF16 if out_bf16 else 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hgf.cache_append(p.cache, k, v, slots, starts, done=done)
        hgf.diff_attention_cached(p.cache, q, slots, starts, 0.6, out=out, workspace=ws, flags=flags)
    bits_ = [[rows(p.rng, n, w * dh) for w in (2 * H, H, 2 * H * group)] for _ in range(pieces)]
    new, outs = [[bf16(x) for x in piece_] for piece_ in bits_], []
    for nk, nv, nq in new:
        k.copy_(nk), v.copy_(nv), q.copy_(nq)
        graph.replay()
        outs.append(out.clone())
    again = hgf.diff_attention_cached(p.cache, q, slots, starts, 0.6, flags=flags)
    assert torch.equal(again, outs[-1])
    hgf.check_status()
    for (kb, vb, qb), got in zip(bits_, outs):
        p.ref.append([1, 0], [0, piece, n], kb, vb)
        got = got.float().cpu().numpy().astype(np.float64).reshape(n, H * group, dh)
        qf = bf16_bits_to_f32(qb).astype(np.float64).reshape(n, 2, H * group, dh)
        for i, s in enumerate([1, 0]):
            want, tol = attention(p.ref.values(s), qf[i * piece:(i + 1) * piece], piece, H * group, 0.6, 1.0, coarse=out_bf16)
            tol = tol[:, :, None] + (2.0 ** -8 * np.abs(want) if out_bf16 else 0)
            assert (np.abs(got[i * piece:(i + 1) * piece] - want) <= tol).all()
    p.check()


def test_on_another_stream(hgf):
    p = Pair(hgf, 2, 64)
    p.fill([300, 70])
    q = rows(p.rng, 4, 256)
    want = hgf.diff_attention_cached(p.cache, bf16(q), ints([0, 1]), ints([0, 2, 4]), 0.5)
    qd, slots, starts = bf16(q), ints([0, 1]), ints([0, 2, 4])
    first, rstarts, two, want2 = ints([0, 0]), ints([0, 300, 370]), ints([2]), ints([70])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    k, v = hgf.cache_read(p.cache, slots, first, rstarts, 370, stream=side)
    got = hgf.diff_attention_cached(p.cache, qd, slots, starts, 0.5, stream=side)
    done = hgf.cache_reserve(p.cache, two, want2, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and done.tolist() == [1]
    k2, v2 = hgf.cache_read(p.cache, slots, first, rstarts, 370)
    assert torch.equal(k, k2) and torch.equal(v, v2)


def test_same_inputs_give_the_same_bits(hgf):
    p = Pair(hgf, 3, 64, n_pages=90, n_slots=16)
    p.fill(LENGTHS)
    for counts, group in (([1] * 16, 1), ([1, 2] * 8, 2)):
        n = sum(counts)
        q, slots, starts = bf16(rows(p.rng, n, 6 * group * 64)), ints(range(16)), ints(np.concatenate([[0], np.cumsum(counts)]).tolist())
        first = hgf.diff_attention_cached(p.cache, q, slots, starts, 0.5)
        for _ in range(5):
            assert torch.equal(first, hgf.diff_attention_cached(p.cache, q, slots, starts, 0.5))


def test_a_serving_loop(hgf):
    """The operators as they are used: prompts of a batch through the whole-sequence attention and into the cache, then decode steps with a
    fork, a sequence that ends, one that is admitted in its place, and drafts that are taken back."""
    H, dh, lam = 2, 64, 0.8
    p = Pair(hgf, H, dh, n_pages=24, n_slots=6, max_pages=8, seed=4)
    L = 150
    rng = p.rng
    q, k, v = rows(rng, 2 * L, 2 * H * dh), rows(rng, 2 * L, 2 * H * dh), rows(rng, 2 * L, H * dh)
    prompt = hgf.diff_attention_forward(bf16(q), bf16(k), bf16(v), 2, L, H, dh, lam).cpu().numpy()
    p.reserve([0, 1], [L + 100, L + 100])
    assert hgf.cache_append(p.cache, bf16(k), bf16(v), ints([0, 1]), ints([0, L, 2 * L])).tolist() == p.ref.append([0, 1], [0, L, 2 * L], k, v)
    # the prompt's last row over the cache: the whole-sequence result but for the cache's rounding, half a step of 1/127 of each block's maximum
    # on keys and values.  A key's half step moves a score by up to h |q|_1 / sqrt(d) (h: half a step), so a probability by twice the exponent of it
    last = p.attend([0, 1], [1, 1], lam=lam, q=np.concatenate([q[[L - 1, 2 * L - 1]], q[:2]]))
    kf, vf, qf = (bf16_bits_to_f32(a).astype(np.float64) for a in (k, v, q))
    for i in range(2):
        own = slice(i * L, (i + 1) * L)
        hk, hv = np.abs(kf[own]).max() / 254, np.abs(vf[own]).max() / 254
        qrow = qf[(i + 1) * L - 1].reshape(2, H, dh)
        moved = np.expm1(2 * hk * np.abs(qrow).sum(-1).max() / np.sqrt(dh))
        bound = (1 + lam) * (hv + moved * (np.abs(vf[own]).max() + hv)) + 4e-3 * (1 + lam) * np.abs(vf[own]).max()   # (the last: the other kernel's bf16 probabilities)
        assert np.abs(last[i].reshape(-1) - prompt[(i + 1) * L - 1]).max() <= bound
    active = [0, 1]
    for step in range(12):
        if step == 3:
            assert hgf.cache_fork(p.cache, ints([0]), ints([2])).tolist() == p.ref.fork([0], [2]) == [1]
            p.reserve([2], [L + 100])
            active = [0, 1, 2]
        if step == 6:
            hgf.cache_free(p.cache, ints([1]))
            p.ref.free([1])
            p.reserve([4], [200])
            p.append([4], [130])
            active = [0, 2, 4]
        if step == 9:                          # drafts: five tokens, two stay
            before = [len(p.ref.tokens[s]) for s in active]
            p.append(active, [5] * 3)
            p.attend(active, [5] * 3, lam=lam)
            for s, n in zip(active, before):
                if (n + 5) // BLOCK == (n + 2) // BLOCK:
                    p.cache.length[s] = n + 2
                    p.ref.tokens[s] = p.ref.tokens[s][:n + 2]
        p.append(active, [1] * len(active))
        p.attend(active, [1] * len(active), lam=lam)
    p.check()
    hgf.check_status()
