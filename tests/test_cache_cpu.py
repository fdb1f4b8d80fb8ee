"""The K/V cache's entry points on a machine without a GPU: what they refuse before any launch, sizes, and the tests' own reference."""
import ctypes

import numpy as np
import pytest

from cache_reference import BLOCK, Reference, attention, page_bytes, quantise, rows, tile_index
from paper_2602_05269_b200 import build as hgf_build


@pytest.fixture(scope="module")
def hgf():
    hgf_build.build()
    from paper_2602_05269_b200 import hgf as binding
    binding.lib()
    return binding


def _struct(hgf, **change):
    v = {"codes": 4096, "scales": 4096, "open": 4096, "table": 4096, "held": 4096, "length": 4096, "refs": 4096, "arrivals": 4096, "n_pages": 8,
         "n_slots": 4, "max_pages": 3, "n_heads": 2, "head_dim": 64}
    v.update(change)
    return ctypes.byref(hgf.Cache(*(v[n] for n, _ in hgf.Cache._fields_)))


def _calls(hgf):
    """Each entry point as a function of the cache and of changed arguments; the pointers are never followed, since every call is refused."""
    L, p = hgf.lib(), ctypes.c_void_p
    ok = p(4096)

    def call(fn, order, **default):
        return lambda cache, **kw: fn(cache, *({**default, **kw}[n] for n in order), None)
    return {
        "reserve": call(L.hgf_cache_reserve, ("slots", "tokens", "n", "done"), slots=ok, tokens=ok, n=2, done=None),
        "append": call(L.hgf_cache_append, ("k", "v", "rows", "slots", "starts", "n", "done"), k=ok, v=ok, rows=4, slots=ok, starts=ok, n=2, done=None),
        "read": call(L.hgf_cache_read, ("slots", "first", "starts", "n", "rows", "k", "v", "flags"), slots=ok, first=ok, starts=ok, n=2, rows=4, k=ok, v=ok, flags=0),
        "fork": call(L.hgf_cache_fork, ("slots", "dst", "n", "done"), slots=ok, dst=ok, n=2, done=None),
        "free": call(L.hgf_cache_free, ("slots", "n"), slots=ok, n=2),
        "attend": call(L.hgf_diff_attention_cached, ("q", "rows", "heads", "slots", "starts", "n", "lam", "scale", "out", "ws", "ws_bytes", "flags"), q=ok, rows=4, heads=2,
                       slots=ok, starts=ok, n=2, lam=ctypes.c_float(0.5), scale=ctypes.c_float(1.0), out=ok, ws=ok, ws_bytes=1 << 30, flags=0),
    }


@pytest.mark.parametrize("name", ["reserve", "append", "read", "fork", "free", "attend"])
def test_bad_caches_and_lists_are_refused(hgf, name):
    call, before = _calls(hgf)[name], hgf.launch_count()
    assert call(None) == 1
    for field in ("codes", "scales", "open", "table", "held", "length", "refs", "arrivals"):
        assert call(_struct(hgf, **{field: None})) == 1
        assert call(_struct(hgf, **{field: 4096 + 8})) == 3
    for field in ("n_pages", "n_slots", "max_pages", "n_heads"):
        assert call(_struct(hgf, **{field: 0})) == 1
    for field, value in (("head_dim", 96), ("head_dim", 0), ("n_pages", 1 << 31), ("n_slots", 1 << 31), ("max_pages", (1 << 24) + 1), ("n_heads", 65536)):
        assert call(_struct(hgf, **{field: value})) == 2
    assert call(_struct(hgf), slots=None) == 1
    assert call(_struct(hgf), n=0) == 1
    assert call(_struct(hgf), n=hgf.CACHE_MAX_SEQS + 1) == 2
    assert hgf.launch_count() == before


def test_other_bad_arguments_are_refused(hgf):
    c, cache, odd, before = _calls(hgf), _struct(hgf), ctypes.c_void_p(4096 + 2), hgf.launch_count()
    assert c["reserve"](cache, tokens=None) == 1
    assert c["fork"](cache, dst=None) == 1
    for name, args in (("append", ("k", "v")), ("read", ("k", "v")), ("attend", ("q", "out"))):
        for a in args:
            assert c[name](cache, **{a: None}) == 1
            assert c[name](cache, **{a: odd}) == 3
        assert c[name](cache, starts=None) == 1
        assert c[name](cache, rows=0) == 1
        assert c[name](cache, rows=(1 << 24) + 1) == 2
    for name in ("read", "attend"):
        assert c[name](cache, flags=2) == 1
    assert c["read"](cache, first=None) == 1
    assert c["attend"](cache, heads=0) == 1
    assert c["attend"](cache, heads=3) == 2
    assert c["attend"](cache, ws=None) == 4
    assert c["attend"](cache, ws_bytes=1000) == 4
    assert c["attend"](cache, ws=ctypes.c_void_p(4096 + 16)) == 3
    assert hgf.launch_count() == before


def test_workspace(hgf):
    bytes_ = hgf.lib().hgf_cached_workspace_bytes
    assert bytes_(None, 1, 1, 2) == 256 and bytes_(_struct(hgf, head_dim=32), 1, 1, 2) == 256
    single, several = bytes_(_struct(hgf), 4, 4, 2), bytes_(_struct(hgf), 4, 5, 2)
    assert 0 < single <= several and single % 256 == 0 and several % 256 == 0
    assert bytes_(_struct(hgf), 4, 4, 4) == several        # shared heads


def test_a_cache_in_host_memory_is_refused(hgf):
    import torch
    cache = hgf.KVCache(2, 64, 4, 2, 2, device="cpu")
    assert cache.codes.shape == (4, 2, 3 * 64 * 64) and cache.open.shape == (2, 2, 3, 64, 64) and cache.table.shape == (2, 2) and cache.scales.shape == (4, 2, 4)
    n, before = torch.zeros(2, dtype=torch.int32), hgf.launch_count()
    k, v, f = (torch.zeros(1, w, dtype=torch.bfloat16) for w in (256, 128, 256))
    out, ws = torch.zeros(1, 128), torch.zeros(1 << 22, dtype=torch.uint8)
    for call in (lambda: hgf.cache_reserve(cache, n, n, granted=n), lambda: hgf.cache_append(cache, k, v, n[:1], n, done=n[:1]), lambda: hgf.cache_free(cache, n),
                 lambda: hgf.cache_fork(cache, n, n, done=n), lambda: hgf.cache_read(cache, n[:1], n[:1], n, k=k, v=v),
                 lambda: hgf.diff_attention_cached(cache, f, n[:1], n, 0.5, out=out, workspace=ws)):
        with pytest.raises(AssertionError, match="not the current device"):
            call()
    assert hgf.launch_count() == before
    with pytest.raises(AssertionError):
        hgf.KVCache.of(2, 64, **{**{name: getattr(cache, name) for name in hgf.KVCache._SHAPES}, "refs": torch.zeros(5, dtype=torch.int32)})


def test_status_string(hgf):
    assert hgf.status_string(8) not in {hgf.status_string(i) for i in (*range(8), 99)}


def test_reference_layout_names_every_byte_once():
    for shape in ((64, 64), (64, 128), (128, 64)):
        assert sorted(tile_index(*shape).ravel()) == list(range(shape[0] * shape[1]))
    # the header's rule, spelled out for one element: row 8 a + g, column 16 h + 4 t + b of the tile
    assert tile_index(64, 128)[16 + 8 + 3, 96 + 16 + 8 + 1] == (1 * 4 + 3) * 512 + (4 * 3 + 2) * 16 + 8 + 4 + 1
    x = np.arange(64 * 64).reshape(64, 64).astype(np.int8)
    page = page_bytes(x, x, x)
    assert page[tile_index(64, 64)[5, 9]] == x[5, 9] and page[2 * 64 * 64 + tile_index(64, 64)[9, 5]] == x[5, 9]


def test_reference_quantiser():
    codes, scale = quantise(np.full((64, 64), 0.5) * np.where(np.arange(64) == 0, 2.0, 1.0))
    assert codes[0, 0] == 127 and codes[0, 1] == 64 and scale == np.float32(np.float32(1) / np.float32(127))   # 63.5 to even
    assert np.isnan(quantise(np.full((64, 64), np.inf))[1]) and quantise(np.zeros((64, 64)))[1] == 0


def test_reference_attention_on_one_token_is_its_value():
    rng = np.random.default_rng(0)
    r = Reference(1, 64, 4, 1, 4)
    r.append([0], [0, 1], rows(rng, 1, 128), rows(rng, 1, 64))
    out, _ = attention(r.values(0), rng.standard_normal((1, 2, 3, 64)), 1, 3, 0.25, 2.0)
    assert np.allclose(out[0], 2.0 * 0.75 * r.values(0)[2, 0, 0])
    assert r.append([0], [0, 63], rows(rng, 63, 128), rows(rng, 63, 64)) == [0]      # no page for the block
    assert r.reserve([0, 0], [BLOCK, BLOCK]) == [1, 0] and r.append([0], [0, 63], rows(rng, 63, 128), rows(rng, 63, 64)) == [1]
