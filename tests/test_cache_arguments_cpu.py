"""What the Python calls of the K/V cache check by themselves, on a machine without a GPU: the library is a stand-in that must not be reached."""
import ctypes

import pytest
import torch

from paper_2602_05269_b200 import build as hgf_build


@pytest.fixture
def hgf(monkeypatch):
    hgf_build.build()
    from paper_2602_05269_b200 import hgf as binding
    binding.lib()

    class Library:
        def hgf_cached_workspace_bytes(self, *args):
            return 1 << 16

        def hgf_diff_attention_cached(self, *args):
            self.called = True
            return 0

    library = Library()
    library.called = False
    monkeypatch.setattr(binding, "_native_cache", None)
    monkeypatch.setattr(binding, "_list", lambda cache, *tensors: None)   # (it refuses a cache in host memory, which stands for the GPU's here)
    monkeypatch.setattr(binding, "_stream", lambda stream: None)
    cache = binding.KVCache(2, 64, 4, 2, 2, device="cpu")
    monkeypatch.setattr(binding, "lib", lambda: library)
    return binding, cache, library


def test_attention_refuses_memory_that_is_not_the_caches(hgf):
    """`out`, the workspace and q on another device (meta stands for it), of another type or shape, or with gaps."""
    binding, cache, library = hgf
    slots, starts = torch.zeros(1, dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32)
    q, out, ws = torch.zeros(3, 256, dtype=torch.bfloat16), torch.zeros(3, 128), torch.zeros(1 << 16, dtype=torch.uint8)

    def call(**change):
        a = {"q": q, "out": out, "workspace": ws, **change}
        return binding.diff_attention_cached(cache, a["q"], slots, starts, 0.5, out=a["out"], workspace=a["workspace"])

    assert call() is out and library.called
    assert call(out=None).shape == (3, 128) and call(workspace=None) is out
    library.called = False
    bad = [{"out": out.to("meta")}, {"out": out.to("meta"), "workspace": None}, {"out": out.bfloat16()}, {"out": torch.zeros(128, 3).t()}, {"out": out[:2]},
           {"workspace": ws.to("meta")}, {"workspace": ws.to("meta"), "out": None}, {"workspace": torch.zeros(1 << 16)}, {"workspace": ws.view(torch.int8)}, {"workspace": ws[::2]},
           {"q": q.to("meta")}, {"q": q.float()}, {"q": torch.zeros(3, 256, 2, dtype=torch.bfloat16)}, {"q": torch.zeros(256, dtype=torch.bfloat16)},
           {"q": torch.zeros(3, 255, dtype=torch.bfloat16)}]
    for change in bad:
        with pytest.raises(AssertionError):
            call(**change)
    assert not library.called


def test_a_caches_arrays_are_changed_in_place_only(hgf):
    """The library goes by the addresses taken when the cache was made: another tensor in an array's place would leave it with memory that is given back."""
    binding, cache, _ = hgf
    cache = binding.KVCache.of(2, 64, **{name: getattr(cache, name) for name in binding.KVCache._SHAPES})
    at = {name: getattr(cache, name).data_ptr() for name in binding.KVCache._SHAPES}
    cache.length.fill_(7)
    for name in binding.KVCache._SHAPES:
        array = getattr(cache, name)
        with pytest.raises(AttributeError, match=name):
            setattr(cache, name, array.clone())
        with pytest.raises(AttributeError, match=name):
            delattr(cache, name)
        assert getattr(cache, name) is array
    with pytest.raises(AttributeError, match="length"):
        cache.length = cache.length - 2
    for name in ("n_heads", "head_dim", "n_pages", "n_slots", "max_pages", "device"):
        with pytest.raises(AttributeError, match=name):
            setattr(cache, name, 1000)
    assert cache.length.tolist() == [7, 7]
    cache.length -= 2                          # (in place: the same tensor)
    cache.length[1] = 3
    cache.note = "a caller's own attributes are theirs"
    assert cache.length.tolist() == [5, 3] and all(getattr(cache, name).data_ptr() == a for name, a in at.items())


def _cache(hgf, **change):
    v = {**{name: 4096 for name in hgf.KVCache._SHAPES}, "n_pages": 8, "n_slots": 4, "max_pages": 3, "n_heads": 2, "head_dim": 64, **change}
    return ctypes.byref(hgf.Cache(*(v[n] for n, _ in hgf.Cache._fields_)))


@pytest.mark.parametrize("dh", [64, 128])
def test_the_attentions_form_does_not_go_by_the_pool(dh):
    """A pool has the size of its longest load, which says nothing of a call: its workspace, and so its form, is the same."""
    from paper_2602_05269_b200 import hgf
    for n_seqs, n_rows in ((40, 40), (40, 90), (40, 500), (40, 4000), (1, 100)):
        assert len({hgf.lib().hgf_cached_workspace_bytes(_cache(hgf, head_dim=dh, n_pages=n), n_seqs, n_rows, 2) for n in (1, 39, 40, 5000)}) == 1


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 8])
def test_one_workspace_for_all_calls_of_a_program(dh, group):
    """The bytes for all of the most rows in one sequence suffice for fewer rows and any number of sequences."""
    from paper_2602_05269_b200 import hgf
    need = lambda n_seqs, n_rows: hgf.lib().hgf_cached_workspace_bytes(_cache(hgf, head_dim=dh), n_seqs, n_rows, 2 * group)  # noqa: E731
    for most in (1, 2, 9, 20, 81, 600):
        enough = need(1, most)
        assert all(need(n_seqs, n_rows) <= enough for n_rows in range(1, most + 1) for n_seqs in (*range(1, 12), 30, 31, 64, 200, 1024))
