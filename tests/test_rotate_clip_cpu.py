"""Norm and rotation of heads, and the clipping of gradients, without a GPU: the 64-bit reference against differences, and refusals."""
import ctypes

import pytest
import torch

import rotate_reference as ref
from paper_2602_05269_b200 import build as hgf_build


@pytest.fixture(scope="module")
def hgf():
    hgf_build.build()
    from paper_2602_05269_b200 import hgf as binding
    binding.lib()
    return binding


@pytest.mark.parametrize("rot,pairs", [(0, False), (8, False), (8, True), (4, False), (4, True)])
def test_the_references_gradients_agree_with_differences(rot, pairs):
    r = torch.Generator().manual_seed(rot)
    n = lambda *s: torch.randn(*s, generator=r, dtype=torch.float64)  # noqa: E731
    x, w, dy, pos = n(3, 16), 1 + 0.3 * n(8), n(3, 16), torch.tensor([0, 5, 77])
    loss = lambda x, w: float((ref.forward(x, pos, 8, w, 1e-3, 100.0, rot, pairs)[0] * dy).sum())  # noqa: E731
    got, step = ref.backward(x, dy, pos, 8, w, 1e-3, 100.0, rot, pairs), 1e-5
    dx, dw = n(3, 16), n(8)
    assert abs((loss(x + step * dx, w) - loss(x - step * dx, w)) / (2 * step) - float((got["dx"][0] * dx).sum())) <= 1e-7
    assert abs((loss(x, w + step * dw) - loss(x, w - step * dw)) / (2 * step) - float((got["dw"][0] * dw).sum())) <= 1e-7


def test_what_the_rotation_refuses(hgf):
    L, p = hgf.lib(), ctypes.c_void_p
    before, at, odd = hgf.launch_count(), p(4096), p(4100)
    inf, nan = float("inf"), float("nan")

    def fwd(q=at, k=at, n=5, hq=4, hk=2, dh=64, pos=at, wq=at, wk=at, eps=1e-6, base=1e4, rot=64, qo=at, ko=at, flags=0):
        return L.hgf_qk_norm_rotate(q, k, n, hq, hk, dh, pos, wq, wk, eps, base, rot, qo, ko, flags, None)

    def bwd(dq=4096, dk=4096, dwq=4096, dwk=4096, ws=at, ws_bytes=1 << 24, grads=True, **a):
        f = {"q": at, "k": at, "n": 5, "hq": 4, "hk": 2, "dh": 64, "pos": at, "wq": at, "wk": at, "eps": 1e-6, "base": 1e4, "rot": 64, "qo": at, "ko": at, "flags": 0, **a}
        g = hgf.RotateGrads(dq, dk, dwq, dwk)
        return L.hgf_qk_norm_rotate_backward(f["q"], f["k"], f["n"], f["hq"], f["hk"], f["dh"], f["pos"], f["wq"], f["wk"], f["eps"], f["base"], f["rot"], f["qo"], f["ko"],
                                             ctypes.byref(g) if grads else None, ws, ws_bytes, f["flags"], None)

    for call in (fwd, bwd):
        assert call(q=None, k=None, dq=None, dk=None, dwq=None, dwk=None) == 1 if call is bwd else call(q=None, k=None) == 1
        for bad in ({"pos": None}, {"n": 0}, {"n": -1}, {"hq": 0}, {"hk": -2}, {"eps": -1.0}, {"eps": nan}, {"eps": inf}, {"base": 0.0}, {"base": nan}, {"base": inf}, {"qo": None}, {"ko": None}, {"flags": 1}):
            assert call(**bad) == 1, bad
        for bad in ({"dh": 96}, {"rot": 8}, {"rot": 80}, {"rot": -16}, {"n": 1 << 31}):
            assert call(**bad) == 2, bad
        for name in ("q", "k", "wq", "wk", "qo", "ko"):
            assert call(**{name: odd}) == 3, name
        assert call(pos=p(4098)) == 3
    assert bwd(grads=False) == bwd(q=None, qo=None, hq=0) == bwd(k=None, ko=None) == 1
    assert bwd(dq=4100) == bwd(dk=4100) == bwd(dwq=4100) == bwd(dwk=4100) == bwd(ws=p(4096 + 64)) == 3
    need = L.hgf_qk_norm_rotate_workspace_bytes(64)
    assert need == L.hgf_qk_norm_rotate_workspace_bytes(128) // 2 > 0 == L.hgf_qk_norm_rotate_workspace_bytes(96)
    assert bwd(ws=None) == bwd(ws_bytes=need - 1) == 4
    assert bwd(dq=None, dk=None, dwq=None, dwk=None, ws=None) == 0   # nothing is asked for
    assert hgf.launch_count() == before


def test_what_a_list_of_gradients_refuses(hgf):
    """Everything is checked before memory is asked for: a good list gets as far as the missing device (5)."""
    L = hgf.lib()

    def create(*entries, n=None, out=True):
        arr, handle = (hgf.TensorEntry * max(len(entries), 1))(*[hgf.TensorEntry(*e) for e in entries]), ctypes.c_void_p()
        return L.hgf_grad_list_create(arr, len(entries) if n is None else n, ctypes.byref(handle) if out else None)

    if not torch.cuda.is_available():
        assert create((4096, 4096, 100, 0), (8192, 16384, 100, 1), (0, 0, 0, 1)) == 5
        assert create((4096, 4096, 100, 0), (4496, 4496, 1, 0), (4500, 8192, 3, 1)) == 5     # one behind the other
        assert create((4096, 8192, 100, 0), (4096, 16384, 100, 0)) == 5                      # one gradient, two outputs
    assert create((4096, 4096, 100, 0), n=0) == create((4096, 4096, 100, 0), out=False) == create((4096, 4096, -1, 0)) == create((0, 4096, 1, 0)) == create((4096, 0, 1, 0)) == 1
    assert create((4096, 4096, 100, 2)) == create((4096, 4096, 100, -1)) == create((4096, 4096, 1 << 60, 0)) == 1
    assert create((4098, 4096, 100, 0)) == create((4096, 4098, 100, 0)) == create((4097, 4097, 100, 1)) == 3
    assert create((4096, 4096, 100, 0), (4096, 4096, 100, 0)) == 1                           # the same twice
    assert create((4096, 4096, 100, 0), (4492, 4492, 1, 0)) == 1                             # the last element again
    assert create((4096, 4100, 100, 0)) == create((4096, 3796, 100, 0)) == 1                 # moved by less than its length
    assert create((4096, 8192, 100, 0), (8588, 16384, 1, 0)) == 1                            # reads what another writes
    assert L.hgf_clip_grad_norm(None, 1.0, None, None) == 1
    L.hgf_grad_list_destroy(None)


def test_the_binding_refuses_what_does_not_fit(hgf, monkeypatch):
    class Library:
        called = False

        def hgf_qk_norm_rotate_workspace_bytes(self, d):
            return 256

        def hgf_qk_norm_rotate(self, *a):
            self.called = True
            return 0

        hgf_qk_norm_rotate_backward = hgf_grad_list_create = hgf_clip_grad_norm = hgf_qk_norm_rotate

        def hgf_grad_list_destroy(self, *a):
            pass

    library, z = Library(), lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)
    monkeypatch.setattr(hgf, "_native_train", None)
    monkeypatch.setattr(hgf, "lib", lambda: library)
    monkeypatch.setattr(hgf, "_stream", lambda s: None)
    q, k, pos, w = z(5, 256), z(5, 128), z(5, dt=torch.int32), z(64, dt=torch.float32)
    with pytest.raises(AssertionError, match="current device"):
        hgf.qk_norm_rotate(q, k, pos, 64)
    with pytest.raises(AssertionError, match="current device"):
        hgf.GradList([w])
    monkeypatch.setattr(hgf, "_current_device", lambda d: None)
    assert hgf.qk_norm_rotate(q, k, pos, 64, w, w, q_out=q)[0] is q and hgf.qk_norm_rotate(q, None, pos, 64)[1] is None
    g = hgf.qk_norm_rotate_backward(q, k, pos, 64, q, k, w)
    assert set(g) == {"dq", "dwq", "dk", "dwk", "_workspace"} and set(hgf.qk_norm_rotate_backward(None, k, pos, 64, None, k)) == {"dk", "dwk", "_workspace"}
    grads = hgf.GradList([w, q])
    assert grads.clip(1.0).shape == (1,)
    library.called = False
    for a in ((None, None, pos), (q.float(), k, pos), (q, k[:4], pos), (q, k, pos[:4]), (q, k, pos.long()), (z(5, 200), k, pos), (q, k.to("meta"), pos), (z(5, 512)[:, ::2], k, pos)):
        with pytest.raises(AssertionError):
            hgf.qk_norm_rotate(*a, 64)
        with pytest.raises(AssertionError):
            hgf.qk_norm_rotate_backward(*a, 64, q, k)
    for bad in ({"wq": w[:32]}, {"wk": w.double()}, {"q_out": k}, {"k_out": k.float()}, {"q_out": q.to("meta")}):
        with pytest.raises(AssertionError):
            hgf.qk_norm_rotate(q, k, pos, 64, **bad)
    with pytest.raises(AssertionError):
        hgf.qk_norm_rotate(q, None, pos, 64, k_out=k)
    for bad in ((k, k), (q, None), (q.float(), k)):
        with pytest.raises(AssertionError):
            hgf.qk_norm_rotate_backward(q, k, pos, 64, *bad)
    for bad in ({**g, "dq": k}, {**g, "dwk": w.double()}, {**g, "_workspace": w}):
        with pytest.raises(AssertionError):
            hgf.qk_norm_rotate_backward(q, k, pos, 64, q, k, out=bad)
    for bad in (([],), ([w, w.half()],), ([w], [w, w]), ([q], [q.float()]), ([q], [q[:4]]), ([z(8, 8)[:, ::2]],), ([w, q.to("meta")],)):
        with pytest.raises(AssertionError):
            hgf.GradList(*bad)
    for bad in (w, z(1), z(1, dt=torch.float32).to("meta")):
        with pytest.raises(AssertionError):
            grads.clip(1.0, norm=bad)
    assert not library.called
