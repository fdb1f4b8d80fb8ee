"""Gradients of the differential attention, without a GPU: the 64-bit reference of the GPU tests against differences of the forward formula, and what the
calls refuse before they launch anything."""
import ctypes

import pytest
import torch

import attention_gradients as ref
from paper_2602_05269_b200 import build as hgf_build


@pytest.fixture(scope="module")
def hgf():
    hgf_build.build()
    from paper_2602_05269_b200 import hgf as binding
    binding.lib()
    return binding


@pytest.mark.parametrize("L,dh", [(1, 4), (2, 4), (7, 8)])
def test_the_formulas_gradients_agree_with_differences(L, dh):
    B, h, lam, scale = 2, 2, 0.7, 0.5
    r = torch.Generator().manual_seed(L)
    x = {"q": torch.randn(B * L, 2 * h * dh, generator=r, dtype=torch.float64), "k": torch.randn(B * L, 2 * h * dh, generator=r, dtype=torch.float64),
         "v": torch.randn(B * L, h * dh, generator=r, dtype=torch.float64)}
    g = torch.randn(B * L, h * dh, generator=r, dtype=torch.float64)

    def loss(lam=lam, **change):
        y = {**x, **change}
        return float((ref.reference(y["q"], y["k"], y["v"], g, B, L, h, dh, lam, scale)["out"][0] * g).sum())

    got, step = ref.reference(x["q"], x["k"], x["v"], g, B, L, h, dh, lam, scale), 1e-5
    for name in x:
        d = torch.randn(x[name].shape, generator=r, dtype=torch.float64)
        slope = (loss(**{name: x[name] + step * d}) - loss(**{name: x[name] - step * d})) / (2 * step)
        # (central differences: step^2 of the third derivative, and 2^-53 / step of the value)
        assert abs(slope - float((got["d" + name][0] * d).sum())) <= 1e-7 * (1 + abs(slope))
    slope = (loss(lam + step) - loss(lam - step)) / (2 * step)
    assert abs(slope - float(got["dlambda"][0])) <= 1e-7 * (1 + abs(slope))


def test_what_the_backward_call_refuses(hgf):
    L, p = hgf.lib(), ctypes.c_void_p
    before, at, odd = hgf.launch_count(), p(4096), p(4100)   # (never dereferenced: the checks come first)
    need = hgf.diff_attention_backward_workspace_bytes(2, 100, 3, 64)
    assert need >= 2 * 3 * 2 * 1024 and hgf.diff_attention_backward_workspace_bytes(2, 100, 3, 96) == 0
    assert hgf.diff_attention_backward_workspace_bytes(0, 100, 3, 64) == hgf.diff_attention_backward_workspace_bytes(1, (1 << 24) + 1, 1, 64) == 0

    def call(q=at, k=at, v=at, dout=at, streams=at, lse=at, B=2, n=100, h=3, dh=64, dq=4096, dk=4096, dv=4096, dlam=4096, ws=at, ws_bytes=need, flags=0, grads=True):
        g = hgf.AttentionGrads(dq, dk, dv, dlam)
        return L.hgf_diff_attention_backward(q, k, v, dout, streams, lse, B, n, h, dh, 0.5, 1.0, ctypes.byref(g) if grads else None, ws, ws_bytes, flags, None)

    for name in ("q", "k", "v", "dout", "streams", "lse"):
        assert call(**{name: None}) == 1 and call(**{name: odd}) == 3
    assert call(B=0) == call(n=0) == call(h=0) == call(h=-1) == call(flags=1) == call(grads=False) == 1
    assert call(dk=None) == call(dv=None) == call(dq=None) == 1
    assert call(dh=96) == call(B=65536) == call(n=(1 << 24) + 1) == call(B=40000, n=1 << 20) == 2
    assert call(dq=4100) == call(dk=4100) == call(dv=4100) == call(dlam=4097) == call(ws=p(4096 + 64)) == 3
    assert call(ws=None) == call(ws_bytes=need - 1) == 4
    assert call(dq=None, dk=None, dv=None, dlam=None) == 0   # nothing is asked for

    def forward(streams=at, lse=at, flags=0, dh=64):
        return L.hgf_diff_attention_forward_train(at, at, at, 2, 100, 3, dh, 0.5, 1.0, at, streams, lse, flags, None)

    assert forward(streams=None) == forward(lse=None) == forward(flags=2) == 1 and forward(dh=32) == 2 and forward(streams=odd) == forward(lse=odd) == 3
    assert hgf.launch_count() == before


def test_the_binding_refuses_what_does_not_fit(hgf, monkeypatch):
    class Library:
        def hgf_diff_attention_backward_workspace_bytes(self, *a):
            return 512

        def hgf_diff_attention_backward(self, *a):
            self.called = True
            return 0

        hgf_diff_attention_forward_train = hgf_diff_attention_backward

    library = Library()
    library.called = False
    monkeypatch.setattr(hgf, "_native_train", None)
    monkeypatch.setattr(hgf, "lib", lambda: library)
    monkeypatch.setattr(hgf, "_stream", lambda s: None)
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    good = {"q": z(10, 256), "k": z(10, 256), "v": z(10, 128), "dout": z(10, 128), "streams": z(10, 256, dt=torch.float32), "lse": z(2, 2, 2, 5, dt=torch.float32)}

    def back(want=None, **change):
        a = {**good, **{n: change.pop(n) for n in list(change) if n in good}}
        return hgf.diff_attention_backward(a["q"], a["k"], a["v"], a["dout"], a["streams"], a["lse"], 2, 5, 2, 64, 0.5, want=want, **change)

    with pytest.raises(AssertionError, match="current device"):   # host memory
        back()
    monkeypatch.setattr(hgf, "_current_device", lambda d: None)
    made = back()
    assert set(made) == {"dq", "dk", "dv", "dlambda", "_workspace"} and made["dq"].shape == (10, 256) and made["dlambda"].shape == (1,)
    assert set(back(want=("dq",))) == {"dq", "_workspace"} and back(out=made)["dv"] is made["dv"]
    library.called = False
    for name, t in good.items():
        for bad in (t.to("meta"), t.double(), t[:-1], torch.zeros(t.shape[::-1], dtype=t.dtype).permute(*range(t.dim() - 1, -1, -1))):
            with pytest.raises(AssertionError):
                back(**{name: bad})
            if name not in ("dout",):
                a = {**good, name: bad}
                with pytest.raises(AssertionError):
                    hgf.diff_attention_forward_train(a["q"], a["k"], a["v"], 2, 5, 2, 64, 0.5, streams=a["streams"], lse=a["lse"])
    for bad in ({**made, "dq": made["dq"].float()}, {**made, "dk": made["dk"][:3]}, {**made, "dlambda": made["dlambda"].double()}, {**made, "dv": made["dv"].to("meta")}):
        with pytest.raises(AssertionError):
            back(out=bad)
    with pytest.raises(AssertionError):
        back(workspace=torch.zeros(512))
    assert not library.called
