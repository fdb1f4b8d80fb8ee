"""hgf_diff_attention_forward_train and hgf_diff_attention_backward against the definition in 64 bits, element by element, within what the documented
roundings to bf16 can move (attention_gradients.py)."""
import pytest
import torch

import attention_gradients as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hgf():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    from paper_2602_05269_b200 import hgf as binding
    binding.lib()
    torch.cuda.set_device(0)
    return binding


def check(hgf, B, L, h, dh, lam=0.8, scale=1.0, seed=0, spread=1.0, flags=None, change=None):
    q, k, v, g = ref.inputs(B, L, h, dh, seed, "cuda", spread)
    if change:
        change(q, k, v, g)
    flags = hgf.FLAG_OUT_BF16 if flags is None else flags
    out, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, lam, scale, flags=flags)
    got = hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, lam, scale)
    hgf.check_status()
    want = ref.reference(q, k, v, g, B, L, h, dh, lam, scale)
    assert (lse.double() - want["lse"][0]).abs().max() <= 2.0 ** -19 * (8 + want["lse"][0].abs().max())   # (the maximum times the scale, and a logarithm: fp32)
    for name, x in (("out", out), ("streams", streams), *got.items()):
        if name == "_workspace":
            continue
        value, bound = want[name]
        over = (x.double() - value).abs() - bound
        assert (over <= 0).all(), f"{name}: {over.max():.3e} over, largest value {value.abs().max():.3e}"
    return got, want


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,L,h", [(1, 1, 1), (2, 2, 3), (1, 63, 2), (1, 64, 1), (2, 65, 2), (3, 127, 1), (1, 128, 2), (2, 129, 3), (1, 257, 5), (1, 700, 2)])
def test_lengths(hgf, B, L, h, dh):
    check(hgf, B, L, h, dh, seed=L)


@pytest.mark.parametrize("B,L,h,dh", [(2, 300, 60, 64), (3, 129, 53, 128), (7, 64, 43, 64), (1, 257, 149, 128)])
def test_more_tiles_than_sms(hgf, B, L, h, dh):
    """Several tiles a CTA, one after the other, so that every buffer changes hands between tiles."""
    check(hgf, B, L, h, dh, seed=L)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("lam,scale", [(0.0, 1.0), (-0.6, 1.0), (1.7, 0.5), (0.2, -3.0), (0.5, 0.0)])
def test_lambda_and_scale(hgf, dh, lam, scale):
    got, _ = check(hgf, 2, 150, 2, dh, lam, scale, seed=5)
    if lam == 0.0:
        w = 2 * dh
        assert not got["dq"][:, w:].any() and not got["dk"][:, w:].any()
    if scale == 0.0:
        assert not any(got[n].any() for n in ("dq", "dk", "dv", "dlambda"))


@pytest.mark.parametrize("dh", [64, 128])
def test_peaked_rows_and_even_rows(hgf, dh):
    check(hgf, 1, 300, 2, dh, seed=6, spread=6.0)
    check(hgf, 1, 300, 2, dh, seed=7, spread=0.0)


@pytest.mark.parametrize("dh", [64, 128])
def test_scores_that_grow_along_the_sequence(hgf, dh):
    def grow(q, k, v, g):
        k *= torch.linspace(0.3, 7.0, k.shape[0], device=k.device).to(k.dtype)[:, None]
    check(hgf, 1, 500, 2, dh, seed=8, change=grow)


@pytest.mark.parametrize("dh", [64, 128])
def test_output_in_fp32(hgf, dh):
    B, L, h, lam, scale = 2, 200, 2, 0.8, 0.5
    q, k, v, _ = ref.inputs(B, L, h, dh, 9, "cuda")
    out, streams, _ = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, lam, scale)
    assert out.dtype == streams.dtype == torch.float32
    value, _ = ref.reference(q, k, v, v, B, L, h, dh, lam, scale)["out"]
    one, two = streams.view(B * L, 2, -1).unbind(1)
    assert (out - scale * (one - lam * two)).abs().max() <= 2.0 ** -20 * streams.abs().max()
    assert (out.double() - value).abs().max() <= (ref.HALF ** 2 + ref.SLACK) * scale * (1 + lam) * v.abs().max()
    near = hgf.diff_attention_forward(q, k, v, B, L, h, dh, lam, scale)
    assert (out.double() - value).norm() < (near.double() - value).norm()


@pytest.mark.parametrize("dh", [64, 128])
def test_sequences_do_not_touch_each_other(hgf, dh):
    """A sequence of a batch whose values are not finite leaves the gradients of the others as they are, at lengths inside a tile."""
    B, L, h, lam = 3, 77, 2, 0.8
    q, k, v, g = ref.inputs(B, L, h, dh, 10, "cuda")
    out, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, lam)
    clean = {"out": out, "streams": streams, **hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, lam)}
    for x in (q, k, v, g):
        x[L:2 * L] = float("nan")
    out, streams, dirty_lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, lam)
    assert torch.equal(lse[0], dirty_lse[0]) and torch.equal(lse[2], dirty_lse[2]) and not dirty_lse[1].isfinite().any()
    dirty = {"out": out, "streams": streams, **hgf.diff_attention_backward(q, k, v, g, streams, dirty_lse, B, L, h, dh, lam)}
    for n in ("out", "streams", "dq", "dk", "dv"):
        assert torch.equal(clean[n][:L], dirty[n][:L]) and torch.equal(clean[n][2 * L:], dirty[n][2 * L:])
        assert not dirty[n][L:2 * L].isfinite().all()


@pytest.mark.parametrize("dh", [64, 128])
def test_equal_calls_give_equal_bits_and_parts_give_the_same(hgf, dh):
    """Whatever the workspace holds, and whichever gradients are asked for."""
    B, L, h, lam = 2, 333, 5, 0.8
    q, k, v, g = ref.inputs(B, L, h, dh, 11, "cuda")
    _, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, lam)
    call = lambda **a: hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, lam, **a)  # noqa: E731
    one = call()
    ws = torch.full((hgf.diff_attention_backward_workspace_bytes(B, L, h, dh),), 255, dtype=torch.uint8, device="cuda")
    for want in (None, ("dq",), ("dk", "dv"), ("dq", "dlambda"), ()):
        ws.fill_(255)
        two = call(workspace=ws, want=want)
        for n in two:
            assert n == "_workspace" or torch.equal(one[n], two[n])


def test_another_stream_and_a_captured_step(hgf):
    B, L, h, dh, lam = 2, 200, 3, 64, 0.8
    q, k, v, g = ref.inputs(B, L, h, dh, 12, "cuda")
    out, streams, lse = hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, lam)
    grads = hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, lam)
    first = {n: grads[n].clone() for n in ("dq", "dk", "dv", "dlambda")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, lam, stream=side)
    side.synchronize()
    assert all(torch.equal(first[n], again[n]) for n in first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hgf.diff_attention_forward_train(q, k, v, B, L, h, dh, lam, out=out, streams=streams, lse=lse)
        hgf.diff_attention_backward(q, k, v, g, streams, lse, B, L, h, dh, lam, out=grads)
    q2, k2, v2, g2 = ref.inputs(B, L, h, dh, 13, "cuda")
    for a, b in ((q, q2), (k, k2), (v, v2), (g, g2)):
        a.copy_(b)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    want = ref.reference(q2, k2, v2, g2, B, L, h, dh, lam, 1.0)
    for n in first:
        assert ((grads[n].double() - want[n][0]).abs() <= want[n][1]).all() and not torch.equal(first[n], grads[n])
