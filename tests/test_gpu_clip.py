"""hgf_clip_grad_norm against 64 bits, and a whole training step of a block's attention whose gradients it clips."""
import math

import pytest
import torch

import attention_gradients
import rotate_reference

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -24   # half a step of fp32


@pytest.fixture(scope="module")
def hgf():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    from paper_2602_05269_b200 import hgf as binding
    binding.lib()
    torch.cuda.set_device(0)
    return binding


def check(hgf, grads, max_norm, in_place=False):
    was = [g.clone() for g in grads]
    out = None if in_place else [torch.full_like(g, 7.0) for g in grads]
    norm = hgf.GradList(grads, out).clip(max_norm)
    want = math.sqrt(sum(float(g.double().square().sum()) for g in was))
    assert abs(float(norm) - want) <= 2 * STEP * want
    factor = min(1.0, max_norm / (want + 1e-6))
    for g, w, y in zip(grads, was, out or grads):
        assert in_place or torch.equal(g, w)
        e = w.double() * factor
        half = 2.0 ** -8 if w.dtype == torch.bfloat16 else STEP
        # the factor is rounded once, the product (of fp32) once, the result to its type; 2^-133: below the smallest normal numbers steps are absolute
        assert ((y.double() - e).abs() <= (2 * STEP + half) * e.abs() + 2.0 ** -133).all()
    return norm


def some(sizes, seed=0, scale=1.0):
    r = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=r) * scale).to(torch.bfloat16 if i % 3 == 1 else torch.float32).cuda() for i, n in enumerate(sizes)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sizes", [(1,), (3, 5), (4096,), (4097, 8193, 16385), (0, 7, 0), tuple(range(1, 200)), (1 << 22, 33, 3 << 20)])
def test_sizes_and_types(hgf, sizes, in_place):
    check(hgf, some(sizes, seed=len(sizes)), 0.5, in_place)
    check(hgf, some(sizes, seed=len(sizes)), 1e9, in_place)   # nothing to clip


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_that_begin_anywhere(hgf, dtype):
    flat, other = torch.randn(20000, device="cuda").to(dtype), torch.empty(20000, dtype=dtype, device="cuda")
    cuts = [0, 1, 2, 9, 40, 41, 4000, 4007, 9999, 20000]
    pieces = lambda x: [x[a:b] for a, b in zip(cuts, cuts[1:])]  # noqa: E731
    check(hgf, pieces(flat), 1.0)
    was = flat.double()
    for shift in (0, 1, 3):    # outputs at other offsets than their gradients
        other.fill_(7.0)
        n = 20000 - shift
        hgf.GradList([flat[:n]], [other[shift:]]).clip(1.0)
        assert (other[:shift] == 7.0).all()
        e = was[:n] / (was[:n].norm() + 1e-6)
        assert ((other[shift:].double() - e).abs() <= (2 * STEP + (2.0 ** -8 if dtype == torch.bfloat16 else STEP)) * e.abs()).all()
    check(hgf, pieces(flat), 1.0, in_place=True)


def test_magnitudes(hgf):
    check(hgf, some((1000, 1000), scale=1e30), 1.0)      # squares beyond fp32
    check(hgf, some((1000, 1000), scale=1e-30), 1.0)
    check(hgf, some((1000, 1000), scale=1e-30), 0.0)
    check(hgf, [torch.zeros(100, device="cuda")], 0.5)
    assert float(hgf.GradList(some((50,))).clip(math.inf)) > 0


def test_values_that_are_not_finite(hgf):
    g = some((100, 100))
    g[1][3] = math.inf
    out = [torch.empty_like(x) for x in g]
    assert float(hgf.GradList(g, out).clip(1.0)) == math.inf
    assert not out[0].any() and out[1][3].isnan() and not out[1][:3].any()
    g[1][3] = math.nan
    assert math.isnan(float(hgf.GradList(g, out).clip(1.0)))
    assert all(y.isnan().all() for y in out)


def test_refusals(hgf):
    x = torch.zeros(64, device="cuda")
    for bad in (([x, x],), ([x, x[3:5]],), ([x[:32]], [x[16:48]]), ([x[:8], x[8:16]], [torch.empty(8, device="cuda"), x[4:12]])):
        with pytest.raises(hgf.HgfError) as e:
            hgf.GradList(*bad)
        assert e.value.status == 1
    for norm in (-1.0, math.nan):
        with pytest.raises(hgf.HgfError):
            hgf.GradList([x]).clip(norm)


def test_equal_bits_streams_and_a_captured_call(hgf):
    g = some((100000, 77, 4096), seed=3)
    out = [torch.empty_like(x) for x in g]
    grads = hgf.GradList(g, out)
    norm = grads.clip(0.1).clone()
    first = [y.clone() for y in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = grads.clip(0.1, stream=side)
    side.synchronize()
    assert torch.equal(norm, again) and all(map(torch.equal, first, out))
    graph, where = torch.cuda.CUDAGraph(), torch.empty(1, device="cuda")
    with torch.cuda.graph(graph):
        grads.clip(0.1, norm=where)
    for x in g:
        x.mul_(2.0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert float(where) == 2 * float(norm)    # (a power of two: every square and sum is four times what it was)
    for a, b in zip(first, out):   # the same up to what 1e-6 weighs beside the norm, and roundings
        assert torch.allclose(a.float(), b.float(), rtol=1e-5 if a.dtype == torch.float32 else 2.0 ** -7, atol=0)


def test_a_training_step_of_the_attention(hgf):
    """Projections, norms with rotation, attention, the way back through all of them, and the gradients clipped: every gradient against 64 bits, given what
    the calls before it left."""
    B, L, d, h, dh, r, lam = 2, 150, 256, 4, 64, 16, 0.8
    gen = torch.Generator(device="cuda").manual_seed(5)
    n = lambda *s, std=1.0: torch.randn(*s, generator=gen, device="cuda") * std  # noqa: E731
    x = n(B * L, d).to(torch.bfloat16)
    layers = {}
    for name, wide in (("q", 2 * h * dh), ("k", 2 * h * dh), ("v", h * dh)):
        packed, gamma = hgf.pack_ternary(n(wide, d, std=0.02))
        layers[name] = (packed, gamma, d, wide, n(r, d, std=d ** -0.5).half(), n(wide, r, std=r ** -0.5).half(), torch.rand(wide, generator=gen, device="cuda"))
    y = {name: hgf.linear_forward(x, *layer, flags=hgf.FLAG_OUT_BF16) for name, layer in layers.items()}
    pos = torch.arange(L, dtype=torch.int32, device="cuda").repeat(B)
    wq, wk = 1 + 0.1 * n(dh), 1 + 0.1 * n(dh)
    q, k = hgf.qk_norm_rotate(y["q"], y["k"], pos, dh, wq, wk)
    out, streams, lse = hgf.diff_attention_forward_train(q, k, y["v"], B, L, h, dh, lam, 0.5, flags=hgf.FLAG_OUT_BF16)
    dout = n(B * L, h * dh, std=0.01).to(torch.bfloat16)
    a = hgf.diff_attention_backward(q, k, y["v"], dout, streams, lse, B, L, h, dh, lam, 0.5)
    want = attention_gradients.reference(q, k, y["v"], dout, B, L, h, dh, lam, 0.5)
    for name in ("dq", "dk", "dv", "dlambda"):
        assert ((a[name].double() - want[name][0]).abs() <= want[name][1]).all()
    g = hgf.qk_norm_rotate_backward(y["q"], y["k"], pos, dh, a["dq"], a["dk"], wq, wk)
    for name, w in (("q", wq), ("k", wk)):
        e = rotate_reference.backward(y[name], a["d" + name], pos, dh, w, 1e-6, 10000.0, dh, False)
        assert ((g["d" + name].double() - e["dx"][0]).abs() <= e["dx"][1]).all() and ((g["dw" + name].double() - e["dw"][0]).abs() <= e["dw"][1]).all()
    left = [a["dlambda"], g["dwq"], g["dwk"]]
    for name, dy in (("q", g["dq"]), ("k", g["dk"]), ("v", a["dv"])):
        packed, gamma, d_in, wide, At, Bt, gate = layers[name]
        back = hgf.linear_backward(x, packed, gamma, d_in, wide, dy, At, Bt, gate)
        left += [back[n] for n in ("dW", "dAt", "dBt", "dgate")]
        T = hgf.unpack_ternary(packed, wide, d_in).double()
        dW = dy.double().t() @ (torch.round(127 * x.double() / x.double().abs().amax(1, keepdim=True)) * x.double().abs().amax(1, keepdim=True) / 127)
        assert (back["dW"].double() - dW).abs().max() <= 1e-2 * dW.abs().max() and T.abs().max() == 1
    hgf.check_status()
    check(hgf, left, 0.25 * float(torch.cat([t.flatten() for t in left]).norm()), in_place=True)
